"""Requests of the paged cache's writes and reads that are large enough for two rows a thread and stores past the caches (2^20 threads'
worth of rows and more), bit for bit against the formula in 32-bit steps, computed on the GPU by elementary operations that
tests/test_gpu_kv_cache.py's host ones check on a sample."""

import numpy as np
import pytest
import torch

import paper_2511_06605_amd as dl

import decode_ref

pytestmark = pytest.mark.gpu


@pytest.fixture(scope="module", autouse=True)
def library():
    torch.cuda.set_device(0)
    dl.dl_init(0)
    yield
    dl.dl_shutdown()


def quantised(x, kind):
    """Codes (as their values) and scales of rows [n, dim] of float32; rows with an infinity (drawn values beyond float16 are) get zeros and NaN."""
    bad = ~torch.isfinite(x).all(-1)
    x = torch.where(bad[:, None], 0.0, x)
    a = x.abs().amax(-1).clamp(min=2.0 ** -100)
    limit = torch.tensor(decode_ref.LIMIT[kind], dtype=torch.float32, device=x.device)
    one = torch.ones((), device=x.device)
    y = x * ((one / a) * limit)[:, None]
    y = y.to(torch.float8_e4m3fn).float() if kind == "fp8" else torch.round(y)
    return y, torch.where(bad, float("nan"), a * (one / limit))


def equal(a, b):
    """NaN equal to itself (and to nothing else: no value here is -777)."""
    return torch.equal(torch.nan_to_num(a, nan=-777.0), torch.nan_to_num(b, nan=-777.0))


# (tokens, heads, dim): lanes a row when written, 16 elements each, and when read, 8: 1 and 2, 2 and 4, 8 and 16, 16 and 32.  Numbers of
# rows are odd, and no multiple of a workgroup's.
@pytest.mark.parametrize("kind,dtype", [("fp8", torch.bfloat16), ("int8", torch.float16), ("fp8", torch.float32), ("int8", torch.float32)])
@pytest.mark.parametrize("tokens,heads,dim,page", [(1048583, 1, 16, 16), (174771, 3, 32, 5), (131075, 1, 128, 16), (43693, 3, 112, 64), (65539, 1, 256, 16),
                                                   (21847, 3, 208, 7)])
def test_large_writes_and_reads(kind, dtype, tokens, heads, dim, page):
    lanes = 1
    while lanes * 16 < dim:
        lanes *= 2
    assert tokens * heads * lanes >= 1 << 20 and tokens * heads % 2 == 1
    g = torch.Generator(device="cuda").manual_seed(tokens)
    pages = tokens // page + 2
    wide = torch.randn((tokens, heads, dim + 3), device="cuda", generator=g)
    wide *= torch.exp(3.0 * torch.randn((tokens, heads, 1), device="cuda", generator=g))
    wide = wide.to(dtype)
    k, v = wide[..., 1:1 + dim], wide[..., 3:3 + dim]  # off every alignment but the element's
    slots = torch.randperm(pages * page, device="cuda", generator=g)[:tokens].contiguous()
    for i, none in ((0, -1), (7, pages * page), (tokens // 2, 1 << 40), (tokens - 1, -(1 << 40))):
        slots[i] = none
    keep = (slots >= 0) & (slots < pages * page)
    made = []
    for _ in range(2):
        made.append(torch.full((pages, page, heads, dim), 0x55, dtype=torch.uint8, device="cuda").view(decode_ref.CODE[kind]))
        made.append(torch.full((pages, page, heads), 5.0, device="cuda"))
    cache = dl.KvCache(made[0], made[2], made[1], made[3])
    stream = torch.cuda.current_stream()
    dl.dl_kv_write(cache, dl.KvRows(k, v, slots), stream)
    back = torch.full((tokens, heads, dim + 5), 3.0, dtype=dtype, device="cuda")
    k2, v2 = back[..., 1:1 + dim], torch.full((tokens, heads, dim), 3.0, dtype=dtype, device="cuda")
    dl.dl_kv_read(cache, dl.KvRows(k2, v2, slots), stream)
    for rows, codes, scale, read in ((k, made[0], made[1], k2), (v, made[2], made[3], v2)):
        x = rows.float().reshape(tokens * heads, dim)
        y, z = quantised(x, kind)
        want = torch.full((pages * page, heads, dim), 0x55, dtype=torch.uint8, device="cuda").view(decode_ref.CODE[kind]).float()
        want_scale = torch.full((pages * page, heads), 5.0, device="cuda")
        want[slots[keep]], want_scale[slots[keep]] = y.view(tokens, heads, dim)[keep], z.view(tokens, heads)[keep]
        assert torch.equal(codes.float().view(pages * page, heads, dim), want)
        assert equal(scale.view(pages * page, heads), want_scale)
        value = torch.where(keep[:, None, None], (y * z[:, None]).view(tokens, heads, dim), 0.0).to(dtype)
        assert equal(read, value)
        some = torch.randint(tokens * heads, (500,), device="cuda", generator=g)
        host = decode_ref.quantised(x[some].double().cpu().numpy(), kind)
        assert np.array_equal(host[0], y[some].double().cpu().numpy()) and np.array_equal(host[1], z[some].cpu().numpy(), equal_nan=True)
    assert bool((back[..., 0] == 3).all()) and bool((back[..., 1 + dim:] == 3).all())
