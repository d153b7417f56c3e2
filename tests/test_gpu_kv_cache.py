"""Quantising a cache as it is written, and reading it back (dl_kv_write, dl_kv_read): every code and scale against the formula in 32-bit
steps, bit for bit, and what the codes stand for against the rows in 64 bits."""

import itertools

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


def empty_cache(kind, pages, page, heads, dim, order=(0, 1, 2, 3)):
    """Codes of 0x55 and scales of 5, laid out in any order of the first three dimensions."""
    shape = (pages, page, heads)
    back = [order.index(i) for i in range(3)]
    codes = lambda: torch.full([shape[i] for i in order[:3]] + [dim], 0x55, dtype=torch.uint8, device="cuda").permute(*back, 3)  # noqa: E731
    scale = lambda: torch.full([shape[i] for i in order[:3]], 5.0, device="cuda").permute(*back)  # noqa: E731
    k, v = codes(), codes()
    return k.view(decode_ref.CODE[kind]), v.view(decode_ref.CODE[kind]), scale(), scale()


def draw(rng, shape, dtype):
    """Rows of very different sizes, some of them zero."""
    x = rng.standard_normal(shape) * 10.0 ** rng.uniform(-4, 3, shape[:-1] + (1,))
    x[rng.random(shape[:-1]) < 0.05] = 0.0
    return torch.from_numpy(x).to(dtype).cuda()


def by_slot(t):
    return t.reshape(t.shape[0] * t.shape[1], *t.shape[2:])


def check_written(cache, rows_k, rows_v, slots, kind):
    k, v, ks, vs = cache
    keep = (slots >= 0) & (slots < k.shape[0] * k.shape[1])
    for codes, scale, rows in ((k, ks, rows_k), (v, vs, rows_v)):
        got, got_scale = by_slot(decode_ref.code_values(codes)), by_slot(scale.cpu().numpy())
        filler = decode_ref.code_values(torch.full((1,), 0x55, dtype=torch.uint8).view(decode_ref.CODE[kind]))[0]
        want, want_scale = np.full(got.shape, filler), np.full(got_scale.shape, np.float32(5))
        if rows is not None:
            y, z = decode_ref.quantised(rows.double().cpu().numpy(), kind)
            want[slots[keep]], want_scale[slots[keep]] = y[keep], z[keep]
        assert np.array_equal(got, want), "codes"
        assert np.array_equal(got_scale, want_scale, equal_nan=True), "scales"


@pytest.mark.parametrize("kind", ["fp8", "int8"])
@pytest.mark.parametrize("dtype", [torch.bfloat16, torch.float16, torch.float32])
@pytest.mark.parametrize("tokens,page,heads,dim", [(1, 16, 8, 128), (5, 1, 1, 16), (37, 16, 3, 80), (130, 5, 2, 256), (64, 64, 1, 32), (33, 7, 12, 48)])
def test_write_then_read(kind, dtype, tokens, page, heads, dim):
    rng = np.random.default_rng(tokens * 1000 + dim)
    pages = tokens // page + 3
    cache = empty_cache(kind, pages, page, heads, dim)
    slots = rng.permutation(pages * page)[:tokens].astype(np.int64)
    slots[rng.random(tokens) < 0.1] = rng.choice([-1, -(1 << 40), pages * page, 1 << 40])
    k, v = draw(rng, (tokens, heads, dim), dtype), draw(rng, (tokens, heads, dim), dtype)
    handle, at = dl.KvCache(*cache), torch.from_numpy(slots).cuda()
    dl.dl_kv_write(handle, dl.KvRows(k, v, at), torch.cuda.current_stream())
    check_written(cache, k, v, slots, kind)
    k2, v2 = torch.full_like(k, 3.0), torch.full_like(v, 3.0)
    dl.dl_kv_read(handle, dl.KvRows(k2, v2, at), torch.cuda.current_stream())
    keep = (slots >= 0) & (slots < pages * page)
    for new, old in ((k2, k), (v2, v)):
        y, z = decode_ref.quantised(old.double().cpu().numpy(), kind)
        want = torch.from_numpy((y.astype(np.float32) * z[..., None]) * keep[:, None, None].astype(np.float32)).to(dtype)
        assert torch.equal(new.cpu(), want)
        # against the rows themselves: half a step of the codes (of a row's largest for int8, of each value for fp8, below
        # 2^-6 of them of that), three roundings to 32 bits on the way and the one to the type
        x, got = old.double().cpu().numpy()[keep], new.double().cpu().numpy()[keep]
        top = np.abs(x).max(-1, keepdims=True)
        step = top / 127 / 2 if kind == "int8" else np.maximum(np.abs(x) * 2.0 ** -4, top / 448 * 2.0 ** -10)
        assert (np.abs(got - x) <= (step + 2.0 ** -21 * np.abs(x)) * (1 + decode_ref.UNIT[dtype]) + decode_ref.UNIT[dtype] * np.abs(x) + 2.0 ** -24).all()


@pytest.mark.parametrize("kind", ["fp8", "int8"])
def test_every_value_of_16_bits(kind):
    """All bfloat16 and float16 values, in rows of 16 that begin with the row's largest: every rounding there is."""
    rng = np.random.default_rng(1)
    for dtype in (torch.bfloat16, torch.float16):
        every = torch.arange(65536, dtype=torch.int32).to(torch.int16).view(dtype)
        every = every[torch.isfinite(every.float())]
        every = every[torch.from_numpy(rng.permutation(every.numel()))][: every.numel() // 16 * 16]
        rows = torch.sort(every.reshape(-1, 16).float().abs(), dim=1, descending=True)[0].to(dtype)
        near = (rng.uniform(-1, 1, rows.shape) * rows[:, :1].double().numpy())  # of the size of the row's largest
        for x in (rows, torch.from_numpy(near).to(dtype)):
            x = x.unsqueeze(1).contiguous().cuda()
            n = x.shape[0]
            cache = empty_cache(kind, (n + 15) // 16, 16, 1, 16)
            slots = np.arange(n, dtype=np.int64)
            dl.dl_kv_write(dl.KvCache(*cache), dl.KvRows(x, None, torch.from_numpy(slots).cuda()), torch.cuda.current_stream())
            check_written(cache, x, None, slots, kind)


@pytest.mark.parametrize("kind", ["fp8", "int8"])
def test_rows_that_are_not_finite_or_tiny(kind):
    x = torch.zeros((9, 1, 32))
    x[0, 0, 3], x[1, 0, 4], x[2, 0, 5] = float("inf"), float("-inf"), float("nan")
    x[0, 0, 7] = 1.0
    x[3] = 1e-45
    x[4] = 2.0 ** -110
    x[5, 0, 0] = 3.0e38
    x[6, 0, :2] = torch.tensor([2.0 ** -100, -(2.0 ** -101)])
    x[7] = -0.0
    x = x.cuda()
    cache = empty_cache(kind, 1, 16, 1, 32)
    slots = torch.arange(9, device="cuda")
    dl.dl_kv_write(dl.KvCache(*cache), dl.KvRows(None, x, slots), torch.cuda.current_stream())
    check_written(cache, None, x, slots.cpu().numpy(), kind)
    back = torch.empty_like(x)
    dl.dl_kv_read(dl.KvCache(*cache), dl.KvRows(None, back, slots), torch.cuda.current_stream())
    back = back.cpu()
    assert torch.isnan(back[:3]).all() and torch.isfinite(back[3:]).all()
    assert abs(float(back[5, 0, 0]) / 3.0e38 - 1) < 1e-6


@pytest.mark.parametrize("order", list(itertools.permutations(range(3))))
def test_any_order_and_stride(order):
    """The cache in every order of its dimensions; rows that are slices of wider ones, off every alignment but the element's."""
    rng = np.random.default_rng(5)
    cache = empty_cache("fp8", 6, 16, 3, 64, order)
    wide = torch.from_numpy(rng.standard_normal(40 * 3 * 2 * 70 + 3)).to(torch.bfloat16).cuda()
    rows = wide[3:].view(40, 3, 2, 70)
    k, v = rows[:, :, 0, 1:65], rows[:, :, 1, 5:69]
    slots = rng.permutation(96)[:40].astype(np.int64)
    handle, at = dl.KvCache(*cache), torch.from_numpy(slots).cuda()
    dl.dl_kv_write(handle, dl.KvRows(k, v, at), torch.cuda.current_stream())
    check_written(cache, k, v, slots, "fp8")
    before = wide.clone()
    dl.dl_kv_read(handle, dl.KvRows(k, v, at), torch.cuda.current_stream())
    inside = torch.zeros_like(wide, dtype=torch.bool)
    inside[3:].view(40, 3, 2, 70)[:, :, 0, 1:65] = True
    inside[3:].view(40, 3, 2, 70)[:, :, 1, 5:69] = True
    assert torch.equal(before[~inside], wide[~inside])
    y, z = decode_ref.quantised(before[3:].view(40, 3, 2, 70)[:, :, 1, 5:69].double().cpu().numpy(), "fp8")
    assert torch.equal(v.cpu(), torch.from_numpy(y.astype(np.float32) * z[..., None]).to(torch.bfloat16))


def test_blocks_that_hold_codes_and_scales():
    """A page as one block: keys, values and both scales behind each other, moved between pools by dl_batch_copy."""
    rng = np.random.default_rng(6)
    pages, page, heads, dim = 7, 16, 2, 64
    codes, scales = page * heads * dim, page * heads * 4
    block = 2 * (codes + scales)

    def views(pool):
        k, v = (pool[:, o:o + codes].view(pages, page, heads, dim).view(torch.float8_e4m3fn) for o in (0, codes))
        ks, vs = (pool[:, o:o + scales].view(torch.float32).view(pages, page, heads) for o in (2 * codes, 2 * codes + scales))
        return k, v, ks, vs

    a, b = (torch.zeros((pages, block), dtype=torch.uint8, device="cuda") for _ in range(2))
    T = pages * page
    k, v = draw(rng, (T, heads, dim), torch.bfloat16), draw(rng, (T, heads, dim), torch.bfloat16)
    order = rng.permutation(pages)
    stream = torch.cuda.current_stream()
    dl.dl_kv_write(dl.KvCache(*views(a)), dl.KvRows(k, v, torch.arange(T, device="cuda")), stream)
    dl.dl_batch_copy([(a.data_ptr() + i * block, b.data_ptr() + int(j) * block, block) for i, j in enumerate(order)], stream)
    slots = torch.from_numpy((order[:, None] * page + np.arange(page)).reshape(-1)).cuda()
    k2, v2 = torch.empty_like(k), torch.empty_like(v)
    dl.dl_kv_read(dl.KvCache(*views(b)), dl.KvRows(k2, v2, slots), stream)
    for new, old in ((k2, k), (v2, v)):
        y, z = decode_ref.quantised(old.double().cpu().numpy(), "fp8")
        assert torch.equal(new.cpu(), torch.from_numpy(y.astype(np.float32) * z[..., None]).to(torch.bfloat16))


def test_cache_beyond_32_bits():
    """Slots whose codes lie more than 4 GiB behind the start of the pool."""
    page, heads, dim = 16, 8, 128
    pages = (5 << 30) // (page * heads * dim)
    pool = torch.empty((pages, page, heads, dim), dtype=torch.uint8, device="cuda").view(torch.int8)
    scale = torch.zeros((pages, page, heads), device="cuda")
    slots = torch.tensor([pages * page - 1, 0, pages * page // 2 + 3, (pages - 1) * page], device="cuda")
    x = torch.randn((4, heads, dim), device="cuda")
    stream = torch.cuda.current_stream()
    cache = dl.KvCache(pool, pool, scale, scale)
    dl.dl_kv_write(cache, dl.KvRows(x, None, slots), stream)
    back = torch.empty_like(x)
    dl.dl_kv_read(cache, dl.KvRows(back, None, slots), stream)
    y, z = decode_ref.quantised(x.double().cpu().numpy(), "int8")
    assert torch.equal(back.cpu(), torch.from_numpy(y.astype(np.float32) * z[..., None]))
    assert torch.equal(pool.view(pages * page, heads, dim)[slots].double().cpu(), torch.from_numpy(y))


def test_on_another_stream_and_in_a_graph():
    side = torch.cuda.Stream()
    cache = empty_cache("fp8", 4, 16, 2, 64)
    x = torch.randn((20, 2, 64), device="cuda")
    back = torch.zeros_like(x)
    slots = torch.randperm(64, device="cuda")[:20].contiguous()
    handle, rows, out = dl.KvCache(*cache), dl.KvRows(x, x, slots), dl.KvRows(back, None, slots)
    side.wait_stream(torch.cuda.current_stream())
    with torch.cuda.stream(side):
        dl.dl_kv_write(handle, rows, side)
        dl.dl_kv_read(handle, out, side)
        side.synchronize()
        graph = torch.cuda.CUDAGraph()
        with torch.cuda.graph(graph, stream=side):
            dl.dl_kv_write(handle, rows, side)
            dl.dl_kv_read(handle, out, side)
    for _ in range(4):
        x.normal_()
        slots.copy_(torch.randperm(64, device="cuda")[:20])
        torch.cuda.synchronize()
        graph.replay()
        torch.cuda.synchronize()
        y, z = decode_ref.quantised(x.double().cpu().numpy(), "fp8")
        assert torch.equal(back.cpu(), torch.from_numpy(y.astype(np.float32) * z[..., None]))


def test_nothing_to_do():
    cache = empty_cache("fp8", 2, 16, 2, 64)
    none = torch.empty((0, 2, 64), device="cuda")
    rows = dl.KvRows(none, none, torch.empty((0,), dtype=torch.int64, device="cuda"))
    dl.dl_kv_write(dl.KvCache(*cache), rows, torch.cuda.current_stream())
    dl.dl_kv_read(dl.KvCache(*cache), rows, torch.cuda.current_stream())
    # a pool without pages: no slot is one
    empty = empty_cache("fp8", 0, 16, 2, 64)
    x = torch.ones((3, 2, 64), device="cuda")
    slots = torch.arange(3, device="cuda")
    dl.dl_kv_write(dl.KvCache(*empty), dl.KvRows(x, x, slots), torch.cuda.current_stream())
    dl.dl_kv_read(dl.KvCache(*empty), dl.KvRows(x, None, slots), torch.cuda.current_stream())
    assert not x.any()
    assert bool((cache[2] == 5).all())
