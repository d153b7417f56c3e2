"""The largest calls that dl_prefix_attention takes."""

import pytest
import torch

import paper_2511_06605_amd as dl

pytestmark = pytest.mark.gpu


@pytest.fixture(scope="module", autouse=True)
def library():
    torch.cuda.set_device(0)
    dl.dl_init(0)
    yield
    dl.dl_shutdown()


def test_as_many_rows_as_a_call_may_have():
    """DL_MAX_ROWS / 2 rows of queries on a prefix of one token: out is its value, lse the score, row by row."""
    batch, heads, dim = 4096, 16384, 16
    assert batch * heads == dl.DL_MAX_ROWS // 2
    g = torch.Generator(device="cuda").manual_seed(1)
    k, v = (torch.randint(-100, 101, (1, 1, 1, dim), device="cuda", generator=g).to(torch.int8) for _ in range(2))
    scale = torch.full((1, 1, 1), 2.0 ** -6, device="cuda")
    q = torch.empty((batch, 1, heads, dim), dtype=torch.bfloat16, device="cuda").normal_(generator=g)
    out, lse = torch.full_like(q, 7.0), torch.full((batch, 1, heads), 7.0, device="cuda")
    r = dl.PrefixAttention(dl.KvCache(k, v, scale, scale), q, out, torch.zeros((batch, 0), dtype=torch.int32, device="cuda"),
                           torch.zeros(batch, dtype=torch.int32, device="cuda"),
                           prefix_pages=torch.zeros(1, dtype=torch.int32, device="cuda"), prefix_tokens=1, lse=lse, scale=0.25)
    r.use_workspace(torch.zeros(dl.dl_prefix_attention_workspace(r), dtype=torch.uint8, device="cuda"))
    dl.dl_prefix_attention(r, torch.cuda.current_stream())
    # a weight divided by itself is 1 but for two roundings of 2^-24; codes of 7 bits are values of bfloat16
    want = v[0, 0, 0].float() * 2.0 ** -6
    for b in range(0, batch, 512):  # (a part at a time)
        assert torch.equal(out[b:b + 512], want.bfloat16().expand_as(out[b:b + 512]))
        score = (q[b:b + 512].float() * k[0, 0, 0].float()).sum(-1) * (0.25 * 2.0 ** -6)
        # 16 products of at most 100 x 6, times 2^-8, in 32 bits in any order, and a logarithm and a power of two on the way
        assert float((lse[b:b + 512] - score).abs().max()) <= 16 * 2.0 ** -24 * 16 * 600 * 2.0 ** -8 + 2.0 ** -15
