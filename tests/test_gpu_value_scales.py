"""Attention over a paged cache whose value rows are of very different sizes (dl_prefix_attention): rows of zeros, scales of zero, rows that
are 2^100 and more apart.  lse does not depend on the values at all, and out is right to what a query gives weight to."""

import numpy as np
import pytest
import torch

import paper_2511_06605_amd as dl

import decode_ref
from test_gpu_prefix_attention import Problem

pytestmark = pytest.mark.gpu

D, PAGE = 64, 16


@pytest.fixture(scope="module", autouse=True)
def library():
    torch.cuda.set_device(0)
    dl.dl_init(0)
    yield
    dl.dl_shutdown()


def check(k, v, dtype, kind, place, v_scale=None, seed=0):
    """k and v [n, D]: one head.  place: "own" (one sequence, one query token, all of them its own tokens), "narrow" (two sequences on a
    prefix) or "wide" (128 rows of queries on a prefix, 2^20 scores and more).  Queries are 8 or 4 in dimension 0, so that k[:, 0]
    alone, the rest of k being zero, sets the scores: k[:, 0] itself in nats, or half of it.  v_scale: scales to put in the place of
    what v's rows get, where it is not NaN."""
    n = len(k)
    rng = np.random.default_rng(seed)
    B, group = {"own": (1, 6), "narrow": (2, 3), "wide": (16, 8)}[place]
    assert place != "wide" or B * group * n >= 1 << 20
    pages = -(-n // PAGE)
    table = rng.permutation(pages)
    made, exact = [], []
    for x, forced in ((k, None), (v, v_scale)):
        y, z = decode_ref.quantised(x, kind)
        if forced is not None:
            z = np.where(np.isnan(forced), z, forced.astype(np.float32))
        exact.append(y * z.astype(np.float64)[:, None])
        codes, scale = np.zeros((pages * PAGE, D)), np.zeros(pages * PAGE, dtype=np.float32)
        slots = table[np.arange(n) // PAGE] * PAGE + np.arange(n) % PAGE
        codes[slots], scale[slots] = y, z
        # what lies behind the last token may hold anything
        behind = table[-1] * PAGE + np.arange(n - (pages - 1) * PAGE, PAGE)
        scale[behind] = rng.choice([np.inf, -np.inf, np.nan, -1.0, 3e38, 1e-45], len(behind))
        made += [torch.from_numpy(codes).float().to(decode_ref.CODE[kind]).view(pages, PAGE, 1, D).cuda(),
                 torch.from_numpy(scale).view(pages, PAGE, 1).cuda()]
    q = torch.from_numpy(rng.standard_normal((B, 1, group, D)))
    q[..., 0] = torch.from_numpy(rng.choice([8.0, 4.0], (B, 1, group)))
    q = q.to(dtype).cuda()
    out, lse = torch.full_like(q, 7.0), torch.full((B, 1, group), 7.0, device="cuda")
    at = torch.from_numpy(table.astype(np.int32)).cuda()
    cache = dl.KvCache(made[0], made[2], made[1], made[3])
    if place == "own":
        r = dl.PrefixAttention(cache, q, out, at[None], torch.tensor([n], dtype=torch.int32, device="cuda"), lse=lse)
    else:
        r = dl.PrefixAttention(cache, q, out, torch.zeros((B, 0), dtype=torch.int32, device="cuda"),
                               torch.zeros(B, dtype=torch.int32, device="cuda"), prefix_pages=at, prefix_tokens=n, lse=lse)
    r.use_workspace(torch.zeros(dl.dl_prefix_attention_workspace(r), dtype=torch.uint8, device="cuda"))
    dl.dl_prefix_attention(r, torch.cuda.current_stream())
    out, lse, q = out.double().cpu().numpy(), lse.double().cpu().numpy(), q.double().cpu().numpy()
    see = np.ones(n, dtype=bool)
    for b in range(B):
        for h in range(group):
            want, whole, mass, reach = decode_ref.attention(q[b, 0, h], *exact, see, D ** -0.5)
            bound, bound_lse = decode_ref.attention_bounds(want, whole, mass, reach, D, dtype)
            assert abs(lse[b, 0, h] - whole) <= bound_lse, ((b, h), lse[b, 0, h], whole, bound_lse)
            off = np.abs(out[b, 0, h] - want)
            assert (off <= bound).all(), ((b, h), float((off / bound).max()), out[b, 0, h][:4], want[:4])


def scores(values):
    k = np.zeros((len(values), D))
    k[:, 0] = values
    return k


EVERYWHERE = pytest.mark.parametrize("place", ["own", "narrow", "wide"])
TYPES = pytest.mark.parametrize("dtype,kind", [(torch.bfloat16, "fp8"), (torch.float16, "int8"), (torch.bfloat16, "int8"), (torch.float16, "fp8")])
N = 8192 + 3


@EVERYWHERE
@TYPES
def test_nothing_but_zeros(dtype, kind, place):
    check(np.zeros((N, D)), np.zeros((N, D)), dtype, kind, place)


@EVERYWHERE
@TYPES
def test_zeros_that_score_higher_and_higher(dtype, kind, place):
    """2^7.9 times the weight from one step to the next, so that no reference has to follow; ordinary rows at the end, or at the beginning."""
    rng = np.random.default_rng(1)
    v = np.zeros((N, D))
    v[-300:] = rng.standard_normal((300, D))
    s = np.full(N, 7.9 * np.log(2.0))
    s[:256] = 0.0
    check(scores(s), v, dtype, kind, place)
    check(scores(s[::-1]), v[::-1], dtype, kind, place)


@EVERYWHERE
@TYPES
def test_whole_pieces_of_zeros(dtype, kind, place):
    rng = np.random.default_rng(2)
    v = rng.standard_normal((N, D))
    v[:N // 4] = 0.0
    check(np.zeros((N, D)), v, dtype, kind, place)
    v = np.zeros((N, D))
    v[5000] = rng.standard_normal(D)  # one among zeros
    check(scores(np.where(np.arange(N) == 5000, 5.0, 0.0)), v, dtype, kind, place)


@EVERYWHERE
@TYPES
def test_scales_of_zero(dtype, kind, place):
    """Places of a zeroed pool that were never written stand for zeros."""
    rng = np.random.default_rng(3)
    v = rng.standard_normal((N, D))
    never = rng.random(N) < 0.5
    never[:1024] = True
    v[never] = 0.0
    check(scores(0.5 * rng.standard_normal(N)), v, dtype, kind, place, v_scale=np.where(never, 0.0, np.nan))
    check(np.zeros((N, D)), np.zeros((N, D)), dtype, kind, place, v_scale=np.zeros(N))


@EVERYWHERE
@pytest.mark.parametrize("kind", ["fp8", "int8"])
@pytest.mark.parametrize("large", [1e8, 1e15, 1e30, 1e36])
def test_large_rows_among_zeros(kind, large, place):
    rng = np.random.default_rng(4)
    v = np.zeros((N, D))
    v[rng.permutation(N)[:80]] = large
    check(np.zeros((N, D)), v, torch.bfloat16, kind, place)


@EVERYWHERE
@TYPES
@pytest.mark.parametrize("large", [1e8, 1e18])
def test_large_rows_without_weight(dtype, kind, large, place):
    """Ordinary rows, and large ones whose score takes them out of the sum: e^-80 (e^-160 with a query of 8) of the others."""
    rng = np.random.default_rng(5)
    v = rng.standard_normal((N, D))
    s = 0.5 * rng.standard_normal(N)
    far = rng.permutation(N)[:200]
    v[far] *= large
    s[far] = -160.0
    check(scores(s), v, dtype, kind, place)


@EVERYWHERE
@pytest.mark.parametrize("kind", ["fp8", "int8"])
@pytest.mark.parametrize("decades", [10, 25, 35])
def test_rows_of_every_size(kind, decades, place):
    """10^-decades to 10^decades: the large ones make the output, all of them lse."""
    rng = np.random.default_rng(decades)
    v = rng.standard_normal((N, D)) * 10.0 ** rng.uniform(-decades, decades, (N, 1))
    check(scores(rng.standard_normal(N)), v, torch.bfloat16, kind, place)
    # and each size by itself
    for size in (10.0 ** -decades, 10.0 ** decades):
        check(scores(rng.standard_normal(N)), rng.standard_normal((N, D)) * size, torch.bfloat16, kind, place)


@TYPES
def test_a_large_draft_is_seen_from_its_own_query_on(dtype, kind):
    """Rows of zeros, and a draft of enormous values: the queries before it do not see it, those from it on do."""
    p = Problem([200, 70], prefix=150, q_tokens=4, group=2, dtype=dtype, kind=kind, seed=6)
    p.v.view(torch.uint8)[p.table[0, :4]] = 0
    p.v_scale[p.table[0, :4]] = 2.0 ** -100 * float(np.float32(1) / np.float32(decode_ref.LIMIT[kind]))
    for b, t in ((0, 198), (1, 67)):
        p.v_scale[int(p.table[b, t // 16]), t % 16] *= 2.0 ** (90 if dtype == torch.bfloat16 else 8)
    p.check(torch.zeros(1 << 24, dtype=torch.uint8, device="cuda"))
