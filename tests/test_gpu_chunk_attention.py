"""Attention of chunks of new tokens over a paged cache (dl_chunk_attention) against a plain implementation in 64 bits on the CPU, query by
query."""

import numpy as np
import pytest
import torch

import paper_2511_06605_amd as dl

from prompt_ref import Packed

pytestmark = pytest.mark.gpu


@pytest.fixture(scope="module", autouse=True)
def library():
    torch.cuda.set_device(0)
    dl.dl_init(0)
    yield
    dl.dl_shutdown()


@pytest.fixture(scope="module")
def workspace():
    """One for all calls, full of what the calls before left behind."""
    w = torch.full((1 << 28,), 0xFF, dtype=torch.uint8, device="cuda")  # (NaN, as numbers)
    w[:65536] = 0
    return w


def request(p, workspace, out=None, q=None, plan=None):
    p.out = torch.full_like(p.q, 7.0) if out is None else out
    p.lse = torch.full(p.q.shape[:2], 7.0, device="cuda")
    r = dl.ChunkAttention(p.cache(), p.q if q is None else q, p.out, *(p.plan() if plan is None else plan), lse=p.lse, scale=p.scale)
    assert dl.dl_chunk_attention_workspace(r) <= workspace.numel()
    r.use_workspace(workspace)
    return r


def check(p, workspace, dead=(), **more):
    dl.dl_chunk_attention(request(p, workspace, **more), torch.cuda.current_stream())
    rows = p.check_attention(p.out, p.lse, dead)
    other = torch.from_numpy(~rows).cuda()
    assert (p.out[other] == 7).all() and (p.lse[other] == 7).all()  # rows of no sequence stay as they are
    return p.out, p.lse


TYPES = [(torch.bfloat16, "fp8"), (torch.float16, "int8"), (torch.bfloat16, "int8"), (torch.float16, "fp8")]


@pytest.mark.parametrize("dtype,kind", TYPES)
@pytest.mark.parametrize("dim,heads,group", [(64, 2, 1), (128, 1, 7), (256, 1, 3), (80, 2, 4), (16, 3, 2), (96, 1, 20), (208, 1, 8)])
def test_types_and_heads(workspace, dtype, kind, dim, heads, group):
    check(Packed([(5, 5), (3, 70), (20, 90)], heads=heads, group=group, dim=dim, dtype=dtype, kind=kind, seed=dim + group, gaps=2), workspace)


@pytest.mark.parametrize("dtype,kind", TYPES[:2])
@pytest.mark.parametrize("page", [1, 5, 8, 16, 24, 64, 128])
def test_pages_that_end_anywhere(workspace, dtype, kind, page):
    check(Packed([(1, 1), (31, 64), (2, 33), (33, 100)], page=page, group=2, heads=1, dtype=dtype, kind=kind, seed=page, spare=2), workspace)


@pytest.mark.parametrize("sizes", [
    [(1, 1)], [(1, 0)], [(0, 5)], [(0, 0)], [(3, 1)], [(5, 0), (2, 7), (0, 3), (4, 4)], [(63, 63)], [(64, 64)], [(65, 65)], [(129, 130)], [(1, 300)],
    [(7, 1000)], [(1, 64), (1, 65), (1, 63)], [(40, 20), (20, 40)], [(1, 9)] * 70])
def test_lengths(workspace, sizes):
    for dtype, kind in TYPES[:2]:
        check(Packed(sizes, heads=1, group=3, dtype=dtype, kind=kind, seed=len(sizes)), workspace)


@pytest.mark.parametrize("heads,group,sizes", [(1, 1, [(130, 1500)]), (1, 8, [(40, 700), (1, 900), (3, 10)]), (2, 4, [(33, 600)]), (1, 3, [(1, 2500)] * 3)])
def test_long_axes_are_cut(workspace, heads, group, sizes):
    """Few tiles: pieces of their keys by several workgroups, joined."""
    for dtype, kind in TYPES[:2]:
        check(Packed(sizes, heads=heads, group=group, dtype=dtype, kind=kind, seed=group), workspace)


def test_batches_of_more_than_64_that_are_cut(workspace):
    check(Packed([(1, 3)] * 80 + [(2, 1200), (5, 40)] + [(0, 9)] * 50 + [(1, 900)], heads=1, group=2, dim=16), workspace)


@pytest.mark.parametrize("dtype,kind", TYPES)
@pytest.mark.parametrize("dim,heads,group,sizes", [
    (64, 1, 16, [(64, 64)]), (128, 1, 16, [(70, 200)]), (80, 2, 20, [(52, 700)]), (16, 1, 64, [(17, 20), (20, 1)]), (128, 1, 32, [(33, 33), (40, 1500), (30, 64)]),
    (96, 1, 100, [(11, 129)]), (48, 1, 128, [(8, 65), (9, 128), (0, 40), (15, 13)])])
@pytest.mark.parametrize("room", [0, 2048])
def test_many_rows(workspace, dtype, kind, dim, heads, group, sizes, room):
    """Enough rows a sequence for the kernel with 256 rows a tile, which tables of 2048 tokens and more have."""
    assert sum(m for m, _ in sizes) * group >= 1024 * len(sizes) or len(sizes) > 3
    check(Packed(sizes, heads=heads, group=group, dim=dim, dtype=dtype, kind=kind, seed=dim, gaps=1, room=room), workspace)


@pytest.mark.parametrize("page", [1, 5, 24, 128])
def test_many_rows_and_pages_that_end_anywhere(workspace, page):
    check(Packed([(35, 300), (33, 40)], page=page, group=32, heads=1, dim=32, seed=page, room=2100), workspace)


def test_many_rows_and_what_is_none(workspace):
    p = Packed([(40, 300)], heads=1, group=32, dim=32, room=2048)
    p.table[0, 1], p.table[0, 7], p.table[0, 18] = -1, 1 << 30, -1
    check(p, workspace, dead=[(0, 1), (0, 7), (0, 18)])
    for side in ("k_scale", "v_scale"):
        p = Packed([(40, 300)], heads=1, group=32, dim=32, room=2048)
        getattr(p, side)[int(p.table[0, 280 // 16]), 280 % 16, 0] = float("nan")
        out, _ = check(p, workspace)
        assert torch.isnan(out).any() and torch.isfinite(out[:19]).all()
    for dtype, kind in TYPES:
        p = Packed([(33, 200)], heads=1, group=32, dim=32, dtype=dtype, kind=kind, room=2048)
        for n, t in enumerate((3, 60, 140, 199)):
            p.v_scale[int(p.table[0, t // 16]), t % 16, 0] *= (2.0 ** -90, 2.0 ** -60, 2.0 ** -45, 0.0)[n]
        check(p, workspace)
    check(Packed([(40, 500)], heads=1, group=32, dim=32, q_size=12.0, spread=1.5, room=2048), workspace)


@pytest.mark.parametrize("order", [(0, 1, 2), (0, 2, 1), (2, 0, 1), (1, 0, 2)])
def test_orders_of_a_cache(workspace, order):
    check(Packed([(3, 50), (9, 20)], order=order, group=2), workspace)


def test_strides_of_queries_and_outputs(workspace):
    p = Packed([(6, 40), (11, 11)], heads=2, group=3, dim=80)
    q = torch.empty((6, p.tokens, 83), dtype=p.dtype, device="cuda").permute(1, 0, 2)[..., 1:81]
    q.copy_(p.q)
    out = torch.full((p.tokens, 7, 85), 7.0, dtype=p.dtype, device="cuda")
    check(p, workspace, q=q, out=out[:, 1:, 3:83])
    out[:, 1:, 3:83] = 7
    assert (out == 7).all()


def test_large_scores(workspace):
    for dtype, kind in TYPES[:2]:
        check(Packed([(30, 100), (5, 300)], dtype=dtype, kind=kind, q_size=12.0, spread=1.5, group=2), workspace)


@pytest.mark.parametrize("sizes", [[(20, 100)], [(3, 1500)]])
def test_pages_that_are_none(workspace, sizes):
    p = Packed(sizes, heads=1, group=2)
    for page, value in ((1, -1), (3, 1 << 30)):
        p.table[0, page] = value
    check(p, workspace, dead=[(0, 1), (0, 3)])
    p = Packed(sizes, heads=1, group=2)
    p.table[:] = -1
    check(p, workspace, dead=[(0, x) for x in range(200)])


@pytest.mark.parametrize("sizes", [[(40, 100)], [(70, 1300)]])
@pytest.mark.parametrize("side", ["k_scale", "v_scale"])
def test_a_scale_of_nan_reaches_those_that_see_it(workspace, sizes, side):
    """The key of a new token: the queries before it do not see it."""
    p = Packed(sizes, heads=2, group=2)
    t = sizes[0][1] - 12
    getattr(p, side)[int(p.table[0, t // 16]), t % 16, 1] = float("nan")
    out, _ = check(p, workspace)
    assert torch.isnan(out).any() and torch.isfinite(out[:, :2]).all()


@pytest.mark.parametrize("dtype,kind", TYPES)
def test_scales_far_apart(workspace, dtype, kind):
    """Values whose scales lie far beyond those that the sums take whole, among ordinary ones."""
    p = Packed([(20, 150)], heads=1, group=2, dtype=dtype, kind=kind)
    for n, t in enumerate((3, 60, 140, 149)):
        p.v_scale[int(p.table[0, t // 16]), t % 16, 0] *= (2.0 ** -90, 2.0 ** -60, 2.0 ** -45, 0.0)[n]
    check(p, workspace)


def test_more_queries_than_tokens(workspace):
    check(Packed([(50, 13), (200, 64)], heads=1, group=2, dim=16), workspace)


def test_starts_that_decrease_or_leave_the_rows(workspace):
    """Nothing outside the rows is read or written, whatever they say."""
    p = Packed([(20, 60), (20, 60), (20, 60)], heads=1, group=2)
    _, pages, lens = p.plan()
    for starts in ([0, 1 << 30, -5, 60], [50, 10, 70, 2], [-(1 << 31), (1 << 31) - 1, 0, (1 << 31) - 1]):
        room = torch.full((p.tokens + 20, 2, 64), 7.0, dtype=p.dtype, device="cuda")
        r = request(p, workspace, out=room[10:-10], plan=(torch.tensor(starts, dtype=torch.int32, device="cuda"), pages, lens))
        dl.dl_chunk_attention(r, torch.cuda.current_stream())
        assert (room[:10] == 7).all() and (room[-10:] == 7).all()


def test_lengths_beyond_the_table(workspace):
    p = Packed([(20, 64), (5, 32)], heads=1, group=2)
    starts, pages, lens = p.plan()
    out, lse = check(p, workspace)
    # 64 tokens fit the table: a longer length counts as that, a negative one as none
    dl.dl_chunk_attention(request(p, workspace, plan=(starts, pages, torch.tensor([1 << 30, -3], dtype=torch.int32, device="cuda"))), torch.cuda.current_stream())
    assert torch.equal(p.out[:20], out[:20]) and torch.equal(p.lse[:20], lse[:20])
    assert not p.out[20:].any() and (p.lse[20:] == -np.inf).all()


def test_nothing_to_do(workspace):
    p = Packed([(4, 4)])
    starts, pages, lens = p.plan()
    none = p.q[:0]
    r = dl.ChunkAttention(p.cache(), none, torch.empty_like(none), torch.zeros(2, dtype=torch.int32, device="cuda"), pages, lens)
    r.use_workspace(workspace)
    dl.dl_chunk_attention(r, torch.cuda.current_stream())
    empty = torch.zeros((0, 2), dtype=torch.int32, device="cuda")
    r = dl.ChunkAttention(p.cache(), p.q, p.q.clone(), torch.zeros(1, dtype=torch.int32, device="cuda"), empty, lens[:0])
    r.use_workspace(workspace)
    dl.dl_chunk_attention(r, torch.cuda.current_stream())


def test_the_same_bits_again(workspace):
    p = Packed([(70, 400), (3, 1700)], heads=2, group=2)
    first = [t.clone() for t in check_free(p, workspace)]
    for _ in range(3):
        again = check_free(p, workspace)
        assert torch.equal(first[0], again[0]) and torch.equal(first[1], again[1])


def check_free(p, workspace):
    dl.dl_chunk_attention(request(p, workspace), torch.cuda.current_stream())
    return p.out, p.lse


def test_as_dl_prefix_attention_has_it(workspace):
    """Both operators on what both can say: a batch whose sequences have the same number of queries."""
    for dtype, kind in TYPES[:2]:
        p = Packed([(6, 200), (6, 77), (6, 6)], heads=2, group=4, dim=128, dtype=dtype, kind=kind)
        out, lse = check_free(p, workspace)
        q = p.q.view(3, 6, 8, 128)
        other, other_lse = torch.empty_like(q), torch.empty((3, 6, 8), device="cuda")
        _, pages, lens = p.plan()
        r = dl.PrefixAttention(p.cache(), q, other, pages, lens, lse=other_lse)
        r.use_workspace(workspace)
        dl.dl_prefix_attention(r, torch.cuda.current_stream())
        unit = 2.0 ** -8 if dtype == torch.bfloat16 else 2.0 ** -11
        # each weight and each output rounded once on either side
        assert (other.flatten(0, 1).float() - out.float()).abs().max() <= 4 * unit * out.float().abs().max()
        assert (other_lse.flatten(0, 1) - lse).abs().max() <= 2.0 ** -15 * (1 + lse.abs().max())
