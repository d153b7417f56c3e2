"""Kernels of the prompt operators that the sizes of the other tests do not reach, and workspaces of exactly the size that a call asks for, with
a guard behind them."""

import pytest
import torch

import paper_2511_06605_amd as dl

import test_gpu_chunk_attention as chunk
import test_gpu_kv_evict as evict
import test_gpu_kv_weigh as weigh
from prompt_ref import Packed
from test_gpu_chunk_attention import TYPES, library  # noqa: F401  (a fixture)

pytestmark = pytest.mark.gpu

GUARD = 1 << 20


class Exact:
    """`size` bytes, the front zero and the rest NaN as numbers, and more behind them that nobody may touch."""

    def __init__(self, size):
        self.room = torch.full((size + GUARD,), 0xFF, dtype=torch.uint8, device="cuda")
        self.room[:65536] = 0
        self.room[size:] = 0xA5
        self.size = size

    def __enter__(self):
        return self.room[:self.size]

    def __exit__(self, *what):
        if what[0] is None:
            assert (self.room[self.size:] == 0xA5).all(), "written behind the workspace"
            assert not self.room[:65536].any(), "the front is zero between calls"


def weigh_size(p):
    weights = torch.empty((p.table.shape[0], p.table.shape[1] * p.page), device="cuda")
    return dl.dl_kv_weigh_workspace(dl.KvWeigh(p.cache(), p.q, torch.empty(p.q.shape[:2], device="cuda"), *p.plan(), weights))


def run_weigh(p, parts):
    """parts: how many workgroups share the heads, in the kernel for many queries (None: that for few)."""
    rows, batch, width = p.tokens * p.group, len(p.sizes), p.table.shape[1] * p.page
    assert (rows > 32 * batch) == (parts is not None)
    size = weigh_size(p)
    assert size == 65536 + (4 * parts * batch * width if parts is not None and parts > 1 else 0)
    for with_before in (True, False):
        with Exact(size) as workspace:
            weigh.check(p, workspace, with_before)


@pytest.mark.parametrize("dtype,kind", TYPES)
@pytest.mark.parametrize("dim", [256, 208, 144])
def test_weights_from_many_queries_of_wide_heads(dtype, kind, dim):
    run_weigh(Packed([(20, 90), (5, 70), (33, 300)], heads=2, group=8, dim=dim, dtype=dtype, kind=kind, seed=dim, gaps=1), 2)


@pytest.mark.parametrize("dtype,kind", TYPES)
@pytest.mark.parametrize("heads,group,sizes", [(8, 4, [(1, 500)]), (2, 2, [(3, 40), (16, 300), (0, 9), (1, 1)]), (1, 32, [(1, 70)])])
def test_weights_from_few_queries_with_heads_of_128(dtype, kind, heads, group, sizes):
    run_weigh(Packed(sizes, heads=heads, group=group, dim=128, dtype=dtype, kind=kind, seed=heads), None)


# (width: blocks of 256 keys; 1024 workgroups are what heads are shared out up to)
@pytest.mark.parametrize("heads,blocks,parts", [(8, 200, 6), (8, 344, 3), (9, 600, 2), (3, 1024, 1), (7, 1030, 1), (2, 150, 2)])
@pytest.mark.parametrize("dim", [64, 128])
def test_workgroups_with_several_heads(heads, blocks, parts, dim):
    for dtype, kind in TYPES[:2]:
        run_weigh(Packed([(14, 520)], heads=heads, group=4, dim=dim, dtype=dtype, kind=kind, seed=blocks, room=256 * blocks), parts)


def test_workgroups_with_several_heads_of_more_than_one_sequence():
    run_weigh(Packed([(14, 520), (40, 40), (0, 30), (23, 700)], heads=5, group=4, dim=256, seed=3, room=256 * 100), 3)


def run_chunk(p, wide):
    assert (p.dim <= 128 and p.tokens * p.group >= 1024 * len(p.sizes) and p.table.shape[1] * p.page >= 2048) == wide
    r = dl.ChunkAttention(p.cache(), p.q, torch.empty_like(p.q), *p.plan(), lse=torch.empty(p.q.shape[:2], device="cuda"))
    with Exact(dl.dl_chunk_attention_workspace(r)) as workspace:
        chunk.check(p, workspace)


@pytest.mark.parametrize("dtype,kind", TYPES)
@pytest.mark.parametrize("heads,group,dim,sizes", [
    (2, 16, 64, [(64, 64)]), (2, 16, 128, [(70, 200)]), (3, 32, 16, [(33, 33), (40, 1500), (30, 64)]), (8, 32, 32, [(34, 300)])])
def test_many_rows_and_several_heads(dtype, kind, heads, group, dim, sizes):
    run_chunk(Packed(sizes, heads=heads, group=group, dim=dim, dtype=dtype, kind=kind, seed=heads + dim, gaps=1, room=2048), True)


@pytest.mark.parametrize("dtype,kind", TYPES[:2])
def test_many_rows_and_several_heads_on_a_long_axis(dtype, kind):
    run_chunk(Packed([(36, 2500)], heads=8, group=30, dim=128, dtype=dtype, kind=kind, seed=5), True)


@pytest.mark.parametrize("heads,group,dim,sizes", [
    (1, 1, 64, [(130, 1500)]), (2, 4, 256, [(33, 900)]), (3, 2, 208, [(5, 1200), (70, 70)]), (8, 4, 128, [(16, 516)]), (5, 3, 16, [(1, 2500)] * 3),
    (1, 2, 16, [(1, 3)] * 20 + [(2, 1200), (5, 40)])])
def test_cut_within_the_workspace(heads, group, dim, sizes):
    for dtype, kind in TYPES[:2]:
        run_chunk(Packed(sizes, heads=heads, group=group, dim=dim, dtype=dtype, kind=kind, seed=dim), False)


def test_evictions_within_the_workspace():
    with Exact(65536) as workspace:
        evict.check(workspace, [100, 3000, 0], 70, first=2, recent=5)
        evict.check(workspace, [40_000], 5000, first=2, recent=5, heads=1, dim=16)
