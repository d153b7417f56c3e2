"""The operators that take a prompt into a bounded cache on streams other than the default one, and captured into graphs.

Collected last: streams stay for the life of a process, the runtime maps them all to a few hardware queues, and armed requests in files
before this one must not find theirs shared with the streams that are made here."""

import numpy as np
import pytest
import torch

import paper_2511_06605_amd as dl

import prompt_ref
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
    w = torch.full((1 << 26,), 0xFF, dtype=torch.uint8, device="cuda")  # (NaN, as numbers)
    w[:65536] = 0
    return w


def test_norms_captured_and_replayed():
    """Positions are read when the kernel runs; on a stream of its own."""
    angle = torch.from_numpy(np.random.default_rng(5).uniform(-4.0, 4.0, (30, 32)))
    table = torch.cat([angle.cos(), angle.sin()], 1).float().cuda()
    q = torch.randn((7, 3, 64), device="cuda").half()
    out, positions = torch.full_like(q, 7.0), torch.zeros(7, dtype=torch.int64, device="cuda")
    r = dl.NormRotate(q, None, out, q_weight=torch.ones(64, device="cuda"), table=table, positions=positions)
    graph = torch.cuda.CUDAGraph()
    stream = torch.cuda.Stream()
    with torch.cuda.graph(graph, stream=stream):
        dl.dl_norm_rotate(r, stream)
    for n in range(4):
        positions.copy_(torch.randint(0, 30, (7,)))
        out.fill_(7)
        graph.replay()
        torch.cuda.synchronize()
        got = out.clone()
        dl.dl_norm_rotate(r, torch.cuda.current_stream())
        torch.cuda.synchronize()
        assert torch.equal(got, out) and not (got == 7).all()


def test_chunks_captured_and_replayed_as_lengths_grow(workspace):
    p = Packed([(8, 200), (3, 90)], heads=2, group=2, spare=3)
    for b in range(2):  # (pages for what is to come)
        used = -(-p.sizes[b][1] // 16)
        p.table[b, used:] = p.table[b, 0]
    starts, pages, lens = p.plan()
    lens.fill_(5)
    p.out, p.lse = torch.full_like(p.q, 7.0), torch.full(p.q.shape[:2], 7.0, device="cuda")
    r = dl.ChunkAttention(p.cache(), p.q, p.out, starts, pages, lens, lse=p.lse, scale=p.scale)
    r.use_workspace(workspace)
    stream = torch.cuda.Stream()
    stream.wait_stream(torch.cuda.current_stream())
    with torch.cuda.stream(stream):
        dl.dl_chunk_attention(r, stream)
    torch.cuda.current_stream().wait_stream(stream)
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        dl.dl_chunk_attention(r, torch.cuda.current_stream())
    for a, b in ((8, 3), (100, 50), (200, 90), (150, 0), (200, 90)):
        lens.copy_(torch.tensor([a, b], dtype=torch.int32))
        p.out.fill_(7)
        graph.replay()
        torch.cuda.synchronize()
        got, got_lse = p.out.clone(), p.lse.clone()
        dl.dl_chunk_attention(r, torch.cuda.current_stream())
        torch.cuda.synchronize()
        assert torch.equal(got, p.out) and torch.equal(got_lse, p.lse)
    p.check_attention(p.out, p.lse)


def test_weights_captured_and_replayed_as_lengths_grow(workspace):
    for sizes, group in (([(4, 300), (2, 90)], 2), ([(40, 300), (20, 90)], 4)):  # both kernels
        p = Packed(sizes, heads=2, group=group)
        starts, pages, lens = p.plan()
        lse = p.put(p.exact_lse()).float()
        weights = torch.zeros((2, p.table.shape[1] * 16), device="cuda")
        r = dl.KvWeigh(p.cache(), p.q, lse, starts, pages, lens, weights, scale=p.scale)
        r.use_workspace(workspace)
        graph = torch.cuda.CUDAGraph()
        with torch.cuda.graph(graph):
            dl.dl_kv_weigh(r, torch.cuda.current_stream())
        for a, b in ((40, 20), (300, 0), (100, 90), (300, 90)):
            lens.copy_(torch.tensor([a, b], dtype=torch.int32))
            weights.fill_(7)
            graph.replay()
            torch.cuda.synchronize()
            got = weights.clone()
            dl.dl_kv_weigh(r, torch.cuda.current_stream())
            torch.cuda.synchronize()
            assert torch.equal(got, weights)


def test_eviction_captured_and_replayed(workspace):
    p = Packed([(0, 300), (0, 90)], more_pages=8)
    weights = torch.rand((2, p.table.shape[1] * 16), device="cuda")
    kept, kept_lens = torch.zeros((2, 50), dtype=torch.int32, device="cuda"), torch.zeros(2, dtype=torch.int32, device="cuda")
    lens = torch.zeros(2, dtype=torch.int32, device="cuda")
    r = dl.KvEvict(p.cache(), weights, p.put(p.table), lens, p.put(p.free[:8].reshape(2, 4)), kept, kept_lens, first=3, recent=7)
    r.use_workspace(workspace)
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        dl.dl_kv_evict(r, torch.cuda.current_stream())
    for a, b in ((300, 90), (20, 51), (0, 50), (299, 89)):
        lens.copy_(torch.tensor([a, b], dtype=torch.int32))
        weights.uniform_()
        kept.fill_(7)
        graph.replay()
        torch.cuda.synchronize()
        for row, n, w in zip(kept.tolist(), (a, b), weights.cpu().numpy()):
            stay = prompt_ref.evicted(w, n, 50, 3, 7)
            assert row == stay + [-1] * (50 - len(stay))
        assert kept_lens.tolist() == [min(a, 50), min(b, 50)]


def test_calls_on_two_streams_at_once():
    """Each with a workspace of its own."""
    ps = [Packed([(40, 900), (9, 30)], heads=2, group=2, seed=s) for s in range(2)]
    streams = [torch.cuda.Stream() for _ in ps]
    asked = []
    for p in ps:
        p.out, p.lse = torch.empty_like(p.q), torch.empty(p.q.shape[:2], device="cuda")
        r = dl.ChunkAttention(p.cache(), p.q, p.out, *p.plan(), lse=p.lse, scale=p.scale)
        r.use_workspace(torch.zeros(dl.dl_chunk_attention_workspace(r), dtype=torch.uint8, device="cuda"))
        asked.append(r)
    torch.cuda.synchronize()
    for _ in range(20):
        for r, s in zip(asked, streams):
            dl.dl_chunk_attention(r, s)
    torch.cuda.synchronize()
    for p in ps:
        p.check_attention(p.out, p.lse)
