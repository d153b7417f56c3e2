"""The operators that take a prompt into a bounded cache where sizes are large: pages further apart than 32 bits count, tables with room for
2^30 tokens, many heads, calls that a launch does not hold."""

import numpy as np
import pytest
import torch

import paper_2511_06605_amd as dl

import prompt_ref
import test_prompt_host as host
from prompt_ref import Packed


@pytest.mark.parametrize("make,size", [(host.chunk, dl.dl_chunk_attention_workspace), (host.weigh, dl.dl_kv_weigh_workspace)])
def test_workspaces_do_not_grow_with_the_table(make, size):
    r = make()
    small = size(r)
    r.desc.max_pages, r.desc.batch = 1 << 26, 1  # 2^30 tokens of 16 a page
    assert size(r) <= max(small, 65536 + 2 * 512 * 128 * (64 * 4 + 8) + (1 << 20))


def test_rows_that_a_call_may_have():
    r = host.chunk()
    for tokens, heads, fine in ((1 << 26, 1, True), ((1 << 26) + 1, 1, False), (1 << 25, 2, True), (1 << 25, 4, False), (1, 65536, True), (1, 65538, False)):
        r.cache.desc.heads = 2 if heads % 2 == 0 else 1
        r.desc.tokens, r.desc.q_heads = tokens, heads
        if fine:
            assert dl.dl_chunk_attention_workspace(r) >= 65536
        else:
            host.refused(lambda: dl.dl_chunk_attention_workspace(r), tokens=tokens, heads=heads)


@pytest.fixture(scope="module")
def library():
    torch.cuda.set_device(0)
    dl.dl_init(0)
    yield
    dl.dl_shutdown()


def spread(p, gap):
    """The cache of p with its pages `gap` bytes of codes (and as many of scales) apart."""
    n = p.k.shape[0]
    made = []
    for codes, scale in ((p.k, p.k_scale), (p.v, p.v_scale)):
        room = torch.empty(((n - 1) * gap + codes[0].numel(),), dtype=torch.int8, device="cuda")
        far = room.as_strided(codes.shape, (gap, *codes[0].contiguous().stride()))
        far.copy_(codes.view(torch.int8))
        scales = torch.empty(((n - 1) * gap // 4 + scale[0].numel(),), device="cuda")
        far_scale = scales.as_strided(scale.shape, (gap // 4, *scale[0].contiguous().stride()))
        far_scale.copy_(scale)
        made.append((far.view(codes.dtype), far_scale))
    (p.k, p.k_scale), (p.v, p.v_scale) = made


@pytest.mark.gpu
def test_pages_further_apart_than_32_bits_count(library):
    p = Packed([(20, 70), (3, 40)], heads=2, group=3, more_pages=4)
    spread(p, 3 << 29)  # 1.5 GiB
    assert p.k.stride()[0] * (p.k.shape[0] - 1) > 1 << 33
    out, lse = torch.empty_like(p.q), torch.empty(p.q.shape[:2], device="cuda")
    r = dl.ChunkAttention(p.cache(), p.q, out, *p.plan(), lse=lse, scale=p.scale)
    r.use_workspace(torch.zeros(dl.dl_chunk_attention_workspace(r), dtype=torch.uint8, device="cuda"))
    dl.dl_chunk_attention(r, torch.cuda.current_stream())
    p.check_attention(out, lse)
    weights = torch.empty((2, p.table.shape[1] * 16), device="cuda")
    r = dl.KvWeigh(p.cache(), p.q, lse, *p.plan(), weights, scale=p.scale)
    r.use_workspace(torch.zeros(dl.dl_kv_weigh_workspace(r), dtype=torch.uint8, device="cuda"))
    dl.dl_kv_weigh(r, torch.cuda.current_stream())
    want, bound = p.weighed(lse.double().cpu().numpy(), None)
    assert (np.abs(weights.double().cpu().numpy() - want) <= bound).all()
    kept, kept_lens = torch.empty((2, 30), dtype=torch.int32, device="cuda"), torch.empty(2, dtype=torch.int32, device="cuda")
    to = p.free[:4].reshape(2, 2)
    r = dl.KvEvict(p.cache(), weights, *p.plan()[1:], p.put(to), kept, kept_lens)
    r.use_workspace(torch.zeros(dl.dl_kv_evict_workspace(r), dtype=torch.uint8, device="cuda"))
    before = p.k.view(torch.int8).cpu().numpy(), p.v_scale.cpu().numpy()
    dl.dl_kv_evict(r, torch.cuda.current_stream())
    after = p.k.view(torch.int8).cpu().numpy(), p.v_scale.cpu().numpy()
    for b, (_, n) in enumerate(p.sizes):
        stay = prompt_ref.evicted(weights[b].cpu().numpy(), n, 30, 0, 0)
        assert kept[b].tolist() == stay
        for j, i in enumerate(stay):
            for x, y in zip(before, after):
                assert np.array_equal(x[p.table[b, i // 16], i % 16], y[to[b, j // 16], j % 16], equal_nan=True)


@pytest.mark.gpu
@pytest.mark.parametrize("batch", [2, 20])
def test_tables_with_room_for_2_to_the_30_tokens(library, batch):
    """Pages of 65536 tokens, most of the table no page."""
    p = Packed([(5, 100)] * (batch - 1) + [(40, 900)], heads=1, group=2, dim=16, page=65536)
    starts, table, lens = p.plan()
    wide = torch.full((batch, 1 << 14), -1, dtype=torch.int32, device="cuda")
    wide[:, :table.shape[1]] = table
    out, lse = torch.empty_like(p.q), torch.empty(p.q.shape[:2], device="cuda")
    r = dl.ChunkAttention(p.cache(), p.q, out, starts, wide, lens, lse=lse, scale=p.scale)
    r.use_workspace(torch.zeros(dl.dl_chunk_attention_workspace(r), dtype=torch.uint8, device="cuda"))
    dl.dl_chunk_attention(r, torch.cuda.current_stream())
    p.check_attention(out, lse)


@pytest.mark.gpu
def test_many_heads(library):
    """More heads of a cache than there are workgroups at once."""
    p = Packed([(2, 90), (3, 3)], heads=1100, group=1, dim=16)
    out, lse = torch.empty_like(p.q), torch.empty(p.q.shape[:2], device="cuda")
    r = dl.ChunkAttention(p.cache(), p.q, out, *p.plan(), lse=lse, scale=p.scale)
    r.use_workspace(torch.zeros(dl.dl_chunk_attention_workspace(r), dtype=torch.uint8, device="cuda"))
    dl.dl_chunk_attention(r, torch.cuda.current_stream())
    p.check_attention(out, lse)
