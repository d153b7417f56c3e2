"""dl_chunk_attention with more tiles times heads than one side of a launch holds: 2^24 workgroups of 256 threads."""

import pytest
import torch

import paper_2511_06605_amd as dl

from decode_ref import UNIT

pytestmark = pytest.mark.gpu

HEADS, DIM, PAGES = 65535, 16, 3


@pytest.fixture(scope="module", autouse=True)
def library():
    torch.cuda.set_device(0)
    dl.dl_init(0)
    yield
    dl.dl_shutdown()


@pytest.mark.parametrize("batch", [256, 257])
def test_a_token_a_sequence(batch):
    """Each of `batch` sequences has one token, which attends to itself alone: the output is its value, the lse its score."""
    assert (batch * HEADS >= 1 << 24) == (batch == 257)
    g = torch.Generator(device="cuda").manual_seed(batch)
    codes = [torch.randint(-127, 128, (PAGES, 1, HEADS, DIM), dtype=torch.int8, device="cuda", generator=g) for _ in range(2)]
    scales = [0.01 + 0.01 * torch.rand((PAGES, 1, HEADS), device="cuda", generator=g) for _ in range(2)]
    q = torch.randn((batch, HEADS, DIM), device="cuda", generator=g).bfloat16()
    room = torch.full((batch + 2, HEADS, DIM), 7.0, dtype=torch.bfloat16, device="cuda")
    lses = torch.full((batch + 2, HEADS), 7.0, device="cuda")
    pages = (torch.arange(batch, dtype=torch.int32, device="cuda") % PAGES).view(batch, 1)
    r = dl.ChunkAttention(dl.KvCache(codes[0], codes[1], scales[0], scales[1]), q, room[1:-1], torch.arange(batch + 1, dtype=torch.int32, device="cuda"), pages,
                          torch.ones(batch, dtype=torch.int32, device="cuda"), lse=lses[1:-1])
    r.use_workspace(torch.zeros(dl.dl_chunk_attention_workspace(r), dtype=torch.uint8, device="cuda"))
    dl.dl_chunk_attention(r, torch.cuda.current_stream())
    k, v = (c[:, 0].double() * s[:, 0].double()[..., None] for c, s in zip(codes, scales))
    unit = UNIT[torch.bfloat16]
    for b in range(batch):
        kb, vb, qb = k[b % PAGES], v[b % PAGES], q[b].double()
        # As decode_ref.attention_bounds has it: an exponent off by e, the weight and the output rounded to bfloat16.
        e = (DIM + 8) * 2.0 ** -24 * (kb.abs() * qb.abs()).sum(-1) * DIM ** -0.5 + 2.0 ** -16
        bound = unit * vb.abs() + (1 + unit) * (unit + torch.expm1(2 * e) + 2.0 ** -16)[:, None] * vb.abs() + 2.0 ** -24
        assert ((room[1 + b].double() - vb).abs() <= bound).all(), b
        score = (kb * qb).sum(-1) * DIM ** -0.5
        assert ((lses[1 + b].double() - score).abs() <= e + 2.0 ** -16 + 2.0 ** -22 * score.abs()).all(), b
    assert (room[0] == 7).all() and (room[-1] == 7).all() and (lses[0] == 7).all() and (lses[-1] == 7).all()
