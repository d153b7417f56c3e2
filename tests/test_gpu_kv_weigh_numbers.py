"""Queries that hold no numbers, and so have no lse (dl_kv_weigh, dl_chunk_attention): they give nothing, and what others give stays as it is."""

import numpy as np
import pytest
import torch

import paper_2511_06605_amd as dl

from prompt_ref import Packed
from test_gpu_kv_weigh import TYPES, check, library, workspace  # noqa: F401  (fixtures)

pytestmark = pytest.mark.gpu

NAN, INF = float("nan"), float("inf")


def spoil(p, rows):
    """Puts what is no number into rows (token, head) of the queries, and gives the lse that those rows then have."""
    lse = p.exact_lse()
    for n, (t, h) in enumerate(rows):
        if n % 3 == 2:
            p.q[t, h] = NAN
        else:
            p.q[t, h, (5 * n) % p.dim] = (NAN, INF)[n % 3] if n % 2 else -INF
        lse[t, h] = (NAN, INF, -INF)[n % 3]
    return lse


# (one row, the first and the last of a sequence, both with rows behind them that are none)
FEW = [([(6, 50)], [(0, 1), (2, 3), (5, 3)]), ([(1, 300)], [(0, 2)]), ([(3, 40), (2, 9), (5, 33)], [(2, 0), (2, 3), (4, 1), (9, 3)])]


@pytest.mark.parametrize("dtype,kind", TYPES)
@pytest.mark.parametrize("dim", [64, 128, 256, 80, 16, 208])
@pytest.mark.parametrize("sizes,rows", FEW)
def test_few_queries(workspace, dtype, kind, dim, sizes, rows):  # noqa: F811
    p = Packed(sizes, heads=2, group=2, dim=dim, dtype=dtype, kind=kind, seed=dim)
    assert p.tokens * p.group <= 32 * len(sizes)
    check(p, workspace, lse=spoil(p, rows))


@pytest.mark.parametrize("dtype,kind", TYPES)
@pytest.mark.parametrize("dim", [64, 128, 256, 80])
def test_many_queries(workspace, dtype, kind, dim):  # noqa: F811
    p = Packed([(33, 100), (2, 900), (41, 20)], heads=2, group=16, dim=dim, dtype=dtype, kind=kind, seed=dim)
    assert p.tokens * p.group > 32 * 3
    check(p, workspace, lse=spoil(p, [(0, 0), (13, 20), (32, 31), (33, 5), (34, 31), (75, 15), (75, 31)]))


def test_no_query_has_a_number(workspace):  # noqa: F811
    for sizes, group in (([(4, 30)], 2), ([(40, 60)], 4)):
        p = Packed(sizes, heads=2, group=group)
        p.q[:] = NAN
        weights, _ = check(p, workspace, lse=np.full((p.tokens, 2 * group), np.nan), with_before=False)
        assert not weights.any()


@pytest.mark.parametrize("sizes,heads,group", [([(20, 70), (5, 300)], 2, 2), ([(40, 100), (64, 64)], 1, 32)])
def test_what_attention_hands_on(workspace, sizes, heads, group):  # noqa: F811
    """An output and an lse of NaN for the queries alone, and weights from the others."""
    p = Packed(sizes, heads=heads, group=group, room=2048)
    for t, h in ((0, 0), (7, 1), (sizes[0][0] - 1, heads * group - 1), (p.tokens - 1, 1)):
        p.q[t, h, 3] = NAN
    p.q[9, 0] = INF
    out, lse = torch.full_like(p.q, 7.0), torch.full(p.q.shape[:2], 7.0, device="cuda")
    r = dl.ChunkAttention(p.cache(), p.q, out, *p.plan(), lse=lse, scale=p.scale)
    r.use_workspace(workspace)
    dl.dl_chunk_attention(r, torch.cuda.current_stream())
    assert torch.isnan(lse).sum() == 5
    p.check_attention(out, lse)
    weights, _ = check(p, workspace, lse=lse.cpu().numpy())
    assert torch.isfinite(weights).all()
