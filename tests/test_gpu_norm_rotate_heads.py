"""dl_norm_rotate with as many heads as either side may have."""

import numpy as np
import pytest
import torch

import paper_2511_06605_amd as dl

import prompt_ref

pytestmark = pytest.mark.gpu


@pytest.fixture(scope="module", autouse=True)
def library():
    torch.cuda.set_device(0)
    dl.dl_init(0)
    yield
    dl.dl_shutdown()


@pytest.mark.parametrize("q_heads,k_heads", [(65535, 1), (65535, 2), (2, 65535), (65535, 65535)])
@pytest.mark.parametrize("tokens", [1, 9])
def test_heads(q_heads, k_heads, tokens):
    rng = np.random.default_rng(q_heads + k_heads)
    q, k = (torch.from_numpy(rng.standard_normal((tokens, h, 16)).astype(np.float32)).bfloat16().cuda() for h in (q_heads, k_heads))
    angle = rng.uniform(-4.0, 4.0, (20, 8))
    table = torch.from_numpy(np.concatenate([np.cos(angle), np.sin(angle)], 1)).float().cuda()
    positions = rng.integers(0, 20, tokens)
    outs = torch.full_like(q, 7.0), torch.full_like(k, 7.0)
    dl.dl_norm_rotate(dl.NormRotate(q, k, *outs, q_weight=torch.ones(16, device="cuda"), eps=1e-5, table=table, positions=torch.from_numpy(positions).cuda()),
                      torch.cuda.current_stream())
    for x, y, w in zip((q, k), outs, (np.ones(16), None)):
        want, bound, _ = prompt_ref.norm_rotate(x.double().cpu().numpy(), w, 1e-5, table.double().cpu().numpy(), positions, False, torch.bfloat16)
        off = np.abs(y.double().cpu().numpy() - want)
        assert (off <= bound).all(), float((off / bound).max())
