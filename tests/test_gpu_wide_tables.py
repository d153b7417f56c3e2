"""Tables with room for more tokens than 32 bits count in steps of 128: 600 sequences of up to 2^30 tokens.  Cut by lengths such a batch
could have had more pieces than its workspace has room for; it is cut by sequences."""

import numpy as np
import pytest
import torch

import paper_2511_06605_amd as dl

import decode_ref
import test_decode_host as host

PAGE, WIDTH, BATCH = 65536, 1 << 14, 600


def workspace_of(parts, batch, dim):
    up = lambda n: -(-n // 16) * 16  # noqa: E731
    return 65536 + up(8 * batch) + up(8 * parts) + 4 * dim * parts


@pytest.mark.parametrize("batch,width", [(BATCH, WIDTH), (256, WIDTH), (1024, WIDTH // 4)])
def test_a_piece_a_sequence(batch, width):
    """2^31 steps of 128 and more."""
    assert batch * width * PAGE // 128 >= 1 << 31
    r = host.attention(host.cache(page=PAGE, heads=1), batch=batch, q_tokens=1, q_heads=1, width=width)
    assert dl.dl_prefix_attention_workspace(r) == workspace_of(batch, batch, 64)


def test_the_largest_tables_that_are_cut_by_lengths():
    r = host.attention(host.cache(page=PAGE, heads=1), batch=255, q_tokens=1, q_heads=1, width=WIDTH)
    assert dl.dl_prefix_attention_workspace(r) > workspace_of(255, 255, 64)


@pytest.mark.gpu
@pytest.mark.parametrize("batch", [255, BATCH])
def test_results(batch):
    torch.cuda.set_device(0)
    dl.dl_init(0)
    try:
        rng = np.random.default_rng(batch)
        dim, pages = 16, 3
        lens = rng.integers(0, 400, batch)
        lens[5] = PAGE + 7
        made, exact = [], []
        for _ in range(2):
            y, z = decode_ref.quantised(rng.standard_normal((pages, PAGE, 1, dim)), "int8")
            exact.append((y * z.astype(np.float64)[..., None])[:, :, 0])
            made += [torch.from_numpy(y).to(torch.int8).cuda(), torch.from_numpy(z).cuda()]
        table = torch.full((batch, WIDTH), -1, dtype=torch.int32, device="cuda")
        first = rng.integers(0, pages, batch)  # (sequences may share pages)
        table[:, 0] = torch.from_numpy(first.astype(np.int32)).cuda()
        table[5, 1] = int(first[5] + 1) % pages
        q = torch.from_numpy(rng.standard_normal((batch, 1, 1, dim))).bfloat16().cuda()
        out, lse = torch.full_like(q, 7.0), torch.full((batch, 1, 1), 7.0, device="cuda")
        r = dl.PrefixAttention(dl.KvCache(made[0], made[2], made[1], made[3]), q, out, table,
                               torch.from_numpy(lens.astype(np.int32)).cuda(), lse=lse)
        r.use_workspace(torch.zeros(dl.dl_prefix_attention_workspace(r), dtype=torch.uint8, device="cuda"))
        dl.dl_prefix_attention(r, torch.cuda.current_stream())
        out, lse, q = out.double().cpu().numpy(), lse.double().cpu().numpy(), q.double().cpu().numpy()
        for b, n in enumerate(lens):
            k, v = (np.concatenate([x[first[b]], x[(first[b] + 1) % pages]])[:n] for x in exact)
            want, whole, mass, reach = decode_ref.attention(q[b, 0, 0], k, v, np.ones(n, dtype=bool), dim ** -0.5)
            if n == 0:
                assert not out[b].any() and lse[b, 0, 0] == -np.inf
                continue
            bound, bound_lse = decode_ref.attention_bounds(want, whole, mass, reach, dim, torch.bfloat16)
            assert (np.abs(out[b, 0, 0] - want) <= bound).all() and abs(lse[b, 0, 0] - whole) <= bound_lse, b
    finally:
        dl.dl_shutdown()
