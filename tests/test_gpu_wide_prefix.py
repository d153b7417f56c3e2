"""Attention over a paged cache where many queries meet a long prefix, 2^20 scores and more (the kernel that turns a tile's codes into elements
once for 128 rows of queries), and batches of more than 1024 sequences (a piece each).  Against a plain implementation in 64 bits, a head
at a time."""

import numpy as np
import pytest
import torch

import paper_2511_06605_amd as dl

import decode_ref
from test_gpu_prefix_attention import TYPES, Problem

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
    w = torch.full((1 << 29,), 0xFF, dtype=torch.uint8, device="cuda")  # (NaN, as numbers)
    w[:65536] = 0
    return w


def attend(q, k, v, see, scale, dtype):
    """q [m, D], k and v [n, D], see [m, n]: outputs, lse and their bounds (decode_ref.attention, for many queries at once)."""
    used = see.any(0)
    k, v, see = k[used], v[used], see[:, used]
    with np.errstate(over="ignore", invalid="ignore"):  # (queries that are not finite, which the caller leaves out)
        s, magnitudes = np.where(see, q @ k.T * scale, -np.inf), np.where(see, np.abs(q) @ np.abs(k).T, 0.0)
    top = s.max(1, initial=-np.inf, keepdims=True)
    none = ~see.any(1)
    top[none] = 0.0
    with np.errstate(invalid="ignore"):
        p = np.exp(s - top)
    total = p.sum(1, keepdims=True)
    p = p / np.where(none[:, None], 1.0, total)
    with np.errstate(divide="ignore"):
        lse = (top + np.log(total))[:, 0]
    out, mass = p @ v, p @ np.abs(v)
    reach = magnitudes.max(1, initial=0.0) * abs(scale)
    bound, bound_lse = decode_ref.attention_bounds(out, lse[:, None], mass, reach[:, None], q.shape[1], dtype)
    return out, lse, bound, bound_lse[:, 0], none


class Large(Problem):
    def check(self, workspace, dead=(), wide=True, nan=(), **more):
        """nan: (b, j, h) of queries that have to come out NaN."""
        rows = len(self.lens) * self.M * self.group
        assert not wide or (rows >= 64 and rows * self.prefix * self.heads >= 1 << 20)
        out, lse = self.run(workspace, **more)
        out, lse = out.double().cpu().numpy(), lse.double().cpu().numpy()
        for where in nan:
            assert np.isnan(out[where]).all() and np.isnan(lse[where]), where
        k, v = (decode_ref.code_values(c) * np.nan_to_num(s.double().cpu().numpy())[..., None] for c, s in ((self.k, self.k_scale), (self.v, self.v_scale)))
        q = np.nan_to_num(self.q.double().cpu().numpy())
        page, M, G = self.page, self.M, self.group
        t = np.arange(self.prefix)
        there = np.array([(None, i) not in dead for i in range(len(self.prefix_table))], dtype=bool)
        prefix_at = np.where(there, self.prefix_table, 0)[t // page] if self.prefix else np.zeros(0, dtype=np.int64)
        prefix_alive = there[t // page] if self.prefix else np.zeros(0, dtype=bool)
        for b, n in enumerate(self.lens):
            i = np.arange(n)
            own_there = np.array([(b, x) not in dead for x in range(-(-n // page))], dtype=bool)
            own_at = np.where(own_there, self.table[b, :len(own_there)], 0)[i // page] if n else np.zeros(0, dtype=np.int64)
            own_alive = own_there[i // page] if n else np.zeros(0, dtype=bool)
            m = M if self.q_lens is None else int(np.clip(self.q_lens[b], 0, M))
            for kh in range(self.heads):
                keys, values = (np.concatenate([x[prefix_at, t % page, kh], x[own_at, i % page, kh]]) for x in (k, v))
                see = np.zeros((M, G, self.prefix + n), dtype=bool)
                for j in range(m):
                    see[j, :, :self.prefix] = prefix_alive
                    see[j, :, self.prefix:] = own_alive & (i <= n - m + j)
                want, whole, bound, bound_lse, none = (
                    x.reshape(M, G, *x.shape[1:]) for x in attend(q[b, :, kh * G:(kh + 1) * G].reshape(M * G, -1), keys, values,
                                                                  see.reshape(M * G, -1), self.scale, self.dtype))
                for j in range(M):
                    for g in range(G):
                        h, where = kh * G + g, (b, j, kh * G + g)
                        if where in nan:
                            continue
                        if none[j, g]:
                            assert not out[b, j, h].any() and lse[b, j, h] == -np.inf, where
                            continue
                        off = np.abs(out[b, j, h] - want[j, g])
                        assert (off <= bound[j, g]).all(), (where, float((off / bound[j, g]).max()))
                        assert abs(lse[b, j, h] - whole[j, g]) <= bound_lse[j, g], (where, lse[b, j, h], whole[j, g])
        return out, lse


@pytest.mark.parametrize("dtype,kind", TYPES)
@pytest.mark.parametrize("dim,heads,group,q_tokens,batch,prefix", [
    (128, 2, 8, 1, 16, 4100), (64, 2, 4, 3, 11, 4001), (80, 1, 5, 4, 13, 4097), (256, 1, 8, 2, 9, 7300), (96, 3, 16, 1, 9, 2500), (208, 1, 20, 1, 13, 4200),
    (16, 4, 3, 5, 17, 1100), (112, 1, 1, 1, 129, 8200)])
def test_many_queries_on_a_long_prefix(workspace, dtype, kind, dim, heads, group, q_tokens, batch, prefix):
    """Whole tiles of rows and a rest; head_dims that fill their tiles and such that do not."""
    lens = [q_tokens + (i * 7) % 30 for i in range(batch)]
    Large(lens, prefix=prefix, q_tokens=q_tokens, heads=heads, group=group, dim=dim, dtype=dtype, kind=kind, seed=dim + batch).check(workspace)


@pytest.mark.parametrize("dtype,kind", TYPES[:2])
@pytest.mark.parametrize("page", [1, 5, 8, 24, 64, 128, 8192])
def test_pages_that_end_anywhere(workspace, dtype, kind, page):
    Large([3] * 33, prefix=8193, q_tokens=2, page=page, heads=1, group=2, dtype=dtype, kind=kind, seed=page).check(workspace)


@pytest.mark.parametrize("prefix", [8192, 8193, 8255, 8256, 16385])
def test_a_last_tile_of_any_length(workspace, prefix):
    Large([0] * 16, prefix=prefix, heads=1, group=8, dim=128, seed=prefix).check(workspace)


@pytest.mark.parametrize("dtype,kind", TYPES[:2])
def test_holes_in_the_table(workspace, dtype, kind):
    """Pages of the prefix that are none of the pool, whole tiles of them among them; the first page of the pool is not read in their place."""
    p = Large([4] * 16, prefix=8200, q_tokens=2, heads=1, group=8, dtype=dtype, kind=kind, seed=1)
    holes = {2, 3, 4, 5, 6, 7, 8, 9, 100, 511, 512} | {int(i) for i in np.flatnonzero(p.prefix_table == 0)}
    for t in (p.k, p.v):
        t.view(torch.uint8)[0] = 0x7F
    for i in holes:
        p.prefix_table[i] = [-1, p.k.shape[0], 2 ** 31 - 1, -2 ** 31][i % 4]
    own = {(b, 0) for b in range(16) if p.table[b, 0] == 0}
    for b, _ in own:
        p.table[b, 0] = -1
    p.check(workspace, dead={(None, i) for i in holes} | own)
    # nothing but holes
    p = Large([0] * 16, prefix=8200, heads=1, group=8, dtype=dtype, kind=kind, seed=2)
    p.prefix_table[:] = -1
    out, lse = p.run(workspace)
    assert not out.any() and bool((lse == -float("inf")).all())


@pytest.mark.parametrize("which", ["k_scale", "v_scale"])
def test_a_row_that_is_nan_reaches_every_reader(workspace, which):
    p = Large([1] * 16, prefix=8200, heads=2, group=8, seed=3)
    getattr(p, which)[int(p.prefix_table[100]), 5, 1] = float("nan")  # in head 1
    p.check(workspace, nan={(b, 0, h) for b in range(16) for h in range(8, 16)})


def test_queries_that_are_not_finite_or_not_there(workspace):
    p = Large([6] * 20, prefix=8200, q_tokens=3, heads=1, group=4, q_lens=[3, 0, 1, 2] * 5, seed=4)
    p.q[4, 1, 2, 3] = float("nan")
    p.q[8, 0, 0, 0] = float("inf")
    p.check(workspace, nan={(4, 1, 2), (8, 0, 0)})


def test_saturated_scores(workspace):
    Large([2] * 16, prefix=8200, heads=1, group=8, q_size=30.0, spread=2.0, seed=5).check(workspace)
    Large([2] * 16, prefix=8200, heads=1, group=8, q_size=30.0, spread=2.0, dtype=torch.float16, kind="int8", seed=6).check(workspace)


@pytest.mark.parametrize("order", [(0, 2, 1), (2, 0, 1), (1, 2, 0)])
def test_any_order_and_stride(workspace, order):
    p = Large([5] * 17, prefix=2500, q_tokens=2, heads=3, group=5, dim=80, order=order, seed=7)
    B, M, H, D = p.q.shape
    wide = torch.full((M, B, H + 1, D + 7), 9.0, dtype=p.dtype, device="cuda")
    q = wide.permute(1, 0, 2, 3)[:, :, 1:, 3:3 + D]
    q.copy_(p.q)
    result = torch.full((B, H, M, D + 3), 9.0, dtype=p.dtype, device="cuda")
    out = result.permute(0, 2, 1, 3)[..., 1:1 + D]
    p.check(workspace, q=q, out=out)
    assert bool((result[..., 0] == 9).all()) and bool((result[..., 1 + D:] == 9).all())


def test_same_bits_again(workspace):
    p = Large([3, 40, 0, 7] * 16, prefix=4100, q_tokens=2, heads=2, group=4, dim=128, seed=8)
    first = [t.clone() for t in p.run(workspace)]
    for _ in range(3):
        again = p.run(workspace)
        assert torch.equal(first[0], again[0]) and torch.equal(first[1], again[1])


def test_pages_far_into_the_pool(workspace):
    """More than 4 GiB behind its start."""
    p = Large([7] * 16, prefix=4100, group=8, dim=128, heads=2, seed=9)
    want = [t.clone() for t in p.run(workspace)]
    pages = (5 << 30) // (16 * 2 * 128)
    shift = pages - p.k.shape[0]
    for name in ("k", "v"):
        big = torch.empty((pages, 16, 2, 128), dtype=torch.uint8, device="cuda").view(getattr(p, name).dtype)
        big.view(torch.uint8)[shift:] = getattr(p, name).view(torch.uint8)
        scale = torch.zeros((pages, 16, 2), device="cuda")
        scale[shift:] = getattr(p, name + "_scale")
        setattr(p, name, big)
        setattr(p, name + "_scale", scale)
    p.prefix_table += shift
    p.table[p.table >= 0] += shift
    got = p.run(workspace)
    assert torch.equal(got[0], want[0]) and torch.equal(got[1], want[1])


@pytest.mark.parametrize("dtype,kind", TYPES[:2])
@pytest.mark.parametrize("batch,prefix,q_tokens", [(1025, 0, 1), (1030, 70, 2), (1100, 2000, 1)])
def test_more_than_1024_sequences(workspace, dtype, kind, batch, prefix, q_tokens):
    """Empty ones, short ones and a long one among them."""
    lens = [(i * 13) % 40 for i in range(batch)]
    lens[3], lens[batch - 1], lens[700] = 1500, 300, 0
    Large(lens, prefix=prefix, q_tokens=q_tokens, heads=1, group=2, dim=32, dtype=dtype, kind=kind, seed=batch).check(workspace, wide=prefix > 1000)


def test_more_than_1024_sequences_with_queries_of_their_own_number(workspace):
    batch = 1027
    Large([(i * 5) % 23 for i in range(batch)], prefix=9, q_tokens=3, heads=2, group=1, dim=16, q_lens=[i % 5 for i in range(batch)],
          seed=10).check(workspace, wide=False)
