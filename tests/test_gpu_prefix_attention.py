"""Attention of a batch that shares a prefix, over a paged cache in 8 bits (dl_prefix_attention), against a plain implementation in 64
bits on the CPU, query by query."""

import numpy as np
import pytest
import torch

import paper_2511_06605_amd as dl

import decode_ref

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


NAN8 = {"fp8": 0x7F, "int8": -128}


class Problem:
    """A cache whose unused places hold NaN (as far as its codes have one) and scales of NaN, and a batch on it."""

    def __init__(self, lens, prefix=0, q_tokens=1, heads=2, group=1, dim=64, page=16, dtype=torch.bfloat16, kind="fp8", seed=0, q_lens=None,
                 spread=1.0, order=(0, 1, 2), q_size=1.0, spare=0):
        rng = np.random.default_rng(seed)
        self.lens, self.prefix, self.M, self.heads, self.group, self.dim, self.page = list(lens), prefix, q_tokens, heads, group, dim, page
        self.dtype, self.kind = dtype, kind
        self.q_lens = None if q_lens is None else list(q_lens)
        B = len(self.lens)
        wide = max(1, max(-(-n // page) for n in self.lens) + spare)
        shared = -(-prefix // page)
        pages = shared + sum(-(-n // page) for n in self.lens) + 2
        table = rng.permutation(pages)
        self.prefix_table = table[:shared].astype(np.int32)
        self.table = np.full((B, wide), -7, dtype=np.int32)  # (no page: it is not to be looked at)
        at = shared
        for b, n in enumerate(self.lens):
            need = -(-n // page)
            self.table[b, :need] = table[at:at + need]
            at += need
        used = np.zeros((pages, page), dtype=bool)
        for t in range(prefix):
            used[self.prefix_table[t // page], t % page] = True
        for b, n in enumerate(self.lens):
            for t in range(n):
                used[self.table[b, t // page], t % page] = True
        self.used = used
        back = [order.index(i) for i in range(3)]
        shape = (pages, page, heads)
        made = []
        for _ in range(2):
            x = rng.standard_normal((*shape, dim)) * np.exp(spread * rng.standard_normal((*shape, 1)))
            y, z = decode_ref.quantised(x, kind)
            codes = torch.from_numpy(y).to(torch.float32).to(decode_ref.CODE[kind])
            codes.view(torch.int8)[torch.from_numpy(~used)] = NAN8[kind]
            z[~used] = np.nan
            put = torch.empty([shape[i] for i in order] + [dim], dtype=torch.int8, device="cuda").permute(*back, 3)
            put.copy_(codes.view(torch.int8))
            scale = torch.empty([shape[i] for i in order], device="cuda").permute(*back)
            scale.copy_(torch.from_numpy(z))
            made += [put.view(decode_ref.CODE[kind]), scale]
        self.k, self.k_scale, self.v, self.v_scale = made
        self.q = torch.from_numpy(q_size * rng.standard_normal((B, q_tokens, heads * group, dim))).to(dtype).cuda()
        self.scale = dim ** -0.5

    def request(self, workspace, q=None, out=None, table=None):
        put = lambda a: torch.from_numpy(np.ascontiguousarray(a)).cuda()  # noqa: E731
        cache = dl.KvCache(self.k, self.v, self.k_scale, self.v_scale)
        q = self.q if q is None else q
        self.out = torch.full_like(self.q, 7.0) if out is None else out
        self.lse = torch.full(self.q.shape[:3], 7.0, device="cuda")
        r = dl.PrefixAttention(cache, q, self.out, put(self.table) if table is None else table, put(np.array(self.lens, dtype=np.int32)),
                               prefix_pages=put(self.prefix_table), prefix_tokens=self.prefix, lse=self.lse, scale=self.scale,
                               q_lens=None if self.q_lens is None else put(np.array(self.q_lens, dtype=np.int32)))
        assert dl.dl_prefix_attention_workspace(r) <= workspace.numel()
        r.use_workspace(workspace)
        return r

    def run(self, workspace, **more):
        dl.dl_prefix_attention(self.request(workspace, **more), torch.cuda.current_stream())
        return self.out, self.lse

    def check(self, workspace, dead=(), **more):
        """dead: (sequence or None for the prefix, page of its table) that is no page of the pool."""
        out, lse = self.run(workspace, **more)
        out, lse = out.double().cpu().numpy(), lse.double().cpu().numpy()
        k, v = (decode_ref.code_values(c) * s.double().cpu().numpy()[..., None] for c, s in ((self.k, self.k_scale), (self.v, self.v_scale)))
        q = self.q.double().cpu().numpy()
        for b, n in enumerate(self.lens):
            m = self.M if self.q_lens is None else int(np.clip(self.q_lens[b], 0, self.M))
            tokens = [(self.prefix_table[t // self.page], t % self.page, (None, t // self.page) not in dead) for t in range(self.prefix)]
            tokens += [(self.table[b, t // self.page], t % self.page, (b, t // self.page) not in dead) for t in range(n)]
            pg, at, alive = (np.array([t[i] for t in tokens], dtype=np.int64) for i in range(3))
            for j in range(self.M):
                see = np.arange(len(tokens)) < self.prefix + max(0, n - m + j + 1) if j < m else np.zeros(len(tokens), dtype=bool)
                see &= alive.astype(bool)
                for h in range(self.heads * self.group):
                    kh, vh = (x[np.clip(pg, 0, x.shape[0] - 1), at, h // self.group] if len(tokens) else np.zeros((0, self.dim)) for x in (k, v))
                    want, whole, mass, reach = decode_ref.attention(q[b, j, h], kh, vh, see, self.scale)
                    bound, bound_lse = decode_ref.attention_bounds(want, whole, mass, reach, self.dim, self.dtype)
                    where = (b, j, h)
                    if not see.any():
                        assert not out[b, j, h].any() and lse[b, j, h] == -np.inf, where
                    elif not np.isfinite(want).all():
                        assert np.isnan(out[b, j, h]).all() and np.isnan(lse[b, j, h]), where
                    else:
                        off = np.abs(out[b, j, h] - want)
                        assert (off <= bound).all(), (where, float((off / bound).max()), int((off / bound).argmax()))
                        assert abs(lse[b, j, h] - whole) <= bound_lse, (where, lse[b, j, h], whole, bound_lse)
        return out, lse


TYPES = [(torch.bfloat16, "fp8"), (torch.float16, "int8"), (torch.bfloat16, "int8"), (torch.float16, "fp8")]


@pytest.mark.parametrize("dtype,kind", TYPES)
@pytest.mark.parametrize("dim,heads,group", [(64, 2, 1), (128, 1, 7), (256, 1, 3), (80, 2, 4), (16, 3, 2), (96, 1, 20), (208, 1, 8)])
def test_types_and_heads(workspace, dtype, kind, dim, heads, group):
    Problem([5, 40, 129], prefix=70, q_tokens=2, heads=heads, group=group, dim=dim, dtype=dtype, kind=kind, seed=dim + group).check(workspace)


@pytest.mark.parametrize("dtype,kind", TYPES[:2])
@pytest.mark.parametrize("page", [1, 5, 8, 16, 24, 64, 128])
def test_pages_that_end_anywhere(workspace, dtype, kind, page):
    Problem([1, 31, 32, 33, 200], prefix=2 * page + 3, page=page, group=4, dtype=dtype, kind=kind, seed=page).check(workspace)


@pytest.mark.parametrize("lens,prefix,q_tokens", [
    ([1], 0, 1), ([0], 1, 1), ([0], 0, 1), ([0, 3, 0], 0, 2), ([2, 1, 0], 5, 3), ([127, 128, 129], 0, 1), ([255, 257, 383], 128, 4),
    ([1000], 0, 1), ([1], 1025, 1), ([3, 700], 513, 8), ([9] * 20, 40, 5), ([1, 2, 3, 4, 5, 600], 0, 6)])
def test_lengths(workspace, lens, prefix, q_tokens):
    for dtype, kind in TYPES[:2]:
        Problem(lens, prefix=prefix, q_tokens=q_tokens, heads=1, group=3, dtype=dtype, kind=kind, seed=prefix + len(lens)).check(workspace)


def test_long_axes_are_split(workspace):
    """A piece for every 128 tokens and more of them than lanes; one long sequence among short ones."""
    Problem([9000], heads=1, group=2, seed=1).check(workspace)
    Problem([20000, 3, 150], prefix=9001, heads=1, group=1, dim=16, seed=2, kind="int8", dtype=torch.float16).check(workspace)


@pytest.mark.parametrize("dtype,kind", TYPES)
@pytest.mark.parametrize("dim,heads,group,q_tokens,batch,prefix", [
    (128, 1, 8, 1, 40, 600), (64, 2, 4, 3, 23, 515), (128, 2, 5, 4, 17, 130), (256, 1, 8, 2, 20, 300), (96, 1, 16, 5, 9, 257), (128, 1, 1, 1, 200, 1000)])
def test_many_queries_on_a_prefix(workspace, dtype, kind, dim, heads, group, q_tokens, batch, prefix):
    """Enough queries for the matrix units: whole tiles of them and a rest."""
    lens = [q_tokens + (i * 7) % 30 for i in range(batch)]
    Problem(lens, prefix=prefix, q_tokens=q_tokens, heads=heads, group=group, dim=dim, dtype=dtype, kind=kind, seed=batch).check(workspace)


def test_queries_that_are_not_there(workspace):
    Problem([10, 10, 10, 2, 7], prefix=20, q_tokens=4, group=2, q_lens=[4, 0, 1, 3, 2], seed=3).check(workspace)
    Problem([10, 0, 1], prefix=0, q_tokens=4, group=2, q_lens=[2, 2, 9], seed=4).check(workspace)  # (9 counts as 4)
    Problem([10, 5] * 30, prefix=300, q_tokens=3, group=4, q_lens=[3, 0, 1, 2] * 15, seed=5).check(workspace)


def test_lengths_beyond_the_table_and_below_zero(workspace):
    p = Problem([32, 16, 5], prefix=17, q_tokens=2, seed=6)
    want = p.check(workspace)
    for lens in ([1000, 16, 5], [32, 16, 5]):
        p.lens = lens
        out, lse = p.run(workspace)
        assert np.array_equal(out.double().cpu().numpy(), want[0]) and np.array_equal(lse.double().cpu().numpy(), want[1])
    p.lens = [32, -5, 5]
    out = p.run(workspace)[0].clone()
    p.lens = [32, 0, 5]
    p.check(workspace)
    assert torch.equal(out, p.out)


def test_holes_in_the_tables(workspace):
    """Pages that are none of the pool: their tokens are not attended to, whatever the first page of the pool holds."""
    p = Problem([70, 20, 33], prefix=150, q_tokens=2, group=3, seed=7)
    free = int(np.flatnonzero(~p.used.any(1))[0])
    first = [int(x) for x in (p.prefix_table[2], p.table[0, 1], p.table[1, 0], p.table[1, 1])]
    assert free not in first
    p.prefix_table[2], p.table[0, 1], p.table[1, 0], p.table[1, 1] = -1, 2 ** 31 - 1, p.k.shape[0], -2 ** 31
    p.check(workspace, dead={(None, 2), (0, 1), (1, 0), (1, 1)})
    # nothing but holes
    p = Problem([20], prefix=0, seed=8)
    p.table[:] = -1
    p.check(workspace, dead={(0, 0), (0, 1)})
    # the first page of the pool is garbage
    p = Problem([64, 64], prefix=64, q_tokens=2, seed=9)
    for t in (p.k, p.v):
        t.view(torch.uint8)[0] = 0x7F
    hit = [(None, i) for i in range(4) if p.prefix_table[i] == 0] + [(b, i) for b in range(2) for i in range(4) if p.table[b, i] == 0]
    p.prefix_table[p.prefix_table == 0] = -1
    p.table[p.table == 0] = -1
    extra = (0, 2)
    p.table[extra] = -3
    p.check(workspace, dead=set(hit) | {extra})


@pytest.mark.parametrize("kind", ["fp8", "int8"])
def test_rows_that_are_nan_reach_their_readers_alone(workspace, kind):
    """A draft whose key or value was not finite: the queries before it do not see it."""
    p = Problem([40, 40, 40], prefix=33, q_tokens=4, group=2, kind=kind, seed=10)
    for b, t, which in ((0, 38, p.v_scale), (1, 37, p.k_scale)):  # visible from query 2 / query 1 on
        which[int(p.table[b, t // 16]), t % 16] = float("nan")
    p.check(workspace)


def test_scales_of_any_size(workspace):
    """Values of very different sizes, down to the smallest scale there is, and saturated scores."""
    for dtype in (torch.bfloat16, torch.float16):
        Problem([200, 3], prefix=100, q_tokens=2, spread=3.0, dtype=dtype, seed=11).check(workspace)
        Problem([200, 3], prefix=100, q_tokens=2, q_size=30.0, dtype=dtype, kind="int8", seed=12).check(workspace)
    p = Problem([100], prefix=50, dtype=torch.bfloat16, seed=13)
    p.v_scale.mul_(2.0 ** -90)
    p.check(workspace)
    p.v_scale.mul_(2.0 ** 90).mul_(2.0 ** 90)
    p.check(workspace)
    p = Problem([64], prefix=40, dtype=torch.float16, seed=14)
    p.v.view(torch.uint8)[int(p.table[0, 1])] = 0
    p.v_scale[int(p.table[0, 1])] = 2.0 ** -100 / 448
    p.check(workspace)


def test_queries_that_are_not_finite(workspace):
    p = Problem([50, 50], prefix=20, q_tokens=2, group=2, seed=15)
    p.q[0, 1, 2, 3] = float("nan")
    p.check(workspace)


@pytest.mark.parametrize("order", [(0, 2, 1), (2, 0, 1), (1, 2, 0)])
def test_any_order_and_stride(workspace, order):
    p = Problem([50, 9], prefix=40, q_tokens=2, heads=3, group=2, dim=80, order=order, seed=16)
    B, M, H, D = p.q.shape
    wide = torch.full((M, B, H + 1, D + 7), 9.0, dtype=p.dtype, device="cuda")
    q = wide.permute(1, 0, 2, 3)[:, :, 1:, 3:3 + D]
    q.copy_(p.q)
    result = torch.full((B, H, M, D + 3), 9.0, dtype=p.dtype, device="cuda")
    out = result.permute(0, 2, 1, 3)[..., 1:1 + D]
    table = torch.full((2, 11), -9, dtype=torch.int32, device="cuda")[:, 3:3 + p.table.shape[1]]
    table.copy_(torch.from_numpy(p.table))
    p.check(workspace, q=q, out=out, table=table)
    assert bool((result[..., 0] == 9).all()) and bool((result[..., 1 + D:] == 9).all())


def test_tables_wider_than_the_lengths(workspace):
    for spare in (0, 7, 900):
        Problem([65, 2], prefix=20, q_tokens=2, spare=spare, seed=17).check(workspace)


def test_same_bits_again_and_no_lse(workspace):
    p = Problem([300, 4, 77, 250] * 8, prefix=700, q_tokens=2, group=4, dim=128, seed=18)
    first = [t.clone() for t in p.run(workspace)]
    for _ in range(3):
        again = p.run(workspace)
        assert torch.equal(first[0], again[0]) and torch.equal(first[1], again[1])
    r = p.request(workspace)
    r.desc.lse = None
    dl.dl_prefix_attention(r, torch.cuda.current_stream())
    assert torch.equal(first[0], p.out) and bool((p.lse == 7).all())


def test_cache_beyond_32_bits(workspace):
    """Pages more than 4 GiB behind the start of the pool."""
    p = Problem([40, 7], prefix=33, q_tokens=1, group=2, dim=128, heads=2, seed=19)
    pages = (5 << 30) // (16 * 2 * 128)
    far = {}
    for name in ("k", "v"):
        big = torch.empty((pages, 16, 2, 128), dtype=torch.uint8, device="cuda").view(getattr(p, name).dtype)
        big.view(torch.uint8)[pages - p.k.shape[0]:] = getattr(p, name).view(torch.uint8)
        scale = torch.zeros((pages, 16, 2), device="cuda")
        scale[pages - p.k.shape[0]:] = getattr(p, name + "_scale")
        far[name], far[name + "_scale"] = big, scale
    shift = pages - p.k.shape[0]
    want = [t.clone() for t in p.run(workspace)]
    p.k, p.v, p.k_scale, p.v_scale = far["k"], far["v"], far["k_scale"], far["v_scale"]
    p.prefix_table += shift
    p.table[p.table >= 0] += shift
    got = p.run(workspace)
    assert torch.equal(got[0], want[0]) and torch.equal(got[1], want[1])


def test_on_another_stream_and_in_a_graph(workspace):
    """A captured step replayed as the sequences grow."""
    side = torch.cuda.Stream()
    p = Problem([100, 60, 30], prefix=300, q_tokens=2, group=4, seed=20)
    r = p.request(torch.zeros(1 << 24, dtype=torch.uint8, device="cuda"))
    lens = r._tensors[3]
    side.wait_stream(torch.cuda.current_stream())
    with torch.cuda.stream(side):
        dl.dl_prefix_attention(r, side)
        side.synchronize()
        graph = torch.cuda.CUDAGraph()
        with torch.cuda.graph(graph, stream=side):
            dl.dl_prefix_attention(r, side)
    out, lse = p.out, p.lse
    for step in range(4):
        now = [100 - 7 * step, 60 - 13 * step, 30 - 9 * step]
        lens.copy_(torch.tensor(now, dtype=torch.int32))
        p.q.normal_()
        torch.cuda.synchronize()
        graph.replay()
        torch.cuda.synchronize()
        p.lens = now
        want = p.check(workspace)
        assert np.array_equal(out.double().cpu().numpy(), want[0]) and np.array_equal(lse.double().cpu().numpy(), want[1])


def test_nothing_to_do(workspace):
    p = Problem([4], seed=21)
    for shape in ((0, 1, 2, 64), (1, 0, 2, 64), (1, 1, 0, 64)):
        q = torch.empty(shape, dtype=torch.bfloat16, device="cuda")
        table, lens = torch.zeros((shape[0], 1), dtype=torch.int32, device="cuda"), torch.zeros((shape[0],), dtype=torch.int32, device="cuda")
        r = dl.PrefixAttention(dl.KvCache(p.k, p.v, p.k_scale, p.v_scale), q, torch.empty_like(q), table, lens)
        r.use_workspace(workspace)
        dl.dl_prefix_attention(r, torch.cuda.current_stream())
    # a table without pages, and a pool without pages
    out = torch.full((1, 1, 2, 64), 7.0, dtype=torch.bfloat16, device="cuda")
    lens = torch.full((1,), 5, dtype=torch.int32, device="cuda")
    for k in (p.k, p.k[:0]):
        v, ks, vs = (t[:k.shape[0]] for t in (p.v, p.k_scale, p.v_scale))
        width = 0 if k.shape[0] else 1
        r = dl.PrefixAttention(dl.KvCache(k, v, ks, vs), p.q, out, torch.zeros((1, width), dtype=torch.int32, device="cuda"), lens)
        r.use_workspace(workspace)
        dl.dl_prefix_attention(r, torch.cuda.current_stream())
        assert not out.any()
        out.fill_(7.0)
