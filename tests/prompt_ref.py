"""Plain implementations, in 64 bits and on the CPU, of the operators that take a prompt into a bounded paged cache, a batch of packed
sequences to call them with, and the bounds that their 32-bit kernels keep."""

import numpy as np
import torch

import paper_2511_06605_amd as dl

import decode_ref
from decode_ref import UNIT

# what a type cannot tell from zero: half its smallest number
TINY = {torch.float32: 2.0 ** -150, torch.bfloat16: 2.0 ** -134, torch.float16: 2.0 ** -25}


def norm_rotate(x, weight, eps, table, positions, neighbours, dtype):
    """x [T, H, D] float64.  Result, bound, and whether a token is written."""
    T, _, D = x.shape
    y = x.copy()
    if weight is not None:
        y = x / np.sqrt((x * x).mean(-1, keepdims=True) + eps) * weight
    size, written = np.abs(y), np.ones(T, dtype=bool)
    if table is not None:
        R = table.shape[1]
        for t, p in enumerate(positions):
            if not 0 <= p < table.shape[0]:
                written[t] = False
                continue
            for i in range(R // 2):
                a, b = (2 * i, 2 * i + 1) if neighbours else (i, i + R // 2)
                c, s = table[p, i], table[p, R // 2 + i]
                u, v = y[t, :, a].copy(), y[t, :, b].copy()
                y[t, :, a], y[t, :, b] = u * c - v * s, v * c + u * s
                size[t, :, a], size[t, :, b] = abs(u * c) + abs(v * s), abs(v * c) + abs(u * s)
    # The sum of squares: 8 terms a lane and 5 sums among lanes, 13 roundings, and one of the mean: 7 halves after the root; that of 1 / D and
    # the root's own, 1 and 2; two products, one of the rotation and its sum: 4.  24 units of 32 bits are ample.
    return y, 24 * 2.0 ** -24 * size + UNIT[dtype] * (1 + 2.0 ** -18) * np.abs(y) + TINY[dtype], written


NAN8 = {"fp8": 0x7F, "int8": -128}


class Packed:
    """A cache whose unused places hold NaN (as far as its codes have one) and scales of NaN, and packed sequences (new, all tokens) on it."""

    def __init__(self, sizes, heads=2, group=1, dim=64, page=16, dtype=torch.bfloat16, kind="fp8", seed=0, spread=1.0, q_size=1.0, spare=0, gaps=0,
                 order=(0, 1, 2), more_pages=0, room=0):
        rng = self.rng = np.random.default_rng(seed)
        self.sizes, self.heads, self.group, self.dim, self.page, self.dtype, self.kind = list(sizes), heads, group, dim, page, dtype, kind
        B = len(self.sizes)
        wide = max(1, max([-(-n // page) for _, n in self.sizes], default=1) + spare, -(-room // page))  # (room: tokens that a row of the table has room for)
        need = [-(-n // page) for _, n in self.sizes]
        pages = sum(need) + 2 + more_pages
        ids = rng.permutation(pages)
        self.free = ids[sum(need):].astype(np.int32)
        self.table = np.full((B, wide), -7, dtype=np.int32)  # (no page: it is not to be looked at)
        used = np.zeros((pages, page), dtype=bool)
        at = 0
        for b, (_, n) in enumerate(self.sizes):
            self.table[b, :need[b]] = ids[at:at + need[b]]
            at += need[b]
            for t in range(n):
                used[self.table[b, t // page], t % page] = True
        self.used = used
        back = [order.index(x) for x in range(3)]
        shape = (pages, page, heads)
        made = []
        for _ in range(2):
            x = rng.standard_normal((*shape, dim)) * np.exp(spread * rng.standard_normal((*shape, 1)))
            y, z = decode_ref.quantised(x, kind)
            codes = torch.from_numpy(y).to(torch.float32).to(decode_ref.CODE[kind])
            codes.view(torch.int8)[torch.from_numpy(~used)] = NAN8[kind]
            z[~used] = np.nan
            put = torch.empty([shape[x] for x in order] + [dim], dtype=torch.int8, device="cuda").permute(*back, 3)
            put.copy_(codes.view(torch.int8))
            scale = torch.empty([shape[x] for x in order], device="cuda").permute(*back)
            scale.copy_(torch.from_numpy(z))
            made += [put.view(decode_ref.CODE[kind]), scale]
        self.k, self.k_scale, self.v, self.v_scale = made
        # (rows of q in front of the first sequence and behind the last belong to none)
        self.starts = np.cumsum([gaps] + [m for m, _ in self.sizes]).astype(np.int32)
        self.tokens = int(self.starts[-1]) + gaps
        self.q = torch.from_numpy(q_size * rng.standard_normal((self.tokens, heads * group, dim))).to(dtype).cuda()
        self.scale = dim ** -0.5

    @staticmethod
    def put(a):
        return torch.from_numpy(np.ascontiguousarray(a)).cuda()

    def cache(self):
        return dl.KvCache(self.k, self.v, self.k_scale, self.v_scale)

    def plan(self):
        """q_starts, pages and lens as the descriptors take them."""
        return self.put(self.starts), self.put(self.table), self.put(np.array([n for _, n in self.sizes], dtype=np.int32))

    def held(self):
        """Keys and values [pages, page, heads, dim] in 64 bits."""
        return tuple(decode_ref.code_values(c) * s.double().cpu().numpy()[..., None] for c, s in ((self.k, self.k_scale), (self.v, self.v_scale)))

    def tokens_of(self, b, dead=()):
        """Pages, places and whether they are any, of the tokens of a sequence."""
        t = np.arange(self.sizes[b][1])
        alive = np.array([(b, int(x) // self.page) not in dead for x in t], dtype=bool)
        return np.where(alive, self.table[b, t // self.page], 0), t % self.page, alive

    def check_attention(self, out, lse, dead=()):
        out, lse = out.double().cpu().numpy(), lse.double().cpu().numpy()
        k, v = self.held()
        q = self.q.double().cpu().numpy()
        rows = np.zeros(self.tokens, dtype=bool)
        for b, (m, n) in enumerate(self.sizes):
            pg, at, alive = self.tokens_of(b, dead)
            for j in range(m):
                t = int(self.starts[b]) + j
                rows[t] = True
                see = alive & (np.arange(n) <= n - m + j)
                for h in range(self.heads * self.group):
                    kh, vh = (x[pg, at, h // self.group] for x in (k, v))
                    want, whole, mass, reach = decode_ref.attention(q[t, h], kh, vh, see, self.scale)
                    bound, bound_lse = decode_ref.attention_bounds(want, whole, mass, reach, self.dim, self.dtype)
                    where = (b, j, h)
                    if not see.any():
                        assert not out[t, h].any() and lse[t, h] == -np.inf, where
                    elif not np.isfinite(want).all():
                        assert np.isnan(out[t, h]).all() and np.isnan(lse[t, h]), where
                    else:
                        off = np.abs(out[t, h] - want)
                        assert (off <= bound).all(), (where, float((off / bound).max()), int((off / bound).argmax()))
                        assert abs(lse[t, h] - whole) <= bound_lse, (where, lse[t, h], whole, bound_lse)
        return rows

    def exact_lse(self, dead=()):
        """[tokens, q_heads] float64."""
        k, v = self.held()
        q = self.q.double().cpu().numpy()
        lse = np.full((self.tokens, self.heads * self.group), 3.0)
        for b, (m, n) in enumerate(self.sizes):
            pg, at, alive = self.tokens_of(b, dead)
            for j in range(m):
                for h in range(self.heads * self.group):
                    see = alive & (np.arange(n) <= n - m + j)
                    lse[self.starts[b] + j, h] = decode_ref.attention(q[self.starts[b] + j, h], k[pg, at, h // self.group], v[pg, at, h // self.group], see, self.scale)[1]
        return lse

    def weighed(self, lse, before, dead=()):
        """(weights, bounds) [batch, width] from lse (as the kernel gets it) and before (float64 or None)."""
        k, _ = self.held()
        q = self.q.double().cpu().numpy()
        B, width = self.table.shape[0], self.table.shape[1] * self.page
        start = np.zeros((B, width)) if before is None else before
        given, off = np.zeros((B, width)), np.zeros((B, width))
        for b, (m, n) in enumerate(self.sizes):
            pg, at, alive = self.tokens_of(b, dead)
            for j in range(m):
                t = int(self.starts[b]) + j
                see = alive & (np.arange(n) <= n - m + j)
                for h in range(self.heads * self.group):
                    kh = k[pg, at, h // self.group]
                    nan = see & np.isnan(kh).any(-1)
                    given[b, :n][nan] = np.nan
                    if not np.isfinite(lse[t, h]):
                        continue
                    s = np.where(see, kh @ q[t, h] * self.scale, -np.inf)
                    with np.errstate(invalid="ignore"):
                        w = np.where(see, np.exp(s - lse[t, h]), 0.0)
                        # A score is a sum of dim products and a factor or two, in any order; it and the lse are brought to powers of two and
                        # subtracted, each rounded once or twice: an absolute error e of the exponent.  The power itself: 2^-22.
                        e = (self.dim + 8) * 2.0 ** -24 * (np.abs(kh) @ np.abs(q[t, h])) * abs(self.scale) + 2.0 ** -22 * (1 + abs(lse[t, h]))
                        off[b, :n] += np.where(see, w * (np.expm1(e) + 2.0 ** -22) + 2.0 ** -126, 0.0)
                    given[b, :n] += w
        # sums of at most rows / 16 + 32 partial sums in a line
        lines = max([m * self.group for m, _ in self.sizes], default=0) * self.heads / 16 + 32
        want = start + given
        return want, off + given * lines * 2.0 ** -24 + 2.0 ** -23 * np.abs(want)


def evicted(weights, n, keep, first, recent):
    """The tokens that stay, in order."""
    if n <= keep:
        return list(range(n))
    w = [(-np.inf if np.isnan(x) else float(x), not np.isnan(x)) for x in weights[:n]]
    others = sorted(range(first, n - recent), key=lambda i: (not w[i][1], -w[i][0], i))
    return sorted(list(range(first)) + others[:keep - first - recent] + list(range(n - recent, n)))
