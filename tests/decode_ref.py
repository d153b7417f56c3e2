"""Plain implementations, in 64 bits and on the CPU, of the operators over a paged cache in 8 bits, and the bounds that their
32-bit kernels keep."""

import numpy as np
import torch

LIMIT = {"fp8": 448.0, "int8": 127.0}
CODE = {"fp8": torch.float8_e4m3fn, "int8": torch.int8}
# half the distance of two neighbours, relative
UNIT = {torch.float32: 2.0 ** -24, torch.bfloat16: 2.0 ** -8, torch.float16: 2.0 ** -11}


def fp8_nearest(y):
    """Values of e4m3 nearest to y (|y| <= 448 or a little more), ties to even: three bits behind the first, steps of 2^-9 and up."""
    e = np.clip(np.floor(np.log2(np.maximum(np.abs(y), 2.0 ** -20))), -6, 8)
    # (log2 may be one off next to a power of two)
    e = np.where(2.0 ** (e + 1) <= np.abs(y), e + 1, np.where((2.0 ** e > np.abs(y)) & (e > -6), e - 1, e))
    step = 2.0 ** (np.clip(e, -6, 8) - 3)
    return np.rint(y / step) * step


def quantised(x, kind):
    """(values of the codes, scales) of rows x (a float64 array whose values are exact in 32 bits), by the formula in 32-bit steps."""
    x = x.astype(np.float32)
    bad = ~np.isfinite(x).all(-1)
    a = np.maximum(np.abs(np.where(np.isfinite(x), x, 0)).max(-1), np.float32(2.0 ** -100))
    limit = np.float32(LIMIT[kind])
    factor = (np.float32(1) / a) * limit
    with np.errstate(invalid="ignore", over="ignore"):
        y = (x * factor[..., None]).astype(np.float64)
    y = fp8_nearest(np.where(np.isfinite(y), y, 0)) if kind == "fp8" else np.rint(np.where(np.isfinite(y), y, 0))
    scale = a * (np.float32(1) / limit)
    return np.where(bad[..., None], 0.0, y), np.where(bad, np.float32(np.nan), scale)


def code_values(codes):
    """A tensor of codes as a float64 array."""
    return codes.float().cpu().numpy().astype(np.float64)


def attention(q, k, v, visible, scale):
    """One query head: q [D], k and v [n, D] (float64), visible [n].  Output, lse, and sum of p |v| (what the weights' rounding acts on),
    and the largest sum of |q k| * scale."""
    D = v.shape[-1]
    if not visible.any():
        return np.zeros(D), -np.inf, np.zeros(D), 0.0
    k, v = k[visible], v[visible]
    s = k @ q * scale
    top = s.max() if np.isfinite(s).all() else np.nan
    p = np.exp(s - top)
    total = p.sum()
    p = p / total
    return p @ v, top + np.log(total), p @ np.abs(v), (np.abs(k) @ np.abs(q)).max() * abs(scale)


def attention_bounds(out, lse, mass, reach, D, dtype):
    """How far the kernel's output and lse may be off.

    A score is a sum of D products in 32 bits (any order: D 2^-24 of the sum of magnitudes), times a scale, plus the logarithm of
    another (|log2 u| < 128, whose own rounding and that of the sum are within 2^-17 each): an absolute error e of the exponent.
    A weight is then off by a factor of e^(2 e) at most (it and the sum it is divided by), plus its rounding to the type of q (a unit, and where
    16-bit floats end 2^-25 of the largest weight, which the unit of a float16 output covers where |v| is of a size), and
    what the 32-bit sums and the joining of pieces lose, for which 2^-16 is ample (up to 64 joins, sums of 32 neighbours at a time).
    """
    e = (D + 8) * 2.0 ** -24 * reach + 2.0 ** -16
    unit = UNIT[dtype]
    weights = unit + np.expm1(2 * e) + 2.0 ** -16
    return unit * np.abs(out) + (1 + unit) * weights * mass + 2.0 ** -24, e + 2.0 ** -16 + 2.0 ** -22 * np.abs(lse)


def verify(target, draft, tokens, uniform, race, length):
    """One sequence: target [n + 1, V], draft [n, V] or None (float64 of values exact in 32 bits), tokens [n], uniform [n], race [V]."""
    f = np.float32
    n = tokens.shape[0]
    V = target.shape[1]
    a = 0
    while a < length:
        x = int(tokens[a])
        if not 0 <= x < V:
            break
        q = f(1) if draft is None else f(draft[a, x])
        with np.errstate(invalid="ignore"):
            if not f(uniform[a]) * q < f(target[a, x]):
                break
        a += 1
    p = target[a].astype(f)
    w = p
    if a < length:
        if draft is not None:
            with np.errstate(invalid="ignore"):
                w = p - draft[a].astype(f)
        elif 0 <= int(tokens[a]) < V:
            w = p.copy()
            w[int(tokens[a])] = 0
    def win(w):
        with np.errstate(all="ignore"):
            score = (w / race.astype(f)).astype(f)
            fit = (w > 0) & (score >= 0)
        return int(np.argmax(np.where(fit, score, -1))) if fit.any() else -1
    x = win(w)
    if x < 0 and a < length:
        x = win(p)
    return list(int(t) for t in tokens[:a]) + [x] + [-1] * (n - a), a
