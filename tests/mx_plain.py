"""The 4-bit format and the operators over it in 64 bits, written from their definitions (cca.h): the oracle of the mx tests."""
import numpy as np

GRID = np.array([0.0, 0.5, 1.0, 1.5, 2.0, 3.0, 4.0, 6.0])


def values(codes, scales):
    """codes (..., w/2), scales (..., w/32), uint8 -> (..., w)"""
    codes, scales = np.asarray(codes), np.asarray(scales)
    c = np.stack([codes & 15, codes >> 4], -1).reshape(*codes.shape[:-1], 2 * codes.shape[-1])
    mag = GRID[c & 7] * np.where(c > 7, -1.0, 1.0)
    s = np.where(scales == 255, np.nan, np.exp2(scales.astype(np.float64) - 127))
    return mag * np.repeat(s, 32, -1)


def store(x):
    """x (..., w) -> codes, scales"""
    g = np.asarray(x, np.float64).reshape(*x.shape[:-1], -1, 32)
    finite = np.isfinite(g).all(-1)
    g = np.where(finite[..., None], g, 0.0)
    amax = np.abs(g).max(-1)
    f, e = np.frexp(amax)  # amax = f 2^e, 0.5 <= f < 1
    e = np.where(amax > 0, e - 1 - 2 + (f > 0.875), -1000)
    scales = np.clip(e + 127, 2, 252)
    y = g / np.exp2(scales.astype(np.float64) - 127)[..., None]
    # nearest of the eight, a tie to the even code
    d = np.abs(np.abs(y)[..., None] - GRID)
    best = d.min(-1, keepdims=True)
    near = d == best
    even = near & (np.arange(8) % 2 == 0)
    code = np.where(even.any(-1), even.argmax(-1), near.argmax(-1)) + 8 * np.signbit(y)
    code = np.where(finite[..., None], code, 0).reshape(x.shape)
    return (code[..., 0::2] + 16 * code[..., 1::2]).astype(np.uint8), np.where(finite, scales, 255).astype(np.uint8)


def attend(q, k, v, scale):
    """q (R, d), k, v (n, d) -> o (R, d), lse (R), p (R, n)"""
    if not len(k):
        return np.zeros_like(q), np.full(len(q), -np.inf), np.zeros((len(q), 0))
    s = q @ k.T * scale
    top = s.max(-1, keepdims=True)
    e = np.exp(s - top)
    total = e.sum(-1, keepdims=True)
    p = e / total
    return p @ v, (top + np.log(total))[:, 0], p


def evict(weight, pos, n, budget, recent):
    """weight, pos of one head's rows -> the row that each of rows 0 ... min(n, budget) - 1 holds afterwards"""
    if n <= budget:
        return list(range(n))
    newest = int(max(pos[:n]))
    w = [-np.inf if np.isnan(x) else x for x in weight[:n]]
    rank = sorted(range(n), key=lambda i: (0, 0, i) if int(pos[i]) > newest - recent else (1, -w[i], np.isnan(weight[i]), i))
    kept = set(rank[:budget])
    late = iter(sorted(i for i in kept if i >= budget))
    return [i if i in kept else next(late) for i in range(budget)]
