"""8-bit experts and scored routing, from their definitions, in float64.

e4m3 (OCP): sign, 4 exponent bits (bias 7), 3 mantissa bits; largest number
448, smallest normal 2^-6, spacing 2^-9 below it, no infinities.  A block of
values is held as e4m3(v / s) with s the smallest power of two (at least
2^-127) for which the block's largest finite magnitude is at most 448 s, s = 1
for a block of zeros; what is not finite becomes NaN.
"""
from __future__ import annotations

import numpy as np

from .numerics import silu

BLK = 128
MAX_E4M3 = 448.0


def round_e4m3(x) -> np.ndarray:
    """Nearest e4m3 value of |x| <= 448, ties to even; NaN for what is not finite."""
    x = np.asarray(x, np.float64)
    fin = np.isfinite(x)
    v = np.where(fin, x, 0.0)
    _, e = np.frexp(v)
    step = np.ldexp(1.0, np.maximum(e - 1, -6) - 3)
    return np.where(fin, np.rint(v / step) * step, np.nan)


def block_scale(amax) -> np.ndarray:
    """Scale of blocks whose largest finite magnitudes are amax."""
    amax = np.asarray(amax, np.float64)
    x = np.full(amax.shape, -127)
    for _ in range(400):  # the smallest exponent that fits, step by step
        low = (amax > MAX_E4M3 * np.ldexp(1.0, x))
        if not low.any():
            break
        x = x + low
    return np.where(amax == 0, 1.0, np.ldexp(1.0, x))


def quantize_rows(v: np.ndarray):
    """(q, s): e4m3 values [R][K] and scales [R][K/128]."""
    b = np.asarray(v, np.float64).reshape(v.shape[0], -1, BLK)
    s = block_scale(np.where(np.isfinite(b), np.abs(b), 0.0).max(axis=2))
    return round_e4m3(b / s[:, :, None]).reshape(v.shape), s


def quantize_blocks(w: np.ndarray):
    """(q, s) of a matrix [N][K] by 128 x 128 blocks."""
    N, K = w.shape
    b = np.asarray(w, np.float64).reshape(N // BLK, BLK, K // BLK, BLK)
    s = block_scale(np.where(np.isfinite(b), np.abs(b), 0.0).max(axis=(1, 3)))
    return round_e4m3(b / s[:, None, :, None]).reshape(N, K), s


def dequantize_blocks(q: np.ndarray, s: np.ndarray) -> np.ndarray:
    return np.asarray(q, np.float64) * np.kron(np.asarray(s, np.float64), np.ones((BLK, BLK)))


U = 2.0 ** -24                # half a step of fp32, relative


def product_bound(x: np.ndarray, y: np.ndarray) -> np.ndarray:
    """How far a kernel's x @ y.T may be off for rows x [R][K], y [N][K] of
    e4m3 values times their blocks' scales (both scales constant over 128
    columns): the matrix instruction drops from each of 8 products less than
    2^-13 of the largest one's power of two (7 of them, the largest loses
    nothing); the K/8 sums of 8, and two roundings for a scale of each of the
    K/128 blocks, are fp32."""
    K = x.shape[1]
    ax, ay = np.abs(x), np.abs(y)
    drop = np.zeros((x.shape[0], y.shape[0]))
    for k in range(0, K, 8):
        drop += (ax[:, None, k:k + 8] * ay[None, :, k:k + 8]).max(axis=2)
    return 7 * 2.0 ** -13 * drop + (K / 8 + 2 * K / BLK + 8) * U * (ax @ ay.T)


def hidden8(a: np.ndarray, gu):
    """h [R][F] before it is quantised, in float64, for rows a [R][H] (bf16
    values) of one expert, and how far a kernel's fp32 h may be off: |silu'| <
    1.1, so 1.1 |up| err(gate) + |silu(gate)| err(up) (+ their product), and 8 U
    |h| for the exponential, the reciprocal and three products."""
    F = gu[0].shape[0] // 2
    q, s = quantize_rows(a)
    x, w = q * np.repeat(s, BLK, axis=1), dequantize_blocks(*gu)
    y, e = x @ w.T, product_bound(x, w)
    g, up, eg, eu = y[:, :F], y[:, F:], e[:, :F], e[:, F:]
    h = silu(g) * up
    return h, 1.1 * np.abs(up) * eg + (np.abs(silu(g)) + 1.1 * eg) * eu + 8 * U * np.abs(h)


def quantised_bound(h: np.ndarray, eh: np.ndarray, s: np.ndarray):
    """For a kernel's quantised h with scales s [R][F/128], given h and the bound
    eh on its fp32 values: whether each scale is the one of some |h| within the
    bound, and how far the e4m3 values times s may be off h (half a step of the
    larger magnitude, and eh)."""
    b, e = np.abs(h).reshape(len(h), -1, BLK), eh.reshape(len(h), -1, BLK)
    lo, hi = block_scale(np.maximum(b - e, 0).max(axis=2)), block_scale((b + e).max(axis=2))
    ok = (s >= lo) & (s <= hi) | (lo == 1) & (s <= hi)  # all of it may be 0
    _, x = np.frexp((b + e) / s[:, :, None])
    half = np.ldexp(1.0, np.maximum(x - 1, -6) - 4) * s[:, :, None]
    return ok, eh + half.reshape(h.shape)


def stored_bound(o: np.ndarray, tol: np.ndarray) -> np.ndarray:
    """How far a kernel's stored bf16 output may be from o itself: it computes
    some o' with |o' - o| <= tol and stores bf16(o'), off by at most half a step,
    2^-8 |o'| <= 2^-8 (|o| + tol)."""
    return tol + 2.0 ** -8 * (np.abs(o) + tol)


def select(z, k: int, *, score: str, balance=None, n_group: int = 1, topk_group: int = 1, group_top: int = 2,
           norm_topk: int = 1, scale: float = 1.0):
    """(idx [T][k], w [T][k], counts [E]) token by token: NaN after every
    number, equal values by the lower id."""
    z = np.asarray(z, np.float64)
    T, E = z.shape
    idx, w = np.zeros((T, k), np.int32), np.zeros((T, k))

    def order(v):  # ids, best first
        return sorted(range(len(v)), key=lambda i: (np.isnan(v[i]), -v[i] if not np.isnan(v[i]) else 0, i))

    with np.errstate(all="ignore"):
        for t in range(T):
            if score == "sigmoid":
                s = 1.0 / (1.0 + np.exp(-z[t]))
            elif np.all(z[t] == -np.inf):
                s = np.zeros(E)
            else:
                e = np.exp(z[t] - z[t].max())
                s = e / e.sum()
            c = s + (0.0 if balance is None else np.asarray(balance, np.float64))
            alive = list(range(E))
            if topk_group < n_group:
                M = E // n_group
                by = np.where(np.isnan(c), -np.inf, c).reshape(n_group, M)
                gs = np.sort(by, axis=1)[:, ::-1][:, :group_top].sum(axis=1)
                kept = set(order(np.where(np.isnan(gs), -np.inf, gs))[:topk_group])
                alive = [e for e in alive if e // M in kept]
            idx[t] = [alive[i] for i in order(c[alive])[:k]]
            p = s[idx[t]]
            w[t] = scale * (p / p.sum() if norm_topk and p.sum() != 0 else p)
    return idx, w, np.bincount(idx.reshape(-1), minlength=E).astype(np.int32)
