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


def expert_ffn8(a: np.ndarray, gu, dn):
    """o [R][H] before its bf16 rounding, and how far a kernel's fp32 sums may
    move it, for rows a [R][H] (bf16 values) of one expert; gu, dn: (q, s).

    The bound counts u = 2^-24 per rounding:
      y: K products, their sum, and two roundings a block for the scales:
         (K + 2 K/128) u sum |a w|;
      h: |silu'| < 1.1, so 1.1 |up| err(gate) + |silu(gate)| err(up), and 8 u |h|
         for the exponential, the reciprocal and three products;
      an h within that error of the middle between two e4m3 values may go to
      the other one, a step away, and a block whose largest |h| is within it of
      448 times a power of two may take the other scale, with steps twice as
      large, where every h of the block may be 1.5 steps off: the sum over such
      h of that times |w|;
      o: the same as y over F.
    """
    u = 2.0 ** -24
    F, H = gu[0].shape[0] // 2, gu[0].shape[1]
    aq, sa = quantize_rows(a)
    ad = aq * np.repeat(sa, BLK, axis=1)
    w, d = dequantize_blocks(*gu), dequantize_blocks(*dn)
    y, ay = ad @ w.T, (H + 2 * H / BLK) * u * (np.abs(ad) @ np.abs(w).T)
    g, up = y[:, :F], y[:, F:]
    h = silu(g) * up
    eh = 1.1 * np.abs(up) * ay[:, :F] + np.abs(silu(g)) * ay[:, F:] + 8 * u * np.abs(h)
    b, eb = h.reshape(len(h), -1, BLK), eh.reshape(len(h), -1, BLK)
    amax = np.abs(b).max(axis=2)
    s = block_scale(amax)
    q = round_e4m3(b / s[:, :, None])
    # the two scales a block can have, and whether its other one can come about
    worst = eb.max(axis=2)
    other = (block_scale(amax + worst) != s) | (block_scale(np.maximum(amax - worst, 0)) != s)
    _, e = np.frexp(b / s[:, :, None])
    step = np.ldexp(1.0, np.maximum(e - 1, -6) - 3) * s[:, :, None]
    near = np.abs(np.abs(b - q * s[:, :, None]) - step / 2) <= eb
    # the neighbour across the middle is one step away; under the other scale a
    # value is rounded by at most half of twice the step instead of half a step
    slack = np.where(other[:, :, None], 1.5 * step, np.where(near, step, 0.0)).reshape(h.shape)
    hd = (q * s[:, :, None]).reshape(h.shape)
    o = hd @ d.T
    tol = (F + 2 * F / BLK) * u * (np.abs(hd) @ np.abs(d).T) + slack @ np.abs(d).T
    return o, tol


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


def stored_bound(o: np.ndarray, tol: np.ndarray) -> np.ndarray:
    """How far a kernel's stored output may be from o itself: it computes some
    o' with |o' - o| <= tol and stores bf16(o'), off by at most half a step,
    2^-8 |o'| <= 2^-8 (|o| + tol).  (From bf16(o), which is off o by another
    half step, it may be 2^-8 |o| further.)"""
    return tol + 2.0 ** -8 * (np.abs(o) + tol)
