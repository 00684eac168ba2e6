"""Steps over request pages (oracle): per-head norms, attention under a
sliding window with sinks, and the 4-bit page format.

Definitions (the paper names none of these; they are what its models and a
serving loop after a composed prefill need):

* norm of a head vector: x / sqrt(mean(x^2) + eps) * w;
* a row at position p with first key lo, window W > 0 and S sinks sees the
  keys j in [lo, p] with j > p - W or j < lo + S; W = 0: all of [lo, p]; a row
  at position -1 sees nothing; a row that sees nothing has output 0, lse -inf;
* 4-bit values: for each 32 dims the smallest 2^k, k >= -126, with max |x| <=
  6 * 2^k (1 if all are zero); x / 2^k to the nearest of 0, .5, 1, 1.5, 2, 3,
  4, 6, ties to the even code; a block holding a NaN or infinity is NaN.

Pins: tests/test_oracle_step.py (loops in plain Python, the grid by hand).
"""
from __future__ import annotations

import math

import numpy as np

E2M1 = np.array([0.0, 0.5, 1.0, 1.5, 2.0, 3.0, 4.0, 6.0])


def rms_norm(x, w, eps):
    x = np.asarray(x, dtype=np.float64)
    y = x / np.sqrt((x * x).mean(-1, keepdims=True) + eps)
    return y if w is None else y * np.asarray(w, dtype=np.float64)


def visible_keys(pos, lo, window, n_sinks, n_keys):
    """[n_keys] mask of the keys a row sees."""
    j = np.arange(n_keys)
    seen = (j >= lo) & (j <= pos)
    if window > 0:
        seen &= (j > pos - window) | (j < lo + n_sinks)
    return seen


def step_attention(q, positions, row_lo, K, V, window=0, n_sinks=0, scale=None):
    """q [T][H_q][d] (rotated), K/V [P][H_kv][d] -> out, lse, and for error
    bounds sum_j p_j |v_j| and max_j scale sum_i |q_i k_ji| over visible keys."""
    q, K, V = (np.asarray(x, dtype=np.float64) for x in (q, K, V))
    T, Hq, d = q.shape
    G = Hq // K.shape[1] if K.shape[0] else 1
    scale = 1.0 / math.sqrt(d) if scale is None else scale
    out, mag = np.zeros((T, Hq, d)), np.zeros((T, Hq, d))
    lse, top = np.full((T, Hq), -np.inf), np.zeros((T, Hq))
    for t in range(T):
        seen = visible_keys(positions[t], row_lo[t], window, n_sinks, K.shape[0])
        if not seen.any():
            continue
        for h in range(Hq):
            k, v = K[seen, h // G], V[seen, h // G]
            s = scale * (k @ q[t, h])
            with np.errstate(invalid="ignore"):
                m = s.max()
                e = np.exp(s - m)
                z = e.sum()
                out[t, h] = e @ v / z
                mag[t, h] = e @ np.abs(v) / z
                lse[t, h] = m + math.log(z) if z == z else np.nan
                top[t, h] = scale * (np.abs(k) @ np.abs(q[t, h])).max()
    return out, lse, mag, top


def e2m1_encode(x):
    """x [..][d] -> codes [..][d/2] uint8, scale bytes [..][d/32] uint8."""
    x = np.asarray(x, dtype=np.float64)
    b = x.reshape(*x.shape[:-1], -1, 32)
    ok = np.isfinite(b).all(-1)
    b = np.where(ok[..., None], b, 0.0)
    amax = np.abs(b).max(-1)
    f, e = np.frexp(amax)                       # amax = f 2^e, f in [0.5, 1)
    k = np.where(f <= 0.75, e - 3, e - 2)       # 6 = 0.75 * 2^3
    k = np.where(amax == 0, 0, np.maximum(k, -126))
    y = np.ldexp(b, -k[..., None])
    a = np.abs(y)
    hi = np.clip(np.searchsorted(E2M1, a), 0, 7)       # E2M1[hi] >= a
    lo = np.maximum(hi - 1, 0)
    dl, dh = a - E2M1[lo], E2M1[hi] - a
    code = np.where((dl < dh) | ((dl == dh) & (lo % 2 == 0)), lo, hi)
    code = np.where(a == 0, 0, code) | np.where(np.signbit(y), 8, 0)
    scale = np.where(ok, k + 127, 255).astype(np.uint8)
    code = code.reshape(x.shape).astype(np.uint8)
    return code[..., 0::2] | (code[..., 1::2] << 4), scale


def e2m1_decode(codes, scale):
    grid = np.concatenate([E2M1, -E2M1])
    codes, scale = np.asarray(codes), np.asarray(scale)
    x = np.stack([grid[codes & 15], grid[codes >> 4]], -1).reshape(*codes.shape[:-1], 2 * codes.shape[-1])
    f = np.where(scale == 255, np.nan, np.ldexp(1.0, scale.astype(np.int64) - 127))
    return x * np.repeat(f, 32, -1)
