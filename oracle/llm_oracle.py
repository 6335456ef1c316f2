"""fp64 definitions of the prompt and 8-bit cache operators (numpy only).

Every function follows its formula key by key or value by value; nothing is shared with the library.
"""
from __future__ import annotations

import math

import numpy as np


def e4m3_values() -> np.ndarray:
    """Values of the 256 e4m3 codes: 1 sign, 4 exponent (bias 7), 3 mantissa bits; 0x7f and 0xff are NaN."""
    out = np.empty(256)
    for code in range(256):
        e, m = code >> 3 & 15, code & 7
        v = m / 8 * 2.0 ** -6 if e == 0 else (1 + m / 8) * 2.0 ** (e - 7)
        out[code] = math.nan if code & 127 == 127 else -v if code & 128 else v
    return out


E4M3 = e4m3_values()


def e4m3_round(x: np.ndarray) -> np.ndarray:
    """Nearest e4m3 value of |x| <= 448, ties to the even code; the sign is kept."""
    mags = E4M3[:127]
    a = np.abs(x)
    hi = np.searchsorted(mags, a, side="left").clip(0, 126)
    lo = np.maximum(hi - 1, 0)
    d_lo, d_hi = a - mags[lo], mags[hi] - a
    code = np.where((d_lo < d_hi) | ((d_lo == d_hi) & (lo % 2 == 0)), lo, hi)
    return np.copysign(mags[code], x)


def cache_write(x: np.ndarray):
    """Rows [..., 128] -> (code values, scales [...]): the smallest power of two s >= 2^-126 with max|x| / s <= 448
    over the finite values; what is not finite becomes NaN; a row without a non-zero finite value has scale 1."""
    finite = np.isfinite(x)
    top = np.where(finite, np.abs(x), 0.0).max(-1)
    scale = np.ones_like(top)
    for i in np.ndindex(top.shape):
        if top[i] > 0:
            s = 2.0 ** -126
            while top[i] / s > 448:
                s *= 2
            scale[i] = s
    code = np.where(finite, e4m3_round(np.where(finite, x, 0.0) / scale[..., None]), math.nan)
    return code, scale


def attention_row(q: np.ndarray, k: np.ndarray, v: np.ndarray):
    """One query over the keys it sees: k, v [n, 128]. Returns (output, log-sum-exp)."""
    if len(k) == 0:
        return np.zeros_like(q), -math.inf
    s = k @ q / math.sqrt(q.shape[-1])
    m = s.max()
    w = np.exp(s - m)
    return w @ v / w.sum(), m + math.log(w.sum())


def prompt_attention(q, k, v, q_offsets, kv_offsets, causal=True):
    """q [rows, heads, 128], k, v [rows, kv heads, 128], packed. Rows of no sequence are NaN."""
    rows, heads, _ = q.shape
    g = heads // k.shape[1]
    out = np.full(q.shape, math.nan)
    lse = np.full((heads, rows), math.nan)
    for b in range(len(q_offsets) - 1):
        q0, q1, k0, k1 = q_offsets[b], q_offsets[b + 1], kv_offsets[b], kv_offsets[b + 1]
        for i in range(q1 - q0):
            see = max(0, min(k1 - k0, (k1 - k0) - (q1 - q0) + i + 1)) if causal else k1 - k0
            for h in range(heads):
                out[q0 + i, h], lse[h, q0 + i] = attention_row(q[q0 + i, h], k[k0:k0 + see, h // g], v[k0:k0 + see, h // g])
    return out, lse


def tree_attention(q, k_new, v_new, new_offsets, mask, k_cache, v_cache, starts, lengths):
    """Per new token: the request's cache rows, then the new tokens whose bit its mask word (a Python int) has."""
    rows, heads, _ = q.shape
    g = heads // k_new.shape[1]
    out = np.full(q.shape, math.nan)
    lse = np.full((heads, rows), math.nan)
    for b in range(len(new_offsets) - 1):
        t0, t1 = new_offsets[b], new_offsets[b + 1]
        c0, c1 = starts[b], starts[b] + lengths[b]
        for i in range(t0, t1):
            seen = [t0 + j for j in range(t1 - t0) if mask[i] >> j & 1]
            for h in range(heads):
                k = np.concatenate([k_cache[c0:c1, h // g], k_new[seen, h // g]])
                v = np.concatenate([v_cache[c0:c1, h // g], v_new[seen, h // g]])
                out[i, h], lse[h, i] = attention_row(q[i, h], k, v)
    return out, lse
