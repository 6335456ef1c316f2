"""Inputs and bounds for the GPU tests of the prompt and 8-bit cache operators.

Bounds, from the rounding points (u = half a unit in the last place of the type, 2^-8 for bf16 and 2^-11 for fp16):
an output is rounded once (u), the weights p of the values once (each by at most u, so that the sum moves by at most
u max|v|; over 8-bit caches weights are fp16, which is finer). 1e-4 covers fp32 scores, exponentials and sums. So
|out - exact| <= (2 u + 1e-4) max|v|, and over a whole output the errors, which are independent, stay below u in the
relative 2-norm (about sqrt(2) u / 2). Log-sum-exps: a score sums 128 products in fp32, at most
128 2^-24 sum|q k| / sqrt(128), about 1e-4 for these inputs at scale 1; 3e-4 max(1, scale).
"""
from __future__ import annotations

import numpy as np
import torch

U = {torch.bfloat16: 2.0 ** -8, torch.float16: 2.0 ** -11}


def offsets(lens):
    return np.concatenate([[0], np.cumsum(lens)]).astype(np.int64)


def check(out, lse, want, want_lse, dtype, v_max, scale=1.0):
    """out, want [rows, heads, 128]; NaN rows of `want` belong to no sequence and are left out."""
    out, lse = out.double().cpu().numpy(), None if lse is None else lse.double().cpu().numpy()
    rows = ~np.isnan(want).all((1, 2))
    assert np.isfinite(out[rows]).all()
    err = np.abs(out[rows] - want[rows])
    assert err.max(initial=0) <= (2 * U[dtype] + 1e-4) * v_max
    norm = np.linalg.norm(want[rows])
    assert np.linalg.norm(err) <= U[dtype] * norm + 1e-30
    if lse is not None:
        a, b = lse[:, rows], want_lse[:, rows]
        assert np.array_equal(np.isneginf(a), np.isneginf(b))
        fin = np.isfinite(b)
        assert np.abs(a[fin] - b[fin]).max(initial=0) <= 3e-4 * max(1.0, scale)


def normal(gen, *shape, dtype=torch.bfloat16, scale=1.0):
    return (torch.randn(*shape, generator=gen) * scale).to(dtype)


def to64(t):
    return t.double().cpu().numpy()
