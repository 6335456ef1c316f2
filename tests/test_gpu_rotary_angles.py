"""fsx_rotary's angles: pairs that are turned so that one of their values all but vanishes, and its own rounding with it.

Bound of a value of a pair (a, b), in units of e = 2^-24 times |a| + |b|. The angle: rates are rounded down to 2^-64 of a turn, a position
of 2^31 times that is 2^-33, and 32 bits behind the point are kept: 2^-33 + 2^-32 < 2^-31 of a turn, 0.05 e. Its rest of at most
pi / 4 in fp32 is rounded three times (the whole number, 2 pi / 2^32, their product): 3 e pi / 4 = 2.4 e. Taylor's series to x^8 of the cosine and x^9 of
the sine leave x^10 / 10! = 0.41 e and x^11 / 11! = 0.03 e out at pi / 4, and their evaluation is off by the rounding of the last sum, e / 2, that of
x^2 in the term before it, 0.3 e, and less than 0.2 e of the others: 1.0 e. The products and their sum: e each at most, 2 e.
Together 6 e < 2^-21; and half a step of the result, 2^-11 of fp16, 2^-25 at least.
"""
from __future__ import annotations

import math
from decimal import Decimal, getcontext

import numpy as np
import pytest
import torch

from paper_2607_15621_gb300 import fsx

from llm_cases import to64

pytestmark = pytest.mark.gpu

POSITIONS = [0, 1, -5, 77, 123456, 10 ** 6 + 1, 2 ** 24 + 1, 2 ** 31 - 1, -(2 ** 31), 2 ** 31]


@pytest.mark.parametrize("adjacent", [False, True])
def test_what_all_but_vanishes_shows_the_angle(adjacent):
    getcontext().prec = 80
    pi2 = Decimal("6.28318530717958647692528676655900576839433879875021164194988918461563281257241799726")
    rng = np.random.default_rng(5)
    rate = [1.0, -1.0, 1e-9, 37.5, 2.0 ** 20, 3.14159, 0.5, -1048575.75] + [10000.0 ** (-j / 64) for j in range(56)]
    t = np.array([[float(Decimal(p) * Decimal(r) % pi2) for r in rate] for p in POSITIONS])
    # head 0: a cos - b sin is small, head 1: a sin + b cos is; the larger of a and b lies in 0.5 .. 1
    long = rng.uniform(0.5, 1, t.shape)
    a, b = long * np.sin(t), long * np.cos(t)
    x = np.stack([np.stack([a, b], -1), np.stack([b, -a], -1)], 1)  # [rows, 2, 64, 2]
    x = torch.from_numpy(x).to(torch.float16)
    x = x.flatten(2) if adjacent else x.transpose(2, 3).flatten(2)
    pairs, out = fsx.RotaryPairs([0] * 64, rate, adjacent), torch.empty(x.shape, dtype=torch.float16, device="cuda")
    st = torch.zeros(1, dtype=torch.int32, device="cuda")
    fsx.rotary(x.cuda(), None, torch.tensor([POSITIONS], device="cuda"), pairs, st, q_out=out)

    def halves(y):
        y = to64(y)
        return (y[..., 0::2], y[..., 1::2]) if adjacent else (y[..., :64], y[..., 64:])

    (a, b), (u, w) = halves(x), halves(out)
    c, s = np.cos(t)[:, None], np.sin(t)[:, None]
    small = 0
    for got, want in ((u, a * c - b * s), (w, a * s + b * c)):
        err = np.abs(got - want)
        assert (err <= 2.0 ** -11 * np.abs(want) + 2.0 ** -21 * (np.abs(a) + np.abs(b)) + 2.0 ** -25).all(), (err / (np.abs(a) + np.abs(b))).max()
        small += int((np.abs(want) < 2.0 ** -10).sum())
    assert int(st) == 0 and small >= 2 * len(POSITIONS) * 60  # what the inputs were made for
