"""fsx_tree_attention with many requests of more than 16 rows each: the plan of the tensor-core kernel over several requests a lane and a
thread (bounds as in llm_cases)."""
from __future__ import annotations

import numpy as np
import pytest

from paper_2607_15621_gb300 import fsx

from test_gpu_tree_attention import agree, make, run

pytestmark = pytest.mark.gpu


@pytest.mark.parametrize("cache8", [True, False])
@pytest.mark.parametrize("B", [24, 33, 641, 1024])
def test_many_requests_of_many_rows(B, cache8):
    rng = np.random.default_rng(B)
    lens, new = rng.integers(0, 50, B), rng.integers(10, 34, B)
    lens[::7], new[5::11] = 0, 0
    if B < 100:
        lens[3], lens[B - 1] = 1500, 1300
    agree(make(lens.tolist(), new.tolist(), heads=1, kv_heads=1, cache8=cache8, seed=B))


def test_bad_requests_among_many():
    rng = np.random.default_rng(7)
    B = 700
    lens, new = rng.integers(1, 40, B), rng.integers(17, 30, B)
    c = make(lens.tolist(), new.tolist(), heads=1, kv_heads=1, seed=7)
    clean, lse, status = run(c)
    assert status == fsx.FSX_OK
    bad = [0, 350, 699]
    starts = c["starts"].copy()
    starts[bad] = -1
    out, lse2, status = run(dict(c, starts=starts))
    assert status == fsx.FSX_ERR_DEVICE_ARG
    for b in range(B):
        rows = slice(int(c["no"][b]), int(c["no"][b + 1]))
        if b in bad:
            assert (out[rows] == 7).all() and (lse2[:, rows] == 7).all()
        else:
            # the plan changes with the work, and with it the order of sums: a unit in the last place of values below 4
            assert (out[rows].float() - clean[rows].float()).abs().max() <= 2.0 ** -6 and (lse[:, rows] - lse2[:, rows]).abs().max() <= 1e-4
