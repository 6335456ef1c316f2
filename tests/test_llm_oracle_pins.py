"""Pins of the fp64 oracle of the prompt and 8-bit cache operators against torch compositions and closed forms."""
from __future__ import annotations

import math

import numpy as np
import pytest
import torch

from oracle import llm_oracle as o


def test_e4m3_values_are_torchs():
    codes = torch.arange(256, dtype=torch.uint8)
    want = codes.view(torch.float8_e4m3fn).double().numpy()
    assert np.array_equal(np.isnan(o.E4M3), np.isnan(want))
    assert np.array_equal(o.E4M3[~np.isnan(want)], want[~np.isnan(want)])


def test_e4m3_rounding_is_nearest_even():
    mids = (o.E4M3[:126] + o.E4M3[1:127]) / 2
    x = np.concatenate([o.E4M3[:127], mids, mids * (1 + 1e-9), mids * (1 - 1e-9), -mids])
    want = torch.from_numpy(x.astype(np.float32)).to(torch.float8_e4m3fn).double().numpy()
    exact = x.astype(np.float32).astype(np.float64)
    assert np.array_equal(o.e4m3_round(exact), want)


@pytest.mark.parametrize("top,scale", [(448.0, 1.0), (448.5, 2.0), (224.0, 0.5), (1.0, 2.0 ** -8), (0.0, 1.0),
                                       (2.0 ** -140, 2.0 ** -126), (3.0e38, 2.0 ** 120)])
def test_scale_is_the_smallest_power_of_two(top, scale):
    x = np.zeros((1, 128))
    x[0, 5] = -top
    code, s = o.cache_write(x)
    assert s[0] == scale
    assert np.abs(code).max() <= 448


def test_write_handles_what_is_not_finite():
    x = np.ones((1, 128))
    x[0, 3], x[0, 4] = math.inf, math.nan
    code, s = o.cache_write(x)
    assert np.isnan(code[0, [3, 4]]).all() and np.isfinite(np.delete(code[0], [3, 4])).all()
    assert s[0] == 2.0 ** -8


@pytest.mark.parametrize("causal", [True, False])
def test_prompt_attention_is_torchs(causal):
    g = torch.Generator().manual_seed(0)
    lens, past = [3, 1, 7], [0, 5, 2]
    qo = np.cumsum([0] + lens)
    ko = np.cumsum([0] + [a + b for a, b in zip(lens, past)])
    q = torch.randn(qo[-1], 4, 128, generator=g, dtype=torch.float64)
    k, v = (torch.randn(ko[-1], 2, 128, generator=g, dtype=torch.float64) for _ in "kv")
    out, lse = o.prompt_attention(q.numpy(), k.numpy(), v.numpy(), qo, ko, causal)
    for b, n in enumerate(lens):
        nk = n + past[b]
        mask = torch.ones(n, nk, dtype=torch.bool).tril(past[b]) if causal else torch.ones(n, nk, dtype=torch.bool)
        kk, vv = (x[ko[b]:ko[b + 1]].repeat_interleave(2, 1).transpose(0, 1) for x in (k, v))
        want = torch.nn.functional.scaled_dot_product_attention(q[qo[b]:qo[b + 1]].transpose(0, 1), kk, vv, attn_mask=mask)
        assert np.allclose(out[qo[b]:qo[b + 1]], want.transpose(0, 1).numpy(), atol=1e-12)


def test_rows_that_see_nothing():
    q = np.ones((3, 1, 128))
    out, lse = o.prompt_attention(q, np.ones((1, 1, 128)), np.full((1, 1, 128), 2.0), [0, 3], [0, 1], True)
    assert (out[:2] == 0).all() and np.isneginf(lse[:, :2]).all() and np.allclose(out[2], 2)
    out, lse = o.tree_attention(q, q, q, [0, 3], [0, 0b101, 0], q[:0], q[:0], [0], [0])
    assert (out[[0, 2]] == 0).all() and np.isneginf(lse[0, [0, 2]]).all() and np.allclose(out[1], 1)


def test_a_chain_over_a_cache_is_the_causal_prompt():
    rng = np.random.default_rng(1)
    q = rng.standard_normal((5, 4, 128))
    k, v = rng.standard_normal((2, 12, 2, 128))
    want, want_lse = o.prompt_attention(q, k, v, [0, 5], [0, 12], True)
    chain = [(1 << (i + 1)) - 1 for i in range(5)]
    out, lse = o.tree_attention(q, k[7:], v[7:], [0, 5], chain, k[:7], v[:7], [0], [7])
    assert np.allclose(out, want, atol=1e-12) and np.allclose(lse, want_lse, atol=1e-12)


def test_siblings_do_not_see_one_another():
    rng = np.random.default_rng(2)
    q, k, v = rng.standard_normal((3, 3, 1, 128))
    kc, vc = rng.standard_normal((2, 4, 1, 128))
    masks = [0b001, 0b011, 0b101]
    out, _ = o.tree_attention(q, k, v, [0, 3], masks, kc, vc, [0], [4])
    v2 = v.copy()
    v2[1] = math.nan
    moved, _ = o.tree_attention(q, k, v2, [0, 3], masks, kc, vc, [0], [4])
    assert np.array_equal(out[[0, 2]], moved[[0, 2]]) and np.isnan(moved[1]).all()
