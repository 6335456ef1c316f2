"""fsx_tree_attention over 8-bit caches whose values are small, zero or of very different size.

Bounds: those of llm_cases.check, held for every request by itself, so that small requests count; a float16 output has a
smallest step of 2^-24, so half of that is allowed beside them.
"""
from __future__ import annotations

import math

import numpy as np
import pytest
import torch

from paper_2607_15621_gb300 import fsx

from llm_cases import U, normal
from test_gpu_tree_attention import caches64, make, oracle, run, to64

pytestmark = pytest.mark.gpu

BF16, F16 = torch.bfloat16, torch.float16
FEW = [(1, 4, 2), (11, 2, 2)]                 # new tokens a request, heads, kv heads: 2 and 11 rows an item
MANY = [(11, 4, 2), (24, 2, 2), (40, 8, 2)]   # 22, 24 and 160


def build(lens, new, heads, kv_heads, dtype, seed, keys=None, values=None, new_values=None):
    """Requests of `new` tokens each; `keys` and `values` change the caches' rows [rows, kv heads, 128] in fp32 before they
    are written, given the row numbers of every request; `new_values` changes the new tokens' values."""
    c = make(lens, [new] * len(lens), heads=heads, kv_heads=kv_heads, dtype=dtype, cache8=True, seed=seed, poison=False)
    gen = torch.Generator().manual_seed(seed + 1000)
    own = [np.arange(s, s + n) for s, n in zip(c["starts"], lens)]
    rows = c["kc"].shape[0]
    k, v = (normal(gen, rows, kv_heads, 128, dtype=torch.float32) for _ in "kv")
    for x, change in ((k, keys), (v, values)):
        if change is not None:
            change(x, own)
    status = torch.zeros(1, dtype=torch.int32, device="cuda")
    fsx.cache_write(k.to(dtype).cuda(), v.to(dtype).cuda(), None, c["kc"], c["vc"], c["ks"], c["vs"], status)
    assert int(status) == fsx.FSX_OK
    if new_values is not None:
        vn = c["vn"].float().cpu()
        new_values(vn)
        c["vn"] = vn.to(dtype).cuda()
    return c


def agree(c, v_max=None, slack=1.0):
    """`slack`: 2 where a key or two carry a row, whose rounded weights then move all of its values alike."""
    out, lse, status = run(c)
    assert status == fsx.FSX_OK
    want, want_lse = oracle(c)
    got, z, dtype = to64(out), to64(lse), c["q"].dtype
    tiny = 2.0 ** -25 if dtype == F16 else 0.0
    _, v = caches64(c)
    vn = to64(c["vn"])
    assert np.isfinite(got).all()
    for b, n in enumerate(c["lens"]):
        t = slice(int(c["no"][b]), int(c["no"][b + 1]))
        top = max(np.abs(v[c["starts"][b]:c["starts"][b] + n]).max(initial=0), np.abs(vn[t]).max(initial=0)) if v_max is None else v_max
        err = got[t] - want[t]
        assert np.abs(err).max() <= (2 * U[dtype] + 1e-4) * top + tiny
        assert np.linalg.norm(err) <= slack * U[dtype] * np.linalg.norm(want[t]) + tiny * math.sqrt(err.size)
    assert np.abs(z - want_lse).max() <= 1e-3
    return out


def small_values(shape, scale, dtype, zeros):
    new, heads, kv_heads = shape

    def values(v, own):
        v *= scale
        for at in own:
            if zeros == "some":
                v[at[::5]] = 0
            elif zeros == "most":
                v[at[:len(at) * 2 // 3]] = 0

    def new_values(vn):
        vn *= scale
        if zeros != "none":
            vn[::3] = 0

    return build([400, 130], new, heads, kv_heads, dtype, 41, values=values, new_values=new_values)


SMALL = [(BF16, s) for s in (1e-2, 1e-3, 1e-4, 1e-5, 2.0 ** -40)] + [(F16, s) for s in (1e-2, 1e-3, 1e-4)]


@pytest.mark.parametrize("zeros", ["none", "some", "most"])
@pytest.mark.parametrize("dtype,scale", SMALL)
@pytest.mark.parametrize("shape", FEW)
def test_small_values_few_rows(shape, dtype, scale, zeros):
    agree(small_values(shape, scale, dtype, zeros))


@pytest.mark.parametrize("shape", FEW)
def test_small_cached_values_beside_large_new_ones(shape):
    """Rows that see no new token of any weight: the new tokens' values leave no trace."""
    new, heads, kv_heads = shape
    c = build([300, 90], new, heads, kv_heads, BF16, 42, values=lambda v, own: v.mul_(1e-5), new_values=lambda v: v.mul_(1e5))
    c["mask"] = [0] * len(c["mask"])
    agree(c, v_max=5e-5)


def a_row_of_little_weight(value):
    """Queries of positive components; a row of keys -6, whose weight is e^-54 or less, with values `value` times as large."""
    def keys(k, own):
        for at in own:
            k[at[len(at) // 3]] = -6

    def values(v, own):
        for at in own:
            v[at[len(at) // 3]] *= value

    return keys, values


@pytest.mark.parametrize("value", [1e4, 1e8])
@pytest.mark.parametrize("shape", FEW)
def test_a_large_row_of_little_weight_few_rows(shape, value):
    keys, values = a_row_of_little_weight(value)
    c = build([500, 150], *shape, BF16, 43, keys=keys, values=values)
    c["q"] = c["q"].abs()
    agree(c, v_max=6.0)


def on_small_rows(order):
    """Keys of 6 (against 0 of the others) on rows with values 2^-40 times as large: they carry all of the weight."""
    def small(n):
        i = np.arange(n)
        return i % 3 == 0 if order == "mixed" else i < n // 2 if order == "first" else i >= n // 2

    def keys(k, own):
        k.zero_()
        for at in own:
            k[at[small(len(at))]] = 6
            k[at[small(len(at))], :, ::7] += 0.5

    def values(v, own):
        for at in own:
            v[at[small(len(at))]] *= 2.0 ** -40

    return keys, values


@pytest.mark.parametrize("order", ["mixed", "first", "last"])
@pytest.mark.parametrize("shape", FEW)
def test_small_rows_that_carry_the_weight_few_rows(shape, order):
    keys, values = on_small_rows(order)
    c = build([700, 260], *shape, BF16, 44, keys=keys, values=values)
    c["q"] = c["q"].abs()
    c["mask"] = [0] * len(c["mask"])
    agree(c, v_max=6 * 2.0 ** -40, slack=2.0)


@pytest.mark.parametrize("shape", FEW)
def test_rows_of_every_size_few_rows(shape):
    def values(v, own):
        v *= torch.exp2(torch.randint(-60, 10, (v.shape[0], 1, 1), generator=torch.Generator().manual_seed(5)).float())

    agree(build([640, 200], *shape, BF16, 45, values=values, new_values=lambda v: v.mul_(1e-6)), slack=2.0)


@pytest.mark.parametrize("zeros", ["none", "some", "most"])
@pytest.mark.parametrize("dtype,scale", SMALL)
@pytest.mark.parametrize("shape", MANY)
def test_small_values_many_rows(shape, dtype, scale, zeros):
    agree(small_values(shape, scale, dtype, zeros))


@pytest.mark.parametrize("value", [1e4, 1e8])
@pytest.mark.parametrize("shape", MANY)
def test_a_large_row_of_little_weight_many_rows(shape, value):
    keys, values = a_row_of_little_weight(value)
    c = build([500, 150], *shape, BF16, 43, keys=keys, values=values)
    c["q"] = c["q"].abs()
    agree(c, v_max=6.0)


@pytest.mark.parametrize("order", ["mixed", "first", "last"])
@pytest.mark.parametrize("shape", MANY)
def test_small_rows_that_carry_the_weight_many_rows(shape, order):
    """`first` and `last`: whole chunks that need no scales behind or before whole chunks that do."""
    keys, values = on_small_rows(order)
    c = build([700, 260], *shape, BF16, 44, keys=keys, values=values)
    c["q"] = c["q"].abs()
    c["mask"] = [0] * len(c["mask"])
    agree(c, v_max=6 * 2.0 ** -40, slack=2.0)


@pytest.mark.parametrize("shape", MANY)
def test_rows_of_every_size_many_rows(shape):
    def values(v, own):
        v *= torch.exp2(torch.randint(-60, 10, (v.shape[0], 1, 1), generator=torch.Generator().manual_seed(5)).float())

    agree(build([640, 200], *shape, BF16, 45, values=values, new_values=lambda v: v.mul_(1e-6)), slack=2.0)


@pytest.mark.parametrize("scale", [2.0 ** -8, 2.0 ** -30])
@pytest.mark.parametrize("shape", MANY)
def test_zeros_then_small_values(shape, scale):
    """A cache that starts with chunks of zeros, whose scales say nothing; new tokens as small as the rest."""
    def values(v, own):
        v *= scale
        for at in own:
            v[at[:512]] = 0

    agree(build([900, 640], *shape, BF16, 46, values=values, new_values=lambda v: v.mul_(scale)))


@pytest.mark.parametrize("scale", [1.0, 1e-5])
@pytest.mark.parametrize("shape", MANY + FEW[1:])
def test_scales_of_any_kind(shape, scale):
    """Scales that are no powers of two, over several chunks."""
    c = build([900, 300], *shape, BF16, 47, values=lambda v, own: v.mul_(scale), new_values=lambda v: v.mul_(scale))
    gen = torch.Generator(device="cuda").manual_seed(3)
    c["vs"] = c["vs"] * (0.6 + 0.3 * torch.rand(c["vs"].shape, generator=gen, device="cuda"))
    c["ks"] = c["ks"] * (0.8 + 0.4 * torch.rand(c["ks"].shape, generator=gen, device="cuda"))
    agree(c)


@pytest.mark.parametrize("value", [1e5, 1e10, 1e30])
@pytest.mark.parametrize("shape", MANY + FEW[1:])
def test_an_unseen_draft_of_any_size_has_no_effect(shape, value):
    c = build([300, 0], *shape, BF16, 48)
    n, hidden = shape[0], 5
    c["mask"] = [m & ~(1 << hidden) for m in c["mask"]]
    c["mask"][hidden] |= 1 << hidden
    clean, lse, _ = run(c)
    for t in (hidden, n + hidden):
        c["vn"][t] = c["vn"][t] * value
    out, lse2, status = run(c)
    blind = [i for i in range(2 * n) if i % n != hidden]
    assert status == fsx.FSX_OK and torch.equal(out[blind], clean[blind]) and torch.equal(lse[:, blind], lse2[:, blind])
    want, _ = oracle(c)
    err = to64(out)[blind] - want[blind]
    assert np.linalg.norm(err) <= U[BF16] * np.linalg.norm(want[blind])


@pytest.mark.parametrize("value", [1e5, 1e10])
@pytest.mark.parametrize("shape", MANY + FEW[1:])
def test_a_large_draft_of_little_weight(shape, value):
    """Everyone sees token 1, whose key is -12 against queries of positive components: a weight of e^-108."""
    c = build([200, 0], *shape, BF16, 49)
    n = shape[0]
    c["q"] = c["q"].abs()
    c["mask"] = [m | 2 for m in c["mask"]]
    for t in (1, n + 1):
        c["kn"][t] = -12
        c["vn"][t] = c["vn"][t] * value
    # (a row that sees nothing else takes it whole: none here, every token sees itself and token 1 another)
    c["mask"][1] |= 1
    c["mask"][n + 1] |= 1
    agree(c, v_max=6.0)
