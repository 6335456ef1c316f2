"""fsx_prompt_attention on the GPU against the fp64 oracle, at the sizes and masks where tiles end."""
from __future__ import annotations

import math

import numpy as np
import pytest
import torch

from oracle import llm_oracle
from paper_2607_15621_gb300 import fsx

from llm_cases import check, normal, offsets, to64

pytestmark = pytest.mark.gpu

BF16, F16 = torch.bfloat16, torch.float16


def make(lens, kv_lens=None, heads=4, kv_heads=2, dtype=BF16, seed=0, scale=1.0, pad=0):
    """Packed inputs on the GPU as columns of one buffer; `pad` rows of NaN in front of and behind the sequences."""
    gen = torch.Generator().manual_seed(seed)
    kv_lens = lens if kv_lens is None else kv_lens
    qo, ko = offsets(lens) + pad, offsets(kv_lens) + pad
    nan = lambda n, h: torch.full((n, h, 128), math.nan, dtype=dtype)
    q = torch.cat([nan(pad, heads), normal(gen, sum(lens), heads, 128, dtype=dtype, scale=scale), nan(pad, heads)])
    k, v = (torch.cat([nan(pad, kv_heads), normal(gen, sum(kv_lens), kv_heads, 128, dtype=dtype), nan(pad, kv_heads)])
            for _ in "kv")
    return dict(q=q.cuda(), k=k.cuda(), v=v.cuda(), qo=qo, ko=ko)


def run(c, causal=True, lse=True, stream=None):
    out = torch.full(c["q"].shape, 7.0, dtype=c["q"].dtype, device="cuda")
    z = torch.full((c["q"].shape[1], c["q"].shape[0]), 7.0, device="cuda") if lse else None
    status = torch.zeros(1, dtype=torch.int32, device="cuda")
    fsx.prompt_attention(c["q"], c["k"], c["v"], torch.as_tensor(c["qo"], device="cuda"),
                         torch.as_tensor(c["ko"], device="cuda"), out, status, lse=z, causal=causal, stream=stream)
    torch.cuda.synchronize()
    return out, z, int(status)


def oracle(c, causal=True):
    with np.errstate(invalid="ignore"):
        return llm_oracle.prompt_attention(to64(c["q"]), to64(c["k"]), to64(c["v"]), c["qo"], c["ko"], causal)


def agree(c, causal=True, scale=1.0):
    out, lse, status = run(c, causal)
    assert status == fsx.FSX_OK
    want, want_lse = oracle(c, causal)
    v = c["v"].double()
    check(out, lse, want, want_lse, c["q"].dtype, float(v[v.isfinite()].abs().max()) if v.isfinite().any() else 0.0, scale)
    own = np.zeros(len(want), bool)
    for a, b in zip(c["qo"][:-1], c["qo"][1:]):
        own[a:b] = True
    assert (out[torch.as_tensor(~own, device="cuda")] == 7).all()  # rows of no sequence stay
    return out, lse


@pytest.mark.parametrize("dtype", [BF16, F16])
@pytest.mark.parametrize("lens", [[1], [2, 0, 1], [63, 64, 65], [127, 128, 129], [200, 3, 257], [385]])
def test_causal_lengths(lens, dtype):
    agree(make(lens, dtype=dtype, seed=len(lens)))


@pytest.mark.parametrize("heads,kv_heads", [(1, 1), (2, 2), (3, 1), (6, 2), (7, 1), (8, 1), (64, 1)])
def test_grouped_heads(heads, kv_heads):
    agree(make([5, 70, 131], heads=heads, kv_heads=kv_heads, seed=heads))


@pytest.mark.parametrize("causal", [True, False])
@pytest.mark.parametrize("lens,kv_lens", [([1, 1], [300, 129]), ([4, 130], [260, 131]), ([100, 20], [128, 400]),
                                          ([5, 140, 3], [0, 7, 3]), ([300], [130]), ([0, 3], [9, 3])])
def test_keys_before_the_queries_and_rows_that_see_nothing(lens, kv_lens, causal):
    agree(make(lens, kv_lens, seed=3), causal)


def test_not_causal():
    agree(make([1, 127, 300], dtype=F16, seed=4), causal=False)


@pytest.mark.parametrize("scale", [0.0, 8.0, 60.0])
def test_flat_and_sharp_scores(scale):
    agree(make([190, 64], seed=5, scale=scale), scale=scale)


@pytest.mark.parametrize("causal", [True, False])
def test_what_lies_between_sequences_has_no_effect(causal):
    """NaN rows in front of and behind the sequences, in tiles that the sequences' last rows share."""
    agree(make([37, 150], pad=70, seed=6), causal)


@pytest.mark.parametrize("value", [math.nan, math.inf, -math.inf])
@pytest.mark.parametrize("where", ["k", "v"])
def test_later_tokens_have_no_effect_whatever_they_hold(where, value):
    c = make([300], seed=7)
    clean, lse, _ = run(c)
    bad = 210
    c[where][bad:] = value
    out, lse2, status = run(c)
    assert status == fsx.FSX_OK
    assert torch.equal(out[:bad], clean[:bad]) and torch.equal(lse[:, :bad], lse2[:, :bad])
    if not (where == "k" and value == -math.inf):
        assert not torch.isfinite(out[bad:]).all()


def test_infinite_values_that_are_seen_show():
    c = make([150], seed=8, heads=2, kv_heads=2)
    c["v"][100, 0, 3] = math.inf
    c["v"][120, 1, 7] = -math.inf
    out, _, _ = run(c)
    assert torch.isfinite(out[:100]).all()
    assert (out[100:, 0, 3] == math.inf).all() and (out[120:, 1, 7] == -math.inf).all()
    assert torch.isfinite(out[:120, 1]).all() and torch.isfinite(out[:, 0, 4:]).all()


def test_strides_and_alignment():
    """q, k and v as columns of one wider buffer, k and v from different places; the same bits as from plain tensors."""
    c = make([130, 9], heads=3, kv_heads=3, seed=9)
    plain, lse, _ = run(c)
    rows = c["q"].shape[0]
    buf = torch.full((rows, 12 * 128 + 8), math.nan, dtype=BF16, device="cuda")
    for at, name in ((1, "q"), (5, "k"), (9, "v")):
        buf[:, at * 128:(at + 3) * 128] = c[name].reshape(rows, -1)
        c[name] = buf[:, at * 128:(at + 3) * 128].unflatten(1, (3, 128))
    out, lse2, status = run(c)
    assert status == fsx.FSX_OK and torch.equal(out, plain) and torch.equal(lse, lse2)


def test_another_stream_and_repeats_give_the_same_bits():
    c = make([257, 64], heads=8, kv_heads=2, seed=10)
    torch.cuda.synchronize()
    a, za, _ = run(c)
    side = torch.cuda.Stream()
    b, zb, _ = run(c, stream=side)
    assert torch.equal(a, b) and torch.equal(za, zb)
    with torch.cuda.stream(side):
        d, _, _ = run(c, lse=False)
    assert torch.equal(a, d)


def test_many_sequences():
    rng = np.random.default_rng(11)
    lens = rng.integers(0, 12, 1024)
    agree(make(lens.tolist(), heads=2, kv_heads=1, seed=11))


@pytest.mark.parametrize("causal", [True, False])
def test_items_of_one_and_two_tiles_of_uneven_length(causal):
    lens = [100, 300, 129, 128, 500, 20, 0, 257]
    past = [700, 0, 260, 900, 5, 130, 40, 128]
    agree(make(lens, [a + b for a, b in zip(lens, past)], heads=32, kv_heads=32, seed=14), causal)


@pytest.mark.parametrize("lens,heads", [([3, 200, 40], 16), ([130, 1, 300], 8)])
def test_sequences_with_more_queries_than_keys(lens, heads):
    agree(make(lens, [n // 2 for n in lens], heads=heads, kv_heads=2, seed=15))


def test_more_items_than_one_wave_of_blocks_takes():
    rng = np.random.default_rng(16)
    agree(make(rng.integers(0, 7, 1000).tolist(), heads=16, kv_heads=16, seed=16))


def test_a_bad_sequence_is_reported_and_passed_over():
    c = make([40, 30, 50], seed=12)
    want, want_lse = oracle(c)
    for qo, ko, spoiled in (([0, 40, 70, 121], [0, 40, 70, 120], [2]), ([0, 40, 70, 120], [-1, 40, 70, 120], [0]),
                            ([0, 40, 70, 120], [0, 40, 70, 1 << 40], [2])):
        out, lse, status = run(dict(c, qo=np.array(qo), ko=np.array(ko)))
        assert status == fsx.FSX_ERR_DEVICE_ARG
        for b, (lo, hi) in enumerate(((0, 40), (40, 70), (70, 120))):
            if b in spoiled:
                assert (out[lo:hi] == 7).all() and (lse[:, lo:hi] == 7).all()
            else:
                check(out[lo:hi], lse[:, lo:hi], want[lo:hi], want_lse[:, lo:hi], BF16, float(c["v"].abs().max()))


def test_status_stays_until_it_is_cleared():
    c = make([4], seed=13)
    status = torch.full((1,), 5, dtype=torch.int32, device="cuda")
    out = torch.empty_like(c["q"])
    fsx.prompt_attention(c["q"], c["k"], c["v"], torch.tensor([0, 9], device="cuda"), torch.tensor([0, 4], device="cuda"),
                         out, status)
    assert int(status) == 5


def test_no_rows():
    c = make([0, 0], seed=14)
    out, _, status = run(c)
    assert status == fsx.FSX_OK and out.numel() == 0


def test_offsets_beyond_32_bits():
    rows = (1 << 31) // (32 * 128) + 600  # k and v of 4.3 GB each: the last rows lie past 2^31 elements
    gen = torch.Generator().manual_seed(15)
    c = make([150], heads=32, kv_heads=32, seed=15)
    k, v = (torch.empty(rows, 32, 128, dtype=BF16, device="cuda") for _ in "kv")
    k[-150:], v[-150:] = c["k"], c["v"]
    q = torch.empty(rows, 32, 128, dtype=BF16, device="cuda")
    q[-150:] = c["q"]
    plain, lse, _ = run(c)
    out = torch.empty_like(q)
    z = torch.empty(32, rows, device="cuda")
    status = torch.zeros(1, dtype=torch.int32, device="cuda")
    off = torch.tensor([rows - 150, rows], device="cuda")
    fsx.prompt_attention(q, k, v, off, off, out, status, lse=z)
    assert int(status) == fsx.FSX_OK
    assert torch.equal(out[-150:], plain) and torch.equal(z[:, -150:], lse)
