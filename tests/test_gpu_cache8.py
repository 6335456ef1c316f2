"""fsx_cache_write_e4m3 and fsx_cache_read_e4m3 on the GPU: every code and scale equal to the fp64 oracle's."""
from __future__ import annotations

import math

import numpy as np
import pytest
import torch

from oracle import llm_oracle
from paper_2607_15621_gb300 import fsx

from llm_cases import to64

pytestmark = pytest.mark.gpu

DTYPES = [torch.bfloat16, torch.float16, torch.float32]


def cache(rows, heads):
    return ([torch.full((rows, heads, 128), 0x55, dtype=torch.uint8, device="cuda").view(torch.float8_e4m3fn) for _ in "kv"],
            [torch.full((heads, rows), 7.0, device="cuda") for _ in "kv"])


def values(n, heads, dtype, seed):
    g = torch.Generator().manual_seed(seed)
    x = torch.randn(n, heads, 128, generator=g) * torch.exp(2 * torch.randn(n, heads, 1, generator=g))
    return x.to(dtype).cuda()


def same(code, want):
    got = code.double().cpu().numpy()
    return np.array_equal(got, want, equal_nan=True)


@pytest.mark.parametrize("dtype", DTYPES)
@pytest.mark.parametrize("n,heads", [(1, 1), (4, 32), (7, 3), (8, 2), (129, 5)])
def test_write_and_read_back(n, heads, dtype):
    k, v = values(n, heads, dtype, n), values(n, heads, dtype, n + 1000)
    if n > 6:
        k[3] = 0
        v[5] = 448 * 2.0 ** -9
    (kc, vc), (ks, vs) = cache(n + 40, heads)
    rows = torch.randperm(n + 40, generator=torch.Generator().manual_seed(n))[:n].cuda()
    status = torch.zeros(1, dtype=torch.int32, device="cuda")
    fsx.cache_write(k, v, rows, kc, vc, ks, vs, status)
    assert int(status) == fsx.FSX_OK
    rest = torch.ones(n + 40, dtype=torch.bool, device="cuda")
    rest[rows] = False
    for x, c, s in ((k, kc, ks), (v, vc, vs)):
        want, scale = llm_oracle.cache_write(to64(x))
        assert same(c.view(torch.uint8)[rows].view(torch.float8_e4m3fn), want)
        assert np.array_equal(s[:, rows].T.double().cpu().numpy(), scale)
        assert (c.view(torch.uint8)[rest] == 0x55).all() and (s[:, rest] == 7).all()
    for out in DTYPES:
        buf = torch.full((n, 2 * heads, 128), 7.0, dtype=out, device="cuda")
        a, b = buf[:, :heads], buf[:, heads:]
        fsx.cache_read(kc, vc, ks, vs, rows, a, b, status)
        assert int(status) == fsx.FSX_OK
        for x, got in ((k, a), (v, b)):
            want, scale = llm_oracle.cache_write(to64(x))
            exact = torch.from_numpy(want * scale[..., None]).float().to(out)  # exact in fp32
            assert torch.equal(got.cpu(), exact)


@pytest.mark.parametrize("dtype", DTYPES)
def test_ties_subnormals_and_the_scale_limits(dtype):
    mids = (llm_oracle.E4M3[:126] + llm_oracle.E4M3[1:127]) / 2
    rows = [np.concatenate([mids[:126], [448, -448]]), np.concatenate([-mids[:126], [447, 0.0]]),
            np.concatenate([llm_oracle.E4M3[:127], [448]]), np.full(128, 448.0), np.full(128, 456.0)]
    if dtype != torch.float16:
        rows += [np.linspace(-1, 1, 128) * 2.0 ** -130, np.linspace(0, 3.0e38, 128), np.r_[2.0 ** -133, np.zeros(127)]]
    x = torch.from_numpy(np.stack(rows)[:, None]).to(dtype).cuda()
    (kc, vc), (ks, vs) = cache(len(rows), 1)
    status = torch.zeros(1, dtype=torch.int32, device="cuda")
    fsx.cache_write(x, -x, None, kc, vc, ks, vs, status)
    for y, c, s in ((x, kc, ks), (-x, vc, vs)):
        want, scale = llm_oracle.cache_write(to64(y))
        assert same(c, want) and np.array_equal(s.T.double().cpu().numpy(), scale)
    assert int(status) == fsx.FSX_OK


def test_values_that_are_not_finite_are_reported():
    k, v = values(9, 2, torch.bfloat16, 1), values(9, 2, torch.bfloat16, 2)
    k[4, 1, 7], k[5, 0, 8], v[0, 0, 127] = math.inf, math.nan, -math.inf
    v[8, 1] = math.nan
    (kc, vc), (ks, vs) = cache(9, 2)
    status = torch.zeros(1, dtype=torch.int32, device="cuda")
    fsx.cache_write(k, v, None, kc, vc, ks, vs, status)
    assert int(status) == fsx.FSX_ERR_RANGE
    for x, c, s in ((k, kc, ks), (v, vc, vs)):
        want, scale = llm_oracle.cache_write(to64(x))
        assert same(c, want) and np.array_equal(s.T.double().cpu().numpy(), scale)


@pytest.mark.parametrize("bad", [-1, 20, 1 << 40])
def test_rows_outside_the_cache_are_left_out(bad):
    k, v = values(3, 2, torch.bfloat16, 3), values(3, 2, torch.bfloat16, 4)
    (kc, vc), (ks, vs) = cache(20, 2)
    rows = torch.tensor([5, bad, 19], device="cuda")
    status = torch.zeros(1, dtype=torch.int32, device="cuda")
    fsx.cache_write(k, v, rows, kc, vc, ks, vs, status)
    assert int(status) == fsx.FSX_ERR_DEVICE_ARG
    written = (kc.view(torch.uint8) != 0x55).any(2).any(1).cpu()
    assert written.nonzero().flatten().tolist() == [5, 19]
    a, b = (torch.full((3, 2, 128), 7.0, device="cuda") for _ in "kv")
    status.zero_()
    fsx.cache_read(kc, vc, ks, vs, rows, a, b, status)
    assert int(status) == fsx.FSX_ERR_DEVICE_ARG
    assert (a[1] == 7).all() and (b[1] == 7).all() and not (a[0] == 7).all() and not (b[2] == 7).all()


def test_fused_columns_and_another_stream():
    buf = values(33, 6, torch.bfloat16, 5)
    k, v = buf[:, 1:3], buf[:, 3:5]
    status = torch.zeros(1, dtype=torch.int32, device="cuda")
    (kc, vc), (ks, vs) = cache(33, 2)
    (kd, vd), (kt, vt) = cache(33, 2)
    torch.cuda.synchronize()
    fsx.cache_write(k, v, None, kc, vc, ks, vs, status)
    side = torch.cuda.Stream()
    with torch.cuda.stream(side):
        fsx.cache_write(k.contiguous(), v.contiguous(), None, kd, vd, kt, vt, status)
    torch.cuda.synchronize()
    assert torch.equal(kc.view(torch.uint8), kd.view(torch.uint8)) and torch.equal(vs, vt)
    want, _ = llm_oracle.cache_write(to64(k))
    assert same(kc, want)


def test_no_rows_and_offsets_beyond_32_bits():
    status = torch.zeros(1, dtype=torch.int32, device="cuda")
    rows = (1 << 32) // (32 * 128) + 9  # caches of 4.3 GB
    (kc, vc), (ks, vs) = cache(rows, 32)
    none = values(1, 32, torch.bfloat16, 6)[:0]
    fsx.cache_write(none, none, None, kc, vc, ks, vs, status)
    k, v = values(5, 32, torch.bfloat16, 7), values(5, 32, torch.bfloat16, 8)
    at = torch.arange(rows - 5, rows, device="cuda")
    fsx.cache_write(k, v, at, kc, vc, ks, vs, status)
    a, b = torch.empty_like(k, dtype=torch.float32), torch.empty_like(v, dtype=torch.float32)
    fsx.cache_read(kc, vc, ks, vs, at, a, b, status)
    assert int(status) == fsx.FSX_OK
    for x, got in ((k, a), (v, b)):
        want, scale = llm_oracle.cache_write(to64(x))
        assert np.array_equal(to64(got), want * scale[..., None])
    assert (kc.view(torch.uint8)[:-5] == 0x55).all()


def test_rows_that_repeat_leave_the_others_alone():
    """Destinations have to be distinct; where they are not, only the row that is named twice is unspecified."""
    n, heads = 64, 3
    k, v = values(n, heads, torch.bfloat16, 9), values(n, heads, torch.bfloat16, 10)
    k[1::2] *= 2.0 ** 40
    v[1::2] *= 2.0 ** -40
    rows = torch.arange(n, device="cuda") + 2
    rows[[5, 6, 30, 63]] = 40  # beside its own writer, row 38
    (kc, vc), (ks, vs) = cache(n + 8, heads)
    status = torch.zeros(1, dtype=torch.int32, device="cuda")
    fsx.cache_write(k, v, rows, kc, vc, ks, vs, status)
    assert int(status) == fsx.FSX_OK
    once = [i for i in range(n) if int(rows[i]) != 40]
    at = rows[once]
    for x, c, s in ((k, kc, ks), (v, vc, vs)):
        want, scale = llm_oracle.cache_write(to64(x[once]))
        assert same(c.view(torch.uint8)[at].view(torch.float8_e4m3fn), want)
        assert np.array_equal(s[:, at].T.double().cpu().numpy(), scale)
        rest = torch.ones(n + 8, dtype=torch.bool, device="cuda")
        rest[rows] = False
        assert (c.view(torch.uint8)[rest] == 0x55).all() and (s[:, rest] == 7).all()
