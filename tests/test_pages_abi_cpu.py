"""Host checks of the operators over a cache in pages: what they refuse before anything is enqueued (no GPU needed)."""
from __future__ import annotations

import ctypes
import math
import os

import pytest
import torch

from paper_2607_15621_gb300 import fsx

FAKE = 1 << 20  # never dereferenced: every case fails host validation, or has nothing to do
BAD, UNS = fsx.FSX_ERR_INVALID_ARG, fsx.FSX_ERR_UNSUPPORTED


@pytest.fixture(scope="module")
def lib():
    if not os.path.exists(fsx.LIB_PATH):
        from paper_2607_15621_gb300 import build
        build.build()
    return fsx.lib()


def ints(*v):
    return (ctypes.c_int * 64)(*v)


def doubles(*v):
    return (ctypes.c_double * 64)(*v)


ROTARY = dict(q=FAKE, qs=512, k=FAKE, v=FAKE, kvs=256, dt=fsx.FSX_BF16, pos=FAKE, axes=2, axis=ints(), rate=doubles(), layout=0, n=5,
              H=4, Hk=2, D=128, qo=FAKE, qos=512, ko=FAKE, kos=256, rows=FAKE, kc=FAKE, vc=FAKE, ks=FAKE, vs=FAKE, cdt=fsx.FSX_E4M3,
              cr=100, status=FAKE, stream=None)
PAGED = dict(q=FAKE, qs=512, dt=fsx.FSX_BF16, kc=FAKE, vc=FAKE, ks=FAKE, vs=FAKE, cdt=fsx.FSX_E4M3, cr=160, P=16, table=FAKE, width=7,
             len=FAKE, B=2, picked=None, np=0, H=4, Hk=2, D=128, out=FAKE, lse=None, ws=FAKE, wsb=1 << 40, status=FAKE, stream=None)
BOUNDS = dict(kc=FAKE, ks=FAKE, cdt=fsx.FSX_E4M3, cr=160, P=16, table=FAKE, width=7, len=FAKE, start=None, B=2, Hk=2, D=128, b=FAKE,
              bs=FAKE, status=FAKE, stream=None)
SELECT = dict(q=FAKE, qs=512, dt=fsx.FSX_BF16, b=FAKE, bs=FAKE, cr=160, P=16, table=FAKE, width=7, len=FAKE, B=2, H=4, Hk=2, D=128,
              first=1, last=1, np=4, picked=FAKE, status=FAKE, stream=None)
STEP = dict(table=FAKE, len=FAKE, refs=FAKE, Bin=3, source=FAKE, new=FAKE, B=2, nr=10, width=7, n=20, P=16, to=FAKE + 64, lo=FAKE + 64,
            ro=FAKE, rows=FAKE, pairs=FAKE, npairs=FAKE, status=FAKE, stream=None)
COMPACT = dict(table=FAKE, len=FAKE, refs=FAKE, B=2, width=7, n=20, P=16, to=FAKE, ro=FAKE, pairs=FAKE, mp=10, npairs=FAKE,
               status=FAKE, stream=None)


def planes(n=1, base=FAKE, page_bytes=4096, stride=0, segments=1):
    return (fsx.PagePlane * n)(*[fsx.PagePlane(base, page_bytes, stride, segments) for _ in range(n)])


COPY = dict(planes=planes(), np=1, n=20, pairs=FAKE, npairs=FAKE, mp=10, status=FAKE, stream=None)


@pytest.mark.parametrize("over,code", [
    (dict(q=None), BAD), (dict(qo=None), BAD), (dict(k=None), BAD), (dict(v=None), BAD), (dict(q=None, qo=None, k=None), BAD),
    (dict(pos=None), BAD), (dict(axis=None), BAD), (dict(rate=None), BAD), (dict(status=None), BAD), (dict(dt=fsx.FSX_F32), BAD),
    (dict(dt=fsx.FSX_E4M3), BAD), (dict(axes=0), BAD), (dict(axes=5), BAD), (dict(axis=ints(2)), BAD), (dict(axis=ints(-1)), BAD),
    (dict(rate=doubles(math.nan)), BAD), (dict(rate=doubles(0, math.inf)), BAD), (dict(rate=doubles(-2.0 ** 20 - 1)), BAD),
    (dict(layout=2), BAD), (dict(n=-1), BAD), (dict(n=1 << 31), UNS), (dict(H=3), BAD), (dict(D=64), UNS), (dict(qs=504), BAD),
    (dict(kvs=260), BAD), (dict(qos=511), BAD), (dict(kos=128), BAD), (dict(q=FAKE + 8), BAD), (dict(ko=FAKE + 8), BAD),
    (dict(vc=None), BAD), (dict(kc=None), BAD), (dict(ks=None), BAD), (dict(cdt=fsx.FSX_F16), BAD), (dict(cr=-1), BAD),
    (dict(cr=1 << 31), UNS), (dict(rows=None, n=101), BAD), (dict(kc=FAKE + 8), BAD), (dict(ko=None, kc=None, vc=None), BAD),
])
def test_rotary_refuses(lib, over, code):
    assert lib.fsx_rotary(*dict(ROTARY, **over).values()) == code
    assert fsx.last_error()


PAGES = [(dict(table=None), BAD), (dict(len=None), BAD), (dict(B=0), BAD), (dict(B=1025), BAD), (dict(P=8), UNS), (dict(P=48), UNS),
         (dict(P=2048), UNS), (dict(P=0), UNS), (dict(width=0), BAD), (dict(width=1 << 27), UNS), (dict(cr=161), BAD), (dict(cr=-16), BAD),
         (dict(cr=1 << 31), UNS), (dict(D=64), UNS), (dict(status=None), BAD), (dict(Hk=0), BAD)]


@pytest.mark.parametrize("over,code", PAGES + [
    (dict(q=None), BAD), (dict(kc=None), BAD), (dict(vc=None), BAD), (dict(ks=None), BAD), (dict(vs=None), BAD), (dict(out=None), BAD),
    (dict(ws=None), BAD), (dict(ws=FAKE + 16), BAD), (dict(wsb=16), BAD), (dict(dt=fsx.FSX_F32), BAD), (dict(cdt=fsx.FSX_F16), BAD),
    (dict(H=3), BAD), (dict(H=130, Hk=2, qs=130 * 128), UNS), (dict(qs=504), BAD), (dict(q=FAKE + 8), BAD), (dict(out=FAKE + 8), BAD),
    (dict(kc=FAKE + 8), BAD), (dict(picked=FAKE, np=0), BAD), (dict(picked=FAKE, np=4097), BAD),
])
def test_paged_attention_refuses(lib, over, code):
    assert lib.fsx_paged_attention(*dict(PAGED, **over).values()) == code
    assert fsx.last_error()


@pytest.mark.parametrize("over,code", PAGES + [
    (dict(kc=None), BAD), (dict(ks=None), BAD), (dict(cdt=fsx.FSX_F32), BAD), (dict(b=None), BAD), (dict(bs=None), BAD),
    (dict(b=FAKE + 8), BAD), (dict(kc=FAKE + 8), BAD), (dict(width=1 << 20, Hk=1024), UNS),
])
def test_page_bounds_refuse(lib, over, code):
    assert lib.fsx_page_bounds(*dict(BOUNDS, **over).values()) == code
    assert fsx.last_error()


@pytest.mark.parametrize("over,code", PAGES + [
    (dict(q=None), BAD), (dict(dt=fsx.FSX_F32), BAD), (dict(b=None), BAD), (dict(bs=None), BAD), (dict(picked=None), BAD),
    (dict(width=32769), UNS), (dict(np=0), BAD), (dict(np=4097), BAD), (dict(first=-1), BAD), (dict(last=-1), BAD),
    (dict(first=3, last=2), BAD), (dict(qs=504), BAD), (dict(cr=0), BAD),
])
def test_page_select_refuses(lib, over, code):
    assert lib.fsx_page_select(*dict(SELECT, **over).values()) == code
    assert fsx.last_error()


@pytest.mark.parametrize("over,code", [
    (dict(table=None), BAD), (dict(len=None), BAD), (dict(refs=None), BAD), (dict(new=None), BAD), (dict(to=None), BAD),
    (dict(lo=None), BAD), (dict(ro=None), BAD), (dict(rows=None), BAD), (dict(pairs=None), BAD), (dict(npairs=None), BAD),
    (dict(status=None), BAD), (dict(Bin=0), BAD), (dict(Bin=1025), BAD), (dict(B=0), BAD), (dict(B=1025), BAD), (dict(nr=-1), BAD),
    (dict(width=0), BAD), (dict(n=0), BAD), (dict(P=24), UNS), (dict(n=1 << 28), UNS), (dict(width=1 << 28), UNS),
    (dict(source=None), BAD), (dict(to=FAKE), BAD), (dict(lo=FAKE), BAD),
])
def test_pages_step_refuses(lib, over, code):
    assert lib.fsx_pages_step(*dict(STEP, **over).values()) == code
    assert fsx.last_error()


@pytest.mark.parametrize("over,code", [
    (dict(table=None), BAD), (dict(len=None), BAD), (dict(refs=None), BAD), (dict(to=None), BAD), (dict(ro=None), BAD),
    (dict(pairs=None), BAD), (dict(npairs=None), BAD), (dict(status=None), BAD), (dict(B=0), BAD), (dict(n=0), BAD),
    (dict(P=3), UNS), (dict(mp=9), BAD),
])
def test_pages_compact_refuses(lib, over, code):
    assert lib.fsx_pages_compact(*dict(COMPACT, **over).values()) == code
    assert fsx.last_error()


@pytest.mark.parametrize("over,code", [
    (dict(planes=None), BAD), (dict(np=0), BAD), (dict(np=513), BAD), (dict(n=0), BAD), (dict(pairs=None), BAD), (dict(npairs=None), BAD),
    (dict(pairs=FAKE + 4), BAD), (dict(mp=-1), BAD), (dict(status=None), BAD), (dict(planes=planes(base=None)), BAD), (dict(planes=planes(base=FAKE + 2)), BAD),
    (dict(planes=planes(page_bytes=0)), BAD), (dict(planes=planes(page_bytes=6)), BAD), (dict(planes=planes(segments=0)), BAD),
    (dict(planes=planes(segments=2, stride=4096 * 20 - 4)), BAD), (dict(planes=planes(segments=2, stride=4096 * 20 + 2)), BAD),
])
def test_pages_copy_refuses(lib, over, code):
    assert lib.fsx_pages_copy(*dict(COPY, **over).values()) == code
    assert fsx.last_error()


def test_nothing_to_do_is_no_error(lib):
    assert lib.fsx_rotary(*dict(ROTARY, n=0, pos=None).values()) == fsx.FSX_OK
    assert lib.fsx_pages_copy(*dict(COPY, mp=0, pairs=None).values()) == fsx.FSX_OK


def test_workspace_size(lib):
    assert fsx.paged_attention_workspace_bytes(1, 1, 1) >= 256
    assert fsx.paged_attention_workspace_bytes(0, 1, 1) == 0 and fsx.paged_attention_workspace_bytes(1, 1, 2) == 0
    assert fsx.paged_attention_workspace_bytes(1, 32, 8) == fsx.paged_attention_workspace_bytes(1024, 32, 8)


def z(*s, dtype=torch.bfloat16):
    return torch.zeros(*s, dtype=dtype)


def refuses(call, good, bad):
    for over in bad:
        with pytest.raises(fsx.FsxError):
            call(**dict(good, stream=0, **over))


def test_binding_refuses_tensors_that_do_not_fit():
    i64, i32, i8, f32, f16 = torch.int64, torch.int32, torch.int8, torch.float32, torch.float16
    st, cache, scale = z(1, dtype=i32), z(160, 2, 128, dtype=torch.uint8), z(2, 160, dtype=f32)
    table, lengths = z(5, 7, dtype=i32), z(5, dtype=i64)
    q, k = z(5, 4, 128), z(5, 2, 128)
    refuses(fsx.rotary, dict(q=q, k=k, positions=z(1, 5, dtype=i64), pairs=fsx.rotary_pairs(), status=st, q_out=q, k_out=k, v=k,
                             rows=z(5, dtype=i64), k_cache=cache, v_cache=cache, k_scale=scale, v_scale=scale),
            [dict(q_out=None), dict(q=None), dict(k=z(4, 2, 128)), dict(k=z(5, 2, 64)), dict(k=z(5, 2, 128, dtype=f16)),
             dict(k=z(5, 128, 2).transpose(1, 2)), dict(v=None), dict(v=z(5, 2, 256)[..., ::2]), dict(k_out=z(5, 3, 128)),
             dict(positions=z(1, 4, dtype=i64)), dict(positions=z(1, 5, dtype=i32)), dict(positions=z(5, dtype=i64)),
             dict(pairs=fsx.rotary_pairs((32, 32))), dict(rows=z(5, dtype=i32)), dict(rows=z(4, dtype=i64)), dict(k_scale=None),
             dict(k_scale=z(160, 2, dtype=f32)), dict(v_cache=None), dict(k_cache=None), dict(k_cache=z(160, 3, 128, dtype=torch.uint8)),
             dict(v_cache=z(160, 2, 128)), dict(k=None), dict(q=q.float(), q_out=q.float()), dict(status=st.long()),
             dict(status=None), dict(status=st[:0])])
    refuses(fsx.paged_attention, dict(q=q, k_cache=cache, v_cache=cache, table=table, lengths=lengths, page_rows=16, out=q, status=st,
                                      workspace=z(256, dtype=torch.uint8), k_scale=scale, v_scale=scale),
            [dict(q=z(5, 4, 64)), dict(out=z(5, 128, 4).transpose(1, 2)), dict(out=q.half()), dict(table=table.long()),
             dict(table=z(4, 7, dtype=i32)), dict(lengths=lengths.int()), dict(k_cache=z(160, 2, 128)), dict(k_scale=None),
             dict(picked=z(5, 4, 3, dtype=i32)), dict(picked=z(5, 2, 3, dtype=i64)), dict(lse=z(5, 4, dtype=f32)),
             dict(page_rows=17), dict()])  # the last: too small a workspace
    bounds, bs = z(10, 2, 2, 128, dtype=i8), z(2, 10, dtype=f32)
    refuses(fsx.page_bounds, dict(k_cache=cache, table=table, lengths=lengths, page_rows=16, bounds=bounds, bound_scale=bs, status=st,
                                  k_scale=scale),
            [dict(k_scale=None), dict(bounds=z(9, 2, 2, 128, dtype=i8)), dict(bounds=bounds.int()), dict(bound_scale=z(10, 2, dtype=f32)),
             dict(start=lengths.int()), dict(start=z(4, dtype=i64)), dict(page_rows=32), dict(page_rows=0), dict(k_cache=cache.int())])
    refuses(fsx.page_select, dict(q=q, bounds=bounds, bound_scale=bs, table=table, lengths=lengths, page_rows=16,
                                  picked=z(5, 2, 4, dtype=i32), status=st),
            [dict(picked=z(5, 4, 4, dtype=i32)), dict(picked=z(5, 2, 4, dtype=i64)), dict(first=5), dict(q=z(4, 4, 128)),
             dict(bounds=z(9, 2, 2, 128, dtype=i8)), dict(picked=z(5, 2, 0, dtype=i32))])
    refs = z(20, dtype=i32)
    refuses(fsx.pages_step, dict(table=table, lengths=lengths, refs=refs, new_offsets=z(4, dtype=i64), page_rows=16,
                                 table_out=z(3, 7, dtype=i32), lengths_out=z(3, dtype=i64), refs_out=refs, rows=z(9, dtype=i64),
                                 pairs=z(3, 2, dtype=i32), n_pairs=z(1, dtype=i32), status=st, source=z(3, dtype=i32)),
            [dict(source=None), dict(source=z(3, dtype=i64)), dict(new_offsets=z(3, dtype=i64)), dict(table_out=z(3, 8, dtype=i32)),
             dict(lengths_out=z(4, dtype=i64)), dict(refs_out=z(19, dtype=i32)), dict(pairs=z(2, 2, dtype=i32)), dict(rows=refs),
             dict(n_pairs=z(2, dtype=i32)), dict(page_rows=12)])
    refuses(fsx.pages_compact, dict(table=table, lengths=lengths, refs=refs, page_rows=16, table_out=table, refs_out=refs,
                                    pairs=z(10, 2, dtype=i32), n_pairs=z(1, dtype=i32), status=st),
            [dict(pairs=z(9, 2, dtype=i32)), dict(table_out=z(5, 8, dtype=i32)), dict(refs_out=refs.long())])
    planes_ = fsx.page_planes(16, [cache], [scale], [bounds], [bs])
    assert [(p.page_bytes, p.segment_stride, p.segments) for p in planes_.array] == [(4096, 0, 1), (64, 640, 2), (512, 0, 1), (4, 40, 2)]
    refuses(fsx.pages_copy, dict(planes=planes_, pairs=z(3, 2, dtype=i32), n_pairs=z(1, dtype=i32), status=st),
            [dict(pairs=z(3, 2, dtype=i64)), dict(pairs=z(6, dtype=i32)), dict(n_pairs=z(2, dtype=i32))])
    with pytest.raises(fsx.FsxError):
        fsx.page_planes(16, [cache], [z(2, 320, dtype=f32)])
    with pytest.raises(fsx.FsxError):
        fsx.page_planes(16)
    for page_rows, wrong in ((48, dict(caches=[cache])), (48, dict(scales=[scale])), (0, dict(caches=[cache])), (512, dict(caches=[cache])),
                             (16, dict(caches=[cache[:0]])), (16, dict(bounds=[bounds[:0]])), (16, dict(scales=[scale[0]])),
                             (16, dict(caches=[torch.zeros(())])), (16, dict(bound_scales=[bs[:0]]))):
        with pytest.raises(fsx.FsxError):  # parts of pages, no pages, too few axes, nothing of a page
            fsx.page_planes(page_rows, **wrong)


def test_binding_refuses_lists_of_no_pages_and_caches_of_no_rows():
    """Tensors of nothing have no memory: they must not be taken for ones that were not given."""
    i32, i64 = torch.int32, torch.int64
    st, cache, q, k = z(1, dtype=i32), z(160, 2, 128), z(5, 4, 128), z(5, 2, 128)
    with pytest.raises(fsx.FsxError) as e:
        fsx.paged_attention(q, cache, cache, z(5, 7, dtype=i32), z(5, dtype=i64), 16, q, st, z(1, dtype=torch.uint8),
                            picked=z(5, 2, 0, dtype=i32), stream=0)
    assert "picked" in str(e.value)
    with pytest.raises(fsx.FsxError) as e:
        fsx.rotary(q, k, z(1, 5, dtype=i64), fsx.rotary_pairs(), st, q_out=q, k_out=k, v=k, rows=z(5, dtype=i64), k_cache=cache[:0],
                   v_cache=cache[:0], stream=0)
    assert "caches" in str(e.value)


def test_rotary_pairs():
    p = fsx.rotary_pairs((16, 24, 24))
    assert list(p.axis) == [0] * 16 + [1] * 24 + [2] * 24 and p.n_axes == 3 and p.layout == fsx.FSX_ROTARY_HALVES
    assert list(p.rate) == [10000.0 ** -(j / 64) for j in range(64)]
    own = fsx.rotary_pairs((32, 32), base=100.0, per_axis=True, adjacent=True)
    assert list(own.rate) == [100.0 ** -(i / 32) for i in range(32)] * 2 and own.layout == fsx.FSX_ROTARY_ADJACENT
    for bad in ((32, 31), (65, -1)):
        with pytest.raises(fsx.FsxError):
            fsx.rotary_pairs(bad)
    with pytest.raises(fsx.FsxError):
        fsx.RotaryPairs([0] * 63, [1.0] * 64)
