"""Host checks of the prompt and 8-bit cache operators: what they refuse before anything is enqueued (no GPU needed)."""
from __future__ import annotations

import os

import pytest
import torch

from paper_2607_15621_gb300 import fsx

FAKE = 1 << 20  # never dereferenced: every case fails host validation, or has nothing to do


@pytest.fixture(scope="module")
def lib():
    if not os.path.exists(fsx.LIB_PATH):
        from paper_2607_15621_gb300 import build
        build.build()
    return fsx.lib()


PROMPT = dict(q=FAKE, qs=512, k=FAKE, v=FAKE, kvs=256, dt=fsx.FSX_BF16, qo=FAKE, ko=FAKE, B=2, qr=10, kr=10, H=4, Hk=2,
              D=128, causal=1, out=FAKE, lse=None, status=FAKE, stream=None)
TREE = dict(q=FAKE, qs=512, kn=FAKE, vn=FAKE, ns=256, dt=fsx.FSX_BF16, no=FAKE, mask=FAKE, nr=10, kc=FAKE, vc=FAKE, ks=FAKE,
            vs=FAKE, cdt=fsx.FSX_E4M3, cr=100, starts=None, off=FAKE, B=2, H=4, Hk=2, D=128, out=FAKE, lse=None, ws=FAKE,
            wsb=1 << 40, status=FAKE, stream=None)
CACHE = dict(k=FAKE, v=FAKE, kvs=256, dt=fsx.FSX_BF16, rows=FAKE, n=5, H=2, D=128, kc=FAKE, vc=FAKE, ks=FAKE, vs=FAKE, cr=100,
             status=FAKE, stream=None)
READ = ["kc", "vc", "ks", "vs", "cr", "rows", "n", "H", "D", "k", "v", "kvs", "dt", "status", "stream"]
BAD, UNS = fsx.FSX_ERR_INVALID_ARG, fsx.FSX_ERR_UNSUPPORTED


@pytest.mark.parametrize("over,code", [
    (dict(q=None), BAD), (dict(k=None), BAD), (dict(v=None), BAD), (dict(qo=None), BAD), (dict(ko=None), BAD),
    (dict(out=None), BAD), (dict(status=None), BAD), (dict(dt=fsx.FSX_F32), BAD), (dict(dt=fsx.FSX_E4M3), BAD),
    (dict(dt=9), BAD), (dict(B=0), BAD), (dict(B=1025), BAD), (dict(qr=-1), BAD), (dict(kr=-1), BAD), (dict(qr=1 << 31), UNS),
    (dict(H=3), BAD), (dict(H=0), BAD), (dict(Hk=0), BAD), (dict(H=130, Hk=2, qs=130 * 128), UNS), (dict(D=64), UNS),
    (dict(causal=2), BAD), (dict(qs=511), BAD), (dict(qs=516), BAD), (dict(kvs=255), BAD), (dict(kvs=260), BAD),
    (dict(q=FAKE + 8), BAD), (dict(k=FAKE + 2), BAD), (dict(v=FAKE + 4), BAD), (dict(out=FAKE + 8), BAD),
])
def test_prompt_attention_refuses(lib, over, code):
    assert lib.fsx_prompt_attention(*dict(PROMPT, **over).values()) == code
    assert fsx.last_error()


@pytest.mark.parametrize("over,code", [
    (dict(q=None), BAD), (dict(kn=None), BAD), (dict(vn=None), BAD), (dict(no=None), BAD), (dict(mask=None), BAD),
    (dict(kc=None), BAD), (dict(vc=None), BAD), (dict(ks=None), BAD), (dict(vs=None), BAD), (dict(off=None), BAD),
    (dict(out=None), BAD), (dict(status=None), BAD), (dict(ws=None), BAD), (dict(ws=FAKE + 16), BAD), (dict(wsb=16), BAD),
    (dict(dt=fsx.FSX_F32), BAD), (dict(cdt=fsx.FSX_F16), BAD), (dict(cdt=fsx.FSX_F32), BAD), (dict(B=0), BAD),
    (dict(B=1025), BAD), (dict(nr=-1), BAD), (dict(cr=-1), BAD), (dict(cr=1 << 31), UNS), (dict(H=3), BAD), (dict(D=64), UNS),
    (dict(H=130, Hk=2, qs=130 * 128), UNS), (dict(qs=504), BAD), (dict(ns=252), BAD), (dict(kc=FAKE + 8), BAD),
    (dict(vn=FAKE + 8), BAD),
])
def test_tree_attention_refuses(lib, over, code):
    assert lib.fsx_tree_attention(*dict(TREE, **over).values()) == code
    assert fsx.last_error()


@pytest.mark.parametrize("over,code", [
    (dict(k=None), BAD), (dict(v=None), BAD), (dict(kc=None), BAD), (dict(vc=None), BAD), (dict(ks=None), BAD),
    (dict(vs=None), BAD), (dict(status=None), BAD), (dict(dt=fsx.FSX_E4M3), BAD), (dict(n=-1), BAD), (dict(cr=-1), BAD),
    (dict(n=1 << 31), UNS), (dict(H=0), BAD), (dict(D=64), UNS), (dict(kvs=248), BAD), (dict(kvs=260), BAD),
    (dict(rows=None, n=101), BAD), (dict(k=FAKE + 8), BAD), (dict(vc=FAKE + 8), BAD),
])
def test_cache_write_and_read_refuse(lib, over, code):
    a = dict(CACHE, **over)
    assert lib.fsx_cache_write_e4m3(*a.values()) == code
    assert fsx.last_error()
    assert lib.fsx_cache_read_e4m3(*[a[n] for n in READ]) == code
    assert fsx.last_error()


def test_prompt_attention_refuses_more_rows_than_it_counts(lib):
    for over in (dict(qr=(1 << 30) - 100), dict(qr=(1 << 31) - 1, H=4096, Hk=4096, qs=4096 * 128, kvs=4096 * 128)):
        assert lib.fsx_prompt_attention(*dict(PROMPT, **over).values()) == UNS
        assert fsx.last_error()


def test_tree_attention_refuses_more_rows_than_it_counts(lib):
    over = dict(nr=(1 << 31) - 1, H=64, Hk=64, qs=64 * 128, ns=64 * 128)
    assert lib.fsx_tree_attention(*dict(TREE, **over).values()) == UNS
    assert fsx.last_error()


def test_nothing_to_do_is_no_error(lib):
    assert lib.fsx_prompt_attention(*dict(PROMPT, qr=0, q=None, out=None).values()) == fsx.FSX_OK
    assert lib.fsx_tree_attention(*dict(TREE, nr=0, q=None, out=None).values()) == fsx.FSX_OK
    assert lib.fsx_cache_write_e4m3(*dict(CACHE, n=0, k=None).values()) == fsx.FSX_OK


def test_workspace_size(lib):
    assert fsx.tree_attention_workspace_bytes(1, 1, 1, 1) >= 256
    assert fsx.tree_attention_workspace_bytes(0, 1, 1, 1) == 0
    assert fsx.tree_attention_workspace_bytes(1, 1, 1, 2) == 0


@pytest.mark.parametrize("B,heads,kv_heads", [(1, 32, 32), (1, 64, 1), (3, 8, 2), (16, 32, 8), (128, 4, 1), (1024, 32, 32)])
def test_workspace_serves_fewer_new_rows(lib, B, heads, kv_heads):
    sizes = [fsx.tree_attention_workspace_bytes(B, r, heads, kv_heads) for r in [*range(0, min(64 * B, 600)), 64 * B]]
    assert sizes == sorted(sizes)


def test_binding_refuses_tensors_that_do_not_fit():
    z = lambda *s, dtype=torch.bfloat16: torch.zeros(*s, dtype=dtype)
    off, st = z(3, dtype=torch.int64), z(1, dtype=torch.int32)
    q, k, out = z(5, 4, 128), z(5, 2, 128), z(5, 4, 128)
    bad = [dict(q=z(5, 4, 128, dtype=torch.float16)), dict(k=z(5, 2, 64)), dict(v=z(4, 2, 128)), dict(out=z(5, 128, 4).transpose(1, 2)),
           dict(q_offsets=off.int()), dict(kv_offsets=z(4, dtype=torch.int64)), dict(lse=z(5, 4, dtype=torch.float32)),
           dict(k=z(5, 128, 2).transpose(1, 2)), dict(q=z(5, 4, 128, dtype=torch.int32))]
    for over in bad:
        a = dict(dict(q=q, k=k, v=k, q_offsets=off, kv_offsets=off, out=out, status=st), **over)
        with pytest.raises(fsx.FsxError):
            fsx.prompt_attention(**a)
    cache, scale = z(9, 2, 128, dtype=torch.uint8), z(2, 9, dtype=torch.float32)
    for over in [dict(k_cache=z(9, 2, 128)), dict(k_scale=z(9, 2, dtype=torch.float32)), dict(rows=off), dict(k=z(5, 3, 128))]:
        a = dict(dict(k=k, v=k, rows=None, k_cache=cache, v_cache=cache, k_scale=scale, v_scale=scale, status=st), **over)
        with pytest.raises(fsx.FsxError):
            fsx.cache_write(**a)
    for over in [dict(mask=z(4, dtype=torch.int64)), dict(k_scale=None), dict(starts=off), dict(offsets=z(2, dtype=torch.int64)),
                 dict(k_cache=z(9, 3, 128, dtype=torch.uint8))]:
        a = dict(dict(q=q, k_new=k, v_new=k, new_offsets=off, mask=z(5, dtype=torch.int64), k_cache=cache, v_cache=cache,
                      offsets=off, out=out, status=st, workspace=z(256, dtype=torch.uint8), k_scale=scale, v_scale=scale), **over)
        with pytest.raises(fsx.FsxError):
            fsx.tree_attention(**a)


def test_binding_asks_for_one_stride_only_where_it_means_something():
    k = torch.zeros(5, 128)[:, None, :]  # one kv head: its stride may be anything
    assert fsx._alike(k.clone(), k.expand(5, 1, 128).as_strided((5, 1, 128), (128, 0, 1)))
    assert fsx._alike(torch.zeros(1, 2, 128), torch.zeros(1, 6, 128)[:, :2])
    assert not fsx._alike(torch.zeros(5, 2, 128), torch.zeros(5, 6, 128)[:, :2])
    assert not fsx._alike(torch.zeros(5, 128, 2).transpose(1, 2), torch.zeros(5, 2, 128))
