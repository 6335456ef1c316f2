"""The extension behind the operators over pages: tensors without memory, sizes beyond the 32 bits of the entry points (no GPU)."""
from __future__ import annotations

import mmap
import os
import subprocess
import sys
import textwrap

import pytest
import torch

from paper_2607_15621_gb300 import build, fsx

ROOT = os.path.dirname(os.path.dirname(os.path.abspath(__file__)))


@pytest.fixture(scope="module", autouse=True)
def built():
    if not os.path.exists(fsx.CALLS_PATH):
        build.build()


def test_a_tensor_without_memory_and_without_rows_is_refused():
    """torch throws where its memory is asked for, of a tensor of no elements only at the call itself."""
    code = textwrap.dedent("""
        import torch
        from paper_2607_15621_gb300 import fsx
        status, positions = torch.zeros(1, dtype=torch.int32), torch.zeros(1, 0, dtype=torch.int64)

        def call(q):
            try:
                fsx.rotary(q, None, positions, fsx.rotary_pairs(), status, q_out=q, stream=0)
            except fsx.FsxError:
                print("refused")
            return q

        torch.vmap(call)(torch.empty(2, 0, 4, 128, dtype=torch.bfloat16))
        torch.vmap(call)(torch.empty(2, 3, 4, 128, dtype=torch.bfloat16))
    """)
    done = subprocess.run([sys.executable, "-c", code], cwd=ROOT, capture_output=True, text=True, timeout=300)
    assert (done.returncode, done.stdout.split()) == (0, ["refused"] * 2), done.stderr[-2000:]


def wide(n, dtype):
    """[1, n] without memory behind it but for what is touched."""
    at = mmap.mmap(-1, n * dtype.itemsize, flags=mmap.MAP_PRIVATE | mmap.MAP_ANONYMOUS | getattr(mmap, "MAP_NORESERVE", 0x4000))
    return torch.frombuffer(at, dtype=dtype).view(1, n)


def test_sizes_beyond_32_bits_are_refused_not_cut():
    i32, i64, bf = torch.int32, torch.int64, torch.bfloat16
    z = lambda *s, dtype=bf: torch.zeros(*s, dtype=dtype)
    table, picked = wide((1 << 32) + 4, i32), wide((1 << 32) + 4, i32).view(1, 1, -1)
    q, cache, st, lengths = z(1, 4, 128), z(64, 1, 128), z(1, dtype=i32), z(1, dtype=i64)
    ws = z(fsx.paged_attention_workspace_bytes(1, 4, 1) + 256, dtype=torch.uint8)
    ws = ws[-ws.data_ptr() % 256:]
    bounds, scale, refs = z(4, 1, 2, 128, dtype=torch.int8), z(1, 4, dtype=torch.float32), z(4, dtype=i32)
    few = z(1, 4, dtype=i32)
    calls = [lambda: fsx.paged_attention(q, cache, cache, table, lengths, 16, q.clone(), st, ws, stream=0),
             lambda: fsx.paged_attention(q, cache, cache, few, lengths, 16, q.clone(), st, ws, picked=picked, stream=0),
             lambda: fsx.page_bounds(cache, table, lengths, 16, bounds, scale, st, stream=0),
             lambda: fsx.page_select(q, bounds, scale, table, lengths, 16, z(1, 1, 3, dtype=i32), st, stream=0),
             lambda: fsx.page_select(q, bounds, scale, few, lengths, 16, picked, st, stream=0)]
    many, long = table.view(-1, 1), wide((1 << 32) + 4, i64).view(-1)  # as many requests
    calls += [lambda: fsx.page_bounds(cache, many, long, 16, bounds, scale, st, stream=0),
              lambda: fsx.pages_compact(many, long, refs, 16, many, refs, z(2, 2, dtype=i32), st, st, stream=0),
              lambda: fsx.pages_step(many, long, refs, z(2, dtype=i64), 16, few[:, :1].contiguous(), lengths, refs, lengths, z(1, 2, dtype=i32),
                                     st, st, source=z(1, dtype=i32), stream=0)]
    for call in calls:
        with pytest.raises(fsx.FsxError) as e:
            call()
        assert e.value.status in (fsx.FSX_ERR_INVALID_ARG, fsx.FSX_ERR_UNSUPPORTED), e.value
