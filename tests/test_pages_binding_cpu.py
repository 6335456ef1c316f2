"""The extension behind the operators over pages: tensors without memory (no GPU)."""
from __future__ import annotations

import os
import subprocess
import sys
import textwrap

import pytest

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
