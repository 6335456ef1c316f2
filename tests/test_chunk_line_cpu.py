"""The counts behind the plan of many drafted rows, on the CPU: ``csrc/chunk_line.h``, which the kernel uses, is compiled with
``tests/cpp/chunk_line_check.cpp`` and compared with 128-bit sums up to the most that the entry point accepts."""
from __future__ import annotations

import os
import shutil
import subprocess
import tempfile

import pytest

ROOT = os.path.dirname(os.path.dirname(os.path.abspath(__file__)))
CSRC = os.path.join(ROOT, "paper_2607_15621_gb300", "csrc")


@pytest.mark.skipif(shutil.which("g++") is None, reason="needs a host C++ compiler")
def test_chunks_are_counted_without_wrapping():
    with tempfile.TemporaryDirectory() as tmp:
        exe = os.path.join(tmp, "chunk_line_check")
        subprocess.run(["g++", "-std=c++17", "-O1", "-I", CSRC, os.path.join(ROOT, "tests", "cpp", "chunk_line_check.cpp"),
                        "-o", exe], check=True, capture_output=True, text=True)
        res = subprocess.run([exe], capture_output=True, text=True, timeout=60)
    assert res.returncode == 0, res.stdout + res.stderr
    assert res.stdout == "ok 32\n"
