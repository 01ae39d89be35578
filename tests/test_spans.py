"""Whether two strided tensors share memory, against the sets of their bytes (CPU)."""

import os
import shutil
import subprocess

import pytest

ROOT = os.path.dirname(os.path.dirname(os.path.abspath(__file__)))


def test_spans_against_sets_of_bytes(tmp_path):
    cc = shutil.which("g++")
    if cc is None:
        pytest.skip("no host compiler")
    exe = tmp_path / "span_check"
    include = os.path.join(ROOT, "paper_2609_30656_gb300", "csrc")
    source = os.path.join(ROOT, "tests", "native", "span_check.cpp")
    subprocess.run([cc, "-std=c++17", "-O1", "-Wall", "-Werror", "-I", include, source, "-o", str(exe)], check=True)
    wrong, sharing = map(int, subprocess.run([str(exe)], check=True, capture_output=True, text=True).stdout.split())
    assert wrong == 0 and 1000 < sharing < 99000
