"""How prompt attention deals its steps out to workgroups, gone through on the CPU with the kernels' own rules."""
import os
import shutil
import subprocess

import pytest

ROOT = os.path.dirname(os.path.dirname(os.path.abspath(__file__)))


def test_no_start_or_length_leads_outside(tmp_path):
    """Starts in any order, lengths and prefixes of every size: all parts and rows lie inside their arrays, and where starts
    ascend each step is taken once and joined."""
    gxx = shutil.which("g++")
    if not gxx:
        pytest.skip("g++ not available")
    out = str(tmp_path / "deal")
    res = subprocess.run([gxx, "-std=c++17", "-g", "-O2", "-fsanitize=address,undefined", "-fno-sanitize-recover=all",
                          "-D__HIP_PLATFORM_AMD__", "-I/opt/rocm/include", os.path.join(ROOT, "tests", "sanitize", "deal_paths.cpp"),
                          "-o", out], capture_output=True, text=True)
    assert res.returncode == 0, res.stderr
    res = subprocess.run([out], capture_output=True, text=True, timeout=300)
    assert res.returncode == 0, res.stdout[-3000:] + res.stderr[-3000:]
