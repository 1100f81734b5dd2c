"""How vp_attend_new cuts its work, compiled with the host compiler and run on
the CPU (tests/line_invariants.cpp), and the refusals that need no GPU."""

import os
import shutil
import subprocess

import pytest

ROOT = os.path.dirname(os.path.dirname(os.path.abspath(__file__)))
CUDA_INC = os.path.join(os.environ.get("CUDA_HOME", "/usr/local/cuda"), "include")


def test_line_invariants(tmp_path):
    cxx = shutil.which("g++")
    if cxx is None or not os.path.exists(os.path.join(CUDA_INC, "cuda.h")):
        pytest.skip("needs g++ and the CUDA headers")
    exe = tmp_path / "line_invariants"
    subprocess.run([cxx, "-std=c++17", "-O2", "-I", os.path.join(ROOT, "paper_2605_31457_gb300", "csrc"),
                    "-I", CUDA_INC, os.path.join(ROOT, "tests", "line_invariants.cpp"), "-o", str(exe)],
                   check=True, capture_output=True, text=True)
    r = subprocess.run([str(exe)], capture_output=True, text=True, timeout=120)
    assert r.returncode == 0, r.stdout + r.stderr
    assert "0 violations" in r.stdout


def test_refusals_without_a_context(lib):
    assert lib.lib.vp_reserve_new(None, 1, 0) == lib.VP_ERR_NOT_INITIALIZED
    assert lib.lib.vp_attend_new(None, 1, 1, *([None] * 11)) == lib.VP_ERR_NOT_INITIALIZED
    assert lib.lib.vp_evict(None, 1, *([None] * 9), 0, None, None) == lib.VP_ERR_NOT_INITIALIZED
