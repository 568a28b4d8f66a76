"""Host-side check of the paged attention's work plan: compiles tests/paged_plan_check.cpp
against the package header with g++ and runs it; and the workspace size through the C ABI."""
import os
import shutil
import subprocess
import tempfile

import pytest

import paper_2608_07915_amd as S

ROOT = os.path.dirname(os.path.dirname(os.path.abspath(__file__)))
CSRC = os.path.join(ROOT, "paper_2608_07915_amd", "csrc")


@pytest.mark.skipif(shutil.which("g++") is None, reason="g++ not available")
def test_paged_plan():
    with tempfile.TemporaryDirectory() as d:
        exe = os.path.join(d, "paged_plan_check")
        subprocess.run(["g++", "-std=c++17", "-O2", "-Wall", f"-I{CSRC}", os.path.join(ROOT, "tests", "paged_plan_check.cpp"),
                        "-o", exe], check=True)
        r = subprocess.run([exe], capture_output=True, text=True, timeout=120)
        assert r.returncode == 0 and r.stdout.strip() == "OK", r.stdout + r.stderr


def test_workspace_never_falls():
    need = S.spectra_paged_attention_workspace_bytes
    last = 0
    for n in (1, 5, 64, 500, 4096, 30000):
        b = need(8, 8 * n, 32, 8, n, 100000)
        assert b >= last and b % 256 == 0
        last = b
    # a decode step alone takes the scan's partials only
    assert need(64, 64, 32, 8, 1, 100000) < 1 << 23
    assert need(64, 64, 32, 8, 1, 2 ** 31) == 0 and need(64, 64, 34, 2, 1, 100) == 0
