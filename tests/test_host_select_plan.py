"""Host-side check of the block selection's work plan: compiles tests/select_plan_check.cpp against the package header with
g++ and runs it; and the workspaces' sizes through the C ABI."""
import os
import shutil
import subprocess
import tempfile

import pytest

import paper_2608_07915_amd as S

ROOT = os.path.dirname(os.path.dirname(os.path.abspath(__file__)))
CSRC = os.path.join(ROOT, "paper_2608_07915_amd", "csrc")


@pytest.mark.skipif(shutil.which("g++") is None, reason="g++ not available")
def test_select_plan():
    with tempfile.TemporaryDirectory() as d:
        exe = os.path.join(d, "select_plan_check")
        subprocess.run(["g++", "-std=c++17", "-O2", "-Wall", f"-I{CSRC}", os.path.join(ROOT, "tests", "select_plan_check.cpp"),
                        "-o", exe], check=True)
        r = subprocess.run([exe], capture_output=True, text=True, timeout=120)
        assert r.returncode == 0 and r.stdout.strip() == "OK", r.stdout + r.stderr


@pytest.mark.parametrize("tokens,q,kv,slots", [(65536, 32, 8, 131072), (65536, 32, 8, 1 << 20), (8192, 128, 8, 1 << 20),
                                               (128, 128, 8, 1 << 22), (2 ** 21, 1, 1, 1 << 20), (1, 32, 8, 1 << 30)])
def test_selection_of_any_size_keeps_some_scores_at_a_time(tokens, q, kv, slots):
    """At most 2^28 scores, or one token's; and a float for every query row and 2^15 more."""
    row = -(-slots // 2048) * 32
    most = max(1 << 28, q * row) + tokens * q + (1 << 15) + 64
    assert S.spectra_paged_select_workspace_bytes(tokens, q, kv, slots) <= 4 * most
