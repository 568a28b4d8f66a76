"""Host-side check of the drafted trees' work plan: compiles tests/tree_plan_check.cpp against the package header with g++
and runs it; and the workspaces' sizes through the C ABI."""
import os
import shutil
import subprocess
import tempfile

import numpy as np
import pytest

import paper_2608_07915_amd as S

ROOT = os.path.dirname(os.path.dirname(os.path.abspath(__file__)))
CSRC = os.path.join(ROOT, "paper_2608_07915_amd", "csrc")


@pytest.mark.skipif(shutil.which("g++") is None, reason="g++ not available")
def test_tree_plan():
    with tempfile.TemporaryDirectory() as d:
        exe = os.path.join(d, "tree_plan_check")
        subprocess.run(["g++", "-std=c++17", "-O2", "-Wall", f"-I{CSRC}", os.path.join(ROOT, "tests", "tree_plan_check.cpp"),
                        "-o", exe], check=True)
        r = subprocess.run([exe], capture_output=True, text=True, timeout=120)
        assert r.returncode == 0 and r.stdout.strip() == "OK", r.stdout + r.stderr


@pytest.mark.parametrize("batch,new,q,kv", [(4096, 4, 32, 8), (16384, 2, 32, 8), (512, 1, 8, 8), (1000, 8, 28, 4), (3, 1, 16, 1)])
def test_tree_workspace_by_the_rows_there_are(batch, new, q, kv):
    """Rows of 136 floats: a sequence's on a KV head in whole units of 16, 32 or 64, and the card's workgroups' (1024 of 16,
    or 512 of 32 or 64, and one more of each KV head)."""
    rows = new * (q // kv)
    unit = 16 if rows <= 16 else 32 if rows <= 32 else 64
    held = batch * kv * (-(-rows // unit) * unit) + (1024 + kv) * max(16, unit // 2) + kv * unit
    assert S.spectra_paged_tree_attention_workspace_bytes(batch, batch * new, q, kv, new, 1000) <= 136 * 4 * held + (1 << 20)


def test_workspaces_serve_every_smaller_call_of_as_many_heads():
    """What the header promises of the calls on trees, selections and lists: counts of tokens, sequences, slots and blocks in
    any combination, heads as they are."""
    rng = np.random.default_rng(0)
    pick = lambda hi: int(np.exp(rng.uniform(0, np.log(hi + 1))))  # noqa: E731
    for _ in range(3000):
        kv, n_qh = pick(300), pick(16)
        most = (1 << 21) // (kv * n_qh)
        batch, new, max_new, tokens, blocks = pick(16384), pick(most), pick(64), pick(1 << 21), pick(4096)
        b, n, m, t, k = pick(batch), pick(new), pick(max_new), pick(tokens), pick(blocks)
        q = kv * n_qh
        for call, large, small in ((S.spectra_paged_tree_attention_workspace_bytes, (batch, new, q, kv, max_new, tokens), (b, n, q, kv, m, t)),
                                   (S.spectra_paged_select_workspace_bytes, (new, q, kv, tokens), (n, q, kv, t)),
                                   (S.spectra_paged_sparse_attention_workspace_bytes, (new, q, kv, blocks), (n, q, kv, k))):
            assert 0 < call(*small) <= call(*large), (call.__name__, large, small)
