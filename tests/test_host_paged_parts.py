"""The calls of test_gpu_paged_parts.py are ones whose slots are split: compiles
tests/paged_parts_check.cpp against the package header with g++ and reads the plan."""
import os
import shutil
import subprocess

import pytest

from paged_cases import KV, SPLIT

ROOT = os.path.dirname(os.path.dirname(os.path.abspath(__file__)))
CSRC = os.path.join(ROOT, "paper_2608_07915_amd", "csrc")


@pytest.mark.skipif(shutil.which("g++") is None, reason="g++ not available")
def test_calls_are_split(tmp_path):
    exe = str(tmp_path / "parts")
    subprocess.run(["g++", "-std=c++17", "-O2", "-Wall", f"-I{CSRC}", os.path.join(ROOT, "tests", "paged_parts_check.cpp"), "-o", exe],
                   check=True)

    def plan(lens, new, n_qh):
        r = subprocess.run([exe, *map(str, (len(lens), sum(new), KV * n_qh, KV, max(new), max(lens), 16))], capture_output=True,
                           text=True, check=True)
        return [int(x) for x in r.stdout.split()]
    for name, (lens, new, n_qh) in {**SPLIT, "widths": ([2900, 64], [50, 20], 3), "far": ([2600], [40], 4)}.items():
        units, parts, slots, _ = plan(lens, new, n_qh)
        assert units > 0 and parts > 1, name
    _, parts, slots, _ = plan(*SPLIT["last_part_of_129"])
    assert 1409 - (parts - 1) * slots == 129
    _, parts, slots, _ = plan(*SPLIT["last_part_of_one"])
    assert 2305 - (parts - 1) * slots == 1
    assert plan([2600] * 130, [40] * 130, 4)[1] == 1


@pytest.mark.skipif(shutil.which("g++") is None, reason="g++ not available")
def test_units_and_chunks_of_any_sequences(tmp_path):
    exe = str(tmp_path / "units")
    subprocess.run(["g++", "-std=c++17", "-O2", "-Wall", f"-I{CSRC}", os.path.join(ROOT, "tests", "paged_units_check.cpp"), "-o", exe],
                   check=True)
    r = subprocess.run([exe], capture_output=True, text=True, timeout=120)
    assert r.returncode == 0 and r.stdout.strip() == "OK", r.stdout + r.stderr
