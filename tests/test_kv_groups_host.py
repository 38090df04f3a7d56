"""Where shared attention looks for a row's part over the common keys (paper_2608_09291_amd/csrc/us_kv_rules.h), compiled
for the host: inside of what the group's rows have left, whatever the tables of sequences and groups hold."""
import os
import shutil
import subprocess

import pytest

ROOT = os.path.dirname(os.path.dirname(os.path.abspath(__file__)))


def test_a_row_is_one_of_its_groups_or_none(tmp_path):
    if shutil.which("g++") is None:
        pytest.skip("g++ not available")
    exe = str(tmp_path / "kv_groups_check")
    r = subprocess.run(["g++", "-std=c++17", "-O1", "-fsanitize=undefined", "-fno-sanitize-recover=all", "-I",
                        os.path.join(ROOT, "paper_2608_09291_amd", "csrc"), os.path.join(ROOT, "tests", "kv_groups_check.cpp"),
                        "-o", exe], capture_output=True, text=True)
    assert r.returncode == 0, r.stderr[-2000:]
    r = subprocess.run([exe], capture_output=True, text=True, timeout=120)
    assert r.returncode == 0 and r.stdout.strip() == "ok", r.stdout + r.stderr
