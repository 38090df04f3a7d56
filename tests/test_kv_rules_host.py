"""What the key/value cache's attention kernels decide by whole numbers (paper_2608_09291_amd/csrc/us_kv_rules.h),
compiled for the host: the order in which blocks pass through the LDS stages of the prompt kernel,
and the range of keys that a query sees."""
import os
import shutil
import subprocess

import pytest

ROOT = os.path.dirname(os.path.dirname(os.path.abspath(__file__)))


@pytest.fixture(scope="module")
def check(tmp_path_factory):
    if shutil.which("g++") is None:
        pytest.skip("g++ not available")
    exe = str(tmp_path_factory.mktemp("kv_rules") / "kv_rules_check")
    r = subprocess.run(["g++", "-std=c++17", "-O1", "-fsanitize=undefined", "-fno-sanitize-recover=all", "-I",
                        os.path.join(ROOT, "paper_2608_09291_amd", "csrc"), os.path.join(ROOT, "tests", "kv_rules_check.cpp"),
                        "-o", exe], capture_output=True, text=True)
    assert r.returncode == 0, r.stderr[-2000:]

    def run(name):
        r = subprocess.run([exe, name], capture_output=True, text=True, timeout=120)
        assert r.returncode == 0 and r.stdout.strip() == "ok", r.stdout + r.stderr
    return run


def test_no_stage_is_overwritten_while_it_may_be_read(check):
    check("stages")


def test_ranges_of_keys(check):
    check("masks")
