"""Registers of the kernels around the key/value cache (host only: compiles to gfx950 assembly)."""
import concurrent.futures as cf
import os
import re
import subprocess

import pytest

from paper_2608_09291_amd import build

UNITS = ("us_kv_rotate", "us_kv_fork", "us_kv_choose", "us_kv_chosen", "us_kv_shared")


@pytest.fixture(scope="module")
def kernels(tmp_path_factory):
    if not os.path.exists(build.HIPCC):
        pytest.skip("hipcc not available")
    tmp = tmp_path_factory.mktemp("kv_more_res")

    def compile_unit(u):
        out = str(tmp / (u + ".s"))
        flags = [f for f in build.hip_flags(u + ".hip") if f != "-fPIC"]
        r = subprocess.run([build.HIPCC, *flags, "-I", build.CSRC, "--cuda-device-only", "-S",
                            os.path.join(build.CSRC, u + ".hip"), "-o", out], capture_output=True, text=True)
        assert r.returncode == 0, r.stderr[-2000:]
        return open(out).read()

    found = {}
    with cf.ThreadPoolExecutor(max_workers=5) as ex:
        for text in ex.map(compile_unit, UNITS):
            for m in re.finditer(r"\.amdhsa_kernel (\S+)(.*?)\.end_amdhsa_kernel", text, re.S):
                get = lambda key, body=m.group(2): int(re.search(r"\.amdhsa_%s (\d+)" % key, body).group(1))  # noqa: E731
                found[m.group(1)] = (get("next_free_vgpr"), get("private_segment_fixed_size"))
    return found


def _of(kernels, name):
    """{template numbers: (registers, scratch)} of a kernel."""
    got = {}
    for k, v in kernels.items():
        m = re.search(name + r"I((?:L[ib]\d+E)+)E", k)
        if m:
            got[tuple(int(x) for x in re.findall(r"L[ib](\d+)E", m.group(1)))] = v
    return got


def test_every_row_width_and_type_is_built(kernels):
    widths, types = (2, 3, 4, 6, 8), (0, 1, 2)
    both = {(w, t) for w in widths for t in types}
    for name in ("us_kv_chosen_kernel", "us_kv_shared_few_kernel", "us_kv_shared_join_kernel"):
        assert set(_of(kernels, name)) == both, name
    assert set(_of(kernels, "us_kv_choose_kernel")) == {(w, t, few) for w, t in both for few in (0, 1)}
    many = _of(kernels, "us_kv_shared_many_kernel")
    assert {k[1:3] for k in many} == both and len(many) == 2 * len(both)
    assert set(_of(kernels, "us_kv_summarise_kernel")) == {(w,) for w in widths}
    assert set(_of(kernels, "us_kv_rotate_kernel")) == {(t, n, v, a) for t in types for n in (4, 8, 16, 32) for v in (0, 1) for a in (0, 1)}


def test_registers_leave_the_waves_that_the_kernels_count_on(kernels):
    for name in ("us_kv_chosen_kernel", "us_kv_shared_few_kernel"):
        for (w, t), (vgpr, _) in _of(kernels, name).items():
            assert vgpr <= (256 if w <= 4 else 512), (name, w, t)             # two wavefronts per SIMD, or one
    for (_, w, t, waves), (vgpr, _) in _of(kernels, "us_kv_shared_many_kernel").items():
        assert waves == (8 if w <= 4 else 4)
        assert vgpr <= (256 if waves == 8 else 512), (w, t)
    for key, (vgpr, _) in _of(kernels, "us_kv_rotate_kernel").items():
        assert vgpr <= 102, key                                               # five wavefronts per SIMD
    for key, (vgpr, _) in _of(kernels, "us_kv_choose_kernel").items():
        assert vgpr <= 128, key                                               # two workgroups of eight per CU


def test_little_spills_but_in_the_widest_float32_prompt(kernels):
    spilled = {k: scratch for k, (_, scratch) in kernels.items() if scratch}
    assert all(re.search(r"us_kv_shared_many_kernelILi\dELi8ELi0E", k) or ("us_kv_shared_many" in k and s <= 8) for k, s in spilled.items()), spilled
