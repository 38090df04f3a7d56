"""Registers of the key/value cache's kernels (host only: compiles to gfx950 assembly)."""
import concurrent.futures as cf
import os
import re
import subprocess

import pytest

from paper_2608_09291_amd import build

UNITS = ("us_kv_store", "us_kv_decode", "us_kv_prompt", "us_kv_evict")


@pytest.fixture(scope="module")
def kernels(tmp_path_factory):
    if not os.path.exists(build.HIPCC):
        pytest.skip("hipcc not available")
    tmp = tmp_path_factory.mktemp("kv_res")

    def compile_unit(u):
        out = str(tmp / (u + ".s"))
        flags = [f for f in build.hip_flags(u + ".hip") if f != "-fPIC"]
        r = subprocess.run([build.HIPCC, *flags, "-I", build.CSRC, "--cuda-device-only", "-S",
                            os.path.join(build.CSRC, u + ".hip"), "-o", out], capture_output=True, text=True)
        assert r.returncode == 0, r.stderr[-2000:]
        return open(out).read()

    found = {}
    with cf.ThreadPoolExecutor(max_workers=4) as ex:
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
    for name, per in (("us_kv_append_kernel", 2), ("us_kv_read_kernel", 2), ("us_kv_decode_kernel", 1),
                      ("us_kv_prompt_kernel", 1), ("us_kv_join_kernel", 1), ("us_kv_weights_kernel", 1)):
        got = _of(kernels, name)
        assert {k[:2] for k in got} == {(w, t) for w in widths for t in types} and len(got) == 15 * per, name
    assert set(_of(kernels, "us_kv_move_kernel")) == {(w,) for w in widths}


def test_registers_leave_the_waves_that_the_kernels_count_on(kernels):
    for (w, t, *_), (vgpr, _) in _of(kernels, "us_kv_decode_kernel").items():
        assert vgpr <= (256 if w <= 4 else 512), (w, t)          # two wavefronts per SIMD, or one
    for (w, t, waves), (vgpr, _) in _of(kernels, "us_kv_prompt_kernel").items():
        assert waves == (8 if w <= 4 else 4)
        assert vgpr <= (256 if waves == 8 else 512), (w, t)


def test_nothing_spills_but_the_widest_float32_prompt(kernels):
    spilled = {k for k, (_, scratch) in kernels.items() if scratch}
    assert all("us_kv_prompt_kernelILi8ELi0E" in k for k in spilled), spilled
