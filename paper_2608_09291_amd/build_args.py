"""Build the Python binding's tensor checks (csrc/python) in-tree.

    python -m paper_2608_09291_amd.build_args

compiles ``csrc/python/us_kv_args.cpp`` with g++ against torch's headers and
links ``_kv_args.so`` next to this file. Host code only.
"""
from __future__ import annotations

import os
import subprocess
import sysconfig

PKG = os.path.dirname(os.path.abspath(__file__))
SOURCE = os.path.join(PKG, "csrc", "python", "us_kv_args.cpp")
LIB = os.path.join(PKG, "_kv_args.so")


def build() -> str:
    """Compile and link the module; returns its path."""
    import torch
    root = os.path.dirname(torch.__file__)
    include = [os.path.join(root, "include"), os.path.join(root, "include", "torch", "csrc", "api", "include"),
               sysconfig.get_paths()["include"]]
    libs = os.path.join(root, "lib")
    tmp = LIB + ".tmp"
    cmd = ["g++", "-O2", "-std=c++17", "-fPIC", "-shared", "-Wall",
           f"-D_GLIBCXX_USE_CXX11_ABI={int(torch._C._GLIBCXX_USE_CXX11_ABI)}",
           *[x for d in include for x in ("-isystem", d)], SOURCE, "-o", tmp, "-L", libs, "-lc10", "-ltorch_cpu", "-ltorch_python"]
    r = subprocess.run(cmd, capture_output=True, text=True)
    if r.returncode != 0:
        raise RuntimeError("compile failed:\n" + " ".join(cmd) + "\n" + r.stdout + r.stderr)
    os.replace(tmp, LIB)
    return LIB


if __name__ == "__main__":
    print(build())
