"""Builds libsamo.so (HIP, gfx950 only) and the binding's native argument marshalling in-tree."""
from __future__ import annotations

import concurrent.futures
import os
import subprocess
import sysconfig
import tempfile

PKG = os.path.dirname(os.path.abspath(__file__))
ROOT = os.path.dirname(PKG)
CSRC = os.path.join(PKG, "csrc")
LIB = os.path.join(PKG, "libsamo.so")
SOURCES = ["api.hip", "attention.hip", "attention_all.hip", "attention_cap.hip", "attention_cap_slope.hip",
           "attention_cap_table.hip", "attention_keys.hip", "attention_slope.hip", "attention_table.hip", "glu.hip", "index.hip", "norm.hip", "pipeline.hip", "step8.hip", "wgrad.hip"]
FLAGS = [
    "-O3", "-std=c++17", "--offload-arch=gfx950", "-fPIC", "-shared",
    "-Wall", "-Wextra", "-Wno-unused-parameter",
    # packed-FP32 forms are kept out of every kernel of this library
    "-Xclang", "-target-feature", "-Xclang", "-packed-fp32-ops",
]


def build(verbose: bool = False, extra_flags: list | None = None, out: str | None = None) -> str:
    hipcc = os.environ.get("HIPCC", "/opt/rocm/bin/hipcc")
    out = out or LIB
    tmp = out + ".tmp%d" % os.getpid()
    flags = FLAGS + (extra_flags or []) + ["-I", os.path.join(ROOT, "include"), "-I", CSRC]
    with tempfile.TemporaryDirectory() as objects:           # the sources side by side, then one link
        def compile_one(source: str) -> str:
            made = os.path.join(objects, source + ".o")
            cmd = [hipcc] + [f for f in flags if f != "-shared"] + ["-c", os.path.join(CSRC, source), "-o", made]
            if verbose:
                print(" ".join(cmd), flush=True)
            subprocess.check_call(cmd)
            return made

        with concurrent.futures.ThreadPoolExecutor(min(8, os.cpu_count() or 1)) as pool:
            made = list(pool.map(compile_one, SOURCES))
        subprocess.check_call([hipcc] + flags + made + ["-o", tmp])
    os.replace(tmp, out)
    return out


def build_marshal(verbose: bool = False, out: str | None = None) -> str:
    """_marshal.so, a CPython extension against the installed torch's headers (host code only)."""
    import torch
    root = os.path.dirname(torch.__file__)
    out = out or os.path.join(PKG, "_marshal.so")
    tmp = out + ".tmp%d" % os.getpid()
    cmd = [os.environ.get("CXX", "g++"), "-O2", "-std=c++17", "-fPIC", "-shared", "-w",
           "-D_GLIBCXX_USE_CXX11_ABI=%d" % int(torch.compiled_with_cxx11_abi()),
           "-I", os.path.join(ROOT, "include"),
           "-I", os.path.join(root, "include"), "-I", os.path.join(root, "include", "torch", "csrc", "api", "include"),
           "-I", sysconfig.get_paths()["include"], os.path.join(CSRC, "marshal.cpp"), "-o", tmp,
           "-L", os.path.join(root, "lib"), "-ltorch_python", "-ltorch_cpu", "-lc10"]
    if verbose:
        print(" ".join(cmd), flush=True)
    subprocess.check_call(cmd)
    os.replace(tmp, out)
    return out


if __name__ == "__main__":
    print(build(verbose=True))
    print(build_marshal(verbose=True))
