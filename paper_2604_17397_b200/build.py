"""Compile the CUDA sources into the in-tree shared library (sm_100a only)."""
from __future__ import annotations

import os
import shutil
import subprocess
import sys

HERE = os.path.dirname(os.path.abspath(__file__))
ROOT = os.path.dirname(HERE)
CSRC = os.path.join(HERE, "csrc")
LIB_PATH = os.path.join(HERE, "libsdvg.so")
SOURCES = ["sdvg_host.cu", "rope_commit.cu", "route.cu", "state.cu", "quant.cu", "steps.cu", "attn_fwd.cu",
           "linear.cu", "gated_norm.cu", "qk_norm.cu"]
BINDING_PATH = os.path.join(HERE, "_binding.so")


def nvcc_path() -> str:
    for cand in (os.environ.get("NVCC"), shutil.which("nvcc"), "/usr/local/cuda/bin/nvcc"):
        if cand and os.path.exists(cand):
            return cand
    raise RuntimeError("nvcc not found")


def needs_build(out: str = LIB_PATH) -> bool:
    if not os.path.exists(out):
        return True
    t = os.path.getmtime(out)
    deps = [os.path.join(CSRC, f) for f in os.listdir(CSRC)] + [os.path.join(ROOT, "include", "sdvg.h")]
    return any(os.path.getmtime(d) > t for d in deps)


def build(force: bool = False, out: str = LIB_PATH, extra_flags=(), verbose: bool = False) -> str:
    if not force and not needs_build(out):
        if out == LIB_PATH:
            build_binding()
        return out
    cmd = [nvcc_path(), "-shared", "-Xcompiler", "-fPIC", "-std=c++17", "-O3", "-lineinfo",
           "-gencode", "arch=compute_100a,code=sm_100a",
           "-I", os.path.join(ROOT, "include"), "-I", CSRC,
           *extra_flags,
           *[os.path.join(CSRC, s) for s in SOURCES], "-o", out]
    if verbose:
        print(" ".join(cmd), file=sys.stderr)
    subprocess.run(cmd, check=True)
    if out == LIB_PATH:
        build_binding(force)
    return out


def build_binding(force: bool = False):
    """The compiled argument marshalling of the dense operators: links the library and torch's Python types, so that it is
    built again for another torch or Python.  Returns its path, or None where there is no torch to build it for (the library
    itself needs none)."""
    try:
        import torch
    except ImportError:
        return None
    import sysconfig

    sources = [os.path.join(CSRC, "binding.cpp"), os.path.join(ROOT, "include", "sdvg.h")]
    made_for, note = f"torch {torch.__version__} {sys.implementation.cache_tag}", BINDING_PATH + ".made_for"
    if not force and os.path.exists(BINDING_PATH) and os.path.exists(note):
        with open(note) as f:
            same = f.read() == made_for
        if same and all(os.path.getmtime(s) <= os.path.getmtime(BINDING_PATH) for s in sources):
            return BINDING_PATH
    torch_dir = os.path.dirname(torch.__file__)
    include = [os.path.join(torch_dir, "include"), os.path.join(torch_dir, "include", "torch", "csrc", "api", "include"),
               sysconfig.get_paths()["include"]]
    libs = os.path.join(torch_dir, "lib")
    subprocess.run([os.environ.get("CXX", "g++"), "-O2", "-std=c++17", "-shared", "-fPIC",
                    f"-D_GLIBCXX_USE_CXX11_ABI={int(torch._C._GLIBCXX_USE_CXX11_ABI)}",
                    *[a for d in include for a in ("-isystem", d)], "-I", os.path.join(ROOT, "include"), sources[0], "-o",
                    BINDING_PATH, "-L" + HERE, "-l:libsdvg.so", "-Wl,-rpath,$ORIGIN", "-L" + libs, "-Wl,-rpath," + libs, "-ltorch_python",
                    "-ltorch_cpu", "-lc10"], check=True)
    with open(note, "w") as f:
        f.write(made_for)
    return BINDING_PATH


if __name__ == "__main__":
    build(force="--force" in sys.argv, verbose=True,
          extra_flags=("-Xptxas", "-v") if "--ptxas" in sys.argv else ())
    print(LIB_PATH)
