"""Build the gfx950 shared library (HIP kernels + C ABI) in-tree."""
from __future__ import annotations

import os
import shutil
import subprocess
import sys

PKG = os.path.dirname(os.path.abspath(__file__))
ROOT = os.path.dirname(PKG)
CSRC = os.path.join(PKG, "csrc")
INCLUDE = os.path.join(ROOT, "include")
LIB_NAME = "libwfplan.so"
LIB_PATH = os.path.join(PKG, LIB_NAME)
BIND_PATH = os.path.join(PKG, "_kvbind.so")
SOURCES = ["host.hip", "score.hip", "score_keys.hip", "argmin.hip", "prefix.hip", "lean.hip",
           "lanes.hip", "kv_host.hip", "kv_step.hip", "kv_store.hip", "kv_attend.hip"]
ARCH = "gfx950"

HIP_FLAGS = [
    "-O3", "-std=c++17", "-fPIC", f"--offload-arch={ARCH}",
    # the objective is two fp32 products and an fp32 sum, each rounded:
    # no contraction into fused multiply-adds
    "-ffp-contract=off",
    # no packed fp32 instructions in generated device code
    "-Xclang", "-target-feature", "-Xclang", "-packed-fp32-ops",
    # the iterative ILP scheduler: 1.8% faster scoring on the 256-activation
    # window and 3% on the 400-activation one than the default schedule
    "-mllvm", "-amdgpu-sched-strategy=iterative-ilp",
    "-Wall", "-Wno-unused-command-line-argument",
]


def flags(src: str) -> list:
    """Compiler flags of a source.  The cache kernels (kv_*) take the default
    schedule: the compiler fails on attention with the other."""
    if not src.startswith("kv_"):
        return HIP_FLAGS
    return [f for f in HIP_FLAGS if "sched-strategy" not in f and f != "-mllvm"]


def bind_command(out: str) -> list:
    """Compiler call for _kvbind.so, the short way from torch tensors to the cache's calls: host
    code only, against the headers and libraries of the installed torch."""
    import sysconfig
    import torch
    at = os.path.dirname(torch.__file__)
    lib = os.path.join(at, "lib")
    return [os.environ.get("CXX", "g++"), "-O2", "-std=c++17", "-fPIC", "-shared", "-fvisibility=hidden", "-w",
            f"-D_GLIBCXX_USE_CXX11_ABI={int(torch._C._GLIBCXX_USE_CXX11_ABI)}", "-I", INCLUDE,
            "-I", os.path.join(at, "include"), "-I", os.path.join(at, "include", "torch", "csrc", "api", "include"),
            "-I", sysconfig.get_paths()["include"], os.path.join(CSRC, "kv_bind.cpp"), "-o", out,
            "-L", lib, "-ltorch_python", "-ltorch_cpu", "-lc10"]


def hipcc() -> str:
    for c in (os.environ.get("HIPCC"), "/opt/rocm/bin/hipcc", shutil.which("hipcc")):
        if c and os.path.exists(c):
            return c
    raise RuntimeError("hipcc not found: the gfx950 library cannot be built")


def start_bind(out: str):
    """The compiler of _kvbind.so as a process, or why there is none: it needs torch and a host compiler,
    which the library does not."""
    try:
        return subprocess.Popen(bind_command(out), stdout=subprocess.PIPE, stderr=subprocess.STDOUT), None
    except (ImportError, OSError) as e:
        return None, str(e)


def build(verbose: bool = False) -> str:
    """Compile every HIP source for gfx950 and link libwfplan.so next to
    this file.  Always recompiles.  _kvbind.so is built beside it where that is possible; where it
    is not, the Python calls take the longer way."""
    build_dir = os.path.join(PKG, "_build")
    os.makedirs(build_dir, exist_ok=True)
    objs = []
    procs = []
    for src in SOURCES:
        obj = os.path.join(build_dir, src.replace(".hip", ".o"))
        cmd = [hipcc(), *flags(src), "-I", INCLUDE, "-c", os.path.join(CSRC, src), "-o", obj]
        if verbose:
            print(" ".join(cmd), file=sys.stderr)
        procs.append((src, subprocess.Popen(cmd, stdout=subprocess.PIPE, stderr=subprocess.STDOUT)))
        objs.append(obj)
    bind = os.path.join(build_dir, "_kvbind.so")
    bind_proc, why = start_bind(bind)
    errors = []
    for src, p in procs:
        out, _ = p.communicate()
        text = out.decode(errors="replace")
        text = "\n".join(l for l in text.splitlines() if "packed-fp32-ops" not in l and l.strip())
        if p.returncode != 0:
            errors.append(f"{src}:\n{text}")
        elif verbose and text:
            print(text, file=sys.stderr)
    if errors:
        raise RuntimeError("HIP build failed:\n" + "\n".join(errors))
    tmp = LIB_PATH + ".tmp"
    cmd = [hipcc(), f"--offload-arch={ARCH}", "-shared", "-fPIC", "-o", tmp, *objs]
    subprocess.check_call(cmd)
    os.replace(tmp, LIB_PATH)
    if bind_proc is not None:
        out, _ = bind_proc.communicate()
        if bind_proc.returncode != 0:
            why = out.decode(errors="replace").strip() or f"exit status {bind_proc.returncode}"
    if why is None:
        os.replace(bind, BIND_PATH)
    else:
        print(f"_kvbind.so is not built: {why}", file=sys.stderr)
        if os.path.exists(BIND_PATH):    # an earlier build's may not fit this one's header
            os.remove(BIND_PATH)
    return LIB_PATH


if __name__ == "__main__":
    print(build(verbose=True))
