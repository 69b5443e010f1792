"""Builds, in-tree (no JIT cache, no pip install), libmuon_b200.so with nvcc for sm_100a and _front.so, the torch front end of the layer operators.

    python -m paper_2609_21594_b200.build [--library] [--force] [-v]        (--library: the C library alone, which needs only nvcc)
"""
from __future__ import annotations

import importlib.util
import os
import shutil
import subprocess
import sys
import sysconfig

HERE = os.path.dirname(os.path.abspath(__file__))
CSRC = os.path.join(HERE, "csrc")
HEADER = os.path.join(HERE, "..", "include", "muon_b200.h")
LIB = os.path.join(HERE, "libmuon_b200.so")
FRONT = os.path.join(HERE, "_front.so")
SOURCES = ["api.cu", "plan.cu", "layout_kernels.cu", "elementwise_kernels.cu", "ns_simt.cu", "ns_tcgen05.cu", "ns_tcgen05_pair.cu", "ns_tables.cu",
           "layer_api.cu", "layer_norm.cu", "rotary.cu", "attention_simt.cu", "attention_fwd.cu", "attention_bwd.cu",
           "feed_forward_api.cu", "pack8.cu", "product_simt.cu", "product_tc.cu", "product_few.cu"]
NVCC_FLAGS = ["-gencode", "arch=compute_100a,code=sm_100a", "-lineinfo", "-O3", "-std=c++17",
              "-Xcompiler", "-fPIC"] + os.environ.get("MUON_NVCC_EXTRA", "").split()


def _nvcc() -> str:
    for cand in (os.environ.get("NVCC"), "/usr/local/cuda/bin/nvcc", "nvcc"):
        if cand and (os.path.isabs(cand) and os.path.exists(cand) or not os.path.isabs(cand)):
            return cand
    return "nvcc"


def _stale(target: str, sources: list) -> bool:
    return not os.path.exists(target) or any(os.path.getmtime(d) > os.path.getmtime(target) for d in sources)


def _library_stale() -> bool:
    return _stale(LIB, [os.path.join(CSRC, f) for f in os.listdir(CSRC) if not f.endswith(".cpp")] + [HEADER])


def _front_stale() -> bool:
    return _stale(FRONT, [os.path.join(CSRC, "front.cpp"), HEADER, LIB])


def needs_build() -> bool:
    return _library_stale() or _front_stale()


def _cuda() -> str:
    return os.path.dirname(os.path.dirname(_nvcc())) or "/usr/local/cuda"


def front_lacks() -> list:
    """What this machine lacks to build the torch front end.  The library needs nvcc alone."""
    torch = importlib.util.find_spec("torch")
    have = {"C++ compiler": shutil.which(os.environ.get("CXX", "g++")), "torch": torch,
            "headers of Python": os.path.exists(os.path.join(sysconfig.get_paths()["include"], "Python.h"))}
    if torch:
        have["headers of torch"] = os.path.isdir(os.path.join(torch.submodule_search_locations[0], "include", "torch"))
    return [what for what, there in have.items() if not there]


def _front_command() -> list:
    """The host compiler's command for csrc/front.cpp, linked with torch and with the library next to it."""
    torch = importlib.util.find_spec("torch").submodule_search_locations[0]
    include = [os.path.join(torch, "include"), os.path.join(torch, "include", "torch", "csrc", "api", "include"), sysconfig.get_paths()["include"],
               os.path.join(_cuda(), "include")]
    return [os.environ.get("CXX", "g++"), "-O2", "-std=c++17", "-fPIC", "-shared", "-DTORCH_EXTENSION_NAME=_front", *[f"-I{d}" for d in include],
            os.path.join(CSRC, "front.cpp"), "-o", FRONT, "-L" + os.path.join(torch, "lib"), "-lc10", "-lc10_cuda", "-ltorch_cpu", "-ltorch", "-ltorch_python",
            "-L" + HERE, "-l:" + os.path.basename(LIB), "-Wl,-rpath,$ORIGIN"]


def build_library(force: bool = False, verbose: bool = False) -> str:
    """Compiles every .cu under csrc/ into one shared library next to this file (nvcc alone); returns its path."""
    if not force and not _library_stale():
        return LIB
    objs = []
    odir = os.path.join(HERE, "build")
    os.makedirs(odir, exist_ok=True)
    procs = []
    for src in SOURCES:
        obj = os.path.join(odir, src.replace(".cu", ".o"))
        cmd = [_nvcc(), *NVCC_FLAGS, "-c", os.path.join(CSRC, src), "-o", obj]
        if verbose:
            cmd.insert(1, "-Xptxas=-v")
        procs.append((src, subprocess.Popen(cmd, stdout=subprocess.PIPE, stderr=subprocess.STDOUT, text=True)))
        objs.append(obj)
    failed = False
    for src, p in procs:
        out, _ = p.communicate()
        if out.strip():
            print(f"[nvcc {src}]\n{out}", file=sys.stderr)
        failed |= p.returncode != 0
    if failed:
        raise RuntimeError("nvcc failed")
    subprocess.check_call([_nvcc(), "-gencode", "arch=compute_100a,code=sm_100a", "-shared", "-o", LIB, *objs, "-lcudart_static", "-ldl", "-lpthread", "-lrt"])
    return LIB


def build(force: bool = False, verbose: bool = False) -> str:
    """Builds the library and the front end beside it; returns the library's path.  A machine that lacks what the front end needs gets the library
    alone, which serves the C ABI, `binding` and `optim` (and is told; importing `functional` fails there)."""
    build_library(force, verbose)
    if force or _front_stale():
        lacking = front_lacks()
        if lacking:
            print(f"{os.path.basename(FRONT)} (the torch front end of the layer operators) is not built: no {', no '.join(lacking)}", file=sys.stderr)
        else:
            subprocess.check_call(_front_command())
    return LIB


if __name__ == "__main__":
    print((build_library if "--library" in sys.argv else build)(force="--force" in sys.argv, verbose="-v" in sys.argv))
