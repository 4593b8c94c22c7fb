"""Builds libgar.so (sm_100a) in-tree with nvcc.  `python -m paper_1905_04374_b200.build`."""
from __future__ import annotations

import os
import shutil
import subprocess
import sys
from concurrent.futures import ThreadPoolExecutor

PKG = os.path.dirname(os.path.abspath(__file__))
ROOT = os.path.dirname(PKG)
CSRC = os.path.join(PKG, "csrc")
OBJ = os.path.join(PKG, "_build")
LIB = os.path.join(PKG, "libgar.so")
WORKER_MODULE = os.path.join(PKG, "_gar_worker.so")

# Slot counts the coordinate kernel is compiled for: keep identical to K3_P_LIST in k3_dispatch.cu.
K3_P = list(range(1, 33)) + [36, 40, 44, 48, 52, 56, 60, 64]     # <= 32: theta fixed at compile time

NVCC_FLAGS = ["-gencode", "arch=compute_100a,code=sm_100a", "-lineinfo", "-O3", "-std=c++17",
              "-Xcompiler", "-fPIC", "-I" + os.path.join(ROOT, "include"), "-I" + CSRC]


def _nvcc() -> str:
    exe = shutil.which("nvcc") or "/usr/local/cuda/bin/nvcc"
    if not os.path.exists(exe):
        raise RuntimeError("nvcc not found: the CUDA toolkit is needed to build libgar.so")
    return exe


def _units():
    units = [("k1_distances.cu", "k1_distances.o", []),
             ("k1_umma.cu", "k1_umma.o", []),
             ("k2_select.cu", "k2_select.o", []),
             ("k3_dispatch.cu", "k3_dispatch.o", []),
             ("gar_api.cu", "gar_api.o", [])]
    for name in ("logprobs", "checkpoint", "wgrad", "api"):
        units.append((f"worker_{name}.cu", f"worker_{name}.o", []))
    for p in K3_P:
        units.append(("k3_inst.cu", f"k3_inst_{p}.o", [f"-DK3_P={p}", f"-DK3_EXACT={1 if p <= 32 else 0}"]))
    return units


def _newest_header(worker: bool) -> float:
    """The newest header a unit depends on: the worker-side operators' own headers concern their units only."""
    hdrs = [os.path.join(CSRC, f) for f in os.listdir(CSRC)
            if f.endswith((".cuh", ".h")) and (worker or not f.startswith("worker_"))]
    hdrs.append(os.path.join(ROOT, "include", "gar.h"))
    if worker:
        hdrs.append(os.path.join(ROOT, "include", "gar_worker.h"))
    hdrs.append(os.path.abspath(__file__))
    return max(os.path.getmtime(h) for h in hdrs)


def build(force: bool = False, verbose: bool = False) -> str:
    """Compile every translation unit that is out of date and link libgar.so."""
    os.makedirs(OBJ, exist_ok=True)
    nvcc = _nvcc()
    hdr_time = {w: _newest_header(w) for w in (False, True)}
    jobs = []
    for src, obj, extra in _units():
        s, o = os.path.join(CSRC, src), os.path.join(OBJ, obj)
        if force or not os.path.exists(o) or os.path.getmtime(o) < max(os.path.getmtime(s), hdr_time[src.startswith("worker_")]):
            jobs.append([nvcc, *NVCC_FLAGS, *extra, "-c", s, "-o", o])

    def run(cmd):
        res = subprocess.run(cmd, capture_output=True, text=True)
        if res.returncode != 0:
            raise RuntimeError("nvcc failed: " + " ".join(cmd) + "\n" + res.stdout + res.stderr)
        if verbose and (res.stdout or res.stderr):
            print(res.stdout + res.stderr)

    if jobs:
        with ThreadPoolExecutor(max_workers=min(len(jobs), os.cpu_count() or 4)) as ex:
            list(ex.map(run, jobs))
    objs = [os.path.join(OBJ, obj) for _, obj, _ in _units()]
    if jobs or not os.path.exists(LIB):
        run([nvcc, "-shared", "-o", LIB, *objs, "-gencode", "arch=compute_100a,code=sm_100a"])
    _build_worker_module(run, force)
    return LIB


def _build_worker_module(run, force: bool) -> None:
    """Compile the tensor marshalling of the worker-side operators against the installed torch."""
    src = os.path.join(CSRC, "worker_binding.cpp")
    deps = [src, os.path.join(ROOT, "include", "gar.h"), os.path.join(ROOT, "include", "gar_worker.h"), os.path.abspath(__file__)]
    if not force and os.path.exists(WORKER_MODULE) and os.path.getmtime(WORKER_MODULE) >= max(map(os.path.getmtime, deps)):
        return
    import sysconfig

    import torch
    base = os.path.dirname(torch.__file__)
    cuda = os.path.dirname(os.path.dirname(_nvcc()))
    libs = os.path.join(base, "lib")
    run(["g++", "-O2", "-std=c++17", "-fPIC", "-shared", f"-D_GLIBCXX_USE_CXX11_ABI={int(torch._C._GLIBCXX_USE_CXX11_ABI)}",
         "-I" + os.path.join(ROOT, "include"), "-isystem", os.path.join(base, "include"), "-isystem", sysconfig.get_paths()["include"],
         "-isystem", os.path.join(cuda, "include"), src, "-o", WORKER_MODULE, "-L" + PKG, "-lgar", "-L" + libs, "-lc10", "-lc10_cuda",
         "-ltorch_cpu", "-ltorch_cuda", "-ltorch_python", "-Wl,-rpath,$ORIGIN", "-Wl,-rpath," + libs])


if __name__ == "__main__":
    print(build(force="--force" in sys.argv, verbose=True))
