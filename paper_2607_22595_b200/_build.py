"""Build libmix.so (sm_100a only) and the two CPython modules that call it, in-tree."""
from __future__ import annotations

import os
import shutil
import subprocess
import sysconfig
import tempfile
from concurrent.futures import ThreadPoolExecutor

import torch

PKG_DIR = os.path.dirname(os.path.abspath(__file__))
ROOT = os.path.dirname(PKG_DIR)
CSRC = os.path.join(PKG_DIR, "csrc")
LIB_PATH = os.path.join(PKG_DIR, "libmix.so")
FAST_PATH = os.path.join(PKG_DIR, "_fastcall.so")      # CPython module of the binding's per-step calls, linked to libmix.so
OPS_PATH = os.path.join(PKG_DIR, "_fastops.so")        # the same for the calls of experts.py, on torch's C++ interface

SOURCES = ["mix_api.cu", "route_probe_steer.cu", "probe_tc.cu", "sae_front.cu", "sae_simt_edit_only.cu", "sae_encode_tc.cu", "sae_tail.cu",
           "sae_static.cu", "router_select.cu", "router_balance.cu", "linear_int.cu"]


def _nvcc() -> str:
    for cand in (os.environ.get("NVCC"), shutil.which("nvcc"), "/usr/local/cuda/bin/nvcc"):
        if cand and os.path.exists(cand):
            return cand
    raise RuntimeError("nvcc not found")


def needs_build() -> bool:
    built = [LIB_PATH, FAST_PATH, OPS_PATH]
    if not all(os.path.exists(p) for p in built):
        return True
    t = min(os.path.getmtime(p) for p in built)
    deps = [os.path.join(CSRC, f) for f in os.listdir(CSRC)] + [os.path.join(ROOT, "include", "mix.h")]
    return any(os.path.getmtime(p) > t for p in deps)


def _ops_command() -> list:
    top = os.path.dirname(torch.__file__)
    cuda = os.path.dirname(os.path.dirname(_nvcc()))
    return [shutil.which("g++") or "g++", "-O2", "-std=c++17", "-shared", "-fPIC", "-D_GLIBCXX_USE_CXX11_ABI=%d" % int(torch.compiled_with_cxx11_abi()),
            "-I", sysconfig.get_paths()["include"], "-I", os.path.join(ROOT, "include"), "-I", os.path.join(top, "include"), "-I",
            os.path.join(top, "include", "torch", "csrc", "api", "include"), "-I", os.path.join(cuda, "include"), "-o", OPS_PATH,
            os.path.join(CSRC, "fastops.cpp"), "-L", os.path.join(top, "lib"), "-lc10", "-lc10_cuda", "-ltorch_cpu", "-ltorch_cuda", "-ltorch_python",
            "-L", PKG_DIR, "-l:libmix.so", "-Wl,-rpath,$ORIGIN"]


def build(force: bool = False, verbose: bool = False) -> str:
    if not force and not needs_build():
        return LIB_PATH
    flags = ["-gencode", "arch=compute_100a,code=sm_100a", "-O3", "-std=c++17", "-lineinfo", "-Xcompiler", "-fPIC",
             "-I", os.path.join(ROOT, "include"), "-I", CSRC]
    extra = os.environ.get("MIX_NVCC_EXTRA")      # e.g. "-DMIX_SOMETHING" for one-off experiments
    flags = (extra.split() if extra else []) + flags + (["-Xptxas", "-v"] if verbose else [])
    with tempfile.TemporaryDirectory() as tmp:    # a process per source: they take half a minute each
        objects = [os.path.join(tmp, s + ".o") for s in SOURCES]
        jobs = [[_nvcc()] + flags + ["-c", os.path.join(CSRC, s), "-o", o] for s, o in zip(SOURCES, objects)]
        with ThreadPoolExecutor(os.cpu_count() or 4) as pool:
            done = list(pool.map(lambda cmd: subprocess.run(cmd, capture_output=True, text=True), jobs))
        bad = [r for r in done if r.returncode != 0]
        if bad:
            raise RuntimeError("nvcc failed:\n" + "".join(r.stdout + r.stderr for r in bad))
        res = subprocess.run([_nvcc(), "-gencode", "arch=compute_100a,code=sm_100a", "-shared", "-o", LIB_PATH] + objects + ["-lcudart"],
                             capture_output=True, text=True)
    if res.returncode != 0:
        raise RuntimeError("nvcc failed:\n" + res.stdout + res.stderr)
    if verbose:
        print("".join(r.stderr for r in done))
    cmd = [shutil.which("gcc") or "gcc", "-O2", "-shared", "-fPIC", "-I", sysconfig.get_paths()["include"], "-I", os.path.join(ROOT, "include"),
           "-o", FAST_PATH, os.path.join(CSRC, "fastcall.c"), "-L", PKG_DIR, "-l:libmix.so", "-Wl,-rpath,$ORIGIN"]
    for cmd in (cmd, _ops_command()):
        res = subprocess.run(cmd, capture_output=True, text=True)
        if res.returncode != 0:
            raise RuntimeError("gcc failed:\n" + res.stdout + res.stderr)
    return LIB_PATH
