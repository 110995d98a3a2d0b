"""Build libmix.so (sm_100a only) in-tree with nvcc."""
from __future__ import annotations

import os
import shutil
import subprocess
import sysconfig

PKG_DIR = os.path.dirname(os.path.abspath(__file__))
ROOT = os.path.dirname(PKG_DIR)
CSRC = os.path.join(PKG_DIR, "csrc")
LIB_PATH = os.path.join(PKG_DIR, "libmix.so")
FAST_PATH = os.path.join(PKG_DIR, "_fastcall.so")      # CPython module of the binding's per-step calls, linked to libmix.so

SOURCES = ["mix_api.cu", "route_probe_steer.cu", "probe_tc.cu", "sae_front.cu", "sae_simt_edit_only.cu", "sae_encode_tc.cu", "sae_tail.cu",
           "sae_static.cu", "router_select.cu", "router_balance.cu", "linear_int.cu"]


def _nvcc() -> str:
    for cand in (os.environ.get("NVCC"), shutil.which("nvcc"), "/usr/local/cuda/bin/nvcc"):
        if cand and os.path.exists(cand):
            return cand
    raise RuntimeError("nvcc not found")


def needs_build() -> bool:
    if not (os.path.exists(LIB_PATH) and os.path.exists(FAST_PATH)):
        return True
    t = min(os.path.getmtime(LIB_PATH), os.path.getmtime(FAST_PATH))
    deps = [os.path.join(CSRC, f) for f in os.listdir(CSRC)] + [os.path.join(ROOT, "include", "mix.h")]
    return any(os.path.getmtime(p) > t for p in deps)


def build(force: bool = False, verbose: bool = False) -> str:
    if not force and not needs_build():
        return LIB_PATH
    cmd = [_nvcc(), "-gencode", "arch=compute_100a,code=sm_100a", "-O3", "-std=c++17", "-lineinfo",
           "-shared", "-Xcompiler", "-fPIC", "-I", os.path.join(ROOT, "include"), "-I", CSRC,
           "-o", LIB_PATH] + [os.path.join(CSRC, s) for s in SOURCES] + ["-lcudart"]
    extra = os.environ.get("MIX_NVCC_EXTRA")      # e.g. "-DMIX_SOMETHING" for one-off experiments
    if extra:
        cmd[1:1] = extra.split()
    if verbose:
        cmd.insert(1, "-Xptxas")
        cmd.insert(2, "-v")
    res = subprocess.run(cmd, capture_output=True, text=True)
    if res.returncode != 0:
        raise RuntimeError("nvcc failed:\n" + res.stdout + res.stderr)
    if verbose:
        print(res.stderr)
    cmd = [shutil.which("gcc") or "gcc", "-O2", "-shared", "-fPIC", "-I", sysconfig.get_paths()["include"], "-I", os.path.join(ROOT, "include"),
           "-o", FAST_PATH, os.path.join(CSRC, "fastcall.c"), "-L", PKG_DIR, "-l:libmix.so", "-Wl,-rpath,$ORIGIN"]
    res = subprocess.run(cmd, capture_output=True, text=True)
    if res.returncode != 0:
        raise RuntimeError("gcc failed:\n" + res.stdout + res.stderr)
    return LIB_PATH
