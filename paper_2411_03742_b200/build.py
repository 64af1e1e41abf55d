"""Compile the CUDA sources into the in-tree shared library `libadacons_b200.so` (sm_100a).

Usage:  python -m paper_2411_03742_b200.build [--force] [--verbose]
nvcc cross-compiles without a GPU, so this also works on a build machine that has none.
"""
from __future__ import annotations

import os
import shutil
import subprocess
import sys

PKG_DIR = os.path.dirname(os.path.abspath(__file__))
ROOT = os.path.dirname(PKG_DIR)
CSRC = os.path.join(PKG_DIR, "csrc")
INCLUDE = os.path.join(ROOT, "include")
LIB_PATH = os.path.join(PKG_DIR, "libadacons_b200.so")
OBJ_DIR = os.path.join(PKG_DIR, "_build")
_COMMON = ["csrc/adacons_common.cuh", "include/adacons.h"]
_OPS = _COMMON + ["csrc/adacons_tc.cuh", "csrc/adacons_host.cuh", "csrc/adacons_status.cuh", "include/adacons_ops.h"]
# translation units and what each includes
SOURCES = {
    "adacons.cu": _COMMON + ["csrc/" + f for f in ("adacons_kernels.cuh", "adacons_pass1.cuh", "adacons_coeff.cuh", "adacons_pass2.cuh",
                                                   "adacons_fused.cuh", "adacons_gram.cuh", "adacons_shift.cuh")],
    "adacons_orth.cu": _OPS + ["csrc/adacons_orth.cuh"],
    "adacons_attn.cu": _OPS + ["csrc/adacons_attn.cuh"],
    "adacons_rope.cu": _OPS + ["csrc/adacons_rope.cuh"],
    "adacons_ffn.cu": _OPS + ["csrc/adacons_ffn.cuh"],
    "adacons_distill.cu": _OPS + ["csrc/adacons_distill.cuh"],
    **{f"adacons_norm{t}.cu": _OPS + ["csrc/adacons_norm.cuh", "csrc/adacons_norm_run.cuh"] for t in ("", "_f32", "_bf16", "_f16")},
}


def _nvcc() -> str:
    for cand in (os.environ.get("NVCC"), shutil.which("nvcc"), "/usr/local/cuda/bin/nvcc"):
        if cand and os.path.exists(cand):
            return cand
    raise RuntimeError("nvcc not found (set NVCC or put it on PATH)")


def _dep_path(name: str) -> str:
    return os.path.join(PKG_DIR if name.startswith("csrc/") else ROOT, name)


def _newest(source: str) -> float:
    return max(os.path.getmtime(p) for p in [os.path.join(CSRC, source), os.path.abspath(__file__)] + [_dep_path(n) for n in SOURCES[source]])


def _object(source: str) -> str:
    return os.path.join(OBJ_DIR, source[:-len(".cu")] + ".o")


def is_stale() -> bool:
    return not os.path.exists(LIB_PATH) or any(_newest(s) > os.path.getmtime(LIB_PATH) for s in SOURCES)


def _run(cmds, verbose: bool) -> None:
    """Run the commands side by side; raise with the output of the first that fails."""
    procs = [(c, subprocess.Popen(c, stdout=subprocess.PIPE, stderr=subprocess.STDOUT, text=True)) for c in cmds]
    done = [(c, p, p.communicate()[0]) for c, p in procs]
    for cmd, p, text in done:
        if p.returncode != 0:
            raise RuntimeError("nvcc failed:\n" + " ".join(cmd) + "\n" + text)
        if verbose:
            sys.stderr.write(text)


def build(force: bool = False, verbose: bool = False) -> str:
    if not force and not is_stale():
        return LIB_PATH
    os.makedirs(OBJ_DIR, exist_ok=True)
    arch = ["-gencode", "arch=compute_100a,code=sm_100a"]
    todo = [s for s in SOURCES if force or not os.path.exists(_object(s)) or _newest(s) > os.path.getmtime(_object(s))]
    _run([[_nvcc()] + (["-Xptxas", "-v"] if verbose else []) + ["-c", "-Xcompiler", "-fPIC", "-O3", "-std=c++17", "-lineinfo"] + arch +
          ["-I", INCLUDE, "-I", CSRC, "-o", _object(s), os.path.join(CSRC, s)] for s in todo], verbose)
    _run([[_nvcc(), "-shared", "-Xcompiler", "-fPIC"] + arch + ["-o", LIB_PATH] + [_object(s) for s in SOURCES]], verbose)
    return LIB_PATH


if __name__ == "__main__":
    print(build(force="--force" in sys.argv, verbose="--verbose" in sys.argv))
