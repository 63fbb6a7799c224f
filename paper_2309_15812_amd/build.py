"""Builds the HIP library ``libo1d.so`` in-tree for gfx950 with hipcc.

Usage: ``python -m paper_2309_15812_amd.build`` (or ``build()`` from Python).
Cross-compiles without a GPU.  Every ``csrc/*.hip`` translation unit is
compiled to an object in parallel (the strip kernels are split per family,
storage type and cell bound for this), then the objects are linked into the
library.  ``_rows.so`` and ``_train.so``, host code that calls the library from torch
tensors, are compiled with g++ beside it.
"""
from __future__ import annotations

import concurrent.futures
import glob
import hashlib
import os
import shutil
import subprocess
import sys
import tempfile

PKG = os.path.dirname(os.path.abspath(__file__))
ROOT = os.path.dirname(PKG)
CSRC = os.path.join(PKG, "csrc")
INCLUDE = os.path.join(ROOT, "include")
LIB = os.path.join(PKG, "libo1d.so")
# Python's calls of the row operators and of group norm, 8-bit products and AdamW (host code only)
BINDINGS = {os.path.join(PKG, "_rows.so"): "o1d_torch.cpp", os.path.join(PKG, "_train.so"): "o1d_torch_train.cpp"}
HIPCC = os.environ.get("HIPCC", "/opt/rocm/bin/hipcc")

FLAGS = [
    "--offload-arch=gfx950",
    "-O3",
    "-std=c++17",
    "-fPIC",
    # Keep the compiler from forming packed FP32 instructions.
    "-Xclang", "-target-feature", "-Xclang", "-packed-fp32-ops",
    "-Wno-unused-command-line-argument",
]


def sources() -> list[str]:
    return sorted(glob.glob(os.path.join(CSRC, "*.hip")))


# The strip kernels are sized to stay in registers (their walks keep a
# window and per-output accumulators of up to 60 values per lane); a spill to
# scratch memory would cost far more than it saves, so their translation
# units are compiled with resource remarks and rejected if any kernel in them
# uses scratch memory.  The general kernels and the row operators are checked the same way.
CHECKED = ("o1d_strip_", "o1d_gen_", "o1d_plane_", "o1d_pw_", "o1d_walk_", "o1d_ln_", "o1d_held", "o1d_mm", "o1d_few_",
           "o1d_gn_", "o1d_f8_", "o1d_adam")
# Kernels that keep some values in scratch memory, with the bytes per lane they may.  In float32 tiles of 128 x 192 the
# gradients reload up to 17 words per step of 4 us; the others touch it outside their loops.
SCRATCH = {
    "2mmIfLi0ELi1ELb0EE": 8, "2mmIfLi1ELi1ELb0EE": 8, "2mmIfLi2ELi1ELb1EE": 12,  # float32, 64 x 64
    "2mmIfLi0ELi5ELb0EE": 8, "2mmIfLi1ELi5ELb0EE": 80, "2mmIfLi2ELi5ELb0EE": 80,  # float32, 128 x 192
    "4f8mmItLi0ELi0E": 48, "4f8mmItLi1ELi0E": 28,  # 8-bit operands, 256 x 256: in the epilogue
    "11ln_bwd_rowsItLi64ELi8ELb1EE": 20,  # layer norm's backward of 4096 bfloat16 features, from a checkpoint
}
REMARK = "-Rpass-analysis=kernel-resource-usage"


def _check_no_scratch(src: str, stderr: str) -> None:
    name, bad = None, []
    for line in stderr.splitlines():
        if "Function Name:" in line:
            name = line.split("Function Name:")[1].split()[0]
        elif "ScratchSize [bytes/lane]:" in line and name is not None:
            used = int(line.split("ScratchSize [bytes/lane]:")[1].split()[0])
            if used > max((n for kernel, n in SCRATCH.items() if kernel in name), default=0):
                bad.append(f"{name} ({used} bytes per lane)")
    if bad:
        raise RuntimeError(f"{os.path.basename(src)}: kernels use scratch memory (register spills): {bad}")


def _run(cmd: list[str], verbose: bool) -> None:
    if verbose:
        print(" ".join(cmd), flush=True)
    res = subprocess.run(cmd, capture_output=True, text=True)
    if res.returncode != 0:
        sys.stderr.write(res.stdout + res.stderr)
        raise RuntimeError(f"{cmd[0]} failed with exit code {res.returncode}: {' '.join(cmd[-3:])}")
    if REMARK in cmd:
        _check_no_scratch(cmd[-1], res.stderr)


def _key(src: str, flags: list[str]) -> str:
    """Hash of a translation unit, every header it may include and the flags."""
    h = hashlib.sha256(" ".join(flags).encode())
    for f in [src, *sorted(glob.glob(os.path.join(CSRC, "*.h"))), os.path.join(INCLUDE, "o1d.h")]:
        with open(f, "rb") as fh:
            h.update(os.path.basename(f).encode() + b"\0" + fh.read())
    return h.hexdigest()[:20]


def build_binding(lib: str, verbose: bool = False) -> str:
    """Compiles a Python module against this torch's headers."""
    import sysconfig

    import torch

    t = os.path.dirname(torch.__file__)
    tmp = lib + ".tmp"
    _run(["g++", "-O2", "-std=c++17", "-fPIC", "-shared", "-DUSE_ROCM", "-D__HIP_PLATFORM_AMD__",
          f"-D_GLIBCXX_USE_CXX11_ABI={int(torch._C._GLIBCXX_USE_CXX11_ABI)}", "-I", INCLUDE,
          "-isystem", os.path.join(t, "include"), "-isystem", os.path.join(t, "include", "torch", "csrc", "api", "include"),
          "-isystem", "/opt/rocm/include", "-isystem", sysconfig.get_paths()["include"],
          os.path.join(CSRC, BINDINGS[lib]), "-o", tmp, "-L", os.path.join(t, "lib"), "-ltorch", "-ltorch_cpu", "-lc10",
          "-lc10_hip", "-ltorch_python"], verbose)
    os.replace(tmp, lib)
    return lib


def build(verbose: bool = False, jobs: int | None = None, incremental: bool = False) -> str:
    """Compiles every translation unit, links libo1d.so and builds _rows.so and _train.so.  With incremental=True, objects whose source,
    headers and flags are unchanged are reused from _build/ (a development aid; the default always
    recompiles everything)."""
    srcs = sources()
    jobs = jobs or min(len(srcs), max(1, min(os.cpu_count() or 1, 16)))
    tmpdir = tempfile.mkdtemp(prefix="o1d_build_")
    cache = os.path.join(PKG, "_build")
    try:
        objs, cmds = [], []
        for src in srcs:
            extra = [REMARK] if os.path.basename(src).startswith(CHECKED) else []
            flags = [*FLAGS, *extra]
            obj = os.path.join(tmpdir, os.path.basename(src) + ".o")
            cached = os.path.join(cache, os.path.basename(src) + "." + _key(src, flags) + ".o")
            if incremental and os.path.exists(cached):
                shutil.copy(cached, obj)
            else:
                cmds.append(([HIPCC, *flags, "-I", INCLUDE, "-I", CSRC, "-c", "-o", obj, src], obj, cached))
            objs.append(obj)
        with concurrent.futures.ThreadPoolExecutor(max_workers=jobs) as ex:
            for fut in [ex.submit(_run, c, verbose) for c, _, _ in cmds]:
                fut.result()
        if incremental:
            os.makedirs(cache, exist_ok=True)
            for _, obj, cached in cmds:
                shutil.copy(obj, cached)
        tmp = LIB + ".tmp"
        _run([HIPCC, "--offload-arch=gfx950", "-shared", "-fPIC", "-o", tmp, *objs], verbose)
        os.replace(tmp, LIB)
        with concurrent.futures.ThreadPoolExecutor(max_workers=len(BINDINGS)) as ex:
            list(ex.map(lambda so: build_binding(so, verbose), BINDINGS))
    finally:
        shutil.rmtree(tmpdir, ignore_errors=True)
    return LIB


if __name__ == "__main__":
    print(build(verbose=True, incremental="--incremental" in sys.argv))
