"""Builds ``libdppf.so`` (CUDA kernels + C ABI) in-tree with nvcc for sm_100a."""
from __future__ import annotations

import os
import shutil
import subprocess
import sys

_PKG = os.path.dirname(os.path.abspath(__file__))
_ROOT = os.path.dirname(_PKG)
# translation units, each with the kernel families that it includes
UNITS = {
    "dppf.cu": ("common.cuh", "round_register.cuh", "adamw_element.cuh", "adamw.cuh", "chunk_ring.cuh", "round_staged.cuh",
                "round_multi.cuh", "round_fused_staged.cuh", "round_general.cuh", "round_generic.cuh", "round_worker.cuh"),
    "local_model.cu": ("common.cuh", "chunk_ring.cuh", "adamw_element.cuh", "local_common.cuh", "local_host.cuh", "embedding.cuh",
                       "policy_loss.cuh", "adamw_tensors.cuh"),
    "block.cu": ("common.cuh", "chunk_ring.cuh", "local_common.cuh", "local_host.cuh", "layer_norm.cuh", "rotary.cuh"),
    "attention.cu": ("common.cuh", "chunk_ring.cuh", "local_common.cuh", "local_host.cuh", "tensor_core.cuh", "attention.cuh"),
}
ABI_HEADER = os.path.join(_ROOT, "include", "dppf.h")


def _csrc(name: str) -> str:
    return os.path.join(_PKG, "csrc", name)


SOURCES = [_csrc(n) for n in UNITS]
HEADERS = [ABI_HEADER] + sorted({_csrc(n) for names in UNITS.values() for n in names})
LIB_PATH = os.path.join(_PKG, "libdppf.so")

NVCC_FLAGS = ["-gencode", "arch=compute_100a,code=sm_100a", "-lineinfo", "-O3", "-std=c++17",
              "-Xcompiler", "-fPIC"]


def nvcc_path() -> str:
    cand = shutil.which("nvcc") or "/usr/local/cuda/bin/nvcc"
    if not os.path.exists(cand):
        raise RuntimeError("nvcc not found: the CUDA library cannot be built")
    return cand


def is_stale() -> bool:
    if not os.path.exists(LIB_PATH):
        return True
    t = os.path.getmtime(LIB_PATH)
    return any(os.path.getmtime(p) > t for p in SOURCES + HEADERS)


def build(force: bool = False, verbose: bool = False) -> str:
    """Compile if the library is missing or older than its sources; return its path."""
    if not force and not is_stale():
        return LIB_PATH
    nvcc, tag = nvcc_path(), f".tmp{os.getpid()}"
    objects, running = [], []
    for unit, includes in UNITS.items():                    # the units compile side by side
        obj = _csrc(unit.replace(".cu", ".o"))
        objects.append(obj)
        needs = [ABI_HEADER, _csrc(unit)] + [_csrc(n) for n in includes]
        if not force and os.path.exists(obj) and all(os.path.getmtime(p) <= os.path.getmtime(obj) for p in needs):
            continue
        cmd = [nvcc, *(["-Xptxas=-v"] if verbose else []), *NVCC_FLAGS, "-I", os.path.join(_ROOT, "include"), "-c", "-o", obj + tag, _csrc(unit)]
        running.append((cmd, obj, subprocess.Popen(cmd)))
    codes = [p.wait() for _, _, p in running]
    for (cmd, obj, _), rc in zip(running, codes):
        if rc:
            raise subprocess.CalledProcessError(rc, cmd)
        os.replace(obj + tag, obj)
    subprocess.run([nvcc, *NVCC_FLAGS, "-shared", "-o", LIB_PATH + tag, *objects], check=True)
    os.replace(LIB_PATH + tag, LIB_PATH)
    return LIB_PATH


if __name__ == "__main__":
    print(build(force="--stale" not in sys.argv, verbose=True))
