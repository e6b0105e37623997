"""Compile the CUDA sources into libinstinfer.so next to this file (sm_100a only)."""
from __future__ import annotations

import os
import shutil
import subprocess
from concurrent.futures import ThreadPoolExecutor
from pathlib import Path

_HERE = Path(__file__).resolve().parent
CSRC = _HERE / "csrc"
INCLUDE = _HERE.parent / "include"
LIBRARY = _HERE / "libinstinfer.so"
CHECKED_LIBRARY = _HERE / "libinstinfer_checked.so"     # the bounds-checking build (-DINSTINFER_BOUNDS_CHECK)
# instinfer_api.cu includes the api_*.inl parts; tree_* and latent_* hold instances of large kernels, one head size or type
# each; the others are parts of the C ABI with kernels of their own
SOURCES = [CSRC / "instinfer_api.cu", CSRC / "tree_d64.cu", CSRC / "tree_d128.cu", CSRC / "tree_d256.cu",
           CSRC / "rope.cu", CSRC / "logits.cu", CSRC / "latent.cu", CSRC / "latent_f16.cu", CSRC / "latent_bf16.cu"]
NVCC_FLAGS = ["-gencode", "arch=compute_100a,code=sm_100a", "-O3", "-std=c++17", "-lineinfo",
              "-Xcompiler", "-fPIC", "-cudart", "static", "-Xptxas", "-v"]


def _nvcc() -> str:
    found = shutil.which("nvcc") or "/usr/local/cuda/bin/nvcc"
    if not os.path.exists(found):
        raise RuntimeError("nvcc not found: the CUDA library cannot be built")
    return found


def _inputs():
    return (list(CSRC.glob("*.cu")) + list(CSRC.glob("*.cuh")) + list(CSRC.glob("*.inl")) +
            list(INCLUDE.glob("*.h")))


def is_current(library: Path = LIBRARY) -> bool:
    return library.exists() and all(library.stat().st_mtime >= f.stat().st_mtime for f in _inputs())


def build(force: bool = False, verbose: bool = False, checked: bool = False) -> Path:
    """nvcc -> libinstinfer.so (or, with checked=True, the bounds-checking build
    libinstinfer_checked.so, in which every data-dependent global offset is tested against the
    extent the call's shapes imply and a violation sets status bit 8 instead of being used);
    skipped when the library is newer than every source."""
    library = CHECKED_LIBRARY if checked else LIBRARY
    if not force and is_current(library):
        return library
    extra = ["-DINSTINFER_BOUNDS_CHECK"] if checked else []
    stem = f"{library.stem}.{os.getpid()}.tmp"
    objects = [library.with_name(f"{stem}.{source.stem}.o") for source in SOURCES]
    tmp = library.with_name(f"{stem}.so")

    def run(*args):
        done = subprocess.run([_nvcc(), *NVCC_FLAGS, *args], capture_output=True, text=True)
        if verbose or done.returncode:
            print(done.stdout + done.stderr)
        if done.returncode:
            raise RuntimeError("nvcc failed")

    try:
        with ThreadPoolExecutor(max_workers=len(SOURCES)) as pool:      # the sources side by side
            jobs = [pool.submit(run, *extra, "-I", str(INCLUDE), "-c", str(source), "-o", str(obj))
                    for source, obj in zip(SOURCES, objects)]
            for job in jobs:
                job.result()
        run("-shared", *map(str, objects), "-o", str(tmp))
    finally:
        for obj in objects:
            obj.unlink(missing_ok=True)
    os.replace(tmp, library)
    return library


if __name__ == "__main__":
    print(build(force=True, verbose=True))
    print(build(force=True, checked=True))
