"""Builds libsawtooth_attn.so (the C-ABI library) in-tree with nvcc for sm_100a."""
from __future__ import annotations

import os
import subprocess

PKG = os.path.dirname(os.path.abspath(__file__))
CSRC = os.path.join(PKG, "csrc")
ROOT = os.path.dirname(PKG)
LIB = os.path.join(PKG, "libsawtooth_attn.so")
OBJ = os.path.join(PKG, "_build")
_HEADER = os.path.join(ROOT, "include", "sawtooth_attn.h")
# Each source with the headers it includes (it is compiled again when one of them is newer than its object file).
SOURCES = {
    "api.cu": ("attn_fwd_sm100.cuh", "ptx.cuh", "schedule.h", "host.h"),
    "paged.cu": ("ptx.cuh", "host.h", "paged_common.cuh", "page_plan.cuh", "qk_norm_rope.cuh"),
}


def _deps(source: str) -> list:
    return [os.path.join(CSRC, f) for f in (source,) + SOURCES[source]] + [_HEADER]


DEPS = sorted({f for source in SOURCES for f in _deps(source)})

NVCC_FLAGS = [
    "-std=c++17", "-O3", "-lineinfo",
    "-gencode", "arch=compute_100a,code=sm_100a",
    "-Xcompiler", "-fPIC",
]


def is_stale() -> bool:
    if not os.path.exists(LIB):
        return True
    t = os.path.getmtime(LIB)
    return any(os.path.getmtime(f) > t for f in DEPS)


def build(force: bool = False, verbose: bool = False) -> str:
    """Compiles the sources that changed (side by side) and links the library."""
    if not force and not is_stale():
        return LIB
    nvcc = os.environ.get("NVCC", "/usr/local/cuda/bin/nvcc")
    os.makedirs(OBJ, exist_ok=True)
    running, objects = [], []
    for source in SOURCES:
        obj = os.path.join(OBJ, source[:-3] + ".o")
        objects.append(obj)
        if force or not os.path.exists(obj) or any(os.path.getmtime(f) > os.path.getmtime(obj) for f in _deps(source)):
            cmd = [nvcc] + NVCC_FLAGS + (["-Xptxas", "-v"] if verbose else []) + ["-c", "-o", obj, os.path.join(CSRC, source)]
            running.append((cmd, obj, subprocess.Popen(cmd)))
    failed = [(cmd, obj, p.returncode) for cmd, obj, p in running if p.wait() != 0]
    if failed:
        for _, obj, _ in failed:
            if os.path.exists(obj):
                os.remove(obj)
        raise subprocess.CalledProcessError(failed[0][2], failed[0][0])
    subprocess.run([nvcc, "-gencode", "arch=compute_100a,code=sm_100a", "-shared", "-cudart", "static", "-o", LIB] + objects, check=True)
    return LIB


HOST_CALL_SRC = os.path.join(ROOT, "profile_host_call.cu")
HOST_CALL_BIN = os.path.join(PKG, "profile_host_call")


def build_host_call_probe(force: bool = False) -> str:
    """Builds the C program that times one attn_fwd call from C (a measuring aid of bench.py) against the in-tree library."""
    build()
    if not force and os.path.exists(HOST_CALL_BIN) and os.path.getmtime(HOST_CALL_BIN) >= max(os.path.getmtime(HOST_CALL_SRC), os.path.getmtime(LIB)):
        return HOST_CALL_BIN
    nvcc = os.environ.get("NVCC", "/usr/local/cuda/bin/nvcc")
    cmd = [nvcc, "-O2", "-std=c++17", "-gencode", "arch=compute_100a,code=sm_100a", "-o", HOST_CALL_BIN, HOST_CALL_SRC,
           "-L" + PKG, "-lsawtooth_attn", "-Xlinker", "-rpath", "-Xlinker", "$ORIGIN"]
    subprocess.run(cmd, check=True, cwd=ROOT)
    return HOST_CALL_BIN


if __name__ == "__main__":
    import sys
    print(build(force=True, verbose="-v" in sys.argv))
    print(build_host_call_probe(force=True))
