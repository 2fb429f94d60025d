"""Builds libsawtooth_attn.so (the C-ABI library) in-tree with nvcc for sm_100a, and beside it the torch module of paged.py."""
from __future__ import annotations

import os
import subprocess

PKG = os.path.dirname(os.path.abspath(__file__))
CSRC = os.path.join(PKG, "csrc")
ROOT = os.path.dirname(PKG)
LIB = os.path.join(PKG, "libsawtooth_attn.so")
TORCH_LIB = os.path.join(PKG, "_torch_binding.so")   # a Python module
OBJ = os.path.join(PKG, "_build")
_HEADER = os.path.join(ROOT, "include", "sawtooth_attn.h")
# Each source with the headers it includes (it is compiled again when one of them is newer than its object file).
SOURCES = {
    "api.cu": ("attn_fwd_sm100.cuh", "ptx.cuh", "schedule.h", "host.h"),
    "paged.cu": ("ptx.cuh", "host.h", "paged_common.cuh", "page_plan.cuh", "qk_norm_rope.cuh", "decode_sm100.cuh", "decode_schedule.h"),
}
TORCH_SOURCE = "torch_binding.cpp"


def _deps(source: str) -> list:
    return [os.path.join(CSRC, f) for f in (source,) + SOURCES.get(source, ())] + [_HEADER]


DEPS = sorted({f for source in list(SOURCES) + [TORCH_SOURCE] for f in _deps(source)})

NVCC_FLAGS = [
    "-std=c++17", "-O3", "-lineinfo",
    "-gencode", "arch=compute_100a,code=sm_100a",
    "-Xcompiler", "-fPIC",
]


def _older(target: str, files: list) -> bool:
    return not os.path.exists(target) or any(os.path.getmtime(f) > os.path.getmtime(target) for f in files)


def is_stale() -> bool:
    return any(_older(LIB, _deps(source)) for source in SOURCES) or _older(TORCH_LIB, _deps(TORCH_SOURCE))


def _torch_commands(obj: str) -> tuple:
    """The compiler calls for the torch module: its object file, and the module linked against the library beside it."""
    import sysconfig

    from torch.utils import cpp_extension
    cxx, cuda = os.environ.get("CXX", "g++"), os.environ.get("CUDA_HOME", "/usr/local/cuda")
    includes = [f"-I{d}" for d in cpp_extension.include_paths() + [os.path.join(cuda, "include"), sysconfig.get_paths()["include"]]]
    libraries = [f"-L{d}" for d in cpp_extension.library_paths()]
    return ([cxx, "-std=c++17", "-O2", "-fPIC", "-DTORCH_EXTENSION_NAME=_torch_binding"] + includes + ["-c", "-o", obj, os.path.join(CSRC, TORCH_SOURCE)],
            [cxx, "-shared", "-o", TORCH_LIB, obj] + libraries + ["-L" + PKG, "-lsawtooth_attn", "-lc10", "-lc10_cuda", "-ltorch_cpu", "-ltorch_cuda", "-ltorch",
                                                                    "-ltorch_python", "-Wl,-rpath,$ORIGIN"])


def build(force: bool = False, verbose: bool = False) -> str:
    """Compiles the sources that changed (side by side) and links the library and the torch module."""
    if not force and not is_stale():
        return LIB
    nvcc = os.environ.get("NVCC", "/usr/local/cuda/bin/nvcc")
    os.makedirs(OBJ, exist_ok=True)
    running, objects = [], []
    for source in SOURCES:
        obj = os.path.join(OBJ, source[:-3] + ".o")
        objects.append(obj)
        if force or _older(obj, _deps(source)):
            cmd = [nvcc] + NVCC_FLAGS + (["-Xptxas", "-v"] if verbose else []) + ["-c", "-o", obj, os.path.join(CSRC, source)]
            running.append((cmd, obj, subprocess.Popen(cmd)))
    torch_obj = os.path.join(OBJ, "torch_binding.o")
    compile_torch, link_torch = _torch_commands(torch_obj)
    if force or _older(torch_obj, _deps(TORCH_SOURCE)):
        running.append((compile_torch, torch_obj, subprocess.Popen(compile_torch)))
    failed = [(cmd, obj, p.returncode) for cmd, obj, p in running if p.wait() != 0]
    if failed:
        for _, obj, _ in failed:
            if os.path.exists(obj):
                os.remove(obj)
        raise subprocess.CalledProcessError(failed[0][2], failed[0][0])
    subprocess.run([nvcc, "-gencode", "arch=compute_100a,code=sm_100a", "-shared", "-cudart", "static", "-o", LIB] + objects, check=True)
    subprocess.run(link_torch, check=True)
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
