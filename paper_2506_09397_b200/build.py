"""Builds the CUDA library (libsled.so) in-tree with nvcc for sm_100a, and the compiled part of the binding (_marshal.so)."""
from __future__ import annotations

import os
import subprocess
import sys
import sysconfig
from concurrent.futures import ThreadPoolExecutor
from importlib.metadata import version

HERE = os.path.dirname(os.path.abspath(__file__))
CSRC = os.path.join(HERE, "csrc")
OBJ = os.path.join(HERE, "_build")
LIB = os.path.join(HERE, "libsled.so")
MARSHAL = os.path.join(HERE, "_marshal.so")
SOURCES = ["engine.cu", "kernels_small.cu", "attention.cu", "attention_mma.cu", "attention_tc.cu", "accept.cu", "gemm_tc.cu", "kv_manager.cpp", "planner.cpp", "no_alloc.cu",
           "paged_attention.cu", "paged_mma.cu", "paged_tc.cu", "paged_f32.cu", "paged_weigh.cu", "paged_blocks.cu", "paged_evict.cu", "paged_slots.cu", "rotary.cu", "paged_append.cu", "paged_scaled.cu", "paged_scaled_tc.cu", "paged_api.cu"]
NVCC_FLAGS = ["-std=c++17", "-O3", "-gencode", "arch=compute_100a,code=sm_100a", "-lineinfo",
              "-Xcompiler", "-fPIC", "-Xcompiler", "-Wall"]


def _nvcc() -> str:
    for cand in (os.environ.get("NVCC"), "/usr/local/cuda/bin/nvcc", "nvcc"):
        if cand and (os.path.isabs(cand) and os.path.exists(cand) or not os.path.isabs(cand)):
            return cand
    return "nvcc"


def _stale(target: str, deps) -> bool:
    if not os.path.exists(target):
        return True
    t = os.path.getmtime(target)
    return any(os.path.getmtime(d) > t for d in deps)


def build(force: bool = False, verbose: bool = False) -> str:
    os.makedirs(OBJ, exist_ok=True)
    headers = [os.path.join(CSRC, f) for f in os.listdir(CSRC) if f.endswith((".h", ".cuh"))]
    headers.append(os.path.join(HERE, "..", "include", "sled.h"))
    nvcc = _nvcc()
    jobs = []
    for src in SOURCES:
        sp = os.path.join(CSRC, src)
        op = os.path.join(OBJ, os.path.splitext(src)[0] + ".o")
        if force or _stale(op, [sp] + headers):
            extra = ["-Xptxas", "-v"] if verbose else []
            jobs.append([nvcc] + NVCC_FLAGS + extra + ["-x", "cu", "-c", sp, "-o", op])

    def run(cmd):
        r = subprocess.run(cmd, capture_output=True, text=True)
        if r.returncode != 0 or verbose:
            sys.stderr.write(r.stdout + r.stderr)
        if r.returncode != 0:
            raise RuntimeError("nvcc failed: " + " ".join(cmd))

    with ThreadPoolExecutor(max_workers=6) as ex:
        list(ex.map(run, jobs))
    objs = [os.path.join(OBJ, os.path.splitext(s)[0] + ".o") for s in SOURCES]
    if force or jobs or _stale(LIB, objs):
        tmp = LIB + f".{os.getpid()}.tmp"
        run([nvcc, "-shared", "-o", tmp] + objs + ["-gencode", "arch=compute_100a,code=sm_100a"])
        os.replace(tmp, LIB)
    build_marshal(force, run)
    return LIB


def marshal_for() -> str:
    """What _marshal.so is tied to: the versions of torch and of Python whose classes it was compiled against."""
    return f"torch {version('torch')}, {sysconfig.get_config_var('SOABI')}"


def build_marshal(force: bool, run) -> None:
    """The binding's argument marshalling, against torch's headers; it finds libsled.so beside itself.  Built again for another torch or
    Python, too."""
    source, note, tied_to = os.path.join(CSRC, "marshal.cpp"), os.path.join(OBJ, "marshal.txt"), marshal_for()
    built_for = ""
    if os.path.exists(note):
        with open(note) as f:
            built_for = f.read()
    if not force and built_for == tied_to and not _stale(MARSHAL, [source, os.path.join(HERE, "..", "include", "sled.h")]):
        return
    import torch
    root = os.path.dirname(torch.__file__)
    cuda = os.path.join(os.path.dirname(os.path.dirname(_nvcc())), "include") if os.path.isabs(_nvcc()) else "/usr/local/cuda/include"
    tmp = MARSHAL + f".{os.getpid()}.tmp"
    run(["g++", "-std=c++17", "-O2", "-shared", "-fPIC", "-Wall", f"-D_GLIBCXX_USE_CXX11_ABI={int(torch._C._GLIBCXX_USE_CXX11_ABI)}",
         "-isystem", os.path.join(root, "include"), "-isystem", os.path.join(root, "include", "torch", "csrc", "api", "include"),
         f'-DSLED_BUILT_FOR="{tied_to}"', "-isystem", sysconfig.get_paths()["include"], "-isystem", cuda, source, "-o", tmp, "-L" + os.path.join(root, "lib"), "-ltorch_python",
         "-ltorch", "-ltorch_cpu", "-lc10", "-lc10_cuda", "-L" + HERE, "-l:libsled.so", "-Wl,-rpath,$ORIGIN"])
    os.replace(tmp, MARSHAL)
    with open(note, "w") as f:
        f.write(tied_to)


if __name__ == "__main__":
    print(build(force="--force" in sys.argv, verbose="-v" in sys.argv))
