"""Builds the C-ABI shared library (liblibra.so) in-tree with nvcc for sm_100a.

nvcc cross-compiles without a GPU, so this also runs on a CPU-only machine.  The CUDA runtime is
linked statically and the driver API is reached through the runtime's entry-point lookup, so the
library loads on machines without a driver (the planner entry point needs no GPU).
"""
from __future__ import annotations

import concurrent.futures
import contextlib
import hashlib
import os
import re
import subprocess
import sys

HERE = os.path.dirname(os.path.abspath(__file__))
ROOT = os.path.dirname(HERE)
CSRC = os.path.join(HERE, "csrc")
INCLUDE = os.path.join(ROOT, "include")
LIB_PATH = os.path.join(HERE, "liblibra.so")
STAMP_PATH = os.path.join(HERE, "liblibra.so.stamp")

SOURCES = ["libra_api.cu", "rope_api.cu", "chunk_api.cu", "norm_api.cu", "table_api.cu", "tree_api.cu",
           "planner.cpp", "sched.cpp", "ring_sched.cpp", "rope.cpp", "chunk_plan.cpp"]
NVCC_FLAGS = [
    "-gencode", "arch=compute_100a,code=sm_100a", "-lineinfo", "-O3", "-std=c++17",
    "--use_fast_math", "-Xcompiler", "-fPIC",
]
LINK_FLAGS = ["-gencode", "arch=compute_100a,code=sm_100a", "-shared", "-cudart", "static"]
OBJ_DIR = os.path.join(HERE, "build")   # objects of the last build, kept so that only what changed is compiled again


def _nvcc() -> str:
    for cand in (os.environ.get("NVCC"), "/usr/local/cuda/bin/nvcc", "nvcc"):
        if cand and (os.path.isabs(cand) and os.path.exists(cand) or not os.path.isabs(cand)):
            return cand
    raise RuntimeError("nvcc not found")


def _source_digest(extra_flags) -> str:
    h = hashlib.sha256()
    names = sorted(os.listdir(CSRC)) + [os.path.join(INCLUDE, "libra.h")]
    for n in names:
        path = n if os.path.isabs(n) else os.path.join(CSRC, n)
        with open(path, "rb") as f:
            h.update(n.encode() + b"\0" + f.read())
    h.update(" ".join(SOURCES + NVCC_FLAGS + LINK_FLAGS + list(extra_flags)).encode())
    return h.hexdigest()


def _object_digest(source: str, extra_flags) -> str:
    """Digest of one source and of every file of csrc / include that it includes, directly or not."""
    h, todo, seen = hashlib.sha256(), [os.path.join(CSRC, source)], set()
    while todo:
        path = todo.pop()
        if path in seen:
            continue
        seen.add(path)
        with open(path, "rb") as f:
            text = f.read()
        h.update(os.path.basename(path).encode() + b"\0" + text)
        for name in re.findall(rb'^\s*#\s*include\s+"([^"]+)"', text, flags=re.M):
            for d in (CSRC, INCLUDE):
                inc = os.path.join(d, name.decode())
                if os.path.exists(inc):
                    todo.append(inc)
                    break
    h.update(" ".join(NVCC_FLAGS + list(extra_flags)).encode())
    return h.hexdigest()


def build_library(force: bool = False, verbose: bool = True, extra_flags=()) -> str:
    """Compile if the sources changed since the last build; returns the library path."""
    digest = _source_digest(extra_flags)
    if not force and os.path.exists(LIB_PATH) and os.path.exists(STAMP_PATH):
        with open(STAMP_PATH) as f:
            if f.read().strip() == digest:
                return LIB_PATH
    os.makedirs(OBJ_DIR, exist_ok=True)
    with contextlib.suppress(FileNotFoundError):   # as for the objects below
        os.remove(STAMP_PATH)

    def run(cmd):
        if verbose:
            print(" ".join(cmd), flush=True)
        return subprocess.run(cmd, capture_output=True, text=True)

    def compile_one(source):
        obj = os.path.join(OBJ_DIR, source + ".o")
        stamp, own = obj + ".stamp", _object_digest(source, extra_flags)
        if not force and os.path.exists(obj) and os.path.exists(stamp):
            with open(stamp) as f:
                if f.read().strip() == own:
                    return obj, None
        with contextlib.suppress(FileNotFoundError):   # it vouches for the object that is about to be overwritten
            os.remove(stamp)
        res = run([_nvcc(), *NVCC_FLAGS, *extra_flags, "-I", INCLUDE, "-I", CSRC, "-c", os.path.join(CSRC, source), "-o", obj])
        if res.returncode == 0:
            with open(stamp, "w") as f:
                f.write(own)
        return obj, res

    with concurrent.futures.ThreadPoolExecutor(max_workers=max(1, os.cpu_count() or 1)) as pool:
        built = list(pool.map(compile_one, SOURCES))
    results = [r for _, r in built if r is not None]
    if all(r.returncode == 0 for r in results):
        results.append(run([_nvcc(), *LINK_FLAGS, *[o for o, _ in built], "-o", LIB_PATH]))
    failed = any(r.returncode != 0 for r in results)
    if verbose or failed:
        sys.stderr.write("".join(r.stdout + r.stderr for r in results))
    if failed:
        raise RuntimeError("nvcc failed")
    with open(STAMP_PATH, "w") as f:
        f.write(digest)
    return LIB_PATH


if __name__ == "__main__":
    build_library(force="--force" in sys.argv, extra_flags=[a for a in sys.argv[1:] if a.startswith(("-X", "-D"))])
