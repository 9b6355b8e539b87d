"""Build the CUDA library in-tree: nvcc, sm_100a only, one shared object.  Sources are compiled side by side and only where they, or a header, are newer than their object."""
from __future__ import annotations

import glob
import os
import shlex
import subprocess
import sys
from concurrent.futures import ThreadPoolExecutor

HERE = os.path.dirname(os.path.abspath(__file__))
CSRC = os.path.join(HERE, "csrc")
SO = os.path.join(HERE, "libwwws.so")
SO_CHECKED = os.path.join(HERE, "libwwws_checked.so")     # -DWWWS_CHECK_INDICES: indices taken from device data are range-checked

NVCC_FLAGS = ["-gencode", "arch=compute_100a,code=sm_100a", "-lineinfo", "-O3", "-std=c++17",
              "-fmad=false", "-Xcompiler", "-fPIC", "-shared", "--use_fast_math=false"]


def sources():
    return sorted(glob.glob(os.path.join(CSRC, "*.cu")))


def needs_build() -> bool:
    if not os.path.exists(SO):
        return True
    t = os.path.getmtime(SO)
    deps = sources() + glob.glob(os.path.join(CSRC, "*.cuh")) + glob.glob(os.path.join(HERE, "..", "include", "*.h"))
    return any(os.path.getmtime(p) > t for p in deps)


def build(force: bool = False, verbose: bool = False, checked: bool = False) -> str:
    """Compile the library; `checked` builds the variant with index checks beside it
    (load it by setting WWWS_LIBRARY to its path)."""
    if not checked and not force and not needs_build():
        return SO
    nvcc = os.environ.get("NVCC", "/usr/local/cuda/bin/nvcc")
    flags = [f for f in NVCC_FLAGS if f != "--use_fast_math=false"] + shlex.split(os.environ.get("WWWS_NVCC_EXTRA", ""))
    flags += (["-DWWWS_CHECK_INDICES"] if checked else []) + (["-Xptxas", "-v"] if verbose else [])
    out = SO_CHECKED if checked else SO
    objects = os.path.join(HERE, "_build", "checked" if checked else "plain")
    os.makedirs(objects, exist_ok=True)
    headers = max(os.path.getmtime(p) for p in glob.glob(os.path.join(CSRC, "*.cuh")) + glob.glob(os.path.join(HERE, "..", "include", "*.h")))

    def compile_one(src):
        obj = os.path.join(objects, os.path.basename(src) + ".o")
        if force or verbose or not os.path.exists(obj) or os.path.getmtime(obj) < max(headers, os.path.getmtime(src)) or "WWWS_NVCC_EXTRA" in os.environ:
            part = f"{obj}.{os.getpid()}"                   # (two builds at once do not read each other's unfinished objects)
            subprocess.check_call([nvcc] + [f for f in flags if f != "-shared"] + ["-c", "-o", part, src])
            os.replace(part, obj)
        return obj

    with ThreadPoolExecutor(max(1, os.cpu_count() or 1)) as pool:
        objs = list(pool.map(compile_one, sorted(sources(), key=os.path.getsize, reverse=True)))
    part = f"{out}.{os.getpid()}"
    subprocess.check_call([nvcc] + flags + ["-o", part] + sorted(objs))
    os.replace(part, out)
    return out


if __name__ == "__main__":
    print(build(force="--force" in sys.argv, verbose="-v" in sys.argv, checked="--checked" in sys.argv))
