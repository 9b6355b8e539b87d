"""Build the CUDA library in-tree: nvcc, sm_100a only, one shared object.  Sources are compiled side by side, and only where something they were made from is newer than
their object or the flags are others."""
from __future__ import annotations

import glob
import hashlib
import os
import shlex
import subprocess
import sys
import time
from concurrent.futures import ThreadPoolExecutor

HERE = os.path.dirname(os.path.abspath(__file__))
CSRC = os.path.join(HERE, "csrc")
SO = os.path.join(HERE, "libwwws.so")
SO_CHECKED = os.path.join(HERE, "libwwws_checked.so")     # -DWWWS_CHECK_INDICES: indices taken from device data are range-checked

NVCC = "/usr/local/cuda/bin/nvcc"
NVCC_FLAGS = ["-gencode", "arch=compute_100a,code=sm_100a", "-lineinfo", "-O3", "-std=c++17",
              "-fmad=false", "-Xcompiler", "-fPIC", "-shared", "--use_fast_math=false"]


def sources():
    return sorted(glob.glob(os.path.join(CSRC, "*.cu")))


def flags_of(checked: bool = False, verbose: bool = False):
    return [f for f in NVCC_FLAGS if f != "--use_fast_math=false"] + shlex.split(os.environ.get("WWWS_NVCC_EXTRA", "")) + \
        (["-DWWWS_CHECK_INDICES"] if checked else []) + (["-Xptxas", "-v"] if verbose else [])


def key_of(flags) -> str:
    """Names what objects are compiled with: those of other flags or another compiler lie in folders of their own."""
    return hashlib.sha256("\0".join([os.environ.get("NVCC", NVCC)] + flags).encode()).hexdigest()[:12]


def linked_with(checked: bool = False) -> str:
    """The file beside the objects that says what the library was last linked from: its key and its sources."""
    return os.path.join(HERE, "_build", "checked.txt" if checked else "plain.txt")


def signature(flags) -> str:
    return " ".join([key_of(flags)] + [os.path.basename(p) for p in sources()])


def needs_build() -> bool:
    if not os.path.exists(SO):
        return True
    if os.path.exists(linked_with()):
        with open(linked_with()) as f:
            if f.read() != signature(flags_of()):
                return True
    t = os.path.getmtime(SO)
    deps = sources() + glob.glob(os.path.join(CSRC, "*.cuh")) + glob.glob(os.path.join(HERE, "..", "include", "*.h"))
    return any(os.path.getmtime(p) > t for p in deps)


def fresh(obj: str) -> bool:
    """Whether an object is newer than everything it was compiled from, which the compiler wrote down beside it (a source may include another one)."""
    if not os.path.exists(obj) or not os.path.exists(obj + ".d"):
        return False
    with open(obj + ".d") as f:
        made_from = shlex.split(f.read().replace("\\\n", " ").partition(":")[2])
    t = os.path.getmtime(obj)
    return bool(made_from) and all(os.path.exists(p) and os.path.getmtime(p) < t for p in made_from)


def build(force: bool = False, verbose: bool = False, checked: bool = False) -> str:
    """Compile the library; `checked` builds the variant with index checks beside it
    (load it by setting WWWS_LIBRARY to its path)."""
    if not checked and not force and not needs_build():
        return SO
    nvcc, flags = os.environ.get("NVCC", NVCC), flags_of(checked, verbose)
    out = SO_CHECKED if checked else SO
    objects = os.path.join(HERE, "_build", key_of(flags))
    os.makedirs(objects, exist_ok=True)
    began = time.time()                                     # what is made counts as old as that: a source saved meanwhile is newer

    def compile_one(src):
        obj = os.path.join(objects, os.path.basename(src) + ".o")
        if force or verbose or not fresh(obj):
            part = f"{obj}.{os.getpid()}"                   # (two builds at once do not read each other's unfinished objects)
            subprocess.check_call([nvcc] + [f for f in flags if f != "-shared"] + ["-c", "-MMD", "-MF", part + ".d", "-o", part, src])
            os.utime(part, (began, began))
            os.replace(part + ".d", obj + ".d")
            os.replace(part, obj)
        return obj

    with ThreadPoolExecutor(max(1, os.cpu_count() or 1)) as pool:
        objs = list(pool.map(compile_one, sorted(sources(), key=os.path.getsize, reverse=True)))
    part = f"{out}.{os.getpid()}"
    subprocess.check_call([nvcc] + flags + ["-o", part] + sorted(objs))
    os.utime(part, (began, began))
    os.replace(part, out)
    with open(linked_with(checked), "w") as f:
        f.write(signature(flags))
    return out


if __name__ == "__main__":
    print(build(force="--force" in sys.argv, verbose="-v" in sys.argv, checked="--checked" in sys.argv))
