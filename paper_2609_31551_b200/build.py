"""In-tree build of the CUDA library (sm_100a only).  nvcc cross-compiles without a GPU."""
from __future__ import annotations
import os
import subprocess
from concurrent.futures import ThreadPoolExecutor

HERE = os.path.dirname(os.path.abspath(__file__))
CSRC = os.path.join(HERE, "csrc")
LIB_PATH = os.path.join(HERE, "libeas_encoder.so")
SOURCES = ["eas_encoder.cu", "eas_language.cu", "serving_host.cpp"]
NVCC_FLAGS = ["-O3", "-std=c++17", "-gencode", "arch=compute_100a,code=sm_100a", "-lineinfo", "-Xcompiler", "-fPIC"]


def _newest_source_mtime() -> float:
    newest = 0.0
    for root in (CSRC, os.path.join(os.path.dirname(HERE), "include")):
        for name in os.listdir(root):
            if not name.endswith((".o", ".d")):
                newest = max(newest, os.path.getmtime(os.path.join(root, name)))
    return newest


def _run(cmd):
    res = subprocess.run(cmd, capture_output=True, text=True)
    if res.returncode != 0:
        raise RuntimeError("nvcc failed:\n" + res.stdout + res.stderr)
    return res.stderr


def _object_is_current(obj: str, deps: str) -> bool:
    """True if the object is newer than everything its last compilation read (the dependency file lists it)."""
    if not (os.path.exists(obj) and os.path.exists(deps)):
        return False
    built = os.path.getmtime(obj)
    with open(deps) as f:
        names = f.read().replace("\\\n", " ").split(":", 1)[1].split()
    return all(os.path.exists(n) and os.path.getmtime(n) < built for n in names)


def build_library(force: bool = False, verbose: bool = False) -> str:
    """Compile csrc/ into libeas_encoder.so next to this file (sources side by side); returns the library path."""
    if not force and os.path.exists(LIB_PATH) and os.path.getmtime(LIB_PATH) >= _newest_source_mtime():
        return LIB_PATH
    nvcc = os.environ.get("NVCC", "/usr/local/cuda/bin/nvcc")

    def compile_one(src):
        path = os.path.join(CSRC, src)
        obj, deps = path + ".o", path + ".d"
        if not force and _object_is_current(obj, deps):
            return obj, ""
        return obj, _run([nvcc] + NVCC_FLAGS + (["-Xptxas", "-v"] if verbose else []) + ["-MD", "-MF", deps, "-c", "-o", obj, path])

    with ThreadPoolExecutor(len(SOURCES)) as pool:
        done = list(pool.map(compile_one, SOURCES))
    _run([nvcc] + NVCC_FLAGS + ["-shared", "-o", LIB_PATH] + [obj for obj, _ in done])
    if verbose:
        print("".join(text for _, text in done))
    return LIB_PATH


if __name__ == "__main__":
    import sys
    print(build_library(force="--incremental" not in sys.argv, verbose=True))
