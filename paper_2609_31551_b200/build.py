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


def _newest_mtime() -> float:
    """Of the sources and objects: the library is newer, or its linking failed."""
    newest = 0.0
    for root in (CSRC, os.path.join(os.path.dirname(HERE), "include")):
        for name in os.listdir(root):
            if not name.endswith(".d"):
                newest = max(newest, os.path.getmtime(os.path.join(root, name)))
    return newest


def _run(cmd):
    res = subprocess.run(cmd, capture_output=True, text=True)
    if res.returncode != 0:
        raise RuntimeError("nvcc failed:\n" + res.stdout + res.stderr)
    return res.stderr


def _paths(src: str):
    path = os.path.join(CSRC, src)
    return path, path + ".o", path + ".d"


def _compiler():
    """The compiler and its flags; the compiler by its real path, which names its version."""
    return [os.path.realpath(os.environ.get("NVCC", "/usr/local/cuda/bin/nvcc"))] + NVCC_FLAGS


_MADE_BY = "# made by: "           # last line of a dependency file: the compiler and the flags that it was written by


def _made_by(src: str):
    """-> the compiler and flags that made a source's object, or None."""
    try:
        with open(_paths(src)[2]) as f:
            last = f.read().rstrip("\n").rsplit("\n", 1)[-1]
    except OSError:
        return None
    return last[len(_MADE_BY):] if last.startswith(_MADE_BY) else None


def _object_is_current(src: str) -> bool:
    """True if the object was made by the present compiler and flags and is newer than everything that compilation read (the dependency file lists it)."""
    _, obj, deps = _paths(src)
    if not os.path.exists(obj) or _made_by(src) != " ".join(_compiler()):
        return False
    built = os.path.getmtime(obj)
    with open(deps) as f:
        names = f.read().split(_MADE_BY)[0].replace("\\\n", " ").split(":", 1)[1].split()
    return all(os.path.exists(n) and os.path.getmtime(n) < built for n in names)


def build_library(force: bool = False, verbose: bool = False) -> str:
    """Compile csrc/ into libeas_encoder.so next to this file (sources side by side); returns the library path."""
    if (not force and os.path.exists(LIB_PATH) and os.path.getmtime(LIB_PATH) >= _newest_mtime()
            and all(_made_by(src) == " ".join(_compiler()) or not os.path.exists(_paths(src)[2]) for src in SOURCES)):
        return LIB_PATH

    def compile_one(src):
        path, obj, deps = _paths(src)
        if not force and _object_is_current(src):
            return obj, ""
        text = _run(_compiler() + (["-Xptxas", "-v"] if verbose else []) + ["-MD", "-MF", deps, "-c", "-o", obj, path])
        with open(deps, "a") as f:
            f.write(_MADE_BY + " ".join(_compiler()) + "\n")
        return obj, text

    with ThreadPoolExecutor(len(SOURCES)) as pool:
        done = list(pool.map(compile_one, SOURCES))
    _run(_compiler() + ["-shared", "-o", LIB_PATH] + [obj for obj, _ in done])
    if verbose:
        print("".join(text for _, text in done))
    return LIB_PATH


if __name__ == "__main__":
    import sys
    print(build_library(force="--incremental" not in sys.argv, verbose=True))
