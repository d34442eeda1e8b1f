"""Builds the C-ABI CUDA library in-tree: ``paper_2502_06833_b200/libead_b200.so``.

sm_100a only (tcgen05 / TMEM / TMA); nvcc cross-compiles without a GPU.
Run as ``python -m paper_2502_06833_b200.build [--force] [--verbose]``.
"""
from __future__ import annotations

import os
import subprocess
import sys

_DIR = os.path.dirname(os.path.abspath(__file__))
_ROOT = os.path.dirname(_DIR)
_CSRC = os.path.join(_DIR, "csrc")
_OBJ = os.path.join(_DIR, "build")
LIB_PATH = os.path.join(_DIR, "libead_b200.so")
SOURCES = [os.path.join(_CSRC, f) for f in ("ead_api.cu", "ead_decoder_api.cu", "ead_pass_api.cu")]
_FLAGS = ["-std=c++17", "-O3", "-lineinfo", "-gencode", "arch=compute_100a,code=sm_100a", "-Xcompiler", "-fPIC,-O2,-Wall"]


def _nvcc() -> str:
    return os.environ.get("NVCC", "/usr/local/cuda/bin/nvcc")


def _object(source: str) -> str:
    return os.path.join(_OBJ, os.path.splitext(os.path.basename(source))[0] + ".o")


def _stale(target: str, deps) -> bool:
    return not os.path.exists(target) or any(not os.path.exists(d) or os.path.getmtime(d) > os.path.getmtime(target) for d in deps)


def _deps(source: str):
    """What the object of a source depends on in this repository: this file (it has the flags), the source, and the headers that it was last compiled
    with; all headers where no list of this checkout says which."""
    headers = [os.path.join(_CSRC, f) for f in os.listdir(_CSRC)] + [os.path.join(_ROOT, "include", "ead.h")]
    try:
        with open(_object(source) + ".d") as f:
            words = f.read().replace("\\\n", " ").split()[1:]
    except OSError:
        words = []
    words = [os.path.normpath(os.path.join(_DIR, w)) for w in words if w != ":"]      # (compiled in _DIR by paths relative to it: a copied tree has its own files)
    if source in words:
        headers = [w for w in words if w.startswith(_ROOT + os.sep)]
    return [os.path.abspath(__file__), source, *headers]


def build(force: bool = False, verbose: bool = False) -> str:
    os.makedirs(_OBJ, exist_ok=True)
    jobs = []
    for s in SOURCES:
        if force or _stale(_object(s), _deps(s)):
            cmd = [_nvcc(), *_FLAGS, "-MD", "-MF", _object(s) + ".d", "-c", os.path.relpath(s, _DIR), "-o", _object(s)]
            jobs.append(subprocess.Popen(cmd[:1] + (["-Xptxas=-v"] if verbose else []) + cmd[1:], cwd=_DIR, text=True,
                                         stdout=subprocess.PIPE, stderr=subprocess.STDOUT))
    said = [j.communicate()[0] for j in jobs]
    if verbose or any(j.returncode for j in jobs):
        sys.stderr.write("".join(said))
    if any(j.returncode for j in jobs):
        raise RuntimeError("nvcc failed building libead_b200.so")
    objects = [_object(s) for s in SOURCES]
    if jobs or _stale(LIB_PATH, objects):
        res = subprocess.run([_nvcc(), "-shared", "-cudart", "static", "-gencode", "arch=compute_100a,code=sm_100a", "-o", LIB_PATH, *objects],
                             capture_output=True, text=True)
        if res.returncode:
            sys.stderr.write(res.stdout + res.stderr)
            raise RuntimeError("nvcc failed linking libead_b200.so")
    return LIB_PATH


if __name__ == "__main__":
    print(build(force="--force" in sys.argv, verbose="--verbose" in sys.argv))
