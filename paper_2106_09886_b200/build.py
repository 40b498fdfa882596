"""Build libqnn.so from csrc/*.cu with nvcc for sm_100a (no torch involved), and the tensor-argument module of the binding,
_binding.so, from csrc/binding.cpp with the host compiler against the installed torch.

    python -m paper_2106_09886_b200.build [--force]
"""
from __future__ import annotations

import hashlib
import importlib.util
import os
import subprocess
import sys
import sysconfig
from concurrent.futures import ThreadPoolExecutor
from pathlib import Path

PKG = Path(__file__).resolve().parent
CSRC = PKG / "csrc"
INCLUDE = PKG.parent / "include"
LIB = PKG / "libqnn.so"
BINDING = PKG / "_binding.so"
STAMP = PKG / "libqnn.so.digest"

COMPILE_FLAGS = [
    "-gencode", "arch=compute_100a,code=sm_100a", "-lineinfo", "-O3", "-std=c++17",
    "--fmad=false",            # no silent contraction: every fused multiply-add is written explicitly
    "-Xcompiler", "-fPIC", "-Xcompiler", "-O2",
]
LINK_FLAGS = ["-gencode", "arch=compute_100a,code=sm_100a", "-shared", "-Xcompiler", "-fPIC"]


def sources() -> list[Path]:
    return sorted(CSRC.glob("*.cu"))


def _digest() -> str:
    """Content digest of everything the library is built from (file times do not survive copies of the tree)."""
    h = hashlib.sha256()
    h.update(" ".join(COMPILE_FLAGS + LINK_FLAGS).encode())
    for path in sources() + sorted(CSRC.glob("*.cuh")) + sorted(CSRC.glob("*.cpp")) + sorted(INCLUDE.glob("*.h")):
        h.update(path.name.encode())
        h.update(path.read_bytes())
    return h.hexdigest()


def needs_build() -> bool:
    return not LIB.exists() or not BINDING.exists() or not STAMP.exists() or STAMP.read_text().strip() != _digest()


def _compile(nvcc: str, src: Path, obj: Path, verbose: bool) -> str:
    cmd = [nvcc, *COMPILE_FLAGS, f"-I{INCLUDE}", f"-I{CSRC}", "-c", "-o", str(obj), str(src)]
    if verbose:
        cmd += ["-Xptxas", "-v"]
    r = subprocess.run(cmd, capture_output=True, text=True)
    if r.returncode != 0:
        raise RuntimeError(f"nvcc failed on {src.name}:\n{r.stdout}\n{r.stderr}")
    return r.stderr


def _build_binding() -> None:
    torch = Path(importlib.util.find_spec("torch").origin).parent
    tmp = BINDING.with_suffix(f".tmp{os.getpid()}.so")
    cmd = [os.environ.get("CXX", "g++"), "-O2", "-std=c++20", "-fPIC", "-shared", f"-I{INCLUDE}", f"-I{sysconfig.get_path('include')}",
           f"-I{torch / 'include'}", f"-I{torch / 'include/torch/csrc/api/include'}", "-I/usr/local/cuda/include", "-o", str(tmp),
           str(CSRC / "binding.cpp"), f"-L{torch / 'lib'}", "-ltorch_python", "-ltorch_cpu", "-lc10", "-lc10_cuda", f"-L{PKG}", "-l:libqnn.so",
           "-Wl,-rpath,$ORIGIN", f"-Wl,-rpath,{torch / 'lib'}"]
    r = subprocess.run(cmd, capture_output=True, text=True)
    if r.returncode != 0:
        raise RuntimeError(f"{cmd[0]} failed on binding.cpp:\n{r.stdout}\n{r.stderr}")
    os.replace(tmp, BINDING)


def build(force: bool = False, verbose: bool = False) -> Path:
    """Compile every csrc/*.cu to an object file (in parallel), link them into libqnn.so, and build the binding's module."""
    if not force and not needs_build():
        return LIB
    nvcc = os.environ.get("NVCC", "/usr/local/cuda/bin/nvcc")
    objdir = PKG / "_build"
    objdir.mkdir(exist_ok=True)
    srcs = sources()
    objs = [objdir / (s.stem + ".o") for s in srcs]
    workers = max(1, min(len(srcs), os.cpu_count() or 1))
    with ThreadPoolExecutor(max_workers=workers) as pool:
        logs = list(pool.map(lambda so: _compile(nvcc, so[0], so[1], verbose), zip(srcs, objs)))
    if verbose:
        print("".join(logs), file=sys.stderr)
    tmp = LIB.with_suffix(f".tmp{os.getpid()}.so")
    subprocess.check_call([nvcc, *LINK_FLAGS, "-o", str(tmp), *map(str, objs)])
    os.replace(tmp, LIB)
    _build_binding()
    STAMP.write_text(_digest() + "\n")
    return LIB


if __name__ == "__main__":
    print(build(force="--force" in sys.argv, verbose="-v" in sys.argv))
