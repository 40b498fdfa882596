"""Build libqnn.so from csrc/*.cu with nvcc for sm_100a (no torch involved), and the tensor-argument module of the binding,
_binding.<ABI tag>.so, from csrc/binding.cpp with the host compiler against the installed torch.  The module holds for one
Python and one torch; its digest covers both, so that another one of either rebuilds it.

    python -m paper_2106_09886_b200.build [--force]
"""
from __future__ import annotations

import hashlib
import importlib.metadata
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
BINDING = PKG / f"_binding{sysconfig.get_config_var('EXT_SUFFIX')}"
BINDING_STAMP = PKG / "_binding.so.digest"
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
    for path in sources() + sorted(CSRC.glob("*.cuh")) + sorted(INCLUDE.glob("*.h")):
        h.update(path.name.encode())
        h.update(path.read_bytes())
    return h.hexdigest()


def _stale(built: Path, stamp: Path, digest: str) -> bool:
    return not built.exists() or not stamp.exists() or stamp.read_text().strip() != digest


def needs_build() -> bool:
    return _stale(LIB, STAMP, _digest()) or _binding_stale()


def _binding_stale() -> bool:
    """(Without torch there is nothing that the module could serve, and the library is built alone.)"""
    return importlib.util.find_spec("torch") is not None and _stale(BINDING, BINDING_STAMP, _binding_digest())


def _compile(nvcc: str, src: Path, obj: Path, verbose: bool) -> str:
    cmd = [nvcc, *COMPILE_FLAGS, f"-I{INCLUDE}", f"-I{CSRC}", "-c", "-o", str(obj), str(src)]
    if verbose:
        cmd += ["-Xptxas", "-v"]
    r = subprocess.run(cmd, capture_output=True, text=True)
    if r.returncode != 0:
        raise RuntimeError(f"nvcc failed on {src.name}:\n{r.stdout}\n{r.stderr}")
    return r.stderr


def _binding_command(out: Path) -> list[str]:
    torch = Path(importlib.util.find_spec("torch").origin).parent
    return [os.environ.get("CXX", "g++"), "-O2", "-std=c++20", "-fPIC", "-shared", f"-I{INCLUDE}", f"-I{sysconfig.get_path('include')}",
            f"-I{torch / 'include'}", f"-I{torch / 'include/torch/csrc/api/include'}", "-I/usr/local/cuda/include", "-o", str(out),
            str(CSRC / "binding.cpp"), f"-L{torch / 'lib'}", "-ltorch_python", "-ltorch_cpu", "-ltorch_cuda", "-lc10", "-lc10_cuda", f"-L{PKG}", "-l:libqnn.so",
            "-Wl,-rpath,$ORIGIN", f"-Wl,-rpath,{torch / 'lib'}"]


def _binding_digest() -> str:
    """Everything the module depends on: its source, the library's header, the command, and the versions of Python and torch."""
    h = hashlib.sha256()
    h.update(" ".join(_binding_command(Path("out"))).replace(str(PKG.parent), "").encode())      # (the tree may be copied elsewhere)
    h.update(f"{sys.version} torch {importlib.metadata.version('torch')}".encode())
    for path in [CSRC / "binding.cpp"] + sorted(INCLUDE.glob("*.h")):
        h.update(path.name.encode())
        h.update(path.read_bytes())
    return h.hexdigest()


def _build_binding() -> None:
    tmp = PKG / f"_binding.tmp{os.getpid()}.so"
    cmd = _binding_command(tmp)
    r = subprocess.run(cmd, capture_output=True, text=True)
    if r.returncode != 0:
        raise RuntimeError(f"{cmd[0]} failed on binding.cpp:\n{r.stdout}\n{r.stderr}")
    os.replace(tmp, BINDING)
    (PKG / "_binding.so").unlink(missing_ok=True)            # the name without a tag, of earlier builds
    BINDING_STAMP.write_text(_binding_digest() + "\n")


def _build_library(verbose: bool) -> None:
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
    STAMP.write_text(_digest() + "\n")


def build(force: bool = False, verbose: bool = False) -> Path:
    """Compile every csrc/*.cu to an object file (in parallel) and link them into libqnn.so; build the binding's module."""
    if force or _stale(LIB, STAMP, _digest()):
        _build_library(verbose)
    if force or _binding_stale():
        _build_binding()
    return LIB


if __name__ == "__main__":
    print(build(force="--force" in sys.argv, verbose="-v" in sys.argv))
