"""Build the JARQ CUDA library (libjarq.so) in-tree for sm_103a.

Each ``csrc/*.cu`` file is compiled in parallel with nvcc
(``-gencode arch=compute_103a,code=sm_103a``) and linked into
``paper_2609_38599_gb300/libjarq.so``.  Object files go to ``_build/``.
"""
from __future__ import annotations

import concurrent.futures
import os
import re
import shutil
import subprocess
import sys

PKG = os.path.dirname(os.path.abspath(__file__))
ROOT = os.path.dirname(PKG)
CSRC = os.path.join(PKG, "csrc")
BUILD = os.path.join(ROOT, "_build")
LIB = os.path.join(PKG, "libjarq.so")
ARCH = ["-gencode", "arch=compute_103a,code=sm_103a"]
FLAGS = ["-O3", "-lineinfo", "-std=c++17", "-Xcompiler", "-fPIC", "-Xcompiler", "-O2",
         "-I" + os.path.join(ROOT, "include")]


# Registers a thread that kernels with roles of different register counts must be
# compiled for: the roles' sum would not fit a smaller block, and they would wait
# for registers that never come.
LAUNCH_REGISTERS = {"k_tc_integer.cu": tuple(
    (f"tc_integer_kernelILi{nt}ELb{groups}ELb{vec}ELb{half}E", registers)
    for nt, vec, half, registers in ((256, 1, 1, 128), (128, 0, 0, 72), (128, 0, 1, 72))
    for groups in (0, 1))}


def check_registers(src: str, ptxas_output: str) -> None:
    """Raises unless ptxas gave the kernels of LAUNCH_REGISTERS their count."""
    found = re.findall(r"Compiling entry function '(\S+)'.*?Used (\d+) registers", ptxas_output, flags=re.S)
    for part, want in LAUNCH_REGISTERS.get(os.path.basename(src), ()):
        counts = [int(n) for name, n in found if part in name]
        if not counts or min(counts) < want:
            raise RuntimeError(f"{src}: {part} compiled for {counts} registers a thread, {want} are needed")


def nvcc() -> str:
    exe = shutil.which("nvcc") or "/usr/local/cuda/bin/nvcc"
    if not os.path.exists(exe):
        raise RuntimeError("nvcc not found: the JARQ CUDA library cannot be built")
    return exe


def _compile(src: str, extra) -> str:
    obj = os.path.join(BUILD, os.path.basename(src)[:-3] + ".o")
    checked = os.path.basename(src) in LAUNCH_REGISTERS
    info = ["-Xptxas", "-v"] if checked and not extra else []
    cmd = [nvcc(), *ARCH, *FLAGS, *extra, *info, "-c", src, "-o", obj]
    res = subprocess.run(cmd, capture_output=True, text=True)
    if res.returncode != 0:
        raise RuntimeError(f"nvcc failed on {src}:\n{res.stdout}\n{res.stderr}")
    if checked:
        try:
            check_registers(src, res.stdout + res.stderr)
        except RuntimeError:
            os.remove(obj)
            raise
    if res.stderr.strip() and "-Xptxas" in " ".join(extra):
        sys.stderr.write(res.stderr)
    return obj


def build(verbose: bool = False, ptxas_info: bool = False) -> str:
    """Compile every CUDA source and link the shared library; returns its path."""
    os.makedirs(BUILD, exist_ok=True)
    srcs = sorted(os.path.join(CSRC, f) for f in os.listdir(CSRC) if f.endswith(".cu"))
    extra = ["-Xptxas", "-v"] if ptxas_info else []
    with concurrent.futures.ThreadPoolExecutor(max_workers=max(1, min(len(srcs), os.cpu_count() or 4))) as ex:
        objs = list(ex.map(lambda s: _compile(s, extra), srcs))
    tmp = LIB + ".tmp"
    cmd = [nvcc(), *ARCH, "-shared", "-o", tmp, *objs]
    res = subprocess.run(cmd, capture_output=True, text=True)
    if res.returncode != 0:
        raise RuntimeError(f"link failed:\n{res.stdout}\n{res.stderr}")
    os.replace(tmp, LIB)
    if verbose:
        print(f"built {LIB} from {len(srcs)} sources")
    return LIB


if __name__ == "__main__":
    build(verbose=True, ptxas_info="-v" in sys.argv)
