"""Build the CUDA library libvbq.so in-tree for GB300 (sm_103a).

Each .cu file under csrc/ is compiled in parallel with nvcc, then linked into
paper_2607_02893_gb300/libvbq.so (CUDA runtime linked statically). The CPython
module native/_decode.c (argument marshalling of decode.py) is compiled beside
them into paper_2607_02893_gb300/_decode.<interpreter's tag>.so.
"""

from __future__ import annotations

import os
import shutil
import subprocess
import sys
import sysconfig
from concurrent.futures import ThreadPoolExecutor

PKG = os.path.dirname(os.path.abspath(__file__))
ROOT = os.path.dirname(PKG)
CSRC = os.path.join(PKG, "csrc")
BUILD = os.path.join(ROOT, "_build", "vbq")
LIB = os.path.join(PKG, "libvbq.so")
MODULE_SRC = os.path.join(PKG, "native", "_decode.c")
MODULE = os.path.join(PKG, "_decode" + sysconfig.get_config_var("EXT_SUFFIX"))      # of the interpreter that builds it

ARCH = ["-gencode", "arch=compute_103a,code=sm_103a"]
NVCC_FLAGS = ["-O3", "-std=c++17", "-lineinfo", "-Xcompiler", "-fPIC,-O2",
              "--expt-relaxed-constexpr", "-I", os.path.join(ROOT, "include")]


def nvcc() -> str:
    cand = shutil.which("nvcc") or "/usr/local/cuda/bin/nvcc"
    if not os.path.exists(cand):
        raise RuntimeError("nvcc not found")
    return cand


def sources():
    return sorted(os.path.join(CSRC, f) for f in os.listdir(CSRC) if f.endswith(".cu"))


def _compile(src: str, verbose_ptxas: bool) -> str:
    obj = os.path.join(BUILD, os.path.basename(src)[:-3] + ".o")
    cmd = [nvcc(), *ARCH, *NVCC_FLAGS, "-c", src, "-o", obj]
    if verbose_ptxas:
        cmd += ["-Xptxas", "-v"]
    r = subprocess.run(cmd, capture_output=True, text=True)
    if r.returncode != 0:
        raise RuntimeError(f"nvcc failed on {src}:\n{r.stdout}\n{r.stderr}")
    if verbose_ptxas:
        sys.stderr.write(r.stderr)
    return obj


def _compile_module() -> None:
    deps = (MODULE_SRC, os.path.join(ROOT, "include", "vbq.h"))
    if os.path.exists(MODULE) and all(os.path.getmtime(d) <= os.path.getmtime(MODULE) for d in deps):
        return
    tmp = MODULE + ".tmp"
    r = subprocess.run([shutil.which("gcc") or "cc", "-O2", "-std=gnu11", "-Wall", "-shared", "-fPIC", "-I", sysconfig.get_paths()["include"],
                        "-I", os.path.join(ROOT, "include"), MODULE_SRC, "-o", tmp], capture_output=True, text=True)
    if r.returncode != 0:
        raise RuntimeError(f"compiling {MODULE_SRC} failed:\n{r.stdout}\n{r.stderr}")
    os.replace(tmp, MODULE)


def build(verbose_ptxas: bool = False, force: bool = False) -> str:
    os.makedirs(BUILD, exist_ok=True)
    _compile_module()
    srcs = sources()
    deps = srcs + [os.path.join(CSRC, f) for f in os.listdir(CSRC) if f.endswith((".cuh", ".h"))]
    deps.append(os.path.join(ROOT, "include", "vbq.h"))
    if not force and os.path.exists(LIB):
        lib_mtime = os.path.getmtime(LIB)
        if all(os.path.getmtime(d) <= lib_mtime for d in deps) and not verbose_ptxas:
            return LIB
    with ThreadPoolExecutor(max_workers=min(8, len(srcs))) as ex:
        objs = list(ex.map(lambda s: _compile(s, verbose_ptxas), srcs))
    tmp = LIB + ".tmp"
    cmd = [nvcc(), *ARCH, "-shared", "-o", tmp, *objs]
    r = subprocess.run(cmd, capture_output=True, text=True)
    if r.returncode != 0:
        raise RuntimeError(f"link failed:\n{r.stdout}\n{r.stderr}")
    os.replace(tmp, LIB)
    return LIB


if __name__ == "__main__":
    print(build(verbose_ptxas="-v" in sys.argv, force="-f" in sys.argv))
