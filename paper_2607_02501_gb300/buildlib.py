"""Build libembqmm.so and libembpaged.so in-tree with nvcc for sm_103a (no cmake, no torch
extension), and the Python module that marshals the latter's calls.

Each .cu is compiled in parallel, then linked into its shared library with the CUDA
runtime linked statically, so the libraries need only the driver at run time.
"""
from __future__ import annotations

import concurrent.futures as cf
import os
import shutil
import subprocess
import sys
import sysconfig

HERE = os.path.dirname(os.path.abspath(__file__))
CSRC = os.path.join(HERE, "csrc")
BUILD = os.path.join(HERE, "_build")
LIB = os.path.join(HERE, "libembqmm.so")
SOURCES = ["api.cu", "quant.cu", "gemv.cu", "gemm_tc.cu", "layer_ops.cu"]
PAGED_LIB = os.path.join(HERE, "libembpaged.so")
PAGED_SOURCES = ["paged_api.cu", "paged_cache.cu", "paged_attention.cu", "paged_many.cu"]
# named for the interpreter and machine that it is compiled for, as the importer looks for it
BINDING = os.path.join(HERE, "_paged_binding" + sysconfig.get_config_var("EXT_SUFFIX"))
ARCH = ["-gencode", "arch=compute_103a,code=sm_103a"]


def _nvcc() -> str:
    for cand in (os.environ.get("NVCC"), shutil.which("nvcc"), "/usr/local/cuda/bin/nvcc"):
        if cand and os.path.exists(cand):
            return cand
    raise RuntimeError("nvcc not found: the CUDA toolkit is required to build libembqmm.so")


def _flags(verbose_ptxas: bool):
    f = ARCH + ["-O3", "-lineinfo", "-std=c++17", "-Xcompiler", "-fPIC",
                "-Xcompiler", "-fvisibility=hidden", "--expt-relaxed-constexpr",
                "-I", os.path.join(HERE, "..", "include")]
    if verbose_ptxas:
        f += ["-Xptxas", "-v"]
    return f


def _stale() -> bool:
    built = (LIB, PAGED_LIB, BINDING)
    if not all(os.path.exists(f) for f in built):
        return True
    t = min(os.path.getmtime(f) for f in built)
    deps = [os.path.join(CSRC, n) for n in os.listdir(CSRC)]
    deps += [os.path.join(HERE, "..", "include", n) for n in ("emb_qmm.h", "emb_paged.h")]
    deps.append(os.path.abspath(__file__))
    return any(os.path.getmtime(d) > t for d in deps)


def build(force: bool = False, verbose_ptxas: bool = False) -> str:
    if not force and not _stale():
        return LIB
    nvcc = _nvcc()
    os.makedirs(BUILD, exist_ok=True)
    flags = _flags(verbose_ptxas)

    def compile_one(src):
        obj = os.path.join(BUILD, src.replace(".cu", ".o"))
        cmd = [nvcc, *flags, "-c", os.path.join(CSRC, src), "-o", obj]
        r = subprocess.run(cmd, capture_output=True, text=True)
        return src, obj, r

    sources = SOURCES + PAGED_SOURCES
    def compile_binding():
        tmp = BINDING + f".tmp{os.getpid()}"
        cmd = [shutil.which("g++") or "g++", "-O2", "-std=c++17", "-shared", "-fPIC", "-fvisibility=hidden",
               "-I", sysconfig.get_paths()["include"], os.path.join(CSRC, "paged_binding.cpp"), "-o", tmp]
        r = subprocess.run(cmd, capture_output=True, text=True)
        if r.returncode == 0:
            os.replace(tmp, BINDING)
        return r

    with cf.ThreadPoolExecutor(max_workers=len(sources) + 1) as ex:
        binding = ex.submit(compile_binding)
        results = list(ex.map(compile_one, sources))
        r = binding.result()
    if r.returncode != 0:
        raise RuntimeError(f"g++ failed:\n{r.stdout}{r.stderr}")
    failed = False
    for src, _, r in results:
        if r.stdout or r.stderr:
            sys.stderr.write(f"--- {src}\n{r.stdout}{r.stderr}")
        failed |= r.returncode != 0
    if failed:
        raise RuntimeError("nvcc failed (see messages above)")
    objects = {src: obj for src, obj, _ in results}
    for lib, parts in ((LIB, SOURCES), (PAGED_LIB, PAGED_SOURCES)):
        tmp = lib + f".tmp{os.getpid()}"
        cmd = [nvcc, *ARCH, "-shared", "-o", tmp] + [objects[src] for src in parts]
        r = subprocess.run(cmd, capture_output=True, text=True)
        if r.returncode != 0:
            raise RuntimeError(f"link failed:\n{r.stdout}{r.stderr}")
        os.replace(tmp, lib)
    return LIB


if __name__ == "__main__":
    print(build(force="--force" in sys.argv, verbose_ptxas="-v" in sys.argv))
