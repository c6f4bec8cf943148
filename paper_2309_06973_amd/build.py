"""Builds libshifter.so (HIP, gfx950) with hipcc and _q8.so (the 8-bit operators' calls from Python,
host code over torch's headers) with g++, both in-tree."""
from __future__ import annotations

import os
import subprocess
import sys
import sysconfig
from concurrent.futures import ThreadPoolExecutor

PKG = os.path.dirname(os.path.abspath(__file__))
ROOT = os.path.dirname(PKG)
CSRC = os.path.join(PKG, "csrc")
OBJ = os.path.join(PKG, "_build")
LIB = os.path.join(PKG, "libshifter.so")
BINDING = os.path.join(PKG, "_q8.so")
SOURCES = ["api.hip", "select.hip", "spec_select.hip", "spec_multi.hip", "mask_scan.hip", "batch.hip", "plan_compact.hip",
           "fixpoint.hip", "fold.hip", "codec.hip", "q8_rows.hip", "q8_product.hip",
           "log_probs.hip", "grad_norm.hip", "adapters.hip"]
FLAGS = ["-O3", "-std=c++17", "--offload-arch=gfx950", "-fPIC", "-Wall",
         "-Wno-unused-result",
         "-Xclang", "-target-feature", "-Xclang", "-packed-fp32-ops",
         "-I", os.path.join(ROOT, "include"), "-I", CSRC]


def _hipcc() -> str:
    for c in (os.environ.get("HIPCC"), "/opt/rocm/bin/hipcc", "hipcc"):
        if c and (os.path.isabs(c) and os.path.exists(c) or not os.path.isabs(c)):
            return c
    return "hipcc"


def _binding_commands():
    """(compile, link): the binding is linked once libshifter.so is there."""
    import torch
    from torch.utils import cpp_extension
    obj = os.path.join(OBJ, "q8_bind.o")
    headers = [sysconfig.get_paths()["include"], *cpp_extension.include_paths()]
    compile_ = ["g++", "-O2", "-std=c++17", "-fPIC", "-Wall", f"-D_GLIBCXX_USE_CXX11_ABI={int(torch.compiled_with_cxx11_abi())}",
                *(a for h in headers for a in ("-isystem", h)), "-I", os.path.join(ROOT, "include"),
                "-c", os.path.join(CSRC, "q8_bind.cpp"), "-o", obj]
    link = ["g++", "-shared", obj, "-L", PKG, "-lshifter", *("-L" + p for p in cpp_extension.library_paths()),
            "-lc10", "-ltorch_cpu", "-ltorch_hip", "-ltorch_python", "-Wl,-rpath,$ORIGIN", "-Wl,--allow-shlib-undefined", "-o", BINDING]
    return compile_, link


def _run(cmd, what: str):
    r = subprocess.run(cmd, capture_output=True, text=True)
    if r.returncode != 0:
        raise RuntimeError(f"{what} failed:\n{r.stdout}\n{r.stderr}")


def build_library(verbose: bool = True) -> str:
    os.makedirs(OBJ, exist_ok=True)
    hipcc = _hipcc()

    def compile_one(src: str) -> str:
        obj = os.path.join(OBJ, src.replace(".hip", ".o"))
        cmd = [hipcc, *FLAGS, "-c", os.path.join(CSRC, src), "-o", obj]
        r = subprocess.run(cmd, capture_output=True, text=True)
        if r.returncode != 0:
            raise RuntimeError(f"hipcc failed for {src}:\n{r.stdout}\n{r.stderr}")
        if verbose:
            warn = [l for l in r.stderr.splitlines()
                    if "warning" in l and "packed-fp32-ops" not in l]
            for l in warn:
                print(l, file=sys.stderr)
        return obj

    bind, link_binding = _binding_commands()
    with ThreadPoolExecutor(max_workers=4) as ex:
        binding = ex.submit(_run, bind, "g++ for q8_bind.cpp")
        objs = list(ex.map(compile_one, SOURCES))
        binding.result()
    _run([hipcc, "--offload-arch=gfx950", "-shared", "-fPIC", *objs, "-o", LIB], "link")
    _run(link_binding, "link of the binding")
    if verbose:
        print(f"built {LIB}")
        print(f"built {BINDING}")
    return LIB


if __name__ == "__main__":
    build_library()
