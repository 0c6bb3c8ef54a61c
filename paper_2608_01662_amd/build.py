"""Build the LSA HIP library (liblsa.so) for gfx950, in-tree.

    python -m paper_2608_01662_amd.build          # or: python paper_2608_01662_amd/build.py
"""
from __future__ import annotations

import os
import shutil
import subprocess
import sys
from concurrent.futures import ThreadPoolExecutor

HERE = os.path.dirname(os.path.abspath(__file__))
CSRC = os.path.join(HERE, "csrc")
INCLUDE = os.path.join(os.path.dirname(HERE), "include")
LIB = os.path.join(HERE, "liblsa.so")
SERVE = os.path.join(HERE, "_serve.so")
SOURCES = ["indexer.hip", "attention.hip", "append.hip", "cache_read.hip", "decode_attn.hip", "prompt_attn.hip", "lsa_api.cpp",
           "serve_api.cpp", "prompt_api.cpp"]
ARCH = "gfx950"

HIPCC_FLAGS = [
    f"--offload-arch={ARCH}", "-O3", "-std=c++17", "-fPIC",
    "-Xclang", "-target-feature", "-Xclang", "-packed-fp32-ops",
    "-Wall", "-Wno-unused-function", "-Wno-unused-variable", "-Wno-format-security",
    f"-I{INCLUDE}", f"-I{CSRC}",
]


# Per-source extra flags. The indexer's MFMA accumulators are reduced by vector code right after
# each product chain: keeping them in VGPRs (not AGPRs) saves a register copy per element.
# The attention kernels never produce a NaN from finite inputs (masked scores are -inf and every
# difference of two -inf is guarded): without NaN semantics the softmax maxima compile to plain
# v_max_f32, without the canonicalising v_max_f32 x, x, x in front of each operand. (The decode attention keeps NaN
# semantics: a masked weight times a NaN is a case of its own there. Its accumulators are rescaled by vector
# code, so they are kept in VGPRs too.)
EXTRA_FLAGS = {"indexer.hip": ["-mllvm", "-amdgpu-mfma-vgpr-form"], "attention.hip": ["-fno-honor-nans"],
               "decode_attn.hip": ["-mllvm", "-amdgpu-mfma-vgpr-form"]}


def _hipcc() -> str:
    h = shutil.which("hipcc") or "/opt/rocm/bin/hipcc"
    if not os.path.exists(h):
        raise RuntimeError("hipcc not found: the LSA library needs ROCm's hipcc")
    return h


def _binding_command(out: str) -> list[str]:
    """The Python module of the serving operators' host side: host code against torch and liblsa.so."""
    import sysconfig
    import torch
    from torch.utils import cpp_extension
    lib = os.path.join(os.path.dirname(torch.__file__), "lib")
    return [shutil.which("g++") or "c++", "-O2", "-std=c++17", "-fPIC", "-shared", "-Wall",
            f"-D_GLIBCXX_USE_CXX11_ABI={int(torch._C._GLIBCXX_USE_CXX11_ABI)}", f"-I{INCLUDE}",
            f"-I{sysconfig.get_paths()['include']}", *(f"-isystem{p}" for p in cpp_extension.include_paths()),
            os.path.join(CSRC, "serve_bind.cpp"), "-o", out, f"-L{HERE}", "-llsa", "-Wl,-rpath,$ORIGIN",
            f"-L{lib}", "-lc10", "-ltorch_cpu", "-ltorch_python"]


def build(verbose: bool = False) -> str:
    """Compile every source for gfx950 and link liblsa.so next to this file, and the binding of the serving
    operators (_serve.so) against it. Always rebuilds."""
    hipcc = _hipcc()
    objdir = os.path.join(HERE, "_build")
    os.makedirs(objdir, exist_ok=True)

    def compile_one(src):
        obj = os.path.join(objdir, os.path.splitext(src)[0] + ".o")
        lang = ["-x", "hip"] if src.endswith(".cpp") else []
        cmd = [hipcc, *HIPCC_FLAGS, *EXTRA_FLAGS.get(src, []), *lang, "-c", os.path.join(CSRC, src), "-o", obj]
        r = subprocess.run(cmd, capture_output=True, text=True)
        out = "\n".join(l for l in (r.stdout + r.stderr).splitlines() if "packed-fp32-ops" not in l)
        if r.returncode != 0:
            raise RuntimeError(f"hipcc failed on {src}:\n{out}")
        if verbose and out.strip():
            print(out)
        return obj

    with ThreadPoolExecutor(max_workers=len(SOURCES)) as ex:
        objs = list(ex.map(compile_one, SOURCES))
    tmp = LIB + ".tmp"
    cmd = [hipcc, f"--offload-arch={ARCH}", "-shared", "-fPIC", "-o", tmp, *objs]
    r = subprocess.run(cmd, capture_output=True, text=True)
    if r.returncode != 0:
        raise RuntimeError(f"link failed:\n{r.stdout}{r.stderr}")
    os.replace(tmp, LIB)
    r = subprocess.run(_binding_command(SERVE + ".tmp"), capture_output=True, text=True)
    if r.returncode != 0:
        raise RuntimeError(f"binding failed:\n{r.stdout}{r.stderr}")
    os.replace(SERVE + ".tmp", SERVE)
    return LIB


if __name__ == "__main__":
    print(build(verbose="-v" in sys.argv))
