"""Builds libst3.so (the C-ABI library) and compiles nothing else.

`hipcc` cross-compiles for gfx950 without a GPU, so this runs anywhere the ROCm
toolchain is installed.  The library is written next to this file so that it
travels with the source tree.
"""
from __future__ import annotations

import os
import shutil
import subprocess
from concurrent.futures import ThreadPoolExecutor

HERE = os.path.dirname(os.path.abspath(__file__))
ROOT = os.path.dirname(HERE)
CSRC = os.path.join(HERE, "csrc")
LIB_PATH = os.path.join(HERE, "libst3.so")

SOURCES = ["st3_api.hip", "st3_decode.hip", "st3_select.hip", "st3_prefill.hip", "st3_prefill_mfma.hip",
           "st3_noalloc.hip", "st3_packed.hip", "st3_block.hip", "st3_block_decode.hip",
           "st3_block_attend.hip", "st3_rotary.hip"]

HIPCC_FLAGS = [
    "--offload-arch=gfx950", "-O3", "-std=c++17", "-fPIC", "-fvisibility=hidden",
    "-Xclang", "-target-feature", "-Xclang", "-packed-fp32-ops",
    "-Wall", "-Wno-unused-function", "-Wno-unknown-attributes",
]


def _hipcc() -> str:
    for cand in (shutil.which("hipcc"), "/opt/rocm/bin/hipcc"):
        if cand and os.path.exists(cand):
            return cand
    raise RuntimeError("hipcc not found: the ROCm toolchain is required to build libst3.so")


def build_library(verbose: bool = False) -> str:
    hipcc = _hipcc()
    objdir = os.path.join(HERE, "_build")
    os.makedirs(objdir, exist_ok=True)
    inc = ["-I", os.path.join(ROOT, "include"), "-I", CSRC]

    def compile_one(src: str) -> str:
        obj = os.path.join(objdir, src.replace(".hip", ".o"))
        cmd = [hipcc, *HIPCC_FLAGS, *inc, "-c", os.path.join(CSRC, src), "-o", obj]
        if verbose:
            print(" ".join(cmd), flush=True)
        r = subprocess.run(cmd, capture_output=True, text=True)
        if r.returncode != 0:
            raise RuntimeError(f"hipcc failed on {src}:\n{r.stdout}\n{r.stderr}")
        if verbose and r.stderr.strip():
            print(r.stderr)
        return obj

    with ThreadPoolExecutor(max_workers=min(8, len(SOURCES))) as ex:
        objs = list(ex.map(compile_one, SOURCES))
    cmd = [hipcc, "--offload-arch=gfx950", "-shared", "-fPIC", *objs, "-o", LIB_PATH]
    r = subprocess.run(cmd, capture_output=True, text=True)
    if r.returncode != 0:
        raise RuntimeError(f"link failed:\n{r.stdout}\n{r.stderr}")
    return LIB_PATH


def build_host_sanitized(driver_src: str, out_path: str) -> str:
    """The library's sources plus a host driver program as ONE executable whose HOST code runs under
    AddressSanitizer and UndefinedBehaviorSanitizer (device code is compiled as usual and never
    launched by such a driver): checks the argument validation and the host-only helpers on a box
    without a GPU."""
    hipcc = _hipcc()
    objdir = os.path.join(HERE, "_build", "san")
    os.makedirs(objdir, exist_ok=True)
    inc = ["-I", os.path.join(ROOT, "include"), "-I", CSRC]
    san = ["-Xarch_host", "-fsanitize=address", "-Xarch_host", "-fsanitize=undefined", "-Xarch_host",
           "-fno-sanitize-recover=undefined", "-Xarch_host", "-fno-omit-frame-pointer", "-g"]
    flags = [f for f in HIPCC_FLAGS if f != "-fvisibility=hidden"]

    def compile_one(path: str) -> str:
        obj = os.path.join(objdir, os.path.basename(path) + ".o")
        lang = ["-x", "hip"] if not path.endswith(".hip") else []
        r = subprocess.run([hipcc, *flags, *san, *inc, *lang, "-c", path, "-o", obj], capture_output=True, text=True)
        if r.returncode != 0:
            raise RuntimeError(f"hipcc (sanitized) failed on {path}:\n{r.stdout}\n{r.stderr}")
        return obj

    srcs = [os.path.join(CSRC, f) for f in SOURCES] + [driver_src]
    with ThreadPoolExecutor(max_workers=min(8, len(srcs))) as ex:
        objs = list(ex.map(compile_one, srcs))
    r = subprocess.run([hipcc, "--offload-arch=gfx950", "-fsanitize=address", "-fsanitize=undefined", *objs, "-o", out_path],
                       capture_output=True, text=True)
    if r.returncode != 0:
        raise RuntimeError(f"link (sanitized) failed:\n{r.stdout}\n{r.stderr}")
    return out_path


if __name__ == "__main__":
    print(build_library(verbose=True))
