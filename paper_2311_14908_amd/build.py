"""Build libsvmx.so (gfx950) in-tree with hipcc, and the binding's list checks with g++.

Every HIP source is compiled for gfx950 only, with packed-fp32 instruction selection
disabled, then linked into ``paper_2311_14908_amd/libsvmx.so`` next to this file.  ``_tensor_list.so``
beside it is the one Python extension (host code against torch's headers).
"""
from __future__ import annotations

import os
import subprocess
import sys
import sysconfig
from concurrent.futures import ThreadPoolExecutor

HERE = os.path.dirname(os.path.abspath(__file__))
ROOT = os.path.dirname(HERE)
CSRC = os.path.join(HERE, "csrc")
INCLUDE = os.path.join(ROOT, "include")
OBJDIR = os.path.join(ROOT, "_build", "svmx")
SOURCES = ["api.cpp", "smo.hip", "ws_smo.hip", "gram.hip", "gram_split.hip", "predict.hip", "warm.hip",
           "layers.cpp", "embed.hip", "norm.hip", "adamw.hip", "svgrad.hip"]
ARCH = "gfx950"
HIPCC = os.environ.get("HIPCC", "/opt/rocm/bin/hipcc")
FLAGS = ["-O3", "-std=c++17", "-fPIC", f"--offload-arch={ARCH}", "-Xclang", "-target-feature", "-Xclang",
         "-packed-fp32-ops", "-Wall", "-Wno-unused-result", "-I", INCLUDE, "-I", CSRC]


def lib_path() -> str:
    return os.path.join(HERE, "libsvmx.so")


def _compile(src: str, verbose: bool) -> str:
    obj = os.path.join(OBJDIR, src + ".o")
    cmd = [HIPCC, *FLAGS, "-x", "hip", "-c", os.path.join(CSRC, src), "-o", obj]
    if verbose:
        print(" ".join(cmd), flush=True)
    r = subprocess.run(cmd, capture_output=True, text=True)
    msg = "\n".join(line for line in (r.stdout + r.stderr).splitlines() if "packed-fp32-ops" not in line)
    if r.returncode != 0:
        raise RuntimeError(f"hipcc failed on {src}:\n{msg}")
    if verbose and msg.strip():
        print(msg, flush=True)
    return obj


def _extension(verbose: bool) -> None:
    import torch

    base = os.path.dirname(torch.__file__)
    libs = os.path.join(base, "lib")
    out = os.path.join(HERE, "_tensor_list.so")
    tmp = out + f".tmp{os.getpid()}"
    cmd = ["g++", "-O2", "-std=c++17", "-fPIC", "-shared", "-Wall", f"-D_GLIBCXX_USE_CXX11_ABI={int(torch.compiled_with_cxx11_abi())}",
           "-I", INCLUDE, "-isystem", os.path.join(base, "include"), "-isystem", sysconfig.get_paths()["include"],
           os.path.join(CSRC, "tensor_list.cpp"), "-o", tmp, "-L", libs, "-ltorch_python", "-ltorch_cpu", "-lc10",
           f"-Wl,-rpath,{libs}"]
    if verbose:
        print(" ".join(cmd), flush=True)
    r = subprocess.run(cmd, capture_output=True, text=True)
    if r.returncode != 0:
        raise RuntimeError(f"g++ failed on tensor_list.cpp:\n{r.stdout}{r.stderr}")
    os.replace(tmp, out)


def build(verbose: bool = False) -> str:
    os.makedirs(OBJDIR, exist_ok=True)
    with ThreadPoolExecutor(max_workers=len(SOURCES) + 1) as ex:
        extension = ex.submit(_extension, verbose)
        objs = list(ex.map(lambda s: _compile(s, verbose), SOURCES))
        extension.result()
    out = lib_path()
    tmp = out + f".tmp{os.getpid()}"
    cmd = [HIPCC, f"--offload-arch={ARCH}", "-shared", "-fPIC", "-o", tmp, *objs]
    if verbose:
        print(" ".join(cmd), flush=True)
    r = subprocess.run(cmd, capture_output=True, text=True)
    if r.returncode != 0:
        raise RuntimeError(f"link failed:\n{r.stdout}{r.stderr}")
    os.replace(tmp, out)
    return out


if __name__ == "__main__":
    print(build(verbose="-v" in sys.argv))
