"""Builds libmaaso.so (hipcc, gfx950) and the marshalling module _marshal.so (host code, against the installed
torch) in-tree.  `python -m paper_2509_06362_amd.build`."""
from __future__ import annotations

import os
import subprocess
import sys
import sysconfig
import tempfile
from concurrent.futures import ThreadPoolExecutor
from pathlib import Path

PKG = Path(__file__).resolve().parent
ROOT = PKG.parent
CSRC = PKG / "csrc"
LIB = PKG / "libmaaso.so"
MARSHAL = PKG / "_marshal.so"

HIPCC_FLAGS = [
    "--offload-arch=gfx950", "-O3", "-std=c++17", "-fPIC",
    # one IEEE operation per source operation: no contraction, correctly rounded division
    "-ffp-contract=off", "-fhip-fp32-correctly-rounded-divide-sqrt",
    # packed fp32 instructions stay off
    "-Xclang", "-target-feature", "-Xclang", "-packed-fp32-ops",
    "-Wall", "-Wextra",
]


def sources():
    return sorted(CSRC.glob("*.hip"))


def build_marshal(verbose: bool = False) -> Path:
    import torch
    from torch.utils import cpp_extension
    tmp = MARSHAL.with_suffix(f".so.tmp{os.getpid()}")
    include = [*cpp_extension.include_paths(), os.path.join(os.environ.get("ROCM_PATH", "/opt/rocm"), "include"),
               sysconfig.get_paths()["include"]]
    cmd = [os.environ.get("CXX", "g++"), "-O2", "-std=c++17", "-fPIC", "-shared", "-D__HIP_PLATFORM_AMD__=1", "-DUSE_ROCM=1",
           f"-D_GLIBCXX_USE_CXX11_ABI={int(torch._C._GLIBCXX_USE_CXX11_ABI)}", *(f"-isystem{p}" for p in include),
           "-Wall", "-Wextra", str(CSRC / "instance_marshal.cpp"), *(f"-L{p}" for p in cpp_extension.library_paths()),
           "-lc10", "-lc10_hip", "-ltorch_cpu", "-ltorch_python", "-o", str(tmp)]
    if verbose:
        print(" ".join(cmd), flush=True)
    res = subprocess.run(cmd, capture_output=True, text=True)
    if res.returncode != 0:
        tmp.unlink(missing_ok=True)
        raise RuntimeError(f"{cmd[0]} failed ({res.returncode}):\n{res.stderr}")
    if verbose and res.stderr.strip():
        print(res.stderr, file=sys.stderr)
    os.replace(tmp, MARSHAL)
    return MARSHAL


def build_library(verbose: bool = False) -> Path:
    """Every source compiled, side by side, and linked."""
    hipcc = os.environ.get("HIPCC", "/opt/rocm/bin/hipcc")
    noise = "is not a recognized feature for this target"

    def run(cmd):
        if verbose:
            print(" ".join(cmd), flush=True)
        res = subprocess.run(cmd, capture_output=True, text=True)
        err = "\n".join(l for l in res.stderr.splitlines() if noise not in l)
        if res.returncode != 0:
            raise RuntimeError(f"hipcc failed ({res.returncode}):\n{err}")
        if verbose and err.strip():
            print(err, file=sys.stderr)

    with tempfile.TemporaryDirectory(prefix="maaso_build") as tmp:
        objects = [str(Path(tmp) / f"{s.stem}.o") for s in sources()]
        with ThreadPoolExecutor(len(objects)) as pool:
            list(pool.map(run, [[hipcc, *HIPCC_FLAGS, f"-I{ROOT / 'include'}", "-c", str(s), "-o", o] for s, o in zip(sources(), objects)]))
        linked = LIB.with_suffix(f".so.tmp{os.getpid()}")
        try:
            run([hipcc, "--offload-arch=gfx950", "-shared", "-fPIC", *objects, "-o", str(linked)])
            os.replace(linked, LIB)
        finally:
            linked.unlink(missing_ok=True)
    build_marshal(verbose)
    return LIB


if __name__ == "__main__":
    print(build_library(verbose=True))
