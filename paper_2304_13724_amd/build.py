"""Build libbgmf.so (HIP, gfx950) in-tree with hipcc, and _ranking.so, the
ranking calls on PyTorch tensors, with g++."""
from __future__ import annotations

import glob
import os
import subprocess
import sys
import sysconfig

PKG = os.path.dirname(os.path.abspath(__file__))
ROOT = os.path.dirname(PKG)
LIB = os.path.join(PKG, "libbgmf.so")
TENSORS = os.path.join(PKG, "_ranking.so")
ARCH = "gfx950"
HIPCC = os.environ.get("HIPCC", "/opt/rocm/bin/hipcc")

FLAGS = [
    f"--offload-arch={ARCH}", "-O3", "-std=c++17", "-fPIC", "-shared", "-parallel-jobs=8",
    # packed fp32 arithmetic stays off (v_pk_*_f32 are not emitted)
    "-Xclang", "-target-feature", "-Xclang", "-packed-fp32-ops",
    "-Wall", "-Wno-unused-function", "-Wno-unused-result", "-Wno-unused-value",
]


def sources():
    return sorted(glob.glob(os.path.join(PKG, "csrc", "*.hip")))


# The HIP runtime is recorded in libbgmf.so under the name libamdhip64.so,
# the name PyTorch's ROCm libraries use for theirs (hipcc would record the
# versioned file name).  The dynamic loader maps a library once per name, so
# a process that loads both gets a single HIP runtime -- whichever loads
# first -- and PyTorch's device pointers and streams are valid in the
# library's calls.  The library's RUNPATH still finds the ROCm installation's
# runtime when it is loaded on its own.  The name comes from linking against
# an empty stand-in that carries only that soname.
def _runtime_name_stub() -> str:
    stub_dir = os.path.join(PKG, "_build", "hipname")
    stub = os.path.join(stub_dir, "libamdhip64.so")
    if not os.path.exists(stub):
        os.makedirs(stub_dir, exist_ok=True)
        src = os.path.join(stub_dir, "empty.c")
        with open(src, "w") as f:
            f.write("void bgmf_runtime_name_stub(void) {}\n")
        subprocess.run(["gcc", "-shared", "-fPIC", "-Wl,-soname,libamdhip64.so", src, "-o",
                        stub], check=True)
    return stub_dir


def _compile(cmd, out: str, verbose: bool) -> None:
    tmp = out + ".tmp"
    cmd = [*cmd, "-o", tmp]
    if verbose:
        print(" ".join(cmd), flush=True)
    res = subprocess.run(cmd, capture_output=True, text=True)
    if res.returncode != 0:
        sys.stderr.write(res.stdout + res.stderr)
        raise RuntimeError(f"{os.path.basename(cmd[0])} failed building {os.path.basename(out)}")
    os.replace(tmp, out)


def build_tensors(verbose: bool = False) -> str:
    """Compile csrc/ranking_tensors.cpp (host code only) against PyTorch's
    headers and libbgmf.so, which it finds beside itself."""
    import torch
    home = os.path.dirname(torch.__file__)
    _compile(["g++", "-O2", "-std=c++17", "-fPIC", "-shared", "-Wall",
              f"-D_GLIBCXX_USE_CXX11_ABI={int(torch._C._GLIBCXX_USE_CXX11_ABI)}",
              "-isystem", os.path.join(home, "include"),
              "-isystem", sysconfig.get_paths()["include"], "-I", os.path.join(ROOT, "include"),
              os.path.join(PKG, "csrc", "ranking_tensors.cpp"), "-L", PKG, "-l:libbgmf.so",
              "-Wl,-rpath,$ORIGIN", "-L", os.path.join(home, "lib"), "-lc10", "-ltorch_cpu",
              "-ltorch_python"], TENSORS, verbose)
    return TENSORS


def build(verbose: bool = False) -> str:
    """Compile every HIP source into paper_2304_13724_amd/libbgmf.so and, where
    PyTorch is installed, paper_2304_13724_amd/_ranking.so (ranking.py raises
    without it; the rest of the package needs the library alone)."""
    _compile([HIPCC, *FLAGS, "-L", _runtime_name_stub(), "-I", os.path.join(ROOT, "include"),
              *sources(), "-lrocprofiler-sdk-roctx"], LIB, verbose)
    try:
        import torch  # noqa: F401
    except ImportError:
        print("PyTorch is not installed: _ranking.so is not built", file=sys.stderr)
    else:
        build_tensors(verbose)
    return LIB


if __name__ == "__main__":
    print(build(verbose=True))
