"""Build liblbscan.so (HIP, gfx950) and _lbscan_torch.so in-tree.  Run as
`python -m paper_2506_15976_amd.build`.

hipcc cross-compiles without a GPU.  Objects go to _build/ at the repo root
(ignored by git); the shared libraries are written next to this file so that they
travel with the tree.  _lbscan_torch.so is host code: the torch side of the operators
around the scan (csrc/lbscan_torch.cpp), a Python module linked against liblbscan.so.
"""
from __future__ import annotations

import concurrent.futures
import glob
import os
import subprocess
import sys
import sysconfig

HERE = os.path.dirname(os.path.abspath(__file__))
ROOT = os.path.dirname(HERE)
CSRC = os.path.join(HERE, "csrc")
OBJDIR = os.path.join(ROOT, "_build", "lbscan")
LIB = os.path.join(HERE, "liblbscan.so")
TORCH_LIB = os.path.join(HERE, "_lbscan_torch.so")

HIPCC = os.environ.get("HIPCC", "/opt/rocm/bin/hipcc")
CXX = os.environ.get("CXX", "g++")
# Packed-FP32 instruction selection is switched off for all device code.
FLAGS = [
    "--offload-arch=gfx950", "-O3", "-std=c++17", "-fPIC", "-fno-gpu-rdc",
    "-Xclang", "-target-feature", "-Xclang", "-packed-fp32-ops",
    "-Wno-unused-command-line-argument", "-Wno-ignored-attributes",
]


def _sources():
    return sorted(glob.glob(os.path.join(CSRC, "*.hip")))


def _headers():
    return glob.glob(os.path.join(CSRC, "*.h")) + glob.glob(os.path.join(CSRC, "*.inc")) + glob.glob(os.path.join(ROOT, "include", "*.h"))


def _torch_sources():
    return sorted(glob.glob(os.path.join(CSRC, "*.cpp")))


def _torch_flags():
    """Compiler and linker flags of the torch side.  torch is only looked up, not imported: importing it takes
    longer than compiling most of the kernels."""
    import importlib.util
    torch = os.path.dirname(importlib.util.find_spec("torch").origin)
    rocm = os.path.dirname(os.path.dirname(HIPCC))
    include = os.path.join(torch, "include")
    compiler = ["-x", "c++", "-D__HIP_PLATFORM_AMD__=1", "-DUSE_ROCM=1", "-DTORCH_EXTENSION_NAME=_lbscan_torch",
                "-D_GLIBCXX_USE_CXX11_ABI=1", "-O2", "-std=c++17", "-fPIC", "-w"]
    compiler += [f"-I{p}" for p in (include, os.path.join(include, "torch", "csrc", "api", "include"),
                                    os.path.join(rocm, "include"), sysconfig.get_paths()["include"])]
    lib = os.path.join(torch, "lib")
    linker = [f"-L{HERE}", "-l:liblbscan.so", f"-L{lib}", "-ltorch_python", "-ltorch", "-ltorch_cpu", "-lc10", "-lc10_hip",
              "-Wl,-rpath,$ORIGIN"]
    return compiler, linker


def _compile(src: str, extra) -> str:
    obj = os.path.join(OBJDIR, os.path.basename(src) + ".o")
    if src.endswith(".cpp"):
        cmd = [CXX, *_torch_flags()[0], "-c", src, "-o", obj]
    else:
        cmd = [HIPCC, *FLAGS, *extra, "-c", src, "-o", obj]
    r = subprocess.run(cmd, capture_output=True, text=True)
    out = "\n".join(l for l in (r.stdout + r.stderr).splitlines()
                    if "packed-fp32-ops" not in l and "is not a recognized feature" not in l)
    if r.returncode != 0:
        raise RuntimeError(f"{cmd[0]} failed for {src}:\n{out}")
    if out.strip():
        print(out, file=sys.stderr)
    return obj


def build(force: bool = True, extra_flags=(), jobs: int = 8, verbose: bool = True) -> str:
    """Compile every source and link the shared libraries.  With force=False
    the build is skipped when both are newer than every source."""
    srcs = _sources()
    host = _torch_sources()
    if not force and os.path.exists(LIB) and os.path.exists(TORCH_LIB):
        newest = max(os.path.getmtime(p) for p in srcs + host + _headers() + [__file__])
        if min(os.path.getmtime(LIB), os.path.getmtime(TORCH_LIB)) >= newest:
            return LIB
    os.makedirs(OBJDIR, exist_ok=True)
    with concurrent.futures.ThreadPoolExecutor(max_workers=jobs) as ex:
        # (the torch side first: it takes longest)
        objs = list(ex.map(lambda s: _compile(s, list(extra_flags)), host + srcs))
    for cmd in ([HIPCC, "--offload-arch=gfx950", "-shared", "-fPIC", "-fno-gpu-rdc", "-o", LIB, *objs[len(host):]],
                [CXX, "-shared", "-fPIC", "-o", TORCH_LIB, *objs[:len(host)], *_torch_flags()[1]]):
        r = subprocess.run(cmd, capture_output=True, text=True)
        if r.returncode != 0:
            raise RuntimeError("link failed:\n" + r.stdout + r.stderr)
    if verbose:
        print(f"built {LIB} and {os.path.basename(TORCH_LIB)} from {len(srcs) + len(host)} sources")
    return LIB


if __name__ == "__main__":
    build(force=True, extra_flags=sys.argv[1:])
