"""Builds libper_hip.so (gfx950) and the Python boundaries of its calls in-tree.  Usable as
``python -m paper_2311_09445_amd.build``."""
from __future__ import annotations

import os
import subprocess
import sysconfig

HERE = os.path.dirname(os.path.abspath(__file__))
CSRC = os.path.join(HERE, "csrc")
OBJECTS = os.path.join(HERE, "build")
LIB = os.path.join(HERE, "libper_hip.so")
BINDING = os.path.join(HERE, "_per_binding.so")
SEQ_BINDING = os.path.join(HERE, "_seq_binding.so")
SOURCES = ["per_kernels.hip", "per_api.hip", "seq_api.hip", "seq_rotate.hip", "seq_attention.hip", "seq_delta.hip", "seq_block.hip"]

# -ffp-contract=off: the tree arithmetic must round after every add and multiply.
# packed-fp32 ops are switched off for the device pass.
FLAGS = ["--offload-arch=gfx950", "-O3", "-std=c++17", "-fPIC", "-ffp-contract=off",
         "-fno-fast-math", "-fno-gpu-flush-denormals-to-zero",
         "-Xclang", "-target-feature", "-Xclang", "-packed-fp32-ops", "-Wall", "-Wno-unused-command-line-argument"]


def build_lib(verbose: bool = False) -> str:
    """One object per source file, compiled side by side, then linked."""
    hipcc = os.environ.get("HIPCC", "/opt/rocm/bin/hipcc")
    os.makedirs(OBJECTS, exist_ok=True)
    running, objects = [], []
    for src in SOURCES:
        obj = os.path.join(OBJECTS, os.path.splitext(src)[0] + ".o")
        cmd = [hipcc, *FLAGS, "-c", os.path.join(CSRC, src), "-o", obj]
        if verbose:
            print(" ".join(cmd), flush=True)
        running.append((cmd, subprocess.Popen(cmd)))
        objects.append(obj)
    failed = [subprocess.CalledProcessError(p.returncode, cmd) for cmd, p in running if p.wait()]
    if failed:
        raise failed[0]
    cmd = [hipcc, "--offload-arch=gfx950", "-fPIC", "-shared", *objects, "-o", LIB]
    if verbose:
        print(" ".join(cmd), flush=True)
    subprocess.check_call(cmd)
    return LIB


def _build_binding(source: str, target: str, verbose: bool) -> str:
    """Host code only (no kernels): a CPython module that takes torch tensors apart for C-ABI calls."""
    from torch.utils import cpp_extension
    torch_lib = os.path.join(os.path.dirname(cpp_extension.include_paths()[0]), "lib")
    include = cpp_extension.include_paths() + ["/opt/rocm/include", sysconfig.get_paths()["include"]]
    cmd = ["g++", "-O2", "-std=c++17", "-fPIC", "-shared", "-fvisibility=hidden", "-Wall", "-D__HIP_PLATFORM_AMD__=1", "-DUSE_ROCM=1"]
    cmd += [x for d in include for x in ("-isystem", d)] + [os.path.join(CSRC, source), "-o", target]
    cmd += ["-L" + HERE, "-l:libper_hip.so", "-Wl,-rpath,$ORIGIN", "-L" + torch_lib, "-lc10", "-lc10_hip", "-ltorch_cpu", "-ltorch_python"]
    if verbose:
        print(" ".join(cmd), flush=True)
    subprocess.check_call(cmd)
    return target


def build_binding(verbose: bool = False) -> str:
    """The calls of one replay buffer."""
    return _build_binding("per_binding.cpp", BINDING, verbose)


def build_seq_binding(verbose: bool = False) -> str:
    """The sequence operators."""
    return _build_binding("seq_binding.cpp", SEQ_BINDING, verbose)


if __name__ == "__main__":
    print(build_lib(verbose=True))
    print(build_binding(verbose=True))
    print(build_seq_binding(verbose=True))
