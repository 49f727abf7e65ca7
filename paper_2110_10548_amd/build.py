"""Build libp2.so (HIP kernels + C ABI) for gfx950, in-tree, and _train.so (the training operators on torch tensors).

The library needs hipcc alone; the extension module needs torch's and Python's headers and is built apart from it.
"""
import importlib.util
import os
import subprocess

HERE = os.path.dirname(os.path.abspath(__file__))
CSRC = os.path.join(HERE, "csrc")
LIB = os.path.join(HERE, "libp2.so")
SOURCES = ["p2_plan.cpp", "p2_literal.hip", "p2_compact.hip", "p2_regs.hip", "p2_shared.hip", "p2_frontier.hip", "p2_graph.hip", "p2_skeleton.hip", "p2_select.hip", "p2_peak.hip", "p2_api.hip",
           "p2_norm.hip", "p2_balance.hip", "p2_newton.hip", "p2_route.hip", "p2_adamw.hip", "p2_linear.hip", "p2_train_api.hip"]
FLAGS = ["--offload-arch=gfx950", "-O3", "-std=c++17", "-fPIC", "-Wall", "-Wno-unused-function",
         "-Xclang", "-target-feature", "-Xclang", "-packed-fp32-ops"]

TENSORS = os.path.join(HERE, "_train.so")                  # extension module: the training operators on torch tensors


def tensors_command():
    """The host compiler's command: only torch's and Python's headers, no device code."""
    import sysconfig
    import torch
    where = os.path.dirname(os.path.abspath(torch.__file__))
    return ["g++", "-O2", "-std=c++17", "-fPIC", "-shared", "-Wall", "-fvisibility=hidden", "-D_GLIBCXX_USE_CXX11_ABI=%d" % torch._C._GLIBCXX_USE_CXX11_ABI,
            "-isystem", os.path.join(where, "include"), "-isystem", os.path.join(where, "include", "torch", "csrc", "api", "include"),
            "-isystem", sysconfig.get_paths()["include"], os.path.join(CSRC, "p2_train_tensors.cpp"), "-o", TENSORS,
            "-L" + os.path.join(where, "lib"), "-ltorch_python", "-ltorch_cpu", "-lc10"]


def build(verbose: bool = False) -> str:
    objs = []
    procs = []
    for src in SOURCES:
        obj = os.path.join(CSRC, os.path.splitext(src)[0] + ".o")
        cmd = ["hipcc", "-x", "hip", "-c", os.path.join(CSRC, src), "-o", obj] + FLAGS
        if verbose:
            print(" ".join(cmd))
        procs.append((subprocess.Popen(cmd), cmd))
        objs.append(obj)
    for p, cmd in procs:
        if p.wait() != 0:
            raise RuntimeError("compile failed: " + " ".join(cmd))
    cmd = ["hipcc", "-shared", "-fPIC", "--offload-arch=gfx950", "-o", LIB] + objs
    if verbose:
        print(" ".join(cmd))
    subprocess.run(cmd, check=True)
    return LIB


def build_tensors(verbose: bool = False):
    """The extension module's path, or None where there is no torch to build it for."""
    if importlib.util.find_spec("torch") is None:
        print("torch is not installed: libp2.so is complete, the training operators on torch tensors are left out")
        return None
    cmd = tensors_command()
    if verbose:
        print(" ".join(cmd))
    if subprocess.run(cmd).returncode != 0:
        raise RuntimeError("compile failed: " + " ".join(cmd))
    return TENSORS


if __name__ == "__main__":
    print(build(verbose=True))
    print(build_tensors(verbose=True))
