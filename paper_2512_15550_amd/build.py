"""Compile the HIP library for gfx950 with hipcc, in-tree: six translation units (the host side with the staged and build kernels; the
single-launch decode kernel; the operators on the paged KV cache; those on 8-bit rows, windows and drafts, whose attention over 8-bit rows has one for
each type of query), compiled side by side, then linked; and the binding's checks of tensors, an extension module of the interpreter."""
import os
import subprocess
import sysconfig

HERE = os.path.dirname(os.path.abspath(__file__))
CSRC = os.path.join(HERE, "csrc")
SOURCES = ["ctkvr.hip", "fused.hip", "cache.hip", "quant.hip", "quant_bf16.hip", "quant_f32.hip"]
LIB = os.path.join(HERE, "libctkvr.so")
MARSHAL = os.path.join(HERE, "_marshal.so")
OBJ_DIR = os.path.join(HERE, "_build")

HIPCC_FLAGS = [
    "--offload-arch=gfx950", "-O3", "-std=c++17", "-fPIC", "-fvisibility=hidden",
    # every fused multiply-add on a path that decides an integer is written as an explicit fmaf
    "-ffp-contract=off",
    # no packed-fp32 instructions
    "-Xclang", "-target-feature", "-Xclang", "-packed-fp32-ops",
    # matrix results in ordinary vector registers: a kernel of 512 registers a wave otherwise gets them in the accumulation
    # half, and every vector instruction on a result first copies it
    "-mllvm", "-amdgpu-mfma-vgpr-form=1",
    # what a statement in assembly leaves open is an error
    "-Werror=inline-asm",
]


def marshal_command():
    import torch
    root = os.path.dirname(os.path.abspath(torch.__file__))
    return [os.environ.get("CXX", "g++"), "-O2", "-std=c++17", "-shared", "-fPIC", "-fvisibility=hidden", f"-D_GLIBCXX_USE_CXX11_ABI={int(torch._C._GLIBCXX_USE_CXX11_ABI)}",
            "-I" + sysconfig.get_paths()["include"], "-I" + os.path.join(root, "include"), "-I" + os.path.join(root, "include", "torch", "csrc", "api", "include"),
            "-o", MARSHAL, os.path.join(CSRC, "marshal.cpp"), "-L" + os.path.join(root, "lib"), "-ltorch_python", "-ltorch_cpu", "-lc10"]


def build_library(verbose: bool = False) -> str:
    hipcc = os.environ.get("HIPCC", "/opt/rocm/bin/hipcc")
    os.makedirs(OBJ_DIR, exist_ok=True)
    jobs = []
    for src in SOURCES:
        obj = os.path.join(OBJ_DIR, src.replace(".hip", ".o"))
        cmd = [hipcc, *HIPCC_FLAGS, "-c", "-o", obj, os.path.join(CSRC, src)]
        if verbose:
            print(" ".join(cmd))
        jobs.append((obj, cmd, subprocess.Popen(cmd, stdout=subprocess.PIPE, stderr=subprocess.STDOUT, text=True)))
    cmd = marshal_command()
    if verbose:
        print(" ".join(cmd))
    jobs.append((None, cmd, subprocess.Popen(cmd, stdout=subprocess.PIPE, stderr=subprocess.STDOUT, text=True)))
    objs = []
    for obj, cmd, proc in jobs:
        out, _ = proc.communicate()
        if proc.returncode != 0:
            raise RuntimeError("compilation failed: " + " ".join(cmd) + "\n" + out)
        if obj:
            objs.append(obj)
    link = [hipcc, "--offload-arch=gfx950", "-shared", "-fPIC", "-o", LIB, *objs]
    if verbose:
        print(" ".join(link))
    proc = subprocess.run(link, capture_output=True, text=True)
    if proc.returncode != 0:
        raise RuntimeError("link failed:\n" + proc.stdout + proc.stderr)
    return LIB


PROBES = ["sync_probe", "latency_probe", "gather_probe", "xcd_probe", "mfma_chain_probe"]
PROBE_DIR = os.path.join(HERE, "probes")


def build_probes(verbose: bool = False):
    """The stand-alone programs under csrc/probes (launch floor, in-launch barriers, visibility,
    latencies; a check of the fp32 matrix instruction): executables in probes/, not used by the library."""
    hipcc = os.environ.get("HIPCC", "/opt/rocm/bin/hipcc")
    os.makedirs(PROBE_DIR, exist_ok=True)
    out = []
    for name in PROBES:
        exe = os.path.join(PROBE_DIR, name)
        cmd = [hipcc, "--offload-arch=gfx950", "-O3", "-std=c++17", "-Xclang", "-target-feature", "-Xclang", "-packed-fp32-ops",
               "-o", exe, os.path.join(CSRC, "probes", name + ".hip")]
        if verbose:
            print(" ".join(cmd))
        proc = subprocess.run(cmd, capture_output=True, text=True)
        if proc.returncode != 0:
            raise RuntimeError("hipcc failed: " + " ".join(cmd) + "\n" + proc.stdout + proc.stderr)
        out.append(exe)
    return out


if __name__ == "__main__":
    import sys
    print(build_library(verbose=True))
    if "--probes" in sys.argv:
        print("\n".join(build_probes(verbose=True)))
