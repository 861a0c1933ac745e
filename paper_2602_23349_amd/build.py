"""Builds in-tree the FlashOptim HIP library for gfx950, paper_2602_23349_amd/libflashoptim.so, and the module that marshals
torch tensors for it, paper_2602_23349_amd/_marshal.so."""
import concurrent.futures
import os
import shutil
import subprocess
import sys
import sysconfig
import tempfile

HERE = os.path.dirname(os.path.abspath(__file__))
ROOT = os.path.dirname(HERE)
CSRC = os.path.join(HERE, "csrc")
LIB = os.path.join(HERE, "libflashoptim.so")
MARSHAL = os.path.join(HERE, "_marshal.so")
MARSHAL_SOURCES = [os.path.join(CSRC, "marshal.cpp"), os.path.join(ROOT, "include", "flashoptim.h")]
SOURCES = [os.path.join(CSRC, n) for n in ("flashoptim_kernels.hip", "flashoptim_api.hip", "flashoptim_mx4.hip", "flashoptim_norm.hip")]
HEADERS = [os.path.join(CSRC, "flashoptim_device.h"), os.path.join(CSRC, "flashoptim_launch.h"), os.path.join(CSRC, "flashoptim_host.h"),
           os.path.join(CSRC, "flashoptim_layers.h"), os.path.join(CSRC, "flashoptim_mx4.h"),
           os.path.join(ROOT, "include", "flashoptim.h")]

# Exact arithmetic is part of the contract: no FMA contraction, IEEE division and square root,
# subnormals kept.  Packed FP32 instructions are disabled.  The command processor loads a kernel's first arguments into
# registers before its wavefronts start (up to 14 words), instead of every wavefront by a load that it waits for.
FLAGS = ["--offload-arch=gfx950", "-O3", "-std=c++17", "-fPIC",
         "-ffp-contract=off", "-fhip-fp32-correctly-rounded-divide-sqrt", "-fno-gpu-flush-denormals-to-zero",
         "-Xclang", "-target-feature", "-Xclang", "-packed-fp32-ops",
         "-mllvm", "-amdgpu-kernarg-preload-count=16",
         "-I" + os.path.join(ROOT, "include"), "-I" + CSRC]


def hipcc() -> str:
    for cand in (os.environ.get("HIPCC"), shutil.which("hipcc"), "/opt/rocm/bin/hipcc"):
        if cand and os.path.exists(cand):
            return cand
    raise RuntimeError("hipcc not found")


def older(built, sources) -> bool:
    if not os.path.exists(built):
        return True
    t = os.path.getmtime(built)
    return any(os.path.getmtime(p) > t for p in sources + [os.path.abspath(__file__)])     # (this file: the flags)


def stale() -> bool:
    return older(LIB, SOURCES + HEADERS)


def marshal_command() -> list:
    """Host code against torch's headers, by the host compiler; the library's entry points are bound at run time."""
    import torch
    from torch.utils import cpp_extension
    libs = cpp_extension.library_paths()
    return (["g++", "-O2", "-std=c++17", "-fPIC", "-shared", "-w", "-fvisibility=hidden",
             f"-D_GLIBCXX_USE_CXX11_ABI={int(torch._C._GLIBCXX_USE_CXX11_ABI)}", "-I" + os.path.join(ROOT, "include"),
             "-I" + sysconfig.get_paths()["include"]] + ["-I" + d for d in cpp_extension.include_paths()] +
            [MARSHAL_SOURCES[0], "-o", MARSHAL] + [a for d in libs for a in ("-L" + d, "-Wl,-rpath," + d)] +
            ["-lc10", "-ltorch_cpu", "-ltorch_python"])


def build(force: bool = True) -> str:
    with concurrent.futures.ThreadPoolExecutor(2) as pool:
        marshal = pool.submit(run, marshal_command()) if force or older(MARSHAL, MARSHAL_SOURCES) else None
        if force or stale():
            build_library()
        if marshal:
            marshal.result()
    return LIB


def build_library() -> None:
    with tempfile.TemporaryDirectory() as tmp, concurrent.futures.ThreadPoolExecutor(4) as pool:
        objects = [os.path.join(tmp, os.path.basename(src) + ".o") for src in SOURCES]
        compiled = pool.map(lambda p: run([hipcc()] + FLAGS + ["-c", p[0], "-o", p[1]]), zip(SOURCES, objects))
        out = "".join(compiled) + run([hipcc(), "--offload-arch=gfx950", "-fPIC", "-shared"] + objects + ["-o", LIB])
    if out.strip():
        print(out, file=sys.stderr)


def run(cmd) -> str:
    r = subprocess.run(cmd, stdout=subprocess.PIPE, stderr=subprocess.STDOUT, text=True)
    # the host pass warns that it does not know the packed-fp32-ops feature: harmless
    out = "\n".join(l for l in r.stdout.splitlines() if "packed-fp32-ops" not in l)
    if r.returncode != 0:
        raise RuntimeError(f"{os.path.basename(cmd[0])} failed:\n" + out)
    return out


if __name__ == "__main__":
    print(build())
