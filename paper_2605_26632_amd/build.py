"""Build librtlynx.so (HIP, gfx950 only) in-tree with hipcc, and the compiled part of its Python binding, _block.so, with g++."""
import os
import subprocess
import sys
import sysconfig

HERE = os.path.dirname(os.path.abspath(__file__))
ROOT = os.path.dirname(HERE)
CSRC = os.path.join(HERE, "csrc")
LIB = os.path.join(HERE, "librtlynx.so")
BLOCK = os.path.join(HERE, "_block.so")
SOURCES = ["api.hip", "pack.hip", "pack_lora.hip", "gemm.hip", "mx.hip", "grouped.hip", "grouped_grad.hip", "few_rows.hip", "gated.hip", "block_norm.hip", "rotary.hip", "diag.hip"]
HIPCC = os.environ.get("HIPCC", "/opt/rocm/bin/hipcc")
FLAGS = ["--offload-arch=gfx950", "-O3", "-std=c++17", "-fPIC", "-fno-gpu-rdc",
         # packed-fp32 instructions are kept out of the generated code: some of their forms have given wrong results on this hardware
         "-Xclang", "-target-feature", "-Xclang", "-packed-fp32-ops",
         "-I" + os.path.join(ROOT, "include"), "-I" + CSRC]


def build(verbose: bool = False) -> str:
    objs = []
    procs = []
    for s in SOURCES:
        src = os.path.join(CSRC, s)
        obj = os.path.join(CSRC, s.replace(".hip", ".o"))
        objs.append(obj)
        procs.append(subprocess.Popen([HIPCC, *FLAGS, "-c", src, "-o", obj],
                                      stdout=subprocess.PIPE, stderr=subprocess.STDOUT, text=True))
    for s, p in zip(SOURCES, procs):
        out, _ = p.communicate()
        out = "\n".join(l for l in out.splitlines() if "packed-fp32-ops" not in l)
        if p.returncode != 0:
            raise RuntimeError("hipcc failed on %s:\n%s" % (s, out))
        if verbose and out.strip():
            print(out)
    subprocess.run([HIPCC, "-shared", "-fPIC", "--offload-arch=gfx950", *objs, "-o", LIB], check=True)
    build_block()
    return LIB


def build_block() -> str:
    """_block.so: host code only, on torch's headers and librtlynx.so beside it."""
    import torch
    home = os.path.join(os.path.dirname(torch.__file__))
    includes = [os.path.join(ROOT, "include"), os.path.join(home, "include"), os.path.join(home, "include", "torch", "csrc", "api", "include"),
                sysconfig.get_paths()["include"]]
    out = subprocess.run([os.environ.get("CXX", "g++"), "-O2", "-std=c++17", "-fPIC", "-shared", "-fvisibility=hidden",
                          "-D_GLIBCXX_USE_CXX11_ABI=%d" % torch._C._GLIBCXX_USE_CXX11_ABI, *("-I" + i for i in includes), os.path.join(CSRC, "block_binding.cpp"),
                          "-L" + HERE, "-l:librtlynx.so", "-L" + os.path.join(home, "lib"), "-ltorch_python", "-ltorch", "-ltorch_cpu", "-lc10",
                          "-Wl,-rpath,$ORIGIN", "-o", BLOCK], stdout=subprocess.PIPE, stderr=subprocess.STDOUT, text=True)
    if out.returncode != 0:
        raise RuntimeError("g++ failed on block_binding.cpp:\n" + out.stdout)
    return BLOCK


if __name__ == "__main__":
    print(build(verbose="-v" in sys.argv))
