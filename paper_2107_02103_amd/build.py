"""Build libdpc.so (HIP kernels for gfx950 + host table builder) in-tree.

    python -m paper_2107_02103_amd.build

Every call recompiles.  The library is written next to this file under
``_lib/`` so that it travels with the source tree."""
import os
import subprocess
import sys

HERE = os.path.dirname(os.path.abspath(__file__))
ROOT = os.path.dirname(HERE)
CSRC = os.path.join(HERE, "csrc")
INCLUDE = os.path.join(ROOT, "include")
LIB_DIR = os.path.join(HERE, "_lib")
LIB = os.path.join(LIB_DIR, "libdpc.so")
ARCH = "gfx950"

SOURCES = ["dpc_table.cpp", "dpc_se_a.hip", "dpc_descriptor.hip", "dpc_env.hip", "dpc_fitting.hip",
           "dpc_nlist.hip", "dpc_route.hip", "dpc_i8.hip", "dpc_gate.hip", "dpc_embed.hip", "dpc_mx4.hip"]

# packed fp32 instructions are disabled for all device code
HIPCC_FLAGS = ["-O3", "-std=c++17", "-fPIC", f"--offload-arch={ARCH}",
               "-Xclang", "-target-feature", "-Xclang", "-packed-fp32-ops",
               "-Wall", "-Wno-unused-result"]


def hipcc():
    for c in (os.environ.get("HIPCC"), "/opt/rocm/bin/hipcc"):
        if c and os.path.exists(c):
            return c
    return "hipcc"


def build(verbose=False):
    os.makedirs(LIB_DIR, exist_ok=True)
    objs = []
    for src in SOURCES:
        obj = os.path.join(LIB_DIR, src + ".o")
        lang = ["-x", "hip"] if src.endswith(".hip") else []
        cmd = [hipcc()] + HIPCC_FLAGS + ["-I", INCLUDE] + lang + ["-c", os.path.join(CSRC, src), "-o", obj]
        if verbose:
            print(" ".join(cmd), flush=True)
        subprocess.check_call(cmd, stderr=subprocess.STDOUT if not verbose else None)
        objs.append(obj)
    tmp = LIB + ".tmp%d" % os.getpid()
    # rocBLAS serves the fitting net's plain GEMMs
    cmd = [hipcc(), f"--offload-arch={ARCH}", "-shared", "-fPIC", "-o", tmp] + objs + ["-lrocblas"]
    if verbose:
        print(" ".join(cmd), flush=True)
    subprocess.check_call(cmd)
    os.replace(tmp, LIB)
    for o in objs:
        os.remove(o)
    return LIB


if __name__ == "__main__":
    print(build(verbose="-v" in sys.argv))
