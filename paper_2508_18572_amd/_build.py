"""Build libkvio.so (HIP kernels + C ABI) for gfx950 with hipcc, in-tree."""
import os
import subprocess
import tempfile
from concurrent.futures import ThreadPoolExecutor

PKG = os.path.dirname(os.path.abspath(__file__))
ROOT = os.path.dirname(PKG)
CSRC = os.path.join(PKG, "csrc")
INCLUDE = os.path.join(ROOT, "include")
LIB = os.path.join(PKG, "libkvio.so")
SOURCES = [os.path.join(CSRC, "kvio_kernels.hip"), os.path.join(CSRC, "kvio_api.cpp"),
           os.path.join(CSRC, "kvio_sched.cpp"), os.path.join(CSRC, "kvio_disk.cpp"),
           os.path.join(CSRC, "kvio_staged.cpp"), os.path.join(CSRC, "kvio_noalloc.hip"),
           os.path.join(CSRC, "kvio_linkpeak.hip")]
# the operators on the paged cache (include/kvio_attn.h), whose sources stand apart
CSRC_ATTN = os.path.join(PKG, "csrc_attn")
SOURCES += [os.path.join(CSRC_ATTN, f) for f in ("kvio_append.hip", "kvio_attend_steps.hip", "kvio_attend_blocks.hip", "kvio_attn_api.cpp")]
HIPCC = os.environ.get("HIPCC", "/opt/rocm/bin/hipcc")

FLAGS = [
    "--offload-arch=gfx950", "-O3", "-std=c++17", "-fPIC", "-shared",
    "-Wall", "-Wextra", "-Werror", "-Wno-unused-parameter",
    # keep the compiler from forming packed fp32 ops
    "-Xclang", "-target-feature", "-Xclang", "-packed-fp32-ops",
    # matrix products in either kind of registers: attention reads their results with ordinary instructions (the
    # transfer kernels, which have no such products, come out the same with and without it)
    "-mllvm", "-amdgpu-mfma-vgpr-form",
    "-I", INCLUDE, "-I", CSRC, "-I", os.path.join(PKG, "csrc_attn"), "-pthread",
]


def build(verbose: bool = False, extra=()) -> str:
    """Compile every source into libkvio.so, a few at a time; always recompiles."""
    tmp = LIB + ".tmp"

    def run(cmd):
        if verbose:
            print(" ".join(cmd), flush=True)
        subprocess.run(cmd, check=True)

    with tempfile.TemporaryDirectory() as d:
        objects = [os.path.join(d, os.path.basename(s) + ".o") for s in SOURCES]
        each = [f for f in FLAGS if f != "-shared"] + list(extra)
        with ThreadPoolExecutor(min(8, os.cpu_count() or 1)) as pool:
            list(pool.map(lambda so: run([HIPCC] + each + ["-x", "hip", "-c", so[0], "-o", so[1]]), zip(SOURCES, objects)))
        run([HIPCC, "--offload-arch=gfx950", "-fPIC", "-shared", "-pthread"] + objects + ["-o", tmp])
    os.replace(tmp, LIB)
    return LIB


if __name__ == "__main__":
    print(build(verbose=True))
