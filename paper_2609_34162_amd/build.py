"""Build libsdp.so for gfx950 with hipcc (in-tree)."""
import os
import subprocess
import sys
import tempfile
from concurrent.futures import ThreadPoolExecutor

HERE = os.path.dirname(os.path.abspath(__file__))
ROOT = os.path.dirname(HERE)
LIB_PATH = os.path.join(HERE, "libsdp.so")
SOURCES = [os.path.join(HERE, "csrc", f)
           for f in ("sdp_runtime.hip", "sdp_stream.hip", "sdp_host_route.hip", "sdp_kernels.hip",
                     "sdp_copy.hip", "sdp_noalloc.hip", "sdp_ops.hip", "sdp_qk.hip", "sdp_grouped.hip",
                     "sdp_distill.hip")]
# host-only lanes, built with the host compiler: no fused multiply-add, so the
# FP64 update rounds every product and sum as written
HOST_SOURCES = [os.path.join(HERE, "csrc", f) for f in ("sdp_host_adamw.cpp", "sdp_schedule.cpp")]
HIPCC = os.environ.get("HIPCC", "/opt/rocm/bin/hipcc")
HOSTCXX = os.environ.get("SDP_HOSTCXX", "/opt/rocm/llvm/bin/clang++")
HOST_FLAGS = ["-O3", "-std=c++17", "-fPIC", "-ffp-contract=off", "-fno-math-errno", "-Wall", "-fvisibility=hidden"]
FLAGS = [
    "--offload-arch=gfx950", "-O3", "-std=c++17", "-fPIC", "-shared",
    # no packed FP32 instructions in device code
    "-Xclang", "-target-feature", "-Xclang", "-packed-fp32-ops",
    "-Wall", "-Wno-unused-function",
    # only the C ABI (SDP_API in sdp.h) is exported
    "-fvisibility=hidden",
]


def build(verbose: bool = False) -> str:
    tmp = LIB_PATH + ".tmp"
    inc = ["-I", os.path.join(ROOT, "include"), "-I", os.path.join(HERE, "csrc")]
    # one compiler process for each source, up to the machine's CPUs (8 at most)
    compile_flags = [f for f in FLAGS if f != "-shared"]
    with tempfile.TemporaryDirectory() as d:
        def compiled(src: str) -> str:
            obj = os.path.join(d, os.path.basename(src) + ".o")
            tool = [HIPCC, *compile_flags] if src in SOURCES else [HOSTCXX, *HOST_FLAGS]
            cmd = [*tool, *inc, "-c", src, "-o", obj]
            if verbose:
                print(" ".join(cmd), flush=True)
            subprocess.check_call(cmd)
            return obj
        with ThreadPoolExecutor(min(8, os.cpu_count() or 1)) as pool:
            objs = list(pool.map(compiled, SOURCES + HOST_SOURCES))
        cmd = [HIPCC, *FLAGS, "-o", tmp, *objs]
        if verbose:
            print(" ".join(cmd), flush=True)
        subprocess.check_call(cmd)
    os.replace(tmp, LIB_PATH)
    return LIB_PATH


if __name__ == "__main__":
    build(verbose=True)
    sys.exit(0)
