"""Builds libppd.so (hand-written HIP for gfx950, with hipcc) and the call module ppd_call (host C, one file per Python ABI) in-tree.  `python -m paper_2603_13358_amd.build`."""
import os
import subprocess
import sys
import sysconfig

HERE = os.path.dirname(os.path.abspath(__file__))
CSRC = os.path.join(HERE, "csrc")
LIB = os.path.join(HERE, "libppd.so")
CALL = os.path.join(HERE, "ppd_call" + sysconfig.get_config_var("EXT_SUFFIX"))  # of this interpreter
CALL_SOURCE = os.path.join(CSRC, "ppd_call.c")
SOURCES = ["ppd_api.hip", "ppd_kernels.hip", "ppd_plan.cpp", "ppd_route.cpp",
           "ppd_ops_api.hip", "ppd_tree_kernels.hip", "ppd_cache_kernels.hip", "ppd_tree_plan.cpp",
           "ppd_rope_api.hip", "ppd_rope_kernels.hip", "ppd_prefix_api.hip", "ppd_prefix_kernels.hip", "ppd_prefix_plan.cpp"]
HEADERS = ["ppd_internal.h", "ppd_context.h", "ppd_device.h", "ppd_ops.h", "ppd_append.h", "ppd_rope.h", "ppd_prefix.h", os.path.join("..", "..", "include", "ppd.h")]

# Packed-FP32 instructions are switched off for all device code (the host pass does not know the feature
# and says so; that warning is harmless).
# Kernel arguments that are plain values and pointers (the append's and the plan upload's) arrive in scalar registers with the
# wave instead of being its first read from memory: an append of 11 decodes 2.66 -> 2.61 us back to back, one decode over
# 4000 keys with its append 18.2 -> 17.7 us a layer, 11 decodes of 300-6500 keys 33.5 -> 33.3.
FLAGS = ["--offload-arch=gfx950", "-O3", "-std=c++17", "-fPIC", "-shared", "-Wall",
         "-Xclang", "-target-feature", "-Xclang", "-packed-fp32-ops", "-mllvm", "-amdgpu-kernarg-preload-count=16"]


def is_stale():
    if not os.path.exists(LIB) or not os.path.exists(CALL):
        return True
    t = os.path.getmtime(LIB)
    return os.path.getmtime(CALL_SOURCE) > os.path.getmtime(CALL) or any(os.path.getmtime(os.path.join(CSRC, f)) > t for f in SOURCES + HEADERS)


def build_call(verbose=False):
    """Compiles the call module (CPython extension, no device code)."""
    cc = os.environ.get("CC", "gcc")
    cmd = [cc, "-O2", "-Wall", "-fPIC", "-shared", "-I" + sysconfig.get_paths()["include"], CALL_SOURCE, "-o", CALL]
    if verbose:
        print(" ".join(cmd), flush=True)
    res = subprocess.run(cmd, stdout=subprocess.PIPE, stderr=subprocess.STDOUT, text=True)
    if res.returncode != 0:
        raise RuntimeError(cc + " failed:\n" + res.stdout)


def build_lib(force=True, verbose=False):
    """Compiles the library and the call module.  force=False skips the compile when the built library is newer than its sources."""
    if not force and not is_stale():
        return LIB
    build_call(verbose)
    hipcc = os.environ.get("HIPCC", "/opt/rocm/bin/hipcc")
    # PPD_EXTRA_HIPCC_FLAGS: tuning macros of the kernels, e.g. "-DPPD_STAGES=2 -DPPD_STREAM_KSETS=2"
    extra = os.environ.get("PPD_EXTRA_HIPCC_FLAGS", "").split()
    cmd = [hipcc] + FLAGS + extra + [os.path.join(CSRC, f) for f in SOURCES] + ["-o", LIB]
    if verbose:
        print(" ".join(cmd), flush=True)
    res = subprocess.run(cmd, stdout=subprocess.PIPE, stderr=subprocess.STDOUT, text=True)
    out = "\n".join(l for l in res.stdout.splitlines() if "packed-fp32-ops" not in l)
    if res.returncode != 0:
        raise RuntimeError("hipcc failed:\n" + out)
    if verbose and out.strip():
        print(out)
    return LIB


if __name__ == "__main__":
    build_lib(force=True, verbose=True)
    print("built", LIB)
    sys.exit(0)
