"""Builds libbyzshield.so (HIP kernels + host library + C-ABI) for gfx950, and _worker_calls.so, in-tree."""
import concurrent.futures
import os
import subprocess
import sys
import warnings

PKG = os.path.dirname(os.path.abspath(__file__))
ROOT = os.path.dirname(PKG)
CSRC = os.path.join(PKG, "csrc")
OBJ = os.path.join(PKG, "_build")
LIB = os.path.join(PKG, "libbyzshield.so")
KERNELS = os.path.join(CSRC, "kernels.hip")
# kernels.hip is compiled once per part (-DBYZ_PART=n): the single-pass kernels are large and
# build in parallel this way
# the slowest parts first: the pool starts them in this order
KERNEL_PARTS = (2, 1, 18, 7, 4, 22, 25, 14, 24, 15, 17, 6, 5, 23, 20, 21, 8, 10, 16, 9, 11, 19, 3, 13, 12, 0)
OTHER_SOURCES = [os.path.join(CSRC, name) for name in
                 ("group_norm.hip", "gated_ffn.hip", "distill.hip", "krum.hip", "host.cpp")]


CALLS = os.path.join(PKG, "_worker_calls.so")


def build_calls(verbose=False):
    """Compiles the Python module of the worker operators' common calls against torch's headers (ten seconds)."""
    import sysconfig

    import torch
    root = os.path.dirname(torch.__file__)
    made = CALLS + ".%d.so" % os.getpid()
    cmd = ["g++", "-std=c++17", "-O2", "-fPIC", "-shared", "-Wall", "-I", os.path.join(ROOT, "include"),
           "-isystem", sysconfig.get_paths()["include"], "-isystem", os.path.join(root, "include"),
           "-isystem", os.path.join(root, "include", "torch", "csrc", "api", "include"),
           os.path.join(CSRC, "worker_calls.cpp"), "-o", made, "-L", PKG, "-lbyzshield",
           "-L", os.path.join(root, "lib"), "-ltorch_python", "-ltorch_cpu", "-lc10", "-Wl,-rpath,$ORIGIN"]
    if verbose:
        print(" ".join(cmd), flush=True)
    if os.path.exists(CALLS):  # one that is left from before would be used with a library it does not belong to
        os.remove(CALLS)
    subprocess.run(cmd, check=True)
    os.replace(made, CALLS)  # whole, also where several processes build it at once
    return CALLS


def build(verbose=False):
    """Always compiles (about six and a half minutes on 8 cores); raises where the library does not build."""
    sys.path.insert(0, CSRC)
    try:
        import gen_selnet
        gen_selnet.main(os.path.join(CSRC, "generated"))
    finally:
        sys.path.remove(CSRC)
    os.makedirs(OBJ, exist_ok=True)
    hipcc = os.environ.get("HIPCC", "/opt/rocm/bin/hipcc")
    flags = ["--offload-arch=gfx950", "-O3", "-std=c++17", "-fPIC",
             "-Wall", "-Wextra", "-Wno-unused-parameter", "-Wno-unused-function",
             "-Xclang", "-target-feature", "-Xclang", "-packed-fp32-ops",
             "-I", os.path.join(ROOT, "include"), "-I", CSRC]
    jobs = []
    for part in KERNEL_PARTS:
        obj = os.path.join(OBJ, "kernels_part%d.o" % part)
        jobs.append(([hipcc] + flags + ["-DBYZ_PART=%d" % part, "-c", KERNELS, "-o", obj], obj))
    for src in OTHER_SOURCES:
        obj = os.path.join(OBJ, os.path.splitext(os.path.basename(src))[0] + ".o")
        jobs.append(([hipcc] + flags + ["-c", src, "-o", obj], obj))

    def run(job):
        cmd, obj = job
        import time
        t0 = time.time()
        subprocess.run(cmd, check=True)
        if verbose:
            print("%6.1f s  %s" % (time.time() - t0, " ".join(cmd[-6:])), flush=True)
        return obj

    workers = min(len(jobs), max(1, len(os.sched_getaffinity(0))), 16)
    with concurrent.futures.ThreadPoolExecutor(max_workers=workers) as pool:
        objects = list(pool.map(run, jobs))
    link = [hipcc, "--offload-arch=gfx950", "-shared", "-fPIC"] + objects + ["-o", LIB]
    if verbose:
        print(" ".join(link), flush=True)
    subprocess.run(link, check=True)
    try:
        build_calls(verbose)
    except (ImportError, OSError, subprocess.CalledProcessError) as e:
        warnings.warn("%s was not built (%s); the binding does without it" % (os.path.basename(CALLS), e), RuntimeWarning)
    return LIB


if __name__ == "__main__":
    print(build(verbose=True))
