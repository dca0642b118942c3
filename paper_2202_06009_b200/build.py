"""Compile the CUDA sources of this package for sm_100a into libzoa.so (in-tree)."""
import os
import subprocess
import tempfile

HERE = os.path.dirname(os.path.abspath(__file__))
CSRC = os.path.join(HERE, "csrc")
LIB = os.path.join(HERE, "libzoa.so")
SOURCES = ["zoa_kernels.cu", "zoa_pipeline.cu", "zoa_reduce_pipeline.cu", "zoa_server_pipeline.cu", "zoa_api.cu", "zoa_noalloc.cu",
           "zoa_ops.cu", "zoa_mx4_quantize.cu", "zoa_mx4_matmul.cu", "zoa_distill.cu"]
HEADERS = ["zoa_device.cuh", "zoa_internal.h", "zoa_ring.cuh", "zoa_ops.h", "zoa_async.cuh", "zoa_mx4.cuh", os.path.join("..", "..", "include", "zoa.h")]

# The arithmetic contract needs IEEE division and square root, subnormals kept,
# and no contraction of a multiply and an add into one fused operation.
NVCC_FLAGS = ["-gencode", "arch=compute_100a,code=sm_100a", "-lineinfo", "-O3", "-std=c++17",
              "--fmad=false", "--ftz=false", "--prec-div=true", "--prec-sqrt=true",
              "-Xcompiler", "-fPIC", "-Xcompiler", "-Wall"]


def _stale() -> bool:
    if not os.path.exists(LIB):
        return True
    built = os.path.getmtime(LIB)
    deps = [os.path.join(CSRC, f) for f in SOURCES + HEADERS] + [os.path.abspath(__file__)]
    return any(os.path.getmtime(d) > built for d in deps)


def build(force: bool = False, verbose: bool = False) -> str:
    if not force and not _stale():
        return LIB
    nvcc = ["nvcc", *NVCC_FLAGS, *(["-Xptxas=-v"] if verbose else [])]
    with tempfile.TemporaryDirectory() as tmp:      # the sources side by side, one process each
        objects = [os.path.join(tmp, s + ".o") for s in SOURCES]
        jobs = [subprocess.Popen([*nvcc, "-c", os.path.join(CSRC, s), "-o", o]) for s, o in zip(SOURCES, objects)]
        for job in jobs:
            job.wait()
        for job in jobs:
            if job.returncode:
                raise subprocess.CalledProcessError(job.returncode, job.args)
        subprocess.check_call([*nvcc, "-shared", "-o", LIB, *objects])
    return LIB


if __name__ == "__main__":
    import sys
    print(build(force=True, verbose="-v" in sys.argv))
