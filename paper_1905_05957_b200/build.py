"""Compile the CUDA library in-tree: paper_1905_05957_b200/csrc/libdsq.so (sm_100a only).

Every translation unit is compiled to an object file on its own (side by side), then linked."""
import os
import subprocess
import sys
import sysconfig
from concurrent.futures import ThreadPoolExecutor

HERE = os.path.dirname(os.path.abspath(__file__))
CSRC = os.path.join(HERE, "csrc")
OBJ = os.path.join(CSRC, "build")
LIB = os.path.join(CSRC, "libdsq.so")
CALL_SRC = os.path.join(CSRC, "dsq_call.c")
# the Python extension through which the short calls go, of this interpreter
CALL_LIB = os.path.join(CSRC, "dsq_call" + (sysconfig.get_config_var("EXT_SUFFIX") or ".so"))
SOURCES = ["dsq_api.cu", "dsq_chunked.cu", "dsq_chunked_sign.cu", "dsq_chunked_sign_l2.cu", "dsq_chunked_qsgd.cu", "dsq_chunked_qsgd_window.cu",
           "dsq_elementwise.cu", "dsq_topk.cu", "dsq_static.cu", "dsq_whole.cu",
           "dsq_mma.cu", "dsq_orth.cu", "dsq_orth_small.cu", "dsq_int8.cu"]
HEADERS = ["dsq_common.cuh", "dsq_chunked.cuh", "dsq_mma.cuh", "dsq_orth.cuh", "dsq_internal.h", os.path.join("..", "..", "include", "dsq.h")]

NVCC_FLAGS = [
    "-gencode", "arch=compute_100a,code=sm_100a", "-lineinfo", "-O3", "-std=c++17",
    "-fmad=false",                      # every multiply and add rounds separately
    "-Xcompiler", "-fPIC",
]


def _stale() -> bool:
    if not os.path.exists(LIB):
        return True
    t = os.path.getmtime(LIB)
    return any(os.path.getmtime(os.path.join(CSRC, f)) > t for f in SOURCES + HEADERS)


def build_call() -> str | None:
    """The extension, where a C compiler and Python.h are there; without it the same calls go through ctypes, a few microseconds slower."""
    tmp = CALL_LIB + ".tmp"
    try:
        subprocess.run([os.environ.get("CC", "gcc"), "-O2", "-shared", "-fPIC", "-I" + sysconfig.get_paths()["include"], CALL_SRC, "-o", tmp],
                       check=True)
    except (OSError, subprocess.CalledProcessError) as e:
        print(f"{os.path.basename(CALL_LIB)} was not built ({e}): short calls go through ctypes", file=sys.stderr)
        return None
    os.replace(tmp, CALL_LIB)
    return CALL_LIB


def build(force: bool = False, verbose: bool = False) -> str:
    if force or not os.path.exists(CALL_LIB) or os.path.getmtime(CALL_SRC) > os.path.getmtime(CALL_LIB):
        build_call()
    if not force and not _stale():
        return LIB
    nvcc = os.environ.get("NVCC", "nvcc")
    os.makedirs(OBJ, exist_ok=True)
    extra = ["-Xptxas", "-v"] if verbose else []

    def compile_one(src: str) -> str:
        obj = os.path.join(OBJ, src[:-3] + ".o")
        subprocess.run([nvcc] + NVCC_FLAGS + extra + ["-c", os.path.join(CSRC, src), "-o", obj], check=True)
        return obj

    with ThreadPoolExecutor(max_workers=min(len(SOURCES), os.cpu_count() or 1)) as pool:
        objs = list(pool.map(compile_one, SOURCES))
    subprocess.run([nvcc, "-gencode", "arch=compute_100a,code=sm_100a", "-shared", "-o", LIB + ".tmp"] + objs, check=True)
    os.replace(LIB + ".tmp", LIB)
    return LIB


if __name__ == "__main__":
    print(build(force="--force" in sys.argv, verbose="-v" in sys.argv))
