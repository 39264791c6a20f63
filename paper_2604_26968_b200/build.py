"""Builds libkvtier.so (the CUDA library behind include/kvtier.h) for sm_100a.

nvcc cross-compiles without a GPU.  The library is placed inside the package
directory so that it travels with the source tree.
"""
import os
import subprocess
import sys

HERE = os.path.dirname(os.path.abspath(__file__))
ROOT = os.path.dirname(HERE)
CSRC = os.path.join(HERE, "csrc")
LIB = os.path.join(HERE, "libkvtier.so")
SOURCES = ["kvtier_host.cu", "kv_attention_host.cu", "kv_score.cu", "kv_select.cu", "kv_select_persist.cu", "kv_blocks.cu", "kv_heads.cu", "kv_prefetch.cu", "kv_dedup.cu", "kv_move.cu", "kv_move_tma.cu",
           "kv_append.cu", "kv_attend.cu", "kv_attend_tiles.cu", "kv_attend_stream.cu", "kv_attention.cu"]

NVCC_FLAGS = [
    "-gencode", "arch=compute_100a,code=sm_100a",
    "-O3", "-lineinfo", "-std=c++17",
    "-diag-suppress", "186",
    "--fmad=false",            # binary32 arithmetic exactly as written, never fused
    "-Xcompiler", "-fPIC", "-shared",
    "-I", os.path.join(ROOT, "include"), "-I", CSRC,
]


def _stale() -> bool:
    if not os.path.exists(LIB):
        return True
    t = os.path.getmtime(LIB)
    deps = [os.path.join(CSRC, f) for f in os.listdir(CSRC)] + [os.path.join(ROOT, "include", "kvtier.h")]
    return any(os.path.getmtime(d) > t for d in deps)


def build(force: bool = False, verbose: bool = False) -> str:
    if not force and not _stale():
        return LIB
    nvcc = os.environ.get("NVCC", "/usr/local/cuda/bin/nvcc")
    tmp = LIB + ".tmp.%d" % os.getpid()
    cmd = [nvcc, *NVCC_FLAGS, *(["-Xptxas", "-v"] if verbose else []),
           *[os.path.join(CSRC, s) for s in SOURCES], "-o", tmp]
    subprocess.run(cmd, check=True)
    os.replace(tmp, LIB)
    return LIB


if __name__ == "__main__":
    print(build(force="--force" in sys.argv, verbose="-v" in sys.argv))
