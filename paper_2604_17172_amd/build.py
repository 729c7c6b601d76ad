"""Build libuzip.so (gfx950) in-tree with hipcc.

    python paper_2604_17172_amd/build.py      (or __graft_entry__.build())
"""
from __future__ import annotations

import os
import shutil
import subprocess
import tempfile
from concurrent.futures import ThreadPoolExecutor

HERE = os.path.dirname(os.path.abspath(__file__))
ROOT = os.path.dirname(HERE)
CSRC = os.path.join(HERE, "csrc")
SRC = os.path.join(CSRC, "uzip.hip")
SOURCES = [SRC] + [os.path.join(CSRC, name) for name in (
    "kv_cache.hip", "kv_attend.hip", *(f"kv_attend_{dim}.hip" for dim in (64, 96, 128, 192, 256)),
    "rotary.hip", "latent.hip", "latent_256.hip", "latent_512.hip",
    "expanded.hip", "expanded_64.hip", "expanded_128.hip")]
LIB_PATH = os.path.join(HERE, "_build", "libuzip.so")

HIPCC_FLAGS = [
    "--offload-arch=gfx950", "-O3", "-std=c++17", "-fPIC",
    # no packed fp32 instructions in any kernel
    "-Xclang", "-target-feature", "-Xclang", "-packed-fp32-ops",
    # the fused reduce is an exact fixed-order binary32 sum
    "-ffp-contract=off",
    "-Wall", "-Wno-unused-command-line-argument",
]

# Sources whose matrix instructions accumulate in vector registers: a tile's scores are read by vector instructions at once,
# and would move there from the accumulation registers (a fifth of the loop's instructions).
SOURCE_FLAGS = {name: ["-mllvm", "-amdgpu-mfma-vgpr-form=1"]
                for name in ("expanded_64.hip", "expanded_128.hip")}


def _hipcc(args: list[str], verbose: bool) -> None:
    res = subprocess.run(["hipcc", *HIPCC_FLAGS, "-I", os.path.join(ROOT, "include"), *args], capture_output=True,
                         text=True)
    if res.returncode != 0:
        raise RuntimeError("hipcc failed:\n" + res.stdout + res.stderr)
    if verbose and res.stderr:
        print(res.stderr)


def build(verbose: bool = False) -> str:
    """Compile every source, side by side, and link the library."""
    os.makedirs(os.path.dirname(LIB_PATH), exist_ok=True)
    objs = tempfile.mkdtemp(prefix="uzip_build_")
    try:
        units = [(src, os.path.join(objs, os.path.basename(src) + ".o")) for src in SOURCES]
        with ThreadPoolExecutor(max_workers=8) as pool:
            for job in [pool.submit(_hipcc, [*SOURCE_FLAGS.get(os.path.basename(src), []), "-c", src, "-o", obj], verbose) for src, obj in units]:
                job.result()
        tmp = LIB_PATH + ".tmp"
        _hipcc(["-shared", *[obj for _, obj in units], "-o", tmp], verbose)
    finally:
        shutil.rmtree(objs, ignore_errors=True)
    os.replace(tmp, LIB_PATH)
    return LIB_PATH


if __name__ == "__main__":
    print(build(verbose=True))
