"""Builds libsom.so (the HIP kernels and the C ABI of include/som.h) for gfx950 with hipcc."""
from __future__ import annotations

import os
import subprocess
import tempfile
from concurrent.futures import ThreadPoolExecutor

HERE = os.path.dirname(os.path.abspath(__file__))
ROOT = os.path.dirname(HERE)
CSRC = os.path.join(HERE, "csrc")
LIB = os.path.join(HERE, "libsom.so")
SOURCES = [os.path.join(CSRC, "som_sweep.hip"), os.path.join(CSRC, "som_rows.hip"),
           os.path.join(CSRC, "som_kernels.hip"), os.path.join(CSRC, "som_update.hip"),
           os.path.join(CSRC, "som_api.cpp"), os.path.join(CSRC, "som_noalloc.hip"),
           os.path.join(CSRC, "som_mm_nn.hip"), os.path.join(CSRC, "som_mm_nt.hip"),
           os.path.join(CSRC, "som_mm_tn.hip"), os.path.join(CSRC, "som_few.hip"), os.path.join(CSRC, "som_route.hip"),
           os.path.join(CSRC, "som_experts.hip"), os.path.join(CSRC, "som_clip.hip"),
           os.path.join(CSRC, "som_dense_api.cpp"), os.path.join(CSRC, "som_norm_rows.hip"),
           os.path.join(CSRC, "som_norm_grad.hip"), os.path.join(CSRC, "som_adamw.hip"),
           os.path.join(CSRC, "som_mx4.hip"), os.path.join(CSRC, "som_mx4_few.hip"),
           os.path.join(CSRC, "som_mx4_half.hip"), os.path.join(CSRC, "som_mx4_packed.hip"),
           os.path.join(CSRC, "som_layer_api.cpp")]

HIPCC = os.environ.get("HIPCC", "/opt/rocm/bin/hipcc")
ARCH = "gfx950"

# Packed fp32 instructions are kept out of every device code object; fp contraction
# is off so that every rounding is the one the source writes.
FLAGS = [
    f"--offload-arch={ARCH}", "-O3", "-std=c++17", "-fPIC", "-shared",
    "-ffp-contract=off",
    "-Xclang", "-target-feature", "-Xclang", "-packed-fp32-ops",
    "-Wall", "-Wno-unused-command-line-argument",
    f"-I{os.path.join(ROOT, 'include')}",
]


# The benchmark's read-stream probe (its bandwidth denominator), a library of its own.
PROBE_LIB = os.path.join(HERE, "libsomprobe.so")
PROBE_SOURCES = [os.path.join(CSRC, "probe.hip")]


def _run(cmd, verbose):
    if verbose:
        print(" ".join(cmd), flush=True)
    subprocess.run(cmd, check=True)


def _compile(sources, out, verbose):
    """Each source to an object of its own, as many at once as there are CPUs (up to eight), then one library."""
    with tempfile.TemporaryDirectory() as tmp:
        objects = [os.path.join(tmp, os.path.basename(s) + ".o") for s in sources]
        flags = [f for f in FLAGS if f != "-shared"]
        with ThreadPoolExecutor(min(8, os.cpu_count() or 1)) as pool:
            list(pool.map(lambda so: _run([HIPCC, *flags, "-c", so[0], "-o", so[1]], verbose), zip(sources, objects)))
        linked = out + ".tmp"
        _run([HIPCC, *FLAGS, *objects, "-o", linked], verbose)
    os.replace(linked, out)


def build(verbose: bool = False) -> str:
    _compile(SOURCES, LIB, verbose)
    _compile(PROBE_SOURCES, PROBE_LIB, verbose)
    return LIB


if __name__ == "__main__":
    print(build(verbose=True))
