"""Builds libmixaq.so (hand-written HIP for gfx950) in-tree with hipcc."""
import os
import subprocess
import tempfile
from concurrent.futures import ThreadPoolExecutor

HERE = os.path.dirname(os.path.abspath(__file__))
CSRC = os.path.join(HERE, "csrc")
LIB = os.path.join(HERE, "libmixaq.so")
SOURCES = ["api.hip", "kernels.hip", "downsample.hip", "scaled_quantize.hip", "scaled_linear.hip", "residual_norm.hip", "token_quantize.hip", "token_linear.hip",
           "group_norm.hip", "cost_sampler.cpp"]
# -ffp-contract=off: the pinned binary32 sequences must not be re-fused;
# packed fp32 instructions are disabled for the device pass.
FLAGS = ["-O3", "--offload-arch=gfx950", "-std=c++17", "-ffp-contract=off", "-fPIC",
         "-Xclang", "-target-feature", "-Xclang", "-packed-fp32-ops", "-Wall", "-Wno-unused-function"]


def _hipcc(args):
    res = subprocess.run(["hipcc"] + args, capture_output=True, text=True)
    noise = "is not a recognized feature for this target"
    err = "\n".join(l for l in res.stderr.splitlines() if noise not in l)
    if res.returncode != 0:
        raise RuntimeError("hipcc failed:\n" + err)
    return err


def build(verbose=False):
    """Every source on its own, side by side, then one library."""
    with tempfile.TemporaryDirectory() as tmp:
        objects = [os.path.join(tmp, s + ".o") for s in SOURCES]
        with ThreadPoolExecutor(max_workers=4) as pool:
            said = list(pool.map(lambda so: _hipcc(FLAGS + ["-c", "-x", "hip", os.path.join(CSRC, so[0]), "-o", so[1]]), zip(SOURCES, objects)))
        said.append(_hipcc(["--offload-arch=gfx950", "-fPIC", "-shared", "-o", LIB] + objects))
    if verbose and "".join(said).strip():
        print("\n".join(said))
    return LIB


if __name__ == "__main__":
    print(build(verbose=True))
