"""Builds libmarl_gfx950.so from csrc/ with hipcc for gfx950 (cross-compiles without a GPU)."""
import os
import subprocess
import sys
from concurrent.futures import ThreadPoolExecutor

HERE = os.path.dirname(os.path.abspath(__file__))
CSRC = os.path.join(HERE, "csrc")
INCLUDE = os.path.join(os.path.dirname(HERE), "include")
LIB = os.path.join(HERE, "libmarl_gfx950.so")
SOURCES = ["api.hip", "env_kernels.hip", "gae_kernels.hip", "policy_kernels.hip", "ppo_kernels.hip",
           "recurrent_kernels.hip", "rollout_v3.hip", "rollout_v5.hip", "rollout_v7.hip"]
# the operators of sequence memories
MEMORY_SOURCES = ["linear_attention.hip", "linear_attention_f32.hip", "linear_attention_bf16.hip", "layer_norm.hip", "rotary.hip"]
# attention over a window, and the norm of heads with their rotation
WINDOW_SOURCES = ["window_attention_f32.hip", "window_attention_bf16.hip", "window_attention.hip", "norm_rotary.hip"]
FLAGS = ["--offload-arch=gfx950", "-O3", "-std=c++17", "-fPIC", "-I", INCLUDE, "-I", CSRC,
         # packed fp32 ALU forms are kept off on this target
         "-Xclang", "-target-feature", "-Xclang", "-packed-fp32-ops",
         "-Wall", "-Wno-unused-function"]

# Window attention's products with their sums in ordinary registers: the compiler otherwise copies 128 of them to the other half of the register file and back for
# every tile where a wavefront has more than 256
EXTRA_FLAGS = {src: ["-mllvm", "-amdgpu-mfma-vgpr-form=1"] for src in ("window_attention_f32.hip", "window_attention_bf16.hip")}


def flags(src):
    return [*FLAGS, *EXTRA_FLAGS.get(src, [])]


def _compile(src):
    obj = os.path.join(CSRC, src.replace(".hip", ".o"))
    subprocess.check_call(["hipcc", *flags(src), "-c", os.path.join(CSRC, src), "-o", obj])
    return obj


def build(verbose=True):
    sources = WINDOW_SOURCES + SOURCES + MEMORY_SOURCES
    with ThreadPoolExecutor(max_workers=min(os.cpu_count() or 8, len(sources))) as ex:
        objs = list(ex.map(_compile, sources))
    subprocess.check_call(["hipcc", "--offload-arch=gfx950", "-shared", "-fPIC", "-o", LIB, *objs])
    if verbose:
        print("built", LIB)
    return LIB


if __name__ == "__main__":
    build()
    sys.exit(0)
