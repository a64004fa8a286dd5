"""Builds libactqkv.so (HIP, gfx950) with hipcc, a call for each source, and the Python extension module that
calls it with one g++ call, both next to this file."""
from __future__ import annotations

import os
import shutil
import subprocess
import sysconfig
import tempfile
from concurrent.futures import ThreadPoolExecutor

HERE = os.path.dirname(os.path.abspath(__file__))
CSRC = os.path.join(HERE, "csrc")
LIB = os.path.join(HERE, "libactqkv.so")
NATIVE = os.path.join(HERE, "_native.so")

SOURCES = ["api.hip", "probe.hip", "score.hip", "select.hip", "attn_prefill_f32.hip",
           "attn_prefill_mfma.hip", "attn_decode.hip", "append.hip", "cutoff.hip", "gather.hip",
           "decode_retrieve.hip", "attn_static.hip", "paged_api.hip", "paged_append.hip",
           "paged_append_rotated.hip", "paged8_append.hip", "paged_chunk.hip",
           "paged_chunk_f32.hip", "paged8_chunk.hip", "paged8_chunk_f32.hip", "paged_step.hip",
           "paged8_step.hip", "paged_selected.hip", "paged_chosen_chunk.hip",
           "paged_chosen_chunk_f32.hip", "paged_select.hip", "paged_weights.hip",
           "paged_evict.hip"]

FLAGS = ["--offload-arch=gfx950", "-O3", "-std=c++17", "-fPIC",
         # packed fp32 instructions are kept out of the generated code
         "-Xclang", "-target-feature", "-Xclang", "-packed-fp32-ops",
         "-Wall", "-Wno-unused-function"]


def _native_command() -> list:
    import torch
    root = os.path.dirname(torch.__file__)
    flags = ["-O2", "-std=c++17", "-fPIC", "-shared", "-D__HIP_PLATFORM_AMD__=1", "-DUSE_ROCM=1"]
    include = ["-I" + sysconfig.get_paths()["include"], "-isystem" + os.path.join(root, "include"),
               "-isystem" + os.path.join(root, "include", "torch", "csrc", "api", "include"), "-isystem/opt/rocm/include"]
    libs = ["-L" + os.path.join(root, "lib"), "-ltorch_python", "-ltorch_cpu", "-lc10_hip", "-lc10", "-ldl"]
    return [shutil.which("g++") or "g++"] + flags + include + [os.path.join(CSRC, "py_native.cpp"), "-o", NATIVE] + libs


def build(verbose: bool = False) -> str:
    """Compiles every source, a few at a time, and links them."""
    hipcc = shutil.which("hipcc") or "/opt/rocm/bin/hipcc"
    noise = "is not a recognized feature for this target"
    with tempfile.TemporaryDirectory() as objects, ThreadPoolExecutor(min(8, os.cpu_count() or 1)) as pool:
        made = [os.path.join(objects, s + ".o") for s in SOURCES]
        commands = [_native_command()] + [[hipcc] + FLAGS + ["-c", os.path.join(CSRC, s), "-o", o] for s, o in zip(SOURCES, made)]
        link = [hipcc] + FLAGS + ["-shared"] + made + ["-o", LIB]

        def run(c):
            if verbose:
                print(" ".join(c))
            r = subprocess.run(c, stdout=subprocess.PIPE, stderr=subprocess.PIPE, text=True)
            err = "\n".join(l for l in r.stderr.splitlines() if noise not in l)
            if verbose and err.strip():
                print(err)
            return "" if r.returncode == 0 else os.path.basename(c[0]) + " failed:\n" + err

        failed = [f for f in pool.map(run, commands) if f] or [f for f in [run(link)] if f]
    if failed:
        raise RuntimeError("\n".join(failed))
    return LIB


if __name__ == "__main__":
    print(build(verbose=True))
