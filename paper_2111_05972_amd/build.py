"""Build the HIP shared library in-tree with hipcc for gfx950, and the Python module that calls it (no torch involved)."""
import os
import subprocess
import sys
import sysconfig
import tempfile
from concurrent.futures import ThreadPoolExecutor

HERE = os.path.dirname(os.path.abspath(__file__))
CSRC = os.path.join(HERE, "csrc")
LIB = os.path.join(HERE, "libtp_layer.so")
SOURCES = ["tp_layer.cpp", "simple_kernels.hip", "gemm_bf16.hip", "attn_bf16.hip", "gemm_f32.hip", "attn_f32.hip", "layernorm.hip",
           "rope.hip", "qk_norm_rope.hip", "dropout.hip", "attn_packed_plan.hip", "attn_packed_bf16.hip", "attn_packed_f32.hip", "lm_loss.hip"]
FLAGS = ["--offload-arch=gfx950", "-O3", "-std=c++17", "-fPIC",
         "-Xclang", "-target-feature", "-Xclang", "-packed-fp32-ops",
         "-Wno-unused-command-line-argument", "-Wno-option-ignored"]
CALLS = os.path.join(HERE, "_calls" + sysconfig.get_config_var("EXT_SUFFIX"))         # the Python module that calls the library
JOBS = 4                    # compilers at once: each takes about 1 GB


def _run(cmd, verbose):
    if verbose:
        print(" ".join(cmd), flush=True)
    r = subprocess.run(cmd, stdout=subprocess.PIPE, stderr=subprocess.STDOUT, text=True)
    out = "\n".join(l for l in r.stdout.splitlines() if "packed-fp32-ops" not in l and l.strip())
    if r.returncode != 0:
        raise RuntimeError("hipcc failed:\n" + out)
    if verbose and out:
        print(out)
    return out


def build(verbose=False, extra=(), out=LIB):
    """Every source is compiled, side by side, and linked into `out`; then, for the package's own library, the module that calls it (without Python's headers
    there is none, and ctypes calls the library)."""
    hipcc = os.environ.get("HIPCC", "/opt/rocm/bin/hipcc")
    with tempfile.TemporaryDirectory() as tmp:
        objects = [os.path.join(tmp, s + ".o") for s in SOURCES]
        compile_one = lambda s, o: _run([hipcc] + FLAGS + list(extra) + ["-x", "hip", "-c", os.path.join(CSRC, s), "-o", o], verbose)  # noqa: E731
        with ThreadPoolExecutor(JOBS) as pool:
            text = list(pool.map(compile_one, SOURCES, objects))
        text.append(_run([hipcc, "--offload-arch=gfx950", "-fPIC", "-shared"] + objects + ["-o", out], verbose))
    include = sysconfig.get_paths()["include"]
    if out == LIB and os.path.exists(os.path.join(include, "Python.h")):
        text.append(_run([os.environ.get("CXX", "g++"), "-O2", "-std=c++17", "-fPIC", "-shared", "-I", include, os.path.join(CSRC, "calls.cpp"), "-o", CALLS, "-ldl"], verbose))
    return "\n".join(t for t in text if t)


if __name__ == "__main__":
    args = sys.argv[1:]
    out = LIB
    if "-o" in args:            # build a variant beside the default library (tuning experiments)
        i = args.index("-o")
        out = os.path.abspath(args[i + 1])
        del args[i:i + 2]
    build(verbose=True, extra=args, out=out)
    print("built", out)
