"""Compile the HIP sources of the runtime into ``libmt.so`` next to this file (gfx950 only), and the calls on torch tensors into ``_answers.so``."""
import os
import subprocess
import sys
import sysconfig

HERE = os.path.dirname(os.path.abspath(__file__))
CSRC = os.path.join(HERE, "csrc")
LIB = os.path.join(HERE, "libmt.so")
CALLS = os.path.join(HERE, "_answers.so")
SOURCES = ["mt_api.cpp", "batcher.hip", "fc_stream.hip", "fc_big.hip", "conv.hip", "conv_first.hip", "small.hip",
           "lm_api.cpp", "lm_norm.hip", "lm_linear4.hip", "lm_score.hip",
           "lm_cache_api.cpp", "lm_kv_write.hip", "lm_attend.hip", "lm_pages.hip", "lm_sample.hip"]
FLAGS = ["--offload-arch=gfx950", "-O3", "-std=c++17", "-fPIC", "-Wall", "-Wno-unused-function", "-Wno-inline-asm",
         # keep the compiler from forming packed-fp32 VALU ops
         "-Xclang", "-target-feature", "-Xclang", "-packed-fp32-ops"]


def compile_one(src: str, verbose: bool) -> str:
    obj = os.path.join(CSRC, os.path.splitext(src)[0] + ".o")
    cmd = ["hipcc", *FLAGS, "-x", "hip", "-c", os.path.join(CSRC, src), "-o", obj]
    if verbose:
        print(" ".join(cmd), flush=True)
    r = subprocess.run(cmd, stdout=subprocess.PIPE, stderr=subprocess.STDOUT, text=True)
    out = "\n".join(l for l in r.stdout.splitlines() if "not a recognized feature for this target" not in l)
    if r.returncode != 0:
        raise RuntimeError("hipcc failed for %s:\n%s" % (src, out))
    if out.strip():
        print(out, file=sys.stderr)
    return obj


def compile_calls(verbose: bool) -> None:
    """csrc/lm_torch.cpp: host code, against torch's headers."""
    import torch
    home = os.path.dirname(torch.__file__)
    cmd = ["g++", "-O2", "-std=c++17", "-Wall", "-fPIC", "-shared", "-D_GLIBCXX_USE_CXX11_ABI=%d" % torch._C._GLIBCXX_USE_CXX11_ABI,
           *("-isystem" + d for d in (os.path.join(home, "include"), os.path.join(home, "include", "torch", "csrc", "api", "include"), sysconfig.get_paths()["include"])),
           os.path.join(CSRC, "lm_torch.cpp"), "-L" + os.path.join(home, "lib"), "-ltorch_python", "-ltorch_cpu", "-lc10", "-o", CALLS]
    if verbose:
        print(" ".join(cmd), flush=True)
    r = subprocess.run(cmd, stdout=subprocess.PIPE, stderr=subprocess.STDOUT, text=True)
    if r.returncode != 0:
        raise RuntimeError("g++ failed for lm_torch.cpp:\n%s" % r.stdout)
    if r.stdout.strip():
        print(r.stdout, file=sys.stderr)


def build(verbose: bool = False) -> str:
    from concurrent.futures import ThreadPoolExecutor
    with ThreadPoolExecutor(max_workers=min(8, os.cpu_count() or 1)) as pool:       # one hipcc per source
        calls = pool.submit(compile_calls, verbose)
        objs = list(pool.map(lambda src: compile_one(src, verbose), SOURCES))
        calls.result()
    cmd = ["hipcc", "--offload-arch=gfx950", "-shared", "-fPIC", "-o", LIB, *objs]
    subprocess.check_call(cmd)
    return LIB


if __name__ == "__main__":
    print(build(verbose=True))
