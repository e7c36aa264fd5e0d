"""Build libaha.so (the gfx950 kernels and their C ABI) in-tree with hipcc, and the binding's look at its tensors with g++."""
from __future__ import annotations

import os
import subprocess
import sys
import sysconfig
from concurrent.futures import ThreadPoolExecutor

HERE = os.path.dirname(os.path.abspath(__file__))
CSRC = os.path.join(HERE, "csrc")
LIB = os.path.join(HERE, "libaha.so")
TENSORS = os.path.join(HERE, "_tensors.so")
OBJDIR = os.path.join(HERE, "_build")

SOURCES = ["aha_api.hip", "value_prior.hip", "score_f32.hip", "score_hold_f32.hip", "score_bf16.hip", "score_full.hip", "score_window.hip", "score_share.hip", "score_given.hip",
           "attn_window.hip", "topk.hip", "compact.hip", "decode.hip",
           "rotate.hip", "shared_attn.hip", "shared_wide.hip", "shared_api.hip",
           "prompt_attn.hip", "prompt_wide.hip", "prompt_mid.hip", "paged_attn.hip", "paged_evict.hip"]

HIPCC_FLAGS = [
    "--offload-arch=gfx950", "-O3", "-std=c++17", "-fPIC",
    "-Xclang", "-target-feature", "-Xclang", "-packed-fp32-ops",
    "-Wno-unused-value", "-Wno-unknown-attributes",
]


def hipcc() -> str:
    for c in (os.environ.get("HIPCC"), "/opt/rocm/bin/hipcc", "hipcc"):
        if c and (os.path.sep not in c or os.path.exists(c)):
            return c
    raise RuntimeError("hipcc not found")


def build_tensors() -> None:
    """Compile the Python module that checks a call's tensors against their description."""
    import torch
    from torch.utils import cpp_extension
    include = cpp_extension.include_paths() + [sysconfig.get_paths()["include"]]
    tmp = TENSORS + ".tmp.%d" % os.getpid()
    cmd = ["g++", "-O2", "-std=c++17", "-shared", "-fPIC", "-D_GLIBCXX_USE_CXX11_ABI=%d" % torch._C._GLIBCXX_USE_CXX11_ABI,
           *("-isystem" + p for p in include), os.path.join(CSRC, "tensors.cpp"), "-o", tmp,
           *("-L" + p for p in cpp_extension.library_paths()), "-ltorch_python", "-ltorch_cpu", "-lc10"]
    r = subprocess.run(cmd, capture_output=True, text=True)
    if r.returncode != 0:
        raise RuntimeError("g++ failed on tensors.cpp:\n%s" % r.stderr[-6000:])
    os.replace(tmp, TENSORS)


def build(verbose: bool = False, jobs: int = 8) -> str:
    """Compile every kernel source for gfx950 and link libaha.so. Always compiles."""
    os.makedirs(OBJDIR, exist_ok=True)
    cc = hipcc()

    def compile_one(src):
        obj = os.path.join(OBJDIR, src.replace(".hip", ".o"))
        cmd = [cc, *HIPCC_FLAGS, "-c", os.path.join(CSRC, src), "-o", obj]
        r = subprocess.run(cmd, capture_output=True, text=True)
        if r.returncode != 0:
            raise RuntimeError("hipcc failed on %s:\n%s" % (src, r.stderr[-6000:]))
        if verbose and r.stderr.strip():
            sys.stderr.write(r.stderr)
        return obj

    with ThreadPoolExecutor(max_workers=jobs) as ex:
        tensors = ex.submit(build_tensors)
        objs = list(ex.map(compile_one, SOURCES))
        failed = tensors.exception()
    if failed is not None:  # (no g++ or none of torch's headers, for one: the binding makes the same checks itself, slower)
        if os.path.exists(TENSORS):
            os.remove(TENSORS)
        sys.stderr.write("_tensors is not built, a call's checks take 7 us instead of 0.5: %s\n" % failed)
    tmp = LIB + ".tmp.%d" % os.getpid()
    cmd = [cc, "--offload-arch=gfx950", "-shared", "-fPIC", "-o", tmp, *objs,
           "-Wl,--version-script=" + os.path.join(CSRC, "aha.map")]
    r = subprocess.run(cmd, capture_output=True, text=True)
    if r.returncode != 0:
        raise RuntimeError("link failed:\n%s" % r.stderr[-6000:])
    os.replace(tmp, LIB)
    return LIB


if __name__ == "__main__":
    print(build(verbose=True))
