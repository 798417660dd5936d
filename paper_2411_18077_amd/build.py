"""Build libminikv.so (hand-written HIP for gfx950) and _bind.so (its binding's quick calls, host code) in-tree.

    python -m paper_2411_18077_amd.build          # compile every translation unit and link

hipcc cross-compiles without a GPU, so this runs anywhere the ROCm toolchain is installed.
"""
import os
import subprocess
import sys
import sysconfig
from concurrent.futures import ThreadPoolExecutor

HERE = os.path.dirname(os.path.abspath(__file__))
ROOT = os.path.dirname(HERE)
CSRC = os.path.join(HERE, "csrc")
OBJ = os.path.join(HERE, "_build")
LIB = os.path.join(HERE, "libminikv.so")
BIND = os.path.join(HERE, "_bind.so")                  # checks and passes on the arguments of the calls between two launches (host code)

SOURCES = ["api.hip", "quantize.hip", "decode_scalar.hip", "decode_tiled.hip", "decode_static.hip", "select.hip",
           "prefill_attn.hip", "pt.hip", "blocks.hip", "decode_blk.hip", "prompt_blk.hip", "norm_rope.hip", "pages.hip"]

FLAGS = [
    "--offload-arch=gfx950", "-O3", "-std=c++17", "-fPIC",
    "-I" + os.path.join(ROOT, "include"), "-I" + CSRC,
    # packed-FP32 VALU forms are kept out of the generated code on the test machines
    "-Xclang", "-target-feature", "-Xclang", "-packed-fp32-ops",
    "-Wall", "-Wno-unused-function",
]
# per-file extras: the quantizer's code decisions are individually rounded binary32 operations
# quantize.hip: no contraction (its operations are separately rounded by definition); inputs are finite by contract, so
# the packed fp16 min / max need no NaN canonicalisation (-fno-honor-nans drops one instruction of three there)
EXTRA = {"quantize.hip": ["-ffp-contract=off", "-fno-honor-nans"], "pt.hip": ["-ffp-contract=off"],
         # finite inputs by contract: the running maximum needs no NaN canonicalisation (an instruction per score)
         "prefill_attn.hip": ["-fno-honor-nans"], "prompt_blk.hip": ["-fno-honor-nans"]}


def hipcc():
    for p in (os.environ.get("HIPCC"), "/opt/rocm/bin/hipcc", "hipcc"):
        if p and (os.path.isabs(p) and os.path.exists(p) or not os.path.isabs(p)):
            return p
    raise RuntimeError("hipcc not found")


def _compile(src):
    obj = os.path.join(OBJ, src.replace(".hip", ".o"))
    cmd = [hipcc(), *FLAGS, *EXTRA.get(src, []), "-c", os.path.join(CSRC, src), "-o", obj]
    r = subprocess.run(cmd, capture_output=True, text=True)
    if r.returncode:
        raise RuntimeError("hipcc failed for %s:\n%s\n%s" % (src, r.stdout, r.stderr))
    warn = "\n".join(l for l in r.stderr.splitlines() if "packed-fp32-ops" not in l and l.strip())
    return obj, warn


def bound_to():
    """What _bind.so is built for and has to run with: it takes tensors and objects as these lay them out."""
    import torch
    return "torch %s, Python %d.%d" % ((torch.__version__,) + sys.version_info[:2])


def _compile_bind():
    import torch
    root = os.path.dirname(torch.__file__)
    obj = os.path.join(OBJ, "bind.o")
    cmd = ["g++", "-O2", "-std=c++17", "-fPIC", "-Wall", '-DMINIKV_BUILT_FOR="%s"' % bound_to(), "-D_GLIBCXX_USE_CXX11_ABI=%d" % torch._C._GLIBCXX_USE_CXX11_ABI,
           "-I" + os.path.join(ROOT, "include"), "-I" + sysconfig.get_paths()["include"], "-isystem", os.path.join(root, "include"),
           "-isystem", os.path.join(root, "include", "torch", "csrc", "api", "include"), "-c", os.path.join(CSRC, "bind.cpp"), "-o", obj]
    r = subprocess.run(cmd, capture_output=True, text=True)
    if r.returncode:
        raise RuntimeError("g++ failed for bind.cpp:\n%s\n%s" % (r.stdout, r.stderr))
    return ["g++", "-shared", obj, "-o", BIND, "-L" + HERE, "-lminikv", "-Wl,-rpath,$ORIGIN", "-L" + os.path.join(root, "lib"), "-ltorch_python",
            "-ltorch_cpu", "-lc10"]


def build(verbose=True):
    os.makedirs(OBJ, exist_ok=True)
    with ThreadPoolExecutor(max_workers=4) as ex:
        bind = ex.submit(_compile_bind)
        results = list(ex.map(_compile, SOURCES))
    objs = [o for o, _ in results]
    for _, w in results:
        if w and verbose:
            print(w, file=sys.stderr)
    cmd = [hipcc(), "--offload-arch=gfx950", "-shared", "-fPIC", *objs, "-o", LIB]
    r = subprocess.run(cmd, capture_output=True, text=True)
    if r.returncode:
        raise RuntimeError("link failed:\n%s\n%s" % (r.stdout, r.stderr))
    link_bind = bind.result()                          # (what was wrong there, now that the library is there)
    r = subprocess.run(link_bind, capture_output=True, text=True)
    if r.returncode:
        raise RuntimeError("link of _bind.so failed:\n%s\n%s" % (r.stdout, r.stderr))
    return LIB


if __name__ == "__main__":
    print(build())
