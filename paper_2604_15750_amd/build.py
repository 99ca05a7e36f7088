"""Compile csrc/*.hip into paper_2604_15750_amd/libdlm.so for gfx950 and csrc/decisions_py.c into _decisions (in-tree, no torch dependency), and
csrc/kv8_py.cpp and csrc/q8_py.cpp into _kv8 and _q8 where torch and its headers are there."""
import os
import shutil
import subprocess
import sys
import sysconfig
from concurrent.futures import ThreadPoolExecutor

HERE = os.path.dirname(os.path.abspath(__file__))
CSRC = os.path.join(HERE, "csrc")
OUT = os.path.join(HERE, "libdlm.so")
# (tagged with the interpreter it was built for: it reads that one's objects, and another does not load it)
OUT_PY = os.path.join(HERE, "_decisions" + sysconfig.get_config_var("EXT_SUFFIX"))
OUT_KV8 = os.path.join(HERE, "_kv8" + sysconfig.get_config_var("EXT_SUFFIX"))
OUT_Q8 = os.path.join(HERE, "_q8" + sysconfig.get_config_var("EXT_SUFFIX"))
HIPCC = os.environ.get("HIPCC", "/opt/rocm/bin/hipcc")
# amdgpu-kernarg-preload-count: a kernel's first arguments (14 dwords at most, up to the first struct) arrive in scalar registers with the
# launch instead of by a trip to memory, so its first loads go out at once (161 launches of an in-block pass of the 8B model: 2888 -> 2864 us;
# the 13 of the fp32 model's 54.0 -> 53.0).
FLAGS = ["--offload-arch=gfx950", "-O3", "-std=c++17", "-fPIC", "-Xclang", "-target-feature", "-Xclang", "-packed-fp32-ops",
         "-mllvm", "-amdgpu-kernarg-preload-count=14", "-Wno-unused-command-line-argument"] + os.environ.get("DLM_EXTRA_HIPCC_FLAGS", "").split()


def build(verbose=False):
    srcs = sorted(f for f in os.listdir(CSRC) if f.endswith(".hip"))
    objdir = os.path.join(HERE, "_build")
    os.makedirs(objdir, exist_ok=True)

    def cc(src):
        obj = os.path.join(objdir, src[:-4] + ".o")
        cmd = [HIPCC, *FLAGS, "-c", os.path.join(CSRC, src), "-o", obj]
        r = subprocess.run(cmd, capture_output=True, text=True)
        err = "\n".join(l for l in r.stderr.splitlines() if "packed-fp32-ops" not in l)
        if r.returncode != 0:
            raise RuntimeError(f"hipcc failed on {src}:\n{err}")
        if verbose and err.strip():
            print(err, file=sys.stderr)
        return obj

    with ThreadPoolExecutor(max_workers=min(8, len(srcs))) as ex:
        objs = list(ex.map(cc, srcs))
    r = subprocess.run([HIPCC, "--offload-arch=gfx950", "-shared", "-fPIC", "-o", OUT, *objs], capture_output=True, text=True)
    if r.returncode != 0:
        raise RuntimeError("link failed:\n" + r.stderr)
    build_extension()
    build_kv8_extension()
    build_q8_extension()
    return OUT


def _compile_extension(source, out, calls, compiler="gcc", flags=(), needed=True):
    """None without the compiler or Python's headers (or, if not `needed`, where it refuses the source): `calls` then go through ctypes."""
    cc, include = shutil.which(compiler), sysconfig.get_paths()["include"]
    if cc is None or not os.path.exists(os.path.join(include, "Python.h")):
        print(f"no {compiler} or no Python.h: {calls} are called through ctypes", file=sys.stderr)
        return None
    r = subprocess.run([cc, "-O2", "-shared", "-fPIC", "-I", include, "-o", out, os.path.join(CSRC, source), *flags], capture_output=True, text=True)
    if r.returncode != 0:
        if needed:
            raise RuntimeError(f"{compiler} failed on {source}:\n" + r.stderr)
        print(f"{compiler} failed on {source} ({calls} are called through ctypes):\n" + r.stderr, file=sys.stderr)
        return None
    return out


def build_extension():
    """The decisions' calls without ctypes; without gcc or Python's headers there is none, and they go through ctypes."""
    for old in (OUT_PY, os.path.join(os.path.dirname(OUT_PY), "_decisions.so")):  # (the latter: without a tag)
        if os.path.exists(old):
            os.remove(old)
    return _compile_extension("decisions_py.c", OUT_PY, "block_boundary and select_parallel")


def build_kv8_extension():
    """The same for the 8-bit cache's operators, against torch's headers: its tensors are read without a call into Python.  It is of use with that
    torch alone, and names it."""
    return _compile_with_torch("kv8_py.cpp", OUT_KV8, "the 8-bit cache's operators")


def build_q8_extension():
    """... and for the 8-bit integer layers'."""
    return _compile_with_torch("q8_py.cpp", OUT_Q8, "the 8-bit integer layers' operators")


def _compile_with_torch(source, out, calls):
    if os.path.exists(out):
        os.remove(out)
    try:
        import torch
    except ImportError:
        print(f"no torch: {calls} are called through ctypes", file=sys.stderr)
        return None
    at = os.path.dirname(torch.__file__)
    flags = [f'-DTORCH_BUILT_WITH="{torch.__version__}"', "-std=c++17", "-I", os.path.join(at, "include"),
             f"-D_GLIBCXX_USE_CXX11_ABI={int(torch._C._GLIBCXX_USE_CXX11_ABI)}", "-L", os.path.join(at, "lib"), "-ltorch_python", "-ltorch_cpu", "-lc10"]
    return _compile_extension(source, out, calls, "g++", flags, needed=False)


if __name__ == "__main__":
    print(build(verbose=True))
