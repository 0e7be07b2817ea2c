"""Builds libkvtc.so (HIP kernels + C ABI for gfx950) in-tree with hipcc."""
from __future__ import annotations

import os
import subprocess
import sys
from concurrent.futures import ThreadPoolExecutor

HERE = os.path.dirname(os.path.abspath(__file__))
CSRC = os.path.join(HERE, "csrc")
LIB = os.path.join(HERE, "libkvtc.so")
# (source, object, macros): the decode kernels' many widths and the attentions' types, formats and widths are compiled in parts, side by side
SOURCES = [(f"{s}.hip", f"{s}.o", []) for s in ("kvtc_api", "kvtc_encode", "kvtc_fp8", "kvtc_rope", "kvtc_probe", "kvtc_entropy", "kvtc_calib", "kvtc_cache", "kvtc_place", "kvtc_rope_scaled", "kvtc_join", "kvtc_many", "kvtc_test")]
SOURCES += [("kvtc_decode.hip", f"kvtc_decode_{k}.o", [f"-DKVTC_DECODE_PART={k}"]) for k in range(5)]
SOURCES += [("kvtc_attend.hip", f"kvtc_attend_{k}.o", [f"-DKVTC_ATTEND_PART={k}"]) for k in range(6)]
SOURCES += [("kvtc_many_mfma.hip", f"kvtc_many_mfma_{k}.o", [f"-DKVTC_MANY_PART={k}"]) for k in range(9)]
FLAGS = ["--offload-arch=gfx950", "-O3", "-std=c++17", "-fPIC",
         "-Xclang", "-target-feature", "-Xclang", "-packed-fp32-ops",
         "-Wno-unused-command-line-argument"]


def _hipcc() -> str:
    for c in (os.environ.get("HIPCC"), "/opt/rocm/bin/hipcc", "hipcc"):
        if c and (os.path.isabs(c) and os.path.exists(c) or not os.path.isabs(c)):
            return c
    return "hipcc"


def build(verbose: bool = False, extra_flags=()) -> str:
    """Compile every source and link the shared library; returns its path."""
    objdir = os.path.join(HERE, "_build")
    os.makedirs(objdir, exist_ok=True)
    hipcc = _hipcc()

    def compile_one(source) -> str:
        src, obj, macros = source
        obj = os.path.join(objdir, obj)
        cmd = [hipcc, *FLAGS, *macros, *extra_flags, "-c", os.path.join(CSRC, src), "-o", obj]
        res = subprocess.run(cmd, capture_output=True, text=True)
        err = "\n".join(l for l in res.stderr.splitlines() if "packed-fp32-ops" not in l)
        if res.returncode != 0:
            raise RuntimeError(f"hipcc failed on {src}:\n{err}")
        if verbose and err.strip():
            print(err, file=sys.stderr)
        return obj

    with ThreadPoolExecutor(max_workers=os.cpu_count() or 4) as ex:
        objs = list(ex.map(compile_one, SOURCES[::-1]))
    cmd = [hipcc, "--offload-arch=gfx950", "-shared", "-fPIC", "-o", LIB, *objs]
    res = subprocess.run(cmd, capture_output=True, text=True)
    if res.returncode != 0:
        raise RuntimeError(f"link failed:\n{res.stderr}")
    return LIB


if __name__ == "__main__":
    print(build(verbose=True))
