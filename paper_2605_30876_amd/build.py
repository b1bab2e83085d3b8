"""Build libdmoe.so in-tree with hipcc for gfx950.

    python -m paper_2605_30876_amd.build [--jobs N] [--debug]

Every HIP source is compiled with packed-fp32 instructions disabled
(``-Xclang -target-feature -Xclang -packed-fp32-ops``); the host pass prints
that it does not know the feature, which is harmless.
"""
from __future__ import annotations

import argparse
import concurrent.futures as cf
import os
import shutil
import subprocess
import sys

PKG = os.path.dirname(os.path.abspath(__file__))
ROOT = os.path.dirname(PKG)
CSRC = os.path.join(PKG, "csrc")
INCLUDE = os.path.join(ROOT, "include")
LIB = os.path.join(PKG, "libdmoe.so")
SOURCES = ["dmoe_api.cpp", "router.hip", "routing.hip", "topp.hip", "schedule.hip", "route.hip", "pack.hip",
           "ffn.hip", "ffn_f32.hip", "combine.hip", "noalloc.hip", "layer.hip", "attn/attn_api.cpp", "attn/rope.hip",
           "attn/append_quant.hip", "attn/pages.hip", "attn/plan.hip", "attn/attention_bf16.hip", "attn/attention_f32.hip",
           "attn/attention_bf16_fp8.hip", "attn/attention_bf16_fp4.hip", "attn/attention_bf16_fp8_fp4.hip",
           "attn/attention_f32_fp8.hip", "attn/attention_f32_fp4.hip", "attn/attention_f32_fp8_fp4.hip"]
ARCH = os.environ.get("DMOE_OFFLOAD_ARCH", "gfx950")


def kernel_source_hash() -> str:
    """Hash of the code of every kernel source of the MoE layer (line comments
    and blank lines left out): hardware-counter figures taken on other code
    are stale."""
    import hashlib
    import re

    h = hashlib.sha256()
    for f in sorted(os.listdir(CSRC)):
        if not f.endswith((".hip", ".h")):
            continue
        with open(os.path.join(CSRC, f), encoding="utf-8") as fh:
            for line in fh:
                code = re.sub(r"//.*", "", line).rstrip()
                if code:
                    h.update(code.encode() + b"\n")
    return h.hexdigest()[:16]


def hipcc() -> str:
    for cand in (os.environ.get("HIPCC"), "/opt/rocm/bin/hipcc", shutil.which("hipcc")):
        if cand and os.path.exists(cand):
            return cand
    raise RuntimeError("hipcc not found (set HIPCC or install ROCm)")


def _flags(debug: bool):
    opt = ["-O1", "-g"] if debug else ["-O3"]
    return opt + ["-std=c++17", "-fPIC", f"--offload-arch={ARCH}", "-I", INCLUDE, "-I", CSRC,
                  "-Xclang", "-target-feature", "-Xclang", "-packed-fp32-ops",
                  "-Wall", "-Wno-unused-function"]


def build(jobs: int = 0, debug: bool = False, verbose: bool = False) -> str:
    cc = hipcc()
    objdir = os.path.join(ROOT, "_build", "obj")
    os.makedirs(objdir, exist_ok=True)
    flags = _flags(debug)

    def compile_one(src):
        obj = os.path.join(objdir, os.path.splitext(src)[0].replace("/", "_") + ".o")
        cmd = [cc, "-x", "hip", "-c", os.path.join(CSRC, src), "-o", obj] + flags
        r = subprocess.run(cmd, capture_output=True, text=True)
        out = "\n".join(l for l in (r.stdout + r.stderr).splitlines()
                        if "packed-fp32-ops' is not a recognized feature" not in l)
        if r.returncode != 0:
            raise RuntimeError(f"hipcc failed on {src}:\n{' '.join(cmd)}\n{out}")
        if verbose and out.strip():
            print(out)
        return obj

    n = jobs or min(len(SOURCES), os.cpu_count() or 1)
    with cf.ThreadPoolExecutor(max_workers=n) as ex:
        objs = list(ex.map(compile_one, SOURCES))
    tmp = LIB + ".tmp"
    cmd = [cc, "-shared", "-fPIC", f"--offload-arch={ARCH}", "-o", tmp] + objs
    r = subprocess.run(cmd, capture_output=True, text=True)
    if r.returncode != 0:
        raise RuntimeError(f"link failed:\n{' '.join(cmd)}\n{r.stdout}{r.stderr}")
    os.replace(tmp, LIB)
    return LIB


def main(argv=None):
    ap = argparse.ArgumentParser(description=__doc__)
    ap.add_argument("--jobs", type=int, default=0)
    ap.add_argument("--debug", action="store_true")
    ap.add_argument("-v", "--verbose", action="store_true")
    a = ap.parse_args(argv)
    print(build(a.jobs, a.debug, a.verbose))


if __name__ == "__main__":
    sys.exit(main())
