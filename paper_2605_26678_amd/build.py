"""Builds libnkv.so (HIP, gfx950) in-tree with hipcc.  Run as ``python -m paper_2605_26678_amd.build``."""
from __future__ import annotations

import os
import subprocess
import sys
from concurrent.futures import ThreadPoolExecutor

HERE = os.path.dirname(os.path.abspath(__file__))
ROOT = os.path.dirname(HERE)
CSRC = os.path.join(HERE, "csrc")
OBJ = os.path.join(HERE, "_build")
LIB = os.path.join(HERE, "libnkv.so")

SOURCES = ["nkv_api.hip", "nkv_score_generic.hip", "nkv_score_fast.hip", "nkv_score_tile.hip", "nkv_finalize.hip", "nkv_finalize_wide.hip", "nkv_budget.hip",
           "nkv_budget_wide.hip", "nkv_budget_heads.hip", "nkv_select.hip", "nkv_select_wide.hip", "nkv_decode.hip",
           "nkv_pages.hip", "nkv_pages_attention.hip", "nkv_pages_prompt.hip", "nkv_pages_prompt_tokens.hip", "nkv_pages_prompt_64.hip", "nkv_pages_prompt_96.hip",
           "nkv_pages_prompt_128.hip", "nkv_pages_prompt_192.hip", "nkv_pages_prompt_256.hip", "nkv_beam.hip"]

# -packed-fp32-ops is switched off on purpose: packed fp32 instructions are not to be generated.
FLAGS = ["--offload-arch=gfx950", "-O3", "-std=c++17", "-fPIC", "-Wall", "-Wno-unused-function",
         "-Xclang", "-target-feature", "-Xclang", "-packed-fp32-ops",
         "-I", os.path.join(ROOT, "include"), "-I", CSRC]


def _hipcc() -> str:
    for c in (os.environ.get("HIPCC"), "/opt/rocm/bin/hipcc", "hipcc"):
        if c and (os.path.isabs(c) and os.path.exists(c) or not os.path.isabs(c)):
            return c
    raise RuntimeError("hipcc not found")


def library_path() -> str:
    return LIB


def is_built() -> bool:
    return os.path.exists(LIB)


def build(verbose: bool = True) -> str:
    """Compile every HIP source for gfx950 and link libnkv.so.  Always compiles."""
    os.makedirs(OBJ, exist_ok=True)
    hipcc = _hipcc()

    def compile_one(src: str) -> str:
        obj = os.path.join(OBJ, src.replace(".hip", ".o"))
        cmd = [hipcc, *FLAGS, "-c", os.path.join(CSRC, src), "-o", obj]
        r = subprocess.run(cmd, capture_output=True, text=True)
        out = "\n".join(l for l in (r.stdout + r.stderr).splitlines()
                        if "packed-fp32-ops" not in l and "is not a recognized feature" not in l)
        if r.returncode != 0:
            raise RuntimeError(f"hipcc failed on {src}:\n{out}")
        if verbose and out.strip():
            print(out, file=sys.stderr)
        return obj

    with ThreadPoolExecutor(max_workers=min(8, len(SOURCES))) as ex:
        objs = list(ex.map(compile_one, SOURCES))
    tmp = LIB + f".tmp{os.getpid()}"
    r = subprocess.run([hipcc, "--offload-arch=gfx950", "-shared", "-fPIC", "-o", tmp, *objs],
                       capture_output=True, text=True)
    if r.returncode != 0:
        raise RuntimeError("link failed:\n" + r.stdout + r.stderr)
    os.replace(tmp, LIB)
    return LIB


if __name__ == "__main__":
    print(build())
