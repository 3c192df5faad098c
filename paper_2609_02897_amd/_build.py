"""Build libasv.so in-tree for gfx950 with hipcc (no GPU needed to compile)."""

from __future__ import annotations

import os
import subprocess

_HERE = os.path.dirname(os.path.abspath(__file__))
ROOT = os.path.dirname(_HERE)
SOURCES = [os.path.join(_HERE, "csrc", f) for f in ("asv_api.hip", "asv_logits.hip",
                                                                "asv_rules.hip")]
HEADERS = [os.path.join(ROOT, "include", "asv.h")] + [
    os.path.join(_HERE, "csrc", f) for f in ("asv_host.h", "asv_k1_host.h", "asv_q8_host.h", "k_common.h",
                                               "k_lmhead.h", "k_reduce.h", "k_accept.h",
                                               "k_draft.h", "k_tree.h", "k_rules.h", "k_fp8.h")]
OUT = os.path.join(_HERE, "libasv.so")
# measurement-only library (achievable-peak microbenchmarks), separate from libasv
MICROBENCH_SOURCES = [os.path.join(_HERE, "csrc", "microbench.hip")]
MICROBENCH_OUT = os.path.join(_HERE, "libasv_microbench.so")

HIPCC_FLAGS = [
    "--offload-arch=gfx950", "-O3", "-std=c++17", "-fPIC",
    # code objects every ROCm 7.x runtime loads (torch may bring an older runtime than hipcc)
    "-mcode-object-version=5",
    # keep the compiler from forming packed fp32 (v_pk_*_f32) instructions
    "-Xclang", "-target-feature", "-Xclang", "-packed-fp32-ops",
]


def hipcc() -> str:
    cand = os.path.join(os.environ.get("ROCM_PATH", "/opt/rocm"), "bin", "hipcc")
    return cand if os.path.exists(cand) else "hipcc"


def build_library(out: str = OUT, verbose: bool = False, sources=None) -> str:
    """Compile the HIP sources (libasv's by default) into ``out`` (written atomically)."""
    tmp = out + ".tmp"
    sources = sources or SOURCES
    objects = [f"{tmp}{i}.o" for i in range(len(sources))]
    flags = [*HIPCC_FLAGS, "-I", os.path.join(ROOT, "include")]
    msgs = ""

    def run(cmds):                  # side by side
        nonlocal msgs
        procs = [subprocess.Popen(c, stdout=subprocess.PIPE, stderr=subprocess.STDOUT, text=True)
                 for c in cmds]
        outs = [p.communicate()[0] for p in procs]
        for c, p, o in zip(cmds, procs, outs):
            o = "\n".join(l for l in o.splitlines() if "packed-fp32-ops" not in l)
            if p.returncode != 0:
                raise RuntimeError(f"hipcc failed ({p.returncode}):\n{' '.join(c)}\n{o}")
            msgs += o

    try:
        run([[hipcc(), *flags, "-c", src, "-o", obj] for src, obj in zip(sources, objects)])
        run([[hipcc(), "--offload-arch=gfx950", "-fPIC", "-shared", "-o", tmp, *objects]])
    finally:
        for obj in objects:
            if os.path.exists(obj):
                os.remove(obj)
    if verbose and msgs.strip():
        print(msgs)
    os.replace(tmp, out)
    return out


def build_microbench(verbose: bool = False) -> str:
    return build_library(MICROBENCH_OUT, verbose, MICROBENCH_SOURCES)


def is_built(out: str = OUT) -> bool:
    return os.path.exists(out)
