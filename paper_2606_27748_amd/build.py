"""Build the gfx950 shared library ``libflexattn.so`` in-tree with hipcc."""
from __future__ import annotations

import concurrent.futures as cf
import os
import subprocess
import sys

HERE = os.path.dirname(os.path.abspath(__file__))
ROOT = os.path.dirname(HERE)
CSRC = os.path.join(HERE, "csrc")
BUILD = os.path.join(HERE, "_build")
LIB = os.path.join(HERE, "libflexattn.so")
SOURCES = ["flex_api.hip", "flex_fwd.hip", "flex_bwd.hip", "flex_bwd_dq.hip", "flex_decode.hip", "flex_awd.hip",
           "flex_seq_api.hip", "flex_attn_fwd.hip", "flex_attn_bwd.hip", "flex_delta_fwd.hip", "flex_delta_bwd.hip",
           "flex_layer_api.hip", "flex_conv.hip", "flex_norm.hip", "flex_scan_fwd.hip", "flex_scan_bwd.hip"]
HIPCC = os.environ.get("HIPCC", "/opt/rocm/bin/hipcc")
FLAGS = [
    "--offload-arch=gfx950", "-O3", "-std=c++17", "-fPIC",
    # never emit packed fp32 arithmetic (v_pk_fma/mul/add_f32)
    "-Xclang", "-target-feature", "-Xclang", "-packed-fp32-ops",
    "-I", os.path.join(ROOT, "include"),
]
# Per-source additions: the dQ sweep places MFMA results in VGPRs (its results
# mostly feed vector code; fewer accumulator-register copies).  Measured slower
# for the other kernels.
_VGPR_FORM = ["-mllvm", "-amdgpu-mfma-vgpr-form"]
FILE_FLAGS = {"flex_bwd_dq.hip": _VGPR_FORM, "flex_delta_fwd.hip": _VGPR_FORM, "flex_delta_bwd.hip": _VGPR_FORM}


def _run(cmd):
    r = subprocess.run(cmd, capture_output=True, text=True)
    err = "\n".join(l for l in r.stderr.splitlines() if "packed-fp32-ops" not in l)
    if r.returncode != 0:
        raise RuntimeError("command failed: %s\n%s" % (" ".join(cmd), err))
    return err


def build(verbose: bool = False) -> str:
    os.makedirs(BUILD, exist_ok=True)
    objs = []
    cmds = []
    for s in SOURCES:
        o = os.path.join(BUILD, s.replace(".hip", ".o"))
        objs.append(o)
        cmds.append([HIPCC] + FLAGS + FILE_FLAGS.get(s, []) + ["-c", os.path.join(CSRC, s), "-o", o])
    with cf.ThreadPoolExecutor(max_workers=min(len(cmds), 4)) as ex:
        for err in ex.map(_run, cmds):
            if verbose and err.strip():
                print(err, file=sys.stderr)
    tmp = LIB + ".tmp"
    _run([HIPCC, "--offload-arch=gfx950", "-shared", "-fPIC", "-o", tmp] + objs)
    os.replace(tmp, LIB)
    return LIB


if __name__ == "__main__":
    print(build(verbose=True))
