"""Build the HIP library in-tree: paper_2604_05417_amd/libmetasd.so (gfx950 only)."""
from __future__ import annotations

import os
import subprocess

HERE = os.path.dirname(os.path.abspath(__file__))
CSRC = os.path.join(HERE, "csrc")
SRCS = [os.path.join(CSRC, n) for n in ("metasd.hip", "pages.hip")]
DEPS = SRCS + [os.path.join(CSRC, n) for n in ("common.h", "kernels.h", "batch.h", "prefill.h", "gemm_tiles.h", "step.h", "attn.h", "attn_plan.h",
                                               "step_f32.h", "chain_f32.h", "chain_plan.h", "pages.h", "pages_attn.h", "pages_plan.h", "pages_host.h",
                                               "accept_probs.h")] + [os.path.join(HERE, "..", "include", "metasd.h")]
LIB = os.path.join(HERE, "libmetasd.so")

HIPCC_FLAGS = ["-O3", "-std=c++17", "--offload-arch=gfx950", "-fPIC",
               "-Xclang", "-target-feature", "-Xclang", "-packed-fp32-ops",   # no packed-fp32 code generation
               "-Wall", "-Wno-unused-function", "-Wno-inline-asm"]   # the direct-load asm declares that it writes m0


def build(force: bool = True, verbose: bool = False) -> str:
    """Compile with hipcc (cross-compiles without a GPU).  force=False skips an up-to-date library."""
    if not force and os.path.exists(LIB) and all(os.path.getmtime(LIB) >= os.path.getmtime(d) for d in DEPS):
        return LIB
    hipcc = os.environ.get("HIPCC", "/opt/rocm/bin/hipcc")
    # one compiler per source, side by side
    objs = [os.path.join(HERE, os.path.basename(src) + ".o") for src in SRCS]
    runs = [(subprocess.Popen([hipcc] + HIPCC_FLAGS + ["-c", "-o", obj, src], stdout=subprocess.DEVNULL, stderr=subprocess.PIPE, text=True))
            for src, obj in zip(SRCS, objs)]
    noise = "is not a recognized feature for this target"
    errs = ["\n".join(ln for ln in r.communicate()[1].splitlines() if noise not in ln) for r in runs]
    err = "\n".join(e for e in errs if e.strip())
    if any(r.returncode != 0 for r in runs):
        raise RuntimeError("hipcc failed:\n" + err)
    res = subprocess.run([hipcc, "--offload-arch=gfx950", "-shared", "-fPIC", "-o", LIB] + objs, capture_output=True, text=True)
    for obj in objs:
        os.remove(obj)
    if res.returncode != 0:
        raise RuntimeError("hipcc failed:\n" + res.stderr)
    if verbose and err.strip():
        print(err)
    return LIB


if __name__ == "__main__":
    print(build(verbose=True))
