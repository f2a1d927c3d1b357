"""Build libasl.so (HIP, gfx950) in-tree with hipcc.  `python -m paper_2601_07667_amd.build`."""
from __future__ import annotations

import os
import subprocess
import sys
from concurrent.futures import ThreadPoolExecutor

PKG = os.path.dirname(os.path.abspath(__file__))
ROOT = os.path.dirname(PKG)
CSRC = os.path.join(PKG, "csrc")
LIB = os.path.join(PKG, "libasl.so")
SOURCES = ["api.hip", "score.hip", "pool.hip", "rank.hip", "rankvar.hip", "select.hip", "gather.hip", "tail.hip",
           "paged_api.hip", "paged.hip", "attend.hip", "attend_64.hip", "attend_128.hip", "attend_tree.hip", "attend_tree_64.hip",
           "attend_tree_128.hip", "rotate.hip", "draft.hip"]
# packed-fp32 instructions are switched off for all device code
FLAGS = ["--offload-arch=gfx950", "-O3", "-std=c++17", "-fPIC", "-fvisibility=hidden",
         "-Xclang", "-target-feature", "-Xclang", "-packed-fp32-ops",
         "-I", os.path.join(ROOT, "include"), "-I", CSRC, "-Wall", "-Wno-unused-function"]


# score.hip never produces NaNs from finite inputs (masked logits are -inf, never inf - inf); telling
# the compiler so lets max() compile to bare v_max_f32 / v_max3_f32 without NaN-quieting moves.
# The attention kernels take NaN as they come, so without the first of the two.
# MFMA results are kept in ordinary VGPRs: the softmax arithmetic reads every accumulator, and
# copies out of accumulation registers would cost one vector instruction per element.
PER_FILE_FLAGS = {"score.hip": ["-fno-honor-nans", "-mllvm", "-amdgpu-mfma-vgpr-form"],
                  **{f: ["-mllvm", "-amdgpu-mfma-vgpr-form"] for f in ("attend.hip", "attend_64.hip", "attend_128.hip", "attend_tree.hip",
                                                                       "attend_tree_64.hip", "attend_tree_128.hip")}}


def _hipcc() -> str:
    for c in (os.environ.get("HIPCC"), "/opt/rocm/bin/hipcc", "hipcc"):
        if c and (os.path.isabs(c) and os.path.exists(c) or not os.path.isabs(c)):
            return c
    raise RuntimeError("hipcc not found")


def build_lib(verbose: bool = True, extra_flags=()) -> str:
    obj_dir = os.path.join(PKG, "_build")
    os.makedirs(obj_dir, exist_ok=True)
    cc = _hipcc()

    def compile_one(src: str) -> str:
        obj = os.path.join(obj_dir, src.replace(".hip", ".o"))
        cmd = [cc, *FLAGS, *PER_FILE_FLAGS.get(src, []), *extra_flags, "-c", os.path.join(CSRC, src), "-o", obj]
        r = subprocess.run(cmd, capture_output=True, text=True)
        msgs = "\n".join(l for l in (r.stdout + r.stderr).splitlines()
                         if "packed-fp32-ops' is not a recognized feature" not in l)
        if r.returncode != 0:
            raise RuntimeError(f"hipcc failed on {src}:\n{msgs}")
        if verbose and msgs.strip():
            print(msgs, file=sys.stderr)
        return obj

    with ThreadPoolExecutor(max_workers=min(8, len(SOURCES))) as ex:
        objs = list(ex.map(compile_one, SOURCES))
    cmd = [cc, "--offload-arch=gfx950", "-shared", "-fPIC", "-o", LIB, *objs]
    r = subprocess.run(cmd, capture_output=True, text=True)
    if r.returncode != 0:
        raise RuntimeError("link failed:\n" + r.stdout + r.stderr)
    if verbose:
        print(f"built {LIB}")
    return LIB


if __name__ == "__main__":
    build_lib()
