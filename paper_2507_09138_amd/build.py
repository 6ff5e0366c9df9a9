"""Builds libhr_ivf.so (HIP, gfx950 only) in-tree with hipcc.

    python -m paper_2507_09138_amd.build [--force]

The sources are compiled one hipcc process per file (in parallel) into ``_build/`` and
linked into ``libhr_ivf.so`` next to this file.  hipcc cross-compiles without a GPU.
"""
import os
import subprocess
import sys
from concurrent.futures import ThreadPoolExecutor

HERE = os.path.dirname(os.path.abspath(__file__))
ROOT = os.path.dirname(HERE)
CSRC = os.path.join(HERE, "csrc")
OBJ = os.path.join(HERE, "_build")
LIB = os.path.join(HERE, "libhr_ivf.so")
SOURCES = ["api.hip", "aux_kernels.hip", "scan_f16.hip", "scan_bf16.hip", "scan_f32.hip", "scan_f32x2.hip",
           "i8.hip", "rows.hip", "norm.hip", "gated.hip",
           "gated_f16.hip", "gated_bf16.hip", "gated_f32.hip", "adamw.hip"]
HEADERS = [os.path.join(CSRC, h) for h in ("common.h", "wave.h", "group.h", "scan_kernel.h", "entry.h", "row_math.h", "i8_few.h", "tile.h", "tile_launch.h", "tile_plan.h")] + \
          [os.path.join(ROOT, "include", h) for h in ("hr_ivf.h", "hr_scores.h", "hr_layers.h")]
FLAGS = ["--offload-arch=gfx950", "-O3", "-std=c++17", "-fPIC", "-Wall", "-Wno-unused-function",
         "-Xclang", "-target-feature", "-Xclang", "-packed-fp32-ops",
         "-I", os.path.join(ROOT, "include"), "-I", CSRC] + os.environ.get("HR_EXTRA_HIPCC_FLAGS", "").split()


def _stale(target, deps):
    if not os.path.exists(target):
        return True
    t = os.path.getmtime(target)
    return any(os.path.getmtime(d) > t for d in deps)


def _compile(src, force):
    obj = os.path.join(OBJ, src.replace(".hip", ".o"))
    path = os.path.join(CSRC, src)
    if force or _stale(obj, [path] + HEADERS):
        cmd = ["hipcc"] + FLAGS + ["-c", path, "-o", obj]
        r = subprocess.run(cmd, capture_output=True, text=True)
        if r.returncode != 0:
            raise RuntimeError(f"hipcc failed on {src}:\n{r.stdout}\n{r.stderr}")
        msgs = [ln for ln in r.stderr.splitlines() if "packed-fp32-ops" not in ln and ln.strip()]
        if any("warning" in m or "error" in m for m in msgs):
            sys.stderr.write("\n".join(msgs) + "\n")
    return obj


def build(force=False, jobs=8):
    os.makedirs(OBJ, exist_ok=True)
    with ThreadPoolExecutor(max_workers=jobs) as ex:
        objs = list(ex.map(lambda s: _compile(s, force), SOURCES))
    if force or _stale(LIB, objs):
        cmd = ["hipcc", "--offload-arch=gfx950", "-shared", "-fPIC", "-o", LIB] + objs
        r = subprocess.run(cmd, capture_output=True, text=True)
        if r.returncode != 0:
            raise RuntimeError(f"link failed:\n{r.stdout}\n{r.stderr}")
    return LIB


if __name__ == "__main__":
    print(build(force="--force" in sys.argv))
