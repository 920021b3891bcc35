"""Build libscheinfer.so (HIP for gfx950 + the host worker) in-tree with hipcc / g++."""
from __future__ import annotations

import os
import subprocess
import sys

HERE = os.path.dirname(os.path.abspath(__file__))
ROOT = os.path.dirname(HERE)
CSRC = os.path.join(HERE, "csrc")
OBJ = os.path.join(HERE, "_build")
LIB = os.path.join(HERE, "libscheinfer.so")
HIPCC = os.environ.get("HIPCC", "/opt/rocm/bin/hipcc")

HIP_SOURCES = ["route.hip", "route_static.hip", "decode.hip", "prefill.hip", "layer.hip", "profiler.hip", "q4.hip", "peaks.hip",
               "norm.hip", "append.hip", "attend.hip", "attend_bf16.hip", "attend_e4m3.hip", "pages.hip"]
CPP_SOURCES = ["cc_worker.cpp", "solver.cpp"]
HIP_FLAGS = ["-O3", "-std=c++17", "-fPIC", "--offload-arch=gfx950", "-Xclang", "-target-feature", "-Xclang",
             "-packed-fp32-ops", "-Wno-unused-command-line-argument", "-I", os.path.join(ROOT, "include"), "-I", CSRC]
CPP_FLAGS = ["-O3", "-std=c++17", "-fPIC", "-mavx2", "-mfma", "-pthread", "-I", os.path.join(ROOT, "include"), "-I", CSRC]


def _run(cmd):
    r = subprocess.run(cmd, capture_output=True, text=True)
    if r.returncode != 0:
        sys.stderr.write(" ".join(cmd) + "\n" + r.stdout + r.stderr)
        raise RuntimeError("build step failed: " + os.path.basename(cmd[-1]))
    # the host pass of hipcc warns that it does not know the packed-fp32 feature: harmless
    noise = "is not a recognized feature for this target"
    out = "\n".join(l for l in (r.stdout + r.stderr).splitlines() if noise not in l).strip()
    if out:
        sys.stderr.write(out + "\n")


def build(force: bool = True, jobs: int = 4) -> str:
    """Compile every source and link the shared library.  ``force=False`` skips up-to-date objects."""
    from concurrent.futures import ThreadPoolExecutor
    os.makedirs(OBJ, exist_ok=True)
    headers = [os.path.join(CSRC, f) for f in os.listdir(CSRC) if f.endswith(".h")] + [os.path.join(ROOT, "include", f) for f in os.listdir(os.path.join(ROOT, "include")) if f.endswith(".h")]
    newest_h = max(os.path.getmtime(h) for h in headers)
    tasks = []
    objs = []
    for src in HIP_SOURCES + CPP_SOURCES:
        s = os.path.join(CSRC, src)
        o = os.path.join(OBJ, src + ".o")
        objs.append(o)
        if not force and os.path.exists(o) and os.path.getmtime(o) >= max(os.path.getmtime(s), newest_h):
            continue
        if src.endswith(".hip"):
            tasks.append([HIPCC] + HIP_FLAGS + ["-c", s, "-o", o])
        else:
            tasks.append(["g++"] + CPP_FLAGS + ["-c", s, "-o", o])
    with ThreadPoolExecutor(max_workers=jobs) as ex:
        list(ex.map(_run, tasks))
    tmp = LIB + ".tmp.%d" % os.getpid()
    _run([HIPCC, "-shared", "-fPIC", "--offload-arch=gfx950", "-o", tmp] + objs + ["-pthread"])
    os.replace(tmp, LIB)
    return LIB


if __name__ == "__main__":
    print(build(force="--incremental" not in sys.argv))
