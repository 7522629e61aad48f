"""Build libekv.so (HIP, gfx950) in-tree with hipcc.

Every call compiles all sources; objects go to ``_build/`` and the shared
library next to this file.  Usage: ``python -m paper_2609_33536_amd.build``
(``--timeline``: the instrumented libekv_timeline.so for the per-launch time
budget of the decode kernel, next to libekv.so).
"""

import os
import shutil
import subprocess
import sys

HERE = os.path.dirname(os.path.abspath(__file__))
ROOT = os.path.dirname(HERE)
CSRC = os.path.join(HERE, "csrc")
INCLUDE = os.path.join(ROOT, "include")
BUILD = os.path.join(ROOT, "_build")
LIB = os.path.join(HERE, "libekv.so")
TIMELINE_LIB = os.path.join(HERE, "libekv_timeline.so")
SOURCES = ["api.hip", "api_serve.hip", "control.hip", "decode.hip", "extend.hip", "prefill.hip", "rope.hip", "shared.hip",
           "transition.hip", "validate.hip"]
ARCH = "gfx950"

FLAGS = [
    f"--offload-arch={ARCH}", "-O3", "-std=c++17", "-fPIC",
    # keep the compiler from forming packed fp32 VALU ops
    "-Xclang", "-target-feature", "-Xclang", "-packed-fp32-ops",
    # MFMA accumulators in ordinary VGPRs (no copies to and from AGPRs)
    "-mllvm", "-amdgpu-mfma-vgpr-form",
    "-Wall", "-Wno-unused-result", "-Wno-unused-command-line-argument",
    f"-I{INCLUDE}", f"-I{CSRC}",
]


def hipcc():
    path = shutil.which("hipcc") or "/opt/rocm/bin/hipcc"
    if not os.path.exists(path):
        raise RuntimeError("hipcc not found")
    return path


def build(verbose=False, extra_flags=(), timeline=False):
    """Compile every source and link LIB; with timeline=True the instrumented
    variant libekv_timeline.so instead (decode workgroups record timestamps,
    see EKV_TIMELINE in decode.hip; for measurement only)."""
    build_dir = os.path.join(BUILD, "timeline") if timeline else BUILD
    lib = TIMELINE_LIB if timeline else LIB
    extra_flags = tuple(extra_flags) + (("-DEKV_TIMELINE",) if timeline else ())
    os.makedirs(build_dir, exist_ok=True)
    cc = hipcc()
    procs = []
    objs = []
    for src in SOURCES:
        obj = os.path.join(build_dir, src.replace(".hip", ".o"))
        objs.append(obj)
        cmd = [cc, *FLAGS, *extra_flags, "-c", os.path.join(CSRC, src), "-o", obj]
        if verbose:
            print(" ".join(cmd), flush=True)
        procs.append((src, subprocess.Popen(cmd, stdout=subprocess.PIPE, stderr=subprocess.STDOUT)))
    failed = []
    for src, p in procs:
        out = p.communicate()[0].decode(errors="replace")
        out = "\n".join(l for l in out.splitlines() if "packed-fp32-ops" not in l)
        if p.returncode != 0:
            failed.append(src)
            print(out, file=sys.stderr)
        elif verbose and out.strip():
            print(out)
    if failed:
        raise RuntimeError(f"hipcc failed for {failed}")
    tmp = lib + ".tmp"
    cmd = [cc, f"--offload-arch={ARCH}", "-shared", "-fPIC", "-o", tmp, *objs]
    if verbose:
        print(" ".join(cmd), flush=True)
    subprocess.run(cmd, check=True)
    os.replace(tmp, lib)
    return lib


if __name__ == "__main__":
    print(build(verbose="-v" in sys.argv, timeline="--timeline" in sys.argv))
