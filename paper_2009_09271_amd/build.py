"""Build libefsparse.so (HIP, gfx950) in-tree with hipcc.

    python paper_2009_09271_amd/build.py      # by path: importing the package needs a built library
"""

import os
import shutil
import subprocess
import sys
import tempfile

HERE = os.path.dirname(os.path.abspath(__file__))
SRCS = [os.path.join(HERE, "csrc", f) for f in ("efsparse.hip", "linear.hip")]
OUT = os.path.join(HERE, "libefsparse.so")

FLAGS = [
    "--offload-arch=gfx950",
    "-O3",
    "-std=c++17",
    "-fPIC",
    "-ffp-contract=off",            # no fused multiply-add contraction: IEEE add / divide only
    "-Wall",
    "-Xclang", "-target-feature", "-Xclang", "-packed-fp32-ops",
]


def hipcc():
    for c in (os.environ.get("HIPCC"), "/opt/rocm/bin/hipcc", shutil.which("hipcc")):
        if c and os.path.exists(c):
            return c
    raise RuntimeError("hipcc not found")


def build(verbose: bool = False) -> str:
    tmp = OUT + ".tmp"
    with tempfile.TemporaryDirectory() as d:
        jobs = []
        for src in SRCS:  # side by side
            cmd = [hipcc()] + FLAGS + ["-c", src, "-o", os.path.join(d, os.path.basename(src) + ".o")]
            if verbose:
                print(" ".join(cmd), flush=True)
            jobs.append((cmd, subprocess.Popen(cmd)))
        failed = [cmd for cmd, p in jobs if p.wait()]
        if failed:
            raise subprocess.CalledProcessError(1, failed[0])
        cmd = [hipcc(), "--offload-arch=gfx950", "-shared", "-fPIC"] + [cmd[-1] for cmd, _ in jobs] + ["-o", tmp]
        if verbose:
            print(" ".join(cmd), flush=True)
        subprocess.check_call(cmd)
    os.replace(tmp, OUT)
    return OUT


if __name__ == "__main__":
    print(build(verbose="-q" not in sys.argv))
