"""Builds the HIP library librheo.so in place (gfx950).

All device code is compiled with -ffp-contract=off (the canonical weights
and the fp64 proxies are defined operation by operation) and without packed
fp32 instructions.
"""

import os
import subprocess
import sys
from concurrent.futures import ThreadPoolExecutor

HERE = os.path.dirname(os.path.abspath(__file__))
ROOT = os.path.dirname(HERE)
CSRC = os.path.join(HERE, "csrc")
LIB = os.path.join(HERE, "librheo.so")
PROBE_LIB = os.path.join(HERE, "libstreamprobe.so")
SOURCES = ["api.hip", "expand.hip", "dense.hip", "prune.hip", "verify.hip", "views.hip",
           "cache_api.hip", "cache_plan.hip", "cache_write.hip", "attention.hip",
           "cache_commit.hip", "logprobs.hip"]
HIPCC = os.environ.get("HIPCC", "/opt/rocm/bin/hipcc")


FLAGS = ["-O3", "--offload-arch=gfx950", "-std=c++17", "-fPIC",
         "-ffp-contract=off", "-fno-fast-math",
         "-Xclang", "-target-feature", "-Xclang", "-packed-fp32-ops",
         "-I", os.path.join(ROOT, "include"), "-I", CSRC]
# The default scheduler leaves every LDS read of the attention loop next to the
# product that takes it; this one keeps the order that the loop asks for
# (64 trees over 4096 tokens: 242 us against 252; one token over 517: 15.4, 17.3).
SOURCE_FLAGS = {"attention.hip": ["-mllvm", "-amdgpu-sched-strategy=iterative-ilp"]}


def _run(cmd, verbose):
    if verbose:
        print(" ".join(cmd), flush=True)
    res = subprocess.run(cmd, capture_output=True, text=True)
    msgs = [l for l in (res.stdout + res.stderr).splitlines()
            if "packed-fp32-ops" not in l]
    if res.returncode != 0:
        raise RuntimeError("hipcc failed:\n" + "\n".join(msgs))
    if verbose and msgs:
        print("\n".join(msgs), flush=True)


def _compile(out, sources, verbose, jobs=None):
    """One object per source, `jobs` compilers at a time, then the library."""
    objs = [os.path.join(HERE, "build", os.path.basename(out) + "." + s + ".o") for s in sources]
    os.makedirs(os.path.join(HERE, "build"), exist_ok=True)

    def one(source, obj):
        _run([HIPCC] + FLAGS + SOURCE_FLAGS.get(source, []) +
             ["-c", os.path.join(CSRC, source), "-o", obj], verbose)

    with ThreadPoolExecutor(jobs or min(4, os.cpu_count() or 1)) as pool:
        list(pool.map(one, sources, objs))
    _run([HIPCC, "--offload-arch=gfx950", "-shared", "-fPIC", "-o", out + ".tmp"] + objs, verbose)
    os.replace(out + ".tmp", out)
    return out


def build(verbose=False, jobs=None):
    """librheo.so, and the streaming-read probe bench.py measures beside it."""
    _compile(PROBE_LIB, ["stream_probe.hip"], verbose, jobs)
    return _compile(LIB, SOURCES, verbose, jobs)


if __name__ == "__main__":
    print(build(verbose="-v" in sys.argv))
