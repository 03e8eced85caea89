"""Builds libshe_hip.so (HIP kernels + C ABI) for gfx950 next to this file."""
from __future__ import annotations

import os
import subprocess
import tempfile
from concurrent.futures import ThreadPoolExecutor

_HERE = os.path.dirname(os.path.abspath(__file__))
CSRC = os.path.join(_HERE, "csrc")
LIB_PATH = os.path.join(_HERE, "libshe_hip.so")
# those that take longest first
SOURCES = ["clear_sample.hip", "clear_attend.hip", "she_kernels.hip", "clear_adapters.hip", "clear_qk.hip", "clear_plan.hip", "she_api.cpp", "she_host.cpp",
           "she_circuits.cpp", "she_leveled.cpp", "she_clear.cpp", "she_clear_step.cpp", "clear_attend_shape.cpp"]
HIPCC = os.environ.get("HIPCC", "/opt/rocm/bin/hipcc")

FLAGS = [
    "--offload-arch=gfx950", "-O3", "-std=c++17", "-fPIC", "-shared", "-ffp-contract=off", "-pthread",
    # keep hipcc from forming packed FP32 instructions
    "-Xclang", "-target-feature", "-Xclang", "-packed-fp32-ops",
    "-Wall", "-Wno-unused-result", "-Wno-unused-value",
]


def build(verbose: bool = False, extra: list[str] | None = None, out: str | None = None) -> str:
    """Compiles every source each time it is called, several at a time, and links them, all with the flags `extra` too; returns the path of
    the shared library."""
    out = out or LIB_PATH
    stderr = None if verbose else subprocess.DEVNULL
    link = FLAGS + (extra or [])
    flags = [f for f in link if f != "-shared"]

    def run(cmd):
        if verbose:
            print(" ".join(cmd), flush=True)
        subprocess.check_call(cmd, stderr=stderr)

    with tempfile.TemporaryDirectory() as tmp, ThreadPoolExecutor(min(8, os.cpu_count() or 1)) as pool:
        objects = [os.path.join(tmp, s + ".o") for s in SOURCES]
        for done in [pool.submit(run, [HIPCC] + flags + ["-c", os.path.join(CSRC, s), "-o", o]) for s, o in zip(SOURCES, objects)]:
            done.result()
        run([HIPCC] + link + objects + ["-o", out + ".tmp"])
    os.replace(out + ".tmp", out)
    return out


if __name__ == "__main__":
    print(build(verbose=True))
