"""Compile the HIP library for gfx950 in-tree (hipcc cross-compiles without a GPU)."""
from __future__ import annotations

import os
import subprocess
import tempfile

HERE = os.path.dirname(os.path.abspath(__file__))
ROOT = os.path.dirname(HERE)
CSRC = os.path.join(HERE, "csrc")
LIB = os.path.join(HERE, "libshareprefill.so")

HIPCC_FLAGS = [
    "--offload-arch=gfx950", "-O3", "-std=c++17", "-fPIC",
    # packed fp32 instructions are kept out of the generated code on purpose
    "-Xclang", "-target-feature", "-Xclang", "-packed-fp32-ops",
    "-I" + os.path.join(ROOT, "include"), "-I" + CSRC,
]
# the translation units and what each is compiled with besides
SOURCES = {
    # the prefill's device code never relies on NaN semantics (the score quantiser tests bits); lets fmax chains
    # compile to v_max3 without a canonicalising v_max per operand
    "shareprefill.hip": ["-Xarch_device", "-fno-honor-nans"],
    # the cache's device code does: a value that is not finite stays with the rows that see it
    "cache.hip": [],
}


def build_library(verbose: bool = False) -> str:
    hipcc = os.environ.get("HIPCC", "/opt/rocm/bin/hipcc")
    with tempfile.TemporaryDirectory() as tmp:
        objects = [os.path.join(tmp, name + ".o") for name in SOURCES]
        jobs = []
        for (name, more), obj in zip(SOURCES.items(), objects):
            cmd = [hipcc] + HIPCC_FLAGS + more + ["-c", os.path.join(CSRC, name), "-o", obj]
            jobs.append(subprocess.Popen(cmd, stdout=subprocess.PIPE, stderr=subprocess.STDOUT, text=True))
        out = [job.communicate()[0] for job in jobs]
        for job, text in zip(jobs, out):
            if job.returncode != 0:
                raise RuntimeError("hipcc failed:\n" + text)
        res = subprocess.run([hipcc, "--offload-arch=gfx950", "-fPIC", "-shared"] + objects + ["-o", LIB],
                             stdout=subprocess.PIPE, stderr=subprocess.STDOUT, text=True)
    if res.returncode != 0:
        raise RuntimeError("hipcc failed:\n" + res.stdout)
    if verbose:
        print("".join(out) + res.stdout)
    return LIB


def library_path(build_if_missing: bool = True) -> str:
    override = os.environ.get("SHAREPREFILL_LIB")      # an explicitly chosen build of the same library
    if override:
        if not os.path.exists(override):
            raise FileNotFoundError(override)
        return override
    if not os.path.exists(LIB):
        if not build_if_missing:
            raise FileNotFoundError(LIB)
        build_library()
    return LIB


if __name__ == "__main__":
    print(build_library(verbose=True))
