"""Builds libhclae.so (HIP, gfx950 only) in-tree next to this file."""
import os
import subprocess
import tempfile

HERE = os.path.dirname(os.path.abspath(__file__))
CSRC = os.path.join(HERE, "csrc")
LIB = os.path.join(HERE, "libhclae.so")
PROBE = os.path.join(HERE, "libhclae_probe.so")      # for the tests: single instructions of the contraction

HIPCC_FLAGS = [
    "-O3", "-std=c++17", "--offload-arch=gfx950", "-shared", "-fPIC",
    "-Xclang", "-target-feature", "-Xclang", "-packed-fp32-ops",
    "-Wall", "-Wno-unused-function",
]


def sources():
    return [os.path.join(CSRC, "hclae.hip"), os.path.join(CSRC, "serve.hip")]


def build(verbose=False, extra=()):
    hipcc = os.environ.get("HIPCC", "/opt/rocm/bin/hipcc")
    flags = HIPCC_FLAGS + list(extra)
    with tempfile.TemporaryDirectory() as tmp:               # every source at the same time, then the library from what they gave
        objects = [os.path.join(tmp, "%d.o" % i) for i in range(len(sources()))]
        each = [f for f in flags if f != "-shared"]
        jobs = [[hipcc] + each + ["-c", "-o", o, s] for o, s in zip(objects, sources())]
        jobs.append([hipcc] + flags + ["-o", PROBE, os.path.join(CSRC, "probe.hip")])
        running = []
        for c in jobs:
            if verbose:
                print(" ".join(c))
            running.append(subprocess.Popen(c))
        failed = [c for c, p in zip(jobs, running) if p.wait() != 0]
        if failed:
            raise subprocess.CalledProcessError(1, failed[0])
        link = [hipcc] + flags + ["-o", LIB] + objects
        if verbose:
            print(" ".join(link))
        subprocess.run(link, check=True)
    return LIB


if __name__ == "__main__":
    build(verbose=True)
    print(LIB)
