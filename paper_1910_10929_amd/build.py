"""Build libdgs.so (gfx950) in-tree with hipcc."""
from __future__ import annotations

import os
import subprocess
import tempfile

HERE = os.path.dirname(os.path.abspath(__file__))
CSRC = os.path.join(HERE, "csrc")
LIB = os.path.join(HERE, "libdgs.so")
SOURCES = ["dgs_stream.hip", "dgs_select.hip", "dgs_chain.hip", "dgs_server.hip", "dgs_api.hip",
           "dgs_edge.hip", "dgs_checkpoint.hip", "dgs_weight_grad.hip", "dgs_head.hip",
           "dgs_orthogonal.hip"]

HIPCC_FLAGS = [
    "--offload-arch=gfx950", "-O3", "-std=c++17", "-fPIC",
    "-ffp-contract=off", "-fno-gpu-flush-denormals-to-zero",
    # packed-fp32 instruction forms are kept out of the generated code
    "-Xclang", "-target-feature", "-Xclang", "-packed-fp32-ops",
    # The first 64 bytes of a kernel's arguments are in registers when it starts (scalars and pointers up to the first
    # struct); fetching them costs every launch 0.4 us (back-to-back launches that copy a word per thread: 2.8 / 2.4 us)
    "-mllvm", "-amdgpu-kernarg-preload-count=16",
    "-Wall", "-Wno-unused-command-line-argument", "-Wno-unknown-warning-option",
]


def build_lib(verbose: bool = False) -> str:
    hipcc = os.environ.get("HIPCC", "/opt/rocm/bin/hipcc")
    with tempfile.TemporaryDirectory() as tmp:
        objects = [os.path.join(tmp, s + ".o") for s in SOURCES]
        compile_ = [[hipcc] + HIPCC_FLAGS + ["-c", os.path.join(CSRC, s), "-o", o] for s, o in zip(SOURCES, objects)]
        link = [hipcc, "--offload-arch=gfx950", "-shared", "-fPIC"] + objects + ["-o", LIB]
        if verbose:
            print("\n".join(" ".join(cmd) for cmd in compile_ + [link]))
        # the sources side by side: one alone takes most of the time that all of them take
        procs = [subprocess.Popen(cmd) for cmd in compile_]
        codes = [p.wait() for p in procs]
        for code, cmd in zip(codes, compile_):
            if code:
                raise subprocess.CalledProcessError(code, cmd)
        subprocess.run(link, check=True)
    return LIB


if __name__ == "__main__":
    print(build_lib(verbose=True))
