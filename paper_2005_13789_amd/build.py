"""Build libne.so (HIP kernels + C ABI) in-tree for gfx950 with hipcc."""
from __future__ import annotations

import os
import subprocess
import sys
import tempfile

PKG = os.path.dirname(os.path.abspath(__file__))
ROOT = os.path.dirname(PKG)
SRCS = [os.path.join(PKG, "csrc", f) for f in ("ne.hip", "ne_shared.hip", "ne_embed.hip", "ne_xent.hip", "ne_logprob.hip", "ne_adamw.hip", "ne_muon.hip")]
OUT = os.path.join(PKG, "libne.so")

HIPCC_FLAGS = [
    "-O3", "-std=c++17", "--offload-arch=gfx950", "-shared", "-fPIC",
    "-I", os.path.join(ROOT, "include"),
    # packed fp32 ops stay off: some of their forms have given wrong results on this hardware
    "-Xclang", "-target-feature", "-Xclang", "-packed-fp32-ops",
    # fp32 atomic adds must become global_atomic_add_f32, not a compare-and-swap loop
    "-munsafe-fp-atomics",
    "-Wall", "-Wno-unused-function",
]


def build(verbose: bool = False) -> str:
    """Compiles the sources side by side, then links them."""
    compile_flags = [f for f in HIPCC_FLAGS if f != "-shared"]
    with tempfile.TemporaryDirectory() as tmp:
        objects = [os.path.join(tmp, os.path.basename(src) + ".o") for src in SRCS]
        commands = [["hipcc", *compile_flags, "-c", src, "-o", obj] for src, obj in zip(SRCS, objects)]
        link = ["hipcc", "-shared", "-fPIC", "--offload-arch=gfx950", *objects, "-o", OUT]
        if verbose:
            for cmd in (*commands, link):
                print(" ".join(cmd), flush=True)
        running = [subprocess.Popen(cmd) for cmd in commands]
        failed = [cmd for cmd, process in zip(commands, running) if process.wait() != 0]
        if failed:
            raise subprocess.CalledProcessError(1, failed[0])
        subprocess.run(link, check=True)
    return OUT


if __name__ == "__main__":
    build(verbose=True)
    print(OUT)
    sys.exit(0)
