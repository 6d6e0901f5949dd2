"""Compile the HIP sources of this package for gfx950 into libbpd.so (in-tree)."""
from __future__ import annotations

import os
import subprocess
import sys
import tempfile

HERE = os.path.dirname(os.path.abspath(__file__))
LIB = os.path.join(HERE, "libbpd.so")
SOURCES = [os.path.join(HERE, "csrc", f) for f in ("bpd.hip", "bpd_cache.hip")]
FLAGS = [
    "--offload-arch=gfx950", "-O3", "-std=c++17", "-shared", "-fPIC",
    # packed-fp32 code generation is kept off on purpose: some packed forms have given wrong results on this hardware
    "-Xclang", "-target-feature", "-Xclang", "-packed-fp32-ops",
    "-Wno-unused-result",
]


def hipcc() -> str:
    for cand in (os.environ.get("HIPCC"), "/opt/rocm/bin/hipcc", "hipcc"):
        if cand and (os.path.isabs(cand) and os.path.exists(cand) or not os.path.isabs(cand)):
            return cand
    return "hipcc"


def build(verbose: bool = False) -> str:
    with tempfile.TemporaryDirectory(prefix="bpd_build_") as tmp:
        objects = [os.path.join(tmp, os.path.basename(s) + ".o") for s in SOURCES]
        compile_flags = [f for f in FLAGS if f != "-shared"]
        cmds = [[hipcc()] + compile_flags + ["-c", s, "-o", o] for s, o in zip(SOURCES, objects)]
        link = [hipcc()] + FLAGS + objects + ["-o", LIB]
        if verbose:
            print("\n".join(" ".join(c) for c in cmds + [link]), flush=True)
        # the sources side by side, then the library
        running = [subprocess.Popen(c, stdout=subprocess.PIPE, stderr=subprocess.STDOUT, text=True) for c in cmds]
        done = [(p.communicate()[0], p.returncode) for p in running]
        if all(rc == 0 for _, rc in done):
            res = subprocess.run(link, stdout=subprocess.PIPE, stderr=subprocess.STDOUT, text=True)
            done.append((res.stdout, res.returncode))
    out = "\n".join(l for text, _ in done for l in text.splitlines() if "not a recognized feature" not in l)
    if any(rc != 0 for _, rc in done):
        raise RuntimeError("hipcc failed:\n" + out)
    if verbose and out.strip():
        print(out)
    return LIB


if __name__ == "__main__":
    print(build(verbose=True))
