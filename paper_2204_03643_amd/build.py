"""Compiles the HIP library for gfx950 in-tree (hipcc cross-compiles without a GPU)."""
from __future__ import annotations

import hashlib
import os
import subprocess
import sys

HERE = os.path.dirname(os.path.abspath(__file__))
CSRC = os.path.join(HERE, "csrc")
LIB = os.path.join(HERE, "libtvprox.so")
STAMP = LIB + ".stamp"          # digest of the sources and flags the library was built from

HIPCC_FLAGS = [
    "--offload-arch=gfx950", "-O3", "-std=c++17", "-fPIC", "-shared",
    # keep the compiler from forming packed-fp32 instructions
    "-Xclang", "-target-feature", "-Xclang", "-packed-fp32-ops",
    "-Wall", "-Wno-unused-function",
]


def sources():
    return [os.path.join(CSRC, f) for f in sorted(os.listdir(CSRC)) if f.endswith(".hip")]


def source_digest() -> str:
    """Digest of everything the library is compiled from (file contents, not time stamps: a
    copy of the tree keeps the one and not necessarily the other)."""
    deps = [os.path.join(CSRC, f) for f in sorted(os.listdir(CSRC))]
    deps.append(os.path.join(os.path.dirname(HERE), "include", "tvprox.h"))
    h = hashlib.sha256(" ".join(HIPCC_FLAGS).encode())
    for d in deps:
        h.update(os.path.basename(d).encode())
        with open(d, "rb") as f:
            h.update(f.read())
    return h.hexdigest()


def is_stale() -> bool:
    """True when the library is missing or was built from other sources than those in the tree."""
    if not (os.path.exists(LIB) and os.path.exists(STAMP)):
        return True
    with open(STAMP) as f:
        return f.read().strip() != source_digest()


def build_library(verbose: bool = False) -> str:
    hipcc = os.environ.get("HIPCC", "/opt/rocm/bin/hipcc")
    tmp = LIB + ".tmp%d" % os.getpid()
    digest = source_digest()
    # a source a process, then the link
    objects = [tmp + ".%d.o" % i for i in range(len(sources()))]
    flags = [f for f in HIPCC_FLAGS if f != "-shared"]
    compiles = [[hipcc] + flags + ["-c", src, "-o", obj] for src, obj in zip(sources(), objects)]
    link = [hipcc, "--offload-arch=gfx950", "-shared", "-fPIC"] + objects + ["-o", tmp]
    try:
        running = []
        for cmd in compiles:
            if verbose:
                print(" ".join(cmd), flush=True)
            running.append(subprocess.Popen(cmd, stdout=subprocess.PIPE, stderr=subprocess.STDOUT, text=True))
        said = [p.communicate()[0] for p in running]
        if any(p.returncode for p in running):
            sys.stderr.write("".join(said))
            raise RuntimeError("hipcc failed")
        res = subprocess.run(link, capture_output=True, text=True)
        if res.returncode != 0:
            sys.stderr.write(res.stdout + res.stderr)
            raise RuntimeError("hipcc failed")
    finally:
        for obj in objects:
            if os.path.exists(obj):
                os.remove(obj)
    os.replace(tmp, LIB)
    with open(STAMP, "w") as f:
        f.write(digest + "\n")
    return LIB


if __name__ == "__main__":
    print(build_library(verbose=True))
