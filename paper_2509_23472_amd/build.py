"""Builds libloract.so (gfx950) in-tree with hipcc.  Run as `python -m paper_2509_23472_amd.build`."""
from __future__ import annotations

import os
import shutil
import subprocess
import sys

PKG_DIR = os.path.dirname(os.path.abspath(__file__))
CSRC = os.path.join(PKG_DIR, "csrc")
LIB_PATH = os.path.join(PKG_DIR, "libloract.so")

HIPCC_FLAGS = [
    "--offload-arch=gfx950", "-O3", "-std=c++17", "-fPIC", "-shared",
    "-Xclang", "-target-feature", "-Xclang", "-packed-fp32-ops",
    "-Wall", "-Wno-unused-function",
]


def hipcc_path() -> str:
    for cand in (os.environ.get("HIPCC"), shutil.which("hipcc"), "/opt/rocm/bin/hipcc"):
        if cand and os.path.exists(cand):
            return cand
    raise RuntimeError("hipcc not found")


def source_hash() -> str:
    """sha256 over the library's sources (csrc/ and the public header), in name order: identifies
    the build a profile was taken from."""
    import hashlib
    h = hashlib.sha256()
    files = sorted(os.path.join(CSRC, f) for f in os.listdir(CSRC) if f.endswith((".h", ".hip")))
    files.append(os.path.join(os.path.dirname(PKG_DIR), "include", "loract.h"))
    for path in files:
        h.update(os.path.basename(path).encode())
        with open(path, "rb") as fh:
            h.update(fh.read())
    return h.hexdigest()[:16]


def build_library(verbose: bool = True) -> str:
    """Compile every HIP source, each in a process of its own, link them into
    paper_2509_23472_amd/libloract.so and return its path."""
    import tempfile
    sources = sorted(os.path.join(CSRC, f) for f in os.listdir(CSRC) if f.endswith(".hip"))
    with tempfile.TemporaryDirectory() as tmp:
        objects, running = [], []
        for src in sources:
            obj = os.path.join(tmp, os.path.basename(src) + ".o")
            cmd = [hipcc_path()] + [f for f in HIPCC_FLAGS if f != "-shared"] + ["-c", src, "-o", obj]
            if verbose:
                print(" ".join(cmd), flush=True)
            objects.append(obj)
            running.append(subprocess.Popen(cmd, stdout=subprocess.PIPE, stderr=subprocess.STDOUT, text=True))
        results = [(proc.communicate()[0], proc.returncode) for proc in running]
        link = subprocess.run([hipcc_path(), "--offload-arch=gfx950", "-fPIC", "-shared"] + objects + ["-o", LIB_PATH + ".tmp"],
                              stdout=subprocess.PIPE, stderr=subprocess.STDOUT, text=True) \
            if all(code == 0 for _, code in results) else None
    if link is not None:
        results.append((link.stdout, link.returncode))
    out = "\n".join(line for text, _ in results for line in text.splitlines() if "packed-fp32-ops" not in line)
    if any(code != 0 for _, code in results):
        raise RuntimeError("hipcc failed:\n" + out)
    if verbose and out.strip():
        print(out)
    os.replace(LIB_PATH + ".tmp", LIB_PATH)
    return LIB_PATH


if __name__ == "__main__":
    build_library()
    sys.exit(0)
