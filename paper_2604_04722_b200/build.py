"""Build ``libkvq.so`` (the C-ABI CUDA library) in-tree with nvcc for sm_100a."""
from __future__ import annotations

import os
import subprocess
import sys

_HERE = os.path.dirname(os.path.abspath(__file__))
CSRC = os.path.join(_HERE, "csrc")
LIB = os.path.join(_HERE, "libkvq.so")
SOURCES = [os.path.join(CSRC, "kvq.cu"), os.path.join(CSRC, "kvq_rows.cu"), os.path.join(CSRC, "kvq_pages.cu")]
NVCC_FLAGS = [
    "-gencode", "arch=compute_100a,code=sm_100a", "-lineinfo", "-O3", "-std=c++17",
    "-Xcompiler", "-fPIC", "-Xptxas", "-v",
]


def _deps():
    out = []
    for root in (CSRC, os.path.join(os.path.dirname(_HERE), "include")):
        for name in os.listdir(root):
            if name.endswith((".cu", ".cuh", ".h")):
                out.append(os.path.join(root, name))
    return out


def stale() -> bool:
    if not os.path.exists(LIB):
        return True
    t = os.path.getmtime(LIB)
    return any(os.path.getmtime(f) > t for f in _deps())


def build(force: bool = False, verbose: bool = False) -> str:
    """Compile the library if missing or older than its sources; returns its path."""
    if not force and not stale():
        return LIB
    nvcc = os.environ.get("NVCC", "nvcc")
    tmp = LIB + ".tmp.%d" % os.getpid()
    objects = ["%s.%d.o" % (tmp, i) for i in range(len(SOURCES))]
    try:
        # the sources are compiled side by side, then linked
        jobs = [([nvcc, *NVCC_FLAGS, "-c", "-o", obj, src], subprocess.Popen(
            [nvcc, *NVCC_FLAGS, "-c", "-o", obj, src], stdout=subprocess.PIPE, stderr=subprocess.STDOUT, text=True))
            for src, obj in zip(SOURCES, objects)]
        done = [(cmd, proc.communicate()[0], proc.returncode) for cmd, proc in jobs]
        if all(rc == 0 for _, _, rc in done):
            cmd = [nvcc, *NVCC_FLAGS, "-shared", "-o", tmp, *objects]
            link = subprocess.run(cmd, stdout=subprocess.PIPE, stderr=subprocess.STDOUT, text=True)
            done.append((cmd, link.stdout, link.returncode))
        for cmd, text, rc in done:
            if verbose or rc != 0:
                sys.stderr.write(text)
            if rc != 0:
                raise RuntimeError("nvcc failed (%d): %s" % (rc, " ".join(cmd)))
    finally:
        for obj in objects:
            if os.path.exists(obj):
                os.remove(obj)
    os.replace(tmp, LIB)
    return LIB


if __name__ == "__main__":
    print(build(force="--force" in sys.argv, verbose=True))
