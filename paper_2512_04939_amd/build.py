"""Compile the HIP sources in csrc/ into liblitevggt.so (gfx950) with hipcc."""
from __future__ import annotations

import os
import subprocess
import sys

HERE = os.path.dirname(os.path.abspath(__file__))
CSRC = os.path.join(HERE, "csrc")
LIB = os.path.join(HERE, "liblitevggt.so")
SOURCES = ["api.hip", "importance.hip", "select.hip", "match.hip", "merge.hip", "attn.hip",
           "block.hip", "cache.hip", "attn_kv.hip", "rope.hip", "mass.hip", "evict.hip", "probe.hip"]
FLAGS = ["-O3", "--offload-arch=gfx950", "-fPIC", "-std=c++17", "-Wall", "-Wno-unused-function",
         # packed fp32 VALU forms are kept out of the generated code on this target
         "-Xclang", "-target-feature", "-Xclang", "-packed-fp32-ops"]


def build(verbose: bool = True, extra: list[str] | None = None, lib: str = LIB) -> str:
    objs = []
    procs = []
    os.makedirs(os.path.join(HERE, "_build"), exist_ok=True)
    for s in SOURCES:
        obj = os.path.join(HERE, "_build", s.replace(".hip", ".o"))
        cmd = ["hipcc", *FLAGS, *(extra or []), "-c", os.path.join(CSRC, s), "-o", obj]
        if verbose:
            print(" ".join(cmd), flush=True)
        procs.append((s, subprocess.Popen(cmd, stdout=subprocess.PIPE, stderr=subprocess.STDOUT)))
        objs.append(obj)
    failed = False
    for s, pr in procs:
        out, _ = pr.communicate()
        text = out.decode()
        # the host pass does not know the device-only target feature: harmless
        text = "\n".join(l for l in text.splitlines() if "is not a recognized feature" not in l)
        if text.strip() and verbose:
            print(text)
        if pr.returncode != 0:
            failed = True
            print(f"hipcc failed on {s}", file=sys.stderr)
    if failed:
        raise RuntimeError("HIP build failed")
    cmd = ["hipcc", "--offload-arch=gfx950", "-shared", "-fPIC", *objs, "-o", lib]
    if verbose:
        print(" ".join(cmd), flush=True)
    subprocess.check_call(cmd)
    return lib


if __name__ == "__main__":
    build()
