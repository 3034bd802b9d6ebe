"""Build the HIP library (libskd.so) in-tree for gfx950 with hipcc."""
from __future__ import annotations

import os
import subprocess
import sys

HERE = os.path.dirname(os.path.abspath(__file__))
CSRC = os.path.join(HERE, "csrc")
LIB = os.path.join(HERE, "libskd.so")
SOURCES = ["skd_schedule.cpp", "skd_engine.hip", "kernels_f32.hip", "kernels_bf16.hip", "team_column.hip", "kv_ops.hip", "sample_rows.hip", "skd_ops.hip"]
HEADERS = [os.path.join(CSRC, "skd_kernels.h"), os.path.join(CSRC, "bf16_device.h"), os.path.join(CSRC, "once_per_device.h"), os.path.join(CSRC, "gave_up.h"), os.path.join(CSRC, "kv_pages.h"), os.path.join(CSRC, "kv_ops.h"), os.path.join(CSRC, "sample_rows.h"), os.path.join(os.path.dirname(HERE), "include", "skd.h")]


def stale() -> bool:
    if not os.path.exists(LIB):
        return True
    t = os.path.getmtime(LIB)
    deps = [os.path.join(CSRC, s) for s in SOURCES] + HEADERS
    return any(os.path.getmtime(d) > t for d in deps)


def build(force: bool = True, verbose: bool = False) -> str:
    if not force and not stale():
        return LIB
    hipcc = os.environ.get("HIPCC", "/opt/rocm/bin/hipcc")
    cmd = [hipcc, "--offload-arch=gfx950", "-O3", "-std=c++17", "-fPIC", "-shared",
           "-Xclang", "-target-feature", "-Xclang", "-packed-fp32-ops",
           "-Wall", "-Wno-unused-function", "-x", "hip"]
    cmd += [os.path.join(CSRC, s) for s in SOURCES]
    cmd += ["-o", LIB]
    res = subprocess.run(cmd, capture_output=True, text=True)
    # the host pass does not know the packed-fp32 feature and says so: harmless
    err = "\n".join(l for l in res.stderr.splitlines() if "packed-fp32-ops" not in l)
    if res.returncode != 0:
        raise RuntimeError("hipcc failed:\n" + err)
    if verbose and err.strip():
        print(err, file=sys.stderr)
    return LIB


if __name__ == "__main__":
    print(build(force=True, verbose=True))
