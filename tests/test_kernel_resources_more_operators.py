"""No kernel for changed scores, 4-bit pages or block tables keeps vector registers or anything else in scratch memory."""
import os
import re
import subprocess

import pytest

from paper_2307_02628_amd import _build


@pytest.mark.parametrize("src,kernels", [("kv_scores.hip", 32), ("kv_scores_fp8.hip", 32), ("kv_scores_fp4.hip", 32), ("kv_fp4.hip", 20), ("kv_table.hip", 11)])
def test_no_kernel_spills(src, kernels, tmp_path):
    hipcc = os.environ.get("HIPCC", "/opt/rocm/bin/hipcc")
    res = subprocess.run([hipcc, "--offload-arch=gfx950", "--cuda-device-only", "-O3", "-std=c++17", "-fPIC", "-Xclang", "-target-feature", "-Xclang", "-packed-fp32-ops",
                          "-Rpass-analysis=kernel-resource-usage", "-x", "hip", "-c", os.path.join(_build.CSRC, src), "-o", str(tmp_path / "k.o")], capture_output=True, text=True)
    assert res.returncode == 0, res.stderr[-2000:]
    usage = {}
    for line in res.stderr.splitlines():
        if m := re.search(r"Function Name: (\S+)", line):
            usage[name := m.group(1)] = {}
        elif m := re.search(r"remark:\s+(ScratchSize \[bytes/lane\]|VGPRs Spill): (\d+)", line):
            usage[name][m.group(1)] = int(m.group(2))
    assert len(usage) >= kernels and all(len(u) == 2 for u in usage.values())
    bad = {k: u for k, u in usage.items() if any(u.values())}
    assert not bad, f"kernels that spill: {bad}"
