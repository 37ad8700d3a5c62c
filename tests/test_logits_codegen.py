"""What the kernels on logits are built around, checked on the generated assembly (no GPU: hipcc cross-compiles gfx950).

Few rows are cut into as many parts as the card holds at once, four workgroups of eight waves a compute unit: eight waves per SIMD,
which 64 vector registers a lane and 80 scalar registers a wave leave.
"""
import os
import re
import shutil
import subprocess

import pytest


def test_four_workgroups_per_compute_unit(tmp_path):
    if shutil.which("hipcc") is None and not os.path.exists("/opt/rocm/bin/hipcc"):
        pytest.skip("hipcc not found")
    from paper_2508_02322_amd import build
    out = tmp_path / "logits.s"
    flags = [f for f in build.FLAGS if f != "-fPIC"]
    res = subprocess.run([build.hipcc(), *flags, "--cuda-device-only", "-S", os.path.join(build.CSRC, "logits.hip"), "-o", str(out)],
                         capture_output=True, text=True)
    assert res.returncode == 0, res.stderr[-2000:]
    entries = re.findall(r"\.group_segment_fixed_size:\s+(\d+).*?\.name:\s+(\S+).*?\.private_segment_fixed_size:\s+(\d+)"
                         r".*?\.sgpr_count:\s+(\d+).*?\.vgpr_count:\s+(\d+)", out.read_text(), re.S)
    passes = {name: (int(lds), *map(int, rest)) for lds, name, *rest in entries if re.search(r"(logprobs|distill)_kernel", name)}
    # two types; log probabilities of whole rows (short and long workgroups) and of parts (long ones), with alternatives or without;
    # distillation with short and long workgroups, with the unlisted class or without
    assert len(passes) == 2 * (3 * 2) + 2 * (2 * 2), sorted(passes)
    for name, (lds, scratch, sgprs, vgprs) in passes.items():
        assert lds <= 160 * 1024 // 4 and scratch == 0 and sgprs <= 80 and vgprs <= 64, (name, lds, scratch, sgprs, vgprs)
