"""Host-only guard on the registers of a decoder block's operators: their loops are timed with so many waves a SIMD and nothing spilled, which a small change of the
source can cost without failing a numerical test (a second copy of the dk/dv kernel's body: 290 spills, thirteen times the time)."""
import os
import re
import shutil
import subprocess

import pytest


def resources(tmp_path, source):
    """{kernel: (vector registers, vector spills)} as the compiler reports them"""
    from paper_2506_24119_amd import build as B
    if not (os.path.exists(B.HIPCC) or shutil.which(B.HIPCC)):
        pytest.skip("hipcc not available")
    cmd = [B.HIPCC] + B._flags() + ["-x", "hip", "--cuda-device-only", "-S", os.path.join(B.CSRC, source), "-o", str(tmp_path / "k.s")]
    r = subprocess.run(cmd, stdout=subprocess.PIPE, stderr=subprocess.STDOUT, text=True)
    assert r.returncode == 0, r.stdout[-2000:]
    return {m.group(1): (int(m.group(2)), int(m.group(3)))
            for m in re.finditer(r"\.name:\s+(\S+)\n(?:.*\n)*?\s+\.vgpr_count:\s+(\d+)\n\s+\.vgpr_spill_count:\s+(\d+)", open(tmp_path / "k.s").read())}


def test_packed_attention(tmp_path):
    """Three workgroups of four waves a compute unit for the forward kernel, two for the gradients'."""
    found = resources(tmp_path, "kernels_pack_attn.hip")
    for kernel, count, most in (("pack_forward_kernel", 6, 168), ("pack_dq_kernel", 6, 256), ("pack_dkv_kernel", 12, 256), ("pack_join_kernel", 2, 64)):
        these = {k: v for k, v in found.items() if kernel in k}
        assert len(these) == count, sorted(found)
        for name, (vgprs, spills) in these.items():
            assert vgprs <= most and spills == 0, (name, vgprs, spills)


def test_rows_stay_in_registers(tmp_path):
    for name, (vgprs, spills) in resources(tmp_path, "kernels_block.hip").items():
        assert vgprs <= 256 and spills == 0, (name, vgprs, spills)
