"""Registers and LDS of the selective scan's kernels (CPU only: cross-compiles
for gfx950): the occupancy that their plans count on."""
import os
import re
import shutil
import subprocess

import pytest

from paper_2505_15112_amd import build as B

pytestmark = pytest.mark.skipif(shutil.which(B.HIPCC) is None and not os.path.exists(B.HIPCC),
                                reason="hipcc not available")


def resources(source, tmp_path):
    out = tmp_path / "kernels.s"
    flags = [f for f in B.CFLAGS if f != "-fPIC"]
    subprocess.run([B.HIPCC, *flags, "--cuda-device-only", "-S", os.path.join(B.CSRC, source),
                    "-o", str(out)], check=True, capture_output=True)
    text = out.read_text()
    found = {}
    for block in text[text.index("amdhsa.kernels"):].split("  - .agpr_count")[1:]:
        def field(key):
            return re.search(r"\." + key + r":\s+(\S+)", block).group(1)
        found[field("name")] = (int(field("vgpr_count")), int(field("group_segment_fixed_size")))
    return found


def test_two_gradient_workgroups_share_a_cu(tmp_path):
    """Up to 32 states: 4 waves of at most 256 registers twice, and their LDS."""
    found = resources("ssm_back.hip", tmp_path)
    some = [(n, v) for n, v in found.items()
            if re.search(r"k_ssm_back\w*(Li8ELi2|Li16ELi1|Li16ELi2)E", n)]
    assert len(some) >= 18
    for name, (vgpr, lds) in some:
        assert vgpr <= 256 and 2 * lds <= 160 * 1024, (name, vgpr, lds)


def test_four_scanning_waves_share_a_simd(tmp_path):
    """Up to 16 states to a lane: at most 128 registers; the tiles as well."""
    found = resources("ssm.hip", tmp_path)
    some = [(n, v) for n, v in found.items()
            if re.search(r"k_ssm_(lanes|ends)\w*Li(8|16)E", n) or "k_ssm_scan" in n]
    assert len(some) >= 30
    for name, (vgpr, lds) in some:
        assert vgpr <= 128 and lds <= 40 * 1024, (name, vgpr, lds)
