"""No kernel of linear attention or layer norm keeps registers in memory, which a bound on
registers alone would not show (CPU only: cross-compiles for gfx950); and the walks of fp16 that two
workgroups of a CU are counted on for."""
import os
import re
import shutil
import subprocess

import pytest

from paper_2505_15112_amd import build as B

pytestmark = pytest.mark.skipif(shutil.which(B.HIPCC) is None and not os.path.exists(B.HIPCC),
                                reason="hipcc not available")


FOUND = {}  # by source


def kernels(source, tmp_path):
    """name: registers, LDS, registers spilled, scratch memory of a thread"""
    if source in FOUND:
        return FOUND[source]
    out = tmp_path / "kernels.s"
    flags = [f for f in B.CFLAGS if f != "-fPIC"]
    subprocess.run([B.HIPCC, *flags, "--cuda-device-only", "-S", os.path.join(B.CSRC, source),
                    "-o", str(out)], check=True, capture_output=True)
    text = out.read_text()
    found = FOUND[source] = {}
    for block in text[text.index("amdhsa.kernels"):].split("  - .agpr_count")[1:]:
        def field(key):
            return re.search(r"\." + key + r":\s+(\S+)", block).group(1)
        found[field("name")] = tuple(int(field(k)) for k in (
            "vgpr_count", "group_segment_fixed_size", "vgpr_spill_count",
            "private_segment_fixed_size"))
    return found


@pytest.mark.parametrize("source,count", [("attend_f32.hip", 18), ("attend_f16.hip", 18),
                                          ("attend_bf16.hip", 18), ("attend.hip", 10),
                                          ("norm.hip", 80)])
def test_nothing_is_spilled(source, count, tmp_path):
    found = kernels(source, tmp_path)
    assert len(found) >= count
    for name, (_, lds, spilled, scratch) in found.items():
        assert spilled == 0 and scratch == 0 and lds <= 160 * 1024, (name, lds, spilled, scratch)


def test_two_walks_of_fp16_share_a_cu(tmp_path):
    """Keys of up to 64 channels, without dots: eight waves of at most 128 registers, and
    their LDS, twice."""
    some = [v for n, v in kernels("attend_f16.hip", tmp_path).items()
            if re.search(r"Li64ELi8ELb[01]ELb0E", n)]
    assert len(some) == 2
    for vgpr, lds, _, _ in some:
        assert vgpr <= 128 and 2 * lds <= 160 * 1024
