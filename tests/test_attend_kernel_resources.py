"""Registers, LDS and spills of linear attention's and layer norm's kernels (CPU only:
cross-compiles for gfx950): the occupancy that their plans count on."""
import os
import re
import shutil

import pytest

from paper_2505_15112_amd import build as B
from test_lm_kernel_resources import resources

pytestmark = pytest.mark.skipif(shutil.which(B.HIPCC) is None and not os.path.exists(B.HIPCC),
                                reason="hipcc not available")


def test_two_walks_share_a_cu(tmp_path):
    """bfloat16, keys of up to 128 channels: eight waves of at most 128 registers, and
    their LDS, twice."""
    found = resources("attend_bf16.hip", tmp_path)
    assert len(found) == 18
    some = [(n, v) for n, v in found.items() if re.search(r"Li(64|128)ELi8E", n)]
    assert len(some) == 6
    for name, (vgpr, lds) in some:
        assert vgpr <= 128 and 2 * lds <= 160 * 1024, (name, vgpr, lds)
    for name, (vgpr, lds) in found.items():
        assert vgpr <= 256 and lds <= 160 * 1024, (name, vgpr, lds)


def test_norm_teams_fill_a_cu(tmp_path):
    """Gradients by 1024 threads of at most 128 registers; forward rows of one vector a thread by
    twice as many."""
    found = resources("norm.hip", tmp_path)
    back = [(n, v) for n, v in found.items() if "k_norm_back" in n]
    assert len(back) >= 36
    for name, (vgpr, lds) in back:
        assert vgpr <= 128 and lds <= 160 * 1024, (name, vgpr, lds)
    front = [(n, v) for n, v in found.items() if re.search(r"6k_norm\w*ELi1EEE", n)]
    assert len(front) >= 35
    for name, (vgpr, _) in front:
        assert vgpr <= 64, (name, vgpr)
