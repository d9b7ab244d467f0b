"""Gradients of layer norms with more groups than one launch's threads could take."""
import pytest
import torch

import attend_ref as R
from attend_ref import BF16, F32
from gpu_util import announce
from paper_2505_15112_amd import ops

pytestmark = pytest.mark.gpu
DEV = "cuda"


@pytest.mark.parametrize("kind", [F32, BF16])
@pytest.mark.parametrize("groups", [(1 << 22) + 8, (1 << 23)])
def test_more_groups_than_threads_of_a_launch(kind, groups):
    """Groups of two channels, 2^22 workgroups of 1024 threads and more in one launch."""
    dim, rows = 2 * groups, 3
    if dim > 1 << 24:
        dim = 1 << 24
    g = torch.Generator(device=DEV).manual_seed(1)
    x, dy = (torch.randn(rows, dim, device=DEV, generator=g).to(kind) for _ in range(2))
    w, b = (torch.randn(dim, device=DEV, generator=g).to(kind) for _ in range(2))
    announce("layer_norm_backward", rows, dim, groups, kind)
    y, _, stats = ops.layer_norm(x, w, b, groups=groups, with_stats=True)
    dx, dw, db = ops.layer_norm_backward(dy, x, stats, w, b, groups=groups)
    width = dim // groups
    for lo in (0, dim // 2 - 32 * width, dim - 64 * width):
        part = slice(lo, lo + 64 * width)
        ref = R.norm(x[:, part].cpu(), w[part].cpu(), b[part].cpu(), groups=64, dy=dy[:, part].cpu())
        r = 4 * 34 * 2.0**-24  # as in the other tests of the norm: two steps of sums and 32 more
        for name, t in (("dx", dx[:, part]), ("dweight", dw[part]), ("dbias", db[part])):
            R.assert_within(t, ref[name], ref["m" + name], r, name)
