"""Layer norm and its gradients: rows of one value far from zero."""
import pytest
import torch

import attend_ref as R
from attend_ref import BF16, F32
from gpu_util import announce
from paper_2505_15112_amd import ops

pytestmark = pytest.mark.gpu
DEV = "cuda"


@pytest.mark.parametrize("kind", [F32, BF16])
@pytest.mark.parametrize("dim,power,eps", [(6, 121, 1e-5), (24, 121, 1e-5), (48, 121, 1e-5),
                                           (96, 121, 1e-5), (768, 110, 1e-12),
                                           (1536, 110, 1e-12), (6144, 110, 1e-12)])
def test_gradients_of_constant_rows_far_from_zero(kind, dim, power, eps):
    """Rows of 2^power, whose sums (of 3 2^n elements) are exact and within fp32: xhat is 0 and dx
    is rstd (u - mean(u)), which is finite, while 2^power rstd is beyond fp32."""
    g = torch.Generator().manual_seed(3)
    x = torch.full((5, dim), 2.0**power).to(kind)
    dy = torch.randn(5, dim, generator=g).to(kind)
    w = torch.randn(dim, generator=g).to(kind)
    announce("layer_norm_backward", (5, dim), kind)
    y, _, stats = ops.layer_norm(x.to(DEV), w.to(DEV), eps=eps, with_stats=True)
    assert not y.any() and bool((stats[:, 0, 0] == 2.0**power).all())
    dx, dw, _ = ops.layer_norm_backward(dy.to(DEV), x.to(DEV), stats, w.to(DEV))
    u = dy.double() * w.double()
    rstd = eps ** -0.5
    want = rstd * (u - u.mean(-1, keepdim=True))
    mag = rstd * (u.abs() + u.abs().mean(-1, keepdim=True))
    R.assert_within(dx, want, mag, (dim / 64 + 32) * 2.0**-24, "dx")
    assert not dw.any()
