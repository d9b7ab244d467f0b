"""Layer norm and its gradients: rows of one value far from zero, and bounds that hold the
variance and the gradients where the mean is far larger than the deviation."""
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


def bounds(x, weight, dy, eps, steps):
    """The definition in 64 bits with the errors of a computation in two passes.  With r =
    steps 2^-24: the mean is off by e = r mean|x|, which is added to every difference;
    squares of differences add up to within r, so the variance is off by e^2 + r var (to first order
    a common shift leaves it), and 1 / sqrt of it by half of that relative to it."""
    v = x.double()
    n = v.shape[-1]
    mean = v.mean(-1, keepdim=True)
    d = v - mean
    var = (d * d).mean(-1, keepdim=True)
    rstd = 1 / torch.sqrt(var + eps)
    hat = d * rstd
    r = steps * 2.0**-24
    e = r * v.abs().mean(-1, keepdim=True)
    off = 0.5 * (e * e + r * var) / (var + eps) + 3 * 2.0**-24  # of rstd, relative
    ehat = e * rstd + (off + 3 * 2.0**-24) * hat.abs()
    u = dy.double() * weight.double()
    m0, m1 = u.mean(-1, keepdim=True), (u * hat).mean(-1, keepdim=True)
    em1 = (u.abs() * ehat).mean(-1, keepdim=True) + r * (u * hat).abs().mean(-1, keepdim=True)
    dx = rstd * (u - m0 - hat * m1)
    edx = rstd * (r * u.abs().mean(-1, keepdim=True) + 4 * 2.0**-24 * (u.abs() + m0.abs()) +
                  ehat * m1.abs() + hat.abs() * em1) + (off + 2 * 2.0**-24) * dx.abs()
    return dict(mean=(mean, e), rstd=(rstd, off * rstd),
                y=(hat * weight.double(), (ehat + 2.0**-24 * hat.abs()) * weight.double().abs()),
                dx=(dx, edx))


@pytest.mark.parametrize("dim", [64, 1024, 4096, 20000])
def test_a_mean_of_a_thousand_deviations(dim):
    g = torch.Generator().manual_seed(4)
    x = torch.randn(6, dim, generator=g) + 1000.0
    dy, w = torch.randn(6, dim, generator=g), torch.randn(dim, generator=g)
    announce("layer_norm", (6, dim))
    y, _, stats = ops.layer_norm(x.to(DEV), w.to(DEV), with_stats=True)
    dx, _, _ = ops.layer_norm_backward(dy.to(DEV), x.to(DEV), stats, w.to(DEV))
    # a thread's chain of at most dim / 64 sums, then some 16 over lanes and waves
    want = bounds(x, w, dy, 1e-5, dim / 64 + 32)
    got = dict(mean=stats[..., 0, :1], rstd=stats[..., 0, 1:], y=y, dx=dx)
    for name, t in got.items():
        ref, tol = want[name]
        # the bounds say something: of most elements they are far below the size
        assert tol.median() < 0.05 * ref.abs().median(), name
        bad = (t.cpu().double() - ref).abs() > tol + 2.0**-24 * ref.abs()
        assert not bad.any(), (name, int(bad.sum()))
