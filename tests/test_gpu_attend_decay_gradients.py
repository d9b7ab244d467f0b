"""The decays' gradients where they are far smaller than the sums around them, against the
definition in 64 bits.

A token's gradient is the sum of W[i,j] over j < t <= i, with W[i,j] = scale D[i,j]
(q[i] . k[j]) (dy[i] . v[j]) and D the product of the decays between.  The kernels
form it of differences of fp32 dots, one of 2-norm s to a token, whose terms do not
include W[t,t].  A dot's roundings are those of a chain of about 80 sums, each at most
2^-24 of a size of s, with signs of their own: 9 * 2^-24 s.  512 tokens' two dots add
up to 32 times that: 1.7e-5 s.  Of decays that are alike all over a row, a
gradient's size is s too, so 1e-4 of the gradient's 2-norm leaves a factor of 6.
"""
import pytest
import torch

from attend_ref import BF16, F16, F32
from gpu_util import announce
from paper_2505_15112_amd import ops
from test_gpu_attend import dev, inputs

pytestmark = pytest.mark.gpu
DEV = "cuda"


def gradient(a, dy, **more):
    announce("linear_attention_backward", tuple(a["q"].shape), tuple(a["v"].shape), a["q"].dtype)
    return ops.linear_attention_backward(dy.to(DEV), **dev(a), **more)[3]


@pytest.mark.parametrize("kind", [F32, F16, BF16])
@pytest.mark.parametrize("steps", [90, 1300])
@pytest.mark.parametrize("clear", [-float("inf"), torch.finfo(torch.float32).min])
def test_rows_of_two_sequences(kind, steps, clear):
    """A decay that clears the state, between two sequences of a row: the first one's
    gradients are those of a call of its own, whatever the second holds."""
    cut = steps // 2 + 3
    a, dy = inputs(1, steps, 2, 1, 40, 24, kind=kind, rate=0.05)
    a["log_decay"][:, cut] = clear
    first = {k: v[:, :cut] if k in ("q", "k", "v", "log_decay") else v for k, v in a.items()}
    want = gradient(first, dy[:, :cut])
    b = dict(a, v=a["v"].clone())
    b["v"][:, cut + 5, :, 3] = float("nan")
    c = dict(a, v=a["v"].clone())
    c["v"][:, cut:] *= 300
    for x in (a, b, c):
        got = gradient(x, dy)
        for h in range(2):
            # twice the 2-norm's bound above: two calls, each with its own roundings
            err = (got[0, :cut, h] - want[0, :, h]).norm()
            assert err <= 2e-4 * want[0, :, h].norm(), h
        assert not got[0, cut].any()
