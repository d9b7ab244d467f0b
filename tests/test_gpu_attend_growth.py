"""Linear attention whose decays grow past fp32 over a piece of a row, where the states do
not: rows that are cut into pieces and rows that are not give the same."""
import pytest
import torch

from attend_ref import BF16, F16, F32
from test_gpu_attend import check_backward, check_forward, inputs

pytestmark = pytest.mark.gpu
STEPS = 1024


@pytest.mark.parametrize("kind", [F32, F16, BF16])
def test_nothing_grows_from_an_empty_state(kind):
    """Factors of e^1.5 a token over the first 64 tokens, e^96 in all, whose keys are 0."""
    a, _ = inputs(1, STEPS, 1, 1, 64, 64, kind=kind)
    a["log_decay"][:, :64] = 1.5
    a["log_decay"][:, 64:] = -0.05
    a["k"][:, :64] = 0
    check_forward(a)


def test_a_first_state_with_zeros_grows_where_it_is_not_zero():
    """The state's columns that are 1e-33 at first are 1e-33 e^96 behind 64 tokens."""
    a, _ = inputs(1, STEPS, 2, 1, 40, 64, state=True)
    a["state"][..., ::2] = 0
    a["state"][..., 1::2] *= 1e-33
    a["log_decay"][:, :64] = 1.5
    a["log_decay"][:, 64:] = -0.05
    a["k"][:, :64] = 0
    check_forward(a)


@pytest.mark.parametrize("kind", [F32, BF16])
@pytest.mark.parametrize("batch", [1, 300])
def test_gradients_of_a_row_that_ends_in_growth(kind, batch):
    """Behind a cleared state, 64 tokens without keys and gradients grow by e^96 (and
    the same where the batch fills the GPU and no row is cut)."""
    a, dy = inputs(1, STEPS, 1, 1, 32, 32, kind=kind, rate=0.05)
    a["log_decay"][:, -96] = -float("inf")
    a["log_decay"][:, -64:] = 1.5
    a["k"][:, -96:] = 0
    dy[:, -96:] = 0
    if batch == 1:
        check_backward(a, dy)
        return
    one = check_backward(a, dy)
    b = {k: v.expand(batch, *v.shape[1:]).contiguous() if isinstance(v, torch.Tensor) else v
         for k, v in a.items()}
    from paper_2505_15112_amd import ops
    got = ops.linear_attention_backward(dy.expand(batch, *dy.shape[1:]).contiguous().cuda(),
                                        **{k: v.cuda() if isinstance(v, torch.Tensor) else v
                                           for k, v in b.items()})
    for g, w in zip(got[:4], one[:4]):
        assert torch.isfinite(g).all()
        # both are within some 2^-16 of the same sums, bf16's last rounding included
        assert (g[-1].float() - w[0].float()).abs().max() <= 2.0**-7 * w.float().abs().max()


def test_a_cleared_state_does_not_grow_back():
    """A row whose first 64 tokens clear the state and whose pieces then grow by 2^2000."""
    a, _ = inputs(1, 2048, 1, 1, 64, 64, state=True)
    a["log_decay"][:, 0] = -float("inf")
    a["log_decay"][:, 1:1000] = 1.4
    a["log_decay"][:, 1000:] = -0.05
    a["k"][:, :1000] = 0
    check_forward(a)
