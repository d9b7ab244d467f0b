"""Linear attention's outputs are rounded once: results that lie just beside the middle of
two numbers of the output's type, of states and scores that fp32 holds exactly."""
import pytest
import torch

from attend_ref import BF16, F16, F32
from gpu_util import announce
from paper_2505_15112_amd import ops

pytestmark = pytest.mark.gpu
DEV = "cuda"
SPACING = {BF16: 2.0**-7, F16: 2.0**-10, F32: 2.0**-23}  # of the numbers from 1 to 2
TINY = {BF16: 2.0**-20, F16: 2.0**-22, F32: 0.0}
KINDS = [F32, F16, BF16]


def parts(kind, *shape):
    """Numbers of the type from 1 to 2, half a spacing of them, and a little more or less."""
    g = torch.Generator().manual_seed(11)
    whole = 1 + SPACING[kind] * torch.randint(0, round(1 / SPACING[kind]) - 1, shape, generator=g)
    little = TINY[kind] * (torch.randint(0, 2, shape, generator=g) * 2 - 1)
    half = torch.full(shape, SPACING[kind] / 2 if kind != F32 else 0.0)
    return whole, half, little


@pytest.mark.parametrize("kind", KINDS)
@pytest.mark.parametrize("steps", [40, 700])
def test_a_state_that_is_read(kind, steps):
    """Every token reads one row of a state that nothing changes."""
    state = sum(parts(kind, 1, 2, 64, 48))
    q = torch.zeros(1, steps, 2, 64)
    q[0, torch.arange(steps), :, torch.arange(steps) % 64] = 1
    zeros = torch.zeros(1, steps, 2, 64).to(kind)
    announce("linear_attention", steps, kind)
    y, last = ops.linear_attention(q.to(kind).to(DEV), zeros.to(DEV), zeros[..., :48].to(DEV),
                                   torch.zeros(1, steps, 2, device=DEV), state.to(DEV), scale=1.0,
                                   with_state=True)
    assert torch.equal(last.cpu(), state)
    want = state[0, :, torch.arange(steps) % 64].transpose(0, 1).to(kind)
    assert torch.equal(y[0].cpu(), want)


@pytest.mark.parametrize("kind", KINDS)
def test_scores(kind):
    """Tokens that see themselves alone, as every decay clears the state: y = (q . k) v,
    dv = (q . k) dy, dq = (dy . v) k and dk = (dy . v) q, each of a score of three products
    and a power of two."""
    steps, g = 130, torch.Generator().manual_seed(12)
    score = torch.stack(parts(kind, 1, steps, 2), -1)  # 1 x steps x 2 x 3
    ones = torch.ones(1, steps, 2, 3)
    power = 2.0 ** torch.randint(-3, 4, (1, steps, 2, 3), generator=g)
    decay = torch.full((1, steps, 2), -float("inf"), device=DEV)
    total = score.sum(-1, keepdim=True)  # exact

    def on(t):
        return t.to(kind).to(DEV)

    announce("linear_attention, backward", kind)
    y, _ = ops.linear_attention(on(score), on(ones), on(power), decay, scale=1.0)
    assert torch.equal(y.cpu(), (total * power).to(kind))
    dv = ops.linear_attention_backward(on(power), on(score), on(ones), on(power), decay,
                                       scale=1.0)[2]
    assert torch.equal(dv.cpu(), (total * power).to(kind))
    dq, dk, _, dg, _ = ops.linear_attention_backward(on(score), on(power), on(power), on(ones),
                                                     decay, scale=1.0)
    assert torch.equal(dq.cpu(), (total * power).to(kind))
    assert torch.equal(dk.cpu(), (total * power).to(kind))
    assert not dg.any()
