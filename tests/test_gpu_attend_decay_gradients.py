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
from test_gpu_attend import check_backward, check_forward, dev, inputs

pytestmark = pytest.mark.gpu
DEV = "cuda"


def pairs(a, dy, b, h, absolute=False):
    """W of row b's head h, on the GPU in 64 bits."""
    per = a["v"].shape[2] // a["q"].shape[2]
    f = torch.abs if absolute else (lambda t: t)
    q, k = (f(a[x][b, :, h // per].to(DEV).double()) for x in ("q", "k"))
    v, d = f(a["v"][b, :, h].to(DEV).double()), f(dy[b, :, h].to(DEV).double())
    g = a["log_decay"]
    c = (g[b, :, h] if g.dim() > 1 else g[h].expand(len(q))).to(DEV).double().cumsum(0)
    over = (c[:, None] - c[None]).masked_fill(
        torch.ones(len(q), len(q), dtype=torch.bool, device=DEV).triu(1), -float("inf"))
    return torch.exp(over) * (q @ k.t().contiguous()) * (d @ v.t().contiguous()) / q.shape[1] ** 0.5


def crossing(w):
    """For each t the sum of w[i,j] over j < t <= i."""
    before = torch.cat((torch.zeros_like(w[:, :1]), w.cumsum(1)[:, :-1]), 1)  # over j < t
    return before.flip(0).cumsum(0).flip(0).diagonal()


def gradient(a, dy, **more):
    announce("linear_attention_backward", tuple(a["q"].shape), tuple(a["v"].shape), a["q"].dtype)
    return ops.linear_attention_backward(dy.to(DEV), **dev(a), **more)[3]


@pytest.mark.parametrize("kind", [F32, F16, BF16])
@pytest.mark.parametrize("heads", [2, 600])
def test_decays_that_leave_little(kind, heads):
    """Decays between e^-8 and e^-16 over 2100 tokens; rows in pieces and whole (600 heads,
    of which the first and last are looked at)."""
    a, dy = inputs(1, 2100, heads, heads, 64, 64, kind=kind)
    a["log_decay"] = -8.0 - 8.0 * torch.rand(*a["log_decay"].shape,
                                             generator=torch.Generator().manual_seed(7))
    got = gradient(a, dy)
    for h in (0, heads - 1):
        want = crossing(pairs(a, dy, 0, h))
        assert (got[0, :, h] - want).norm() <= 1e-4 * want.norm(), h


@pytest.mark.parametrize("kind", [F32, BF16])
def test_one_decay_for_all_tokens(kind):
    """Heads' decays of e^-8 and e^-16: the sums of the tokens' gradients."""
    a, dy = inputs(2, 700, 2, 1, 64, 64, kind=kind, fixed=True)
    a["log_decay"] = torch.tensor([-8.0, -16.0])
    got = gradient(a, dy)
    for h in range(2):
        tokens = torch.stack([crossing(pairs(a, dy, b, h)) for b in range(2)])
        # a sum of 1400 of them: the tokens' errors as they are, at worst all of one sign
        assert (got[h] - tokens.sum()).abs() <= 1e-4 * tokens.norm() * 1400 ** 0.5


@pytest.mark.parametrize("heads", [2, 600])
def test_strong_decays_before_weak_ones(heads):
    """Decays of e^-12, and behind them of e^-0.01: the first tokens' gradients hold no
    roundings of the later ones'.  The last 512 tokens of strong decays may."""
    a, dy = inputs(1, 2100, heads, heads, 64, 64)
    a["log_decay"][:, :1300] = -12.0
    a["log_decay"][:, 1300:] = -0.01
    got = gradient(a, dy)
    for h in (0, heads - 1):
        want = crossing(pairs(a, dy, 0, h))
        for part in (slice(0, 788), slice(1300, None)):
            assert (got[0, part, h] - want[part]).norm() <= 1e-4 * want[part].norm(), (h, part)


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


@pytest.mark.parametrize("steps,dims", [(512, (24, 40)), (513, (24, 40)), (1025, (130, 70)),
                                        (1600, (24, 40))])
def test_rows_around_the_boundaries_of_the_sums(steps, dims):
    """Ragged rows, first states and gradients of last ones, lengths at and around
    multiples of 512, against the definition."""
    a, dy = inputs(3, steps, 2, 1, *dims, kind=BF16, state=True, lengths=[steps, 512, 33],
                   rate=0.05)
    so = torch.randn(*a["state"].shape, generator=torch.Generator().manual_seed(3))
    check_backward(a, dy, so)


@pytest.mark.parametrize("kind", [F16, BF16])
@pytest.mark.parametrize("dims", [(64, 64), (128, 100)])
def test_long_rows_against_the_definition(kind, dims):
    """Rows of 2049 tokens, cut into pieces, forward and gradients."""
    a, dy = inputs(1, 2049, 2, 1, *dims, kind=kind, state=True, rate=0.02)
    check_forward(a)
    check_backward(a, dy, torch.randn(*a["state"].shape,
                                      generator=torch.Generator().manual_seed(3)))


def test_more_rows_than_workgroups_of_a_launch():
    """2^20 + 5 rows of two tokens, whose only pair is that of tokens 0 and 1."""
    rows, d = (1 << 20) + 5, 4
    g = torch.Generator(device=DEV).manual_seed(3)
    q, k, v, dy = (torch.randn(rows, 2, 1, d, device=DEV, generator=g) for _ in range(4))
    decay = -torch.rand(rows, 2, 1, device=DEV, generator=g)
    announce("linear_attention_backward", rows)
    got = ops.linear_attention_backward(dy, q, k, v, decay)[3][:, :, 0]
    qk, dv = ((x[:, 1, 0].double() * y[:, 0, 0].double()) for x, y in ((q, k), (dy, v)))
    a = torch.exp(decay[:, 1, 0].double()) / d ** 0.5
    want, mag = a * qk.sum(1) * dv.sum(1), a * qk.abs().sum(1) * dv.abs().sum(1)
    # two dots of four terms through some eight roundings each, and their difference (token 1's
    # k dq is 0)
    assert ((got[:, 1] - want).abs() <= 32 * 2.0**-24 * mag + 2.0**-126).all()
    assert (got[:, 0].abs() <= 32 * 2.0**-24 * mag + 2.0**-126).all()


def test_a_captured_graph_of_long_rows_replays():
    """Rows of several 512 tokens, ragged, replayed over new inputs with eager work between."""
    size, lengths = (3, 1300, 2, 1, 64, 48), [1300, 1024, 70]
    a, dy = inputs(*size, kind=BF16, state=True, lengths=lengths, rate=0.1)
    d, dy = dev(a), dy.to(DEV)

    def work():
        y, last = ops.linear_attention(**d, with_state=True)
        return (y, last, *ops.linear_attention_backward(dy, **d, dstate_out=last))

    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    with torch.cuda.stream(side):
        first = work()
    torch.cuda.current_stream().wait_stream(side)
    assert all(torch.equal(x, w) for x, w in zip(first, work()))
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        out = work()
    for seed in range(3):
        b, dy2 = inputs(*size, kind=BF16, state=True, lengths=lengths, rate=0.1, seed=20 + seed)
        for k in ("q", "k", "v", "log_decay", "state"):
            d[k].copy_(b[k])
        dy.copy_(dy2)
        want = work()
        torch.cuda.synchronize()
        graph.replay()
        torch.cuda.synchronize()
        assert all(torch.equal(x, w) for x, w in zip(out, want))
