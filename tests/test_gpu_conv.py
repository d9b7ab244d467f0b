"""The causal convolution, its gradients and its single-token step against the
definition in 64 bits (lm_ref.py, where the bounds are derived)."""
import pytest
import torch

import lm_ref as R
from gpu_util import announce
from paper_2505_15112_amd import ops

pytestmark = pytest.mark.gpu
DEV = "cuda"
F32, F16, BF16 = torch.float32, torch.float16, torch.bfloat16


def inputs(batch, steps, dim, width, kind=F32, wkind=None, bias=True, state=False, seed=0):
    g = torch.Generator().manual_seed(seed)

    def normal(*s, dtype=kind):
        return torch.randn(*s, generator=g).to(dtype)

    wkind = wkind or kind
    return (normal(batch, steps, dim), normal(dim, width, dtype=wkind),
            normal(dim, dtype=wkind) if bias else None,
            normal(batch, width - 1, dim) if state else None, normal(batch, steps, dim))


def to(*ts):
    return [t.to(DEV) if t is not None else None for t in ts]


def dbl(*ts):
    return [t.double() if t is not None else None for t in ts]


def check(x, w, bias, state, dy, lengths=None, silu=True, dstate_out=None):
    announce("causal_conv", tuple(x.shape), tuple(w.shape), x.dtype, w.dtype)
    n = torch.tensor(lengths, dtype=torch.int32) if lengths is not None else None
    dx_, dw_, db_, ds_ = to(x, w, bias, state)
    nd = n.to(DEV) if n is not None else None
    y, last = ops.causal_conv(dx_, dw_, db_, state=ds_, lengths=nd, silu=silu, with_state=True)
    args = (*dbl(x, w, bias, state), n, silu)
    ry, rlast, mag, _, _ = R.conv(*args)
    R.assert_within(y, ry, mag, 16, "y")
    assert torch.equal(last.cpu().double(), rlast)
    so = dstate_out
    got = ops.causal_conv_backward(dy.to(DEV), dx_, dw_, db_, state=ds_, lengths=nd, silu=silu,
                                   dstate_out=so.to(DEV) if so is not None else None,
                                   with_dstate=True)
    so = so.double() if so is not None else None
    ref = R.conv_back(dy.double(), *args, dstate_out=so)
    mags = R.conv_back(dy.double(), *args, dstate_out=so, absolute=True)
    terms = x.shape[0] * x.shape[1]
    for name, g, r, m in zip(("dx", "dweight", "dbias", "dstate"), got, ref, mags):
        if g is None:
            assert name == "dbias" and bias is None
            continue
        R.assert_within(g, r, m, 24 + (terms if name in ("dweight", "dbias") else 0), name)
    return got


SIZES = [(1, 1, 1), (1, 2, 5), (2, 15, 8), (1, 16, 64), (3, 17, 130), (2, 33, 9), (1, 257, 24),
         (2, 600, 66)]


@pytest.mark.parametrize("size", SIZES)
@pytest.mark.parametrize("width", [2, 3, 4])
@pytest.mark.parametrize("kind,wkind", [(F32, F32), (F16, F16), (BF16, BF16), (BF16, F32)])
def test_conv_and_gradients(size, width, kind, wkind):
    x, w, bias, state, dy = inputs(*size, width, kind, wkind, state=size[1] % 2 == 1)
    check(x, w, bias, state, dy)


@pytest.mark.parametrize("kind,wkind", [(F32, F32), (BF16, F32), (BF16, BF16)])
def test_conv_gradients_over_many_rows(kind, wkind):
    """Sums over many workgroups, whole ones and others."""
    for size in ((9, 500, 40), (24, 248, 128)):
        x, w, bias, state, dy = inputs(*size, 4, kind, wkind)
        check(x, w, bias, state, dy)


@pytest.mark.parametrize("silu", [True, False])
@pytest.mark.parametrize("bias", [True, False])
def test_conv_without_parts(silu, bias):
    x, w, b, state, dy = inputs(2, 40, 20, 4, F16, bias=bias, state=True)
    so = torch.randn(2, 3, 20, generator=torch.Generator().manual_seed(5)).half()
    check(x, w, b, state, dy, silu=silu, dstate_out=so)


@pytest.mark.parametrize("width", [2, 4])
def test_conv_ragged_rows_do_not_read_past_their_tokens(width):
    lengths = [0, 1, 2, 3, 16, 19, 39, 70, -1]
    x, w, b, state, dy = inputs(9, 39, 37, width, BF16, state=True)
    for r, n in enumerate(lengths):
        x[r, max(n, 0):] = float("nan")
        dy[r, max(n, 0):] = float("inf")
    so = torch.randn(9, width - 1, 37, generator=torch.Generator().manual_seed(5)).bfloat16()
    check(x, w, b, state, dy, lengths=lengths, dstate_out=so)


def test_conv_strided_inputs():
    x, w, b, state, dy = inputs(3, 40, 30, 4, BF16, state=True)
    want = ops.causal_conv(*to(x, w, b, state), with_state=True)
    wg = ops.causal_conv_backward(*to(dy, x, w, b), state=state.to(DEV))
    big = torch.full((40, 3, 61), float("nan"), dtype=BF16, device=DEV)
    xs, dys = big[:, :, :30].transpose(0, 1), big[:, :, 31:].transpose(0, 1)
    xs.copy_(x)
    dys.copy_(dy)
    got = ops.causal_conv(xs, *to(w, b, state), with_state=True)
    assert torch.equal(got[0], want[0]) and torch.equal(got[1], want[1])
    gg = ops.causal_conv_backward(dys, xs, *to(w, b), state=state.to(DEV))
    assert all(torch.equal(p, q) for p, q in zip(gg, wg))


@pytest.mark.parametrize("batch,steps,dim", [(0, 4, 8), (2, 0, 8), (2, 4, 0)])
def test_conv_empty(batch, steps, dim):
    x, w, b, state, dy = to(*inputs(batch, steps, dim, 4, F32, state=True))
    y, last = ops.causal_conv(x, w, b, state=state, with_state=True)
    assert y.shape == (batch, steps, dim)
    if steps == 0:
        assert torch.equal(last, state)
    so = torch.randn_like(state)
    dx, dw, db, ds = ops.causal_conv_backward(dy, x, w, b, state=state, dstate_out=so)
    assert not dw.any() and not db.any()
    if steps == 0:
        assert torch.equal(ds, so)


def test_conv_gradients_against_differences():
    x, w, b, state, dy = inputs(2, 21, 12, 4, F32, state=True)
    got = check(x, w, b, state, dy)
    args = dict(zip("xwbs", dbl(x, w, b, state)))

    def f(a):
        return (R.conv(a["x"], a["w"], a["b"], a["s"], None, True)[0] * dy.double()).sum()

    for name, g in zip("xwbs", got):
        v = torch.randn(args[name].shape, generator=torch.Generator().manual_seed(7)).double()
        slope = (f(dict(args, **{name: args[name] + 1e-5 * v}))
                 - f(dict(args, **{name: args[name] - 1e-5 * v}))) / 2e-5
        terms = g.double().cpu() * v
        assert abs(slope - terms.sum()) <= 1e-5 * terms.abs().sum() + 1e-6, name


@pytest.mark.parametrize("batch,dim", [(1, 1), (3, 65), (64, 256)])
@pytest.mark.parametrize("width", [2, 3, 4])
@pytest.mark.parametrize("kind", [F32, F16, BF16])
def test_step_moves_the_window(batch, dim, width, kind):
    x, w, b, state, _ = inputs(batch, 5, dim, width, kind, state=True)
    xd, wd, bd, pool = to(x, w, b, state)
    announce("causal_conv_step", batch, dim, width, kind)
    ry, rlast, mag, _, _ = R.conv(*dbl(x, w, b, state), None, True)
    for t in range(5):
        y = ops.causal_conv_step(xd[:, t], pool, wd, bd)
        R.assert_within(y, ry[:, t], mag[:, t], 16, f"y[{t}]")
    assert torch.equal(pool.cpu().double(), rlast)


def test_step_slots():
    x, w, b, _, _ = to(*inputs(5, 1, 33, 4, BF16))
    pool = torch.randn(9, 3, 33, device=DEV).bfloat16()
    before = pool.clone()
    slots = torch.tensor([7, -1, 0, 9, 3], dtype=torch.int32, device=DEV)
    y = ops.causal_conv_step(x[:, 0], pool, w, b, slots=slots)
    rows, used = [0, 2, 4], [7, 0, 3]
    dense = before[used].clone()
    assert torch.equal(y[rows], ops.causal_conv_step(x[rows, 0], dense, w, b))
    assert torch.equal(pool[used], dense) and not y[[1, 3]].any()
    rest = [i for i in range(9) if i not in used]
    assert torch.equal(pool[rest], before[rest])


def test_refusals():
    x, w, b, state, dy = to(*inputs(2, 6, 8, 4, F32, state=True))
    bad = [(dict(x=x.double()), TypeError), (dict(weight=w.half()), TypeError),
           (dict(weight=w[:7]), ValueError), (dict(bias=b.half()), TypeError),
           (dict(state=state[:, :2]), ValueError), (dict(x=x[0]), ValueError),
           (dict(lengths=torch.zeros(3, dtype=torch.int32, device=DEV)), ValueError),
           (dict(x=x.cpu()), ValueError), (dict(weight=w.cpu()), ValueError)]
    for change, error in bad:
        with pytest.raises(error):
            ops.causal_conv(**dict(dict(x=x, weight=w, bias=b, state=state), **change))
    with pytest.raises(ops._lib.LibscanError):  # width 5
        ops.causal_conv(x, torch.zeros(8, 5, device=DEV))
    with pytest.raises(ops._lib.LibscanError):  # in place
        ops.causal_conv(x, w, out=x)
    with pytest.raises(ops._lib.LibscanError):  # the state over itself
        ops.causal_conv(x, w, state=state, state_out=state)
    with pytest.raises(ValueError):
        ops.causal_conv_step(x[:, 0], state[:1], w)


def check_dweight(x, w, b, state, dy, lengths=None, silu=True):
    n = torch.tensor(lengths, dtype=torch.int32) if lengths is not None else None
    xd, wd, bd, sd, dyd = to(x, w, b, state, dy)
    announce("causal_conv_backward", tuple(x.shape), tuple(w.shape), x.dtype)
    got = ops.causal_conv_backward(dyd, xd, wd, bd, state=sd,
                                   lengths=n.to(DEV) if n is not None else None, silu=silu)[1]
    args = (dy.double(), *dbl(x, w, b, state), n, silu)
    want, mag = R.conv_back(*args)[1], R.conv_back(*args, absolute=True)[1]
    g, odd = got.cpu(), ~want.isfinite()
    assert torch.equal(g.isnan(), want.isnan()) and torch.equal(g[odd & ~want.isnan()].double(),
                                                                 want[odd & ~want.isnan()])
    R.assert_within(g.masked_fill(odd, 0), want.masked_fill(odd, 0),
                    mag.masked_fill(~mag.isfinite(), 0), 24 + x.shape[0] * x.shape[1], "dweight")


@pytest.mark.parametrize("width", [2, 3, 4])
@pytest.mark.parametrize("value", [float("nan"), float("inf")])
def test_conv_weights_that_a_last_input_does_not_meet(width, value):
    """The last input meets the last weight only; an infinity or NaN there is in no
    other weight's gradient."""
    for lengths in (None, [40, 17]):
        x, w, b, state, dy = inputs(2, 40, 37, width, F32, state=True)
        x[0, 39, 5] = value
        x[1, 16 if lengths else 39, 8] = value
        check_dweight(x, w, b, state, dy, lengths, silu=False)


@pytest.mark.parametrize("silu", [True, False])
def test_conv_weights_and_a_row_without_tokens(silu):
    """What the first state of an empty row holds is in no weight's gradient."""
    x, w, b, state, dy = inputs(3, 40, 37, 4, BF16, state=True)
    state[1] = float("nan")
    state[2] = float("inf")
    check_dweight(x, w, b, state, dy, [40, 0, -2], silu)


def test_step_refuses_slots_that_are_no_tensor():
    x, w, _, state, _ = to(*inputs(2, 1, 8, 4, F32, state=True))
    for slots in ([0, 1], 1, torch.zeros(2, dtype=torch.int64, device=DEV)):
        with pytest.raises(TypeError, match="slots"):
            ops.causal_conv_step(x[:, 0], state, w, slots=slots)
    for slots in (torch.zeros(2, dtype=torch.int32),
                  torch.zeros(3, dtype=torch.int32, device=DEV)):
        with pytest.raises(ValueError, match="slots"):
            ops.causal_conv_step(x[:, 0], state, w, slots=slots)
