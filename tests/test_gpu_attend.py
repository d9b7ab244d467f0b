"""Linear attention, its gradients and its single-token step against the
definition in 64 bits (attend_ref.py, where the bounds are derived)."""
import pytest
import torch

import attend_ref as R
from attend_ref import BF16, F16, F32
from gpu_util import announce
from paper_2505_15112_amd import ops

pytestmark = pytest.mark.gpu
DEV = "cuda"
NAMES = ("dq", "dk", "dv", "dlog_decay", "dstate")


def inputs(batch, steps, heads, groups, dk, dv, kind=F32, state=False, fixed=False, lengths=None,
           seed=0, rate=0.3):
    """On the CPU: kind for the activations, fp32 for the rest; and dy."""
    g = torch.Generator().manual_seed(seed)

    def normal(*s, dtype=kind):
        return torch.randn(*s, generator=g).to(dtype)

    shape = (heads,) if fixed else (batch, steps, heads)
    a = dict(q=normal(batch, steps, groups, dk), k=normal(batch, steps, groups, dk),
             v=normal(batch, steps, heads, dv),
             log_decay=-rate * torch.rand(*shape, generator=g) ** 3,
             state=normal(batch, heads, dk, dv, dtype=F32) if state else None,
             lengths=torch.tensor(lengths, dtype=torch.int32) if lengths is not None else None)
    return a, normal(batch, steps, heads, dv)


def dev(a):
    return {k: v.to(DEV) if isinstance(v, torch.Tensor) else v for k, v in a.items()}


def ref_args(a):
    return {k: v.double() if isinstance(v, torch.Tensor) and v.is_floating_point() else v
            for k, v in a.items()}


def steps_of(a, c):
    return c * (a["q"].shape[1] + a["q"].shape[3] + a["v"].shape[3] + 32) * 2.0**-24


def check_forward(a, **more):
    announce("linear_attention", tuple(a["q"].shape), tuple(a["v"].shape), a["q"].dtype)
    y, last = ops.linear_attention(**dev(a), with_state=True, **more)
    ref, mag = (R.attend(**ref_args(a), absolute=m, **more) for m in (False, True))
    r = steps_of(a, 4)
    R.assert_within(y, ref["y"], mag["y"], r + R.OPERANDS[y.dtype], "y")
    R.assert_within(last, ref["state"], mag["state"], r, "state")
    return y, last


def check_backward(a, dy, dstate_out=None, **more):
    announce("linear_attention_backward", tuple(a["q"].shape), tuple(a["v"].shape), a["q"].dtype)
    so = dstate_out.to(DEV) if dstate_out is not None else None
    got = ops.linear_attention_backward(dy.to(DEV), **dev(a), dstate_out=so, with_dstate=True,
                                        **more)
    grads = dict(dy=dy.double(), dstate_out=dstate_out.double() if so is not None else None, **more)
    ref, mag = (R.attend(**ref_args(a), **grads, absolute=m) for m in (False, True))
    r = steps_of(a, 8)
    for name, g in zip(NAMES, got):
        more_r = R.OPERANDS[g.dtype] if g.dtype != F32 else 0.0
        R.assert_within(g, ref[name], mag[name], r + more_r, name)
    return got


SIZES = [  # batch, steps, heads, groups, dk, dv
    (1, 1, 1, 1, 1, 1), (2, 1, 2, 1, 64, 64), (1, 15, 2, 2, 16, 33), (2, 63, 2, 2, 64, 128),
    (1, 64, 3, 3, 128, 64), (1, 65, 4, 2, 128, 128), (2, 130, 3, 1, 48, 80), (1, 97, 1, 1, 256, 256),
    (1, 129, 2, 2, 33, 200), (3, 31, 6, 3, 7, 5), (1, 333, 2, 2, 32, 32),
]


@pytest.mark.parametrize("size", SIZES)
@pytest.mark.parametrize("kind", [F32, F16, BF16])
def test_attention(size, kind):
    check_forward(inputs(*size, kind=kind, state=size[1] % 2 == 1, fixed=size[2] == 2)[0])


@pytest.mark.parametrize("size", SIZES)
@pytest.mark.parametrize("kind", [F32, F16, BF16])
def test_gradients(size, kind):
    a, dy = inputs(*size, kind=kind, state=size[1] % 2 == 1, fixed=size[2] == 2)
    so = torch.randn(*a["state"].shape, generator=torch.Generator().manual_seed(5)) \
        if size[2] == 3 and a["state"] is not None else None
    check_backward(a, dy, so)


def test_gradients_of_the_last_state_alone():
    a, dy = inputs(2, 70, 2, 1, 40, 24)
    so = torch.randn(2, 2, 40, 24, generator=torch.Generator().manual_seed(5))
    check_backward(a, dy, so)
    check_backward(a, torch.zeros_like(dy), so)


@pytest.mark.parametrize("scale", [1.0, -0.25, 0.0])
def test_scale(scale):
    a, dy = inputs(1, 70, 2, 1, 40, 24, kind=BF16, state=True)
    check_forward(a, scale=scale)
    check_backward(a, dy, scale=scale)


def test_gradients_against_differences():
    """fp32 gradients as central differences of the definition in 64 bits."""
    a, dy = inputs(1, 20, 2, 1, 8, 6, state=True)
    so = torch.randn(1, 2, 8, 6, generator=torch.Generator().manual_seed(5))
    got = dict(zip(NAMES, ops.linear_attention_backward(dy.to(DEV), **dev(a),
                                                        dstate_out=so.to(DEV))))
    g = torch.Generator().manual_seed(9)
    for name, key in (("dq", "q"), ("dk", "k"), ("dv", "v"), ("dlog_decay", "log_decay"),
                      ("dstate", "state")):
        at = ref_args(a)
        way = torch.randn(at[key].shape, generator=g, dtype=torch.double)

        def value(eps):
            out = R.attend(**dict(at, **{key: at[key] + eps * way}))
            return (out["y"] * dy.double()).sum() + (out["state"] * so.double()).sum()

        eps = 1e-5
        want = (value(eps) - value(-eps)) / (2 * eps)
        # the differences' own error is eps^2 times third derivatives, about 1e-10 of the
        # values here; the kernel's is that of 20 x 8 x 6 fp32 sums
        have = (got[name].cpu().double() * way).sum()
        size = (got[name].cpu().double() * way).abs().sum()
        assert abs(have - want) <= 1e-5 * size + 1e-6, name


@pytest.mark.parametrize("kind", [F32, BF16])
@pytest.mark.parametrize("dims", [(64, 64), (40, 130)])
def test_ragged_rows_do_not_read_past_their_tokens(kind, dims):
    """Lengths of 0, 1, a chunk's edges and beyond the steps; NaN past the tokens."""
    lengths = [0, 1, 64, 65, 33, 140, 200, -3]
    a, dy = inputs(8, 140, 2, 1, *dims, kind=kind, state=True, lengths=lengths)
    clean = {k: v.clone() if isinstance(v, torch.Tensor) else v for k, v in a.items()}
    dy_clean = dy.clone()
    for b, n in enumerate(lengths):
        n = max(n, 0)
        for k in ("q", "k", "v", "log_decay"):
            a[k][b, n:] = float("nan")
            clean[k][b, n:] = 0
        dy[b, n:] = float("inf")
        dy_clean[b, n:] = 0
    y, last = check_forward(clean)
    y2, last2 = ops.linear_attention(**dev(a), with_state=True)
    assert torch.equal(y, y2) and torch.equal(last, last2)
    for b, n in enumerate(lengths):
        assert not y2[b, max(n, 0):].any()
    assert torch.equal(last2[0].cpu(), a["state"][0])
    so = torch.randn(*a["state"].shape, generator=torch.Generator().manual_seed(3))
    want = check_backward(clean, dy_clean, so)
    got = ops.linear_attention_backward(dy.to(DEV), **dev(a), dstate_out=so.to(DEV))
    for name, g, w in zip(NAMES, got, want):
        assert torch.equal(g, w), name
    assert torch.equal(got[4][0].cpu(), so[0])


@pytest.mark.parametrize("kind", [F32, F16, BF16])
@pytest.mark.parametrize("dims", [(32, 16), (100, 130)])
def test_ragged_rows_in_pieces(kind, dims):
    """Rows long enough to be cut: lengths that end in every piece and at their edges."""
    lengths = [640, 0, 64, 129, 320, 577]
    a, dy = inputs(6, 640, 2, 1, *dims, kind=kind, state=True, lengths=lengths, rate=0.05)
    so = torch.randn(*a["state"].shape, generator=torch.Generator().manual_seed(3))
    check_forward(a)
    check_backward(a, dy, so)


def test_rows_beyond_32_bit_offsets():
    """2.4e9 elements: what lies behind 2^31 of them against a call of its own."""
    steps, heads, d = 150000, 64, 128
    if torch.cuda.mem_get_info()[0] < 90 << 30:
        pytest.skip("needs 70 GB")
    g = torch.Generator(device=DEV).manual_seed(1)
    q, k, v, dy = (torch.empty(2, steps, heads, d, dtype=BF16, device=DEV).normal_(generator=g)
                   for _ in range(4))
    decay = torch.full((heads,), -0.02, device=DEV)
    announce("linear_attention", tuple(q.shape))
    y, last = ops.linear_attention(q, k, v, decay, with_state=True)
    one, end = ops.linear_attention(q[1:], k[1:], v[1:], decay, with_state=True)
    # rows may be cut into other pieces: sums in another order, one unit of bfloat16
    assert (y[1, -500:].float() - one[0, -500:].float()).abs().max() <= 2.0**-7 * one.abs().max()
    assert (last[1] - end[0]).abs().max() <= 1e-5 * end.abs().max()
    del y, one
    announce("linear_attention_backward", tuple(q.shape))
    grads = ops.linear_attention_backward(dy, q, k, v, decay)
    part = ops.linear_attention_backward(dy[1:], q[1:], k[1:], v[1:], decay)
    for x, w in zip(grads[:3], part[:3]):
        assert (x[1, -500:].float() - w[0, -500:].float()).abs().max() <= 2.0**-7 * w.abs().max()


def test_strided_operands():
    """q, k, v as parts of one projection, decays and dy as slices, all unaligned."""
    a, dy = inputs(2, 90, 4, 2, 40, 24, kind=BF16)
    d = dev(a)
    parts = torch.zeros(2, 90, 1 + 2 * 80 + 96, dtype=BF16, device=DEV)
    q, k, v = parts[..., 1:].split((80, 80, 96), -1)
    q, k, v = q.unflatten(-1, (2, 40)), k.unflatten(-1, (2, 40)), v.unflatten(-1, (4, 24))
    q.copy_(d["q"]), k.copy_(d["k"]), v.copy_(d["v"])
    g = torch.zeros(2, 90, 7, device=DEV)[..., 2:6].copy_(d["log_decay"])
    turned = torch.zeros(90, 4, 2, 25, dtype=BF16, device=DEV).permute(2, 0, 1, 3)[..., :24]
    turned.copy_(dy.to(DEV))
    s = dict(d, q=q, k=k, v=v, log_decay=g)
    for x, w in zip(ops.linear_attention(**s, with_state=True),
                    ops.linear_attention(**d, with_state=True)):
        assert torch.equal(x, w)
    for x, w in zip(ops.linear_attention_backward(turned, **s)[:4],
                    ops.linear_attention_backward(dy.to(DEV), **d)[:4]):
        assert torch.equal(x, w)


@pytest.mark.parametrize("kind", [F32, BF16])
def test_decays_that_clear_keep_and_grow(kind):
    """Decays of -infinity in the middle and at the edges of chunks, of 0, very strong
    ones, and some that grow."""
    a, dy = inputs(1, 200, 2, 1, 32, 48, kind=kind, state=True)
    g = a["log_decay"]
    g[:, [0, 5, 63, 64, 100, 199], 0] = -float("inf")
    g[:, 20:40] = 0
    g[:, 110:150] = -50.0
    g[:, 160:170] = 0.2
    check_forward(a)
    got = check_backward(a, dy)
    assert not got[3][0, [0, 5, 63, 64, 100, 199], 0].any()
    # what a cleared head gives does not depend on what came before
    b = {k: v.clone() if isinstance(v, torch.Tensor) else v for k, v in a.items()}
    b["v"][:, :100, 0] *= 3
    y, last = ops.linear_attention(**dev(a), with_state=True)
    y2, last2 = ops.linear_attention(**dev(b), with_state=True)
    assert torch.equal(y[:, 100:, 0], y2[:, 100:, 0]) and torch.equal(last[:, 0], last2[:, 0])


@pytest.mark.parametrize("kind", [F32, F16, BF16])
@pytest.mark.parametrize("bad", [float("inf"), float("nan")])
def test_what_comes_later_does_not_reach_back(kind, bad):
    """An infinity or a NaN at token 75 leaves the tokens before it as they were, and
    gradients of outputs before it those of the tokens behind it."""
    a, dy = inputs(1, 160, 2, 2, 40, 72, kind=kind)
    want, _ = ops.linear_attention(**dev(a))
    for key in ("q", "k", "v", "log_decay"):
        b = {k: v.clone() if isinstance(v, torch.Tensor) else v for k, v in a.items()}
        if key == "log_decay":
            b[key][0, 75, 0] = bad
        else:
            b[key][0, 75, 0, 3] = bad
        announce("linear_attention, bad", key, kind)
        y, _ = ops.linear_attention(**dev(b))
        assert torch.equal(y[:, :75], want[:, :75]), key
        assert torch.equal(y[:, :, 1], want[:, :, 1]), key  # another head
        at = y[0, 75, 0]
        if key == "v":
            assert not torch.isfinite(at[3]) and torch.isfinite(at[4]), key
        else:
            assert key == "log_decay" and bad > 0 or not torch.isfinite(at).any(), key
        if key != "q":
            assert not torch.isfinite(y[0, 100, 0]).all()
    grads = ops.linear_attention_backward(dy.to(DEV), **dev(a))
    dy[0, 75, 0, 3] = bad
    again = ops.linear_attention_backward(dy.to(DEV), **dev(a))
    for name, g, w in zip(NAMES[1:3], again[1:3], grads[1:3]):
        assert torch.equal(g[:, 76:], w[:, 76:]), name
        assert not torch.isfinite(g[0, 75, 0]).all(), name
    assert torch.equal(again[0][:, :75], grads[0][:, :75])
    assert torch.equal(again[0][:, 76:], grads[0][:, 76:])
    assert torch.equal(again[3][:, 76:], grads[3][:, 76:])


def test_long_rows_keep_their_precision():
    """A long row with slow decays, against the same row in two halves through the state,
    and its decays' gradients against the definition by chunks in 64 bits."""
    a, dy = inputs(1, 5000, 2, 2, 64, 64, rate=0.01)
    d, half = dev(a), 2345
    y, last = ops.linear_attention(**d, with_state=True)
    cut = [{k: v[:, s] if k in ("q", "k", "v", "log_decay") else v for k, v in d.items()}
           for s in (slice(None, half), slice(half, None))]
    y0, mid = ops.linear_attention(**cut[0], with_state=True)
    y1, end = ops.linear_attention(**dict(cut[1], state=mid), with_state=True)
    # both are within some 2^-20 of the exact sums of terms of the size of the largest
    big = y.abs().max()
    assert (torch.cat((y0, y1), 1) - y).abs().max() <= 2.0**-18 * big
    assert (end - last).abs().max() <= 2.0**-18 * last.abs().max()
    got = ops.linear_attention_backward(dy.to(DEV), **d)
    at = {k: d[k].double().requires_grad_() for k in ("q", "k", "v", "log_decay")}
    c = at["log_decay"].cumsum(1)
    over = (c[:, :, None] - c[:, None]).masked_fill(
        torch.ones(5000, 5000, dtype=torch.bool, device=DEV).triu(1)[None, :, :, None],
        -float("inf"))
    for h in range(2):
        p = torch.exp(over[0, :, :, h]) * (at["q"][0, :, h] @ at["k"][0, :, h].t())
        out = (p @ at["v"][0, :, h]) / 8
        want = torch.autograd.grad((out * dy[0, :, h].to(DEV).double()).sum(), list(at.values()),
                                   retain_graph=True)
        for name, g, w in zip(NAMES, got, want):
            g, w = g[0, :, h].double(), w[0, :, h]
            # 2-norm: fp32 sums over some hundred tokens
            assert (g - w).norm() <= 1e-5 * w.norm(), name


def test_the_same_call_twice_gives_the_same_bits():
    a, dy = inputs(2, 300, 4, 2, 64, 64, kind=BF16)
    d = dev(a)
    first = ops.linear_attention(**d, with_state=True) + ops.linear_attention_backward(
        dy.to(DEV), **d)[:4]
    for _ in range(3):
        again = ops.linear_attention(**d, with_state=True) + ops.linear_attention_backward(
            dy.to(DEV), **d)[:4]
        assert all(torch.equal(x, w) for x, w in zip(again, first))


def test_given_outputs_and_scratch():
    """The caller's outputs, and scratch of just the size that is asked for, whatever it holds."""
    a, dy = inputs(2, 300, 4, 2, 64, 96, kind=BF16, state=True, fixed=True)
    d, dy = dev(a), dy.to(DEV)
    y, last = ops.linear_attention(**d, with_state=True)
    grads = ops.linear_attention_backward(dy, **d, dstate_out=last)
    p = ops._args.attend(d["q"], d["k"], d["v"], d["log_decay"], d["state"], None, None, False)
    front, back = ops._sizes("linear_attention_bytes", p, 2)
    assert front > 0 and back > 0
    for fill in (0xff, 0x7f, 0):
        out, end = torch.full_like(y, 3.0), torch.full_like(last, 3.0)
        got = ops.linear_attention(**d, out=out, state_out=end, scratch_buf=torch.full(
            (front,), fill, dtype=torch.uint8, device=DEV))
        assert got[0] is out and got[1] is end
        assert torch.equal(out, y) and torch.equal(end, last)
        again = ops.linear_attention_backward(dy, **d, dstate_out=last, scratch_buf=torch.full(
            (back,), fill, dtype=torch.uint8, device=DEV))
        assert all(torch.equal(g, w) for g, w in zip(again, grads))
    with pytest.raises(ops._lib.LibscanError):
        ops.linear_attention(**d, scratch_buf=torch.empty(front - 1, dtype=torch.uint8, device=DEV))


# ---------------------------------------------------------------- single tokens

@pytest.mark.parametrize("size", [(1, 1, 1, 1, 1), (3, 4, 2, 64, 64), (2, 3, 3, 128, 128),
                                  (5, 2, 1, 33, 49), (1, 2, 2, 256, 256), (130, 1, 1, 16, 7)])
@pytest.mark.parametrize("kind", [F32, F16, BF16])
@pytest.mark.parametrize("fixed", [True, False])
def test_step(size, kind, fixed):
    batch, heads, groups, dk, dv = size
    a, _ = inputs(batch, 1, heads, groups, dk, dv, kind=kind, state=True, fixed=fixed)
    ref, mag = (R.attend(**ref_args(a), absolute=m) for m in (False, True))
    d = dev(a)
    pool = torch.full((batch + 2, heads, dk, dv), 7.0, device=DEV)
    slots = torch.randperm(batch + 2, generator=torch.Generator().manual_seed(1))[:batch]
    pool[slots.to(DEV)] = d["state"]
    announce("linear_attention_step", size, kind)
    g = d["log_decay"] if fixed else d["log_decay"][:, 0]
    y = ops.linear_attention_step(d["q"][:, 0], d["k"][:, 0], d["v"][:, 0], g, pool,
                                  slots=slots.to(torch.int32).to(DEV))
    r = steps_of(a, 4)
    R.assert_within(y, ref["y"][:, 0], mag["y"][:, 0], r, "y")
    R.assert_within(pool[slots.to(DEV)], ref["state"], mag["state"], 4 * 2.0**-24, "state")
    rest = torch.ones(batch + 2, dtype=torch.bool)
    rest[slots] = False
    assert bool((pool[rest.to(DEV)] == 7.0).all())


def test_step_rows_without_a_state():
    a, _ = inputs(4, 1, 2, 1, 40, 24, kind=BF16)
    d = dev(a)
    pool = torch.randn(3, 2, 40, 24, device=DEV)
    was = pool.clone()
    slots = torch.tensor([-1, 2, 3, 1 << 30], dtype=torch.int32, device=DEV)
    y = ops.linear_attention_step(d["q"][:, 0], d["k"][:, 0], d["v"][:, 0], d["log_decay"][:, 0],
                                  pool, slots=slots)
    assert not y[[0, 2, 3]].any() and bool(y[1].any())
    assert torch.equal(pool[:2], was[:2]) and not torch.equal(pool[2], was[2])


def test_step_of_a_pool_beyond_32_bit_offsets():
    n, heads, dk, dv = 40000, 14, 64, 64  # 2.3e9 elements
    if torch.cuda.mem_get_info()[0] < 12 << 30:
        pytest.skip("needs 9.2 GB")
    pool = torch.zeros(n, heads, dk, dv, device=DEV)
    a, _ = inputs(2, 1, heads, heads, dk, dv, state=True)
    d = dev(a)
    slots = torch.tensor([n - 1, 39000], dtype=torch.int32, device=DEV)
    pool[slots.long()] = d["state"]
    y = ops.linear_attention_step(d["q"][:, 0], d["k"][:, 0], d["v"][:, 0], d["log_decay"][:, 0],
                                  pool, slots=slots)
    small = d["state"].clone()
    want = ops.linear_attention_step(d["q"][:, 0], d["k"][:, 0], d["v"][:, 0],
                                     d["log_decay"][:, 0], small)
    assert torch.equal(y, want) and torch.equal(pool[slots.long()], small)
    assert not pool[:30000].any()


def test_steps_follow_the_prompt():
    """A prompt, then tokens one by one, against all of it at once (fp32)."""
    a, _ = inputs(2, 90, 4, 2, 64, 48)
    d = dev(a)
    want, last = ops.linear_attention(**d, with_state=True)
    cut = {k: v[:, :71] if k in ("q", "k", "v", "log_decay") else v for k, v in d.items()}
    _, state = ops.linear_attention(**cut, with_state=True)
    for t in range(71, 90):
        y = ops.linear_attention_step(d["q"][:, t], d["k"][:, t], d["v"][:, t],
                                      d["log_decay"][:, t], state)
        assert (y - want[:, t]).abs().max() <= 1e-5 * want.abs().max()
    assert (state - last).abs().max() <= 1e-5 * last.abs().max()


# ---------------------------------------------------------------- streams, graphs

def test_a_captured_graph_replays():
    """Forward, gradients and a step in one graph, replayed over new inputs with eager
    work between, against the eager results."""
    a, dy = inputs(2, 150, 4, 2, 64, 64, kind=BF16, state=True)
    d, dy = dev(a), dy.to(DEV)
    pool = d["state"].clone()

    def work():
        y, last = ops.linear_attention(**d, with_state=True)
        grads = ops.linear_attention_backward(dy, **d, dstate_out=last)
        one = ops.linear_attention_step(d["q"][:, 0], d["k"][:, 0], d["v"][:, 0],
                                        d["log_decay"][:, 0], pool)
        return (y, last, *grads, one, pool.clone())

    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    with torch.cuda.stream(side):
        work()
    torch.cuda.current_stream().wait_stream(side)
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        out = work()
    for seed in range(3):
        b, dy2 = inputs(2, 150, 4, 2, 64, 64, kind=BF16, state=True, seed=10 + seed)
        for k in ("q", "k", "v", "log_decay", "state"):
            d[k].copy_(b[k])
        dy.copy_(dy2)
        pool.copy_(d["state"])
        want = work()
        pool.copy_(d["state"])
        torch.cuda.synchronize()
        graph.replay()
        torch.cuda.synchronize()
        for x, w in zip(out, want):
            assert torch.equal(x, w)


def test_on_another_stream():
    a, dy = inputs(2, 150, 4, 2, 64, 64, kind=BF16)
    d = dev(a)
    want, _ = ops.linear_attention(**d)
    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    with torch.cuda.stream(side):
        y, _ = ops.linear_attention(**d)
    side.synchronize()
    assert torch.equal(y, want)


# ---------------------------------------------------------------- arguments

def test_refusals():
    a, dy = inputs(2, 9, 4, 2, 8, 6)
    d, dy = dev(a), dy.to(DEV)
    for bad, error, what in (
            (dict(k=d["k"][:, :, :1]), ValueError, "k"), (dict(v=d["v"][:1]), ValueError, "v"),
            (dict(v=d["v"][:, :, :3]), ValueError, "heads"), (dict(q=d["q"][0]), ValueError, "q"),
            (dict(k=d["k"].half()), TypeError, "k"), (dict(v=None), TypeError, "v"),
            (dict(log_decay=d["log_decay"].half()), TypeError, "log_decay"),
            (dict(log_decay=d["log_decay"][:, :3]), ValueError, "log_decay"),
            (dict(q=d["q"].transpose(2, 3)), ValueError, "q|k"),
            (dict(state=torch.zeros(2, 4, 6, 8, device=DEV)), ValueError, "state"),
            (dict(lengths=torch.zeros(3, dtype=torch.int32, device=DEV)), ValueError, "lengths"),
            (dict(lengths=torch.zeros(2, dtype=torch.int64, device=DEV)), TypeError, "lengths"),
            (dict(k=d["k"].cpu()), ValueError, "k")):
        with pytest.raises(error, match=what):
            ops.linear_attention(**dict(d, **bad))
        with pytest.raises(error, match=what):
            ops.linear_attention_backward(dy, **dict(d, **bad))
    with pytest.raises(TypeError):
        ops.linear_attention(**d, scale="large")
    with pytest.raises(ValueError, match="out"):
        ops.linear_attention(**d, out=torch.zeros(2, 9, 4, 5, device=DEV))
    with pytest.raises(ops._lib.LibscanError):
        ops.linear_attention(**d, out=d["v"])
    with pytest.raises(ops._lib.LibscanError):
        ops.linear_attention(**dev(inputs(1, 2, 1, 1, 257, 8)[0]))
    with pytest.raises(ValueError, match="dy"):
        ops.linear_attention_backward(dy[:, :8], **d)
    small = torch.zeros(16, dtype=torch.uint8, device=DEV)
    with pytest.raises(ops._lib.LibscanError):
        ops.linear_attention_backward(dy, **d, scratch_buf=small)
    one = (d["q"][:, 0], d["k"][:, 0], d["v"][:, 0], d["log_decay"][:, 0])
    pool = torch.zeros(2, 4, 8, 6, device=DEV)
    with pytest.raises(ValueError, match="states"):
        ops.linear_attention_step(*one, pool[:1])
    with pytest.raises(ValueError, match="states"):
        ops.linear_attention_step(*one, pool.transpose(2, 3).contiguous())
    with pytest.raises(TypeError, match="slots"):
        ops.linear_attention_step(*one, pool, slots=torch.zeros(2, device=DEV))


def test_nothing_to_do():
    for size in ((0, 9, 2, 1, 8, 6), (2, 0, 2, 1, 8, 6), (2, 9, 0, 1, 8, 6)):
        a, dy = inputs(*size, state=True)
        y, last = ops.linear_attention(**dev(a), with_state=True)
        assert y.numel() == 0 and torch.equal(last.cpu(), a["state"])
        got = ops.linear_attention_backward(dy.to(DEV), **dev(a),
                                            dstate_out=a["state"].to(DEV))
        assert torch.equal(got[4].cpu(), a["state"])
        assert all(g.shape == d.shape for g, d in zip(got, (a["q"], a["k"], a["v"])))


def test_no_graph_is_said_so():
    a, dy = inputs(1, 9, 2, 1, 8, 6)
    d = dev(a)
    with pytest.warns(UserWarning, match="linear_attention_backward"):
        ops.linear_attention(**dict(d, log_decay=d["log_decay"].clone().requires_grad_()))
    with pytest.warns(UserWarning, match="no gradients"):
        ops.linear_attention_step(d["q"][:, 0].clone().requires_grad_(), d["k"][:, 0],
                                  d["v"][:, 0], d["log_decay"][:, 0],
                                  torch.zeros(1, 2, 8, 6, device=DEV))
