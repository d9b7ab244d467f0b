"""The selective scan, its gradients and its single-token step against the
definition in 64 bits (lm_ref.py, where the bounds are derived)."""
import pytest
import torch

import lm_ref as R
from gpu_util import announce
from paper_2505_15112_amd import ops

pytestmark = pytest.mark.gpu
DEV = "cuda"
F32, F16, BF16 = torch.float32, torch.float16, torch.bfloat16


def inputs(batch, steps, dim, n, groups=1, kind=F32, gate=True, skip=True, bias=True, state=False,
           lengths=None, seed=0):
    """On the CPU: kind for the activations, fp32 for the rest."""
    g = torch.Generator().manual_seed(seed)

    def normal(*s, scale=1.0, dtype=kind):
        return (torch.randn(*s, generator=g) * scale).to(dtype)

    a = dict(x=normal(batch, steps, dim), dt=normal(batch, steps, dim, scale=0.5),
             A=-(torch.rand(dim, n, generator=g) * n + 0.2),
             B=normal(batch, steps, groups, n), C=normal(batch, steps, groups, n),
             D=normal(dim, dtype=F32) if skip else None,
             z=normal(batch, steps, dim) if gate else None,
             dt_bias=normal(dim, dtype=F32) - 2.0 if bias else None,
             state=normal(batch, dim, n, dtype=F32) if state else None,
             lengths=torch.tensor(lengths, dtype=torch.int32) if lengths is not None else None)
    dy = normal(batch, steps, dim)
    return a, dy


def dev(a):
    return {k: v.to(DEV) if isinstance(v, torch.Tensor) else v for k, v in a.items()}


def ref_args(a):
    return {k: v.double() if isinstance(v, torch.Tensor) and v.is_floating_point() else v
            for k, v in a.items()}


NAMES = ("dx", "ddt", "dA", "dB", "dC", "dD", "dz", "ddt_bias", "dstate")


def check_forward(a, softplus=True):
    batch, steps, dim = a["x"].shape
    announce("selective_scan", tuple(a["x"].shape), tuple(a["B"].shape), a["x"].dtype)
    y, last, _ = ops.selective_scan(**dev(a), softplus=softplus, with_state=True)
    ref = R.scan(**ref_args(a), softplus_on=softplus)
    mag = R.scan(**ref_args(a), softplus_on=softplus, absolute=True)
    c = 4 * (steps + 32)
    R.assert_within(y, ref["y"], mag["y"], c, "y")
    R.assert_within(last, ref["state"], mag["state"], c, "state")


def check_backward(a, dy, dstate_out=None, softplus=True):
    batch, steps, dim = a["x"].shape
    d = dev(a)
    announce("selective_scan_backward", tuple(a["x"].shape), tuple(a["B"].shape), a["x"].dtype)
    _, _, kept = ops.selective_scan(**d, softplus=softplus, with_checkpoints=True)
    so = dstate_out.to(DEV) if dstate_out is not None else None
    got = ops.selective_scan_backward(dy.to(DEV), kept, **d, softplus=softplus, dstate_out=so,
                                      with_dstate=True)
    more = dict(dy=dy.double(), dstate_out=dstate_out.double() if so is not None else None,
                softplus_on=softplus)
    ref = R.scan(**ref_args(a), **more)
    mag = R.scan(**ref_args(a), **more, absolute=True)
    c = 8 * (steps + 32)
    for name, g in zip(NAMES, got):
        if g is None:
            assert a[{"dD": "D", "dz": "z", "ddt_bias": "dt_bias"}[name]] is None
            continue
        extra = dim + batch * steps if name in ("dA", "dB", "dC", "dD", "ddt_bias") else 0
        R.assert_within(g, ref[name], mag[name], c + extra, name)
    return got


SIZES = [  # batch, steps, dim, n, groups
    (1, 1, 1, 1, 1), (1, 1, 64, 16, 1), (2, 15, 16, 16, 1), (1, 16, 17, 5, 1), (2, 17, 130, 16, 2),
    (1, 33, 66, 8, 3), (3, 70, 100, 17, 2), (1, 65, 40, 33, 1), (2, 31, 20, 64, 4),
    (1, 300, 24, 16, 1), (130, 5, 128, 16, 1),
]


@pytest.mark.parametrize("size", SIZES)
@pytest.mark.parametrize("kind", [F32, F16, BF16])
def test_scan(size, kind):
    check_forward(inputs(*size, kind=kind, state=size[1] % 2 == 1)[0])


@pytest.mark.parametrize("size", SIZES)
@pytest.mark.parametrize("kind", [F32, F16, BF16])
def test_scan_gradients(size, kind):
    a, dy = inputs(*size, kind=kind, state=size[1] % 2 == 1)
    check_backward(a, dy)


@pytest.mark.parametrize("gate", [True, False])
@pytest.mark.parametrize("skip,bias", [(False, False), (True, False), (False, True)])
@pytest.mark.parametrize("softplus", [True, False])
def test_scan_without_parts(gate, skip, bias, softplus):
    a, dy = inputs(2, 20, 70, 16, kind=BF16, gate=gate, skip=skip, bias=bias)
    if not softplus:  # step sizes must not be negative: the state would grow by e^32 a step
        a["dt"] = a["dt"].abs() * 0.2
        a["dt_bias"] = a["dt_bias"].abs() if bias else None
    check_forward(a, softplus)
    check_backward(a, dy, softplus=softplus)


@pytest.mark.parametrize("dim", [40, 4500])  # both lane layouts at n = 16
def test_scan_ragged_rows_do_not_read_past_their_tokens(dim):
    """Lengths of 0, 1, a block's edges and beyond the steps; NaN past the tokens."""
    lengths = [0, 1, 16, 33, 47, 60, -3]
    a, dy = inputs(7, 47, dim, 16, groups=2, kind=BF16, state=True, lengths=lengths)
    clean = {k: v.clone() if isinstance(v, torch.Tensor) else v for k, v in a.items()}
    dy_clean = dy.clone()
    for b, n in enumerate(lengths):
        n = max(n, 0)
        for k in ("x", "dt", "z", "B", "C"):
            a[k][b, n:] = float("nan")
            clean[k][b, n:] = 0
        dy[b, n:] = float("inf")
        dy_clean[b, n:] = 0
    y, last, kept = ops.selective_scan(**dev(a), with_state=True, with_checkpoints=True)
    y2, last2, kept2 = ops.selective_scan(**dev(clean), with_state=True, with_checkpoints=True)
    assert torch.equal(y, y2) and torch.equal(last, last2)
    for b, n in enumerate(lengths):
        assert not y[b, max(n, 0):].any()
    assert torch.equal(last[0].cpu(), a["state"][0])
    so = torch.randn(7, dim, 16, generator=torch.Generator().manual_seed(3))
    got = ops.selective_scan_backward(dy.to(DEV), kept, **dev(a), dstate_out=so.to(DEV))
    want = ops.selective_scan_backward(dy_clean.to(DEV), kept2, **dev(clean), dstate_out=so.to(DEV))
    for name, g, w in zip(NAMES, got, want):
        assert torch.equal(g, w), name
    assert torch.equal(got[8][0].cpu(), so[0])
    if dim < 100:
        check_forward(clean)
        check_backward(clean, dy_clean, dstate_out=so)


@pytest.mark.parametrize("n,groups", [(1, 1), (8, 1), (16, 2), (20, 1), (64, 2)])
@pytest.mark.parametrize("kind", [F32, BF16])
def test_scan_long_ragged_rows(n, groups, kind):
    """Rows cut into chunks: lengths at, around and between the cuts, on strided
    inputs with NaN behind the tokens."""
    lengths = [0, 5, 32, 33, 64, 95, 150, 200]
    a, dy = inputs(8, 150, 130, n, groups, kind=kind, state=True, lengths=lengths)
    for b, count in enumerate(lengths):
        for k in ("x", "dt", "z", "B", "C"):
            a[k][b, count:] = float("nan")
        dy[b, count:] = float("nan")
    check_forward(a)
    check_backward(a, dy, dstate_out=torch.randn(8, 130, n))
    d = dev(a)
    y = ops.selective_scan(**d)[0]
    both = torch.full((8, 150, 3 * 130 + 1), float("nan"), dtype=kind, device=DEV)
    for i, k in enumerate(("x", "dt", "z")):
        both[:, :, 1 + i * 130:1 + (i + 1) * 130] = d[k]
        d[k] = both[:, :, 1 + i * 130:1 + (i + 1) * 130]
    assert torch.equal(ops.selective_scan(**d)[0], y)


@pytest.mark.parametrize("n,groups", [(5, 1), (16, 2), (20, 1), (64, 1)])
def test_scan_rows_in_chunks(n, groups):
    """Few channels and many steps: the rows are cut into chunks, forward and
    backward.  Lengths that end chunks early, leave some empty, or are 0; the
    same without lengths, with a first state and a gradient of the last one."""
    steps, dim = 1537, 100
    lengths = [1537, 0, 700, 33]
    for case in (lengths, None):
        rows = 4 if case else 1
        a, dy = inputs(rows, steps, dim, n, groups, kind=F32, state=True, lengths=case)
        d = dev(a)
        p = ops._args.ssm(*(d[k] for k in ("x", "dt", "A", "B", "C", "D", "z", "dt_bias", "state",
                                           "lengths")), True, False)
        assert ops._sizes("selective_scan_bytes", p, 3)[1] > 0     # it is the chunks that run
        for b, count in enumerate(case or []):
            for k in ("x", "dt", "z", "B", "C"):
                a[k][b, count:] = float("nan")
            dy[b, count:] = float("nan")
        check_forward(a)
        check_backward(a, dy, dstate_out=torch.randn(rows, dim, n))


def test_scan_wide_layout():
    """Enough channels for a quad of lanes per channel, in both directions."""
    a, dy = inputs(2, 35, 8200, 16, groups=2, kind=BF16, state=True)
    check_forward(a)
    check_backward(a, dy, dstate_out=torch.randn(2, 8200, 16))


@pytest.mark.parametrize("batch,dim", [(1, 48), (4, 4096)])
def test_scan_many_steps(batch, dim):
    a, dy = inputs(batch, 700, dim, 16, kind=F32, state=True)
    if dim > 100:  # the definition on some channels, each of which stands by itself
        y, last, _ = ops.selective_scan(**dev(a), with_state=True)
        some = torch.arange(0, dim, 171)
        part = {k: (v[..., some] if k in ("x", "dt", "z", "D", "dt_bias") else
                    v[some] if k == "A" else v[:, some] if k == "state" else v)
                if v is not None else None for k, v in a.items()}
        ref, mag = R.scan(**ref_args(part)), R.scan(**ref_args(part), absolute=True)
        R.assert_within(y[..., some.to(DEV)], ref["y"], mag["y"], 4 * 732, "y")
        R.assert_within(last[:, some.to(DEV)], ref["state"], mag["state"], 4 * 732, "state")
    else:
        check_forward(a)
        check_backward(a, dy)


def test_scan_in_pieces_is_the_scan():
    """A row continued from the state of its first part: the same to the bounds."""
    a, _ = inputs(2, 90, 70, 16, kind=F32, state=True)
    d = dev(a)
    whole, last, _ = ops.selective_scan(**d, with_state=True)
    head = {k: v[:, :37] if k in ("x", "dt", "z", "B", "C") else v for k, v in d.items()}
    tail = {k: v[:, 37:] if k in ("x", "dt", "z", "B", "C") else v for k, v in d.items()}
    y0, s0, _ = ops.selective_scan(**head, with_state=True)
    y1, s1, _ = ops.selective_scan(**dict(tail, state=s0), with_state=True)
    mag = R.scan(**ref_args(a), absolute=True)
    c = 8 * 122
    R.assert_within(torch.cat((y0, y1), 1), whole.double().cpu(), mag["y"], c, "y")
    R.assert_within(s1, last.double().cpu(), mag["state"], c, "state")


def test_scan_strided_inputs_and_odd_alignment():
    """Slices of wider tensors, time before batch, addresses off 16 bytes."""
    a, dy = inputs(3, 21, 33, 9, groups=3, kind=BF16)
    d = dev(a)
    want = ops.selective_scan(**d, with_state=True, with_checkpoints=True)
    wide = {}
    for k in ("x", "dt", "z"):
        big = torch.full((21, 3, 2 * 33 + 1), float("nan"), dtype=BF16, device=DEV)
        v = big[:, :, 33:66].transpose(0, 1)
        v.copy_(d[k])
        wide[k] = v
    both = torch.full((3, 21, 1 + 2 * 27), float("nan"), dtype=BF16, device=DEV)
    wide["B"] = both[:, :, 1:28].unflatten(2, (3, 9))
    wide["C"] = both[:, :, 28:].unflatten(2, (3, 9))
    wide["B"].copy_(d["B"])
    wide["C"].copy_(d["C"])
    got = ops.selective_scan(**dict(d, **wide), with_state=True, with_checkpoints=True)
    assert all(torch.equal(g, w) for g, w in zip(got, want))
    dyw = torch.zeros(21, 3, 40, dtype=BF16, device=DEV)[:, :, 3:36].transpose(0, 1)
    dyw.copy_(dy.to(DEV))
    g0 = ops.selective_scan_backward(dy.to(DEV), want[2], **d)
    g1 = ops.selective_scan_backward(dyw, want[2], **dict(d, **wide))
    for name, p, q in zip(NAMES, g0, g1):
        assert (p is None and q is None) or torch.equal(p, q), name


def test_scan_broadcast_inputs():
    """One row's inputs for the whole batch (stride 0)."""
    a, _ = inputs(1, 18, 50, 16, kind=F32)
    d = dev(a)
    y, last, _ = ops.selective_scan(**d, with_state=True)
    e = {k: v.expand(4, *v.shape[1:]) if k in ("x", "dt", "z", "B", "C") else v
         for k, v in d.items()}
    ye, le, _ = ops.selective_scan(**e, with_state=True)
    assert torch.equal(ye, y.expand(4, -1, -1)) and torch.equal(le, last.expand(4, -1, -1))


@pytest.mark.parametrize("batch,steps,dim", [(0, 5, 8), (2, 0, 8), (2, 5, 0)])
def test_scan_empty(batch, steps, dim):
    a, dy = inputs(batch, steps, dim, 4, kind=F32, state=True)
    d = dev(a)
    y, last, kept = ops.selective_scan(**d, with_state=True, with_checkpoints=True)
    assert y.shape == (batch, steps, dim)
    if steps == 0:
        assert torch.equal(last, d["state"])
    so = torch.randn(batch, dim, 4, device=DEV)
    got = ops.selective_scan_backward(dy.to(DEV), kept, **d, dstate_out=so)
    for name, g in zip(NAMES[:-1], got):
        assert not g.any(), name
    if steps == 0:
        assert torch.equal(got[8], so)


def test_scan_gradients_are_the_same_every_time():
    a, dy = inputs(4, 80, 4096, 16, kind=BF16)
    d = dev(a)
    _, _, kept = ops.selective_scan(**d, with_checkpoints=True)
    first = ops.selective_scan_backward(dy.to(DEV), kept, **d)
    for _ in range(3):
        again = ops.selective_scan_backward(dy.to(DEV), kept, **d)
        assert all(p is q or torch.equal(p, q) for p, q in zip(first, again))


def test_scan_gradients_against_differences():
    """<gradient, v> against a central difference of the definition along v.

    The difference's own error, with steps of 1e-5 in 64 bits, is about 1e-9 of
    the value; the kernel's is within 1e-4 of the terms' absolute sum."""
    a, dy = inputs(2, 23, 20, 8, groups=2, kind=F32, state=True)
    got = check_backward(a, dy)
    r = ref_args(a)
    names = ("x", "dt", "A", "B", "C", "D", "z", "dt_bias", "state")
    for name, g in zip(names, got):
        v = torch.randn(r[name].shape, generator=torch.Generator().manual_seed(7)).double()
        f = [(R.scan(**dict(r, **{name: r[name] + s * 1e-5 * v}))["y"] * dy.double()).sum()
             for s in (1, -1)]
        slope, terms = (f[0] - f[1]) / 2e-5, g.double().cpu() * v
        assert abs(slope - terms.sum()) <= 1e-4 * terms.abs().sum() + 1e-6, name


@pytest.mark.parametrize("batch,dim,n,groups", [(1, 1, 1, 1), (3, 65, 16, 1), (5, 48, 5, 3),
                                                (2, 130, 33, 2), (64, 256, 64, 4)])
@pytest.mark.parametrize("kind", [F32, F16, BF16])
def test_step(batch, dim, n, groups, kind):
    a, _ = inputs(batch, 1, dim, n, groups, kind=kind, state=True)
    d = dev(a)
    pool = d["state"].clone()
    announce("selective_scan_step", batch, dim, n, groups, kind)
    y = ops.selective_scan_step(d["x"][:, 0], d["dt"][:, 0], pool, d["A"], d["B"][:, 0],
                                d["C"][:, 0], D=d["D"], z=d["z"][:, 0], dt_bias=d["dt_bias"])
    ref, mag = R.scan(**ref_args(a)), R.scan(**ref_args(a), absolute=True)
    R.assert_within(y, ref["y"][:, 0], mag["y"][:, 0], 4 * 33, "y")
    R.assert_within(pool, ref["state"], mag["state"], 4 * 33, "state")


def test_step_slots():
    """States named by slot; idle rows (-1, or outside the pool) touch nothing."""
    a, _ = inputs(5, 1, 70, 16, kind=BF16, state=True)
    d = dev(a)
    pool = torch.randn(9, 70, 16, device=DEV)
    before = pool.clone()
    slots = torch.tensor([7, -1, 0, 9, 3], dtype=torch.int32, device=DEV)
    args = (d["x"][:, 0], d["dt"][:, 0])
    more = dict(D=d["D"], z=d["z"][:, 0], dt_bias=d["dt_bias"])
    y = ops.selective_scan_step(*args, pool, d["A"], d["B"][:, 0], d["C"][:, 0], slots=slots, **more)
    rows, used = [0, 2, 4], [7, 0, 3]
    dense = before[used].clone()
    yd = ops.selective_scan_step(*(v[rows] for v in args), dense, d["A"], d["B"][rows, 0],
                                 d["C"][rows, 0], **dict(more, z=d["z"][rows, 0]))
    assert torch.equal(y[rows], yd) and torch.equal(pool[used], dense)
    assert not y[[1, 3]].any()
    rest = [i for i in range(9) if i not in used]
    assert torch.equal(pool[rest], before[rest])


def test_step_pool_beyond_32_bits():
    """A pool of more than 2^32 bytes and 2^31 elements: the last slots."""
    dim, n = 5120, 16
    count = 2**31 // (dim * n) + 40
    pool = torch.empty(count, dim, n, device=DEV)
    a, _ = inputs(2, 1, dim, n, kind=BF16, state=True)
    d = dev(a)
    slots = torch.tensor([count - 1, 2**30 // (dim * n) + 1], dtype=torch.int32, device=DEV)
    pool[slots.long()] = d["state"]
    small = d["state"].clone()
    args = (d["x"][:, 0], d["dt"][:, 0])
    more = dict(D=d["D"], z=d["z"][:, 0], dt_bias=d["dt_bias"])
    y = ops.selective_scan_step(*args, pool, d["A"], d["B"][:, 0], d["C"][:, 0], slots=slots, **more)
    want = ops.selective_scan_step(*args, small, d["A"], d["B"][:, 0], d["C"][:, 0], **more)
    assert torch.equal(y, want) and torch.equal(pool[slots.long()], small)


def test_steps_continue_a_prompt():
    """Prompt, then tokens one by one: the scan over all of them."""
    a, _ = inputs(3, 40, 70, 16, kind=F32)
    d = dev(a)
    whole, last, _ = ops.selective_scan(**d, with_state=True)
    head = {k: v[:, :33] if k in ("x", "dt", "z", "B", "C") else v for k, v in d.items()}
    _, pool, _ = ops.selective_scan(**head, with_state=True)
    mag = R.scan(**ref_args(a), absolute=True)
    for t in range(33, 40):
        y = ops.selective_scan_step(d["x"][:, t], d["dt"][:, t], pool, d["A"], d["B"][:, t],
                                    d["C"][:, t], D=d["D"], z=d["z"][:, t], dt_bias=d["dt_bias"])
        R.assert_within(y, whole[:, t].double().cpu(), mag["y"][:, t], 8 * 72, f"y[{t}]")
    R.assert_within(pool, last.double().cpu(), mag["state"], 8 * 72, "state")


def test_scan_special_values():
    """Infinities and NaN stay in their channel (and row); the step sizes' ends."""
    a, _ = inputs(2, 20, 40, 16, kind=F32)
    clean = ops.selective_scan(**dev(a))[0]
    a["x"][0, 5, 3] = float("nan")
    a["z"][1, 7, 11] = float("inf")
    a["dt"][0, 9, 20] = float("inf")    # the state is forgotten: exp(-inf) = 0, times x it is inf
    a["dt"][1, 2, 30] = -200.0          # a step of (nearly) nothing
    y = ops.selective_scan(**dev(a))[0]
    assert torch.isnan(y[0, 5:, 3]).all()
    touched = torch.zeros(2, 20, 40, dtype=torch.bool, device=DEV)
    touched[0, 5:, 3] = touched[1, 7, 11] = touched[0, 9:, 20] = touched[1, 2:, 30] = True
    assert torch.equal(y[~touched], clean[~touched])
    assert torch.isfinite(y[1, :, 30]).all()
    ref, mag = R.scan(**ref_args(a)), R.scan(**ref_args(a), absolute=True)
    R.assert_within(y[1, :, 30], ref["y"][1, :, 30], mag["y"][1, :, 30], 4 * 52, "small steps")


def test_scan_on_another_stream_and_in_a_graph():
    a, _ = inputs(2, 50, 70, 16, kind=BF16)
    d = dev(a)
    want = ops.selective_scan(**d)[0]
    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    with torch.cuda.stream(side):
        got = ops.selective_scan(**d)[0]
    side.synchronize()
    assert torch.equal(got, want)
    pool = torch.randn(2, 70, 16, device=DEV)
    start = pool.clone()
    args = (d["x"][:, 0], d["dt"][:, 0], pool, d["A"], d["B"][:, 0], d["C"][:, 0])
    out = torch.empty(2, 70, dtype=BF16, device=DEV)
    ops.selective_scan_step(*args, z=d["z"][:, 0], out=out)
    torch.cuda.synchronize()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        ops.selective_scan_step(*args, z=d["z"][:, 0], out=out)
    other = start.clone()
    pool.copy_(start)
    for _ in range(4):
        graph.replay()
        torch.cuda.synchronize()
        want = ops.selective_scan_step(*args[:2], other, *args[3:], z=d["z"][:, 0])
        assert torch.equal(out, want) and torch.equal(pool, other)


def test_refusals():
    a, dy = inputs(2, 6, 8, 4, kind=F32, state=True)
    d = dev(a)
    bad = [("x", d["x"].double(), TypeError), ("dt", d["dt"].half(), TypeError),
           ("A", d["A"][:, :3], ValueError), ("A", d["A"].half(), TypeError),
           ("B", d["B"][:, :5], ValueError), ("C", d["C"][:, :, :, :3], ValueError),
           ("B", d["B"][:, :, 0], TypeError), ("z", d["z"][:, :, :7], ValueError),
           ("D", d["D"][:7], ValueError), ("dt_bias", d["dt_bias"].cpu(), ValueError),
           ("state", d["state"].transpose(1, 2).contiguous().transpose(1, 2), ValueError),
           ("lengths", torch.zeros(2, dtype=torch.int64, device=DEV), TypeError),
           ("x", d["x"].transpose(1, 2).contiguous().transpose(1, 2), ValueError),
           ("out", torch.empty(2, 6, 7, device=DEV), ValueError)]
    for name, v, error in bad:
        with pytest.raises(error):
            ops.selective_scan(**dict(d, **{name: v}))
    with pytest.raises(ops._lib.LibscanError):  # three groups of eight channels
        ops.selective_scan(**dict(d, B=d["B"].expand(2, 6, 3, 4), C=d["C"].expand(2, 6, 3, 4)))
    with pytest.raises(ops._lib.LibscanError):  # more states than the kernels hold
        wide = torch.zeros(2, 6, 1, 65, device=DEV)
        ops.selective_scan(**dict(d, A=torch.zeros(8, 65, device=DEV), B=wide, C=wide, state=None))
    with pytest.raises(ops._lib.LibscanError):  # over its own input
        ops.selective_scan(**d, out=d["x"])
    with pytest.raises(ValueError):             # checkpoints of another call
        ops.selective_scan_backward(dy.to(DEV), torch.empty(5, device=DEV), **d)
    with pytest.raises(ValueError):             # fewer states than rows
        ops.selective_scan_step(d["x"][:, 0], d["dt"][:, 0], d["state"][:1], d["A"], d["B"][:, 0],
                                d["C"][:, 0])


@pytest.mark.parametrize("size", [(2, 32, 32, 16, 1), (3, 64, 64, 16, 2), (1, 32, 32, 32, 1),
                                  (2, 64, 64, 32, 2), (1, 32, 32, 64, 1), (2, 32, 64, 64, 2),
                                  (4, 32, 4096, 16, 2), (1, 1024, 64, 16, 1), (1, 768, 64, 32, 2),
                                  (1, 512, 32, 64, 1)])
@pytest.mark.parametrize("kind", [F32, F16, BF16])
def test_scan_whole_tiles(size, kind):
    """Steps, channels and states that leave no tile in part filled."""
    for state in (False, True):
        a, dy = inputs(*size, kind=kind, state=state)
        check_forward(a)
    check_backward(a, dy, dstate_out=torch.randn(size[0], size[2], size[3],
                                                 generator=torch.Generator().manual_seed(4)))


# ---------------------------------------------------------------- edges

def cut(a):
    """Whether the call's rows are cut into chunks: (forward, backward)."""
    p = ops._args.ssm(*(dev(a)[k] for k in ("x", "dt", "A", "B", "C", "D", "z", "dt_bias", "state",
                                            "lengths")), True, False)
    (batch, steps, dim), (groups, n) = a["x"].shape, a["B"].shape[2:]
    _, forward, backward = ops._sizes("selective_scan_bytes", p, 3)
    per = 32 if n <= 16 and batch * dim >= 16384 else 16  # channels of a workgroup, uncut
    parts = -(-dim // groups // per)
    whole = sum((v + 15) // 16 * 16 for v in (parts * batch * steps * groups * n * 8,
                                               batch * dim * n * 4, batch * dim * 4, batch * dim * 4))
    return forward > 0, backward != whole


@pytest.mark.parametrize("first", [False, True])
def test_chunks_of_growing_systems(first):
    """Negative step sizes: the decay over a chunk is beyond fp32, the states are
    not, as nothing (or next to nothing) is there to grow.  Forwards over the
    first steps, backwards over the last."""
    a, dy = inputs(1, 1537, 100, 16, skip=True, bias=False, state=True)
    assert cut(a) == (True, True)
    a["A"] = torch.full((100, 16), -8.0)
    a["A"][:, ::2] = -6.0
    a["dt"] = torch.full_like(a["dt"], 0.05)
    so = None
    if first:                       # a small start grows by e^112 in 40 steps
        a["state"] *= 1e-30
        a["dt"][:, :40] = -0.35
        a["x"][:, :38] = 0
        check_forward(a, softplus=False)
        a, dy = inputs(1, 1537, 100, 16, skip=True, bias=False, state=True)
        a["A"] = torch.full((100, 16), -8.0)
        a["dt"] = torch.full_like(a["dt"], 0.05)
        a["dt"][:, 1472:1512] = -0.35
        a["x"][:, 1400:] = 0
        dy[:, 1400:] = 0
        so = torch.randn(1, 100, 16, generator=torch.Generator().manual_seed(6)) * 1e-30
    else:                           # from nothing, by e^179 in 64
        a["state"] = None
        a["dt"][:, :64] = -0.35
        a["x"][:, :62] = 0
        dy[:, 10:] = 0
        check_forward(a, softplus=False)
    check_backward(a, dy, dstate_out=so, softplus=False)


def assert_same(got, ref, mag, c, what):
    """NaN where the definition has NaN, its infinities, and the bounds elsewhere."""
    g = got.detach().cpu().double()
    assert torch.equal(g.isnan(), ref.isnan()), \
        f"{what}: NaN at {(g.isnan() != ref.isnan()).nonzero()[:3].tolist()}"
    assert torch.equal(g[ref.isinf()], ref[ref.isinf()]), what
    odd = ~ref.isfinite()
    R.assert_within(got.detach().cpu().masked_fill(odd, 0), ref.masked_fill(odd, 0),
                    mag.masked_fill(~mag.isfinite(), 0), c, what)


def check_same(a, dy=None, softplus=True, dstate_out=None):
    """The call against the definition where inputs may be infinite or NaN."""
    batch, steps, dim = a["x"].shape
    d = dev(a)
    announce("selective_scan", tuple(a["x"].shape), tuple(a["B"].shape), a["x"].dtype)
    y, last, kept = ops.selective_scan(**d, softplus=softplus, with_state=True,
                                       with_checkpoints=True)
    more = dict(softplus_on=softplus)
    if dy is not None:
        more.update(dy=dy.double(),
                    dstate_out=dstate_out.double() if dstate_out is not None else None)
    ref = R.scan(**ref_args(a), **more)
    mag = R.scan(**ref_args(a), **more, absolute=True)
    assert_same(y, ref["y"], mag["y"], 4 * (steps + 32), "y")
    assert_same(last, ref["state"], mag["state"], 4 * (steps + 32), "state")
    if dy is None:
        return
    got = ops.selective_scan_backward(
        dy.to(DEV), kept, **d, softplus=softplus, with_dstate=True,
        dstate_out=dstate_out.to(DEV) if dstate_out is not None else None)
    for name, g in zip(NAMES, got):
        extra = dim + batch * steps if name in ("dA", "dB", "dC", "dD", "ddt_bias") else 0
        assert_same(g, ref[name], mag[name], 8 * (steps + 32) + extra, name)


def positive(*size, **kw):
    """Inputs whose products are all positive, so that infinities do not cancel."""
    a, dy = inputs(*size, state=True, **kw)
    for k in ("x", "B", "C", "D", "z", "state"):
        a[k] = a[k].abs() + 0.1
    a["A"] = -(a["A"].abs() * 0.02 + 0.01)
    return a, dy.abs() + 0.1


PADDED = [(2, 20, 40, 1, 1), (1, 35, 34, 5, 2), (1, 20, 17, 7, 1), (1, 33, 20, 16, 1),
          (2, 18, 40, 17, 1), (1, 20, 33, 33, 1), (1, 17, 20, 62, 1), (1, 18, 16400, 5, 1),
          (1, 18, 16400, 8, 2), (1, 801, 40, 3, 1), (1, 801, 40, 11, 2), (1, 801, 33, 20, 1),
          (1, 801, 20, 50, 1)]


@pytest.mark.parametrize("size", PADDED)
def test_infinities_where_states_or_channels_do_not_fill_the_lanes(size):
    """An infinite input, step size, gradient or C gives the infinities that the
    definition has, whatever n and the channels are padded to."""
    a, _ = positive(*size)
    if size[1] > 800:
        assert cut(a) == (True, True)
    a["x"][0, 5, 3] = a["dt"][0, 9, 12] = float("inf")
    check_same(a)
    a, dy = positive(*size)
    dy[0, 6, 3] = float("inf")
    check_same(a, dy)
    a, dy = positive(*size)
    a["C"][0, 7, 0, 0] = float("inf")
    check_same(a, dy)


@pytest.mark.parametrize("n", [1, 3, 8, 18, 64])
def test_step_infinities(n):
    a, _ = positive(2, 1, 40, n)
    a["x"][0, 0, 3] = a["dt"][1, 0, 9] = float("inf")
    d = dev(a)
    y = ops.selective_scan_step(d["x"][:, 0], d["dt"][:, 0], d["state"], d["A"], d["B"][:, 0],
                                d["C"][:, 0], D=d["D"], z=d["z"][:, 0], dt_bias=d["dt_bias"])
    ref, mag = R.scan(**ref_args(a)), R.scan(**ref_args(a), absolute=True)
    assert_same(y, ref["y"][:, 0], mag["y"][:, 0], 4 * 33, "y")
    assert_same(d["state"], ref["state"], mag["state"], 4 * 33, "state")


@pytest.mark.parametrize("size", [(1, 20, 40, 16, 1), (2, 33, 20, 20, 2), (1, 5, 34, 64, 1),
                                  (1, 18, 16400, 16, 1), (1, 801, 40, 16, 1)])
@pytest.mark.parametrize("ragged", [False, True])
def test_nothing_follows_a_rows_last_token(size, ragged):
    """A NaN or an infinity in the last token's x is in none of the gradients that
    it has no part in (A's among them)."""
    batch, steps = size[:2]
    count = steps - 3 if ragged else steps
    a, dy = positive(*size, lengths=[count] * batch if ragged else None)
    a["x"][0, count - 1, 3] = float("nan")
    a["x"][0, count - 1, 5] = float("inf")
    check_same(a, dy, dstate_out=torch.rand(
        batch, *a["A"].shape, generator=torch.Generator().manual_seed(9)))


@pytest.mark.parametrize("size", PADDED)
def test_an_infinite_state_beyond_the_last_token(size):
    """An infinity in B stays in the states to the end; steps that are not the row's
    have no part in the gradients."""
    a, dy = positive(*size)
    a["B"][0, 7, 0, 0] = float("inf")
    check_same(a, dy)


@pytest.mark.parametrize("size", PADDED)
def test_an_infinite_gradient_of_the_last_state(size):
    """It comes in before the steps that are not the row's, and passes them by."""
    a, dy = positive(*size)
    so = torch.rand(size[0], *a["A"].shape, generator=torch.Generator().manual_seed(9))
    so[0, 3, 0] = float("inf")
    check_same(a, dy, dstate_out=so)


CHUNKED = [  # gate, skip, bias, softplus, ragged
    (True, True, True, True, True), (False, True, True, True, True), (True, False, False, True, False),
    (False, False, True, False, True), (True, True, False, False, False),
    (False, True, False, True, False),
]


@pytest.mark.parametrize("n,groups", [(1, 1), (8, 1), (16, 2), (20, 1), (50, 2), (64, 1)])
@pytest.mark.parametrize("kind", [F32, F16, BF16])
def test_chunks_without_parts(n, groups, kind):
    """Rows that are cut, with and without a gate, D, a bias, the softplus and
    lengths, against the definition."""
    steps = 801 if n <= 32 else 1201
    i = [1, 8, 16, 20, 50, 64].index(n) + 2 * [F32, F16, BF16].index(kind)
    for gate, skip, bias, softplus, ragged in (CHUNKED[i % 6], CHUNKED[(i + 3) % 6]):
        lengths = [steps, 0, 33, 500] if ragged else None
        rows = 4 if ragged else 2
        a, dy = inputs(rows, steps, 70, n, groups, kind=kind, gate=gate, skip=skip, bias=bias,
                       state=ragged, lengths=lengths)
        if not softplus:
            a["dt"] = a["dt"].abs() * 0.2
            a["dt_bias"] = a["dt_bias"].abs() * 0.1 if bias else None
        assert cut(a) == (True, True)
        for b, count in enumerate(lengths or []):
            for k in ("x", "dt", "z", "B", "C"):
                if a[k] is not None:
                    a[k][b, count:] = float("nan")
            dy[b, count:] = float("nan")
        check_forward(a, softplus)
        so = torch.randn(rows, 70, n, generator=torch.Generator().manual_seed(8))
        check_backward(a, dy, dstate_out=so, softplus=softplus)


@pytest.mark.parametrize("n,groups", [(16, 1), (20, 2), (64, 1)])
@pytest.mark.parametrize("kind", [F32, BF16])
def test_chunks_of_strided_rows(n, groups, kind):
    """Cut rows on slices of wider tensors, time before batch, off 16 bytes, and
    one row's inputs for several (stride 0), against the definition."""
    a, dy = inputs(3, 801, 34, n, groups, kind=kind, state=True)
    a["dt"] = a["dt"][:1].expand(3, 801, 34)
    assert cut(a) == (True, True)
    ref, mag = (R.scan(**ref_args(a), dy=dy.double(), absolute=v) for v in (False, True))
    d = dev(a)
    wide = torch.full((801, 3, 3 * 34 + 1), float("nan"), dtype=kind, device=DEV)
    views = [wide[:, :, 1 + 34 * i:35 + 34 * i].transpose(0, 1) for i in range(3)]
    for v, t in zip(views, (a["x"], a["z"], dy)):
        v.copy_(t)
    both = torch.full((3, 801, 1 + 2 * groups * n), float("nan"), dtype=kind, device=DEV)
    for i, k in enumerate("BC"):
        v = both[:, :, 1 + i * groups * n:1 + (i + 1) * groups * n].unflatten(2, (groups, n))
        v.copy_(d[k])
        d[k] = v
    d["x"], d["z"] = views[:2]
    d["dt"] = a["dt"][:1].to(DEV).expand(3, 801, 34)
    y, last, kept = ops.selective_scan(**d, with_state=True, with_checkpoints=True)
    R.assert_within(y, ref["y"], mag["y"], 4 * 833, "y")
    R.assert_within(last, ref["state"], mag["state"], 4 * 833, "state")
    got = ops.selective_scan_backward(views[2], kept, **d)
    for name, g in zip(NAMES, got):
        extra = 34 + 3 * 801 if name in ("dA", "dB", "dC", "dD", "ddt_bias") else 0
        R.assert_within(g, ref[name], mag[name], 8 * 833 + extra, name)
