"""Layer norm and its gradients against the definition in 64 bits
(attend_ref.py)."""
import pytest
import torch

import attend_ref as R
from attend_ref import BF16, F16, F32
from gpu_util import announce
from paper_2505_15112_amd import ops

pytestmark = pytest.mark.gpu
DEV = "cuda"


def inputs(rows, dim, kind, weights=None, residual=False, seed=0, shift=0.5):
    g = torch.Generator().manual_seed(seed)
    weights = weights or kind

    def normal(*s, dtype=kind):
        return torch.randn(*s, generator=g).to(dtype)

    lead = rows if isinstance(rows, tuple) else (rows,)
    a = dict(x=(torch.randn(*lead, dim, generator=g) + shift).to(kind),
             weight=normal(dim, dtype=weights), bias=normal(dim, dtype=weights),
             residual=normal(*lead, dim) if residual else None)
    return a, normal(*lead, dim), normal(*lead, dim)


def dev(a):
    return {k: v.to(DEV) if isinstance(v, torch.Tensor) else v for k, v in a.items()}


def roundings(dim, groups):
    """Sums of dim / groups terms by at most 64 lanes' partial sums, each a chain, and
    about 16 roundings beside them."""
    return (dim // groups / 64 + 32) * 2.0**-24


def check(a, dy, dsum, groups=1, eps=1e-5):
    dim, x = a["x"].shape[-1], a["x"]
    announce("layer_norm", tuple(x.shape), x.dtype, groups)
    d = dev(a)
    y, total, stats = ops.layer_norm(**d, groups=groups, eps=eps, with_stats=True)
    dsum = dsum if a["residual"] is not None else None
    ref = R.norm(**a, groups=groups, eps=eps, dy=dy, dsum=dsum)
    r = 2 * roundings(dim, groups)
    R.assert_within(y, ref["y"], ref["my"], r, "y")
    R.assert_within(stats[..., 0], ref["mean"], ref["mmean"], r, "mean")
    R.assert_within(stats[..., 1], ref["rstd"], ref["mrstd"], r, "rstd")
    if total is None:
        assert a["residual"] is None
    else:
        assert torch.equal(total.cpu(), ref["sum"])
    announce("layer_norm_backward", tuple(x.shape), x.dtype, groups)
    back = ops.layer_norm_backward(dy.to(DEV), d["x"] if total is None else total, stats,
                                   d["weight"], d["bias"],
                                   dsum=dsum.to(DEV) if dsum is not None else None, groups=groups)
    rows = x.numel() // dim
    for name, got, more in zip(("dx", "dweight", "dbias"), back, (0, rows, rows)):
        if got is None:
            assert a[name[1:]] is None
            continue
        R.assert_within(got, ref[name], ref["m" + name], 2 * r + more * 2.0**-24, name)
    return (y, total, stats, *back)


SIZES = [(1, 1, 1), (1, 64, 1), (3, 65, 1), (2, 7, 7), (5, 128, 2), (70, 96, 3), (33, 512, 16),
         (9, 1000, 1), (4, 2048, 1), (130, 1024, 8), (3, 4096, 1), (2, 5120, 1), (5, 4099, 1),
         (3, 8192, 1), (2, 16389, 1), (1, 33000, 1), (2, 40000, 2), (300, 40, 1), (3, 70001, 1)]


@pytest.mark.parametrize("size", SIZES)
@pytest.mark.parametrize("kind", [F32, F16, BF16])
def test_norm(size, kind):
    rows, dim, groups = size
    a, dy, dsum = inputs(rows, dim, kind, residual=rows % 2 == 1)
    check(a, dy, dsum, groups)


@pytest.mark.parametrize("kind", [F16, BF16])
@pytest.mark.parametrize("size", [(5, 96, 3), (9, 4096, 1), (2, 20000, 1)])
def test_fp32_weights(kind, size):
    rows, dim, groups = size
    a, dy, dsum = inputs(rows, dim, kind, weights=F32, residual=True)
    check(a, dy, dsum, groups)


@pytest.mark.parametrize("without", [("weight",), ("bias",), ("weight", "bias")])
@pytest.mark.parametrize("dim", [48, 1000, 33000])
def test_without_weight_or_bias(without, dim):
    a, dy, dsum = inputs(7, dim, BF16)
    check(dict(a, **{k: None for k in without}), dy, dsum)


def test_many_rows():
    """Enough rows for every workgroup to have several, of two kinds of rows."""
    for rows, dim, groups in ((20011, 64, 1), (5003, 256, 4), (3001, 1024, 1)):
        a, dy, dsum = inputs(rows, dim, F32)
        check(a, dy, dsum, groups)


def test_more_groups_than_one_launch_takes():
    """2^21 + 3 rows of 8 groups of 4 channels: the groups come in turns."""
    rows = (1 << 21) + 3
    x = torch.randn(rows, 32, device=DEV, generator=torch.Generator(device=DEV).manual_seed(1))
    y, _, stats = ops.layer_norm(x, groups=8, with_stats=True)
    dx, _, _ = ops.layer_norm_backward(y, x, stats, groups=8)
    for part in (slice(0, 50), slice(rows - 50, rows), slice(rows // 2, rows // 2 + 50)):
        ref = R.norm(x[part].cpu(), groups=8, dy=y[part].cpu())
        R.assert_within(y[part], ref["y"], ref["my"], 2 * roundings(32, 8), "y")
        R.assert_within(dx[part], ref["dx"], ref["mdx"], 4 * roundings(32, 8), "dx")


def test_rows_beyond_32_bit_offsets():
    """2.2e9 elements."""
    rows, dim = 135000, 16384
    if torch.cuda.mem_get_info()[0] < 30 << 30:
        pytest.skip("needs 18 GB")
    x = torch.empty(rows, dim, dtype=BF16, device=DEV).normal_(
        generator=torch.Generator(device=DEV).manual_seed(1))
    announce("layer_norm", tuple(x.shape))
    y, _, stats = ops.layer_norm(x, with_stats=True)
    dx, _, _ = ops.layer_norm_backward(y, x, stats)
    want, _, st = ops.layer_norm(x[-40:], with_stats=True)
    assert torch.equal(y[-40:], want) and torch.equal(stats[-40:], st)
    assert torch.equal(dx[-40:], ops.layer_norm_backward(want, x[-40:], st)[0])


def test_rows_far_from_zero():
    """A mean of 1000 times the deviation: the variance is that of the differences."""
    a, dy, dsum = inputs(4, 1024, F32, shift=1000.0)
    check(a, dy, dsum)


def test_constant_rows_and_eps():
    x = torch.full((2, 512), 3.0, device=DEV)
    y, _, stats = ops.layer_norm(x, with_stats=True)
    assert not y.any() and bool((stats[:, 0, 0] == 3.0).all())
    # 1 / sqrt(1e-5) to three roundings
    assert (stats[:, 0, 1] - 1e5 ** 0.5).abs().max() <= 3 * 2.0**-24 * 1e5 ** 0.5
    a, dy, dsum = inputs(4, 512, F32)
    check(a, dy, dsum, eps=10.0)
    check(a, dy, dsum, eps=0.0)


def test_batches_strides_and_outputs():
    """batch x steps x dim in slices of wider tensors, unaligned; given outputs."""
    a, dy, dsum = inputs((3, 5), 200, BF16, residual=True)
    want = check(a, dy, dsum, 4)
    d = dev(a)

    def wide(t):
        w = torch.zeros(3, 6, 403, dtype=BF16, device=DEV)[:, 1:, 1:201]
        return w.copy_(t)

    y, s, st = (torch.empty_like(t) for t in want[:3])
    got = ops.layer_norm(wide(d["x"]), d["weight"], d["bias"], residual=wide(d["residual"]),
                         groups=4, out=y, sum_out=s, stats_out=st)
    assert got[0] is y and got[1] is s and got[2] is st
    for g, w in zip(got, want):
        assert torch.equal(g, w)
    back = ops.layer_norm_backward(wide(dy.to(DEV)), wide(s), st, d["weight"], d["bias"],
                                   dsum=wide(dsum.to(DEV)), groups=4)
    for g, w in zip(back, want[3:]):
        assert torch.equal(g, w)
    flat = ops.layer_norm(d["x"].flatten(0, 1), d["weight"], d["bias"],
                          residual=d["residual"].flatten(0, 1), groups=4)
    assert torch.equal(flat[0], want[0].flatten(0, 1))
    turned = d["x"].transpose(0, 1)  # batch and steps the other way round
    y2, _, _ = ops.layer_norm(turned, d["weight"], d["bias"], groups=4)
    y3, _, _ = ops.layer_norm(turned.contiguous(), d["weight"], d["bias"], groups=4)
    assert torch.equal(y2, y3)


@pytest.mark.parametrize("bad", [float("inf"), float("nan")])
@pytest.mark.parametrize("dim", [64, 4096, 33000])
def test_a_bad_value_stays_in_its_row_and_group(bad, dim):
    a, dy, _ = inputs(6, dim, BF16)
    d = dev(a)
    want = ops.layer_norm(**d, groups=2, with_stats=True)
    d["x"][3, 1] = bad
    got = ops.layer_norm(**d, groups=2, with_stats=True)
    rest = [0, 1, 2, 4, 5]
    assert torch.equal(got[0][rest], want[0][rest]) and torch.equal(got[2][rest], want[2][rest])
    assert torch.equal(got[0][3, dim // 2:], want[0][3, dim // 2:])
    assert bool(torch.isnan(got[0][3, :dim // 2]).all())


def test_gradients_against_differences():
    a, dy, _ = inputs(3, 24, F32)
    d = dev(a)
    _, _, stats = ops.layer_norm(**d, groups=2, with_stats=True)
    got = ops.layer_norm_backward(dy.to(DEV), d["x"], stats, d["weight"], d["bias"], groups=2)
    g = torch.Generator().manual_seed(9)
    at = {k: v.double() for k, v in a.items() if v is not None}
    for grad, key in zip(got, ("x", "weight", "bias")):
        way = torch.randn(at[key].shape, generator=g, dtype=torch.double)

        def value(e):
            return (R.norm(**dict(at, **{key: at[key] + e * way}), groups=2)["y"] *
                    dy.double()).sum()

        want = (value(1e-5) - value(-1e-5)) / 2e-5
        have, size = ((f(grad.cpu().double() * way)).sum() for f in (lambda t: t, torch.abs))
        assert abs(have - want) <= 1e-5 * size + 1e-6, key


def test_graph_and_stream():
    a, dy, dsum = inputs(50, 1024, BF16, residual=True)
    d, dy, dsum = dev(a), dy.to(DEV), dsum.to(DEV)

    def work():
        y, s, st = ops.layer_norm(**d, with_stats=True)
        return (y, s, st, *ops.layer_norm_backward(dy, s, st, d["weight"], d["bias"], dsum=dsum))

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
        b, dy2, ds2 = inputs(50, 1024, BF16, residual=True, seed=3 + seed)
        for k in d:
            d[k].copy_(b[k])
        dy.copy_(dy2), dsum.copy_(ds2)
        want = work()
        torch.cuda.synchronize()
        graph.replay()
        torch.cuda.synchronize()
        assert all(torch.equal(x, w) for x, w in zip(out, want))


def test_refusals_and_nothing_to_do():
    a, dy, dsum = inputs(6, 64, BF16, residual=True)
    d = dev(a)
    for bad, error, what in (
            (dict(weight=d["weight"][:32]), ValueError, "weight"),
            (dict(weight=d["weight"].float()), TypeError, "bias"),
            (dict(bias=d["bias"].half()), TypeError, "bias"), (dict(groups=3), ValueError, "groups"),
            (dict(groups=0), ValueError, "groups"), (dict(residual=d["x"][:3]), ValueError, "res"),
            (dict(x=d["x"].t()), ValueError, "x|weight"), (dict(x=d["x"][0]), ValueError, "x"),
            (dict(x=d["x"].double()), TypeError, "x"), (dict(eps="small"), TypeError, "real number|float")):
        with pytest.raises(error, match=what):
            ops.layer_norm(**dict(d, **bad))
    for bad in (dict(eps=-1.0), dict(eps=float("nan")), dict(out=d["x"]), dict(sum_out=d["x"])):
        with pytest.raises(ops._lib.LibscanError):
            ops.layer_norm(**dict(d, **bad))
    with pytest.raises(ValueError, match="residual"):
        ops.layer_norm(d["x"], sum_out=torch.empty_like(d["x"]))
    y, s, st = ops.layer_norm(**d, with_stats=True)
    with pytest.raises(TypeError, match="stats"):
        ops.layer_norm_backward(dy.to(DEV), s, None, d["weight"])
    with pytest.raises(ValueError, match="stats"):
        ops.layer_norm_backward(dy.to(DEV), s, st, d["weight"], groups=2)
    with pytest.raises(ValueError, match="dsum"):
        ops.layer_norm_backward(dy.to(DEV), s, st, dsum=dsum[:2].to(DEV))
    with pytest.warns(UserWarning, match="layer_norm_backward"):
        ops.layer_norm(d["x"].clone().requires_grad_())
    y, s, st = ops.layer_norm(d["x"][:0], d["weight"], d["bias"], with_stats=True)
    back = ops.layer_norm_backward(dy[:0].to(DEV), d["x"][:0], st, d["weight"], d["bias"])
    assert y.shape == (0, 64) and back[0].shape == (0, 64)
    assert not back[1].any() and not back[2].any()
