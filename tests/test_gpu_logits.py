"""Penalties, biases, grammar masks and the softmax behind them against the
definition in 64 bits (lm_ref.py, where the bounds are derived)."""
import pytest
import torch

import lm_ref as R
from gpu_util import announce
from paper_2505_15112_amd import _lib, ops

pytestmark = pytest.mark.gpu
DEV = "cuda"
F32, F16, BF16 = torch.float32, torch.float16, torch.bfloat16


def inputs(rows, vocab, kind=F32, hist=0, biases=0, grammar=False, seed=0):
    g = torch.Generator().manual_seed(seed)
    a = dict(logits=(torch.randn(rows, vocab, generator=g) * 4).to(kind))
    if hist:
        a["history"] = torch.randint(-2, vocab + 2, (rows, hist), generator=g).int()
        a["history"][:, hist // 2:] = torch.randint(0, min(vocab, 7), (rows, hist - hist // 2),
                                                    generator=g).int()
        a["history_len"] = torch.randint(0, hist + 1, (rows,), generator=g).int()
        a["prompt_len"] = torch.randint(0, hist + 1, (rows,), generator=g).int()
        a["repetition"] = torch.rand(rows, generator=g) + 0.7
        a["presence"] = torch.rand(rows, generator=g)
        a["frequency"] = torch.rand(rows, generator=g) * 0.3
    if biases:
        # ids repeat and fall outside
        a["bias_ids"] = torch.randint(-1, vocab + 1, (rows, biases), generator=g).int()
        a["bias_ids"][:, biases // 2] = a["bias_ids"][:, 0]
        a["bias_values"] = torch.randn(rows, biases, generator=g) * 3
    if grammar:
        a["allowed"] = torch.randint(-2**31, 2**31, (rows, (vocab + 31) // 32), generator=g).int()
    return a


def dev(a):
    return {k: v.to(DEV) for k, v in a.items()}


def ref(a):
    a = {k: v.double() if v.is_floating_point() else v for k, v in a.items()}
    return R.logits(a.pop("logits"), **a)


def check(a, temperature=None):
    announce("logits", tuple(a["logits"].shape), a["logits"].dtype, sorted(a))
    x, mag = ref(a)
    got = ops.logits_process(**dev(a))
    inf = x == R.NEG_INF
    assert torch.equal(got.cpu() == R.NEG_INF, inf)
    R.assert_within(got.masked_fill(inf.to(DEV), 0), x.masked_fill(inf, 0), mag, 8, "logits")
    d = dev(a)
    same = ops.logits_process(**dict(d, out=d["logits"]))  # in place
    assert torch.equal(same, got)
    p = ops.logits_probs(**dev(a),
                         temperature=temperature.to(DEV) if temperature is not None else None)
    want = R.probs(x, temperature)
    # the exponent's argument is off by its own size's roundings; so much for p
    t = torch.ones(x.shape[0]) if temperature is None else temperature
    size = (mag.max(1, keepdim=True).values + mag) / t.double()[:, None].clamp(min=1e-30)
    # the sum's roundings: one for each of the at most 64 places a thread adds,
    # and a few over threads and segments
    R.assert_within(p, want, want * (8 * size + 128), 1, "probs")
    assert not p.cpu()[inf].any()


@pytest.mark.parametrize("rows,vocab", [(1, 1), (3, 2), (2, 31), (5, 33), (2, 1000), (3, 8191),
                                        (2, 8192), (2, 8193), (1, 20001), (3, 50257)])
@pytest.mark.parametrize("kind", [F32, F16, BF16])
def test_all_parts(rows, vocab, kind):
    check(inputs(rows, vocab, kind, hist=50, biases=9, grammar=True),
          torch.linspace(0.3, 1.5, rows))


@pytest.mark.parametrize("hist,biases,grammar", [(0, 0, False), (30, 0, False), (0, 5, False),
                                                 (0, 0, True), (1, 1, False)])
@pytest.mark.parametrize("vocab", [700, 9001])
def test_parts_alone(hist, biases, grammar, vocab):
    check(inputs(4, vocab, BF16, hist, biases, grammar))


def test_history_defaults_and_long_history():
    """No lengths: all columns are generated tokens; counts beyond 16 bits."""
    a = inputs(2, 300, F32, hist=90000)
    a["history"][1] = 5
    for k in ("history_len", "prompt_len", "presence"):
        del a[k]
    check(a)


def test_many_rows():
    check(inputs(700, 300, F16, hist=20, biases=3, grammar=True))


@pytest.mark.parametrize("rows,vocab", [(40, 60000), (129, 16387), (300, 8193)])
@pytest.mark.parametrize("named", [True, False])
@pytest.mark.parametrize("kind", [F32, F16, BF16])
def test_many_long_rows(rows, vocab, named, kind):
    """Rows of several segments, enough of them for the wide workgroups."""
    a = (inputs(rows, vocab, kind, hist=60, biases=9, grammar=True) if named
         else inputs(rows, vocab, kind))
    check(a, torch.linspace(0.3, 1.5, rows))


def test_rows_that_the_mask_leaves_empty():
    a = inputs(4, 20000, F32, grammar=True)
    a["allowed"][1] = 0
    a["allowed"][2] = 0
    a["allowed"][2, 600] = 1 << 7
    p = ops.logits_probs(**dev(a)).cpu()
    assert not p[1].any()
    assert p[2, 600 * 32 + 7] == 1 and p[2].sum() == 1
    check(a)


def test_special_values():
    """The type's lowest value, infinities and NaN, in masked and open places."""
    a = inputs(8, 9000, F32, grammar=True)
    x, al = a["logits"], a["allowed"]
    al[:] = -1
    x[0, 5] = float("nan")
    al[0, 0] = ~(1 << 5)                    # masked: no trace of it
    x[1, 8500] = float("inf")
    al[1, 8500 // 32] = ~(1 << (8500 % 32))
    x[2, :] = torch.finfo(F32).min          # equal shares of the lowest value
    x[3, 10] = R.NEG_INF                    # open, but nothing there
    x[4, 20] = float("nan")
    x[5, 30] = float("inf")
    x[6, :] = R.NEG_INF
    x[7, :8999] = R.NEG_INF
    p = ops.logits_probs(**dev(a)).cpu()
    want = R.probs(*ref(a)[:1])
    assert torch.equal(p.isnan(), want.isnan())
    assert p[4].isnan().all() and p[5].isnan().all() and not p[6].any() and p[7, 8999] == 1
    ok = [0, 1, 2, 3, 7]
    R.assert_within(p[ok], want[ok], want[ok] * 400, 1, "probs")
    hot = torch.zeros(8)
    cold = ops.logits_probs(**dev(a), temperature=hot.to(DEV)).cpu()
    wcold = R.probs(ref(a)[0], hot)
    assert torch.equal(cold.isnan(), wcold.isnan()) and cold[5, 30] == 1
    assert ((cold - wcold).nan_to_num().abs() <= 2.0**-23 * wcold.nan_to_num()).all()


def test_low_masks_of_half_types():
    for kind in (F16, BF16):
        a = inputs(2, 600, kind)
        a["logits"][0, :599] = torch.finfo(kind).min
        a["logits"][1, :] = torch.finfo(kind).min
        p = ops.logits_probs(**dev(a)).cpu()
        assert p[0, 599] == 1 and not p[0, :599].any()
        R.assert_within(p[1], torch.full((600,), 1 / 600).double(), torch.full((600,), 1 / 600), 64,
                        "equal")


@pytest.mark.parametrize("vocab", [900, 20001])
def test_negative_temperature(vocab):
    """The shares of the negated logits, bit for bit; masked and empty places have none."""
    a = inputs(3, vocab, F32, grammar=True)
    a["logits"][1, 5:90] = R.NEG_INF
    other = dict(a, logits=(-a["logits"]).masked_fill(a["logits"] == R.NEG_INF, R.NEG_INF))
    t = torch.tensor([1.0, 0.7, 2.0], device=DEV)
    got = ops.logits_probs(**dev(a), temperature=-t)
    assert torch.equal(got, ops.logits_probs(**dev(other), temperature=t))
    assert got.sum(1).sub(1).abs().max() < 1e-4 and not got[1, 5:90].any()


def test_temperature_zero_shares_ties():
    a = inputs(2, 10000, F32)
    a["logits"][0, [3, 9000]] = 50.0
    p = ops.logits_probs(**dev(a), temperature=torch.tensor([0.0, 1.0], device=DEV)).cpu()
    assert p[0, 3] == 0.5 and p[0, 9000] == 0.5 and p[0].sum() == 1
    assert abs(float(p[1].double().sum()) - 1) < 1e-5


@pytest.mark.parametrize("vocab", [999, 16385])
def test_strides(vocab):
    a = inputs(3, vocab, BF16, hist=12, grammar=True)
    d = dev(a)
    want = ops.logits_process(**d)
    big = torch.full((3, vocab + 7), float("nan"), dtype=BF16, device=DEV)
    big[:, 3:3 + vocab] = d["logits"]
    hist = torch.full((3, 20), 1, dtype=torch.int32, device=DEV)
    hist[:, 4:16] = d["history"]
    allowed = torch.zeros(3, d["allowed"].shape[1] + 1, dtype=torch.int32, device=DEV)
    allowed[:, 1:] = d["allowed"]
    s = dict(d, logits=big[:, 3:3 + vocab], history=hist[:, 4:16], allowed=allowed[:, 1:])
    assert torch.equal(ops.logits_process(**s), want)
    assert torch.equal(ops.logits_probs(**s), ops.logits_probs(**d))
    into = torch.zeros(3, vocab + 5, dtype=BF16, device=DEV)
    ops.logits_process(**s, out=into[:, 2:2 + vocab])
    assert torch.equal(into[:, 2:2 + vocab], want)
    assert not into[:, :2].any() and not into[:, 2 + vocab:].any()


def test_empty():
    for rows, vocab in ((0, 10), (3, 0)):
        x = torch.zeros(rows, vocab, device=DEV)
        assert ops.logits_process(x).shape == (rows, vocab)
        assert ops.logits_probs(x).shape == (rows, vocab)


def test_probabilities_go_into_the_sampler():
    """A grammar's tokens only, and the most likely at temperature 0."""
    a = inputs(16, 40000, BF16, hist=64, biases=4, grammar=True)
    d = dev(a)
    p = ops.logits_probs(**d, temperature=torch.full((16,), 0.8, device=DEV))
    tok = ops.topp_sample_f32(p, torch.rand(16, device=DEV), 0.9).cpu().long()
    bits = (a["allowed"].gather(1, (tok // 32)[:, None])[:, 0] >> (tok % 32)) & 1
    assert bits.all()
    cold = ops.logits_probs(**d, temperature=torch.zeros(16, device=DEV))
    tok = ops.topp_sample_f32(cold, torch.rand(16, device=DEV) * 0.4, 0.9).cpu().long()
    best = ops.logits_process(**dict(d, logits=d["logits"].float())).cpu()
    assert torch.equal(best.gather(1, tok[:, None])[:, 0], best.max(1).values)


def test_in_a_graph():
    a = dev(inputs(4, 30000, BF16, hist=40, grammar=True))
    want = ops.logits_probs(**a)
    out = torch.empty_like(want)
    buf = torch.empty(1 << 16, dtype=torch.uint8, device=DEV)
    ops.logits_probs(**a, out=out, scratch_buf=buf)
    torch.cuda.synchronize()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        ops.logits_probs(**a, out=out, scratch_buf=buf)
    for i in range(4):
        out.zero_()
        buf.fill_(i)
        graph.replay()
        torch.cuda.synchronize()
        assert torch.equal(out, want)


def test_refusals():
    a = dev(inputs(2, 100, F32, hist=5, biases=3, grammar=True))
    bad = [(dict(logits=a["logits"].double()), TypeError), (dict(logits=a["logits"][0]), ValueError),
           (dict(history=a["history"].long()), TypeError), (dict(history=None), ValueError),
           (dict(history_len=a["history_len"][:1]), ValueError),
           (dict(repetition=a["repetition"].half()), TypeError),
           (dict(bias_ids=None), ValueError), (dict(bias_values=a["bias_values"][:, :2]), ValueError),
           (dict(allowed=a["allowed"][:, :3]), ValueError), (dict(presence=1.0), TypeError),
           (dict(allowed=a["allowed"].cpu()), ValueError),
           (dict(out=torch.empty(2, 99, device=DEV)), ValueError)]
    for change, error in bad:
        with pytest.raises(error):
            ops.logits_process(**dict(a, **change))
    with pytest.raises(_lib.LibscanError):  # over its input, a place further on
        buf = torch.zeros(2 * 100 + 1, device=DEV)
        ops.logits_process(buf[:200].view(2, 100), out=buf[1:].view(2, 100))
    with pytest.raises(_lib.LibscanError):  # too little scratch
        ops.logits_probs(torch.zeros(2, 50000, device=DEV),
                         scratch_buf=torch.empty(16, dtype=torch.uint8, device=DEV))


@pytest.mark.parametrize("vocab", [900, 20001])
@pytest.mark.parametrize("masked", [False, True])
def test_temperature_of_negative_zero(vocab, masked):
    """-0.0 is 0: the largest logit's places, as for +0.0."""
    a = inputs(3, vocab, F32, hist=20, grammar=masked)
    a["logits"][1, [4, 800]] = 60.0
    zero = torch.zeros(3)
    got = ops.logits_probs(**dev(a), temperature=(-zero).to(DEV)).cpu()
    assert torch.equal(got, ops.logits_probs(**dev(a), temperature=zero.to(DEV)).cpu())
    want = R.probs(ref(a)[0], zero)
    assert ((got - want).abs() <= 2.0**-23 * want).all()


@pytest.mark.parametrize("vocab", [3000, 20001])
def test_repetition_divides(vocab):
    """Seen tokens alone: one rounding, that of l / repetition or l * repetition."""
    x = inputs(3, vocab, F32)["logits"]
    x[2] *= 1e-30
    rep = torch.tensor([1.1, 0.7, 1e-39])  # the last one's reciprocal is beyond fp32
    got = ops.logits_process(x.to(DEV), history=torch.arange(vocab).int().expand(3, -1).to(DEV),
                             prompt_len=torch.full((3,), vocab).int().to(DEV),
                             repetition=rep.to(DEV)).cpu()
    assert torch.equal(got, torch.where(x > 0, x / rep[:, None], x * rep[:, None]))


@pytest.mark.parametrize("vocab,biases", [(40, 700), (5000, 4000), (20001, 3001)])
@pytest.mark.parametrize("hist", [0, 300])
def test_biases_that_repeat_add_up_in_the_lists_order(vocab, biases, hist):
    """Single-precision additions one by one, so the same bits."""
    a = inputs(2, vocab, F32, hist=hist)
    base = ops.logits_process(**dev(a)).cpu() if hist else a["logits"]
    g = torch.Generator().manual_seed(3)
    ids = torch.randint(-1, vocab + 1, (2, biases), generator=g).int()
    ids[1, ::3] = 7                     # one id in a third of the list
    ids[0, biases // 2:] = ids[0, :biases - biases // 2].clone()
    values = torch.randn(2, biases, generator=g) * 3
    got = ops.logits_process(**dev(dict(a, bias_ids=ids, bias_values=values))).cpu()
    want = base.clone().numpy()
    for r in range(2):
        for tok, v in zip(ids[r].tolist(), values[r].numpy()):
            if 0 <= tok < vocab:
                want[r, tok] += v
    assert torch.equal(got, torch.from_numpy(want))


def test_repeated_biases_take_no_quadratic_time():
    """A long list with every id twice, or one id alone, against one without
    repeats: a few walks over the list, where a search for each entry's repeats
    took 1600 times as long (50 times are room for noise)."""
    g = torch.Generator(device=DEV).manual_seed(1)
    x = torch.randn(1, 131072, device=DEV, generator=g)
    once = torch.randperm(131072, device=DEV, generator=g)[None, :16384].int().contiguous()
    twice = torch.cat((once[:, :8192], once[:, :8192]), 1)
    values = torch.randn(1, 16384, device=DEV, generator=g)

    def time(ids):
        ops.logits_process(x, bias_ids=ids, bias_values=values)
        each = []
        for _ in range(5):
            a, b = (torch.cuda.Event(enable_timing=True) for _ in range(2))
            a.record()
            ops.logits_process(x, bias_ids=ids, bias_values=values)
            b.record()
            torch.cuda.synchronize()
            each.append(a.elapsed_time(b))
        return sorted(each)[2]

    limit = 50 * time(once)
    assert time(twice) < limit and time(torch.full_like(once, 77)) < limit


@pytest.mark.parametrize("rows,vocab", [(1, 200003), (4, 600001)])
@pytest.mark.parametrize("named", [True, False])
def test_rows_of_more_than_64_segments(rows, vocab, named):
    """More segments than a wave has lanes, small ones and large ones: the maximum
    and most of the sum beyond the first 64, and among them."""
    a = (inputs(rows, vocab, BF16, hist=60, biases=9, grammar=True) if named
         else inputs(rows, vocab, BF16))
    for at in (vocab - 3, 5):
        a["logits"][:, at] = 25.0
        if named:
            a["allowed"][:, at // 32] = -1
        check(a, torch.linspace(0.5, 1.5, rows))


def test_repetition_divides_at_its_ends():
    """Penalties and logits from the smallest to the largest, 0, infinities and NaN: the
    quotient's bits (results below the normal range aside)."""
    g = torch.Generator().manual_seed(5)
    rep = torch.cat((torch.tensor([0.0, 1e-45, 1e-39, 2.0**-126, 2.0**-125, 1.0, 3.0, 2.0**126,
                                   3.4e38, float("inf"), float("nan")]),
                     torch.exp2(torch.rand(53, generator=g) * 250 - 125),
                     torch.rand(192, generator=g) + 0.5))
    x = torch.exp2(torch.rand(len(rep), 4001, generator=g) * 250 - 125)
    x[:, ::2] = torch.rand(len(rep), 2001, generator=g) * 8
    x[:, :4] = torch.tensor([0.0, float("inf"), 3.4e38, 1e-38])
    rows, vocab = x.shape
    got = ops.logits_process(x.to(DEV), history=torch.arange(vocab).int().expand(rows, -1).to(DEV),
                             prompt_len=torch.full((rows,), vocab).int().to(DEV),
                             repetition=rep.to(DEV)).cpu()
    want = torch.where(x > 0, x / rep[:, None], x * rep[:, None])
    assert torch.equal(got.isnan(), want.isnan())
    normal = (want >= 2.0**-126) | (want == 0)
    assert normal.double().mean() > 0.7 and torch.equal(got[normal], want[normal])
