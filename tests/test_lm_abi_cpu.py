"""The language model operators' entry points on the CPU: every call here is
refused (or has nothing to do) before any HIP call, by its arguments."""
import ctypes
import os
import struct

import pytest
import torch

from paper_2505_15112_amd import _lib, ops

if not os.path.exists(_lib.LIB_PATH):
    from paper_2505_15112_amd import build as _build
    _build.build()

A = 0x10000000  # fake addresses, never dereferenced, 256 MiB apart
STEP = 0x10000000


def at(i):
    return A + i * STEP


@pytest.fixture(scope="module")
def lib():
    return _lib.load()


CONV = ("type weight_type batch steps dim width silu x x_batch x_step weight bias state "
        "lengths").split()
SSM = ("type batch steps dim n groups softplus x x_batch x_step dt dt_batch dt_step z z_batch "
       "z_step B B_batch B_step B_group C C_batch C_step C_group A D dt_bias state lengths").split()
LOGITS = ("type rows vocab logits logits_row history history_row history_cols history_len "
          "prompt_len repetition presence frequency bias_ids bias_values biases allowed allowed_row "
          "temperature").split()


def pack(names, values):
    assert set(values) <= set(names)
    return struct.pack(f"{len(names)}q", *(values.get(n, 0) for n in names))


def conv(**kw):
    base = dict(type=_lib.BF16, weight_type=_lib.BF16, batch=2, steps=100, dim=64, width=4, silu=1,
                x=at(0), x_batch=6400, x_step=64, weight=at(1), bias=at(2))
    return pack(CONV, dict(base, **kw))


def ssm(**kw):
    base = dict(type=_lib.BF16, batch=2, steps=100, dim=64, n=16, groups=1, softplus=1, x=at(0),
                x_batch=6400, x_step=64, dt=at(1), dt_batch=6400, dt_step=64, B=at(2), B_batch=1600,
                B_step=16, B_group=16, C=at(3), C_batch=1600, C_step=16, C_group=16, A=at(4))
    return pack(SSM, dict(base, **kw))


def logits(**kw):
    base = dict(type=_lib.F32, rows=4, vocab=1000, logits=at(0), logits_row=1000)
    return pack(LOGITS, dict(base, **kw))


def test_conv_refusals(lib):
    f = lib.causal_conv
    assert f(None, at(5), None, None) == _lib.EINVAL
    for bad in (dict(type=3), dict(weight_type=_lib.F16), dict(width=1), dict(width=5),
                dict(batch=-1), dict(steps=-1), dict(dim=-1), dict(x=0), dict(weight=0),
                dict(x_batch=-1), dict(x_step=-64), dict(x_step=1 << 60)):
        assert f(conv(**bad), at(5), None, None) == _lib.EINVAL, bad
    assert f(conv(), None, None, None) == _lib.EINVAL
    assert f(conv(), at(0) + 64, None, None) == _lib.EINVAL           # over x
    assert f(conv(), at(5), at(5) + 2, None) == _lib.EINVAL           # outputs over each other
    assert f(conv(state=at(6)), at(5), at(6), None) == _lib.EINVAL    # the state over itself
    for big in (dict(steps=1 << 31), dict(batch=1 << 40), dict(dim=1 << 30)):
        assert f(conv(**big), at(5), None, None) == _lib.ERANGE, big
    for empty in (dict(batch=0), dict(dim=0)):
        assert f(conv(**empty, x=0, weight=0, bias=0), None, None, None) == _lib.OK


def test_conv_backward_refusals(lib):
    size = ctypes.c_size_t(0)
    assert lib.causal_conv_scratch_bytes(conv(), ctypes.byref(size)) == _lib.OK
    assert size.value >= 5 * 64 * 4
    assert lib.causal_conv_scratch_bytes(conv(), None) == _lib.EINVAL
    assert lib.causal_conv_scratch_bytes(conv(width=9), ctypes.byref(size)) == _lib.EINVAL

    def f(p=conv(), dy=at(4), so=None, dx=at(5), dw=at(6), db=at(7), ds=None, scratch=at(8),
          n=size.value):
        return lib.causal_conv_backward(p, dy, 6400, 64, so, dx, dw, db, ds, scratch, n, None)

    for bad in (dict(dy=None), dict(dx=None), dict(dw=None), dict(scratch=None),
                dict(scratch=at(8) + 4), dict(dx=at(4)), dict(dw=at(5)), dict(db=at(1)),
                dict(ds=at(6)), dict(scratch=at(5))):
        assert f(**bad) == _lib.EINVAL, bad
    assert f(n=size.value - 1) == _lib.ENOSPACE
    assert lib.causal_conv_backward(conv(), at(4), -1, 64, None, at(5), at(6), at(7), None, at(8),
                                    size.value, None) == _lib.EINVAL


def test_step_refusals(lib):
    one = dict(steps=1)
    c, s = lib.causal_conv_step, lib.selective_scan_step
    for f, p, bad in ((c, conv, conv(steps=2)), (s, ssm, ssm(steps=2))):
        assert f(bad, at(8), 4, None, at(9), None) == _lib.EINVAL
        assert f(p(**one, state=at(7)), at(8), 4, None, at(9), None) == _lib.EINVAL
        assert f(p(**one, lengths=at(7)), at(8), 4, None, at(9), None) == _lib.EINVAL
        assert f(p(**one), None, 4, None, at(9), None) == _lib.EINVAL
        assert f(p(**one), at(8), -1, None, at(9), None) == _lib.EINVAL
        assert f(p(**one), at(8), 4, None, None, None) == _lib.EINVAL
        assert f(p(**one), at(8), 4, None, at(8) + 16, None) == _lib.EINVAL  # y in the pool
        assert f(p(**one), at(0), 4, None, at(9), None) == _lib.EINVAL       # the pool over x
        assert f(p(**one), at(8), 4, at(8), at(9), None) == _lib.EINVAL      # slots in the pool
        assert f(p(**one), at(8), 1 << 60, None, at(9), None) == _lib.ERANGE
        assert f(p(**one, batch=0), None, 0, None, None, None) == _lib.OK


def test_scan_refusals(lib):
    f = lib.selective_scan
    n = [ctypes.c_size_t(0) for _ in range(3)]
    assert lib.selective_scan_bytes(ssm(), *map(ctypes.byref, n)) == _lib.OK
    assert n[0].value == 2 * 7 * 64 * 16 * 4      # a state before every 16th of 100 tokens
    big = 1 << 30

    def run(p=ssm(), y=at(10), so=None, ck=None, scratch=at(12), size=big):
        return f(p, y, so, ck, scratch, size, None)

    for bad in (dict(type=9), dict(n=0), dict(groups=0), dict(groups=3), dict(dim=-4), dict(x=0),
                dict(dt=0), dict(B=0), dict(C=0), dict(A=0), dict(x_batch=-1), dict(C_group=-1),
                dict(B_step=1 << 60)):
        assert run(ssm(**bad)) == _lib.EINVAL, bad
    assert run(ssm(n=65)) == _lib.ERANGE
    assert run(ssm(batch=1 << 30)) == _lib.ERANGE
    assert run(y=None) == _lib.EINVAL
    assert run(y=at(3)) == _lib.EINVAL
    assert run(so=at(10)) == _lib.EINVAL
    assert run(ck=at(4)) == _lib.EINVAL
    assert run(ssm(state=at(11)), so=at(11)) == _lib.EINVAL
    if n[1].value:
        assert run(scratch=None) == _lib.EINVAL
        assert run(scratch=at(12) + 8) == _lib.EINVAL
        assert run(size=n[1].value - 1) == _lib.ENOSPACE
        assert run(scratch=at(10)) == _lib.EINVAL


def test_scan_backward_refusals(lib):
    n = [ctypes.c_size_t(0) for _ in range(3)]
    full = ssm(D=at(5), z=at(6), z_batch=6400, z_step=64, dt_bias=at(7))
    assert lib.selective_scan_bytes(full, *map(ctypes.byref, n)) == _lib.OK
    names = "dx ddt dA dB dC dD dz ddt_bias dstate".split()
    good = dict(zip(names, (at(20 + i) for i in range(9))), dy=at(18), ck=at(19), so=None,
                scratch=at(30), size=n[2].value)

    def run(p=full, **kw):
        v = dict(good, **kw)
        return lib.selective_scan_backward(p, v["dy"], 6400, 64, v["ck"], v["so"],
                                           *(v[k] for k in names), v["scratch"], v["size"], None)

    for k in names[:-1] + ["dy", "ck", "scratch"]:
        assert run(**{k: None}) == _lib.EINVAL, k
    for k in names:
        assert run(**{k: at(18)}) == _lib.EINVAL, k        # over dy
        assert run(**{k: at(30)}) == _lib.EINVAL, k        # over the scratch
    assert run(so=at(28)) == _lib.EINVAL                   # dstate over dstate_out
    assert run(size=n[2].value - 1) == _lib.ENOSPACE


def test_logits_refusals(lib):
    f = lib.logits_process
    for bad in (dict(type=-1), dict(rows=-1), dict(vocab=-1), dict(logits=0), dict(biases=3),
                dict(history_cols=-1), dict(biases=-1), dict(logits_row=-5),
                dict(history=at(5), history_row=-1, history_cols=7)):
        assert f(logits(**bad), at(9), 1000, None) == _lib.EINVAL, bad
    assert f(logits(), None, 1000, None) == _lib.EINVAL
    assert f(logits(), at(9), 999, None) == _lib.EINVAL               # rows over each other
    assert f(logits(), at(0) + 4, 1000, None) == _lib.EINVAL          # nearly in place
    assert f(logits(), at(0), 1001, None) == _lib.EINVAL
    assert f(logits(allowed=at(9), allowed_row=32), at(9), 1000, None) == _lib.EINVAL
    assert f(logits(vocab=1 << 31), at(9), 1 << 31, None) == _lib.ERANGE
    assert f(logits(rows=1 << 40), at(9), 1000, None) == _lib.ERANGE
    assert f(logits(rows=0, logits=0), None, 0, None) == _lib.OK
    size = ctypes.c_size_t(0)
    assert lib.logits_scratch_bytes(logits(vocab=50000), ctypes.byref(size)) == _lib.OK
    assert size.value > 0
    g = lib.logits_probs
    assert g(logits(vocab=50000, logits_row=50000), at(9), at(10), size.value - 1,
             None) == _lib.ENOSPACE
    assert g(logits(vocab=50000, logits_row=50000), at(9), None, 1 << 20, None) == _lib.EINVAL
    assert g(logits(vocab=50000, logits_row=50000), at(9), at(10) + 4, 1 << 20,
             None) == _lib.EINVAL
    assert g(logits(vocab=50000, logits_row=50000), at(9), at(9) + 64, 1 << 20,
             None) == _lib.EINVAL
    assert g(logits(), at(0), at(10), 1 << 20, None) == _lib.EINVAL   # probabilities over logits


def test_binding_needs_gpu_tensors():
    x, w = torch.zeros(1, 4, 8), torch.zeros(8, 4)
    with pytest.raises(ValueError, match="GPU"):
        ops.causal_conv(x, w)
    with pytest.raises(ValueError, match="GPU"):
        ops.selective_scan(x, x, torch.zeros(8, 2), torch.zeros(1, 4, 1, 2), torch.zeros(1, 4, 1, 2))
    with pytest.raises(ValueError, match="GPU"):
        ops.logits_probs(torch.zeros(2, 10))
    with pytest.raises(TypeError, match="torch.Tensor"):
        ops.logits_process([1.0])
    with pytest.raises(TypeError, match="float32, float16 or bfloat16"):
        ops.logits_process(torch.zeros(2, 10, dtype=torch.float64))


def test_scratch_of_another_gpu_is_refused(monkeypatch):
    """(Stand-ins: a kernel of one GPU must not get memory of another.)"""
    class On:
        def __init__(self, i):
            self.i, self.device = i, f"cuda:{i}"

        def get_device(self):
            return self.i

    monkeypatch.setattr(ops, "_check", lambda *a, **k: None)
    here, there = On(0), On(1)
    assert ops._scratch_for(here, 16, On(0)) is here
    with pytest.raises(ValueError, match="scratch_buf"):
        ops._scratch_for(there, 16, On(0))
