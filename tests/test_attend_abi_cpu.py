"""The entry points of linear attention and layer norm on the CPU: every call here
is refused (or has nothing to do) before any HIP call, by its arguments."""
import ctypes
import os
import struct

import pytest
import torch

from paper_2505_15112_amd import _lib, ops

if not os.path.exists(_lib.LIB_PATH):
    from paper_2505_15112_amd import build as _build
    _build.build()

ATTEND = ("type batch steps heads groups dk dv fixed q q_batch q_step q_head k k_batch k_step "
          "k_head v v_batch v_step v_head log_decay decay_batch decay_step scale state "
          "lengths").split()
NORM = ("type weight_type batch steps dim groups eps x x_batch x_step residual residual_batch "
        "residual_step weight bias").split()


def at(i):
    """Fake addresses, never dereferenced, 256 MiB apart."""
    return 0x10000000 * (i + 1)


def pack(names, values):
    assert set(values) <= set(names)
    return b"".join(struct.pack("d" if n in ("scale", "eps") else "q", values.get(n, 0))
                    for n in names)


def attend(**kw):
    base = dict(type=_lib.BF16, batch=2, steps=100, heads=4, groups=2, dk=16, dv=24, q=at(0),
                q_batch=3200, q_step=32, q_head=16, k=at(1), k_batch=3200, k_step=32, k_head=16,
                v=at(2), v_batch=9600, v_step=96, v_head=24, log_decay=at(3), decay_batch=400,
                decay_step=4, scale=0.25)
    return pack(ATTEND, dict(base, **kw))


def norm(**kw):
    base = dict(type=_lib.BF16, weight_type=_lib.BF16, batch=2, steps=50, dim=64, groups=1,
                eps=1e-5, x=at(0), x_batch=3200, x_step=64, weight=at(1), bias=at(2))
    return pack(NORM, dict(base, **kw))


@pytest.fixture(scope="module")
def lib():
    return _lib.load()


def sizes(lib, p):
    n = [ctypes.c_size_t(0) for _ in range(2)]
    return lib.linear_attention_bytes(p, *map(ctypes.byref, n)), n[0].value, n[1].value


BAD = (dict(type=3), dict(type=-1), dict(batch=-1), dict(steps=-1), dict(heads=-2), dict(groups=0),
       dict(groups=3), dict(dk=0), dict(dv=0), dict(dk=-1))
BIG = (dict(dk=257), dict(dv=257), dict(heads=1 << 20), dict(batch=1 << 40), dict(steps=1 << 31),
       dict(batch=1 << 20, heads=64))


def test_attention_refusals(lib):
    status, need, _ = sizes(lib, attend())
    assert status == _lib.OK
    assert lib.linear_attention_bytes(attend(), None, None) == _lib.OK

    def run(p=attend(), y=at(10), so=None, scratch=at(12), size=need):
        return lib.linear_attention(p, y, so, scratch, size, None)

    assert run(None) == _lib.EINVAL
    for bad in BAD:
        assert run(attend(**bad)) == sizes(lib, attend(**bad))[0] == _lib.EINVAL, bad
    for big in BIG:
        assert run(attend(**big)) == sizes(lib, attend(**big))[0] == _lib.ERANGE, big
    for bad in (dict(q=0), dict(k=0), dict(v=0), dict(log_decay=0), dict(q_batch=-1),
                dict(k_head=-1), dict(v_step=1 << 60), dict(decay_step=-4)):
        assert run(attend(**bad)) == _lib.EINVAL, bad
    assert run(y=None) == _lib.EINVAL
    for over in (at(0), at(1), at(2), at(3)):
        assert run(y=over) == _lib.EINVAL and run(so=over) == _lib.EINVAL
    assert run(so=at(10)) == _lib.EINVAL
    assert run(attend(state=at(11)), so=at(11)) == _lib.EINVAL
    assert run(attend(lengths=at(10))) == _lib.EINVAL


def test_attention_scratch_is_checked(lib):
    """A long row of few heads, which is cut into pieces and needs scratch."""
    p = attend(batch=1, steps=20000, q_batch=0, k_batch=0, v_batch=0, decay_batch=0)
    status, need, back = sizes(lib, p)
    assert status == _lib.OK and back > 0
    if need:
        f = lib.linear_attention
        assert f(p, at(10), None, at(12), need - 1, None) == _lib.ENOSPACE
        assert f(p, at(10), None, None, need, None) == _lib.EINVAL
        assert f(p, at(10), None, at(12) + 8, need, None) == _lib.EINVAL
        assert f(p, at(10), None, at(2), need, None) == _lib.EINVAL


def test_attention_backward_refusals(lib):
    _, _, need = sizes(lib, attend(state=at(4)))
    names = "dq dk dv dg dstate".split()
    good = dict(zip(names, (at(20 + i) for i in range(5))), dy=at(18), so=at(19), scratch=at(30),
                size=need, strides=(9600, 96, 24))

    def run(p=attend(state=at(4)), **kw):
        v = dict(good, **kw)
        return lib.linear_attention_backward(p, v["dy"], *v["strides"], v["so"],
                                             *(v[k] for k in names), v["scratch"], v["size"], None)

    for bad in BAD:
        assert run(attend(**bad)) == _lib.EINVAL, bad
    for k in names[:-1] + ["dy", "scratch"]:
        assert run(**{k: None}) == _lib.EINVAL, k
    for k in names:
        for over in (at(18), at(19), at(30), at(0), at(4)):
            assert run(**{k: over}) == _lib.EINVAL, (k, over)
    assert run(strides=(9600, -96, 24)) == _lib.EINVAL
    assert run(size=need - 1) == _lib.ENOSPACE
    assert run(scratch=at(30) + 4) == _lib.EINVAL
    assert run(attend(fixed=1, log_decay=0)) == _lib.EINVAL


def test_attention_step_refusals(lib):
    f = lib.linear_attention_step
    one = dict(steps=1)
    assert f(attend(steps=2), at(8), 4, None, at(9), None) == _lib.EINVAL
    assert f(attend(**one, state=at(7)), at(8), 4, None, at(9), None) == _lib.EINVAL
    assert f(attend(**one, lengths=at(7)), at(8), 4, None, at(9), None) == _lib.EINVAL
    assert f(attend(**one), None, 4, None, at(9), None) == _lib.EINVAL
    assert f(attend(**one), at(8), -1, None, at(9), None) == _lib.EINVAL
    assert f(attend(**one), at(8), 4, None, None, None) == _lib.EINVAL
    assert f(attend(**one), at(8), 4, None, at(8) + 16, None) == _lib.EINVAL  # y in the pool
    assert f(attend(**one), at(0), 4, None, at(9), None) == _lib.EINVAL       # the pool over q
    assert f(attend(**one), at(8), 4, at(8), at(9), None) == _lib.EINVAL      # slots in the pool
    assert f(attend(**one), at(8), 1 << 60, None, at(9), None) == _lib.ERANGE
    assert f(attend(**one, batch=0), None, 0, None, None, None) == _lib.OK


def test_norm_refusals(lib):
    def run(p=norm(), y=at(4), total=None, stats=None):
        return lib.layer_norm(p, y, total, stats, None)

    assert run(None) == _lib.EINVAL
    for bad in (dict(type=7), dict(weight_type=_lib.F16), dict(groups=0), dict(groups=5),
                dict(eps=-1e-9), dict(eps=float("nan")), dict(batch=-1), dict(steps=-1),
                dict(dim=-64), dict(x=0), dict(x_step=-1), dict(x_batch=1 << 60),
                dict(residual=at(3), residual_step=-1)):
        assert run(norm(**bad)) == _lib.EINVAL, bad
    for big in (dict(dim=1 << 30), dict(batch=1 << 40), dict(steps=1 << 31)):
        assert run(norm(**big)) == _lib.ERANGE, big
    assert run(y=None) == _lib.EINVAL
    for over in (at(0), at(1), at(2)):
        assert run(y=over) == run(total=over) == run(stats=over) == _lib.EINVAL
    assert run(total=at(4)) == run(stats=at(4) + 64) == _lib.EINVAL
    assert run(norm(residual=at(4))) == _lib.EINVAL
    for empty in (dict(batch=0), dict(steps=0), dict(dim=0)):
        assert run(norm(**empty, x=0), None) == _lib.OK, empty


def test_norm_backward_refusals(lib):
    size = ctypes.c_size_t(0)
    assert lib.layer_norm_scratch_bytes(norm(), ctypes.byref(size)) == _lib.OK
    assert lib.layer_norm_scratch_bytes(norm(), None) == _lib.EINVAL
    assert lib.layer_norm_scratch_bytes(norm(groups=0), ctypes.byref(size)) == _lib.EINVAL
    names = "dx dw db".split()

    def run(p=norm(), **kw):
        v = dict(dict(dy=at(4), ds=at(5), stats=at(6), dx=at(7), dw=at(8), db=at(9),
                      scratch=at(10), size=size.value, step=64), **kw)
        return lib.layer_norm_backward(p, v["dy"], 3200, v["step"], v["ds"], 3200, 64, v["stats"],
                                       *(v[k] for k in names), v["scratch"], v["size"], None)

    assert run(norm(residual=at(3))) == _lib.EINVAL
    for k in ("dy", "stats", "dx", "scratch"):
        assert run(**{k: None}) == _lib.EINVAL, k
    for k in names + ["scratch"]:
        for over in (at(0), at(1), at(4), at(5), at(6)):
            assert run(**{k: over}) == _lib.EINVAL, (k, over)
    assert run(dw=at(9)) == run(step=-1) == run(scratch=at(10) + 8) == _lib.EINVAL
    assert run(size=size.value - 1) == _lib.ENOSPACE


def test_binding_needs_gpu_tensors():
    q, v = torch.zeros(1, 4, 2, 8), torch.zeros(1, 4, 2, 6)
    with pytest.raises(ValueError, match="GPU"):
        ops.linear_attention(q, q, v, torch.zeros(2))
    with pytest.raises(TypeError, match="torch.Tensor"):
        ops.linear_attention([1.0], q, v, torch.zeros(2))
    with pytest.raises(ValueError, match="GPU"):
        ops.layer_norm(torch.zeros(3, 8))
    with pytest.raises(TypeError, match="float32, float16 or bfloat16"):
        ops.layer_norm(torch.zeros(3, 8, dtype=torch.float64))
