"""Linear attention without heads, whose groups' gradients are sums over none."""
import ctypes

import pytest
import torch

from gpu_util import announce
from paper_2505_15112_amd import _lib, ops
from test_attend_abi_cpu import at, attend, lib  # noqa: F401

DEV = "cuda"


def test_arguments(lib):  # noqa: F811
    """On the CPU: the groups' gradients have to be there, and groups are bounded."""
    p = attend(heads=0)
    n = [ctypes.c_size_t(7) for _ in range(2)]
    assert lib.linear_attention_bytes(p, *map(ctypes.byref, n)) == _lib.OK
    assert n[0].value == n[1].value == 0

    def run(p, dq, dk):
        return lib.linear_attention_backward(p, None, 0, 0, 0, None, dq, dk, None, None, None,
                                             None, 0, None)

    assert run(p, None, at(9)) == run(p, at(8), None) == _lib.EINVAL
    assert run(p, at(0), at(9)) == run(p, at(8), at(8)) == _lib.EINVAL  # over q; both the same
    assert run(attend(heads=0, groups=1 << 17), at(8), at(9)) == _lib.ERANGE
    assert run(attend(heads=0, groups=1 << 60), at(8), at(9)) == _lib.ERANGE


@pytest.mark.gpu
@pytest.mark.parametrize("kind", [torch.float32, torch.float16, torch.bfloat16])
@pytest.mark.parametrize("fixed", [False, True])
def test_gradients_of_groups_without_heads(kind, fixed):
    q = torch.randn(2, 300, 3, 40, device=DEV).to(kind)
    v = torch.zeros(2, 300, 0, 24, device=DEV, dtype=kind)
    decay = torch.zeros(0, device=DEV) if fixed else torch.zeros(2, 300, 0, device=DEV)
    # what the gradients' memory may hold
    old = [torch.full_like(q, float("nan")) for _ in range(4)]
    torch.cuda.synchronize()
    del old
    announce("linear_attention_backward", tuple(q.shape), tuple(v.shape), kind)
    dq, dk, dv, dg, _ = ops.linear_attention_backward(v, q, q.clone(), v, decay)
    assert dq.shape == q.shape and dk.shape == q.shape
    assert not dq.any() and not dk.any()
    assert dv.shape == v.shape and dg.shape == decay.shape


@pytest.mark.gpu
@pytest.mark.parametrize("batch,steps", [(0, 9), (2, 0)])
def test_nothing_at_all(batch, steps):
    q, v = torch.zeros(batch, steps, 3, 40, device=DEV), torch.zeros(batch, steps, 0, 24, device=DEV)
    decay = torch.zeros(batch, steps, 0, device=DEV)
    got = ops.linear_attention_backward(v, q, q.clone(), v, decay)
    assert [t.numel() for t in got[:4]] == [0, 0, 0, 0]
