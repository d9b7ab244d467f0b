"""Tensor-level binding of libscan: argument marshalling only.

Each function checks dtype / device / contiguity, allocates missing outputs and
the workspace with torch (device memory plumbing), and calls the C entry point
of the same name on the current torch stream.  Every step of the computation
runs in libscan's HIP kernels; there is no fallback path.
"""
import ctypes
import importlib.util
import os

import torch

from . import _lib

_DT = {torch.int32: "i32", torch.float32: "f32", torch.float16: "f16", torch.uint8: "u8"}


def _check(t, dtype, name, dims=None):
    if not isinstance(t, torch.Tensor):
        raise TypeError(f"{name}: expected a torch.Tensor")
    if t.dtype != dtype:
        raise TypeError(f"{name}: expected {dtype}, got {t.dtype}")
    if not t.is_cuda:
        raise ValueError(f"{name}: expected a GPU tensor, got {t.device}")
    if not t.is_contiguous():
        raise ValueError(f"{name}: must be contiguous")
    if dims is not None and t.dim() not in dims:
        raise ValueError(f"{name}: expected {dims} dims, got {t.dim()}")


def _ptr(t):
    return t.data_ptr() if t is not None and t.numel() > 0 else None


def _launch(cname, t, *args):
    """Call entry point cname with args and, last, the current stream of t's
    device, which is made the current device if it is not.  Plain integers and
    the raw stream handle: a device context, a Stream object and a pointer
    object per argument cost more than the call itself (11.1 us a call of a
    65536-element scan with them, 6.4 without; its kernel takes 4.5)."""
    i = t.get_device()
    stream = torch._C._cuda_getCurrentRawStream(i)
    if i == torch.cuda.current_device():
        _lib.call(cname, *args, stream)
    else:
        with torch.cuda.device(i):
            _lib.call(cname, *args, stream)


def workspace(op: int, device, n: int = 0, rows: int = 0, length: int = 0, bits: int = 0):
    """A ready (zero-filled) device workspace big enough for op at these sizes.

    It can be reused by any later call of any op on the same stream."""
    nbytes = _lib.workspace_bytes(op, n, rows, length, bits)
    nbytes = max(16, (nbytes + 15) // 16 * 16)
    ws = torch.empty(nbytes, dtype=torch.uint8, device=device)
    _launch("libscan_workspace_init", ws, _ptr(ws), nbytes)
    return ws


def workspace_error(ws, reset=True):
    """The workspace's error word (0 or 1), read back to the host (this
    synchronises the stream); reset clears it.  1 means a call since the last
    reset gave up a bounded wait for another workgroup, so its outputs are
    unspecified (a workspace not zero-filled before first use, written by
    something else, or shared by concurrent calls)."""
    out = torch.zeros(1, dtype=torch.int32, device=ws.device)
    _launch("libscan_workspace_error", ws, _ptr(ws), ws.numel(), out.data_ptr(), int(bool(reset)))
    return int(out.item())


# Checked mode: every call below then reads the workspace's error word after
# it (one stream synchronisation per call) and raises if it is set.
CHECKED = os.environ.get("LIBSCAN_CHECKED", "0") == "1"


def set_checked(on: bool):
    global CHECKED
    CHECKED = bool(on)


def _done(ws, name):
    if CHECKED and workspace_error(ws) != 0:
        raise _lib.LibscanError(name + " (workspace error word set)", _lib.EHIP, _lib.load())


def _out(x, out, dtype, shape=None):
    if out is None and type(x) is torch.Tensor:  # half the time of torch.empty on the device
        return torch.empty_like(x, dtype=dtype) if shape is None \
            else x.new_empty(shape, dtype=dtype)
    shape = x.shape if shape is None else shape
    if out is None:
        return torch.empty(shape, dtype=dtype, device=x.device)
    _check(out, dtype, "out")
    if tuple(out.shape) != tuple(shape):
        raise ValueError(f"out: expected shape {tuple(shape)}, got {tuple(out.shape)}")
    return out


def _scan1d(cname, x, in_dtype, out_dtype, out, ws, extra=()):
    _check(x, in_dtype, "x")
    y = _out(x, out, out_dtype)
    n = x.numel()
    op = _lib.OP_SCAN_RSS if "_rss_" in cname else _lib.OP_SCAN
    if ws is None:
        ws = workspace(op, x.device, n)
    _launch(cname, x, _ptr(x), _ptr(y), n, *extra, _ptr(ws), ws.numel())
    _done(ws, cname)
    return y


def scan_inclusive_i32(x, out=None, ws=None):
    return _scan1d("scan_inclusive_i32", x, torch.int32, torch.int32, out, ws)


def scan_exclusive_i32(x, out=None, ws=None):
    return _scan1d("scan_exclusive_i32", x, torch.int32, torch.int32, out, ws)


def scan_inclusive_f32(x, out=None, ws=None):
    return _scan1d("scan_inclusive_f32", x, torch.float32, torch.float32, out, ws)


def scan_exclusive_f32(x, out=None, ws=None):
    return _scan1d("scan_exclusive_f32", x, torch.float32, torch.float32, out, ws)


def scan_inclusive_f16f32(x, out=None, ws=None):
    return _scan1d("scan_inclusive_f16f32", x, torch.float16, torch.float32, out, ws)


def scan_exclusive_f16f32(x, out=None, ws=None):
    return _scan1d("scan_exclusive_f16f32", x, torch.float16, torch.float32, out, ws)


def scan_inclusive_f16f32_mfma(x, out=None, ws=None):
    """Inclusive fp16 -> fp32 scan with the row scans on the matrix cores."""
    return _scan1d("scan_inclusive_f16f32_mfma", x, torch.float16, torch.float32, out, ws)


def scan_inclusive_f16f32_wave(x, out=None, ws=None):
    """Inclusive fp16 -> fp32 scan on the wavefront tiles only."""
    return _scan1d("scan_inclusive_f16f32_wave", x, torch.float16, torch.float32, out, ws)


def _scan_u8(cname, x, out, total, ws):
    if total is None:
        total = torch.empty(1, dtype=torch.int32, device=x.device)
    else:
        _check(total, torch.int32, "total")
    y = _scan1d(cname, x, torch.uint8, torch.int32, out, ws,
                extra=(total.data_ptr(),))
    return y, total


def scan_exclusive_u8i32(x, out=None, total=None, ws=None):
    """Returns (y, total) -- total is a 1-element int32 device tensor."""
    return _scan_u8("scan_exclusive_u8i32", x, out, total, ws)


def scan_exclusive_u8i32_mfma(x, out=None, total=None, ws=None):
    """The byte scan with the row scans on the matrix cores (x 16-byte aligned)."""
    return _scan_u8("scan_exclusive_u8i32_mfma", x, out, total, ws)


def scan_exclusive_u8i32_wave(x, out=None, total=None, ws=None):
    """The byte scan on the wavefront tiles only."""
    return _scan_u8("scan_exclusive_u8i32_wave", x, out, total, ws)


def _carry(cname, dtype, x, carry_in, out, total_out, ws):
    if carry_in is not None:
        _check(carry_in, dtype, "carry_in")
    if total_out is None:
        total_out = torch.empty(1, dtype=dtype, device=x.device)
    else:
        _check(total_out, dtype, "total_out")
    cin = carry_in.data_ptr() if carry_in is not None else None
    y = _scan1d(cname, x, dtype, dtype, out, ws,
                extra=(cin, total_out.data_ptr()))
    return y, total_out


def scan_inclusive_i32_carry(x, carry_in=None, out=None, total_out=None, ws=None):
    return _carry("scan_inclusive_i32_carry", torch.int32, x, carry_in, out, total_out, ws)


def scan_exclusive_i32_carry(x, carry_in=None, out=None, total_out=None, ws=None):
    return _carry("scan_exclusive_i32_carry", torch.int32, x, carry_in, out, total_out, ws)


def scan_inclusive_f32_carry(x, carry_in=None, out=None, total_out=None, ws=None):
    return _carry("scan_inclusive_f32_carry", torch.float32, x, carry_in, out, total_out, ws)


def scan_exclusive_f32_carry(x, carry_in=None, out=None, total_out=None, ws=None):
    return _carry("scan_exclusive_f32_carry", torch.float32, x, carry_in, out, total_out, ws)


def scan_inclusive_rss_i32(x, out=None, ws=None):
    return _scan1d("scan_inclusive_rss_i32", x, torch.int32, torch.int32, out, ws)


def scan_inclusive_rss_f32(x, out=None, ws=None):
    return _scan1d("scan_inclusive_rss_f32", x, torch.float32, torch.float32, out, ws)


def _rows(cname, x, dtype, exclusive, out, ws):
    _check(x, dtype, "x", dims=(2,))
    rows, length = x.shape
    y = _out(x, out, dtype)
    if ws is None:
        ws = workspace(_lib.OP_SCAN_ROWS, x.device, rows=rows, length=length)
    _launch(cname, x, _ptr(x), _ptr(y), rows, length, int(bool(exclusive)), _ptr(ws), ws.numel())
    _done(ws, cname)
    return y


def scan_rows_i32(x, exclusive=False, out=None, ws=None):
    """Independent scan of every row of a 2-D int32 tensor."""
    return _rows("scan_rows_i32", x, torch.int32, exclusive, out, ws)


def scan_rows_f32(x, exclusive=False, out=None, ws=None):
    """Independent scan of every row of a 2-D fp32 tensor."""
    return _rows("scan_rows_f32", x, torch.float32, exclusive, out, ws)


def topp_cutoff_f32(probs, p, out=None, ws=None):
    """Per row of descending-sorted probabilities: first index whose running
    sum reaches p (int32 tensor of shape [rows])."""
    _check(probs, torch.float32, "probs", dims=(2,))
    rows, length = probs.shape
    cut = _out(probs, out, torch.int32, shape=(rows,))
    if ws is None:
        ws = workspace(_lib.OP_SCAN_ROWS, probs.device, rows=rows, length=length)
    _launch("topp_cutoff_f32", probs, _ptr(probs), _ptr(cut), rows, length, float(p), _ptr(ws),
            ws.numel())
    _done(ws, "topp_cutoff_f32")
    return cut


def compact_by_mask_f32(x, mask, with_idx=False, out=None, idx_out=None, count=None, ws=None):
    """torch.masked_select order.  Returns (out, idx_out or None, count) with
    out/idx_out sized n (the first count entries are valid) and count a
    1-element int32 device tensor."""
    _check(x, torch.float32, "x")
    if mask.dtype == torch.bool:
        mask = mask.view(torch.uint8)
    _check(mask, torch.uint8, "mask")
    if mask.numel() != x.numel():
        raise ValueError("mask and x differ in size")
    n = x.numel()
    out = _out(x, out, torch.float32, shape=(n,))
    if with_idx and idx_out is None:
        idx_out = torch.empty(n, dtype=torch.int32, device=x.device)
    if count is None:
        count = torch.empty(1, dtype=torch.int32, device=x.device)
    if ws is None:
        ws = workspace(_lib.OP_COMPACT, x.device, n)
    _launch("compact_by_mask_f32", x, _ptr(x), _ptr(mask), _ptr(out), _ptr(idx_out),
            count.data_ptr(), n, _ptr(ws), ws.numel())
    _done(ws, "compact_by_mask_f32")
    return out, idx_out, count


def split_by_flags_u32(keys, flags, idx_in=None, with_idx=True, keys_out=None, idx_out=None,
                       n_true=None, ws=None):
    """Stable split: flagged keys first.  keys are uint32 values held in an
    int32 tensor (torch has no uint32 arithmetic); returns
    (keys_out, idx_out or None, n_true)."""
    _check(keys, torch.int32, "keys")
    if flags.dtype == torch.bool:
        flags = flags.view(torch.uint8)
    _check(flags, torch.uint8, "flags")
    n = keys.numel()
    if flags.numel() != n:
        raise ValueError("flags and keys differ in size")
    if idx_in is not None:
        _check(idx_in, torch.int32, "idx_in")
    keys_out = _out(keys, keys_out, torch.int32, shape=(n,))
    if with_idx and idx_out is None:
        idx_out = torch.empty(n, dtype=torch.int32, device=keys.device)
    if n_true is None:
        n_true = torch.empty(1, dtype=torch.int32, device=keys.device)
    if ws is None:
        ws = workspace(_lib.OP_COMPACT, keys.device, n)
    _launch("split_by_flags_u32", keys, _ptr(keys), _ptr(idx_in), _ptr(flags), _ptr(keys_out),
            _ptr(idx_out), n_true.data_ptr(), n, _ptr(ws), ws.numel())
    _done(ws, "split_by_flags_u32")
    return keys_out, idx_out, n_true


def radix_sort_u32(keys, bits_per_pass=8, with_perm=True, keys_out=None, perm_out=None,
                   keys_tmp=None, perm_tmp=None, ws=None):
    """Stable ascending sort of uint32 keys (held in an int32 tensor; compare
    them as unsigned), 1, 4 or 8 key bits per pass (8, the fewest passes, by
    default).  Returns (keys_out, perm_out or None)."""
    _check(keys, torch.int32, "keys")
    n = keys.numel()
    dev = keys.device
    keys_out = _out(keys, keys_out, torch.int32, shape=(n,))
    keys_tmp = torch.empty(n, dtype=torch.int32, device=dev) if keys_tmp is None else keys_tmp
    if with_perm:
        perm_out = torch.empty(n, dtype=torch.int32, device=dev) if perm_out is None else perm_out
        perm_tmp = torch.empty(n, dtype=torch.int32, device=dev) if perm_tmp is None else perm_tmp
    else:
        perm_out = perm_tmp = None
    if ws is None:
        ws = workspace(_lib.OP_RADIX_SORT, dev, n, bits=bits_per_pass)
    _launch("radix_sort_u32", keys, _ptr(keys), _ptr(keys_out), _ptr(perm_out), _ptr(keys_tmp),
            _ptr(perm_tmp), n, int(bits_per_pass), _ptr(ws), ws.numel())
    _done(ws, "radix_sort_u32")
    return keys_out, perm_out


def _radix_sort_typed(cname, keys, dtype, descending, with_perm, keys_out, perm_out, keys_tmp,
                      perm_tmp, ws):
    _check(keys, dtype, "keys")
    n = keys.numel()
    dev = keys.device
    keys_out = _out(keys, keys_out, dtype, shape=(n,))
    keys_tmp = torch.empty(n, dtype=dtype, device=dev) if keys_tmp is None else keys_tmp
    if with_perm:
        perm_out = torch.empty(n, dtype=torch.int32, device=dev) if perm_out is None else perm_out
        perm_tmp = torch.empty(n, dtype=torch.int32, device=dev) if perm_tmp is None else perm_tmp
    else:
        perm_out = perm_tmp = None
    if ws is None:
        ws = workspace(_lib.OP_RADIX_SORT, dev, n, bits=8)
    _launch(cname, keys, _ptr(keys), _ptr(keys_out), _ptr(perm_out), _ptr(keys_tmp), _ptr(perm_tmp),
            n, int(bool(descending)), _ptr(ws), ws.numel())
    _done(ws, cname)
    return keys_out, perm_out


def radix_sort_i32(keys, descending=False, with_perm=True, keys_out=None, perm_out=None,
                   keys_tmp=None, perm_tmp=None, ws=None):
    """Stable sort of int32 keys, ascending or descending.  Returns (keys_out, perm_out or None)."""
    return _radix_sort_typed("radix_sort_i32", keys, torch.int32, descending, with_perm, keys_out,
                             perm_out, keys_tmp, perm_tmp, ws)


def radix_sort_f32(keys, descending=False, with_perm=True, keys_out=None, perm_out=None,
                   keys_tmp=None, perm_tmp=None, ws=None):
    """Stable sort of float32 keys in IEEE 754 totalOrder (-NaN < -Inf < ... < -0 < +0 < ... <
    +Inf < +NaN), ascending or descending.  Returns (keys_out, perm_out or None)."""
    return _radix_sort_typed("radix_sort_f32", keys, torch.float32, descending, with_perm,
                             keys_out, perm_out, keys_tmp, perm_tmp, ws)


def radix_sort_f16(keys, descending=False, with_perm=True, keys_out=None, perm_out=None,
                   keys_tmp=None, perm_tmp=None, ws=None):
    """Stable sort of float16 keys in IEEE 754 totalOrder, ascending or descending."""
    return _radix_sort_typed("radix_sort_f16", keys, torch.float16, descending, with_perm,
                             keys_out, perm_out, keys_tmp, perm_tmp, ws)


def radix_sort_rows_f32(keys, descending=False, with_perm=True, keys_out=None, perm_out=None,
                        keys_tmp=None, perm_tmp=None, ws=None):
    """Stable sort of every row of a 2-D float32 tensor on its own (IEEE 754
    totalOrder).  perm_out holds indices within the row.  Returns (keys_out,
    perm_out or None)."""
    _check(keys, torch.float32, "keys", dims=(2,))
    rows, length = keys.shape
    dev = keys.device
    keys_out = _out(keys, keys_out, torch.float32)
    keys_tmp = torch.empty_like(keys) if keys_tmp is None else keys_tmp
    if with_perm:
        perm_out = _out(keys, perm_out, torch.int32)
        perm_tmp = torch.empty(keys.shape, dtype=torch.int32, device=dev) if perm_tmp is None \
            else perm_tmp
    else:
        perm_out = perm_tmp = None
    if ws is None:
        ws = workspace(_lib.OP_SORT_ROWS, dev, rows=rows, length=length)
    _launch("radix_sort_rows_f32", keys, _ptr(keys), _ptr(keys_out), _ptr(perm_out), _ptr(keys_tmp),
            _ptr(perm_tmp), rows, length, int(bool(descending)), _ptr(ws), ws.numel())
    _done(ws, "radix_sort_rows_f32")
    return keys_out, perm_out


def weighted_sample_f32(w, theta, out=None, ws=None):
    """Per row of non-negative weights: the index drawn by inverse transform
    with the uniform draw theta[row] (int32 tensor of shape [rows])."""
    _check(w, torch.float32, "w", dims=(2,))
    rows, length = w.shape
    _check(theta, torch.float32, "theta", dims=(1,))
    if theta.numel() != rows:
        raise ValueError(f"theta: expected {rows} draws, got {theta.numel()}")
    tok = _out(w, out, torch.int32, shape=(rows,))
    if ws is None:
        ws = workspace(_lib.OP_WEIGHTED_SAMPLE, w.device, rows=rows, length=length)
    _launch("weighted_sample_f32", w, _ptr(w), _ptr(theta), _ptr(tok), rows, length, _ptr(ws),
            ws.numel())
    _done(ws, "weighted_sample_f32")
    return tok


def scratch(op: int, device, rows: int, length: int, k: int = 0):
    """Scratch device memory for op at these sizes (no initialisation needed)."""
    nbytes = max(16, _lib.scratch_bytes(op, rows, length, k))
    return torch.empty(nbytes, dtype=torch.uint8, device=device)


def topp_sample_f32(probs, theta, p, with_cutoff=False, out=None, cutoff_out=None, ws=None,
                    scratch_buf=None):
    """Top-p sampling on unsorted rows: per row, the token drawn with the
    uniform draw theta[row] from the smallest descending-sorted prefix whose
    mass reaches p.  Returns the int32 tokens, and the cutoffs (index in the
    sorted row) when with_cutoff."""
    _check(probs, torch.float32, "probs", dims=(2,))
    rows, length = probs.shape
    _check(theta, torch.float32, "theta", dims=(1,))
    if theta.numel() != rows:
        raise ValueError(f"theta: expected {rows} draws, got {theta.numel()}")
    tok = _out(probs, out, torch.int32, shape=(rows,))
    cut = _out(probs, cutoff_out, torch.int32, shape=(rows,)) if with_cutoff else None
    if ws is None:
        ws = workspace(_lib.OP_TOPP_SAMPLE, probs.device, rows=rows, length=length)
    if scratch_buf is None:
        scratch_buf = scratch(_lib.OP_TOPP_SAMPLE, probs.device, rows, length)
    _launch("topp_sample_f32", probs, _ptr(probs), _ptr(theta), float(p), _ptr(tok), _ptr(cut),
            rows, length, _ptr(scratch_buf), scratch_buf.numel(), _ptr(ws), ws.numel())
    _done(ws, "topp_sample_f32")
    return (tok, cut) if with_cutoff else tok


def topk_rows_f32(x, k, largest=True, values_out=None, idx_out=None, ws=None, scratch_buf=None):
    """Per row of a 2-D float32 tensor, the k largest (or smallest) values in
    IEEE 754 totalOrder, in order, equal values by index.  Returns (values,
    int32 indices within the row), both rows x k."""
    _check(x, torch.float32, "x", dims=(2,))
    rows, length = x.shape
    k = int(k)
    vals = _out(x, values_out, torch.float32, shape=(rows, k))
    idx = _out(x, idx_out, torch.int32, shape=(rows, k))
    if ws is None:
        ws = workspace(_lib.OP_TOPK, x.device, k, rows=rows, length=length)
    if scratch_buf is None:
        scratch_buf = scratch(_lib.OP_TOPK, x.device, rows, length, k)
    _launch("topk_rows_f32", x, _ptr(x), _ptr(vals), _ptr(idx), rows, length, k, int(bool(largest)),
            _ptr(scratch_buf), scratch_buf.numel(), _ptr(ws), ws.numel())
    _done(ws, "topk_rows_f32")
    return vals, idx


# ---------------------------------------------------------------- language model operators
#
# None of these records an autograd graph; where an argument would have it recorded,
# a UserWarning says so.  A torch.autograd.Function that calls an operator and its
# *_backward is what training takes (examples/state_space_lm.py has one for each).

class _Args:
    """The compiled checks of torch_args.cpp, loaded at the first use: conv, ssm, attend,
    norm and logits check an operator's tensors and return its struct's bytes."""

    def __getattr__(self, name):
        path = os.path.join(_lib.PKG, "_torch_args.so")
        if not os.path.exists(path):
            raise RuntimeError(f"{path} is not built; run `python -m paper_2505_15112_amd.build`")
        spec = importlib.util.spec_from_file_location("_torch_args", path)
        module = importlib.util.module_from_spec(spec)
        spec.loader.exec_module(module)
        names = ("conv", "ssm", "attend", "norm", "logits", "dense", "empty", "sizes", "memory", "floats")
        self.__dict__.update({k: getattr(module, k) for k in names})
        return self.__dict__[name]


_args = _Args()


def _into(out, like, shape=None, f32=False, name="out"):
    """The given output, checked, or a new one: of like's shape and type unless said."""
    if out is None:
        if shape is None:
            return _args.empty(like, f32)
        return torch.empty(shape, dtype=torch.float32 if f32 else like.dtype, device=like.device)
    _args.dense(out, name, like, tuple(like.shape) if shape is None else shape, f32)
    return out


def _scratch_for(buf, nbytes, like):
    """Scratch memory of at least nbytes: the caller's, or new."""
    if buf is None:
        return _args.memory(max(16, nbytes), like)
    _check(buf, torch.uint8, "scratch_buf")
    if buf.get_device() != like.get_device():
        raise ValueError(f"scratch_buf: expected memory on the operands' GPU, got {buf.device}")
    return buf


def causal_conv(x, weight, bias=None, state=None, lengths=None, silu=True, with_state=False,
                out=None, state_out=None):
    """Causal depthwise convolution over time: x is batch x steps x dim, weight
    dim x width (2 to 4; its last column meets the newest input), state the
    batch x (width-1) x dim inputs before the first.  Returns (y, state_out): the
    last width-1 inputs of every row when with_state (or state_out is given),
    else None."""
    p = _args.conv(x, weight, bias, state, lengths, silu, False)
    y = _into(out, x)
    if with_state or state_out is not None:
        state_out = _into(state_out, x, (x.shape[0], weight.shape[1] - 1, x.shape[2]),
                          name="state_out")
    _launch("causal_conv", x, p, _ptr(y), _ptr(state_out))
    return y, state_out


def causal_conv_backward(dy, x, weight, bias=None, state=None, lengths=None, silu=True,
                         dstate_out=None, with_dstate=None, scratch_buf=None):
    """Gradients of causal_conv from those of its outputs.  Returns (dx, dweight
    fp32, dbias fp32 or None, dstate or None: by default formed when there is
    a state)."""
    p = _args.conv(x, weight, bias, state, lengths, silu, False)
    (batch, _, dim), width = x.shape, weight.shape[1]
    pdy = _strided(dy, "dy", x)
    pso = _args.dense(dstate_out, "dstate_out", x, (batch, width - 1, dim), False)
    dx = _args.empty(x, False)
    dweight = _args.empty(weight, True)
    dbias = _args.empty(bias, True) if bias is not None else None
    if with_dstate is None:
        with_dstate = state is not None
    dstate = _into(None, x, (batch, width - 1, dim)) if with_dstate else None
    need = _sizes("causal_conv_scratch_bytes", p, 1)[0]
    buf = _scratch_for(scratch_buf, need, x)
    _launch("causal_conv_backward", x, p, pdy, dy.stride(0), dy.stride(1), pso, _ptr(dx),
            _ptr(dweight), _ptr(dbias), _ptr(dstate), _ptr(buf), buf.numel())
    return dx, dweight, dbias, dstate


def _strided(t, name, like):
    """Check an operand of like's type, shape and GPU whose last dimension has unit
    stride; returns its address."""
    if not isinstance(t, torch.Tensor):
        raise TypeError(f"{name}: expected a torch.Tensor")
    if t.dtype != like.dtype:
        raise TypeError(f"{name}: expected {like.dtype}, got {t.dtype}")
    if t.shape != like.shape or t.get_device() != like.get_device():
        raise ValueError(f"{name}: expected shape {tuple(like.shape)} on {like.device}, got "
                         f"{tuple(t.shape)} on {t.device}")
    if t.shape[-1] > 1 and t.stride(-1) != 1 and t.numel() > 0:
        raise ValueError(f"{name}: the last dimension must have unit stride")
    return _ptr(t)


def _sizes(cname, p, count):
    """What a size query of libscan.h reports for a struct."""
    status, *got = _args.sizes(_lib.address(cname), p, count)
    if status != _lib.OK:
        raise _lib.LibscanError(cname, status, _lib.load())
    return got


def _pool(states, x, tail, f32, slots):
    """Check a pool of states and the rows' numbers in it."""
    if not isinstance(states, torch.Tensor):
        raise TypeError("states: expected a torch.Tensor")
    count = states.shape[0] if states.dim() else 0
    ps = _args.dense(states, "states", x, (count, *tail), f32)
    if slots is None:
        if count < x.shape[0]:
            raise ValueError("states: fewer than the rows of x")
        return ps, count, None
    _check(slots, torch.int32, "slots", (1,))
    if slots.shape[0] != x.shape[0] or slots.get_device() != x.get_device():
        raise ValueError("slots: expected one for each row of x, on its GPU")
    return ps, count, _ptr(slots)


def causal_conv_step(x, states, weight, bias=None, slots=None, silu=True, out=None):
    """One token of every row: x is batch x dim, states a pool of (width-1) x dim
    windows (row b's is number slots[b], or b), which move on in place.
    Returns y, batch x dim."""
    p = _args.conv(x, weight, bias, None, None, silu, True)
    pool = _pool(states, x, (weight.shape[1] - 1, x.shape[1]), False, slots)
    y = _into(out, x)
    _launch("causal_conv_step", x, p, *pool, _ptr(y))
    return y


def selective_scan(x, dt, A, B, C, D=None, z=None, dt_bias=None, state=None, lengths=None,
                   softplus=True, with_state=False, with_checkpoints=False, out=None,
                   state_out=None, scratch_buf=None):
    """The selective state space scan: h[t] = exp(delta A) h[t-1] + delta B x,
    y = C h + D x, gated by silu(z), with delta = softplus(dt + dt_bias).  x, dt, z:
    batch x steps x dim; A: dim x n fp32; B, C: batch x steps x groups x n; D and
    dt_bias: dim fp32; state: batch x dim x n fp32.  Returns (y, state_out or
    None, checkpoints or None): the last state when with_state (or state_out is
    given), and what selective_scan_backward needs when with_checkpoints."""
    p = _args.ssm(x, dt, A, B, C, D, z, dt_bias, state, lengths, softplus, False)
    batch, _, dim = x.shape
    y = _into(out, x)
    if with_state or state_out is not None:
        state_out = _into(state_out, x, (batch, dim, A.shape[1]), True, "state_out")
    kept, need, _ = _sizes("selective_scan_bytes", p, 3)
    ckpt = _args.floats(kept // 4, x) if with_checkpoints else None
    buf = _scratch_for(scratch_buf, need, x) if need else None
    _launch("selective_scan", x, p, _ptr(y), _ptr(state_out), _ptr(ckpt), _ptr(buf),
            buf.numel() if buf is not None else 0)
    return y, state_out, ckpt


def selective_scan_backward(dy, checkpoints, x, dt, A, B, C, D=None, z=None, dt_bias=None,
                            state=None, lengths=None, softplus=True, dstate_out=None,
                            with_dstate=None, scratch_buf=None):
    """Gradients of selective_scan from those of its outputs (dy, and dstate_out
    of its last state), with its inputs and its checkpoints.  Returns (dx, ddt,
    dA, dB, dC, dD or None, dz or None, ddt_bias or None, dstate or None): those
    of A, D, dt_bias and state in fp32, the last by default formed when there is
    a state.  The scratch holds partial sums of dB and dC, up to n / 2 bytes for each
    token and channel (include/libscan.h, selective_scan_bytes)."""
    p = _args.ssm(x, dt, A, B, C, D, z, dt_bias, state, lengths, softplus, False)
    batch, _, dim = x.shape
    kept, _, need = _sizes("selective_scan_bytes", p, 3)
    pdy = _strided(dy, "dy", x)
    pk = _args.dense(checkpoints, "checkpoints", x, (kept // 4,), True)
    pso = _args.dense(dstate_out, "dstate_out", x, (batch, dim, A.shape[1]), True)
    if with_dstate is None:
        with_dstate = state is not None

    new = _args.empty
    dx, ddt, dA, dB, dC = new(x, False), new(x, False), new(A, True), new(B, False), new(B, False)
    dD = new(D, True) if D is not None else None
    dz = new(x, False) if z is not None else None
    dbias = new(dt_bias, True) if dt_bias is not None else None
    dstate = _into(None, x, (batch, dim, A.shape[1]), True) if with_dstate else None
    buf = _scratch_for(scratch_buf, need, x)
    _launch("selective_scan_backward", x, p, pdy, dy.stride(0), dy.stride(1), pk, pso, _ptr(dx),
            _ptr(ddt), _ptr(dA), _ptr(dB), _ptr(dC), _ptr(dD), _ptr(dz), _ptr(dbias),
            _ptr(dstate), _ptr(buf), buf.numel())
    return dx, ddt, dA, dB, dC, dD, dz, dbias, dstate


def selective_scan_step(x, dt, states, A, B, C, D=None, z=None, dt_bias=None, slots=None,
                        softplus=True, out=None):
    """One token of every row: x, dt, z: batch x dim; B, C: batch x groups x n;
    states a pool of dim x n fp32 states (row b's is number slots[b], or b),
    which move on in place.  Returns y, batch x dim."""
    p = _args.ssm(x, dt, A, B, C, D, z, dt_bias, None, None, softplus, True)
    pool = _pool(states, x, tuple(A.shape), True, slots)
    y = _into(out, x)
    _launch("selective_scan_step", x, p, *pool, _ptr(y))
    return y


def linear_attention(q, k, v, log_decay, state=None, lengths=None, scale=None, with_state=False,
                     out=None, state_out=None, scratch_buf=None):
    """Linear attention with a decay for each head: S[t] = exp(log_decay) S[t-1] +
    k v^T, y = scale q S (scale: dk ** -0.5 by default).  q, k: batch x steps x groups
    x dk; v: batch x steps x heads x dv, heads a multiple of groups; log_decay: fp32,
    batch x steps x heads, or heads: one for all tokens; state: batch x heads x dk x dv
    fp32.  Returns (y, state_out): the last state when with_state (or state_out is
    given), else None."""
    p = _args.attend(q, k, v, log_decay, state, lengths, scale, False)
    y = _into(out, v)
    if with_state or state_out is not None:
        state_out = _into(state_out, v, (v.shape[0], v.shape[2], q.shape[3], v.shape[3]), True,
                          "state_out")
    need, _ = _sizes("linear_attention_bytes", p, 2)
    buf = _scratch_for(scratch_buf, need, v) if need else None
    _launch("linear_attention", q, p, _ptr(y), _ptr(state_out), _ptr(buf),
            buf.numel() if buf is not None else 0)
    return y, state_out


def linear_attention_backward(dy, q, k, v, log_decay, state=None, lengths=None, scale=None,
                              dstate_out=None, with_dstate=None, scratch_buf=None):
    """Gradients of linear_attention from those of its outputs (dy, and dstate_out of
    its last state).  Returns (dq, dk, dv, dlog_decay fp32, dstate fp32 or None: by
    default formed when there is a state)."""
    p = _args.attend(q, k, v, log_decay, state, lengths, scale, False)
    shape = (v.shape[0], v.shape[2], q.shape[3], v.shape[3])
    pdy = _strided(dy, "dy", v)
    pso = _args.dense(dstate_out, "dstate_out", v, shape, True)
    if with_dstate is None:
        with_dstate = state is not None
    new = _args.empty
    dq, dk, dv, dg = new(q, False), new(k, False), new(v, False), new(log_decay, True)
    dstate = _into(None, v, shape, True) if with_dstate else None
    _, need = _sizes("linear_attention_bytes", p, 2)
    buf = _scratch_for(scratch_buf, need, v)
    _launch("linear_attention_backward", q, p, pdy, *dy.stride()[:3], pso, _ptr(dq), _ptr(dk),
            _ptr(dv), _ptr(dg), _ptr(dstate), _ptr(buf), buf.numel())
    return dq, dk, dv, dg, dstate


def linear_attention_step(q, k, v, log_decay, states, slots=None, scale=None, out=None):
    """One token of every row: q, k: batch x groups x dk; v: batch x heads x dv;
    log_decay: batch x heads, or heads; states a pool of heads x dk x dv fp32 states (row
    b's is number slots[b], or b), which move on in place.  Returns y, batch x heads x dv."""
    p = _args.attend(q, k, v, log_decay, None, None, scale, True)
    pool = _pool(states, v, (v.shape[1], q.shape[2], v.shape[2]), True, slots)
    y = _into(out, v)
    _launch("linear_attention_step", q, p, *pool, _ptr(y))
    return y


def layer_norm(x, weight=None, bias=None, residual=None, groups=1, eps=1e-5, with_stats=False,
               out=None, sum_out=None, stats_out=None):
    """Layer norm over each of `groups` groups of neighbouring channels: x is batch x
    steps x dim or rows x dim, weight and bias dim.  With a residual of x's shape,
    what is normalised is x + residual, rounded to x's type.  Returns (y, that sum or
    None, stats or None): the groups' means and 1 / sqrt(variance + eps), fp32, for
    layer_norm_backward, when with_stats (or stats_out is given)."""
    p = _args.norm(x, weight, bias, residual, groups, eps)
    y = _into(out, x)
    if residual is not None:
        sum_out = _into(sum_out, x, name="sum_out")
    elif sum_out is not None:
        raise ValueError("sum_out: there is no residual")
    if with_stats or stats_out is not None:
        stats_out = _into(stats_out, x, (*x.shape[:-1], groups, 2), True, "stats_out")
    _launch("layer_norm", x, p, _ptr(y), _ptr(sum_out), _ptr(stats_out))
    return y, sum_out, stats_out


def layer_norm_backward(dy, x, stats, weight=None, bias=None, dsum=None, groups=1,
                        scratch_buf=None):
    """Gradients of layer_norm from those of its outputs (dy, and dsum of the sum with the
    residual), with x what it normalised (that sum, if there was a residual) and its
    stats.  Returns (dx, which is the residual's too, dweight fp32 or None, dbias fp32
    or None)."""
    p = _args.norm(x, weight, bias, None, groups, 0.0)
    pdy = _strided(dy, "dy", x)
    more = (None, 0, 0)
    if dsum is not None:
        more = (_strided(dsum, "dsum", x), *_row_strides(dsum))
    ps = _args.dense(stats, "stats", x, (*x.shape[:-1], groups, 2), True)
    if stats is None:
        raise TypeError("stats: expected a torch.Tensor")
    dx = _args.empty(x, False)
    dweight = _args.empty(weight, True) if weight is not None else None
    dbias = _args.empty(bias, True) if bias is not None else None
    need = _sizes("layer_norm_scratch_bytes", p, 1)[0]
    buf = _scratch_for(scratch_buf, need, x)
    _launch("layer_norm_backward", x, p, pdy, *_row_strides(dy), *more, ps, _ptr(dx),
            _ptr(dweight), _ptr(dbias), _ptr(buf), buf.numel())
    return dx, dweight, dbias


def _row_strides(t):
    """The strides over batch and steps of batch x steps x dim, or rows x dim."""
    return t.stride()[:2] if t.dim() == 3 else (0, t.stride(0))


def logits_process(logits, history=None, history_len=None, prompt_len=None, repetition=None,
                   presence=None, frequency=None, bias_ids=None, bias_values=None, allowed=None,
                   out=None):
    """Penalties, biases and grammar masks on rows x vocab logits.

    history: rows x tokens int32 ids (others are skipped), of which the first
    history_len count and the first prompt_len are the prompt.  Seen tokens'
    logits are divided (positive) or multiplied by repetition; generated ones
    lose presence, and frequency per occurrence.  bias_values are added at
    bias_ids (rows x entries).  allowed holds a bit per place, lowest first, in
    rows x ceil(vocab / 32) int32 words: 0 gives -infinity.  All per row.  out may
    be logits itself."""
    p = _args.logits(logits, history, history_len, prompt_len, repetition, presence, frequency,
                     bias_ids, bias_values, allowed, None)
    if out is None:
        out = _args.empty(logits, False)
    else:
        _strided(out, "out", logits)
    _launch("logits_process", logits, p, _ptr(out), out.stride(0))
    return out


def logits_probs(logits, history=None, history_len=None, prompt_len=None, repetition=None,
                 presence=None, frequency=None, bias_ids=None, bias_values=None, allowed=None,
                 temperature=None, out=None, scratch_buf=None):
    """softmax(logits_process(...) / temperature) as fp32 rows x vocab
    probabilities, what topp_sample_f32 takes.  A temperature of 0 gives the
    largest logit's places equal shares; a row with no place left is all 0."""
    p = _args.logits(logits, history, history_len, prompt_len, repetition, presence, frequency,
                     bias_ids, bias_values, allowed, temperature)
    probs = _into(out, logits, f32=True)
    need = _sizes("logits_scratch_bytes", p, 1)[0]
    buf = _scratch_for(scratch_buf, need, logits) if need else None
    _launch("logits_probs", logits, p, _ptr(probs), _ptr(buf),
            buf.numel() if buf is not None else 0)
    return probs
