"""Linear attention and layer norm in 64 bits, written from their definitions
(CPU, torch double), and the error bounds their tests use.

Bounds.  |got - ref| <= u |ref| + r M: u is half a unit in the last place of the
output's type, M the same sums with every term replaced by its absolute value.
r for linear attention is c 2^-24 for the fp32 roundings that a term passes
through, and for outputs of 16 bits what the matrix products round of their
operands besides: scores and states are read as two bfloat16 terms, which leave
out 2^-15 of them (half a unit in the last place, 2^-8, of a rest of at most
2^-7), and so are fp16's inputs, which two terms hold exactly; the product of two
second terms, 2^-14 of the whole, is left out in each of the products that make
an output (q k, then with v; q S).  That is 2 * 2^-14 + 2^-15 < 2^-12 for fp16, and
2^-15 < 2^-14 for bfloat16, whose inputs are one term.  In fp32 three terms hold
every operand, and the products left out are below 2^-20 in all, 16 * 2^-24.
"""
import torch

from lm_ref import TINY, U, lens

F32, F16, BF16 = torch.float32, torch.float16, torch.bfloat16
OPERANDS = {F32: 0.0, F16: 2.0**-12, BF16: 2.0**-14}


def assert_within(got, ref, mag, r, what):
    g = got.detach().cpu().double()
    assert g.shape == ref.shape, (what, g.shape, ref.shape)
    tol = U[got.dtype] * ref.abs() + r * mag + TINY[got.dtype]
    bad = ~((g - ref).abs() <= tol)
    if bad.any():
        i = tuple(bad.nonzero()[0].tolist())
        raise AssertionError(f"{what}: {int(bad.sum())} of {bad.numel()} out of bounds, first at "
                             f"{i}: got {g[i]!r}, ref {ref[i]!r}, tol {tol[i]!r}")


def attend(q, k, v, log_decay, state=None, lengths=None, scale=None, dy=None, dstate_out=None,
           absolute=False):
    """Token by token.  Returns a dict: y, state and, with dy, the gradients; with
    absolute, the magnitudes of all of them (dlog_decay's are those of the sums over
    the later tokens that it is formed of)."""
    f = torch.abs if absolute else (lambda t: t)
    batch, steps, groups, dk = q.shape
    heads, dv = v.shape[2:]
    per = heads // groups
    scale = dk ** -0.5 if scale is None else scale
    scale = abs(scale) if absolute else scale
    zeros = lambda *s: torch.zeros(*s, dtype=torch.double)  # noqa: E731
    fixed = log_decay.dim() == 1
    out = dict(y=zeros(batch, steps, heads, dv), state=zeros(batch, heads, dk, dv))
    if dy is not None:
        out.update(dq=zeros(*q.shape), dk=zeros(*k.shape), dv=zeros(*v.shape),
                   dlog_decay=zeros(*log_decay.shape), dstate=zeros(batch, heads, dk, dv))
    for b, n in enumerate(lens(lengths, batch, steps)):
        h = f(state[b]) if state is not None else zeros(heads, dk, dv)
        hs = [h]
        rows = []
        for t in range(n):
            a = torch.exp(log_decay if fixed else log_decay[b, t])[:, None, None]
            qt, kt = (f(x[b, t]).repeat_interleave(per, 0) for x in (q, k))
            vt = f(v[b, t])
            h = a * h + kt[:, :, None] * vt[:, None, :]
            out["y"][b, t] = scale * (qt[:, :, None] * h).sum(1)
            hs.append(h)
            rows.append((a, qt, kt, vt))
        out["state"][b] = h
        if dy is None:
            continue
        grad = f(dstate_out[b]) if dstate_out is not None else zeros(heads, dk, dv)
        later = (grad * h).sum((1, 2))  # absolute: what the decays' sums have added up so far
        for t in reversed(range(n)):
            a, qt, kt, vt = rows[t]
            d = f(dy[b, t]) * scale
            grad = grad + qt[:, :, None] * d[:, None, :]
            dq, dk_ = (hs[t + 1] * d[:, None, :]).sum(2), (grad * vt[:, None, :]).sum(2)
            out["dq"][b, t] += dq.view(groups, per, dk).sum(1)
            out["dk"][b, t] += dk_.view(groups, per, dk).sum(1)
            out["dv"][b, t] = (grad * kt[:, :, None]).sum(1)
            later = later + (qt * dq).sum(1) + (kt * dk_).sum(1)
            dg = later if absolute else (a * grad * hs[t]).sum((1, 2))
            if fixed:
                out["dlog_decay"] += dg
            else:
                out["dlog_decay"][b, t] = dg
            grad = a * grad
        out["dstate"][b] = grad
    return out


def norm(x, weight=None, bias=None, residual=None, groups=1, eps=1e-5, dy=None, dsum=None):
    """Returns a dict: y, sum, mean, rstd and, with dy, the gradients; and the same
    of magnitudes under "m" + name.  x and residual are of their own type: their sum
    is rounded to it."""
    total = (x.double() + residual.double()).to(x.dtype) if residual is not None else x
    v = total.double().unflatten(-1, (groups, -1))
    n = v.shape[-1]
    mean = v.mean(-1, keepdim=True)
    d = v - mean
    rstd = 1 / torch.sqrt((d * d).mean(-1, keepdim=True) + eps)
    # d is off by the roundings of the mean, of at most the largest element's size
    md = v.abs() + v.abs().mean(-1, keepdim=True)
    hat, mhat = (d * rstd).flatten(-2), (md * rstd).flatten(-2)
    w = weight.double() if weight is not None else torch.ones(x.shape[-1], dtype=torch.double)
    y, my = hat * w, (mhat + hat.abs()) * w.abs()
    if bias is not None:
        y, my = y + bias.double(), my + bias.double().abs()
    out = dict(y=y, my=my, sum=total if residual is not None else None, mean=mean[..., 0],
               mmean=v.abs().mean(-1), rstd=rstd[..., 0],
               mrstd=rstd[..., 0] * (1 + 2 * (md * md).mean(-1) * rstd[..., 0] ** 2))
    if dy is not None:
        g = dy.double()
        u = (g * w).unflatten(-1, (groups, -1))
        h, mh = hat.view_as(u), (mhat + hat.abs()).view_as(u)
        dx = rstd * (u - u.mean(-1, keepdim=True) - h * (u * h).mean(-1, keepdim=True))
        mu = u.abs()
        mdx = rstd * (mu + mu.mean(-1, keepdim=True) + mh * (mu * mh).mean(-1, keepdim=True))
        dx, mdx = dx.flatten(-2), mdx.flatten(-2)
        if dsum is not None:
            dx, mdx = dx + dsum.double(), mdx + dsum.double().abs()
        lead = tuple(range(x.dim() - 1))
        out.update(dx=dx, mdx=mdx, dweight=(g * hat).sum(lead),
                   mdweight=(g.abs() * (mhat + hat.abs())).sum(lead), dbias=g.sum(lead),
                   mdbias=g.abs().sum(lead))
    return out
