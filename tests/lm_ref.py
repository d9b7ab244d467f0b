"""Language model operators in 64 bits, written from their definitions (CPU,
torch double), and the error bounds their tests use.

Bounds.  A kernel reads its inputs exactly, computes in fp32 and rounds an
output once.  So |got - ref| <= u |ref| + c 2^-24 M: u is half a unit in the
last place of the output's type, M the same sums with every term replaced by
its absolute value, and c counts the fp32 roundings that a term passes through
(each instruction used here, exp2, rcp and log included, is good to about one
unit).  A chain of `steps` decays multiplies `steps` rounded factors, so there
c grows with steps.
"""
import torch

U = {torch.float32: 2.0**-24, torch.float16: 2.0**-11, torch.bfloat16: 2.0**-8}
TINY = {torch.float32: 2.0**-126, torch.float16: 2.0**-24, torch.bfloat16: 2.0**-126}


def assert_within(got, ref, mag, c, what):
    g = got.detach().cpu().double()
    assert g.shape == ref.shape, (what, g.shape, ref.shape)
    tol = U[got.dtype] * ref.abs() + c * 2.0**-24 * mag + TINY[got.dtype]
    bad = ~((g - ref).abs() <= tol)
    if bad.any():
        i = tuple(bad.nonzero()[0].tolist())
        raise AssertionError(f"{what}: {int(bad.sum())} of {bad.numel()} out of bounds, first at "
                             f"{i}: got {g[i]!r}, ref {ref[i]!r}, tol {tol[i]!r}")


def lens(lengths, batch, steps):
    return [steps] * batch if lengths is None else [min(max(int(v), 0), steps) for v in lengths]


def sigmoid(v):
    return 1 / (1 + torch.exp(-v))


def softplus(v):
    return torch.logaddexp(v, torch.zeros_like(v))


# ---------------------------------------------------------------- convolution

def conv(x, weight, bias, state, lengths, silu):
    """(y, last state), their magnitudes, and the preactivations u with the padded inputs."""
    batch, steps, dim = x.shape
    width = weight.shape[1]
    y, mag = torch.zeros_like(x), torch.zeros_like(x)
    last = torch.zeros(batch, width - 1, dim, dtype=torch.double)
    us, fulls = [], []
    for b, n in enumerate(lens(lengths, batch, steps)):
        before = state[b] if state is not None else torch.zeros(width - 1, dim, dtype=torch.double)
        full = torch.cat((before, x[b, :n]))
        u = torch.zeros(n, dim, dtype=torch.double)
        m = torch.zeros(n, dim, dtype=torch.double)
        if bias is not None:
            u, m = u + bias, m + bias.abs()
        for j in range(width):
            u = u + full[j:j + n] * weight[:, j]
            m = m + (full[j:j + n] * weight[:, j]).abs()
        # |d silu| <= 1.1, so an error of u comes through at most that much larger
        y[b, :n], mag[b, :n] = (u * sigmoid(u) if silu else u), 1.1 * m
        last[b] = full[n:]
        us.append(u)
        fulls.append(full)
    return y, last, mag, us, fulls


def conv_back(dy, x, weight, bias, state, lengths, silu, dstate_out=None, absolute=False):
    """dx, dweight, dbias, dstate; with absolute, their magnitudes."""
    f = torch.abs if absolute else (lambda v: v)
    batch, steps, dim = x.shape
    width = weight.shape[1]
    _, _, mag, us, fulls = conv(x, weight, bias, state, lengths, silu)
    dx, dstate = torch.zeros_like(x), torch.zeros(batch, width - 1, dim, dtype=torch.double)
    dw, db = torch.zeros_like(weight), torch.zeros(dim, dtype=torch.double)
    for b, n in enumerate(lens(lengths, batch, steps)):
        u, full = us[b], f(fulls[b])
        sig = sigmoid(u)
        slope = sig * (1 + u * (1 - sig)) if silu else torch.ones_like(u)
        if absolute:  # an error of u moves the slope by at most half of it
            slope = 1.1 + 0.5 * mag[b, :n] if silu else slope
        g = f(dy[b, :n]) * slope
        dfull = torch.zeros(n + width - 1, dim, dtype=torch.double)
        for j in range(width):
            dfull[j:j + n] += g * f(weight[:, j])
            dw[:, j] += (g * full[j:j + n]).sum(0)
        db += g.sum(0)
        if dstate_out is not None:
            dfull[n:] += f(dstate_out[b])
        dstate[b], dx[b, :n] = dfull[:width - 1], dfull[width - 1:]
    return dx, dw, db, dstate


# ---------------------------------------------------------------- selective scan

def scan(x, dt, A, B, C, D=None, z=None, dt_bias=None, state=None, lengths=None, softplus_on=True,
         dy=None, dstate_out=None, absolute=False):
    """Step by step, one row after the other.  Returns a dict: y, state and, with
    dy, the gradients; with absolute, the magnitudes of all of them."""
    f = torch.abs if absolute else (lambda v: v)
    batch, steps, dim = x.shape
    groups, n = B.shape[2:]
    per = dim // groups
    zeros = lambda *s: torch.zeros(*s, dtype=torch.double)  # noqa: E731
    out = dict(y=zeros(batch, steps, dim), state=zeros(batch, dim, n))
    if dy is not None:
        out.update(dx=zeros(batch, steps, dim), ddt=zeros(batch, steps, dim), dA=zeros(dim, n),
                   dB=zeros(batch, steps, groups, n), dC=zeros(batch, steps, groups, n),
                   dD=zeros(dim), dz=zeros(batch, steps, dim), ddt_bias=zeros(dim),
                   dstate=zeros(batch, dim, n))
    for b, count in enumerate(lens(lengths, batch, steps)):
        h = f(state[b]) if state is not None else zeros(dim, n)
        hs, decays, deltas, cores = [h], [], [], []
        for t in range(count):
            v = dt[b, t] + (dt_bias if dt_bias is not None else 0)
            delta = softplus(v) if softplus_on else v
            a = torch.exp(delta[:, None] * A)
            Bt = f(B[b, t]).repeat_interleave(per, 0)
            Ct = f(C[b, t]).repeat_interleave(per, 0)
            h = a * h + (f(delta) * f(x[b, t]))[:, None] * Bt
            core = (h * Ct).sum(1)
            if D is not None:
                core = core + f(D) * f(x[b, t])
            gate = f(z[b, t] * sigmoid(z[b, t])) if z is not None else 1.0
            out["y"][b, t] = core * gate
            hs.append(h)
            decays.append(a)
            deltas.append((v, delta, Bt, Ct))
            cores.append(core)
        out["state"][b] = h
        if dy is None:
            continue
        later = f(dstate_out[b]) if dstate_out is not None else zeros(dim, n)
        for t in reversed(range(count)):
            v, delta, Bt, Ct = deltas[t]
            w, xt = f(dy[b, t]), f(x[b, t])
            if z is not None:
                zt = z[b, t]
                sig = sigmoid(zt)
                slope = f(sig * (1 + zt * (1 - sig)))
                if absolute:
                    slope = slope + 0.5 * zt.abs()
                out["dz"][b, t] = w * cores[t] * slope
                w = w * f(zt * sig)
            G = w[:, None] * Ct + later
            later = decays[t] * G
            r = later * hs[t]
            du = (G * Bt).sum(1)
            ddelta = (r * f(A)).sum(1) + du * xt
            out["dx"][b, t] = du * f(delta)
            if D is not None:
                out["dx"][b, t] += f(D) * w
            ddt = ddelta * (sigmoid(v) if softplus_on else 1.0)
            out["ddt"][b, t] = ddt
            out["dA"] += r * f(delta)[:, None]
            out["dB"][b, t] = (G * (f(delta) * xt)[:, None]).view(groups, per, n).sum(1)
            out["dC"][b, t] = (w[:, None] * hs[t + 1]).view(groups, per, n).sum(1)
            out["dD"] += w * xt
            out["ddt_bias"] += ddt
        out["dstate"][b] = later
    return out


# ---------------------------------------------------------------- logits

NEG_INF = -float("inf")


def logits(x, history=None, history_len=None, prompt_len=None, repetition=None, presence=None,
           frequency=None, bias_ids=None, bias_values=None, allowed=None):
    """Processed logits, and the sums of the absolute values that made them."""
    x = x.clone()
    rows, vocab = x.shape
    mag = x.abs()
    for r in range(rows):
        if history is not None:
            cols = history.shape[1]
            n = cols if history_len is None else min(max(int(history_len[r]), 0), cols)
            first = 0 if prompt_len is None else min(max(int(prompt_len[r]), 0), cols)
            ids = history[r, :n].tolist()
            seen, made = set(), {}
            for i, tok in enumerate(ids):
                if 0 <= tok < vocab:
                    seen.add(tok)
                    if i >= first:
                        made[tok] = made.get(tok, 0) + 1
            rep = 1.0 if repetition is None else float(repetition[r])
            for tok in seen:
                v = float(x[r, tok])
                x[r, tok] = v / rep if v > 0 else v * rep
                mag[r, tok] = abs(float(x[r, tok])) * 2
            for tok, c in made.items():
                fall = (c * float(frequency[r]) if frequency is not None else 0.0) + (
                    float(presence[r]) if presence is not None else 0.0)
                x[r, tok] -= fall
                mag[r, tok] += 2 * abs(fall)
        if bias_ids is not None:
            for tok, v in zip(bias_ids[r].tolist(), bias_values[r].tolist()):
                if 0 <= tok < vocab:
                    x[r, tok] += v
                    mag[r, tok] += 2 * abs(v)
        if allowed is not None:
            for w, word in enumerate(allowed[r].tolist()):
                word &= 0xffffffff
                for i in range(32):
                    if not (word >> i) & 1 and w * 32 + i < vocab:
                        x[r, w * 32 + i] = NEG_INF
                        mag[r, w * 32 + i] = 0
    return x, mag


def probs(x, temperature=None):
    """softmax(x / temperature) by row, as logits_probs defines it at its edges."""
    out = torch.zeros_like(x)
    for r in range(x.shape[0]):
        t = 1.0 if temperature is None else float(temperature[r])
        row = x[r]
        open_ = row != NEG_INF
        if not open_.any():
            continue
        v = row[open_]
        if v.isnan().any() or (t != 0 and (v == float("inf")).any()):
            out[r, open_] = float("nan")
        elif t == 0:
            best = (v == v.max()).double()
            out[r, open_] = best / best.sum()
        else:
            e = torch.exp(v / t - (v / t).max())
            out[r, open_] = e / e.sum()
    return out
