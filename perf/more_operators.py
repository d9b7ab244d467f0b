"""More language model operators whose speed is measured: linear attention with a
decay for each head (prompts, gradients, single tokens) and layer norm with its
gradients.

A case is a dict of plain values.  listed() names twelve, draw() gives more
over the same ranges, prepare() makes what a program holds before the call,
run() is one pass: through the library's entry points where `own` is true,
in elementary torch operations in 32 bits where it is not.  exact() is the
same result in 64 bits from the definitions.
"""
import math

import torch

own = False

DEV = "cuda"
TYPES = {"f32": torch.float32, "f16": torch.float16, "bf16": torch.bfloat16}
CHUNK = 64             # tokens of a chunk of the plain form
MAX_ATTEND = 1 << 25   # rows x steps x heads x (dk + dv)
MAX_STEP = 1 << 25     # rows x heads x dk x dv
MAX_NORM = 1 << 25     # rows x dim


def listed():
    return [
        # A prompt of one request.
        dict(name="attend_prompt_1x4096x16x128", op="attend", kind="bf16", batch=1, steps=4096,
             heads=16, groups=16, dk=128, dv=128, fixed=False, ragged=False, first=False),
        # A long prompt of odd length, continued from a state; each head's decay is a constant.
        dict(name="attend_long_1x16389x8x64", op="attend", kind="f16", batch=1, steps=16389,
             heads=8, groups=8, dk=64, dv=128, fixed=True, ragged=False, first=True),
        # Prompts of many lengths in one batch; the heads of a group share q and k.
        dict(name="attend_ragged_16x777x32x64", op="attend", kind="bf16", batch=16, steps=777,
             heads=32, groups=2, dk=128, dv=64, fixed=False, ragged=True, first=False),
        # A training batch, forward and all gradients.
        dict(name="attend_train_4x2048x16x128", op="attend_train", kind="bf16", batch=4, steps=2048,
             heads=16, groups=16, dk=128, dv=128, fixed=False, ragged=False, first=False),
        # A small model in single precision, odd sizes, shared heads, with a first state.
        dict(name="attend_train_f32_3x515x6x48", op="attend_train", kind="f32", batch=3, steps=515,
             heads=6, groups=3, dk=48, dv=80, fixed=True, ragged=True, first=True),
        # One token of a single request: all latency.
        dict(name="attend_step_1x16x64", op="attend_step", kind="bf16", batch=1, heads=16,
             groups=16, dk=64, dv=64, fixed=True),
        # One token of each of 64 running requests.
        dict(name="attend_step_64x32x128", op="attend_step", kind="bf16", batch=64, heads=32,
             groups=32, dk=128, dv=128, fixed=False),
        # One token of a single request, with the residual sum: all latency.
        dict(name="norm_1x2048", op="norm", kind="bf16", rows=1, dim=2048, groups=1, residual=True),
        # A prompt's tokens, with the residual sum.
        dict(name="norm_8192x4096", op="norm", kind="bf16", rows=8192, dim=4096, groups=1,
             residual=True),
        # Long rows of an odd number of channels.
        dict(name="norm_501x16389", op="norm", kind="f16", rows=501, dim=16389, groups=1,
             residual=False),
        # A training batch, forward and all gradients, in a residual stream.
        dict(name="norm_train_8192x4096", op="norm_train", kind="bf16", rows=8192, dim=4096,
             groups=1, residual=True),
        # The norm behind the heads of an attention layer, each head by itself, in
        # single precision, with gradients.
        dict(name="norm_train_heads_4099x2048", op="norm_train", kind="f32", rows=4099, dim=2048,
             groups=16, residual=False),
    ]


# ---------------------------------------------------------------- drawn cases

def _log_int(rng, lo, hi):
    hi = max(lo, hi)
    return max(lo, min(hi, int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))))


def draw(rng):
    op = rng.choice(["attend", "attend", "attend", "attend_train", "attend_train", "attend_step",
                     "attend_step", "norm", "norm", "norm_train", "norm_train"])
    kind = rng.choice(["bf16", "bf16", "f16", "f32"])
    if op.startswith("norm"):
        dim = _log_int(rng, 32, 20000)
        if rng.random() < 0.7:
            dim = dim // 32 * 32
        rows = _log_int(rng, 1, min(65536, MAX_NORM // 2 // dim))
        return dict(op=op, kind=kind, rows=rows, dim=dim,
                    groups=rng.choice([g for g in (1, 1, 1, 4, 16) if dim % g == 0]),
                    residual=rng.random() < 0.6)
    dk = rng.choice([64, 128, 128, 256, 32, 96, 80, 33])
    dv = rng.choice([64, 128, 128, 256, 32, 96, 80, 49])
    heads = _log_int(rng, 1, 32)
    case = dict(op=op, kind=kind, heads=heads,
                groups=rng.choice([g for g in (heads, heads, 1, 2, 4) if heads % g == 0]),
                dk=dk, dv=dv, fixed=rng.random() < 0.4)
    if op == "attend_step":
        return dict(case, batch=_log_int(rng, 1, min(256, MAX_STEP // (heads * dk * dv))))
    most = MAX_ATTEND // 2 // (heads * (dk + dv))
    # (one token alone has no gradient of its decay)
    steps = _log_int(rng, 1, min(16384, most)) if op == "attend" else _log_int(
        rng, 2, min(4096, most))
    return dict(case, steps=steps, batch=_log_int(rng, 1, min(32, most // steps)),
                ragged=rng.random() < 0.4, first=rng.random() < 0.4)


# ---------------------------------------------------------------- inputs

def _lengths(case, g):
    """Token counts of a ragged batch: the same counts in every batch of the
    case, in an order of their own (the first is the whole length)."""
    if not case["ragged"]:
        return None
    b = case["batch"]
    share = torch.linspace(1.0, 0.05, b, device=DEV) if b > 1 else torch.full((1,), 0.8, device=DEV)
    order = torch.randperm(b, generator=g, device=DEV)
    return (share * case["steps"]).ceil().to(torch.int32)[order].contiguous()


def prepare(case, seed):
    g = torch.Generator(device=DEV).manual_seed(seed)

    def normal(*shape, scale=1.0, dtype=torch.float32):
        return (torch.randn(shape, generator=g, device=DEV) * scale).to(dtype)

    op, kind = case["op"], TYPES[case["kind"]]
    s = dict(case=case)
    if op.startswith("norm"):
        rows, dim = case["rows"], case["dim"]
        s["x"] = normal(rows, dim, dtype=kind) + 0.25
        s["residual"] = normal(rows, dim, scale=2.0, dtype=kind) if case["residual"] else None
        s["weight"] = (normal(dim, scale=0.2) + 1.0).to(kind)
        s["bias"] = normal(dim, scale=0.1, dtype=kind)
        if op == "norm_train":
            s["dy"] = normal(rows, dim, dtype=kind)
            s["dsum"] = normal(rows, dim, dtype=kind) if case["residual"] else None
        return s

    batch, heads, groups, dk, dv = (case[k] for k in ("batch", "heads", "groups", "dk", "dv"))
    lead = (batch,) if op == "attend_step" else (batch, case["steps"])
    # q, k and v are parts of one projection's output.
    parts = normal(*lead, 2 * groups * dk + heads * dv, dtype=kind).split(
        (groups * dk, groups * dk, heads * dv), -1)
    s["q"], s["k"] = (p.unflatten(-1, (groups, dk)) for p in parts[:2])
    s["v"] = parts[2].unflatten(-1, (heads, dv))
    # The heads remember between about 5 and 1000 tokens; what a token says of its
    # own decay varies around that.
    rate = torch.exp(torch.linspace(math.log(0.2), math.log(0.001), heads, device=DEV))
    if case["fixed"]:
        s["log_decay"] = -rate * torch.exp(normal(heads, scale=0.1))
    else:
        s["log_decay"] = -rate * torch.exp(normal(*lead, heads, scale=0.5))
    if op == "attend_step":
        s["state"] = normal(batch, heads, dk, dv)
        return s
    s["state"] = normal(batch, heads, dk, dv) if case["first"] else None
    s["lengths"] = _lengths(case, g)
    if op == "attend_train":
        s["dy"] = normal(*lead, heads, dv, dtype=kind)
        s["dstate"] = normal(batch, heads, dk, dv, scale=0.1) if case["first"] else None
    return s


# ---------------------------------------------------------------- one pass

def run(state):
    op = state["case"]["op"]
    return (_own if own else _plain)[op](state)


def _own_attend(s):
    from paper_2505_15112_amd import ops
    y, state = ops.linear_attention(s["q"], s["k"], s["v"], s["log_decay"], state=s["state"],
                                    lengths=s["lengths"], with_state=True)
    return dict(y=y, state=state)


def _own_attend_train(s):
    from paper_2505_15112_amd import ops
    args = (s["q"], s["k"], s["v"], s["log_decay"])
    more = dict(state=s["state"], lengths=s["lengths"])
    y, _ = ops.linear_attention(*args, **more)
    grads = ops.linear_attention_backward(s["dy"], *args, **more, dstate_out=s["dstate"])
    return dict(zip(("dq", "dk", "dv", "dlog_decay", "dstate"), grads), y=y)


def _own_attend_step(s):
    from paper_2505_15112_amd import ops
    y = ops.linear_attention_step(s["q"], s["k"], s["v"], s["log_decay"], s["state"])
    return dict(y=y, state=s["state"])


def _own_norm(s):
    from paper_2505_15112_amd import ops
    y, total, _ = ops.layer_norm(s["x"], s["weight"], s["bias"], residual=s["residual"],
                                 groups=s["case"]["groups"])
    return dict(y=y, sum=total)


def _own_norm_train(s):
    from paper_2505_15112_amd import ops
    groups = s["case"]["groups"]
    y, total, stats = ops.layer_norm(s["x"], s["weight"], s["bias"], residual=s["residual"],
                                     groups=groups, with_stats=True)
    dx, dweight, dbias = ops.layer_norm_backward(s["dy"], s["x"] if total is None else total, stats,
                                                 s["weight"], s["bias"], dsum=s["dsum"],
                                                 groups=groups)
    return dict(y=y, sum=total, dx=dx, dweight=dweight, dbias=dbias)


_own = dict(attend=_own_attend, attend_train=_own_attend_train, attend_step=_own_attend_step,
            norm=_own_norm, norm_train=_own_norm_train)


# ---------------------------------------------------------------- plain forms

def _by_head(t, heads):
    """batch x steps x some heads x d to batch x heads x steps x d, in 32 bits."""
    return t.float().transpose(1, 2).repeat_interleave(heads // t.shape[2], 1)


def _sides(s):
    """q, k, v by head, the log decays (batch x heads x steps), and which tokens there are."""
    batch, steps, heads, _ = s["v"].shape
    q, k, v = (_by_head(s[n], heads) for n in ("q", "k", "v"))
    g = s["log_decay"]
    g = g.transpose(1, 2) if g.dim() == 3 else g[None, :, None].expand(batch, heads, steps)
    valid = None
    if s["lengths"] is not None:
        valid = (torch.arange(steps, device=DEV)[None] < s["lengths"][:, None])[:, None]
        g, k, v, q = g * valid, k * valid[..., None], v * valid[..., None], q * valid[..., None]
    return q, k, v, g, valid


def _recurrence(a, h):
    """h[n] += a[n] h[n-1] for all n, in place: the reach doubles each time."""
    steps, reach = a.shape[2], 1
    while reach < steps:
        h[:, :, reach:] = h[:, :, reach:] + a[:, :, reach:] * h[:, :, :-reach]
        a[:, :, reach:] = a[:, :, reach:] * a[:, :, :-reach]
        reach *= 2
    return h


def _attend(q, k, v, g, state):
    """sum over j <= i of e^(g[j+1] + .. + g[i]) (q[i] . k[j]) v[j], and the last state."""
    steps = q.shape[2]
    pad = -steps % CHUNK
    q, k, v = (torch.nn.functional.pad(t, (0, 0, 0, pad)).unflatten(2, (-1, CHUNK)).contiguous()
               for t in (q, k, v))
    # sums of decays are differences of far larger ones: 64 bits
    c = torch.nn.functional.pad(g.double(), (0, pad)).unflatten(2, (-1, CHUNK)).cumsum(-1)
    over = (c[..., :, None] - c[..., None, :]).float()
    later = torch.ones(CHUNK, CHUNK, dtype=torch.bool, device=DEV).triu(1)
    near = torch.matmul(q, k.transpose(-1, -2).contiguous()) * torch.exp(
        over.masked_fill(later, -math.inf))
    y = torch.matmul(near, v)
    left = torch.exp((c[..., -1:] - c).float())[..., None]
    local = torch.matmul((k * left).transpose(-1, -2).contiguous(), v)
    whole = torch.exp(c[..., -1].float())[..., None, None]
    if state is not None:
        local[:, :, 0] += whole[:, :, 0] * state
    after = _recurrence(whole.clone(), local)
    first = torch.zeros_like(after[:, :, 0]) if state is None else state
    before = torch.cat((first[:, :, None], after[:, :, :-1]), 2)
    y = y + torch.exp(c.float())[..., None] * torch.matmul(q, before)
    return y.flatten(2, 3)[:, :, :steps], after[:, :, -1]


def _plain_attend(s):
    q, k, v, g, valid = _sides(s)
    y, last = _attend(q, k, v, g, s["state"])
    y = y * q.shape[-1] ** -0.5
    if valid is not None:
        y = y * valid[..., None]
    return dict(y=y.transpose(1, 2).to(s["v"].dtype).contiguous(), state=last.contiguous())


def _per_group(t, like):
    """Gradients by head to those of the groups that the heads share."""
    batch, steps, groups, d = like.shape
    t = t.unflatten(1, (groups, -1)).sum(2)
    return t.transpose(1, 2).to(like.dtype).contiguous()


def _plain_attend_train(s):
    kind, heads = s["v"].dtype, s["v"].shape[2]
    q, k, v, g, valid = _sides(s)
    dy = s["dy"].float().transpose(1, 2)
    if valid is not None:
        dy = dy * valid[..., None]
    scale = q.shape[-1] ** -0.5
    q, dy = q, dy * scale
    first, end = s["state"], s["dstate"]
    y, last = _attend(q, k, v, g, first)
    turned = first.transpose(-1, -2) if first is not None else None
    dq, _ = _attend(dy, v, k, g, turned)
    # the same backwards in time, with the next token's decay
    later = torch.cat((g[:, :, 1:], torch.zeros_like(g[:, :, :1])), 2).flip(2)
    rq, rk, rv, rdy = (t.flip(2) for t in (q, k, v, dy))
    turned = end.transpose(-1, -2) if end is not None else None
    dk = _attend(rv, rdy, rq, later, turned)[0].flip(2)
    dv, back = _attend(rk, rq, rdy, later, end)
    dv = dv.flip(2)
    own_part = ((q * dq).sum(-1) - (k * dk).sum(-1)).double()
    if end is not None:
        own_part[:, :, -1] += (end * last).sum((-1, -2), dtype=torch.double)
    dg = own_part.flip(2).cumsum(2).flip(2)
    if valid is not None:
        dg, dq, dk, dv = dg * valid, dq * valid[..., None], dk * valid[..., None], dv * valid[..., None]
        y = y * valid[..., None]
    dg = dg.transpose(1, 2).contiguous() if s["log_decay"].dim() == 3 else dg.sum((0, 2))
    return dict(dq=_per_group(dq, s["q"]), dk=_per_group(dk, s["k"]),
                dv=dv.transpose(1, 2).to(kind).contiguous(), dlog_decay=dg.float(),
                dstate=torch.exp(g[:, :, 0])[..., None, None] * back if first is not None else None,
                y=(y * scale).transpose(1, 2).to(kind).contiguous())


def _plain_attend_step(s):
    heads, dk = s["v"].shape[1], s["q"].shape[2]
    q, k = (s[n].float().repeat_interleave(heads // s[n].shape[1], 1) for n in ("q", "k"))
    v = s["v"].float()
    h = torch.exp(s["log_decay"])[..., None, None] * s["state"] + k[..., :, None] * v[..., None, :]
    y = (q[..., :, None] * h).sum(-2) * dk ** -0.5
    s["state"].copy_(h)
    return dict(y=y.to(s["v"].dtype), state=s["state"])


EPS = 1e-5


def _plain_norm(s):
    x, total, kind = s["x"], None, s["x"].dtype
    if s["residual"] is not None:
        total = (x.float() + s["residual"].float()).to(kind)  # what the layers pass on
        x = total
    x = x.float().unflatten(1, (s["case"]["groups"], -1))
    mean = x.mean(-1, keepdim=True)
    rstd = torch.rsqrt(((x - mean) ** 2).mean(-1, keepdim=True) + EPS)
    hat = (x - mean) * rstd
    y = (hat.flatten(1) * s["weight"].float() + s["bias"].float()).to(kind)
    if s["case"]["op"] == "norm_train":
        return y, total, hat, rstd
    return dict(y=y, sum=total)


def _plain_norm_train(s):
    y, total, hat, rstd = _plain_norm(s)
    dy = s["dy"].float()
    w = (dy * s["weight"].float()).view_as(hat)
    dx = rstd * (w - w.mean(-1, keepdim=True) - hat * (w * hat).mean(-1, keepdim=True))
    dx = dx.flatten(1)
    if s["dsum"] is not None:
        dx = dx + s["dsum"].float()
    return dict(y=y, sum=total, dx=dx.to(s["x"].dtype), dweight=(dy * hat.flatten(1)).sum(0),
                dbias=dy.sum(0))


_plain = dict(attend=_plain_attend, attend_train=_plain_attend_train,
              attend_step=_plain_attend_step, norm=_plain_norm, norm_train=_plain_norm_train)


# ---------------------------------------------------------------- least work

def work(case):
    op = case["op"]
    e = 4 if case["kind"] == "f32" else 2
    if op.startswith("norm"):
        cells = case["rows"] * case["dim"]
        more = 2 if case["residual"] else 0
        if op == "norm":
            return dict(bytes=cells * e * (2 + more), flops=cells * 8)
        # the forward, then its input and dy to dx, with the stream's gradient
        return dict(bytes=cells * e * (5 + more + more // 2), flops=cells * 24)
    heads, groups, dk, dv, batch = (case[k] for k in ("heads", "groups", "dk", "dv", "batch"))
    state = heads * dk * dv
    if op == "attend_step":
        gates = 0 if case["fixed"] else heads * 4
        return dict(bytes=batch * (state * 8 + 2 * groups * dk * e + 2 * heads * dv * e + gates),
                    flops=batch * state * 5)
    steps = case["steps"]
    tokens = batch * steps
    if case["ragged"]:
        share = [1 - 0.95 * i / (batch - 1) for i in range(batch)] if batch > 1 else [0.8]
        tokens = sum(math.ceil(f * steps) for f in share)
    gates = 0 if case["fixed"] else tokens * heads * 4
    side, wide = 2 * groups * dk * e, heads * dv * e  # of one token: q and k, and v
    states = batch * state * 4
    first = states if case["first"] else 0
    if op == "attend":
        # past a row's tokens the outputs are zeros
        return dict(bytes=tokens * (side + wide) + gates + batch * steps * wide + states + first,
                    flops=tokens * state * 5)
    # the forward, then its inputs and dy to all gradients
    return dict(bytes=tokens * (2 * side + 3 * wide) + 3 * gates
                + batch * steps * (side + 2 * wide) + 4 * first, flops=tokens * state * 16)


# ---------------------------------------------------------------- 64 bits

ROWS = 2048  # queries at a time


def exact(case, seed):
    s = prepare(case, seed)
    if case["op"].startswith("norm"):
        return _exact_norm(s)
    for k, v in list(s.items()):
        if isinstance(v, torch.Tensor) and v.is_floating_point():
            s[k] = v.double()
    return _exact[case["op"]](s)


def _exact_row(q, k, v, g, state):
    """One head of one row: (tokens x dk, tokens x dk, tokens x dv, tokens) to its
    outputs and its last state, by all pairs of tokens."""
    n = q.shape[0]
    c, at, outs = g.cumsum(0), torch.arange(n, device=DEV), []
    for lo in range(0, n, ROWS):
        hi = min(n, lo + ROWS)
        over = (c[lo:hi, None] - c[None, :hi]).masked_fill(at[None, :hi] > at[lo:hi, None], -math.inf)
        outs.append((torch.exp(over) * (q[lo:hi] @ k[:hi].t())) @ v[:hi])
    y = torch.cat(outs) if outs else v * 0
    last = (k * torch.exp(c[-1:] - c)[:, None]).t() @ v
    if state is not None:
        y = y + torch.exp(c)[:, None] * (q @ state)
        last = last + (torch.exp(c[-1]) * state if n else state)
    return y * q.shape[1] ** -0.5, last


def _exact_attend(s):
    batch, steps, heads, dv = s["v"].shape
    per = heads // s["q"].shape[2]
    count = [steps] * batch if s["lengths"] is None else s["lengths"].tolist()
    ys, states = [], []
    for b, n in enumerate(count):
        for h in range(heads):
            g = s["log_decay"][b, :n, h] if s["log_decay"].dim() == 3 else s["log_decay"][h].expand(n)
            y, last = _exact_row(s["q"][b, :n, h // per], s["k"][b, :n, h // per], s["v"][b, :n, h],
                                 g, s["state"][b, h] if s["state"] is not None else None)
            ys.append(torch.nn.functional.pad(y, (0, 0, 0, steps - n)))
            states.append(last)
    return dict(y=torch.stack(ys).unflatten(0, (batch, heads)).transpose(1, 2).contiguous(),
                state=torch.stack(states).unflatten(0, (batch, heads)))


def _exact_attend_train(s):
    """Row by row and head by head, so that no more than one head's pairs are held."""
    batch, steps, heads, dv = s["v"].shape
    per = heads // s["q"].shape[2]
    count = [steps] * batch if s["lengths"] is None else s["lengths"].tolist()
    each = s["log_decay"].dim() == 3
    out = {"d" + n: torch.zeros_like(s[n], memory_format=torch.contiguous_format)
           for n in ("q", "k", "v", "log_decay")}
    out["dstate"] = torch.zeros_like(s["state"]) if s["state"] is not None else None
    out["y"] = torch.zeros(batch, steps, heads, dv, dtype=torch.double, device=DEV)
    for b, n in enumerate(count):
        for h in range(heads):
            g = s["log_decay"][b, :n, h] if each else s["log_decay"][h].expand(n)
            leaf = [t.detach().clone().requires_grad_() for t in (
                s["q"][b, :n, h // per], s["k"][b, :n, h // per], s["v"][b, :n, h], g)]
            if s["state"] is not None:
                leaf.append(s["state"][b, h].detach().clone().requires_grad_())
            y, last = _exact_row(*leaf[:4], leaf[4] if len(leaf) > 4 else None)
            total = (y * s["dy"][b, :n, h]).sum()
            if s["dstate"] is not None:
                total = total + (last * s["dstate"][b, h]).sum()
            got = torch.autograd.grad(total, leaf)
            out["y"][b, :n, h] = y.detach()
            out["dq"][b, :n, h // per] += got[0]
            out["dk"][b, :n, h // per] += got[1]
            out["dv"][b, :n, h] = got[2]
            if each:
                out["dlog_decay"][b, :n, h] = got[3]
            else:
                out["dlog_decay"][h] += got[3].sum()
            if s["state"] is not None:
                out["dstate"][b, h] = got[4]
    return out


def _exact_attend_step(s):
    per = s["v"].shape[1] // s["q"].shape[1]
    q, k = (s[n].repeat_interleave(per, 1) for n in ("q", "k"))
    h = torch.exp(s["log_decay"])[..., None, None] * s["state"] + torch.einsum(
        "bhi,bhj->bhij", k, s["v"])
    return dict(y=torch.einsum("bhi,bhij->bhj", q, h) * q.shape[2] ** -0.5, state=h)


def _exact_norm(s):
    kind, total = s["x"].dtype, None
    x = s["x"].double()
    if s["residual"] is not None:
        # the layers pass the sum on, in the stream's own type, and that is what is normalised
        x = (x + s["residual"].double()).to(kind).double()
        total = x
    train = s["case"]["op"] == "norm_train"
    leaf = [t.clone().requires_grad_(train) for t in (x, s["weight"].double(), s["bias"].double())]
    rows = leaf[0].unflatten(1, (s["case"]["groups"], -1))
    var, mean = torch.var_mean(rows, -1, correction=0, keepdim=True)
    y = ((rows - mean) / torch.sqrt(var + EPS)).flatten(1) * leaf[1] + leaf[2]
    out = dict(y=y.detach(), sum=total)
    if train:
        got = torch.autograd.grad((y * s["dy"].double()).sum(), leaf)
        dx = got[0] + s["dsum"].double() if s["dsum"] is not None else got[0]
        out.update(dx=dx, dweight=got[1], dbias=got[2])
    return out


_exact = dict(attend=_exact_attend, attend_train=_exact_attend_train,
              attend_step=_exact_attend_step)
