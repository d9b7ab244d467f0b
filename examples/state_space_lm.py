"""A small state space language model on the library's operators, with random
weights: prompts of different lengths at once, then token by token with
penalties, a grammar's mask and the top-p sampler; and a training step.

    python examples/state_space_lm.py

Torch does the embeddings and the projections; causal_conv, selective_scan,
their single-token steps and gradients, logits_probs and topp_sample_f32 do
the rest.
"""
import os
import sys

import torch
import torch.nn.functional as F

sys.path.insert(0, os.path.dirname(os.path.dirname(os.path.abspath(__file__))))

from paper_2505_15112_amd import ops  # noqa: E402


class Conv(torch.autograd.Function):
    """ops.causal_conv on rows that start from nothing (no first state, which
    causal_conv_backward has a gradient for)."""

    @staticmethod
    def forward(ctx, x, weight, bias, lengths):
        y, _ = ops.causal_conv(x, weight, bias, lengths=lengths)
        ctx.save_for_backward(x, weight, bias, lengths)
        return y

    @staticmethod
    def backward(ctx, dy):
        x, weight, bias, lengths = ctx.saved_tensors
        dx, dweight, dbias, _ = ops.causal_conv_backward(dy.contiguous(), x, weight, bias,
                                                         lengths=lengths)
        return dx, dweight.to(weight.dtype), dbias.to(bias.dtype), None


class Scan(torch.autograd.Function):
    """ops.selective_scan on rows that start from nothing, as Conv."""

    @staticmethod
    def forward(ctx, x, dt, A, B, C, D, z, dt_bias, lengths):
        y, _, kept = ops.selective_scan(x, dt, A, B, C, D=D, z=z, dt_bias=dt_bias,
                                        lengths=lengths, with_checkpoints=True)
        ctx.save_for_backward(kept, x, dt, A, B, C, D, z, dt_bias, lengths)
        return y

    @staticmethod
    def backward(ctx, dy):
        kept, x, dt, A, B, C, D, z, dt_bias, lengths = ctx.saved_tensors
        g = ops.selective_scan_backward(dy.contiguous(), kept, x, dt, A, B, C, D=D, z=z,
                                        dt_bias=dt_bias, lengths=lengths)
        return (*g[:8], None)


class Layer:
    """One mixing layer: width `dim`, `inner` channels of `n` states."""

    def __init__(self, dim, inner, n, rank, dtype, generator, device):
        def w(*shape, scale):
            return (torch.randn(*shape, generator=generator, device=device) * scale).to(dtype)

        self.n, self.rank, self.inner = n, rank, inner
        self.norm = torch.ones(dim, dtype=dtype, device=device)
        self.w_in = w(2 * inner, dim, scale=dim ** -0.5)
        self.conv_w = w(inner, 4, scale=0.5)
        self.conv_b = w(inner, scale=0.1)
        self.w_bc = w(rank + 2 * n, inner, scale=inner ** -0.5)
        self.w_dt = w(inner, rank, scale=rank ** -0.5)
        self.w_out = w(dim, inner, scale=inner ** -0.5)
        rates = torch.arange(1, n + 1, device=device, dtype=torch.float32)
        self.log_A = rates.log().expand(inner, n).contiguous()
        self.D = torch.ones(inner, device=device)
        step = torch.exp(torch.rand(inner, generator=generator, device=device) * 4.6 - 6.9)
        self.dt_bias = step + torch.log(-torch.expm1(-step))

    def parameters(self):
        return [self.norm, self.w_in, self.conv_w, self.conv_b, self.w_bc, self.w_dt, self.w_out,
                self.log_A, self.D, self.dt_bias]

    def split(self, u):
        """The scan's inputs that depend on its input: dt, B, C."""
        dt, B, C = F.linear(u, self.w_bc).split((self.rank, self.n, self.n), -1)
        return F.linear(dt, self.w_dt), B.unsqueeze(-2), C.unsqueeze(-2)

    def prompt(self, h, lengths):
        """batch x steps x dim, and the states behind the rows' last tokens."""
        x, z = F.linear(F.rms_norm(h, h.shape[-1:], self.norm), self.w_in).split(self.inner, -1)
        u, window = ops.causal_conv(x, self.conv_w, self.conv_b, lengths=lengths, with_state=True)
        dt, B, C = self.split(u)
        y, state, _ = ops.selective_scan(u, dt, -self.log_A.exp(), B, C, D=self.D, z=z,
                                         dt_bias=self.dt_bias, lengths=lengths, with_state=True)
        return h + F.linear(y, self.w_out), (window, state)

    def token(self, h, states):
        """batch x dim; the states move on in place."""
        x, z = F.linear(F.rms_norm(h, h.shape[-1:], self.norm), self.w_in).split(self.inner, -1)
        u = ops.causal_conv_step(x, states[0], self.conv_w, self.conv_b)
        dt, B, C = self.split(u)
        y = ops.selective_scan_step(u, dt, states[1], -self.log_A.exp(), B, C, D=self.D, z=z,
                                    dt_bias=self.dt_bias)
        return h + F.linear(y, self.w_out)

    def train(self, h, lengths):
        """prompt() with gradients."""
        x, z = F.linear(F.rms_norm(h, h.shape[-1:], self.norm), self.w_in).split(self.inner, -1)
        u = Conv.apply(x, self.conv_w, self.conv_b, lengths)
        dt, B, C = self.split(u)
        y = Scan.apply(u, dt, -self.log_A.exp(), B, C, self.D, z, self.dt_bias, lengths)
        return h + F.linear(y, self.w_out)


class Model:
    def __init__(self, vocab=32000, dim=256, layers=2, n=16, dtype=torch.bfloat16, seed=0,
                 device="cuda"):
        g = torch.Generator(device=device).manual_seed(seed)
        self.embed = (torch.randn(vocab, dim, generator=g, device=device) * dim ** -0.5).to(dtype)
        self.layers = [Layer(dim, 2 * dim, n, dim // 16, dtype, g, device) for _ in range(layers)]
        self.norm = torch.ones(dim, dtype=dtype, device=device)

    def parameters(self):
        return [self.embed, self.norm] + [p for layer in self.layers for p in layer.parameters()]

    def logits(self, h):
        return F.linear(F.rms_norm(h, h.shape[-1:], self.norm), self.embed)

    def prompt(self, ids, lengths):
        """Logits behind each row's last token, and the states to go on from."""
        h, states = F.embedding(ids, self.embed), []
        for layer in self.layers:
            h, s = layer.prompt(h, lengths)
            states.append(s)
        rows = torch.arange(ids.shape[0], device=ids.device)
        return self.logits(h[rows, (lengths - 1).clamp(min=0).long()]), states

    def token(self, ids, states):
        h = F.embedding(ids, self.embed)
        for layer, s in zip(self.layers, states):
            h = layer.token(h, s)
        return self.logits(h)

    def loss(self, ids, lengths):
        """Mean cross entropy of the next tokens inside the rows."""
        h = F.embedding(ids, self.embed)
        for layer in self.layers:
            h = layer.train(h, lengths)
        scores = self.logits(h[:, :-1]).float().flatten(0, 1)
        inside = torch.arange(1, ids.shape[1], device=ids.device) < lengths[:, None]
        target = torch.where(inside, ids[:, 1:], -100).flatten().long()
        return F.cross_entropy(scores, target, ignore_index=-100)


@torch.no_grad()
def generate(model, ids, lengths, steps, top_p=0.9, temperature=0.8, repetition=1.1, presence=0.2,
             frequency=0.1, allowed=None, seed=0):
    """`steps` tokens for every prompt (rows of ids, the first lengths of each)."""
    rows, dev = ids.shape[0], ids.device
    g = torch.Generator(device=dev).manual_seed(seed)

    def per_row(v):
        return torch.full((rows,), float(v), device=dev)

    history = torch.full((rows, ids.shape[1] + steps), -1, dtype=torch.int32, device=dev)
    history[:, :ids.shape[1]] = ids
    held = lengths.clone()
    each = torch.arange(rows, device=dev)
    more = dict(repetition=per_row(repetition), presence=per_row(presence),
                frequency=per_row(frequency), temperature=per_row(temperature), allowed=allowed)
    logits, states = model.prompt(ids, lengths)
    out = torch.empty(rows, steps, dtype=torch.int32, device=dev)
    for i in range(steps):
        probs = ops.logits_probs(logits, history=history, history_len=held, prompt_len=lengths,
                                 **more)
        draws = torch.rand(rows, generator=g, device=dev)
        token = ops.topp_sample_f32(probs, draws, top_p)
        out[:, i] = token
        history[each, held.long()] = token
        held += 1
        if i + 1 < steps:
            logits = model.token(token, states)
    return out


def train_step(model, ids, lengths, rate=0.05):
    """One step of gradient descent; returns the loss before it."""
    params = [p.requires_grad_() for p in model.parameters()]
    loss = model.loss(ids, lengths)
    grads = torch.autograd.grad(loss, params)
    with torch.no_grad():
        for p, g in zip(params, grads):
            p -= rate * g
            p.requires_grad_(False)
    return float(loss.detach())


def main():
    model = Model()
    g = torch.Generator(device="cuda").manual_seed(1)
    ids = torch.randint(0, 32000, (4, 100), generator=g, device="cuda", dtype=torch.int32)
    lengths = torch.tensor([100, 37, 1, 64], dtype=torch.int32, device="cuda")
    print("losses", [round(train_step(model, ids, lengths), 3) for _ in range(4)])
    print("tokens", generate(model, ids, lengths, 12).tolist())


if __name__ == "__main__":
    main()
