"""A small language model of linear attention layers on the library's operators, with
random weights: prompts of different lengths at once, then token by token, and a
training step, as examples/state_space_lm.py has them.

    python examples/linear_attention_lm.py

Torch does the embeddings and the projections; linear_attention and layer_norm (in front
of every layer, with the residual sum, and behind the heads, each by itself), their
gradients and the single-token step do the rest.
"""
import os
import sys

import torch
import torch.nn.functional as F

HERE = os.path.dirname(os.path.abspath(__file__))
for path in (os.path.dirname(HERE), HERE):
    if path not in sys.path:
        sys.path.insert(0, path)

from paper_2505_15112_amd import ops  # noqa: E402
from state_space_lm import generate, train_step  # noqa: E402


class Attention(torch.autograd.Function):
    """ops.linear_attention on rows that start from nothing."""

    @staticmethod
    def forward(ctx, q, k, v, log_decay, lengths):
        ctx.save_for_backward(q, k, v, log_decay, lengths)
        return ops.linear_attention(q, k, v, log_decay, lengths=lengths)[0]

    @staticmethod
    def backward(ctx, dy):
        q, k, v, log_decay, lengths = ctx.saved_tensors
        grads = ops.linear_attention_backward(dy.contiguous(), q, k, v, log_decay, lengths=lengths)
        return (*grads[:4], None)


class Norm(torch.autograd.Function):
    """ops.layer_norm of x, or of x + residual, which is returned too."""

    @staticmethod
    def forward(ctx, x, weight, bias, residual, groups):
        y, total, stats = ops.layer_norm(x, weight, bias, residual=residual, groups=groups,
                                         with_stats=True)
        ctx.save_for_backward(x if total is None else total, stats, weight, bias)
        ctx.groups, ctx.summed = groups, total is not None
        return y, total

    @staticmethod
    def backward(ctx, dy, dsum):
        x, stats, weight, bias = ctx.saved_tensors
        dsum = dsum.contiguous() if ctx.summed and dsum is not None else None
        dx, dweight, dbias = ops.layer_norm_backward(dy.contiguous(), x, stats, weight, bias,
                                                     dsum=dsum, groups=ctx.groups)
        return (dx, dweight.to(weight.dtype), dbias.to(bias.dtype), dx if ctx.summed else None,
                None)


class Layer:
    """One layer of `heads` heads of d channels, whose keys are shared by `share` of them.
    It takes the stream of the residual sums and what the layer before adds to it."""

    def __init__(self, dim, heads, d, share, dtype, generator, device):
        def w(*shape, scale):
            return (torch.randn(*shape, generator=generator, device=device) * scale).to(dtype)

        def norm(n):
            return [torch.ones(n, dtype=dtype, device=device),
                    torch.zeros(n, dtype=dtype, device=device)]

        self.heads, self.groups, self.d = heads, heads // share, d
        self.norm, self.head_norm = norm(dim), norm(heads * d)
        self.parts = (self.groups * d, self.groups * d, heads * d, heads)
        self.w_in = w(sum(self.parts), dim, scale=dim ** -0.5)
        self.w_out = w(dim, heads * d, scale=(heads * d) ** -0.5)
        # decays from about e^-1 to e^-0.01 a token
        self.rate = torch.linspace(0.0, -4.6, heads, device=device)

    def parameters(self):
        return [*self.norm, *self.head_norm, self.w_in, self.w_out, self.rate]

    def split(self, x):
        """q, k, v and the log decays of every token."""
        q, k, v, g = F.linear(x, self.w_in).split(self.parts, -1)
        q, k = (t.unflatten(-1, (self.groups, self.d)) for t in (q, k))
        decay = -F.softplus(g.float() + self.rate)
        return q, k, v.unflatten(-1, (self.heads, self.d)), decay

    def prompt(self, h, more, lengths):
        """batch x steps x dim; and the states behind the rows' last tokens."""
        x, h, _ = ops.layer_norm(more, *self.norm, residual=h)
        y, state = ops.linear_attention(*self.split(x), lengths=lengths, with_state=True)
        y, _, _ = ops.layer_norm(y.flatten(2), *self.head_norm, groups=self.heads)
        return h, F.linear(y, self.w_out), state

    def token(self, h, more, state):
        """batch x dim; the state moves on in place."""
        x, h, _ = ops.layer_norm(more, *self.norm, residual=h)
        y = ops.linear_attention_step(*self.split(x), state)
        y, _, _ = ops.layer_norm(y.flatten(1), *self.head_norm, groups=self.heads)
        return h, F.linear(y, self.w_out)

    def train(self, h, more, lengths):
        """prompt() with gradients."""
        x, h = Norm.apply(more, *self.norm, h, 1)
        y = Attention.apply(*self.split(x), lengths)
        y, _ = Norm.apply(y.flatten(2), *self.head_norm, None, self.heads)
        return h, F.linear(y, self.w_out)


class Model:
    def __init__(self, vocab=32000, dim=256, layers=2, heads=4, d=64, share=2, dtype=torch.bfloat16,
                 seed=0, device="cuda"):
        g = torch.Generator(device=device).manual_seed(seed)
        self.embed = (torch.randn(vocab, dim, generator=g, device=device) * dim ** -0.5).to(dtype)
        self.layers = [Layer(dim, heads, d, share, dtype, g, device) for _ in range(layers)]
        self.norm = [torch.ones(dim, dtype=dtype, device=device),
                     torch.zeros(dim, dtype=dtype, device=device)]

    def parameters(self):
        return [self.embed, *self.norm] + [p for layer in self.layers for p in layer.parameters()]

    def prompt(self, ids, lengths):
        """Logits behind each row's last token, and the states to go on from."""
        more, states = F.embedding(ids, self.embed), []
        h = torch.zeros_like(more)
        for layer in self.layers:
            h, more, s = layer.prompt(h, more, lengths)
            states.append(s)
        rows, at = torch.arange(ids.shape[0], device=ids.device), (lengths - 1).clamp(min=0).long()
        x, _, _ = ops.layer_norm(more[rows, at], *self.norm, residual=h[rows, at])
        return F.linear(x, self.embed), states

    def token(self, ids, states):
        more = F.embedding(ids, self.embed)
        h = torch.zeros_like(more)
        for layer, s in zip(self.layers, states):
            h, more = layer.token(h, more, s)
        x, _, _ = ops.layer_norm(more, *self.norm, residual=h)
        return F.linear(x, self.embed)

    def loss(self, ids, lengths):
        """Mean cross entropy of the next tokens inside the rows."""
        more = F.embedding(ids, self.embed)
        h = torch.zeros_like(more)
        for layer in self.layers:
            h, more = layer.train(h, more, lengths)
        x, _ = Norm.apply(more, *self.norm, h, 1)
        scores = F.linear(x[:, :-1], self.embed).float().flatten(0, 1)
        inside = torch.arange(1, ids.shape[1], device=ids.device) < lengths[:, None]
        target = torch.where(inside, ids[:, 1:], -100).flatten().long()
        return F.cross_entropy(scores, target, ignore_index=-100)


def main():
    model = Model()
    g = torch.Generator(device="cuda").manual_seed(1)
    ids = torch.randint(0, 32000, (4, 100), generator=g, device="cuda", dtype=torch.int32)
    lengths = torch.tensor([100, 37, 1, 64], dtype=torch.int32, device="cuda")
    print("losses", [round(train_step(model, ids, lengths), 3) for _ in range(4)])
    print("tokens", generate(model, ids, lengths, 12).tolist())


if __name__ == "__main__":
    main()
