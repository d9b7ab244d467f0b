"""The example model of linear attention layers: its parts used together give what
they give apart, and its gradients are those of the same layers in torch."""
import importlib.util
import os

import pytest
import torch
import torch.nn.functional as F

pytestmark = pytest.mark.gpu

PATH = os.path.join(os.path.dirname(os.path.dirname(os.path.abspath(__file__))), "examples",
                    "linear_attention_lm.py")


@pytest.fixture(scope="module")
def lm():
    spec = importlib.util.spec_from_file_location("linear_attention_lm", PATH)
    module = importlib.util.module_from_spec(spec)
    spec.loader.exec_module(module)
    return module


def data(vocab, rows=3, steps=40):
    g = torch.Generator(device="cuda").manual_seed(2)
    ids = torch.randint(0, vocab, (rows, steps), generator=g, device="cuda", dtype=torch.int32)
    return ids, torch.tensor([40, 17, 1], dtype=torch.int32, device="cuda")


def test_tokens_one_by_one_follow_the_prompt(lm):
    """A prompt extended token by token against the longer prompt at once, in fp32 (the two
    sum in different orders: 1e-4 of the logits' size)."""
    model = lm.Model(vocab=500, dim=64, d=24, dtype=torch.float32)
    ids, lengths = data(500)
    start = lengths - torch.tensor([7, 7, 0], dtype=torch.int32, device="cuda")
    logits, states = model.prompt(ids, start)
    for i in range(7):
        nxt = ids.gather(1, (start + i).clamp(max=39)[:, None].long())[:, 0]
        logits = model.token(nxt, states)
    want, last = model.prompt(ids, lengths)
    assert (logits[:2] - want[:2]).abs().max() <= 1e-4 * want.abs().max()
    for state, s2 in zip(states, last):
        assert (state[:2] - s2[:2]).abs().max() <= 1e-4 * s2.abs().max()


def test_generation_repeats(lm):
    model = lm.Model(vocab=1000, dim=64, d=32)
    ids, lengths = data(1000)
    a, b = (lm.generate(model, ids, lengths, 10) for _ in range(2))
    assert torch.equal(a, b) and bool(((a >= 0) & (a < 1000)).all())


def plain_loss(model, ids, lengths):
    """Model.loss in elementary operations, in 64 bits."""
    def norm(x, w, groups):
        rows = x.unflatten(-1, (groups, -1))
        var, mean = torch.var_mean(rows, -1, correction=0, keepdim=True)
        return ((rows - mean) / torch.sqrt(var + 1e-5)).flatten(-2) * w[0] + w[1]

    more = F.embedding(ids, model.embed)
    h = torch.zeros_like(more)
    steps = ids.shape[1]
    inside = torch.arange(steps, device=ids.device) < lengths[:, None]
    for layer in model.layers:
        h = h + more
        q, k, v, g = F.linear(norm(h, layer.norm, 1), layer.w_in).split(layer.parts, -1)
        q, k = (t.unflatten(-1, (layer.groups, layer.d)).repeat_interleave(
            layer.heads // layer.groups, 2) for t in (q, k))
        v = v.unflatten(-1, (layer.heads, layer.d))
        c = -F.softplus(g + layer.rate).cumsum(1)
        over = (c[:, :, None] - c[:, None]).masked_fill(
            torch.ones(steps, steps, dtype=torch.bool, device=ids.device).triu(1)[None, :, :, None],
            -float("inf"))
        near = (q[:, :, None] * k[:, None]).sum(-1) * torch.exp(over) * layer.d ** -0.5
        y = (near[..., None] * v[:, None]).sum(2) * inside[..., None, None]
        more = F.linear(norm(y.flatten(2), layer.head_norm, layer.heads), layer.w_out)
    x = norm(h + more, model.norm, 1)
    scores = F.linear(x[:, :-1], model.embed).flatten(0, 1)
    target = torch.where(inside[:, 1:], ids[:, 1:], -100).flatten().long()
    return F.cross_entropy(scores, target, ignore_index=-100)


def test_gradients_of_a_training_step(lm):
    """The loss and all parameters' gradients in fp32 against 64 bits: 1e-4 of each
    gradient's norm, some hundred fp32 roundings through two layers."""
    model = lm.Model(vocab=60, dim=48, d=16, dtype=torch.float32)
    ids, lengths = data(60)
    params = [p.requires_grad_() for p in model.parameters()]
    loss = model.loss(ids, lengths)
    got = torch.autograd.grad(loss, params)
    twin = lm.Model(vocab=60, dim=48, d=16, dtype=torch.float64)
    for layer in twin.layers:
        layer.rate = layer.rate.double()
    with torch.no_grad():
        for p, t in zip(params, twin.parameters()):
            t.copy_(p)
    leaves = [p.requires_grad_() for p in twin.parameters()]
    want_loss = plain_loss(twin, ids, lengths)
    want = torch.autograd.grad(want_loss, leaves)
    loss, want_loss = float(loss.detach()), float(want_loss.detach())
    assert abs(loss - want_loss) <= 1e-5 * abs(want_loss)
    for g, w in zip(got, want):
        assert (g.double() - w).norm() <= 1e-4 * w.norm() + 1e-9


def test_a_training_step_runs(lm):
    model = lm.Model(vocab=300, dim=64, d=32)
    ids, lengths = data(300)
    before = [p.clone() for p in model.parameters()]
    loss = lm.train_step(model, ids, lengths)
    assert loss == loss and loss > 0
    assert all(torch.isfinite(p).all() for p in model.parameters())
    assert any(not torch.equal(p, b) for p, b in zip(model.parameters(), before))
