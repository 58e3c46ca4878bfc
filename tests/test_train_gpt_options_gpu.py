"""The small GPT with rotated queries and keys and with dropout: its per-worker gradients against automatic differentiation of the
same model with the same masks in 32 bits, and a few steps of it."""
import pytest
import torch

import model_operators_ref as ref
from paper_2302_00845_b200 import binding
from paper_2302_00845_b200.train_gpt import Gpt, sequences, train

pytestmark = pytest.mark.gpu


def turned(x, w):
    """[heads][t][d]: normed, weighed and rotated"""
    t, d = x.shape[-2:]
    n = x / torch.sqrt(x.square().mean(-1, keepdim=True) + 1e-6) * w
    angle = torch.arange(t, device="cuda").double()[:, None] * 10000.0 ** (-2.0 * torch.arange(d // 2, device="cuda").double() / d)
    c, s = torch.cos(angle).float(), torch.sin(angle).float()
    a, b = n[..., :d // 2], n[..., d // 2:]
    return torch.cat((a * c - b * s, a * s + b * c), -1)


def reference_loss(model, p, tokens, drop):
    t, h, hk = model.length, model.heads, model.kv_heads
    F = torch.nn.functional
    inp, want = tokens[:-1], tokens[1:]
    x = p["embed"][inp]
    if not model.rotary:
        x = x + p["pos"]
    for l in range(model.layers):
        y = F.layer_norm(x, (model.width,), p[f"{l}.ln1.w"], p[f"{l}.ln1.b"])
        qkv = (y @ p[f"{l}.qkv"].T).view(t, h + 2 * hk, model.head_dim).transpose(0, 1)
        q, k, v = qkv[:h], qkv[h:h + hk], qkv[h + hk:].repeat_interleave(h // hk, 0)
        if model.rotary:
            q, k = turned(q, p[f"{l}.q.w"]), turned(k, p[f"{l}.k.w"])
        s = q @ k.repeat_interleave(h // hk, 0).transpose(1, 2) * model.head_dim ** -0.5
        s = s.masked_fill(torch.triu(torch.ones(t, t, dtype=torch.bool, device="cuda"), 1), float("-inf"))
        o = (torch.softmax(s, -1) @ v).transpose(0, 1).reshape(t, -1)
        x = x + drop(2 * l, o @ p[f"{l}.out"].T)
        y = F.layer_norm(x, (model.width,), p[f"{l}.ln2.w"], p[f"{l}.ln2.b"])
        x = x + drop(2 * l + 1, F.gelu(y @ p[f"{l}.up"].T) @ p[f"{l}.down"].T)
    y = F.layer_norm(x, (model.width,), p["ln.w"], p["ln.b"])
    return F.cross_entropy(y @ p["head"].T, want)


@pytest.mark.parametrize("rotary,dropout", [(True, 0.0), (False, 0.2), (True, 0.1)])
def test_gradients_of_each_worker(rotary, dropout):
    model = Gpt(vocab=32, width=64, heads=4, kv_heads=2, layers=2, length=70, rotary=rotary, dropout=dropout, seed=5)
    assert ("pos" in model.p) != rotary and ("0.q.w" in model.p) == rotary
    m = 3
    tokens = sequences(m, 1, model.length, model.vocab)[:, 0]
    buf = torch.full((2, m, model.d), float("nan"), device="cuda")
    model.loss_and_gradients(tokens, buf[0])             # the step before draws other masks
    losses = model.loss_and_gradients(tokens, buf[1])
    assert binding.operators_status() == binding.OK
    assert torch.equal(model.grad(buf[0], "embed"), model.grad(buf[1], "embed")) == (dropout == 0.0)
    t, c = model.length, model.width
    limit = int(65536 * dropout + 0.5)
    for i in range(m):
        def drop(call, y):
            if not dropout:
                return y
            keep = torch.from_numpy(ref.keep(range(i * t * c, (i + 1) * t * c), dropout, 5, call, 1)).view(t, c).cuda()
            return torch.where(keep, y * (65536 / (65536 - limit)), 0.0)
        p = {n: w.detach().clone().requires_grad_(True) for n, w in model.p.items()}
        loss = reference_loss(model, p, tokens[i], drop)
        loss.backward()
        assert abs(float(loss) - float(losses[i])) <= 2e-2
        for n, w in p.items():
            got = model.grad(buf[1], n)[i]
            # a dozen bf16 products deep, each rounding by up to 2^-8 and mostly independently: about 1 % of the norm
            assert float((got - w.grad).norm()) <= 3e-2 * float(w.grad.norm()) + 1e-6, n


def test_the_same_gradients_every_time():
    model = Gpt(vocab=32, width=64, heads=4, kv_heads=2, layers=1, length=33, rotary=True, dropout=0.1)
    tokens = sequences(5, 1, model.length, model.vocab)[:, 0]
    bufs = torch.zeros(2, 5, model.d, device="cuda")
    for b in bufs:
        model.steps = 3
        model.loss_and_gradients(tokens, b)
    assert torch.equal(bufs[0], bufs[1])


def test_it_runs_in_coordinated_order():
    model = Gpt(vocab=32, width=64, heads=2, kv_heads=1, layers=1, length=64, rotary=True, dropout=0.1)
    history = train(model, workers=4, examples=4, epochs=2, log=lambda *_: None)
    assert all(torch.isfinite(torch.tensor(history)))
