"""The training operators together: per-worker gradients of a small GPT against automatic differentiation of the
same model in 32 bits, and a few epochs in coordinated order."""
import pytest
import torch

from paper_2302_00845_b200 import binding
from paper_2302_00845_b200.train_gpt import Gpt, sequences, train

pytestmark = pytest.mark.gpu


def reference_loss(model, p, tokens):
    t, h, hk = model.length, model.heads, model.kv_heads
    F = torch.nn.functional
    inp, want = tokens[:-1], tokens[1:]
    x = p["embed"][inp] + p["pos"]
    for l in range(model.layers):
        y = F.layer_norm(x, (model.width,), p[f"{l}.ln1.w"], p[f"{l}.ln1.b"])
        qkv = (y @ p[f"{l}.qkv"].T).view(t, h + 2 * hk, model.head_dim).transpose(0, 1)
        q, k, v = qkv[:h], qkv[h:h + hk].repeat_interleave(h // hk, 0), qkv[h + hk:].repeat_interleave(h // hk, 0)
        s = q @ k.transpose(1, 2) * model.head_dim ** -0.5
        s = s.masked_fill(torch.triu(torch.ones(t, t, dtype=torch.bool, device="cuda"), 1), float("-inf"))
        o = (torch.softmax(s, -1) @ v).transpose(0, 1).reshape(t, -1)
        x = x + o @ p[f"{l}.out"].T
        y = F.layer_norm(x, (model.width,), p[f"{l}.ln2.w"], p[f"{l}.ln2.b"])
        x = x + F.gelu(y @ p[f"{l}.up"].T) @ p[f"{l}.down"].T
    y = F.layer_norm(x, (model.width,), p["ln.w"], p["ln.b"])
    return F.cross_entropy(y @ p["head"].T, want)


def test_gradients_of_each_worker():
    model = Gpt(vocab=32, width=64, heads=4, kv_heads=2, layers=2, length=70)
    m = 3
    tokens = sequences(m, 1, model.length, model.vocab)[:, 0]
    buf = torch.full((2, m, model.d), float("nan"), device="cuda")
    losses = model.loss_and_gradients(tokens, buf[1])
    assert binding.operators_status() == binding.OK
    assert torch.isnan(buf[0]).all()
    for i in range(m):
        p = {n: w.detach().clone().requires_grad_(True) for n, w in model.p.items()}
        loss = reference_loss(model, p, tokens[i])
        loss.backward()
        assert abs(float(loss) - float(losses[i])) <= 2e-2
        for n, w in p.items():
            got = model.grad(buf[1], n)[i]
            # a dozen bf16 products deep, each rounding by up to 2^-8 and mostly independently: about 1 % of the norm
            assert float((got - w.grad).norm()) <= 3e-2 * float(w.grad.norm()) + 1e-6, n


def test_training_in_coordinated_order():
    model = Gpt(vocab=32, width=64, heads=2, kv_heads=1, layers=1, length=64)
    history = train(model, workers=4, examples=16, epochs=4, log=lambda *_: None)
    assert all(torch.isfinite(torch.tensor(history)))
    assert history[-1] < 0.9 * history[0]
