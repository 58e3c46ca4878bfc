"""A small GPT trained in coordinated order: every operator of the library in one training loop.

    python -m paper_2302_00845_b200.train_gpt [--workers M] [--examples N] [--epochs E] [--order cdgrab|random] ...

m workers hold n sequences each (an order-1 Markov source of their own, so that workers differ).  Per pair of
positions every worker's two sequences go through the model; the per-worker gradients land in the gather buffer
[2][m][d] that the order server balances: those of the layer norms straight from layer_norm_backward, the embedding's
from embedding_backward, those of the matrices from one product per worker.  Optionally queries and keys are normed
and rotated by position in place of learned positions, and the residual branches dropped out.  step_mean balances
the pair and averages it; the averages of the matrices, with momentum, are orthogonalised, those of vectors and
embeddings follow their root mean square.
The paper's workers compute their gradients the same way (Algorithm 3); the model is its GPT-2 in small.
"""
from __future__ import annotations

import argparse
import math
import time

import torch

from . import binding


class Gpt:
    """Pre-norm transformer with its backward pass written out; parameters are views of one flat float32
    vector, gradients of worker i views of row i of a gather buffer."""

    def __init__(self, vocab=64, width=128, heads=4, kv_heads=2, layers=2, length=128, seed=0, rotary=False, dropout=0.0):
        self.vocab, self.width, self.heads, self.kv_heads, self.layers, self.length = vocab, width, heads, kv_heads, layers, length
        self.rotary, self.dropout, self.seed, self.steps = rotary, dropout, seed, 0      # steps: masks drawn so far
        self.head_dim = width // heads
        qkv = (heads + 2 * kv_heads) * self.head_dim
        spec = [("embed", (vocab, width))] + ([] if rotary else [("pos", (length, width))])
        for l in range(layers):
            spec += [(f"{l}.q.w", (self.head_dim,)), (f"{l}.k.w", (self.head_dim,))] if rotary else []
            spec += [(f"{l}.ln1.w", (width,)), (f"{l}.ln1.b", (width,)), (f"{l}.qkv", (qkv, width)), (f"{l}.out", (width, width)),
                     (f"{l}.ln2.w", (width,)), (f"{l}.ln2.b", (width,)), (f"{l}.up", (4 * width, width)), (f"{l}.down", (width, 4 * width))]
        spec += [("ln.w", (width,)), ("ln.b", (width,)), ("head", (vocab, width))]
        self.shapes, self.offset, at = dict(spec), {}, 0
        for name, shape in spec:
            self.offset[name] = at
            at += (math.prod(shape) + 7) // 8 * 8
        self.d = at
        self.flat = torch.zeros(self.d, device="cuda")
        self.p = {n: self.flat[self.offset[n]:][:math.prod(s)].view(s) for n, s in spec}
        gen = torch.Generator(device="cuda").manual_seed(seed)
        for n, w in self.p.items():
            if n.endswith(".w"):
                w.fill_(1.0)
            elif w.dim() == 2:
                w.normal_(0.0, 0.02 if n in ("embed", "pos") else w.shape[1] ** -0.5, generator=gen)
        self.matrices = [n for n, s in spec if len(s) == 2 and n not in ("embed", "pos", "head")]

    def grad(self, buf, name):
        """The workers' gradients of one parameter: a view [m][...] of a gather buffer's slab [m][d]."""
        s = self.shapes[name]
        return buf[:, self.offset[name]:self.offset[name] + math.prod(s)].view(buf.shape[0], *s)

    def loss_and_gradients(self, tokens, buf):
        """tokens [m][length + 1]: one sequence per worker.  Fills buf [m][d]; returns the workers' mean losses [m]."""
        m, t, c, p = tokens.shape[0], self.length, self.width, self.p
        h, hk, hd = self.heads, self.kv_heads, self.head_dim
        bf = {n: p[n].bfloat16() for n in self.matrices + ["head"]}
        want = tokens[:, 1:].long()
        per = lambda y: y.view(m, t, -1)  # noqa: E731

        def weight_gradient(name, dy, x):        # worker i's dW = dy_i^T x_i
            self.grad(buf, name).copy_(torch.bmm(per(dy).transpose(1, 2), per(x)))

        def branch(call, y, x):                  # x + y, with y dropped out
            if not self.dropout:
                return x + y.float()
            return binding.dropout_forward(y, self.dropout, self.seed, call, self.steps, residual=x)

        def branch_backward(call, dx):           # y's gradient
            if not self.dropout:
                return dx.bfloat16()
            return binding.dropout_backward(dx, self.dropout, self.seed, call, self.steps, dtype=torch.bfloat16)

        def norm_backward(name, dy, x, stats):
            return binding.layer_norm_backward(dy, x, p[name + ".w"], *stats, self.grad(buf, name + ".w"), self.grad(buf, name + ".b"))

        x = binding.embedding_forward(tokens[:, :-1], p["embed"])
        if not self.rotary:
            x = (x.view(m, t, c) + p["pos"]).view(m * t, c)
        tape = []
        for l in range(self.layers):
            y1, *s1 = binding.layer_norm_forward(x, p[f"{l}.ln1.w"], p[f"{l}.ln1.b"])
            y1 = y1.bfloat16()
            qkv = (y1 @ bf[f"{l}.qkv"].T).view(m, t, h + 2 * hk, hd)
            q, k, v = qkv[:, :, :h], qkv[:, :, h:h + hk], qkv[:, :, h + hk:]
            q2, k2 = binding.rotary_forward(q, k, p[f"{l}.q.w"], p[f"{l}.k.w"]) if self.rotary else (q, k)
            o, lse = binding.attention_forward(q2, k2, v, causal=True)
            x1 = branch(2 * l, o.view(m * t, c) @ bf[f"{l}.out"].T, x)
            y2, *s2 = binding.layer_norm_forward(x1, p[f"{l}.ln2.w"], p[f"{l}.ln2.b"])
            y2 = y2.bfloat16()
            u = y2 @ bf[f"{l}.up"].T
            a = torch.nn.functional.gelu(u)
            tape.append((x, s1, y1, qkv, q2, k2, o, lse, x1, s2, y2, u, a))
            x = branch(2 * l + 1, a @ bf[f"{l}.down"].T, x1)
        y, *s = binding.layer_norm_forward(x, p["ln.w"], p["ln.b"])
        y = y.bfloat16()
        logits = (y @ bf["head"].T).float()
        logp = torch.log_softmax(logits, dim=1)
        losses = -logp.gather(1, want.reshape(-1, 1)).view(m, t).mean(dim=1)

        dlogits = logp.exp()
        dlogits.scatter_add_(1, want.reshape(-1, 1), torch.full((m * t, 1), -1.0, device="cuda"))
        dlogits = (dlogits / t).bfloat16()
        weight_gradient("head", dlogits, y)
        dx = norm_backward("ln", (dlogits @ bf["head"]).float(), x, s)
        for l in reversed(range(self.layers)):
            x0, s1, y1, qkv, q2, k2, o, lse, x1, s2, y2, u, a = tape[l]
            dy = branch_backward(2 * l + 1, dx)
            weight_gradient(f"{l}.down", dy, a)
            du = torch.ops.aten.gelu_backward(dy @ bf[f"{l}.down"], u)
            weight_gradient(f"{l}.up", du, y2)
            dx = dx + norm_backward(f"{l}.ln2", (du @ bf[f"{l}.up"]).float(), x1, s2)
            dy = branch_backward(2 * l, dx)
            weight_gradient(f"{l}.out", dy, o.view(m * t, c))
            d_o = (dy @ bf[f"{l}.out"]).view(m, t, h, hd)
            dqkv = torch.empty_like(qkv)
            dq, dk, dv = dqkv[:, :, :h], dqkv[:, :, h:h + hk], dqkv[:, :, h + hk:]
            binding.attention_backward(d_o, q2, k2, qkv[:, :, h + hk:], o, lse, causal=True, dq=dq, dk=dk, dv=dv)
            if self.rotary:
                binding.rotary_backward(dq, dk, qkv[:, :, :h], qkv[:, :, h:h + hk], p[f"{l}.q.w"], p[f"{l}.k.w"],
                                        dq_weight=self.grad(buf, f"{l}.q.w"), dk_weight=self.grad(buf, f"{l}.k.w"), q_out=dq, k_out=dk)
            dqkv = dqkv.view(m * t, -1)
            weight_gradient(f"{l}.qkv", dqkv, y1)
            dx = dx + norm_backward(f"{l}.ln1", (dqkv @ bf[f"{l}.qkv"]).float(), x0, s1)
        if not self.rotary:
            self.grad(buf, "pos").copy_(dx.view(m, t, c))
        binding.embedding_backward(dx, tokens[:, :-1], self.grad(buf, "embed"))
        self.steps += 1
        return losses


class Update:
    """Momentum; matrices take the orthogonalised direction, the rest divides by its root mean square."""

    def __init__(self, model: Gpt, lr=0.02, momentum=0.9):
        self.model, self.lr, self.momentum = model, lr, momentum
        self.mom, self.sq, self.count = torch.zeros_like(model.flat), torch.zeros_like(model.flat), 0
        # matrices of one shape go through the products as one batch
        self.groups = {}
        for n in model.matrices:
            self.groups.setdefault(model.shapes[n], []).append(n)

    def step(self, g):
        mdl, self.count = self.model, self.count + 1
        self.mom.mul_(self.momentum).add_(g)
        self.sq.mul_(0.95).addcmul_(g, g, value=0.05)
        look = g + self.momentum * self.mom
        rms = (self.sq / (1 - 0.95 ** self.count)).sqrt().add_(1e-8)
        rest = (look * (1 - self.momentum) / rms).mul_(-0.25 * self.lr)
        for shape, names in self.groups.items():
            size = math.prod(shape)
            u = torch.stack([look[mdl.offset[n]:mdl.offset[n] + size].view(shape) for n in names])
            o = binding.orthogonalise(u).float()
            scale = max(1.0, shape[0] / shape[1]) ** 0.5
            for n, w in zip(names, o):
                rest[mdl.offset[n]:mdl.offset[n] + size] = (w * (-self.lr * scale)).view(-1)
        mdl.flat.add_(rest)


def sequences(m, n, length, vocab, seed=0):
    """[m][n][length + 1] tokens; each worker has its own order-1 source over a shared skeleton."""
    gen = torch.Generator(device="cuda").manual_seed(seed + 77)
    shared = torch.randn(vocab, vocab, generator=gen, device="cuda") * 2.0
    own = torch.randn(m, vocab, vocab, generator=gen, device="cuda") * 1.5
    prob = torch.softmax(shared + own, dim=2)
    out = torch.empty(m, n, length + 1, dtype=torch.int64, device="cuda")
    out[:, :, 0] = torch.randint(vocab, (m, n), generator=gen, device="cuda")
    rows = torch.arange(m, device="cuda")[:, None]
    for i in range(length):
        out[:, :, i + 1] = torch.multinomial(prob[rows, out[:, :, i]].view(m * n, vocab), 1, generator=gen).view(m, n)
    return out


def train(model: Gpt, workers=8, examples=16, epochs=4, order="cdgrab", lr=0.02, seed=0, log=print):
    """Mean training loss of each epoch."""
    m, n = workers, examples
    data = sequences(m, n, model.length, model.vocab, seed)
    update = Update(model, lr)
    grads = torch.zeros(2, m, model.d, device="cuda")
    mean = torch.empty(2, model.d, device="cuda")
    perms = torch.empty(m, n, dtype=torch.int32, device="cuda")
    gen = torch.Generator(device="cuda").manual_seed(seed)
    rows, history = torch.arange(m, device="cuda"), []
    with binding.CdGrab(m, n, model.d, "f32") as server:
        current = server.perms().long()
        for epoch in range(epochs):
            if order == "random":
                current = torch.argsort(torch.rand(m, n, generator=gen, device="cuda"), dim=1)
            server.begin_epoch()
            start, total = time.perf_counter(), torch.zeros((), device="cuda")
            for k in range(n // 2):
                for slab in range(2):
                    total += model.loss_and_gradients(data[rows, current[:, 2 * k + slab]], grads[slab]).mean()
                server.step_mean(grads, mean)
                update.step(mean.mean(dim=0))
            server.end_epoch(perms)
            server.check_status()
            binding._check(binding.operators_status(), "cdgrab_operators_status")
            current = perms.long().clone()
            history.append(float(total) / (n // 2 * 2))
            log(f"epoch {epoch}: loss {history[-1]:.4f}  ({time.perf_counter() - start:.2f} s, order {order})")
    return history


def main():
    ap = argparse.ArgumentParser(description=__doc__.splitlines()[0])
    ap.add_argument("--workers", type=int, default=8)
    ap.add_argument("--examples", type=int, default=32)
    ap.add_argument("--epochs", type=int, default=6)
    ap.add_argument("--width", type=int, default=128)
    ap.add_argument("--layers", type=int, default=2)
    ap.add_argument("--length", type=int, default=128)
    ap.add_argument("--lr", type=float, default=0.02)
    ap.add_argument("--rotary", action="store_true", help="norms and rotation of queries and keys in place of learned positions")
    ap.add_argument("--dropout", type=float, default=0.0)
    ap.add_argument("--order", choices=("cdgrab", "random"), default="cdgrab")
    a = ap.parse_args()
    model = Gpt(width=a.width, layers=a.layers, length=a.length, rotary=a.rotary, dropout=a.dropout)
    print(f"{model.d} parameters, {a.workers} workers x {a.examples} sequences of {a.length}")
    train(model, a.workers, a.examples, a.epochs, a.order, a.lr)


if __name__ == "__main__":
    main()
