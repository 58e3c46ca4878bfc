"""The training operators beside the order server: what is timed, and their plain forms.

Five operators produce or consume what the order server works on.  Layer normalisation and
attention, forward and backward, are the parts of a transformer block that are no matrix
product with a weight; their backward passes make the stale gradients that are balanced (the
layer norm's weight gradient comes out per worker, a row of the gather buffer each).  The
orthogonalised update turns the averaged gradient of a weight matrix into the step taken.

    layer_norm_forward    y = (x - mean) * rstd * w + b, with mean and rstd per row
    layer_norm_backward   dx per row, dw and db summed over each worker's own rows
    attention_forward     o = softmax(scale q k^T) v, with the log-sum-exp of every row
    attention_backward    dq, dk, dv from the recomputed probabilities
    orthogonalise         five steps X <- a X + (b A + c A^2) X, A = X X^T, from X = g / |g|

Sizes are those of the framework's workloads (the GPT-2-sized model's width of 768 in 12 heads of
64 with 64 workers, the LSTM's width of 650 with gate matrices of 650 x 2600) or generic ones.
"""
import math

import torch

own = False          # False: the plain forms; True: the framework's kernels

COEFFS = (3.4445, -4.7750, 2.0315)
STEPS = 5
EPS_NORM = 1e-5
EPS_ORTH = 1e-7
TORCH = {"f32": torch.float32, "bf16": torch.bfloat16}
SIZE = {"f32": 4, "bf16": 2}


# ------------------------------------------------------------------------------------- cases
def listed():
    return [
        # one short sequence for each of four workers in a narrow model: all launch latency
        dict(name="ln fwd 4x8x64 f32", op="ln_fwd", workers=4, rows=8, cols=64, dtype="f32"),
        # the LSTM's width (650: rows that are no multiple of 16 bytes), 32 workers, 512 tokens each
        dict(name="ln fwd 32x512x650 bf16", op="ln_fwd", workers=32, rows=512, cols=650, dtype="bf16"),
        # odd rows and columns, seven workers, full precision
        dict(name="ln bwd 7x333x1025 f32", op="ln_bwd", workers=7, rows=333, cols=1025, dtype="f32", grads="f32"),
        # the GPT-2-sized model's width, a 1024-token sequence for each of 64 workers
        dict(name="ln bwd 64x1024x768 bf16", op="ln_bwd", workers=64, rows=1024, cols=768, dtype="bf16", grads="bf16"),
        # a toy model on short odd sequences
        attn("attn fwd b4 t33 h2 d32", "attn_fwd", 4, 33, 33, 2, 2, 32, causal=True),
        # one layer of the GPT-2-sized model, sixteen sequences, q k v in one projection's output
        attn("attn fwd b16 t1024 h12 d64", "attn_fwd", 16, 1024, 1024, 12, 12, 64, causal=True, packed=True),
        # long padded sequences of unequal length, four query heads to a key head
        attn("attn fwd b2 t4096 h16/4 d128", "attn_fwd", 2, 4096, 4096, 16, 4, 128, ragged=True),
        # odd lengths, more queries than keys: under the causal rule 100 rows see no key
        attn("attn bwd b3 t357/257 h6/2 d80", "attn_bwd", 3, 357, 257, 6, 2, 80, causal=True),
        # the same layer of the GPT-2-sized model, backward
        attn("attn bwd b16 t1024 h12 d64", "attn_bwd", 16, 1024, 1024, 12, 12, 64, causal=True, packed=True),
        # one long sequence, causal, shared key heads
        attn("attn bwd b1 t4096 h16/4 d128", "attn_bwd", 1, 4096, 4096, 16, 4, 128, causal=True),
        # the LSTM's gate matrix: its averaged gradient
        dict(name="orth 1x650x2600 f32", op="orth", batch=1, rows=650, cols=2600, dtype="f32"),
        # the attention projections of twelve layers, tall matrices
        dict(name="orth 12x2304x768 bf16", op="orth", batch=12, rows=2304, cols=768, dtype="bf16"),
    ]


def attn(name, op, batch, len_q, len_kv, heads, kv_heads, head_dim, causal=False, ragged=False, packed=False):
    return dict(name=name, op=op, batch=batch, len_q=len_q, len_kv=len_kv, heads=heads, kv_heads=kv_heads,
                head_dim=head_dim, causal=causal, ragged=ragged, packed=packed)


def spread(rng, lo, hi):
    """A whole number between lo and hi, uniform in its logarithm."""
    return max(lo, min(hi, round(math.exp(rng.uniform(math.log(lo), math.log(hi))))))


def draw(rng):
    op = rng.choice(("ln_fwd", "ln_bwd", "attn_fwd", "attn_bwd", "orth"))
    if op in ("ln_fwd", "ln_bwd"):
        cols = spread(rng, 32, 8192)
        workers = spread(rng, 1, 64)
        rows = spread(rng, 1, max(1, min(4096, 25_000_000 // (cols * workers))))
        case = dict(op=op, workers=workers, rows=rows, cols=cols, dtype=rng.choice(("f32", "bf16")))
        if op == "ln_bwd":
            case["grads"] = rng.choice(("f32", "bf16"))
        return case
    if op == "orth":
        batch = spread(rng, 1, 12)
        small = spread(rng, 16, 1024)
        wide = min(spread(rng, small, 8 * small), 21_000_000 // (batch * small))
        wide = max(wide, small) + rng.choice((0, 0, 1, 5))
        rows, cols = rng.choice(((small, wide), (wide, small)))
        cost = STEPS * small * small * (3 * wide + small)
        batch = max(1, min(batch, 270_000_000_000 // cost))
        return dict(op=op, batch=batch, rows=rows, cols=cols, dtype=rng.choice(("f32", "bf16")))
    head_dim = rng.choice((16, 32, 40, 64, 64, 80, 96, 128))
    kv_heads = rng.choice((1, 2, 4, 6))
    heads = kv_heads * rng.choice((1, 1, 2, 4))
    # with a single key the probability is one whatever the score, and dq and dk are zero but for rounding:
    # the backward pass is drawn from two keys on
    least = 2 if op == "attn_bwd" else 1
    most = min(4096, math.isqrt(130_000_000 // heads))
    len_q = spread(rng, least, most)
    len_kv = rng.choice((len_q, len_q, spread(rng, max(least, len_q // 2), min(most, 2 * len_q))))
    batch = spread(rng, 1, max(1, min(32, 100_000_000 // (len_q * len_kv * heads))))
    return dict(op=op, batch=batch, len_q=len_q, len_kv=len_kv, heads=heads, kv_heads=kv_heads, head_dim=head_dim,
                causal=rng.random() < 0.6, ragged=rng.random() < 0.3, packed=len_q == len_kv and rng.random() < 0.5)


def lengths(case):
    """The padded batch's lengths (queries, keys) of each sequence: part of the case, not of the seed."""
    b, tq, tk = case["batch"], case["len_q"], case["len_kv"]
    if not case["ragged"]:
        return [tq] * b, [tk] * b
    # the first sequence full, the others between about a third of the length and all of it
    part = [1.0] + [0.35 + 0.65 * ((i * 0.6180339887) % 1.0) for i in range(1, b)]
    return [max(1, int(tq * p)) for p in part], [max(1, int(tk * p)) for p in part]


# ------------------------------------------------------------------------------------ inputs
def prepare(case, seed):
    gen = torch.Generator(device="cuda").manual_seed(int(seed) * 7919 + 17)

    def randn(*shape):
        return torch.randn(*shape, generator=gen, device="cuda")

    op, st = case["op"], dict(case)
    if op in ("ln_fwd", "ln_bwd"):
        w, r, c, dt = case["workers"], case["rows"], case["cols"], TORCH[case["dtype"]]
        # residual-stream activations: a mean and a scale of their own for each token, some channels larger
        x = randn(w * r, c) * (0.5 + 1.5 * torch.rand(w * r, 1, generator=gen, device="cuda")) + 0.3 * randn(w * r, 1)
        x = x * (1.0 + 4.0 * (torch.rand(c, generator=gen, device="cuda") < 0.02))
        st["x"] = x.to(dt)
        st["weight"] = 1.0 + 0.1 * randn(c)
        st["bias"] = 0.1 * randn(c)
        if op == "ln_bwd":
            st["dy"] = (randn(w * r, c) * 1e-2).to(dt)
            xf = st["x"].float()
            st["mean"] = xf.mean(dim=1)
            st["rstd"] = torch.rsqrt((xf - st["mean"][:, None]).square().mean(dim=1) + EPS_NORM)
            # this parameter's columns [weight | bias] in the workers' rows of the gather buffer
            st["grad_rows"] = torch.zeros(w, 2 * c, dtype=TORCH[case["grads"]], device="cuda")
        return st
    if op == "orth":
        b, r, c = case["batch"], case["rows"], case["cols"]
        # a gradient of the GPT-2-sized workload's kind: half its energy in a rank-16 part
        k = min(16, r, c)
        g = torch.matmul(randn(b, r, k), randn(b, k, c)) / math.sqrt(2.0 * k) + randn(b, r, c) / math.sqrt(2.0)
        st["g"] = (g * 1e-2).to(TORCH[case["dtype"]])
        return st
    b, tq, tk, h, hk, d = (case[n] for n in ("batch", "len_q", "len_kv", "heads", "kv_heads", "head_dim"))
    if case["packed"]:   # one projection's output [batch][token][heads + 2 kv_heads][head_dim]
        qkv = randn(b, tq, h + 2 * hk, d).to(torch.bfloat16)
        st["q"], st["k"], st["v"] = qkv[:, :, :h], qkv[:, :, h:h + hk], qkv[:, :, h + hk:]
    else:
        st["q"] = randn(b, tq, h, d).to(torch.bfloat16)
        st["k"] = randn(b, tk, hk, d).to(torch.bfloat16)
        st["v"] = randn(b, tk, hk, d).to(torch.bfloat16)
    st["q_lens"] = st["kv_lens"] = None
    if case["ragged"]:
        lq, lk = lengths(case)
        st["q_lens"] = torch.tensor(lq, dtype=torch.int32, device="cuda")
        st["kv_lens"] = torch.tensor(lk, dtype=torch.int32, device="cuda")
    if op == "attn_bwd":
        st["do"] = randn(b, tq, h, d).to(torch.bfloat16)
        st["o"], st["lse"] = attention_forward_plain(st)
    return st


# ------------------------------------------------------------------------------- plain forms
def seen(st):
    """Which keys each query sees, [batch][1][1][len_q][len_kv], or None where all see all.  Sequence b has its
    first q_lens[b] queries and kv_lens[b] keys; the causal rule aligns their ends."""
    tq, tk, dev = st["len_q"], st["len_kv"], st["q"].device
    if not st["causal"] and st["q_lens"] is None:
        return None
    i = torch.arange(tq, device=dev)[:, None]
    j = torch.arange(tk, device=dev)[None, :]
    if st["q_lens"] is None:
        return (j <= i + (tk - tq))[None, None, None]
    lq, lk = st["q_lens"][:, None, None], st["kv_lens"][:, None, None]
    m = (i < lq) & (j < lk)
    if st["causal"]:
        m = m & (j <= i + (lk - lq))
    return m[:, None, None]


def by_head(t, groups):
    """[b][t][heads][d] in 32 bits as [b][kv heads][heads per kv head][t][d]."""
    b, n, h, d = t.shape
    return t.float().permute(0, 2, 1, 3).reshape(b, groups, h // groups, n, d)


def by_token(t):
    b, g, r, n, d = t.shape
    return t.reshape(b, g * r, n, d).permute(0, 2, 1, 3).to(torch.bfloat16).contiguous()


def scores(st):
    q, k = by_head(st["q"], st["kv_heads"]), by_head(st["k"], st["kv_heads"])
    return q, k, torch.matmul(q, k.transpose(-1, -2)) * (1.0 / math.sqrt(st["head_dim"]))


def attention_forward_plain(st):
    v = by_head(st["v"], st["kv_heads"])
    s = scores(st)[2]
    m = seen(st)
    if m is not None:
        s = s.masked_fill(~m, -math.inf)
    top = s.amax(dim=-1, keepdim=True)
    top = torch.where(torch.isfinite(top), top, torch.zeros_like(top))
    p = torch.exp(s - top)
    total = p.sum(dim=-1, keepdim=True)
    o = torch.matmul(p, v) / torch.where(total > 0, total, torch.ones_like(total))
    lse = (top + torch.log(total))[..., 0]
    return by_token(o), lse.reshape(lse.shape[0], -1, lse.shape[-1]).contiguous()


def attention_backward_plain(st):
    hk = st["kv_heads"]
    scale = 1.0 / math.sqrt(st["head_dim"])
    v, do, o = by_head(st["v"], hk), by_head(st["do"], hk), by_head(st["o"], hk)
    q, k, s = scores(st)
    lse = st["lse"].reshape(s.shape[:-1])[..., None]
    p = torch.exp(s - torch.where(torch.isfinite(lse), lse, torch.zeros_like(lse)))
    m = seen(st)
    if m is not None:
        p = p.masked_fill(~m, 0.0)
    delta = (do * o).sum(dim=-1, keepdim=True)
    ds = p * (torch.matmul(do, v.transpose(-1, -2)) - delta)
    dq = torch.matmul(ds, k) * scale
    dk = torch.matmul(ds.transpose(-1, -2), q).sum(dim=2, keepdim=True) * scale
    dv = torch.matmul(p.transpose(-1, -2), do).sum(dim=2, keepdim=True)
    return by_token(dq), by_token(dk), by_token(dv)


def layer_norm_forward_plain(st):
    x = st["x"].float()
    mean = x.mean(dim=1)
    dev = x - mean[:, None]
    rstd = torch.rsqrt(dev.square().mean(dim=1) + EPS_NORM)
    y = dev * rstd[:, None] * st["weight"] + st["bias"]
    return y.to(st["x"].dtype), mean, rstd


def layer_norm_backward_plain(st):
    w, r, c = st["workers"], st["rows"], st["cols"]
    dy = st["dy"].float()
    n = (st["x"].float() - st["mean"][:, None]) * st["rstd"][:, None]
    g = dy * st["weight"]
    dx = st["rstd"][:, None] * (g - g.mean(dim=1, keepdim=True) - n * (g * n).mean(dim=1, keepdim=True))
    dw = (dy * n).reshape(w, r, c).sum(dim=1)
    db = dy.reshape(w, r, c).sum(dim=1)
    return dx.to(st["x"].dtype), torch.cat((dw, db), dim=1).to(st["grad_rows"].dtype)


def orthogonalise_plain(st):
    a, b, c = COEFFS
    x = st["g"].float()
    tall = x.shape[1] > x.shape[2]
    if tall:
        x = x.transpose(1, 2)
    x = x / (x.square().sum(dim=(1, 2), keepdim=True).sqrt() + EPS_ORTH)
    for _ in range(STEPS):
        gram = torch.matmul(x, x.transpose(1, 2))
        x = a * x + torch.matmul(b * gram + c * torch.matmul(gram, gram), x)
    return (x.transpose(1, 2) if tall else x).to(torch.bfloat16).contiguous()


# --------------------------------------------------------------------------------------- run
def run(state):
    op = state["op"]
    if own:
        return run_own(op, state)
    if op == "ln_fwd":
        return dict(zip(("y", "mean", "rstd"), layer_norm_forward_plain(state)))
    if op == "ln_bwd":
        return dict(zip(("dx", "grads"), layer_norm_backward_plain(state)))
    if op == "attn_fwd":
        return dict(zip(("o", "lse"), attention_forward_plain(state)))
    if op == "attn_bwd":
        return dict(zip(("dq", "dk", "dv"), attention_backward_plain(state)))
    return {"o": orthogonalise_plain(state)}


def run_own(op, st):
    from paper_2302_00845_b200 import binding
    if op == "ln_fwd":
        return dict(zip(("y", "mean", "rstd"),
                        binding.layer_norm_forward(st["x"], st["weight"], st["bias"], eps=EPS_NORM)))
    if op == "ln_bwd":
        c, rows = st["cols"], st["grad_rows"]
        dx = binding.layer_norm_backward(st["dy"], st["x"], st["weight"], st["mean"], st["rstd"],
                                         rows[:, :c], rows[:, c:])
        return {"dx": dx, "grads": rows}
    if op == "attn_fwd":
        return dict(zip(("o", "lse"), binding.attention_forward(
            st["q"], st["k"], st["v"], causal=st["causal"], q_lens=st["q_lens"], kv_lens=st["kv_lens"])))
    if op == "attn_bwd":
        return dict(zip(("dq", "dk", "dv"), binding.attention_backward(
            st["do"], st["q"], st["k"], st["v"], st["o"], st["lse"], causal=st["causal"], q_lens=st["q_lens"],
            kv_lens=st["kv_lens"])))
    return {"o": binding.orthogonalise(st["g"], steps=STEPS, coeffs=COEFFS, eps=EPS_ORTH)}


# -------------------------------------------------------------------------------------- work
def pairs(case):
    """Query-key pairs that are not masked, over the batch, for one head."""
    total = 0
    for lq, lk in zip(*lengths(case)):
        if not case["causal"]:
            total += lq * lk
        else:      # query i sees the first i + lk - lq + 1 keys
            first = max(0, lq - lk)          # the first query that sees any
            n = lq - first
            total += n * (first + lk - lq + 1 + lk) // 2
    return total


def work(case):
    op = case["op"]
    if op in ("ln_fwd", "ln_bwd"):
        n, c, w, e = case["workers"] * case["rows"], case["cols"], case["workers"], SIZE[case["dtype"]]
        if op == "ln_fwd":      # x in, y out, two statistics a row, weight and bias
            return {"bytes": 2 * n * c * e + 8 * n + 8 * c, "flops": 8 * n * c}
        # dy and x in, dx out, two statistics a row, the weight, a row of dw and db for each worker
        return {"bytes": 3 * n * c * e + 8 * n + 4 * c + 2 * w * c * SIZE[case["grads"]], "flops": 14 * n * c}
    if op == "orth":
        b, r, c = case["batch"], case["rows"], case["cols"]
        m, n = min(r, c), max(r, c)
        # per step: X X^T and A^2 are symmetric (half the entries), B X is whole
        return {"bytes": b * r * c * (SIZE[case["dtype"]] + 2), "flops": b * STEPS * (m * m * n + m * m * m + 2 * m * m * n)}
    h, hk, d = case["heads"], case["kv_heads"], case["head_dim"]
    tq, tk = (sum(v) for v in lengths(case))
    p = pairs(case) * h
    # padded rows of o, dq, dk, dv are written (as zeros) like the others
    fq, fk = case["batch"] * case["len_q"], case["batch"] * case["len_kv"]
    if op == "attn_fwd":        # q k v in, o and the log-sum-exp out; two products
        return {"bytes": 2 * d * (h * tq + 2 * hk * tk + h * fq) + 4 * h * fq, "flops": 4 * d * p}
    # do q o k v and the log-sum-exp in, dq dk dv out; five products
    return {"bytes": 2 * d * (3 * h * tq + 2 * hk * tk + h * fq + 2 * hk * fk) + 4 * h * tq, "flops": 10 * d * p}


# ------------------------------------------------------------------------------------- exact
def exact(case, seed):
    """The definitions in 64 bits, one matrix or one head at a time."""
    st = prepare(case, seed)
    op = case["op"]
    if op in ("ln_fwd", "ln_bwd"):
        x = st["x"].double()
        var, mean = torch.var_mean(x, dim=1, correction=0, keepdim=True)
        rstd = 1.0 / torch.sqrt(var + EPS_NORM)
        n = (x - mean) * rstd
        if op == "ln_fwd":
            return {"y": torch.addcmul(st["bias"].double(), n, st["weight"].double()), "mean": mean[:, 0], "rstd": rstd[:, 0]}
        dy = st["dy"].double()
        g = dy * st["weight"].double()
        # the Jacobian of the normalisation: it takes out the constant and the n components of g
        c, w = case["cols"], case["workers"]
        dx = rstd * (g - g.sum(1, keepdim=True) / c - n * (torch.einsum("rc,rc->r", g, n)[:, None] / c))
        per = lambda t: torch.stack([p.sum(0) for p in t.chunk(w)])  # noqa: E731
        return {"dx": dx, "grads": torch.cat((per(dy * n), per(dy)), 1)}
    if op == "orth":
        out = torch.empty(st["g"].shape, dtype=torch.float64, device="cuda")
        for i, g in enumerate(st["g"].double()):
            wide = g if g.shape[0] <= g.shape[1] else g.T
            x = wide / (torch.linalg.matrix_norm(wide) + EPS_ORTH)
            # every step multiplies by a polynomial of X X^T, whose eigenvectors stay: O = U h(lambda) U^T X
            lam, u = torch.linalg.eigh(x @ x.T)
            lam, h = lam.clamp(min=0.0), torch.ones_like(lam)
            for _ in range(STEPS):
                f = COEFFS[0] + COEFFS[1] * lam + COEFFS[2] * lam * lam
                h, lam = h * f, lam * f * f
            o = (u * h) @ (u.T @ x)
            out[i] = o if wide is g else o.T
        return {"o": out}
    b, tq, tk, h, hk, d = (case[n] for n in ("batch", "len_q", "len_kv", "heads", "kv_heads", "head_dim"))
    f64 = dict(dtype=torch.float64, device="cuda")
    o, lse = torch.zeros(b, tq, h, d, **f64), torch.full((b, h, tq), -math.inf, **f64)
    dq, dk, dv = torch.zeros(b, tq, h, d, **f64), torch.zeros(b, tk, hk, d, **f64), torch.zeros(b, tk, hk, d, **f64)
    for i, (lq, lk) in enumerate(zip(*lengths(case))):
        for j in range(h):
            kv = j // (h // hk)
            q, k, v = st["q"][i, :lq, j].double(), st["k"][i, :lk, kv].double(), st["v"][i, :lk, kv].double()
            s = (q @ k.T) / math.sqrt(d)
            if case["causal"]:
                s += torch.triu(torch.full((lq, lk), -math.inf, **f64), diagonal=lk - lq + 1)
            l = torch.logsumexp(s, dim=1)
            p = torch.exp(s - l.clamp(min=-1e300)[:, None])
            if op == "attn_fwd":
                o[i, :lq, j], lse[i, j, :lq] = p @ v, l
                continue
            g = st["do"][i, :lq, j].double()
            dp = g @ v.T
            ds = p * (dp - (p * dp).sum(1, keepdim=True)) / math.sqrt(d)
            dq[i, :lq, j] = ds @ k
            dk[i, :lk, kv] += ds.T @ q
            dv[i, :lk, kv] += p.T @ g
    return {"o": o, "lse": lse} if op == "attn_fwd" else {"dq": dq, "dk": dk, "dv": dv}
