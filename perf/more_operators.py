"""The operators around a model's attention and at its input: what is timed, and their plain forms.

They stand beside layer normalisation, attention and the orthogonalised update: the parts of a training
step that make the stale gradients which the order server balances, so that gradients of parameters come
out per worker, a row of the gather buffer each.

    embedding_forward     y = scale * table[token], zero for the padding token
    embedding_backward    every worker's gradient of the table: the sum of dy over its rows of each token
    dropout_forward       y = residual + x * keep / (1 - p), keep from a counter-based generator
    dropout_backward      dx = dy * keep / (1 - p), with the mask generated again
    rotary_forward        queries and keys, each head divided by its root mean square, times a weight, then
                          rotated by the token's position
    rotary_backward       their gradients, and the weights' gradients of each worker

The generator is Philox4x32-10 (Salmon et al., SC 2011) with the seed as key and the counter (block low, block
high, call, step): element i of a tensor takes 16 bits of block i // 8 and is dropped where they are below
T = round(65536 p); 1 - p stands for (65536 - T) / 65536.

Sizes are those of the framework's workloads (the GPT-2-sized model's width of 768 in 12 heads of 64 and its
vocabulary, the LSTM's width of 650) or generic ones.
"""
import math

import torch

own = False          # False: the plain forms; True: the framework's kernels

TORCH = {"f32": torch.float32, "bf16": torch.bfloat16, "i32": torch.int32, "i64": torch.int64}
SIZE = {"f32": 4, "bf16": 2, "i32": 4, "i64": 8}
EPS = 1e-6
PADDING = -1


# ------------------------------------------------------------------------------------- cases
def listed():
    return [
        # one short sequence for each of four workers over characters: all launch latency
        emb("emb fwd 4x16 v64 c64 f32", "emb_fwd", 4, 16, 64, 64, "f32"),
        # a 1024-token sequence for each of 64 workers in the GPT-2-sized model, with the usual factor of sqrt(width)
        emb("emb fwd 64x1024 v50257 c768 bf16", "emb_fwd", 64, 1024, 50257, 768, "bf16", scaled=True),
        # the LSTM's width and its twenty truncated sequences of 35 words for each of 32 workers, padded at the end
        emb("emb bwd 32x700 v10000 c650 f32", "emb_bwd", 32, 700, 10000, 650, "f32", grads="f32", ragged=True),
        # the GPT-2-sized model, a sequence for each of 16 workers: most of the table's gradient is zero
        emb("emb bwd 16x1024 v50257 c768 bf16", "emb_bwd", 16, 1024, 50257, 768, "bf16", grads="bf16", scaled=True),
        # a toy model's activations
        drop("drop fwd 132x32 f32", "drop_fwd", 132, 32, "f32", "f32", 0.1, residual=True),
        # the end of a block of the GPT-2-sized model: a 16-bit product's output onto the 32-bit residual stream
        drop("drop fwd 16384x768 bf16 onto f32", "drop_fwd", 16384, 768, "bf16", "f32", 0.1, residual=True),
        # between the LSTM's layers: 32 workers, 20 sequences of 35, an odd width
        drop("drop bwd 22400x650 bf16", "drop_bwd", 22400, 650, "bf16", "bf16", 0.5),
        # the activations of all 64 workers of the GPT-2-sized model
        drop("drop bwd 65536x768 bf16", "drop_bwd", 65536, 768, "bf16", "bf16", 0.1),
        # one new token for each of eight sequences, far into them
        rot("rot fwd b8 t1 h12/4 d64", "rot_fwd", 8, 1, 12, 4, 64, start=100_000),
        # one layer of the GPT-2-sized model, sixteen sequences, q and k slices of one projection's output
        rot("rot fwd b16 t1024 h12 d64", "rot_fwd", 16, 1024, 12, 12, 64, packed=True),
        # three workers, odd and padded lengths, full precision, neighbouring values rotated together
        rot("rot bwd b3 t357 h6/2 d80 f32", "rot_bwd", 3, 357, 6, 2, 80, workers=3, dtype="f32", interleaved=True, ragged=True),
        # long sequences of two workers, four query heads to a key head
        rot("rot bwd b4 t4096 h16/4 d128", "rot_bwd", 4, 4096, 16, 4, 128, workers=2),
    ]


def emb(name, op, workers, rows, vocab, cols, dtype, grads="bf16", tokens="i64", scaled=False, ragged=False):
    return dict(name=name, op=op, workers=workers, rows=rows, vocab=vocab, cols=cols, dtype=dtype, grads=grads,
                tokens=tokens, scaled=scaled, ragged=ragged)


def drop(name, op, rows, cols, dtype, out, p, residual=False):
    return dict(name=name, op=op, rows=rows, cols=cols, dtype=dtype, out=out, p=p, residual=residual)


def rot(name, op, batch, length, heads, kv_heads, head_dim, workers=1, dtype="bf16", rotary_dim=None, interleaved=False,
        start=0, packed=False, ragged=False):
    return dict(name=name, op=op, batch=batch, length=length, heads=heads, kv_heads=kv_heads, head_dim=head_dim,
                workers=workers, dtype=dtype, rotary_dim=rotary_dim or head_dim, interleaved=interleaved, start=start,
                packed=packed, ragged=ragged)


def spread(rng, lo, hi):
    """A whole number between lo and hi, uniform in its logarithm."""
    return max(lo, min(hi, round(math.exp(rng.uniform(math.log(lo), math.log(hi))))))


def draw(rng):
    op = rng.choice(("emb_fwd", "emb_bwd", "drop_fwd", "drop_bwd", "rot_fwd", "rot_bwd"))
    if op in ("emb_fwd", "emb_bwd"):
        cols = spread(rng, 16, 2048)
        workers = spread(rng, 1, 64)
        dtype, grads = rng.choice(("f32", "bf16")), rng.choice(("f32", "bf16"))
        tokens = 50_000_000 // cols
        most = 50257
        if op == "emb_bwd":
            tokens //= 2
            most = min(most, 600_000_000 // (cols * workers * SIZE[grads]))
        vocab = spread(rng, 32, max(32, most))
        rows = spread(rng, 1, max(1, min(8192, tokens // workers)))
        return emb("", op, workers, rows, vocab, cols, dtype, grads, rng.choice(("i32", "i64")), rng.random() < 0.5, rng.random() < 0.4)
    if op in ("drop_fwd", "drop_bwd"):
        cols = spread(rng, 8, 8192)
        rows = spread(rng, 1, 16_000_000 // cols)
        residual = op == "drop_fwd" and rng.random() < 0.7
        return drop("", op, rows, cols, rng.choice(("f32", "bf16")), rng.choice(("f32", "bf16")),
                    rng.choice((0.05, 0.1, 0.2, 0.25, 0.5)), residual)
    head_dim = rng.choice((16, 32, 40, 64, 64, 80, 96, 128, 128, 192, 256))
    kv_heads = rng.choice((1, 2, 4, 6))
    heads = kv_heads * rng.choice((1, 1, 2, 4))
    workers = spread(rng, 1, 16) if op == "rot_bwd" else 1
    per_token = (heads + kv_heads) * head_dim
    length = rng.choice((1, spread(rng, 2, 8192), spread(rng, 2, 8192), spread(rng, 2, 8192)))
    length = min(length, max(1, 12_000_000 // (per_token * workers)))
    batch = workers * spread(rng, 1, max(1, min(32, 12_000_000 // (per_token * length * workers))))
    return rot("", op, batch, length, heads, kv_heads, head_dim, workers, rng.choice(("f32", "bf16", "bf16")),
               rng.choice((head_dim, head_dim, head_dim // 16 * 8)), rng.random() < 0.4, rng.choice((0, 0, 4096, 131_072, 900_001)),
               rng.random() < 0.4, rng.random() < 0.3)


def shares(n, full):
    """The lengths of n padded sequences: part of the case, not of the seed.  The first one full, the others between a
    third of the length and all of it."""
    part = [1.0] + [0.35 + 0.65 * ((i * 0.6180339887) % 1.0) for i in range(1, n)]
    return [max(1, int(full * p)) for p in part]


# ------------------------------------------------------------------------------------ inputs
def prepare(case, seed):
    gen = torch.Generator(device="cuda").manual_seed(int(seed) * 6007 + 29)

    def randn(*shape):
        return torch.randn(*shape, generator=gen, device="cuda")

    op, st = case["op"], dict(case)
    if op in ("emb_fwd", "emb_bwd"):
        w, r, v, c, dt = case["workers"], case["rows"], case["vocab"], case["cols"], TORCH[case["dtype"]]
        # words by frequency: the i-th most frequent with a probability of about 1 / (i + 2.7), by the inverse of its sum
        u = torch.rand(w, r, generator=gen, dtype=torch.float64, device="cuda")
        t = (2.7 * (v / 2.7 + 1.0) ** u - 2.7).long().clamp(0, v - 1)
        if case["ragged"]:
            t = t.masked_fill(torch.arange(r, device="cuda") >= torch.tensor(shares(w, r), device="cuda")[:, None], PADDING)
        st["ids"] = t.to(TORCH[case["tokens"]])
        st["scale"] = math.sqrt(c) if case["scaled"] else 1.0
        if op == "emb_fwd":
            st["table"] = (randn(v, c) * 0.02).to(dt)
        else:
            st["dy"] = (randn(w * r, c) * 1e-2).to(dt)
            # the table's columns of the workers' rows of the gather buffer
            st["grad_rows"] = torch.zeros(w, v, c, dtype=TORCH[case["grads"]], device="cuda")
        return st
    if op in ("drop_fwd", "drop_bwd"):
        n, c = case["rows"], case["cols"]
        st["x"] = (randn(n, c) if op == "drop_fwd" else randn(n, c) * 1e-2).to(TORCH[case["dtype"]])
        st["res"] = randn(n, c).to(TORCH[case["out"]]) if case["residual"] else None
        # one generator for the run; which layer and which step draw from it
        st["seed"] = 0x9E3779B97F4A7C15 ^ (int(seed) * 0x1000193)
        st["call"], st["step"] = 11, 1000 + int(seed)
        return st
    b, t, h, hk, d, dt = (case[n] for n in ("batch", "length", "heads", "kv_heads", "head_dim", "dtype"))
    dt = TORCH[dt]
    if case["packed"]:      # one projection's output [batch][token][heads + 2 kv_heads][head_dim]
        qkv = randn(b, t, h + 2 * hk, d).to(dt)
        st["q"], st["k"] = qkv[:, :, :h], qkv[:, :, h:h + hk]
    else:
        st["q"], st["k"] = randn(b, t, h, d).to(dt), randn(b, t, hk, d).to(dt)
    st["q_weight"], st["k_weight"] = 1.0 + 0.1 * randn(d), 1.0 + 0.1 * randn(d)
    # where each sequence's tokens stand
    first = case["start"] + 17 * torch.arange(b, device="cuda")
    st["positions"] = None if case["start"] == 0 else first[:, None] + torch.arange(t, device="cuda")
    st["lens"] = torch.tensor(shares(b, t), dtype=torch.int32, device="cuda") if case["ragged"] else None
    if op == "rot_bwd":
        st["dq"], st["dk"] = (randn(b, t, h, d) * 1e-2).to(dt), (randn(b, t, hk, d) * 1e-2).to(dt)
        # the two weights' columns of the workers' rows of the gather buffer
        st["grad_rows"] = torch.zeros(case["workers"], 2 * d, device="cuda")
    return st


# ------------------------------------------------------------------------------- plain forms
def embedding_forward_plain(st):
    t = st["ids"].reshape(-1).long()
    used = t != PADDING
    y = st["table"][t.clamp(min=0)].float() * st["scale"]
    return (y * used[:, None]).to(st["table"].dtype)


def embedding_backward_plain(st):
    w, v, c = st["workers"], st["vocab"], st["cols"]
    t = st["ids"].long()
    used = t != PADDING
    row = (t.clamp(min=0) + v * torch.arange(w, device="cuda")[:, None]).reshape(-1)
    g = torch.zeros(w * v, c, device="cuda")
    g.index_add_(0, row, st["dy"].float() * (used.reshape(-1, 1) * st["scale"]))
    st["grad_rows"].copy_(g.view(w, v, c))
    return st["grad_rows"]


def draws(n, seed, call, step):
    """The 16 bits of elements 0 to n - 1: Philox4x32-10 on 32-bit words held in 64."""
    low = 0xFFFFFFFF
    block = torch.arange((n + 7) // 8, device="cuda")
    c0, c1, c2, c3 = block & low, block >> 32, torch.full_like(block, call), torch.full_like(block, step & low)
    k0, k1 = seed & low, (seed >> 32) & low

    def product(const, word):       # 32 x 32 bits: low and high words, by halves so that 64 bits with a sign hold them
        a, b = word & 0xFFFF, word >> 16
        lo = const * a
        hi = const * b + (lo >> 16)
        return ((hi & 0xFFFF) << 16) | (lo & 0xFFFF), hi >> 16

    for _ in range(10):
        lo0, hi0 = product(0xD2511F53, c0)
        lo1, hi1 = product(0xCD9E8D57, c2)
        c0, c1, c2, c3 = hi1 ^ c1 ^ k0, lo1, hi0 ^ c3 ^ k1, lo0
        k0, k1 = (k0 + 0x9E3779B9) & low, (k1 + 0xBB67AE85) & low
    words = torch.stack((c0, c1, c2, c3), dim=1)
    return torch.stack((words & 0xFFFF, words >> 16), dim=2).reshape(-1)[:n]


def kept(st):
    """Which elements stay, and the factor that keeps the mean."""
    limit = math.floor(65536 * st["p"] + 0.5)
    keep = draws(st["rows"] * st["cols"], st["seed"], st["call"], st["step"]) >= limit
    return keep.view(st["rows"], st["cols"]), 65536 / (65536 - limit)


def dropout_plain(st):
    keep, factor = kept(st)
    y = torch.where(keep, st["x"].float() * factor, 0.0)
    if st["res"] is not None:
        y = st["res"].float() + y
    return y.to(TORCH[st["out"]])


def turns(st):
    """cos and sin of every token's angles [batch or 1][length][1][rotary_dim / 2], taken in 64 bits: a far position
    times a frequency is many turns."""
    half = st["rotary_dim"] // 2
    freq = 10000.0 ** (-torch.arange(half, dtype=torch.float64, device="cuda") / half)
    pos = torch.arange(st["length"], device="cuda")[None] if st["positions"] is None else st["positions"]
    angle = pos.double()[:, :, None, None] * freq
    return torch.cos(angle).float(), torch.sin(angle).float()


def rotate(x, cos, sin, st):
    """The pairs of the first rotary_dim values turned; sin with its sign changed turns back."""
    r = st["rotary_dim"]
    if st["interleaved"]:
        a, b = x[..., 0:r:2], x[..., 1:r:2]
        turned = torch.stack((a * cos - b * sin, a * sin + b * cos), dim=-1).flatten(-2)
    else:
        a, b = x[..., :r // 2], x[..., r // 2:r]
        turned = torch.cat((a * cos - b * sin, a * sin + b * cos), dim=-1)
    return torch.cat((turned, x[..., r:]), dim=-1)


def in_use(st):
    """[batch][length][1][1]: the tokens before the padding."""
    if st["lens"] is None:
        return None
    return (torch.arange(st["length"], device="cuda") < st["lens"][:, None])[:, :, None, None]


def rotary_forward_plain(st):
    cos, sin = turns(st)
    used, out = in_use(st), []
    for x, w in ((st["q"], st["q_weight"]), (st["k"], st["k_weight"])):
        x = x.float()
        y = rotate(x * torch.rsqrt(x.square().mean(dim=-1, keepdim=True) + EPS) * w, cos, sin, st)
        out.append((y if used is None else y * used).to(st["q"].dtype))
    return out


def rotary_backward_plain(st):
    cos, sin = turns(st)
    used, out, d = in_use(st), [], st["head_dim"]
    for i, (dy, x, w) in enumerate(((st["dq"], st["q"], st["q_weight"]), (st["dk"], st["k"], st["k_weight"]))):
        x = x.float()
        rstd = torch.rsqrt(x.square().mean(dim=-1, keepdim=True) + EPS)
        n = x * rstd
        g = rotate(dy.float(), cos, -sin, st)
        if used is not None:
            g = g * used
        h = g * w
        out.append((rstd * (h - n * (h * n).mean(dim=-1, keepdim=True))).to(st["q"].dtype))
        st["grad_rows"][:, i * d:(i + 1) * d] = (g * n).reshape(st["workers"], -1, d).sum(dim=1)
    return out


# --------------------------------------------------------------------------------------- run
def run(state):
    op = state["op"]
    if own:
        return run_own(op, state)
    if op == "emb_fwd":
        return {"y": embedding_forward_plain(state)}
    if op == "emb_bwd":
        return {"grads": embedding_backward_plain(state)}
    if op in ("drop_fwd", "drop_bwd"):
        return {"y": dropout_plain(state)}
    if op == "rot_fwd":
        return dict(zip(("q", "k"), rotary_forward_plain(state)))
    return dict(zip(("dq", "dk"), rotary_backward_plain(state)), grads=state["grad_rows"])


def run_own(op, st):
    from paper_2302_00845_b200 import binding
    if op == "emb_fwd":
        return {"y": binding.embedding_forward(st["ids"], st["table"], scale=st["scale"], padding=PADDING)}
    if op == "emb_bwd":
        binding.embedding_backward(st["dy"], st["ids"], st["grad_rows"], scale=st["scale"], padding=PADDING)
        return {"grads": st["grad_rows"]}
    if op == "drop_fwd":
        return {"y": binding.dropout_forward(st["x"], st["p"], st["seed"], call=st["call"], step=st["step"], residual=st["res"],
                                             dtype=TORCH[st["out"]])}
    if op == "drop_bwd":
        return {"y": binding.dropout_backward(st["x"], st["p"], st["seed"], call=st["call"], step=st["step"],
                                              dtype=TORCH[st["out"]])}
    kw = dict(positions=st["positions"], rotary_dim=st["rotary_dim"], interleaved=st["interleaved"], eps=EPS, lens=st["lens"])
    if op == "rot_fwd":
        return dict(zip(("q", "k"), binding.rotary_forward(st["q"], st["k"], st["q_weight"], st["k_weight"], **kw)))
    d, rows = st["head_dim"], st["grad_rows"]
    dq, dk = binding.rotary_backward(st["dq"], st["dk"], st["q"], st["k"], st["q_weight"], st["k_weight"],
                                     dq_weight=rows[:, :d], dk_weight=rows[:, d:], **kw)
    return {"dq": dq, "dk": dk, "grads": rows}


# -------------------------------------------------------------------------------------- work
def work(case):
    op = case["op"]
    if op in ("emb_fwd", "emb_bwd"):
        w, r, v, c, e = case["workers"], case["rows"], case["vocab"], case["cols"], SIZE[case["dtype"]]
        used = sum(shares(w, r)) if case["ragged"] else w * r
        if op == "emb_fwd":     # tokens in, each row that some token names (their expected number) once, y out
            total = math.log(v / 2.7 + 1.0)
            rows = sum(-math.expm1(used * math.log1p(-math.log1p(1.0 / (i + 2.7)) / total)) for i in range(v))
            return {"bytes": w * r * SIZE[case["tokens"]] + int(rows) * c * e + w * r * c * e, "flops": used * c}
        # tokens and the rows of dy in use in, every worker's gradient of the table out
        return {"bytes": w * r * SIZE[case["tokens"]] + used * c * e + w * v * c * SIZE[case["grads"]], "flops": 2 * used * c}
    if op in ("drop_fwd", "drop_bwd"):
        n = case["rows"] * case["cols"]
        out = SIZE[case["out"]]
        # ten rounds of two products and four exclusive ors for eight elements, a comparison and a product for each
        return {"bytes": n * (SIZE[case["dtype"]] + out * (2 if case["residual"] else 1)), "flops": n * 10}
    b, t, h, hk, d, e = (case[n] for n in ("batch", "length", "heads", "kv_heads", "head_dim", "dtype"))
    e = SIZE[e]
    used = (sum(shares(b, t)) if case["ragged"] else b * t) * (h + hk) * d
    full = b * t * (h + hk) * d
    pos = 0 if case["start"] == 0 else 8 * b * t
    if op == "rot_fwd":     # q and k in, both out (padded tokens as zeros), two weights
        return {"bytes": (used + full) * e + 8 * d + pos, "flops": 8 * used}
    # dq, dk, q and k in, two gradients out, two weights, two sums for each worker
    return {"bytes": (2 * used + full) * e + 8 * d + pos + 8 * case["workers"] * d, "flops": 16 * used}


# ------------------------------------------------------------------------------------- exact
def exact(case, seed):
    """The definitions in 64 bits."""
    st = prepare(case, seed)
    op = case["op"]
    f64 = dict(dtype=torch.float64, device="cuda")
    if op == "emb_fwd":
        t = st["ids"].flatten().long()
        y = torch.zeros(t.numel(), case["cols"], **f64)
        at = (t >= 0).nonzero()[:, 0]
        y[at] = torch.index_select(st["table"], 0, t[at]).double() * st["scale"]
        return {"y": y}
    if op == "emb_bwd":
        # one worker at a time: its rows sorted by token, summed within each run
        g = torch.zeros(case["workers"], case["vocab"], case["cols"], **f64)
        for i, (t, dy) in enumerate(zip(st["ids"].long(), st["dy"].view(case["workers"], case["rows"], -1))):
            at = (t >= 0).nonzero()[:, 0]
            which, inverse = torch.unique(t[at], return_inverse=True)
            part = torch.zeros(which.numel(), case["cols"], **f64)
            part.scatter_add_(0, inverse[:, None].expand(-1, case["cols"]), dy[at].double())
            g[i, which] = part * st["scale"]
        return {"grads": g}
    if op in ("drop_fwd", "drop_bwd"):
        keep = philox_mask(case["rows"] * case["cols"], st["seed"], st["call"], st["step"], case["p"])
        share = (65536 - int(65536 * case["p"] + 0.5)) / 65536
        y = torch.zeros(case["rows"] * case["cols"], **f64)
        y[keep] = st["x"].flatten()[keep].double() / share
        y = y.view(case["rows"], case["cols"])
        return {"y": y if st["res"] is None else y + st["res"].double()}
    # a rotation of a pair is a product of complex numbers
    b, t, d, r = (case[n] for n in ("batch", "length", "head_dim", "rotary_dim"))
    i = torch.arange(0, r, 2, **f64)
    pos = torch.arange(t, **f64).expand(b, t) if st["positions"] is None else st["positions"].double()
    phase = torch.polar(torch.ones(1, **f64), pos[:, :, None, None] * torch.exp(-math.log(10000.0) * i / r))
    if st["interleaved"]:
        order = torch.arange(r, device="cuda").view(-1, 2)
    else:
        order = torch.arange(r, device="cuda").view(2, -1).T
    live = torch.ones(b, t, 1, 1, dtype=torch.bool, device="cuda")
    if st["lens"] is not None:
        live = (torch.arange(t, device="cuda")[None] < st["lens"].long()[:, None])[..., None, None]

    def turned(x, by):
        y = x.clone()
        z = torch.complex(x[..., order[:, 0]], x[..., order[:, 1]]) * by
        y[..., order[:, 0]], y[..., order[:, 1]] = z.real, z.imag
        return torch.where(live, y, 0.0)

    out, sums = [], []
    for name in ("q", "k"):
        x, w = st[name].double(), st[name + "_weight"].double()
        rms = torch.sqrt(torch.linalg.vector_norm(x, dim=-1, keepdim=True) ** 2 / d + EPS)
        if op == "rot_fwd":
            out.append(turned(x / rms * w, phase))
            continue
        g = turned(st["d" + name].double(), phase.conj())
        along = torch.einsum("bthd,bthd,d->bth", g, x, w)[..., None]
        out.append(g * w / rms - x * along / (d * rms ** 3))
        sums.append((g * x / rms).view(case["workers"], -1, d).sum(dim=1))
    if op == "rot_fwd":
        return dict(zip(("q", "k"), out))
    return dict(zip(("dq", "dk"), out), grads=torch.cat(sums, dim=1))


def philox_mask(n, seed, call, step, p):
    """keep of every element, the generator written with numpy's unsigned words."""
    import numpy as np
    block = np.arange((n + 7) // 8, dtype=np.uint64)
    mask, shift = np.uint64(0xFFFFFFFF), np.uint64(32)
    c = [block & mask, block >> shift, np.full_like(block, call), np.full_like(block, step & 0xFFFFFFFF)]
    for rnd in range(10):
        k = [np.uint64(((seed >> s) + rnd * inc) & 0xFFFFFFFF) for s, inc in ((0, 0x9E3779B9), (32, 0xBB67AE85))]
        a, b = c[0] * np.uint64(0xD2511F53), c[2] * np.uint64(0xCD9E8D57)
        c = [(b >> shift) ^ c[1] ^ k[0], b & mask, (a >> shift) ^ c[3] ^ k[1], a & mask]
    words = np.stack(c, axis=1).astype("<u4").view("<u2").reshape(-1)[:n]
    return torch.from_numpy((words >= int(65536 * p + 0.5))).cuda()
