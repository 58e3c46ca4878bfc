"""Embedding, dropout and the norms and rotation of queries and keys in 64 bits, with bounds summed from the roundings
that a kernel makes whose sums are held in 32 bits."""
import numpy as np
import torch

from operators_ref import SLACK, U16, U32


# ---- embedding ---------------------------------------------------------------------------------------
def embedding_forward(tokens, table, scale, padding, out_dtype):
    """(value, bound)"""
    t = tokens.reshape(-1).long()
    ok = (t >= 0) & (t < table.shape[0])
    if padding is not None:
        ok &= t != padding
    y = torch.zeros(t.numel(), table.shape[1], dtype=torch.float64, device=table.device)
    y[ok] = table.double()[t[ok]] * float(np.float32(scale))
    return y, SLACK * (U32 + U16[out_dtype]) * y.abs()


def embedding_backward(dy, tokens, m, vocab, scale, padding, grad_dtype, old=None):
    """(value, bound) of [m][vocab][cols]; old: what the sums are added to"""
    cols = dy.shape[1]
    t = tokens.reshape(m, -1).long()
    ok = (t >= 0) & (t < vocab)
    if padding is not None:
        ok &= t != padding
    key = (torch.where(ok, t, 0) + vocab * torch.arange(m, device=dy.device)[:, None]).reshape(-1)[ok.reshape(-1)]
    d = dy.double()[ok.reshape(-1)]
    f64 = dict(dtype=torch.float64, device=dy.device)
    add = lambda v: torch.zeros(m * vocab, v.shape[1], **f64).index_add_(0, key, v)  # noqa: E731
    total, size, count = add(d), add(d.abs()), add(torch.ones(d.shape[0], 1, **f64))
    s = float(np.float32(scale))
    g, err = s * total, (count + 2) * U32 * abs(s) * size          # a chain of additions as long as the run, the product
    if old is not None:
        before = old.double().reshape(m * vocab, cols)
        g = g + before
        err = torch.where(count > 0, err + U32 * g.abs(), 0.0)
    err = err + torch.where(count > 0, U16[grad_dtype] * g.abs(), 0.0)
    return g.view(m, vocab, cols), SLACK * err.view(m, vocab, cols)


# ---- dropout -----------------------------------------------------------------------------------------
def philox(block, call, step, seed):
    """Four words of Philox4x32-10 for each block number (Salmon et al., SC 2011)."""
    block = np.asarray(block, dtype=np.uint64)
    low, half = np.uint64(0xFFFFFFFF), np.uint64(32)
    c = [block & low, block >> half, np.full_like(block, call), np.full_like(block, step)]
    k = [seed & 0xFFFFFFFF, seed >> 32]
    for _ in range(10):
        p0, p1 = np.uint64(0xD2511F53) * c[0], np.uint64(0xCD9E8D57) * c[2]
        c = [(p1 >> half) ^ c[1] ^ np.uint64(k[0]), p1 & low, (p0 >> half) ^ c[3] ^ np.uint64(k[1]), p0 & low]
        k = [(k[0] + 0x9E3779B9) & 0xFFFFFFFF, (k[1] + 0xBB67AE85) & 0xFFFFFFFF]
    return np.stack(c, axis=-1).astype(np.uint32)


def keep(index, p, seed, call, step):
    """Which elements of these indices stay."""
    index = np.asarray(index, dtype=np.int64)
    words = philox(index // 8, call, step, seed)
    e = index % 8
    bits = (np.take_along_axis(words, (e // 2)[..., None], -1)[..., 0] >> (16 * (e % 2)).astype(np.uint32)) & 0xFFFF
    return bits >= int(np.floor(65536 * p + 0.5))


def dropout(x, p, seed, call, step, residual, out_dtype):
    """(value, bound)"""
    rows, cols = x.shape
    stay = torch.from_numpy(keep(np.arange(rows * cols).reshape(rows, cols), p, seed, call, step)).to(x.device)
    limit = int(np.floor(65536 * p + 0.5))
    y = torch.where(stay, x.double() / ((65536 - limit) / 65536 if limit < 65536 else 1.0), 0.0)
    err = 2 * U32 * y.abs()                                # the factor and the product
    if residual is not None:
        y = y + residual.double()
        err = err + U32 * y.abs()
    return y, SLACK * (err + U16[out_dtype] * y.abs())


# ---- norms and rotation ----------------------------------------------------------------------------
def pairs(rotary_dim, interleaved):
    i = torch.arange(rotary_dim // 2)
    return (2 * i, 2 * i + 1) if interleaved else (i, i + rotary_dim // 2)


def turned(x, err, angle, far, rotary_dim, interleaved, back=False):
    """x [b][t][h][d] with its pairs turned by angle [b][t][rotary_dim / 2], and the error that goes with it: `far`
    is how far the angle itself may be off."""
    if rotary_dim == 0:
        return x, err
    a, b = (i.to(x.device) for i in pairs(rotary_dim, interleaved))
    c, s = torch.cos(angle)[:, :, None], torch.sin(angle)[:, :, None] * (-1 if back else 1)
    y, e = x.clone(), err.clone()
    y[..., a], y[..., b] = x[..., a] * c - x[..., b] * s, x[..., a] * s + x[..., b] * c
    # the angle's fraction is rounded to 32 bits (half a unit of 1/2 turn: pi 2^-24), the functions are within two
    # units, the two products and the sum round once each
    size = x[..., a].abs() + x[..., b].abs()
    per = size * (8 * U32 + far[:, :, None]) + err[..., a] + err[..., b]
    e[..., a], e[..., b] = per, per
    return y, e


def rotary(x, w, pos, base, rotary_dim, interleaved, eps, lens, dy=None, m=1, grad_dtype=None):
    """(y, bound), or with dy: ((dx, bound), (dw [m][d], bound))"""
    b, t, h, d = x.shape
    dev, dt = x.device, x.dtype
    live = torch.ones(b, t, 1, 1, dtype=torch.bool, device=dev)
    if lens is not None:
        live = (torch.arange(t, device=dev)[None] < lens.long()[:, None])[:, :, None, None]
    x = torch.where(live, x.double(), 0.0)
    w = torch.ones(d, dtype=torch.float64, device=dev) if w is None else w.double()
    pos = (torch.arange(t, device=dev).expand(b, t) if pos is None else pos.expand(b, t)).double()
    half = rotary_dim // 2
    freq = float(base) ** (-2.0 * torch.arange(half, dtype=torch.float64, device=dev) / max(rotary_dim, 1))
    angle = pos[:, :, None] * freq
    far = angle.abs() * 2.0 ** -50            # products of 53 bits on both sides
    rstd = 1.0 / torch.sqrt(x.square().mean(-1, keepdim=True) + float(np.float32(eps)))
    rstd = torch.where(live, rstd, 0.0)       # (with eps = 0 what is padded has none)
    rel = (d / 2 + 6) * U32                   # a sum of d squares, halved by the root; the root, the division
    n = x * rstd
    if dy is None:
        g = n * w
        y, err = turned(g, (rel + 2 * U32) * g.abs(), angle, far, rotary_dim, interleaved)
        y = torch.where(live, y, 0.0)
        return y, SLACK * torch.where(live, err + U16[dt] * y.abs(), 0.0)
    dy = torch.where(live, dy.double(), 0.0)
    g, gerr = turned(dy, torch.zeros_like(dy), angle, far, rotary_dim, interleaved, back=True)
    n_err = (rel + U32) * n.abs()
    hh, herr = g * w, gerr * w.abs() + U32 * (g * w).abs()
    c = (hh * n).mean(-1, keepdim=True)
    cerr = (herr * n.abs() + hh.abs() * n_err).mean(-1, keepdim=True) + (d + 4) * U32 * (hh * n).abs().mean(-1, keepdim=True)
    dx = rstd * (hh - n * c)
    derr = rstd * (herr + n.abs() * cerr + n_err * c.abs() + 3 * U32 * (hh.abs() + (n * c).abs())) + rel * dx.abs() + U16[dt] * dx.abs()
    part = lambda v: v.reshape(m, -1, d).sum(1)  # noqa: E731
    dw = part(g * n)
    terms = b // m * t * h
    werr = part(gerr * n.abs() + g.abs() * n_err) + (terms + 8) * U32 * part((g * n).abs()) + U16[grad_dtype or torch.float32] * dw.abs()
    return (dx, SLACK * derr), (dw, SLACK * werr)
