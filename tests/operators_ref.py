"""The training operators in 64 bits, and how far a kernel that holds its sums in 32 bits and its matrix
operands in 16 may be from them: every bound is summed from the roundings that are made."""
import math

import torch

U32 = 2.0 ** -24           # unit roundoff: 24 significant bits
U16 = {torch.float32: 2.0 ** -24, torch.bfloat16: 2.0 ** -8}   # bfloat16 has 8
SLACK = 1.25               # second-order terms


def rows64(x, w, b, eps):
    x = x.double()
    mean = x.mean(dim=1, keepdim=True)
    var = (x - mean).square().mean(dim=1, keepdim=True)
    rstd = 1.0 / torch.sqrt(var + eps)
    n = (x - mean) * rstd
    w = torch.ones(x.shape[1], dtype=torch.float64, device=x.device) if w is None else w.double()
    b = torch.zeros_like(w) if b is None else b.double()
    return x, mean, rstd, n, w, b


def layer_norm_forward(x, w, b, eps):
    """(y, bound), (mean, bound), (rstd, bound)"""
    dt = x.dtype
    x, mean, rstd, n, w, b = rows64(x, w, b, eps)
    cols = x.shape[1]
    # a sum of c values in any order of adding partial sums: at most (log2 c + c / 1024 + 4) roundings deep
    depth = (math.log2(cols + 1) + cols / 1024 + 36) * U32
    mean_err = depth * x.abs().mean(dim=1, keepdim=True) + U32 * mean.abs()
    # 1/sqrt(var + eps): half the relative error of var, and the function's own two units
    rstd_err = rstd * (depth + 4 * U32 + mean_err.square() * rstd.square())
    n_err = mean_err * rstd + (2 * U32 + depth) * n.abs() + U32 * (x.abs() + mean.abs()) * rstd
    y = n * w + b
    y_err = w.abs() * n_err + 2 * U32 * (n * w).abs() + U32 * b.abs() + U16[dt] * y.abs()
    return (y, SLACK * y_err), (mean[:, 0], SLACK * mean_err[:, 0]), (rstd[:, 0], SLACK * rstd_err[:, 0])


def layer_norm_backward(dy, x, w, mean, rstd, m, grad_dtype):
    """(dx, bound), (dw, bound), (db, bound) from the statistics as they are given"""
    dt = x.dtype
    x, dy, mu, rs = x.double(), dy.double(), mean.double()[:, None], rstd.double()[:, None]
    cols, rows = x.shape[1], x.shape[0] // m
    w = torch.ones(cols, dtype=torch.float64, device=x.device) if w is None else w.double()
    n = (x - mu) * rs
    n_err = U32 * (3 * n.abs() + (x.abs() + mu.abs()) * rs)
    g = dy * w
    depth = (math.log2(cols + 1) + cols / 1024 + 36) * U32
    c1, c2 = g.mean(dim=1, keepdim=True), (g * n).mean(dim=1, keepdim=True)
    c1_err = depth * g.abs().mean(dim=1, keepdim=True)
    c2_err = depth * (g * n).abs().mean(dim=1, keepdim=True) + (g.abs() * n_err).mean(dim=1, keepdim=True)
    dx = rs * (g - c1 - n * c2)
    dx_err = rs * (c1_err + n.abs() * c2_err + n_err * c2.abs() + 6 * U32 * (g.abs() + c1.abs() + (n * c2).abs()))
    dx_err = dx_err + U16[dt] * dx.abs()
    part = lambda t: t.reshape(m, rows, cols).sum(dim=1)  # noqa: E731
    deep = (rows + 8) * U32          # the longest chain of additions is a worker's whole column
    dw, db = part(dy * n), part(dy)
    dw_err = deep * part((dy * n).abs()) + part(dy.abs() * n_err) + U16[grad_dtype] * dw.abs()
    db_err = deep * part(dy.abs()) + U16[grad_dtype] * db.abs()
    return (dx, SLACK * dx_err), (dw, SLACK * dw_err), (db, SLACK * db_err)


def visible(tq, tk, lq, lk, causal, dev):
    i = torch.arange(tq, device=dev)[:, None]
    j = torch.arange(tk, device=dev)[None, :]
    m = (i < lq) & (j < lk)
    return m & (j <= i + (lk - lq)) if causal else m


def attention(q, k, v, causal, scale, q_lens=None, kv_lens=None, do=None):
    """Dict of name -> (value, bound).  o and lse always; dq, dk, dv where do is given.  What lies in masked
    rows is replaced by zeros first: it must not matter."""
    b, tq, h, d = q.shape
    tk, hk = k.shape[1], k.shape[2]
    dev, u = q.device, U16[torch.bfloat16]
    f64 = dict(dtype=torch.float64, device=dev)
    names = ["o", "lse"] + (["dq", "dk", "dv"] if do is not None else [])
    shapes = dict(o=q.shape, lse=(b, h, tq), dq=q.shape, dk=k.shape, dv=v.shape)
    out = {n: (torch.zeros(shapes[n], **f64), torch.zeros(shapes[n], **f64)) for n in names}
    out["lse"][0].fill_(-math.inf)
    for bi in range(b):
        lq = tq if q_lens is None else int(q_lens[bi])
        lk = tk if kv_lens is None else int(kv_lens[bi])
        m = visible(tq, tk, lq, lk, causal, dev)
        if not m.any():
            continue
        rq, rk = torch.arange(tq, device=dev)[:, None] < lq, torch.arange(tk, device=dev)[:, None] < lk
        for hi in range(h):
            g = hi // (h // hk)
            qq = torch.where(rq, q[bi, :, hi].double(), 0.0)
            kk, vv = torch.where(rk, k[bi, :, g].double(), 0.0), torch.where(rk, v[bi, :, g].double(), 0.0)
            s = scale * (qq @ kk.T)
            # the score: d products added in 32 bits, then a product with the scale (and log2 e)
            s_abs = abs(scale) * (qq.abs() @ kk.abs().T)
            s_err = (d / 8 + 8) * U32 * s_abs
            s = torch.where(m, s, -math.inf)
            lse = torch.logsumexp(s, dim=1)
            some = m.any(dim=1)
            p = torch.where(m, torch.exp(s - torch.where(some, lse, 0.0)[:, None]), 0.0)
            worst = torch.where(m, s_err, 0.0).amax(dim=1)
            o = p @ vv
            # the exponential's own error, that of its argument, the stored probability's rounding
            p_rel = s_err + worst[:, None] + 16 * U32 + 2 * U32 * (lse.abs().nan_to_num(posinf=0.0)[:, None] + s_abs)
            out["o"][0][bi, :, hi] = o
            out["o"][1][bi, :, hi] = SLACK * ((p * (u + 2 * p_rel)) @ vv.abs() + u * o.abs())
            out["lse"][0][bi, hi] = lse
            out["lse"][1][bi, hi] = SLACK * (worst + (16 + tk / 16) * U32 + 4 * U32 * lse.abs().nan_to_num(posinf=0.0) + 2 * U32 * s_abs.amax(dim=1))
            if do is None:
                continue
            dd = torch.where(rq, do[bi, :, hi].double(), 0.0)
            dp = dd @ vv.T
            delta = (p * dp).sum(dim=1, keepdim=True)
            # o is read as the forward pass rounded it, twice its bound
            delta_err = (dd.abs() * (out["o"][1][bi, :, hi] + d * U32 * o.abs())).sum(dim=1, keepdim=True)
            ds = p * (dp - delta)
            ds_err = p * (delta_err + (d / 8 + 4) * U32 * (dd.abs() @ vv.abs().T)) + ds.abs() * (u + 2 * p_rel)
            a = abs(scale)
            dq, dk, dv = scale * ds @ kk, scale * ds.T @ qq, p.T @ dd
            out["dq"][0][bi, :, hi] = dq
            out["dq"][1][bi, :, hi] = SLACK * (a * ds_err @ kk.abs() + u * dq.abs() + a * tk / 16 * U32 * ds.abs() @ kk.abs())
            out["dk"][0][bi, :, g] += dk
            out["dk"][1][bi, :, g] += SLACK * (a * ds_err.T @ qq.abs() + a * tq / 16 * U32 * ds.abs().T @ qq.abs())
            out["dv"][0][bi, :, g] += dv
            out["dv"][1][bi, :, g] += SLACK * ((p * (u + 2 * p_rel)).T @ dd.abs() + tq / 16 * U32 * p.T @ dd.abs())
    for n in ("dk", "dv"):
        if n in out:        # one rounding of the whole sum
            out[n][1].add_(SLACK * u * out[n][0].abs())
    return out


def orthogonalise(g, steps=5, coeffs=(3.4445, -4.7750, 2.0315), eps=1e-7):
    a, b, c = coeffs
    x = g.double()
    tall = x.shape[-2] > x.shape[-1]
    x = x.mT if tall else x
    x = x / (x.square().sum(dim=(-2, -1), keepdim=True).sqrt() + eps)
    for _ in range(steps):
        s = x @ x.mT
        x = a * x + (b * s + c * s @ s) @ x
    return x.mT if tall else x


def assert_within(got, want, bound, name=""):
    got = got.double()
    assert got.shape == want.shape, name
    inf = torch.isinf(want)
    assert torch.equal(got[inf], want[inf]), name
    assert torch.isfinite(got[~inf]).all(), f"{name}: not finite"
    over = ((got - want).abs() - bound)[~inf]
    tiny = 1e-30
    if over.numel():
        worst = float(((got - want).abs()[~inf] / (bound[~inf] + tiny)).max())
        assert float(over.max()) <= tiny, f"{name}: {worst:.3g} times the bound"
