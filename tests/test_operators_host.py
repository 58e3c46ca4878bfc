"""Argument checks of the training operators, which come before any use of a device, and the 64-bit formulas
that the GPU tests compare with, against automatic differentiation."""
import ctypes as C
import math
import os
import subprocess
import sys

import pytest
import torch

import operators_ref as ref
from paper_2302_00845_b200 import binding, build


@pytest.fixture(scope="module")
def lib():
    build.build()
    return binding.lib()


P = 1 << 20       # a non-null, aligned address that is never read


def shape(**kw):
    s = dict(batch=2, len_q=16, len_kv=16, heads=4, kv_heads=2, head_dim=64, causal=1, scale=0.125)
    strides = {n: kw.pop(n, None) for n in ("q", "k", "v", "o", "do", "dq", "dk", "dv")}
    s.update(kw)
    sh = binding.AttentionShape(*[s[n] for n in ("batch", "len_q", "len_kv", "heads", "kv_heads", "head_dim", "causal", "scale")])
    for n, v in strides.items():
        h = s["heads"] if n in ("q", "o", "do", "dq") else s["kv_heads"]
        v = v or (16 * h * s["head_dim"], h * s["head_dim"], s["head_dim"])
        for i in range(3):
            getattr(sh, n + "_stride")[i] = v[i]
    return sh


def test_layer_norm_arguments(lib):
    def fwd(rows=4, cols=8, dtype=0, x=P, xs=8, w=P, b=P, eps=1e-5, y=P, ys=8, mean=P, rstd=P):
        return lib.cdgrab_layer_norm_forward(rows, cols, dtype, x, xs, w, b, eps, y, ys, mean, rstd, None)
    for bad in (dict(rows=-1), dict(rows=1 << 31), dict(cols=0), dict(dtype=2), dict(x=None), dict(y=None), dict(xs=7), dict(ys=7),
                dict(eps=-1e-9), dict(eps=math.nan), dict(x=P + 2), dict(dtype=1, y=P + 1), dict(w=P + 2), dict(mean=P + 1)):
        assert fwd(**bad) == binding.ERR_INVALID, bad
    assert fwd(rows=0) == binding.OK

    def bwd(m=2, rows=4, cols=8, dtype=0, dy=P, dys=8, x=P, xs=8, w=P, mean=P, rstd=P, dx=P, dxs=8, gd=0, dw=P, db=P,
            ws=8, work=P, size=1 << 30):
        return lib.cdgrab_layer_norm_backward(m, rows, cols, dtype, dy, dys, x, xs, w, mean, rstd, dx, dxs, gd, dw, db, ws,
                                              work, size, None)
    for bad in (dict(m=0), dict(rows=-1), dict(cols=0), dict(dtype=5), dict(gd=5), dict(dy=None), dict(x=None), dict(mean=None),
                dict(rstd=None), dict(dys=7), dict(xs=7), dict(dxs=7), dict(ws=7), dict(work=None), dict(size=0),
                dict(work=P + 8), dict(dw=P + 2), dict(m=1 << 15, rows=1 << 16)):
        assert bwd(**bad) == binding.ERR_INVALID, bad
    assert lib.cdgrab_layer_norm_workspace_bytes(0, 1, 1) == -1
    assert lib.cdgrab_layer_norm_workspace_bytes(4, 100, 64) >= 0


def test_attention_arguments(lib):
    def fwd(sh, q=P, k=P, v=P, ql=None, kl=None, o=P, lse=P):
        return lib.cdgrab_attention_forward(C.byref(sh) if sh else None, q, k, v, ql, kl, o, lse, None)
    assert fwd(None) == binding.ERR_INVALID
    for bad in (dict(batch=-1), dict(len_q=-1), dict(len_kv=-1), dict(heads=0), dict(kv_heads=0), dict(heads=3), dict(head_dim=0),
                dict(head_dim=20), dict(head_dim=136), dict(causal=2), dict(scale=math.inf), dict(scale=math.nan),
                dict(q=(4096, 256, 60)), dict(k=(4096, 32, 64)), dict(v=(-8, 128, 64)), dict(o=(0, 256, 64)), dict(o=(4096, 256, 32))):
        assert fwd(shape(**bad)) == binding.ERR_INVALID, bad
        if set(bad) <= {"batch", "len_q", "len_kv", "heads", "kv_heads", "head_dim", "causal", "scale"}:
            assert lib.cdgrab_attention_workspace_bytes(C.byref(shape(**bad))) == -1
    for bad in (dict(q=None), dict(k=None), dict(v=None), dict(o=None), dict(lse=None), dict(q=P + 8), dict(k=P + 2), dict(v=P + 4),
                dict(o=P + 8), dict(lse=P + 2), dict(ql=P + 1), dict(kl=P + 2)):
        assert fwd(shape(), **bad) == binding.ERR_INVALID, bad
    assert fwd(shape(batch=0)) == binding.OK and fwd(shape(len_q=0)) == binding.OK

    def bwd(sh, do=P, q=P, k=P, v=P, o=P, lse=P, dq=P, dk=P, dv=P, work=P, size=1 << 30):
        return lib.cdgrab_attention_backward(C.byref(sh), do, q, k, v, o, lse, None, None, dq, dk, dv, work, size, None)
    for bad in (dict(do=None), dict(q=None), dict(k=None), dict(v=None), dict(o=None), dict(lse=None), dict(dq=None), dict(dk=None),
                dict(dv=None), dict(work=None), dict(size=16), dict(work=P + 8), dict(dk=P + 8), dict(do=P + 2)):
        assert bwd(shape(), **bad) == binding.ERR_INVALID, bad
    for bad in (dict(dq=(0, 256, 64)), dict(dk=(2048, 128, 0)), dict(dv=(2048, 0, 64)), dict(do=(4096, 256, 4))):
        assert bwd(shape(**bad)) == binding.ERR_INVALID, bad


def test_orthogonalise_arguments(lib):
    def call(batch=2, rows=8, cols=16, dtype=0, g=P, gb=128, gs=16, steps=5, co=(1.0, 1.0, 1.0), eps=0.0, o=P, ob=128, os=16,
             work=P, size=1 << 40):
        return lib.cdgrab_orthogonalise(batch, rows, cols, dtype, g, gb, gs, steps, (C.c_float * 3)(*co) if co else None, eps, o,
                                        ob, os, work, size, None)
    for bad in (dict(batch=-1), dict(rows=-1), dict(cols=-1), dict(dtype=2), dict(g=None), dict(o=None), dict(work=None), dict(steps=0),
                dict(steps=65), dict(co=None), dict(co=(math.nan, 0, 0)), dict(eps=-1.0), dict(eps=math.nan), dict(gs=15), dict(os=15),
                dict(ob=100), dict(gb=-1), dict(size=0), dict(work=P + 8), dict(g=P + 2), dict(o=P + 1), dict(rows=1 << 21)):
        assert call(**bad) == binding.ERR_INVALID, bad
    assert call(batch=0) == binding.OK and call(rows=0) == binding.OK and call(cols=0) == binding.OK
    assert lib.cdgrab_orthogonalise_workspace_bytes(-1, 8, 8) == -1


def test_no_cpu_fallback(lib):
    if torch.cuda.is_available():
        pytest.skip("a CUDA device is present")
    assert lib.cdgrab_layer_norm_forward(4, 8, 0, P, 8, None, None, 1e-5, P, 8, None, None, None) == binding.ERR_DEVICE
    assert lib.cdgrab_attention_forward(C.byref(shape()), P, P, P, None, None, P, P, None) == binding.ERR_DEVICE
    assert lib.cdgrab_operators_status() == binding.ERR_DEVICE


def test_attention_formulas_against_autograd():
    torch.manual_seed(0)
    b, tq, tk, h, hk, d = 2, 9, 7, 4, 2, 8
    q, k, v, do = (torch.randn(b, t, n, d, dtype=torch.float64) for t, n in ((tq, h), (tk, hk), (tk, hk), (tq, h)))
    for causal, ql, kl in ((False, None, None), (True, None, None), (True, [5, 9], [7, 3]), (False, [0, 9], [7, 0])):
        for t in (q, k, v):
            t.requires_grad_(True)
            t.grad = None
        s = torch.einsum("bihd,bjhd->bhij", q, k.repeat_interleave(h // hk, 2)) * 0.3
        m = torch.stack([ref.visible(tq, tk, tq if ql is None else ql[i], tk if kl is None else kl[i], causal, "cpu") for i in range(b)])[:, None]
        p = torch.where(m, torch.exp(s), 0.0)
        p = p / p.sum(-1, keepdim=True).clamp(min=1e-300)
        o = torch.einsum("bhij,bjhd->bihd", p, v.repeat_interleave(h // hk, 2))
        o.backward(do)
        got = ref.attention(q.detach(), k.detach(), v.detach(), causal, 0.3, ql, kl, do)
        for name, want in (("o", o.detach()), ("dq", q.grad), ("dk", k.grad), ("dv", v.grad)):
            assert torch.allclose(got[name][0], want, rtol=1e-10, atol=1e-12), name


def test_layer_norm_formulas_against_autograd():
    torch.manual_seed(0)
    m, rows, cols = 3, 4, 11
    x, dy = torch.randn(m * rows, cols, dtype=torch.float64), torch.randn(m * rows, cols, dtype=torch.float64)
    for i in range(m):
        xs = x[i * rows:(i + 1) * rows].clone().requires_grad_(True)
        w, b = torch.randn(cols, dtype=torch.float64, requires_grad=True), torch.randn(cols, dtype=torch.float64, requires_grad=True)
        y = torch.nn.functional.layer_norm(xs, (cols,), w, b, 1e-5)
        y.backward(dy[i * rows:(i + 1) * rows])
        x64, mean, rstd, n, _, _ = ref.rows64(xs.detach(), w, b, 1e-5)
        n_err = 1e-6
        g = dy[i * rows:(i + 1) * rows] * w.detach()
        dx = rstd * (g - g.mean(1, keepdim=True) - n * (g * n).mean(1, keepdim=True))
        assert torch.allclose(dx, xs.grad, atol=n_err)
        assert torch.allclose((dy[i * rows:(i + 1) * rows] * n).sum(0), w.grad, atol=n_err)


def test_wait_limit_arguments(lib):
    for bad in (-1, (1 << 40) + 1):
        assert lib.cdgrab_operators_wait_limit(bad) == binding.ERR_INVALID
    assert lib.cdgrab_operators_wait_limit(1 << 40) == binding.OK and lib.cdgrab_operators_wait_limit(0) == binding.OK


def test_coefficients_that_leave_the_range_of_16_bits(lib):
    """X, A and B are held in fp16: where a singular value could outgrow that, the call is refused; before any use of a
    device, so that the others get as far as finding none here."""
    def call(co, steps):
        return lib.cdgrab_orthogonalise(2, 8, 16, 0, P, 128, 16, steps, (C.c_float * 3)(*co), 0.0, P, 128, 16, P, 1 << 40, None)
    for co, steps in (((2.0, 0.0, 0.0), 10), ((2.0, 0.0, 0.0), 64), ((1e5, 0.0, 0.0), 1), ((0.0, 300.0, 0.0), 2), ((4.0, 0.0, 1.0), 3),
                      ((0.0, 0.0, -250.0), 2), ((1.0, 1.0, 1.0), 8), ((3e38, -3e38, 3e38), 2)):
        assert call(co, steps) == binding.ERR_INVALID, (co, steps)
    if torch.cuda.is_available():
        return               # (the addresses are not real)
    for co, steps in (((3.4445, -4.7750, 2.0315), 64), ((1.5, -0.5, 0.0), 64), ((1.875, -1.25, 0.375), 64), ((2.0, -1.5, 0.5), 64),
                      ((3.0, -3.2, 1.2), 30), ((1.0, 0.0, 0.0), 64), ((0.0, 0.0, 0.0), 64), ((2.0, 0.0, 0.0), 8), ((0.0, 300.0, 0.0), 1), ((-1.0, 0.5, 0.0), 9)):
        assert call(co, steps) == binding.ERR_DEVICE, (co, steps)


def test_the_binding_loads_without_torch(lib):
    """torch provides buffers to the calls that take them; the module and the library need none of it."""
    code = ("import sys; sys.modules['torch'] = None\n"
            "from paper_2302_00845_b200 import binding\n"
            "assert binding.lib().cdgrab_strerror(-1) and binding.lib().cdgrab_layer_norm_workspace_bytes(4, 100, 64) >= 0\n")
    subprocess.run([sys.executable, "-c", code], check=True, cwd=os.path.dirname(os.path.dirname(os.path.abspath(__file__))), timeout=120)


def test_layer_norm_reference_against_autograd():
    """ref.layer_norm_backward itself, which the GPU tests compare with, and its forward pass."""
    torch.manual_seed(1)
    m, rows, cols = 3, 4, 11
    x, dy = torch.randn(m * rows, cols), torch.randn(m * rows, cols)
    w, b = torch.randn(cols), torch.randn(cols)
    for weight in (w, None):
        (y, _), (mean, _), (rstd, _) = ref.layer_norm_forward(x, weight, None if weight is None else b, 1e-5)
        (dx, _), (dw, _), (db, _) = ref.layer_norm_backward(dy, x, weight, mean, rstd, m, torch.float32)
        for i in range(m):
            own = slice(i * rows, (i + 1) * rows)
            xs = x[own].double().requires_grad_(True)
            ws = (torch.ones(cols) if weight is None else weight).double().requires_grad_(True)
            bs = (torch.zeros(cols) if weight is None else b).double().requires_grad_(True)
            out = torch.nn.functional.layer_norm(xs, (cols,), ws, bs, 1e-5)
            out.backward(dy[own].double())
            for got, want in ((y[own], out.detach()), (dx[own], xs.grad), (dw[i], ws.grad), (db[i], bs.grad)):
                assert torch.allclose(got, want, rtol=1e-11, atol=1e-12)


def test_attention_backward_refuses_too_many_tiles_before_anything_runs(lib):
    b, h, t, d = 65535, 4096, 129, 8          # two tiles for each of 2^28 - 4096 heads
    sh = shape(batch=b, len_q=t, len_kv=1, heads=h, kv_heads=h, head_dim=d, causal=0,
               **{n: (256 * h * d, h * d, d) for n in ("q", "k", "v", "o", "do", "dq", "dk", "dv")})
    assert lib.cdgrab_attention_workspace_bytes(C.byref(sh)) > 0
    assert lib.cdgrab_attention_backward(C.byref(sh), P, P, P, P, P, P, None, None, P, P, P, P, 1 << 60, None) == binding.ERR_INVALID
