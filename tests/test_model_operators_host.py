"""Argument checks of embedding, dropout and the rotation, which come before any use of a device, and the 64-bit forms that
the GPU tests compare with: against automatic differentiation and against the oracle's generator."""
import ctypes as C
import math

import numpy as np
import pytest
import torch

import model_operators_ref as ref
from paper_2302_00845_b200 import binding, build

P = 1 << 20       # a non-null, aligned address that is never read


@pytest.fixture(scope="module")
def lib():
    build.build()
    return binding.lib()


def test_embedding_arguments(lib):
    def fwd(groups=2, length=4, cols=8, vocab=10, bits=64, tok=P, ts=4, pad=-1, scale=1.0, dtype=0, table=P, tabs=8, out=0, y=P, ys=8):
        return lib.cdgrab_embedding_forward(groups, length, cols, vocab, bits, tok, ts, pad, scale, dtype, table, tabs, out, y, ys, None)
    for bad in (dict(groups=-1), dict(length=-1), dict(groups=1 << 16, length=1 << 15), dict(groups=1 << 40, length=1 << 40), dict(cols=0), dict(vocab=0),
                dict(bits=16), dict(tok=None), dict(ts=3), dict(scale=math.inf), dict(scale=math.nan), dict(dtype=2), dict(out=-1), dict(table=None),
                dict(tabs=7), dict(y=None), dict(ys=7), dict(tok=P + 4), dict(bits=32, tok=P + 2), dict(table=P + 2), dict(out=1, y=P + 1)):
        assert fwd(**bad) == binding.ERR_INVALID, bad
    assert fwd(groups=0) == binding.OK and fwd(length=0) == binding.OK
    assert fwd(cols=(1 << 24) + 1, tabs=1 << 25, ys=1 << 25) == binding.ERR_INVALID
    assert lib.cdgrab_embedding_workspace_bytes(1, 1, (1 << 24) + 1, 1) == -1

    def bwd(m=2, groups=1, length=4, cols=8, vocab=10, bits=64, tok=P, ts=4, pad=-1, scale=1.0, dtype=0, dy=P, dys=8, gd=0, dt=P, ws=80, rs=8,
            acc=0, work=P, size=1 << 40):
        return lib.cdgrab_embedding_backward(m, groups, length, cols, vocab, bits, tok, ts, pad, scale, dtype, dy, dys, gd, dt, ws, rs, acc, work, size, None)
    for bad in (dict(m=0), dict(m=65536), dict(groups=-1), dict(length=-1), dict(m=1 << 15, length=1 << 16), dict(cols=0), dict(vocab=0), dict(bits=8), dict(tok=None),
                dict(ts=3), dict(scale=math.inf), dict(dtype=3), dict(dy=None), dict(dys=7), dict(gd=2), dict(dt=None), dict(ws=79), dict(rs=7), dict(acc=2),
                dict(work=None), dict(size=0), dict(work=P + 8), dict(dt=P + 2), dict(dy=P + 1), dict(tok=P + 4)):
        assert bwd(**bad) == binding.ERR_INVALID, bad
    assert bwd(length=0, acc=1) == binding.OK
    for bad in ((0, 1, 1, 1), (1, -1, 1, 1), (1, 1, 0, 1), (1, 1, 1, 0), (65536, 1, 1, 1), (2, 1 << 30, 1, 1)):
        assert lib.cdgrab_embedding_workspace_bytes(*bad) == -1, bad
    assert lib.cdgrab_embedding_workspace_bytes(64, 1024, 768, 50257) > 0


def test_dropout_arguments(lib):
    def fwd(rows=4, cols=8, dtype=0, x=P, xs=8, out=0, res=P, rs=8, y=P, ys=8, p=0.1, at=None):
        return lib.cdgrab_dropout_forward(rows, cols, dtype, x, xs, out, res, rs, y, ys, p, 1, 2, 3, at, None)

    def bwd(rows=4, cols=8, dtype=0, x=P, xs=8, out=0, y=P, ys=8, p=0.1, at=None):
        return lib.cdgrab_dropout_backward(rows, cols, dtype, x, xs, out, y, ys, p, 1, 2, 3, at, None)
    both = (dict(rows=-1), dict(cols=-1), dict(rows=1 << 31), dict(cols=1 << 31), dict(dtype=2), dict(out=2), dict(x=None), dict(y=None), dict(xs=7), dict(ys=7),
            dict(p=-1e-9), dict(p=1.0000001), dict(p=math.nan), dict(x=P + 2), dict(out=1, y=P + 1), dict(at=P + 4))
    for bad in both:
        assert fwd(**bad) == binding.ERR_INVALID, bad
        assert bwd(**bad) == binding.ERR_INVALID, bad
    assert fwd(rows=1 << 21, cols=1 << 21, xs=1 << 21, ys=1 << 21, res=None) == binding.ERR_INVALID
    assert fwd(rs=7) == binding.ERR_INVALID and fwd(res=P + 2) == binding.ERR_INVALID
    for call in (fwd, bwd):
        assert call(rows=0) == binding.OK and call(cols=0) == binding.OK


def rotary_shape(**kw):
    s = dict(batch=2, len=6, heads=4, kv_heads=2, head_dim=64, rotary_dim=64, interleaved=0, dtype=1, base=10000.0, eps=1e-6, reserved=0)
    strides = {n: kw.pop(n, None) for n in ("q", "k", "q_out", "k_out", "dq", "dk")}
    s.update(kw)
    sh = binding.RotaryShape(*s.values())
    for n, v in strides.items():
        h = s["heads"] if "q" in n else s["kv_heads"]
        getattr(sh, n + "_stride")[:] = v or (6 * h * 64, h * 64, 64)
    return sh


def test_rotary_arguments(lib):
    def fwd(sh, q=P, k=P, qw=P, kw=P, pos=None, bits=64, ps=0, lens=None, qo=P, ko=P):
        return lib.cdgrab_rotary_forward(C.byref(sh) if sh else None, q, k, qw, kw, pos, bits, ps, lens, qo, ko, None)

    def bwd(sh, m=2, dq=P, dk=P, q=P, k=P, qw=P, kw=P, pos=None, bits=64, ps=0, lens=None, qo=P, ko=P, gd=0, dqw=P, dkw=P, ws=64, work=P, size=1 << 40):
        return lib.cdgrab_rotary_backward(C.byref(sh) if sh else None, m, dq, dk, q, k, qw, kw, pos, bits, ps, lens, qo, ko, gd, dqw, dkw, ws, work, size, None)
    assert fwd(None) == binding.ERR_INVALID and bwd(None) == binding.ERR_INVALID
    for bad in (dict(batch=-1), dict(len=-1), dict(heads=-1), dict(kv_heads=-1), dict(heads=65536), dict(head_dim=0), dict(head_dim=12), dict(head_dim=264),
                dict(rotary_dim=-8), dict(rotary_dim=4), dict(rotary_dim=72), dict(interleaved=2), dict(dtype=2), dict(base=0.0), dict(base=-1.0), dict(base=math.inf),
                dict(base=math.nan), dict(eps=-1e-9), dict(eps=math.nan), dict(eps=math.inf), dict(reserved=1), dict(batch=1 << 16, len=1 << 15),
                dict(q=(1536, 256, 60)), dict(k=(-8, 128, 64)), dict(q_out=(1536, 0, 64)), dict(k_out=(768, 128, 0)),
                dict(q_out=(0, 256, 64)), dict(q_out=(1528, 256, 64)), dict(k_out=(768, 120, 64)), dict(k_out=(64, 128, 128)), dict(k=(1 << 41, 128, 64))):
        assert fwd(rotary_shape(**bad)) == binding.ERR_INVALID, bad
        assert bwd(rotary_shape(**bad)) == binding.ERR_INVALID, bad
        if not {"q", "k", "q_out", "k_out"} & set(bad):
            assert lib.cdgrab_rotary_workspace_bytes(C.byref(rotary_shape(**bad)), 1) == -1, bad
    for bad in (dict(q=None), dict(k=None), dict(qo=None), dict(ko=None), dict(q=P + 8), dict(k=P + 2), dict(qo=P + 8), dict(ko=P + 4), dict(qw=P + 2), dict(kw=P + 1),
                dict(pos=P, bits=16), dict(pos=P, ps=-1), dict(pos=P + 4), dict(pos=P + 2, bits=32), dict(lens=P + 2)):
        assert fwd(rotary_shape(), **bad) == binding.ERR_INVALID, bad
        assert bwd(rotary_shape(), **bad) == binding.ERR_INVALID, bad
    for bad in (dict(m=0), dict(m=3), dict(m=65536), dict(dq=None), dict(dk=None), dict(dq=P + 8), dict(dk=P + 2), dict(gd=2), dict(dqw=P + 2), dict(dkw=P + 1),
                dict(ws=63)):
        assert bwd(rotary_shape(), **bad) == binding.ERR_INVALID, bad
    # long sequences need a workspace, short ones none
    long = rotary_shape(len=100_000)
    need = lib.cdgrab_rotary_workspace_bytes(C.byref(long), 2)
    assert need > 0 and lib.cdgrab_rotary_workspace_bytes(C.byref(rotary_shape()), 2) == 0
    for bad in (dict(work=None), dict(size=need - 1), dict(work=P + 8)):
        assert bwd(long, **bad) == binding.ERR_INVALID, bad
    for bad in (dict(dq=(1536, 256, 4)), dict(dk=(768, 0, 64))):
        assert bwd(rotary_shape(**bad)) == binding.ERR_INVALID, bad
    assert fwd(rotary_shape(batch=0)) == binding.OK and fwd(rotary_shape(len=0)) == binding.OK
    assert fwd(rotary_shape(heads=0, kv_heads=0)) == binding.OK


def test_no_cpu_fallback(lib):
    if torch.cuda.is_available():
        pytest.skip("a CUDA device is present")
    assert lib.cdgrab_embedding_forward(2, 4, 8, 10, 64, P, 4, -1, 1.0, 0, P, 8, 0, P, 8, None) == binding.ERR_DEVICE
    assert lib.cdgrab_dropout_forward(4, 8, 0, P, 8, 0, None, 0, P, 8, 0.5, 1, 2, 3, None, None) == binding.ERR_DEVICE
    assert lib.cdgrab_rotary_forward(C.byref(rotary_shape()), P, P, None, None, None, 0, 0, None, P, P, None) == binding.ERR_DEVICE


def test_the_masks_generator_against_the_oracle():
    """The generator that the GPU tests compare with gives the oracle's words (pinned by the published vectors)."""
    import oracle
    for block, call, step, seed in ((0, 0, 0, 0), (7, 1, 2, 3), (2 ** 40 + 5, 2 ** 32 - 1, 2 ** 31, 2 ** 64 - 1), (123, 9, 8, 0xDEADBEEF12345678)):
        want = oracle.philox4x32_10((block & 0xFFFFFFFF, block >> 32, call, step), (seed & 0xFFFFFFFF, seed >> 32))
        assert np.array_equal(ref.philox([block], call, step, seed)[0], want)
    bits = ref.philox([3], 1, 2, 9)[0]
    halves = [int(w) >> s & 0xFFFF for w in bits for s in (0, 16)]
    for p in (0.1, 0.5, 0.9):
        assert list(ref.keep(np.arange(24, 32), p, 9, 1, 2)) == [h >= int(65536 * p + 0.5) for h in halves]


def test_embedding_forms_against_autograd():
    torch.manual_seed(0)
    t = torch.tensor([[1, 4, 1, 0], [4, -1, 4, 4]])
    table = torch.randn(6, 5, dtype=torch.float64, requires_grad=True)
    dy = torch.randn(8, 5, dtype=torch.float64)
    for i in range(2):
        table.grad = None
        use = t[i] >= 0
        y = torch.where(use[:, None], 1.5 * table[t[i].clamp(min=0)], 0.0)
        y.backward(dy[4 * i:4 * i + 4])
        assert torch.allclose(ref.embedding_forward(t[i], table.detach(), 1.5, -1, torch.float32)[0], y.detach(), rtol=1e-12)
        assert torch.allclose(ref.embedding_backward(dy, t, 2, 6, 1.5, -1, torch.float32)[0][i], table.grad, rtol=1e-12)


@pytest.mark.parametrize("interleaved", [False, True])
@pytest.mark.parametrize("rotary_dim", [0, 8, 16])
def test_rotary_forms_against_autograd(rotary_dim, interleaved):
    torch.manual_seed(0)
    b, t, h, d = 2, 5, 3, 16
    x, w = torch.randn(b, t, h, d, dtype=torch.float64), torch.randn(d, dtype=torch.float64)
    dy, lens = torch.randn(b, t, h, d, dtype=torch.float64), torch.tensor([5, 3])
    pos = torch.tensor([3, 0, 7, 100, 4])
    ref.U16[torch.float64] = 0.0
    eps = float(np.float32(1e-3))
    for i in range(b):
        xs, ws = x[i].clone().requires_grad_(True), w.clone().requires_grad_(True)
        n = xs / torch.sqrt(xs.square().mean(-1, keepdim=True) + eps) * ws
        out = []
        for s in range(t):
            v = n[s]
            for p in range(rotary_dim // 2):
                angle = float(pos[s]) * 100.0 ** (-2 * p / rotary_dim)
                one, two = (2 * p, 2 * p + 1) if interleaved else (p, p + rotary_dim // 2)
                turn = torch.zeros(d, d, dtype=torch.float64)
                turn[one, one] = turn[two, two] = math.cos(angle) - 1
                turn[one, two], turn[two, one] = -math.sin(angle), math.sin(angle)
                v = v + n[s] @ turn.T
            out.append(v * (s < int(lens[i])))
        y = torch.stack(out)
        y.backward(dy[i])
        args = (pos, 100.0, rotary_dim, interleaved, 1e-3, lens)
        assert torch.allclose(ref.rotary(x, w, *args)[0][i], y.detach(), rtol=1e-9, atol=1e-12)
        (dx, _), (dw, _) = ref.rotary(x, w, *args, dy=dy, m=b)
        assert torch.allclose(dx[i], xs.grad, rtol=1e-9, atol=1e-12) and torch.allclose(dw[i], ws.grad, rtol=1e-9, atol=1e-12)
    del ref.U16[torch.float64]


def test_records(lib):
    """cdgrab_call takes the same arguments in the same order: each kind of call gets as far as the call itself, and a number that
    its parameter does not hold is refused."""
    import struct
    if torch.cuda.is_available():
        pytest.skip("the addresses are not real")
    shape = bytes(rotary_shape())
    good = {1: ("8qd7q", [2, 4, 8, 10, 64, P, 4, -1, 1.0, 0, P, 8, 0, P, 8, 0]),
            2: ("9qd11q", [2, 1, 4, 8, 10, 64, P, 4, -1, 1.0, 0, P, 8, 0, P, 80, 8, 0, P, 1 << 40, 0]),
            3: ("10qdQ4q", [4, 8, 0, P, 8, 0, P, 8, P, 8, 0.1, 2 ** 64 - 1, 2 ** 32 - 1, 2 ** 32 - 1, 0, 0]),
            4: ("8qdQ4q", [4, 8, 0, P, 8, 0, P, 8, 0.1, 1, 2, 3, 0, 0]),
            5: ("11q", [P, P, P, P, 0, 0, 0, 0, P, P, 0]),
            6: ("20q", [2, P, P, P, P, P, P, 0, 0, 0, 0, P, P, 0, P, P, 64, 0, 0, 0])}
    call = lambda n, fmt, v: lib.cdgrab_call(n, (shape if n > 4 else b"") + struct.pack(fmt, *v))  # noqa: E731
    for n, (fmt, v) in good.items():
        assert call(n, fmt, v) == binding.ERR_DEVICE, n
    bad = [(1, 2, 2 ** 32 + 8), (1, 3, -2 ** 32 + 10), (1, 4, 2 ** 32 + 64), (1, 5, 0), (1, 6, 3), (1, 8, math.inf), (1, 8, 1e300), (1, 9, 2 ** 32), (1, 11, 7),
           (1, 12, 2), (1, 13, 0), (1, 14, 7), (2, 0, 2 ** 32 + 2), (2, 2, -1), (2, 7, 3), (2, 12, 7), (2, 13, 2 ** 33), (2, 15, 79), (2, 16, 7), (2, 17, 2), (2, 18, 0),
           (2, 19, 15), (3, 0, -1), (3, 4, 7), (3, 5, 2 ** 32), (3, 7, 7), (3, 9, 7), (3, 10, 1.5), (3, 12, 2 ** 32), (3, 13, -1), (3, 14, P + 4), (4, 4, 7), (4, 7, 7),
           (4, 8, -0.5), (4, 10, 2 ** 32), (4, 12, P + 4), (5, 0, P + 8), (5, 1, 0), (5, 2, P + 2), (5, 7, P + 2), (5, 9, 0), (6, 0, 2 ** 32 + 2), (6, 1, 0), (6, 4, P + 4),
           (6, 11, 0), (6, 13, 2 ** 32), (6, 13, 2), (6, 16, 63)]
    for n, at, value in bad:
        fmt, v = good[n]
        assert call(n, fmt, v[:at] + [value] + v[at + 1:]) == binding.ERR_INVALID, (n, at, value)
    assert lib.cdgrab_call(1, None) == binding.ERR_INVALID
    for n in (0, 7, -1):
        assert lib.cdgrab_call(n, bytes(400)) == binding.ERR_INVALID
