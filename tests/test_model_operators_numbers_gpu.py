"""Numbers that are no Python integers, sizes past 32 bits, and the C calls beside those with one record."""
import ctypes as C

import numpy as np
import pytest
import torch

from paper_2302_00845_b200 import binding

pytestmark = pytest.mark.gpu


def gen(seed):
    return torch.Generator(device="cuda").manual_seed(seed)


def test_steps_of_numpy():
    """A step is a number of any integer type."""
    x = torch.randn(16, 40, generator=gen(1), device="cuda")
    for kind in (np.int64, np.int32, np.uint32, np.uint8):
        assert torch.equal(binding.dropout_forward(x, 0.3, kind(5), kind(6), kind(7)), binding.dropout_forward(x, 0.3, 5, 6, 7))
        assert torch.equal(binding.dropout_backward(x, 0.3, kind(5), kind(6), kind(7)), binding.dropout_backward(x, 0.3, 5, 6, 7))
    for bad in (np.int64(-1), np.int64(2 ** 32)):
        with pytest.raises(ValueError):
            binding.dropout_forward(x, 0.3, 5, 6, bad)
    for bad in (1.5, np.float32(2), "3", None):
        with pytest.raises(TypeError):
            binding.dropout_forward(x, 0.3, 5, 6, bad)


@pytest.mark.parametrize("rows,cols", [(140_000, 16_384), (58_500_000, 37), (1_700_000, 1377)])
def test_lookups_beyond_32_bits(rows, cols):
    """Outputs of more than 2^31 elements (bf16, some 4.5 GB): rows accessed wide, eight values across rows, one by one."""
    table = torch.randn(50, cols, generator=gen(cols), device="cuda").bfloat16()
    tokens = torch.randint(0, 50, (rows,), generator=gen(rows), device="cuda").int()
    y = torch.full((rows + 1, cols), 7.0, dtype=torch.bfloat16, device="cuda")
    binding.embedding_forward(tokens, table, out=y[:rows])
    for r in range(0, rows, 1 << 20):
        n = min(1 << 20, rows - r)
        step = max(1, (1 << 28) // cols)
        for q in range(r, r + n, step):
            part = slice(q, min(q + step, r + n))
            assert torch.equal(y[part], table[tokens[part].long()])
    assert (y[rows] == 7).all()
    assert binding.operators_status() == binding.OK


def test_calls_with_one_record_and_without():
    """Every call through the C interface gives the bits that the binding gives."""
    L = binding.lib()
    r = lambda *s: torch.randn(*s, generator=gen(sum(s)), device="cuda")  # noqa: E731
    stream = C.c_void_p(torch.cuda.current_stream().cuda_stream)
    ptr = lambda t: C.c_void_p(t.data_ptr())  # noqa: E731
    m, length, vocab, cols = 3, 70, 40, 33
    tokens = torch.randint(0, vocab, (m, length), generator=gen(2), device="cuda")
    table, dy = r(vocab, cols), r(m * length, cols).bfloat16()
    want, got = binding.embedding_forward(tokens, table, 1.5, 3), torch.empty(m * length, cols, device="cuda")
    assert L.cdgrab_embedding_forward(m, length, cols, vocab, 64, ptr(tokens), length, 3, 1.5, binding.F32, ptr(table), cols, binding.F32, ptr(got), cols,
                                      stream) == binding.OK
    assert torch.equal(got, want)
    want, got = binding.embedding_backward(dy, tokens, torch.empty(m, vocab, cols, device="cuda"), 1.5, 3), torch.empty(m, vocab, cols, device="cuda")
    size = L.cdgrab_embedding_workspace_bytes(m, length, cols, vocab)
    work = torch.empty(size, dtype=torch.uint8, device="cuda")
    assert L.cdgrab_embedding_backward(m, 1, length, cols, vocab, 64, ptr(tokens), length, 3, 1.5, binding.BF16, ptr(dy), cols, binding.F32, ptr(got), vocab * cols,
                                       cols, 0, ptr(work), size, stream) == binding.OK
    assert torch.equal(got, want)
    x, res, seed = r(50, 24).bfloat16(), r(50, 24), 2 ** 64 - 3
    want, got = binding.dropout_forward(x, 0.3, seed, 2 ** 32 - 1, 9, residual=res), torch.empty(50, 24, device="cuda")
    assert L.cdgrab_dropout_forward(50, 24, binding.BF16, ptr(x), 24, binding.F32, ptr(res), 24, ptr(got), 24, 0.3, seed, 2 ** 32 - 1, 9, None, stream) == binding.OK
    assert torch.equal(got, want)
    want, got = binding.dropout_backward(x, 0.3, seed, 2 ** 32 - 1, 9), torch.empty_like(x)
    assert L.cdgrab_dropout_backward(50, 24, binding.BF16, ptr(x), 24, binding.BF16, ptr(got), 24, 0.3, seed, 2 ** 32 - 1, 9, None, stream) == binding.OK
    assert torch.equal(got, want)
    b, t, h, hk, d = 4, 30, 3, 2, 64
    q, k, dq, dk = (r(b, t, n, d).bfloat16() for n in (h, hk, h, hk))
    qw, kw = r(d), r(d)
    pos, lens = torch.randint(0, 10 ** 6, (b, t), generator=gen(3), device="cuda"), torch.tensor([30, 4, 0, 29], dtype=torch.int32, device="cuda")
    sh = binding.RotaryShape(b, t, h, hk, d, 32, 1, binding.BF16, 500.0, 1e-5, 0)
    for n, heads in (("q", h), ("k", hk)):
        for name in (n + "_stride", n + "_out_stride", "d" + n + "_stride"):
            getattr(sh, name)[:] = (t * heads * d, heads * d, d)
    opts = dict(positions=pos, base=500.0, rotary_dim=32, interleaved=True, eps=1e-5, lens=lens)
    want, got = binding.rotary_forward(q, k, qw, kw, **opts), (torch.empty_like(q), torch.empty_like(k))
    assert L.cdgrab_rotary_forward(C.byref(sh), ptr(q), ptr(k), ptr(qw), ptr(kw), ptr(pos), 64, t, ptr(lens), ptr(got[0]), ptr(got[1]), stream) == binding.OK
    assert all(torch.equal(a, c) for a, c in zip(got, want))
    dw, dw2 = torch.empty(2, 2, d, device="cuda"), torch.empty(2, 2, d, device="cuda")
    want = binding.rotary_backward(dq, dk, q, k, qw, kw, dq_weight=dw[0], dk_weight=dw[1], **opts)
    size = L.cdgrab_rotary_workspace_bytes(C.byref(sh), 2)
    work = torch.empty(max(size, 1), dtype=torch.uint8, device="cuda")
    assert L.cdgrab_rotary_backward(C.byref(sh), 2, ptr(dq), ptr(dk), ptr(q), ptr(k), ptr(qw), ptr(kw), ptr(pos), 64, t, ptr(lens), ptr(got[0]), ptr(got[1]), binding.F32,
                                    ptr(dw2[0]), ptr(dw2[1]), d, ptr(work), size, stream) == binding.OK
    assert all(torch.equal(a, c) for a, c in zip(got, want)) and torch.equal(dw, dw2)
