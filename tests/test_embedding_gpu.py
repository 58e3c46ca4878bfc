"""Embedding lookup and its per-worker gradient against the formulas in 64 bits."""
import pytest
import torch

import model_operators_ref as ref
from operators_ref import assert_within
from paper_2302_00845_b200 import binding

pytestmark = pytest.mark.gpu
TYPES = {"f32": torch.float32, "bf16": torch.bfloat16}


def gen(seed):
    return torch.Generator(device="cuda").manual_seed(seed)


def draw(groups, length, vocab, cols, dtype="f32", bits=torch.int64, seed=0, skew=2.0):
    g = gen(seed * 7919 + groups + length + vocab + cols)
    # the low tokens often, the high ones rarely
    t = (torch.rand(groups, length, generator=g, device="cuda") ** skew * vocab).long().clamp(max=vocab - 1).to(bits)
    table = torch.randn(vocab, cols, generator=g, device="cuda").to(TYPES[dtype])
    dy = torch.randn(groups * length, cols, generator=g, device="cuda").to(TYPES[dtype])
    return t, table, dy


def check(t, table, dy, m, grads="f32", scale=1.0, padding=None, accumulate=False, out_dtype=None, status=binding.OK):
    y = binding.embedding_forward(t, table, scale, padding, dtype=out_dtype)
    want, bound = ref.embedding_forward(t, table, scale, padding, out_dtype or table.dtype)
    assert_within(y, want, bound, "y")
    assert binding.operators_status() == status
    vocab, cols = table.shape
    buf = torch.full((m, vocab, cols), 3.0 if accumulate else float("nan"), dtype=TYPES[grads], device="cuda")
    old = buf.clone() if accumulate else None
    got = binding.embedding_backward(dy, t, buf, scale, padding, accumulate)
    assert got is buf
    want, bound = ref.embedding_backward(dy, t, m, vocab, scale, padding, TYPES[grads], old)
    assert_within(buf, want, bound, "dtable")
    assert binding.operators_status() == status
    again = torch.full_like(buf, 3.0)
    assert torch.equal(binding.embedding_backward(dy, t, again, scale, padding, accumulate), buf)      # the same bits
    binding.operators_status()
    return y, buf


# around the vector widths and the columns that a warp takes
@pytest.mark.parametrize("dtype", ["f32", "bf16"])
@pytest.mark.parametrize("cols", [1, 2, 3, 7, 8, 31, 33, 64, 100, 255, 256, 257, 264, 512, 650, 768, 1025, 2048, 5000])
def test_columns(cols, dtype):
    check(*draw(2, 37, 19, cols, dtype), 2, "f32")


@pytest.mark.parametrize("vocab", [2 ** 24 - 1, 2 ** 24, 2 ** 26])
def test_large_vocabularies(vocab):
    """Three and four digits of a sort."""
    check(*draw(1, 5000, vocab, 1, skew=1.0), 1)


# vocabularies around the digits of a sort and single rows; lengths from one token to more than a block takes at once
@pytest.mark.parametrize("vocab", [1, 2, 31, 255, 256, 257, 511, 4095, 65535, 65536, 70001])
@pytest.mark.parametrize("bits", [torch.int32, torch.int64])
def test_vocabularies(vocab, bits):
    check(*draw(2, 300, vocab, 24, bits=bits), 2)


@pytest.mark.parametrize("m,length", [(1, 1), (1, 2), (3, 1), (1, 31), (1, 32), (1, 33), (2, 63), (2, 64), (2, 65), (5, 127), (1, 1023), (1, 1024),
                                      (2, 1025), (1, 2047), (1, 4097), (3, 8191), (1, 8193), (1, 16385), (2, 33000), (1, 70000), (1, 140001),
                                      (64, 17), (300, 3), (2000, 1)])
def test_workers_and_lengths(m, length):
    check(*draw(m, length, 300, 40, "bf16"), m, "bf16")


@pytest.mark.parametrize("length", [32, 64, 65, 96, 97, 128, 160, 1000, 5000, 40000])
@pytest.mark.parametrize("accumulate", [False, True])
def test_one_token_throughout(length, accumulate):
    """A run as long as the sequence, from the first position and from the middle of a window on."""
    t, table, dy = draw(1, length, 50, 300)
    t.fill_(7)
    check(t, table, dy, 1, accumulate=accumulate)
    for lead in (1, 31, 32, 33):
        if lead < length:
            t[:, :lead] = torch.arange(lead, device="cuda") % 7
            check(t, table, dy, 1, accumulate=accumulate)


def test_runs_of_every_length_from_every_start():
    """Runs of lengths around one and two windows of 32, each from 32 consecutive starts."""
    for run in (1, 2, 30, 31, 32, 33, 34, 62, 63, 64, 65, 66, 95, 96, 97, 129):
        rows = []
        for start in range(32):
            rows.append(torch.cat((torch.arange(start), torch.full((run,), 40), torch.arange(41, 41 + 200 - run - start))))
        t = torch.stack(rows).cuda()
        _, table, dy = draw(32, 200, 250, 12, seed=run)
        check(t, table, dy, 32)


@pytest.mark.parametrize("dtype,out", [("f32", "bf16"), ("bf16", "f32"), ("bf16", "bf16"), ("f32", "f32")])
@pytest.mark.parametrize("scale", [1.0, 27.71281, -0.37, 0.0])
def test_types_and_scales(dtype, out, scale):
    check(*draw(3, 50, 90, 72, dtype), 3, out, scale, out_dtype=TYPES[out])
    check(*draw(3, 50, 90, 72, dtype), 3, out, scale, out_dtype=TYPES[out], accumulate=True)


@pytest.mark.parametrize("padding", [-1, 0, 5, 89, -100, 10 ** 12])
def test_padding(padding):
    t, table, dy = draw(4, 60, 90, 40)
    if abs(padding) < 1000:
        t[1:, 40:] = padding
        t[3] = padding                 # a worker with no tokens at all
    dy[(t == padding).reshape(-1)] = float("nan")          # not used
    y, buf = check(t, table, dy, 4, padding=padding)
    assert (y[(t == padding).reshape(-1)] == 0).all()
    if abs(padding) < 1000:
        assert (buf[3] == 0).all()
    check(t, table, dy, 4, padding=padding, accumulate=True)


def test_tokens_outside_the_vocabulary_are_reported():
    for bad in (-1, 90, 91, 2 ** 31, 2 ** 32 + 3, -2 ** 63, 2 ** 63 - 1):
        t, table, dy = draw(2, 60, 90, 40)
        t[1, 17] = bad
        status = binding.OK if bad == -2 ** 63 else binding.ERR_INVALID           # (the number for no padding)
        check(t, table, dy, 2, status=status)
    t, table, dy = draw(2, 60, 90, 40, bits=torch.int32)
    t[0, 0] = -2 ** 31
    check(t, table, dy, 2, status=binding.ERR_INVALID)
    check(t, table, dy, 2, padding=-2 ** 31)


def test_several_rows_to_a_worker_and_strided_tokens():
    long, table, dy = draw(6, 41, 77, 16, "bf16")
    t = long[:, :-1]                       # a slice of longer sequences
    dy = dy[:240]
    a = check(t, table, dy, 3)
    b = check(t.contiguous().view(3, 80), table, dy, 3)
    assert all(torch.equal(x, y) for x, y in zip(a, b))
    y = binding.embedding_forward(t[0], table)             # one dimension
    assert torch.equal(y, a[0][:40])
    one = torch.empty(77, 16, device="cuda")
    assert binding.embedding_backward(dy, t, one) is one
    flat = torch.empty(1, 77, 16, device="cuda")
    assert torch.equal(binding.embedding_backward(dy, t.reshape(-1), flat)[0], one)


@pytest.mark.parametrize("m,rows", [(1, 1), (1, 200), (4, 50), (200, 1)])
def test_single_tokens(m, rows):
    """One token of each sequence, the newest of longer rows: rows of one token, far apart."""
    long, table, dy = draw(m * rows, 9, 60, 72, "bf16")
    dy = dy[:m * rows]
    a = check(long[:, -1:], table, dy, m)
    b = check(long[:, -1].contiguous().view(m, rows), table, dy, m)
    assert all(torch.equal(x, y) for x, y in zip(a, b))


def test_strides_and_what_lies_between():
    m, vocab, cols = 3, 50, 72
    t, table, dy = draw(m, 40, vocab, cols, "bf16")
    wide_t = torch.zeros(vocab, 200, dtype=torch.bfloat16, device="cuda")
    wide_d = torch.zeros(m * 40, 201, dtype=torch.bfloat16, device="cuda")
    for lo in (0, 8, 1, 3):               # from 16-byte aligned down to odd starts
        tab, d = wide_t[:, lo:lo + cols], wide_d[:, lo:lo + cols]
        tab.copy_(table)
        d.copy_(dy)
        out = torch.full((m * 40, cols + 5), 7.0, dtype=torch.bfloat16, device="cuda")
        want, bound = ref.embedding_forward(t, tab, 1.5, None, torch.bfloat16)
        assert_within(binding.embedding_forward(t, tab, 1.5, out=out[:, 2:2 + cols]), want, bound)
        assert (out[:, :2] == 7).all() and (out[:, 2 + cols:] == 7).all()
        for dt in (torch.float32, torch.bfloat16):
            # the table's part of the workers' rows of a gather buffer
            buf = torch.full((2, m, 9000), 5.0, dtype=dt, device="cuda")
            part = buf[1, :, 100 + lo:100 + lo + vocab * cols].view(m, vocab, cols)
            want, bound = ref.embedding_backward(d, t, m, vocab, 1.5, None, dt)
            assert_within(binding.embedding_backward(d, t, part, 1.5), want, bound)
            assert (buf[0] == 5).all() and (buf[1, :, :100 + lo] == 5).all() and (buf[1, :, 100 + lo + vocab * cols:] == 5).all()
            # rows with room between them
            buf = torch.full((m, vocab, cols + 9), 5.0, dtype=dt, device="cuda")
            assert_within(binding.embedding_backward(d, t, buf[:, :, lo:lo + cols], 1.5), want, bound)
            assert (buf[:, :, :lo] == 5).all() and (buf[:, :, lo + cols:] == 5).all()


def test_accumulate_leaves_other_rows_as_they_are():
    t, table, dy = draw(2, 30, 64, 40)
    t.clamp_(max=20)
    t[:, :3] = 63
    buf = torch.full((2, 64, 40), float("nan"), device="cuda")
    buf[:, :21] = 1.0
    buf[:, 63] = 1.0
    binding.embedding_backward(dy, t, buf, accumulate=True)
    assert torch.isnan(buf[:, 21:63]).all() and torch.isfinite(buf[:, 63]).all()
    seen = torch.zeros(2, 64, dtype=torch.bool, device="cuda").scatter_(1, t, True)
    assert (buf[:, :21][~seen[:, :21]] == 1).all()


def test_infinities_stay_in_their_rows():
    t, table, dy = draw(2, 50, 30, 16)
    table[4], dy[7] = float("inf"), float("nan")
    t[:, 7] = 29
    y = binding.embedding_forward(t, table)
    assert torch.equal(torch.isinf(y).all(1), t.reshape(-1) == 4)
    buf = binding.embedding_backward(dy, t, torch.empty(2, 30, 16, device="cuda"))
    assert torch.isnan(buf[0, 29]).all() and torch.isfinite(buf[0, :29]).all() and torch.isfinite(buf[1]).all()


def test_nothing_to_do():
    table = torch.ones(10, 8, device="cuda")
    for shape in ((0,), (0, 5), (3, 0)):
        t = torch.empty(shape, dtype=torch.int64, device="cuda")
        assert binding.embedding_forward(t, table).shape == (0, 8)
    t, dy = torch.empty(3, 0, dtype=torch.int64, device="cuda"), torch.empty(0, 8, device="cuda")
    buf = torch.full((3, 10, 8), 5.0, device="cuda")
    assert (binding.embedding_backward(dy, t, buf, accumulate=True) == 5).all()
    assert (binding.embedding_backward(dy, t, buf) == 0).all()


def test_a_table_gradient_beyond_32_bits():
    """Three workers' tables that end past 2^31 elements (bf16, 4.8 GB)."""
    m, vocab, cols = 3, 50000, 16000
    t, _, dy = draw(m, 200, vocab, 64, "bf16")
    t[:, -1] = vocab - 1
    dy = torch.randn(m * 200, cols, generator=gen(1), device="cuda").bfloat16()
    buf = torch.full((m, vocab, cols), 9.0, dtype=torch.bfloat16, device="cuda")
    binding.embedding_backward(dy, t, buf)
    for i in range(m):
        want = torch.zeros(vocab, 1, device="cuda").index_add_(0, t[i], dy[i * 200:(i + 1) * 200].float().abs().sum(1, keepdim=True))[:, 0]
        total = torch.cat([buf[i, v:v + 5000].float().abs().sum(1) for v in range(0, vocab, 5000)])
        assert torch.equal(total > 0, want > 0)
        last = torch.zeros(cols, device="cuda").double()
        for j in (t[i] == vocab - 1).nonzero()[:, 0]:
            last += dy[i * 200 + j].double()
        assert (buf[i, vocab - 1].double() - last).abs().max() <= 2.0 ** -7 * last.abs().max()


def test_refusals():
    t, table, dy = draw(2, 30, 64, 40)
    buf = torch.empty(2, 64, 40, device="cuda")
    for bad in (lambda: binding.embedding_forward(t.float(), table), lambda: binding.embedding_forward(t, table.half()),
                lambda: binding.embedding_forward(t, table[0]), lambda: binding.embedding_forward(t[None], table),
                lambda: binding.embedding_forward(t.t(), table), lambda: binding.embedding_forward(t, table.t()),
                lambda: binding.embedding_forward(t, table, out=torch.empty(5, 40, device="cuda")),
                lambda: binding.embedding_forward(t.cpu(), table), lambda: binding.embedding_forward(t, table, dtype=torch.float16),
                lambda: binding.embedding_forward(t, table, dtype=torch.bfloat16, out=torch.empty(60, 40, device="cuda")),
                lambda: binding.embedding_backward(dy, t, buf.half()), lambda: binding.embedding_backward(dy[:-1], t, buf),
                lambda: binding.embedding_backward(dy, t, buf[:, :, ::2]), lambda: binding.embedding_backward(dy, t, torch.empty(3, 64, 40, device="cuda")),
                lambda: binding.embedding_backward(dy, t, buf.view(-1))):
        with pytest.raises(ValueError):
            bad()
    for bad in (lambda: binding.embedding_forward(t, table, scale=float("inf")), lambda: binding.embedding_backward(dy, t, buf, scale=float("nan")),
                lambda: binding.embedding_backward(dy, t, buf[:1].expand(2, 64, 40)),
                lambda: binding.embedding_backward(dy, t, buf[:, :1].expand(2, 64, 40))):
        with pytest.raises(binding.CdgrabError):
            bad()
