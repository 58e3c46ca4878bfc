"""Dropout against the formula in 64 bits, with the mask from the generator's published definition."""
import numpy as np
import pytest
import torch

import model_operators_ref as ref
from operators_ref import assert_within
from paper_2302_00845_b200 import binding

pytestmark = pytest.mark.gpu
TYPES = {"f32": torch.float32, "bf16": torch.bfloat16}
SEED = 0xDEADBEEF12345678


def draw(rows, cols, dtype, out, seed=0):
    g = torch.Generator(device="cuda").manual_seed(seed * 31 + rows * 7 + cols)
    return (torch.randn(rows, cols, generator=g, device="cuda").to(TYPES[dtype]),
            torch.randn(rows, cols, generator=g, device="cuda").to(TYPES[out]))


def check(x, res, out, p=0.3, seed=SEED, call=3, step=5, to=None):
    want, bound = ref.dropout(x, p, seed, call, step, res, TYPES[out])
    y = binding.dropout_forward(x, p, seed, call, step, residual=res, dtype=TYPES[out], out=to)
    assert_within(y, want, bound, "y")
    want, bound = ref.dropout(x, p, seed, call, step, None, TYPES[out])
    dx = binding.dropout_backward(x, p, seed, call, step, dtype=TYPES[out])
    assert_within(dx, want, bound, "dx")
    return y, dx


# around the generator's blocks of eight and what a thread takes; odd widths
@pytest.mark.parametrize("dtype", ["f32", "bf16"])
@pytest.mark.parametrize("out", ["f32", "bf16"])
@pytest.mark.parametrize("rows,cols", [(1, 1), (1, 7), (1, 8), (1, 9), (3, 5), (2, 12), (5, 16), (7, 31), (1, 4096), (13, 650), (9, 1023), (33, 768),
                                       (1, 70001), (70001, 1), (600, 1000)])
def test_sizes_and_types(rows, cols, dtype, out):
    x, res = draw(rows, cols, dtype, out)
    check(x, res, out)
    check(x, None, out)


@pytest.mark.parametrize("p", [0.0, 1.0, 0.5, 0.1, 1e-6, 2.0 ** -17, 2.0 ** -16, 1 - 2.0 ** -16, 1 - 2.0 ** -18, 0.999])
def test_probabilities(p):
    x, res = draw(40, 300, "f32", "f32")
    y, dx = check(x, res, "f32", p)
    if p == 0.0:
        assert torch.equal(dx, x)
    if p == 1.0:
        assert torch.equal(y, res) and (dx == 0).all()


@pytest.mark.parametrize("seed,call,step", [(0, 0, 0), (2 ** 64 - 1, 2 ** 32 - 1, 2 ** 32 - 1), (2 ** 32, 1, 0), (1, 0, 2 ** 31)])
def test_seeds_calls_and_steps(seed, call, step):
    x, res = draw(20, 111, "f32", "f32")
    check(x, res, "f32", 0.4, seed, call, step)


def test_the_mask_depends_on_neither_types_nor_strides():
    x = torch.ones(50, 77, device="cuda")
    want = binding.dropout_forward(x, 0.25, 9) > 0
    assert torch.equal(binding.dropout_forward(x.bfloat16(), 0.25, 9) > 0, want)
    wide = torch.ones(50, 200, device="cuda")
    for lo in (0, 1, 4, 8):
        out = torch.full((50, 99), 7.0, device="cuda")
        got = binding.dropout_forward(wide[:, lo:lo + 77], 0.25, 9, out=out[:, 3:80])
        assert torch.equal(got > 0, want) and (out[:, :3] == 7).all() and (out[:, 80:] == 7).all()
    assert torch.equal(binding.dropout_backward(x, 0.25, 9) > 0, want)
    for other in (dict(seed=10), dict(seed=9, call=1), dict(seed=9, step=1)):
        assert not torch.equal(binding.dropout_forward(x, 0.25, **other) > 0, want)


@pytest.mark.parametrize("dtype", ["f32", "bf16"])
@pytest.mark.parametrize("cols,lo", [(72, 0), (72, 8), (72, 1), (72, 3), (650, 2), (8, 8)])
def test_strided_rows(cols, lo, dtype):
    x, res = draw(30, cols, dtype, dtype)
    wx, wr = (torch.zeros(30, cols + 24, dtype=TYPES[dtype], device="cuda") for _ in range(2))
    vx, vr = wx[:, lo:lo + cols], wr[:, lo:lo + cols]
    vx.copy_(x)
    vr.copy_(res)
    out = torch.full((30, cols + 16), 7.0, dtype=TYPES[dtype], device="cuda")
    check(vx, vr, dtype, to=out[:, 8:8 + cols])
    assert (out[:, :8] == 7).all() and (out[:, 8 + cols:] == 7).all()


def test_in_place():
    for dtype in ("f32", "bf16"):
        x, res = draw(33, 96, dtype, dtype)
        y = binding.dropout_forward(x, 0.2, 1, residual=res)
        a, b = x.clone(), res.clone()
        assert torch.equal(binding.dropout_forward(a, 0.2, 1, residual=res, out=a), y)
        assert torch.equal(binding.dropout_forward(x, 0.2, 1, residual=b, out=b), y)
        a = x.clone()
        assert torch.equal(binding.dropout_backward(a, 0.2, 1, out=a), binding.dropout_backward(x, 0.2, 1))


def test_dropped_values_do_not_matter():
    x, res = draw(64, 64, "f32", "f32")
    stay = binding.dropout_forward(torch.ones_like(x), 0.5, 4) > 0
    want = binding.dropout_forward(x, 0.5, 4, residual=res)
    for bad in (float("nan"), float("inf")):
        assert torch.equal(binding.dropout_forward(torch.where(stay, x, bad), 0.5, 4, residual=res), want)
    y = binding.dropout_forward(torch.where(stay, float("nan"), x), 0.5, 4, residual=res)
    assert torch.equal(torch.isnan(y), stay)


def test_share_and_mean():
    """16 million draws: the share of kept elements is within six standard deviations of 1 - p."""
    n, p = 1 << 24, 0.1
    y = binding.dropout_forward(torch.ones(1, n, device="cuda"), p, 123456789)
    q = 1 - round(p * 65536) / 65536
    share = float((y > 0).double().mean())
    assert abs(share - q) <= 6 * (q * (1 - q) / n) ** 0.5
    assert abs(float(y.double().mean()) - 1) <= 6 * ((1 - q) / q / n) ** 0.5 + 1e-7


def test_elements_past_32_bits():
    """The index, not its low 32 bits, chooses the draw: 4.4e9 elements, the last of them checked."""
    rows, cols = 66000, 66000
    x = torch.ones(rows, cols, dtype=torch.bfloat16, device="cuda")
    y = binding.dropout_forward(x, 0.5, 77, out=x)
    for r in (0, 32537, 65075, 65999):
        want = ref.keep(np.arange(r * cols, (r + 1) * cols), 0.5, 77, 0, 0)
        assert np.array_equal((y[r] > 0).cpu().numpy(), want)


def test_a_step_counted_on_the_device():
    x, res = draw(16, 200, "f32", "f32")
    count = torch.tensor([40], dtype=torch.int64, device="cuda")
    assert torch.equal(binding.dropout_forward(x, 0.3, 5, 6, count), binding.dropout_forward(x, 0.3, 5, 6, 40))
    count.fill_(2 ** 32 + 41)              # its low 32 bits
    assert torch.equal(binding.dropout_backward(x, 0.3, 5, 6, count), binding.dropout_backward(x, 0.3, 5, 6, 41))
    count.fill_(-1)
    assert torch.equal(binding.dropout_backward(x, 0.3, 5, 6, count), binding.dropout_backward(x, 0.3, 5, 6, 2 ** 32 - 1))
    count.fill_(0)
    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    with torch.cuda.stream(side):
        binding.dropout_forward(x, 0.3, 5, 6, count)
    torch.cuda.synchronize()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        y = binding.dropout_forward(x, 0.3, 5, 6, count, residual=res)
        count.add_(1)
    for k in range(3):
        graph.replay()
        assert torch.equal(y, binding.dropout_forward(x, 0.3, 5, 6, k, residual=res))


def test_nothing_to_do():
    for shape in ((0, 8), (8, 0)):
        assert binding.dropout_forward(torch.empty(shape, device="cuda"), 0.1, 0).shape == shape


def test_refusals():
    x, res = draw(8, 16, "f32", "f32")
    for bad in (dict(seed=-1), dict(seed=2 ** 64), dict(call=-1), dict(call=2 ** 32), dict(step=-1), dict(step=2 ** 32),
                dict(step=torch.zeros(2, dtype=torch.int64, device="cuda")), dict(step=torch.zeros(1, device="cuda")), dict(residual=res.bfloat16(), dtype=torch.float32),
                dict(residual=res[:, :8]), dict(out=torch.empty(8, 15, device="cuda")), dict(dtype=torch.float16),
                dict(dtype=torch.bfloat16, out=torch.empty(8, 16, device="cuda")), dict(residual=res.cpu())):
        kw = dict(seed=0) | bad
        with pytest.raises(ValueError):
            binding.dropout_forward(x, 0.1, **kw)
    for t in (x.half(), x[0], x.t()):
        with pytest.raises(ValueError):
            binding.dropout_forward(t, 0.1, 0)
    for p in (-0.1, 1.1, float("nan")):
        with pytest.raises(binding.CdgrabError):
            binding.dropout_forward(x, p, 0)
        with pytest.raises(binding.CdgrabError):
            binding.dropout_backward(x, p, 0)
    with pytest.raises(binding.CdgrabError):
        binding.dropout_forward(x, 0.1, 0, out=x[:1].expand(8, 16))
