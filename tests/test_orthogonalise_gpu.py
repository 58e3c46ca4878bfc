"""The orthogonalised update against the iteration in 64 bits.

The products' operands are held in 16 bits with 11 significant ones.  Modelled in 64 bits with that rounding of
X, A and B, the result is at most 3.9e-3 off (2-norm, relative) for 16 x 16 and 2.5e-3 from 64 x 64 on, the
output's own rounding to 8 bits (1.7e-3) included; the tests allow 6e-3 and 4e-3."""
import pytest
import torch

import operators_ref as ref
from paper_2302_00845_b200 import binding

pytestmark = pytest.mark.gpu


def gradient(batch, rows, cols, seed=0, dtype=torch.float32, scale=1e-2):
    g = torch.Generator(device="cuda").manual_seed(seed + 31 * rows + cols)
    k = min(16, rows, cols)
    x = torch.matmul(torch.randn(batch, rows, k, generator=g, device="cuda"),
                     torch.randn(batch, k, cols, generator=g, device="cuda")) / (2 * k) ** 0.5
    return ((x + torch.randn(batch, rows, cols, generator=g, device="cuda") / 2 ** 0.5) * scale).to(dtype)


def off(got, want):
    return float((got.double() - want).norm() / want.norm())


def check(g, **kw):
    o = binding.orthogonalise(g, **kw)
    assert binding.operators_status() == binding.OK
    want = ref.orthogonalise(g, **kw)
    assert o.dtype == torch.bfloat16 and o.shape == g.shape
    assert off(o, want) <= (4e-3 if min(g.shape[-2:]) >= 64 else 6e-3)
    return o


@pytest.mark.parametrize("rows,cols", [(16, 16), (17, 40), (40, 17), (31, 33), (64, 64), (65, 64), (64, 200), (127, 129),
                                       (128, 128), (129, 257), (257, 129), (200, 1000), (1000, 200), (255, 384),
                                       (650, 650), (500, 777), (1030, 640), (128, 576), (576, 128), (128, 577), (100, 321), (449, 65), (64, 385),
                                       (129, 130), (33, 515)])
@pytest.mark.parametrize("dtype", [torch.float32, torch.bfloat16])
def test_shapes(rows, cols, dtype):
    check(gradient(1, rows, cols, dtype=dtype)[0])


@pytest.mark.parametrize("rows,cols", [(1, 1), (1, 5), (5, 1), (1, 300), (300, 1), (2, 2), (3, 700), (8, 8)])
def test_tiny(rows, cols):
    """Well-conditioned small matrices: each singular value goes through the same five polynomials."""
    u = torch.linalg.qr(torch.randn(max(rows, cols), min(rows, cols), dtype=torch.float64))[0]
    g = (u if rows > cols else u.T).float().cuda()
    check(g)


@pytest.mark.parametrize("batch,rows,cols", [(2, 64, 96), (7, 130, 100), (3, 33, 20), (5, 256, 512)])
def test_batches(batch, rows, cols):
    g = gradient(batch, rows, cols)
    g[1] *= 1e4              # each matrix has its own norm
    o = check(g)
    for i in range(batch):
        assert off(o[i], ref.orthogonalise(g[i])) <= 6e-3
        assert torch.equal(o[i], binding.orthogonalise(g[i]))


@pytest.mark.parametrize("scale", [1e-18, 1e-6, 1.0, 1e6, 1e18])
def test_scales(scale):
    check(gradient(1, 96, 160, scale=scale)[0], eps=0.0)


def test_eps_and_steps_and_coefficients():
    g = gradient(1, 80, 120)[0]
    check(g, steps=1)
    check(g, steps=10, coeffs=(1.5, -0.5, 0.0))
    check(g, steps=3, coeffs=(2.0, -1.5, 0.5))
    check(g * 1e-8, eps=1e-3)


def test_zeros():
    g = torch.zeros(2, 40, 70, device="cuda")
    g[1] = gradient(1, 40, 70)[0]
    o = binding.orthogonalise(g)
    assert (o[0] == 0).all() and off(o[1], ref.orthogonalise(g[1])) <= 6e-3
    g[1, 10:20] = 0          # rows without a gradient keep none
    o = binding.orthogonalise(g)
    assert (o[1, 10:20] == 0).all() and off(o[1], ref.orthogonalise(g[1])) <= 6e-3


def test_one_large_entry():
    g = gradient(1, 64, 64)[0]
    g[3, 5] = 50.0           # nearly all of the norm in one place
    check(g)


def test_strides():
    wide = torch.zeros(3, 100, 211, device="cuda")
    for lo in (0, 3, 4):
        g = wide[:, 10:90, lo:lo + 150]
        g.copy_(gradient(3, 80, 150))
        out = torch.full((3, 81, 155), 2.0, dtype=torch.bfloat16, device="cuda")
        o = binding.orthogonalise(g, out=out[:, :80, lo:lo + 150])
        assert torch.equal(o, binding.orthogonalise(g.contiguous()))
        assert (out[:, 80] == 2).all() and (out[:, :, :lo] == 2).all() and (out[:, :, lo + 150:] == 2).all()
    tall = wide[:, :, 1:81].transpose(0, 0)
    g = tall[:, :100]
    g.copy_(gradient(3, 100, 80))
    assert torch.equal(binding.orthogonalise(g), binding.orthogonalise(g.contiguous()))


def test_transposed_matrices_agree():
    g = gradient(1, 70, 190)[0]
    assert off(binding.orthogonalise(g.T.contiguous()).T, binding.orthogonalise(g).double()) <= 2e-3


def test_nothing_to_do():
    for shape in ((0, 5, 5), (2, 0, 5), (2, 5, 0)):
        assert binding.orthogonalise(torch.empty(shape, device="cuda")).shape == shape


def test_same_bits_every_time_and_on_another_stream():
    g = gradient(4, 300, 200)
    first = binding.orthogonalise(g)
    s = torch.cuda.Stream()
    s.wait_stream(torch.cuda.current_stream())
    for _ in range(3):
        o = binding.orthogonalise(g, stream=s)
        s.synchronize()
        assert torch.equal(o, first)


def test_refusals():
    g = gradient(1, 32, 48)[0]
    for bad in (lambda: binding.orthogonalise(g.half()), lambda: binding.orthogonalise(g[0]), lambda: binding.orthogonalise(g.T),
                lambda: binding.orthogonalise(g.cpu()), lambda: binding.orthogonalise(g, coeffs=(1.0, 2.0)),
                lambda: binding.orthogonalise(g, out=torch.empty_like(g))):
        with pytest.raises(ValueError):
            bad()
    for kw in (dict(steps=0), dict(steps=65), dict(eps=-1.0), dict(coeffs=(float("nan"), 0.0, 0.0))):
        with pytest.raises(binding.CdgrabError):
            binding.orthogonalise(g, **kw)


@pytest.mark.parametrize("rows,cols", [(40, 70), (300, 700)])
def test_coefficients_at_the_edge_of_the_range(rows, cols):
    """One singular value that doubles with every step: 128 is the last that X is stored with; one step more is refused."""
    g = torch.zeros(rows, cols, device="cuda")
    g[3, 5] = 1.0
    want = torch.zeros(rows, cols, device="cuda")
    want[3, 5] = 256.0
    assert torch.equal(binding.orthogonalise(g, steps=8, coeffs=(2.0, 0.0, 0.0), eps=0.0).float(), want)
    for steps in (9, 10):
        with pytest.raises(binding.CdgrabError):
            binding.orthogonalise(g, steps=steps, coeffs=(2.0, 0.0, 0.0), eps=0.0)


# tiles of 256 columns (there are as many of them as SMs), several to a block and product, batches in two parts of unequal
# size, remainders in both directions; then tiles of 128 with more of them than SMs
@pytest.mark.parametrize("batch,rows,cols,dtype", [(12, 2304, 768, torch.bfloat16), (13, 770, 2310, torch.float32), (7, 1030, 1300, torch.bfloat16),
                                                   (7, 1300, 1030, torch.float32), (200, 100, 600, torch.float32), (31, 600, 1021, torch.bfloat16),
                                                   (1, 1960, 2040, torch.float32), (1, 2041, 1961, torch.bfloat16), (2, 1300, 1290, torch.float32)])
def test_more_tiles_than_multiprocessors(batch, rows, cols, dtype):
    g = gradient(batch, rows, cols, dtype=dtype)
    o = check(g)
    want = ref.orthogonalise(g)
    for i in range(batch):
        assert off(o[i], want[i]) <= 4e-3
    for _ in range(3):
        assert torch.equal(binding.orthogonalise(g), o)


@pytest.mark.parametrize("rows,cols", [(2, 40), (130, 70)])
def test_output_rows_further_apart_than_32_bits(rows, cols):
    g = gradient(1, rows, cols)[0]
    far = torch.empty((rows - 1) * (1 << 24) + cols if rows > 2 else (1 << 31) + 8 + cols, dtype=torch.bfloat16, device="cuda")
    out = far.as_strided((rows, cols), ((1 << 24) if rows > 2 else (1 << 31) + 8, 1))        # 4 GB, the last row past 2^31
    assert torch.equal(binding.orthogonalise(g, out=out), binding.orthogonalise(g))
