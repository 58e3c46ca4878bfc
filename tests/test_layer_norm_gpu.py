"""Layer norm, forward and backward, against the formulas in 64 bits."""
import pytest
import torch

import operators_ref as ref
from paper_2302_00845_b200 import binding

pytestmark = pytest.mark.gpu
TYPES = {"f32": torch.float32, "bf16": torch.bfloat16}


def draw(m, rows, cols, dtype, seed=0):
    g = torch.Generator(device="cuda").manual_seed(seed * 1000 + m + rows + cols)
    x = torch.randn(m * rows, cols, generator=g, device="cuda") * 2 + torch.randn(m * rows, 1, generator=g, device="cuda")
    dy = torch.randn(m * rows, cols, generator=g, device="cuda")
    w = 1 + 0.2 * torch.randn(cols, generator=g, device="cuda")
    b = 0.3 * torch.randn(cols, generator=g, device="cuda")
    return x.to(TYPES[dtype]), dy.to(TYPES[dtype]), w, b


def check(x, dy, w, b, m, grads, eps=1e-5, dweight=None, dbias=None, **kw):
    y, mean, rstd = binding.layer_norm_forward(x, w, b, eps=eps, out=kw.get("out"))
    for got, (want, bound), name in zip((y, mean, rstd), ref.layer_norm_forward(x, w, b, eps), ("y", "mean", "rstd")):
        ref.assert_within(got, want, bound, name)
    if dweight is None:
        buf = torch.full((m, 2 * x.shape[1]), float("nan"), dtype=TYPES[grads], device="cuda")
        dweight, dbias = buf[:, :x.shape[1]], buf[:, x.shape[1]:]
    want = ref.layer_norm_backward(dy, x, w, mean, rstd, m, TYPES[grads])
    dx = binding.layer_norm_backward(dy, x, w, mean, rstd, dweight, dbias, dx=kw.get("dx"))
    for got, (val, bound), name in zip((dx, dweight, dbias), want, ("dx", "dweight", "dbias")):
        ref.assert_within(got, val, bound, name)
    assert binding.operators_status() == binding.OK
    return y, mean, rstd, dx, dweight, dbias


# around the vector widths, the register tiles and the switch from a warp to a block per row
COLS = [1, 2, 3, 8, 31, 33, 64, 100, 256, 257, 512, 650, 768, 1000, 1024, 1025, 1026, 1032, 2048, 4097, 8192]


@pytest.mark.parametrize("dtype", ["f32", "bf16"])
@pytest.mark.parametrize("cols", COLS)
def test_columns(cols, dtype):
    check(*draw(3, 5, cols, dtype), 3, "f32")


@pytest.mark.parametrize("cols,dtype", [(16384, "bf16"), (16385, "f32"), (40000, "bf16"), (70001, "f32")])
def test_very_long_rows(cols, dtype):
    check(*draw(2, 3, cols, dtype), 2, "bf16")


@pytest.mark.parametrize("m,rows", [(1, 1), (1, 2), (2, 1), (5, 7), (64, 1), (1, 4097), (64, 33), (300, 3), (3, 1001)])
@pytest.mark.parametrize("grads", ["f32", "bf16"])
def test_workers_and_rows(m, rows, grads):
    check(*draw(m, rows, 96, "bf16"), m, grads)


def test_strided_rows_and_gather_buffer_views():
    m, rows, cols = 4, 9, 72
    x, dy, w, b = draw(m, rows, cols, "bf16")
    wide = torch.zeros(m * rows, 200, dtype=torch.bfloat16, device="cuda")
    for lo in (0, 8, 1, 3):           # from 16-byte aligned down to odd starts
        xs = wide[:, lo:lo + cols]
        xs.copy_(x)
        out = torch.full((m * rows, cols + 5), 7.0, dtype=torch.bfloat16, device="cuda")
        buf = torch.full((2, m, 500), 5.0, device="cuda")
        check(xs, dy, w, b, m, "f32", dweight=buf[1, :, 100 + lo:100 + lo + cols], dbias=buf[1, :, 300:300 + cols],
              out=out[:, 2:2 + cols])
        assert (out[:, :2] == 7).all() and (out[:, 2 + cols:] == 7).all()
        assert (buf[0] == 5).all() and (buf[1, :, :100 + lo] == 5).all() and (buf[1, :, 300 + cols:] == 5).all()
        assert (buf[1, :, 100 + lo + cols:300] == 5).all()


def test_in_place():
    x, dy, w, b = draw(2, 6, 130, "f32")
    y, mean, rstd = binding.layer_norm_forward(x, w, b)
    z = x.clone()
    y2, _, _ = binding.layer_norm_forward(z, w, b, out=z)
    assert torch.equal(y, y2)
    dw = torch.empty(2, 130, device="cuda")
    dx = binding.layer_norm_backward(dy, x, w, mean, rstd, dw)
    dw2 = torch.empty(2, 130, device="cuda")
    g = dy.clone()
    assert torch.equal(binding.layer_norm_backward(g, x, w, mean, rstd, dw2, dx=g), dx) and torch.equal(dw, dw2)
    g = x.clone()
    assert torch.equal(binding.layer_norm_backward(dy, g, w, mean, rstd, dw2, dx=g), dx) and torch.equal(dw, dw2)


def test_without_weight_or_bias():
    x, dy, _, _ = draw(2, 4, 48, "f32")
    check(x, dy, None, None, 2, "f32")
    y, mean, rstd = binding.layer_norm_forward(x)
    dw, db = torch.empty(2, 48, device="cuda"), torch.empty(2, 48, device="cuda")
    dx = binding.layer_norm_backward(dy, x, None, mean, rstd, dw, db)
    only = torch.empty(2, 48, device="cuda")
    assert torch.equal(binding.layer_norm_backward(dy, x, None, mean, rstd, None, only), dx) and torch.equal(only, db)
    assert torch.equal(binding.layer_norm_backward(dy, x, None, mean, rstd), dx)


def test_constant_and_large_rows():
    x, dy, w, b = draw(1, 4, 200, "f32")
    x[0] = 3.0                 # no variance: y = bias
    x[1] = x[1] * 1e-3 + 1e3   # mean far above the spread
    x[2] *= 1e15
    check(x, dy, w, b, 1, "f32")


def test_nothing_to_do():
    w = torch.ones(16, device="cuda")
    x = torch.empty(0, 16, device="cuda")
    y, mean, rstd = binding.layer_norm_forward(x, w)
    assert y.shape == (0, 16) and mean.shape == (0,)
    dw = torch.full((3, 16), 9.0, device="cuda")
    binding.layer_norm_backward(x, x, w, mean, rstd, dw)
    assert (dw == 0).all()


def test_gradient_against_differences():
    """Central differences of sum(r * y) in 64 bits of the forward pass in 32: h^2 and rounding over h."""
    m, rows, cols = 2, 3, 24
    x, dy, w, b = draw(m, rows, cols, "f32", seed=5)
    _, mean, rstd = binding.layer_norm_forward(x, w, b)
    dw, db = torch.empty(m, cols, device="cuda"), torch.empty(m, cols, device="cuda")
    dx = binding.layer_norm_backward(dy, x, w, mean, rstd, dw, db)

    def loss(x_, w_, b_, i=None):
        y = binding.layer_norm_forward(x_, w_, b_)[0].double() * dy.double()
        return float((y if i is None else y[i * rows:(i + 1) * rows]).sum())

    h = 2.0 ** -8
    tol = 4e-3                # h^2 times third derivatives of order ten, and 1e-5 of rounding over 2 h
    for r, c in ((0, 0), (2, 7), (5, 23)):
        up, dn = x.clone(), x.clone()
        up[r, c] += h
        dn[r, c] -= h
        assert abs((loss(up, w, b) - loss(dn, w, b)) / (2 * h) - float(dx[r, c])) <= tol
    for i, c in ((0, 3), (1, 20)):
        up, dn = w.clone(), w.clone()
        up[c] += h
        dn[c] -= h
        assert abs((loss(x, up, b, i) - loss(x, dn, b, i)) / (2 * h) - float(dw[i, c])) <= tol
        up, dn = b.clone(), b.clone()
        up[c] += h
        dn[c] -= h
        assert abs((loss(x, w, up, i) - loss(x, w, dn, i)) / (2 * h) - float(db[i, c])) <= tol


def test_same_bits_every_time_and_on_another_stream():
    x, dy, w, b = draw(7, 211, 650, "bf16")
    first = check(x, dy, w, b, 7, "f32")
    s = torch.cuda.Stream()
    s.wait_stream(torch.cuda.current_stream())
    for _ in range(3):
        y, mean, rstd = binding.layer_norm_forward(x, w, b, stream=s)
        dw, db = torch.empty(7, 650, device="cuda"), torch.empty(7, 650, device="cuda")
        dx = binding.layer_norm_backward(dy, x, w, mean, rstd, dw, db, stream=s)
        s.synchronize()
        for got, want in zip((y, mean, rstd, dx, dw, db), first):
            assert torch.equal(got, want)


def test_refusals():
    x, dy, w, b = draw(2, 3, 16, "f32")
    _, mean, rstd = binding.layer_norm_forward(x, w, b)
    with pytest.raises(ValueError):
        binding.layer_norm_forward(x.half())
    with pytest.raises(ValueError):
        binding.layer_norm_forward(x.t())
    with pytest.raises(ValueError):
        binding.layer_norm_forward(x, w[:8])
    with pytest.raises(ValueError):
        binding.layer_norm_forward(x, w.double())
    with pytest.raises(ValueError):
        binding.layer_norm_forward(x.cpu(), w)
    with pytest.raises(ValueError):
        binding.layer_norm_backward(dy, x, w, mean, rstd, torch.empty(4, 16, device="cuda"))   # 6 rows, 4 workers
    with pytest.raises(ValueError):
        binding.layer_norm_backward(dy.bfloat16(), x, w, mean, rstd)
    with pytest.raises(binding.CdgrabError):
        binding.layer_norm_forward(x, w, b, eps=-1.0)
    with pytest.raises(binding.CdgrabError):
        binding.layer_norm_forward(x, w, b, eps=float("nan"))


def test_one_worker_with_gradients_in_different_buffers():
    """With a single worker there is no distance from row to row: views of buffers of any width go together."""
    x, dy, w, b = draw(1, 6, 40, "f32")
    wide, narrow = torch.full((1, 90), 3.0, device="cuda"), torch.full((1, 55), 3.0, device="cuda")
    check(x, dy, w, b, 1, "f32", dweight=wide[:, 20:60], dbias=narrow[:, 4:44])
    assert (wide[:, :20] == 3).all() and (wide[:, 60:] == 3).all() and (narrow[:, :4] == 3).all() and (narrow[:, 44:] == 3).all()
    x, dy, w, b = draw(2, 3, 40, "f32")
    _, mean, rstd = binding.layer_norm_forward(x, w, b)
    with pytest.raises(ValueError):
        binding.layer_norm_backward(dy, x, w, mean, rstd, torch.empty(2, 90, device="cuda")[:, :40], torch.empty(2, 40, device="cuda"))


@pytest.mark.parametrize("cols", [8192, 8193, 16384])
def test_sums_over_many_rows_are_no_single_chain(cols):
    """20,000 rows that all add 0.1: one chain of 32-bit additions drifts by 1e-4 of the sum.  The rows are added up in
    parts, so that no value goes through more than about a thousand additions, whatever the number of columns."""
    rows = 20000
    g = torch.Generator(device="cuda").manual_seed(cols)
    x = torch.randn(rows, cols, generator=g, device="cuda")
    x[:, ::2] = x[:, ::2].abs() + 0.5          # the sums of dy n have a sign too
    dy = torch.full_like(x, 0.1)
    _, mean, rstd = binding.layer_norm_forward(x)
    dw, db = torch.empty(1, cols, device="cuda"), torch.empty(1, cols, device="cuda")
    binding.layer_norm_backward(dy, x, None, mean, rstd, dw, db)
    value = dy[0, 0].double()
    n = torch.zeros(cols, dtype=torch.float64, device="cuda")
    size, off = n.clone(), n.clone()
    for i in range(0, rows, 2000):
        part = (x[i:i + 2000].double() - mean[i:i + 2000, None].double()) * rstd[i:i + 2000, None].double()
        n += part.sum(0)
        size += part.abs().sum(0)
        off += 3 * part.abs().sum(0) + (x[i:i + 2000].abs() + mean[i:i + 2000, None].abs()).mul(rstd[i:i + 2000, None]).double().sum(0)
    chain = 1088 * ref.U32
    assert (db[0].double() - rows * value).abs().max() <= chain * rows * value
    assert ((dw[0].double() - value * n).abs() <= value * (chain * size + ref.U32 * off)).all()


@pytest.mark.parametrize("m,rows,cols,dtype", [(1, 4097, 8193, "bf16"), (5, 333, 16384, "bf16"), (3, 50, 9001, "f32"), (64, 17, 8200, "f32")])
@pytest.mark.parametrize("grads", ["f32", "bf16"])
def test_long_rows_of_workers(m, rows, cols, dtype, grads):
    check(*draw(m, rows, cols, dtype), m, grads)


@pytest.mark.parametrize("rows,cols,dtype", [(9473, 64, "bf16"), (20001, 650, "bf16"), (30011, 33, "f32"), (40000, 1000, "bf16"), (3111, 1025, "f32"),
                                             (7001, 1026, "bf16"), (5003, 2048, "f32"), (1500, 8192, "bf16"), (1301, 8191, "f32")])
def test_more_rows_than_the_grid_takes_at_once(rows, cols, dtype):
    """Warps, and blocks, that go on to further rows with the next one already requested."""
    check(*draw(1, rows, cols, dtype), 1, "f32")
