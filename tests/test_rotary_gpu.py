"""The norms of queries and keys with the rotation, forward and backward, against the formulas in 64 bits."""
import pytest
import torch

import model_operators_ref as ref
from operators_ref import assert_within
from paper_2302_00845_b200 import binding

pytestmark = pytest.mark.gpu
TYPES = {"f32": torch.float32, "bf16": torch.bfloat16}


def draw(b, t, h, hk, d, dtype="bf16", seed=0, packed=False):
    g = torch.Generator(device="cuda").manual_seed(seed * 101 + b + t + h + hk + d)
    r = lambda *s: torch.randn(*s, generator=g, device="cuda")  # noqa: E731
    dt = TYPES[dtype]
    if packed:
        qkv, dqkv = r(b, t, h + 2 * hk, d).to(dt), r(b, t, h + 2 * hk, d).to(dt)
        (q, k), (dq, dk) = ((v[:, :, :h], v[:, :, h:h + hk]) for v in (qkv, dqkv))
    else:
        q, k, dq, dk = (r(b, t, n, d).to(dt) for n in (h, hk, h, hk))
    return q, k, 1 + 0.2 * r(d), 1 + 0.2 * r(d), dq, dk


def check(q, k, qw, kw, dq, dk, m=1, grads="f32", positions=None, base=10000.0, rotary_dim=None, interleaved=False, eps=1e-6, lens=None,
          **out):
    d = q.shape[3]
    opts = dict(positions=positions, base=base, rotary_dim=rotary_dim, interleaved=interleaved, eps=eps, lens=lens)
    args = (positions, base, d if rotary_dim is None else rotary_dim, interleaved, eps, lens)
    buf = torch.full((m, 2 * d), float("nan"), dtype=TYPES[grads], device="cuda")
    y = binding.rotary_forward(q, k, qw, kw, **opts, **out)
    for got, x, w, name in zip(y, (q, k), (qw, kw), "qk"):
        assert_within(got, *ref.rotary(x, w, *args), name)
    dx = binding.rotary_backward(dq, dk, q, k, qw, kw, dq_weight=buf[:, :d], dk_weight=buf[:, d:], **opts)
    for i, (got, g, x, w) in enumerate(zip(dx, (dq, dk), (q, k), (qw, kw))):
        (val, bound), (dw, wbound) = ref.rotary(x, w, *args, dy=g, m=m, grad_dtype=TYPES[grads])
        assert_within(got, val, bound, "d" + "qk"[i])
        assert_within(buf[:, i * d:(i + 1) * d], dw, wbound, "dw " + "qk"[i])
    assert binding.operators_status() == binding.OK
    again = torch.empty_like(buf)
    dx2 = binding.rotary_backward(dq, dk, q, k, qw, kw, dq_weight=again[:, :d], dk_weight=again[:, d:], **opts)
    assert torch.equal(buf, again) and torch.equal(dx[0], dx2[0]) and torch.equal(dx[1], dx2[1])
    return y, dx, buf


@pytest.mark.parametrize("dtype", ["f32", "bf16"])
@pytest.mark.parametrize("interleaved", [False, True])
@pytest.mark.parametrize("d", [8, 16, 24, 32, 40, 48, 56, 64, 72, 80, 96, 104, 112, 128, 136, 160, 192, 200, 248, 256])
def test_head_dimensions(d, interleaved, dtype):
    check(*draw(2, 5, 3, 2, d, dtype), interleaved=interleaved)


@pytest.mark.parametrize("dtype", ["f32", "bf16"])
@pytest.mark.parametrize("interleaved", [False, True])
@pytest.mark.parametrize("d,rot", [(64, 0), (64, 8), (64, 16), (64, 32), (64, 56), (80, 40), (80, 64), (128, 64), (96, 24), (40, 32), (256, 128), (256, 248),
                                   (8, 0), (24, 16)])
def test_part_of_a_head(d, rot, interleaved, dtype):
    check(*draw(2, 7, 2, 1, d, dtype), rotary_dim=rot, interleaved=interleaved)


@pytest.mark.parametrize("b,t,h,hk", [(1, 1, 1, 1), (1, 1, 12, 4), (8, 1, 12, 4), (1, 2, 1, 7), (3, 33, 5, 5), (2, 129, 16, 1), (1, 1000, 4, 2), (5, 31, 40, 8),
                                      (1, 3, 300, 2), (700, 1, 2, 1), (1, 5000, 1, 1)])
def test_lengths_and_heads(b, t, h, hk):
    check(*draw(b, t, h, hk, 64))


@pytest.mark.parametrize("m,per,t", [(1, 1, 1), (2, 1, 5), (3, 4, 7), (16, 1, 65), (64, 1, 3), (300, 1, 2), (5, 2, 200), (2, 1, 3001)])
@pytest.mark.parametrize("grads", ["f32", "bf16"])
def test_workers(m, per, t, grads):
    check(*draw(m * per, t, 3, 2, 40), m=m, grads=grads)


@pytest.mark.parametrize("bits", [torch.int32, torch.int64])
def test_positions(bits):
    x = draw(3, 20, 2, 2, 64, "f32")
    one = torch.arange(20, device="cuda", dtype=bits) * 3 + 7
    check(*x, positions=one)
    each = torch.randint(0, 100_000, (3, 20), device="cuda", dtype=bits)
    check(*x, positions=each)
    wide = torch.zeros(3, 50, device="cuda", dtype=bits)
    wide[:, 5:25] = each
    check(*x, positions=wide[:, 5:25])
    check(*x, positions=-each)
    same = binding.rotary_forward(*x[:4], positions=one[None].expand(3, 20))
    assert all(torch.equal(a, c) for a, c in zip(same, binding.rotary_forward(*x[:4], positions=one)))


@pytest.mark.parametrize("start", [131_072, 1_000_003, 16_777_217, 2 ** 31 - 40])
def test_far_positions(start):
    """A product of 32-bit numbers would be whole radians off there."""
    check(*draw(2, 33, 2, 1, 128, "f32"), positions=start + torch.arange(33, device="cuda"))


def test_rotation_keeps_products_of_equal_distance():
    """q at i with k at j depends on i - j alone."""
    q, k, *_ = draw(1, 1, 1, 1, 64, "f32")
    at = lambda x, p: binding.rotary_forward(x, None, positions=torch.tensor([p], device="cuda"))[0].double()  # noqa: E731
    near, far = (at(q, 5) * at(k, 2)).sum(), (at(q, 500_005) * at(k, 500_002)).sum()
    # 64 products of values with the errors of two rotations each
    assert abs(float(near - far)) <= 64 * 40 * 2.0 ** -24 * 3


@pytest.mark.parametrize("base", [10000.0, 500_000.0, 1.0, 0.5, 2.0])
def test_bases(base):
    check(*draw(2, 40, 2, 2, 64, "f32"), base=base)


def test_lengths_hide_what_lies_past_them():
    q, k, qw, kw, dq, dk = draw(4, 30, 3, 2, 64)
    lens = torch.tensor([30, 17, 0, 1], dtype=torch.int32, device="cuda")
    for i, n in enumerate(lens.tolist()):
        for t in (q, k, dq, dk):
            t[i, n:] = float("nan")
    y, dx, _ = check(q, k, qw, kw, dq, dk, m=4, lens=lens)
    for i, n in enumerate(lens.tolist()):
        assert all((v[i, n:] == 0).all() for v in (*y, *dx))
    check(q[:2], k[:2], qw, kw, dq[:2], dk[:2], lens=torch.tensor([40, -3], dtype=torch.int32, device="cuda").clamp(0, 30))


def test_lengths_outside_the_range():
    """More than there are: all; less than none: none."""
    x = draw(2, 9, 2, 1, 32)
    y = binding.rotary_forward(*x[:4], lens=torch.tensor([2 ** 31 - 1, -5], dtype=torch.int32, device="cuda"))
    full = binding.rotary_forward(*x[:4])
    assert torch.equal(y[0][0], full[0][0]) and (y[0][1] == 0).all() and (y[1][1] == 0).all()


def test_no_epsilon():
    """Padded tokens have no size, and with eps = 0 no norm: they are left out all the same."""
    x = draw(2, 30, 3, 2, 40, "f32")
    check(*x, m=2, eps=0.0, lens=torch.tensor([30, 4], dtype=torch.int32, device="cuda"))


def test_slices_of_one_projection_and_of_its_gradient():
    q, k, qw, kw, dq, dk = x = draw(3, 50, 6, 2, 64, packed=True)
    assert not q.is_contiguous()
    y, dx, buf = check(*x, m=3)
    out = torch.full((3, 50, 10, 64), 7.0, dtype=torch.bfloat16, device="cuda")
    z = binding.rotary_forward(q, k, qw, kw, q_out=out[:, :, :6], k_out=out[:, :, 6:8])
    assert torch.equal(z[0], y[0]) and torch.equal(z[1], y[1]) and (out[:, :, 8:] == 7).all()
    z = binding.rotary_backward(dq, dk, q, k, qw, kw, q_out=out[:, :, :6], k_out=out[:, :, 6:8])
    assert torch.equal(z[0], dx[0]) and torch.equal(z[1], dx[1]) and (out[:, :, 8:] == 7).all()


def test_heads_before_tokens():
    """[batch][head][token] memory through strides."""
    x = [v.permute(0, 2, 1, 3).contiguous().permute(0, 2, 1, 3) if v.dim() == 4 else v for v in draw(2, 11, 4, 2, 80, "f32")]
    check(*x, m=2, interleaved=True)


@pytest.mark.parametrize("dtype", ["f32", "bf16"])
def test_in_place(dtype):
    q, k, qw, kw, dq, dk = draw(2, 40, 4, 2, 96, dtype, packed=True)
    y = binding.rotary_forward(q, k, qw, kw)
    a, b = q.clone(), k.clone()
    binding.rotary_forward(a, b, qw, kw, q_out=a, k_out=b)
    assert torch.equal(a, y[0]) and torch.equal(b, y[1])
    dx = binding.rotary_backward(dq, dk, q, k, qw, kw)
    for first in (True, False):            # over the gradients, over the inputs
        a, b = (dq.clone(), dk.clone()) if first else (q.clone(), k.clone())
        if first:
            binding.rotary_backward(a, b, q, k, qw, kw, q_out=a, k_out=b)
        else:
            binding.rotary_backward(dq, dk, a, b, qw, kw, q_out=a, k_out=b)
        assert torch.equal(a, dx[0]) and torch.equal(b, dx[1])


def test_without_weights_or_keys():
    q, k, qw, kw, dq, dk = draw(2, 13, 3, 2, 48, "f32")
    check(q, k, None, None, dq, dk, m=2)
    y, none = binding.rotary_forward(q, None, qw)
    assert none is None and torch.equal(y, binding.rotary_forward(q, k, qw, kw)[0])
    dw = torch.empty(2, 48, device="cuda")
    both = torch.empty(2, 2, 48, device="cuda")
    dx = binding.rotary_backward(dq, dk, q, k, qw, kw, dq_weight=both[0], dk_weight=both[1])
    got, none = binding.rotary_backward(dq, None, q, None, qw, dq_weight=dw)
    assert none is None and torch.equal(got, dx[0]) and torch.equal(dw, both[0])
    binding.rotary_backward(dq, dk, q, k, qw, kw, dk_weight=dw)
    assert torch.equal(dw, both[1])


def test_zero_and_large_heads():
    q, k, qw, kw, dq, dk = draw(1, 6, 2, 1, 64, "f32")
    q[0, 0] = 0.0                          # no size at all: zeros, and a gradient of 1 / sqrt(eps)
    q[0, 1] *= 1e-18
    q[0, 2] *= 1e15
    k[0, 3, 0, :] = 1e18                   # a square beyond 32 bits' range times 64 stays within it
    check(q, k, qw, kw, dq, dk)


def test_weights_inside_a_flat_vector():
    """Parameters start anywhere a float may."""
    q, k, _, _, dq, dk = draw(2, 5, 2, 1, 64)
    flat = 1 + 0.1 * torch.randn(300, device="cuda")
    check(q, k, flat[3:67], flat[101:165], dq, dk)


def test_gradients_against_differences():
    """A second check of dx and dw, without the formula: central differences of the forward pass in 32 bits.  With steps of
    2^-6 they are within h^2 / 6 of the third derivative (of size 1 here) and 2^-24 / h of rounding, times 200 terms."""
    q, k, qw, kw, dq, dk = draw(1, 2, 2, 1, 16, "f32")
    dw = torch.empty(2, 1, 16, device="cuda")
    got = binding.rotary_backward(dq, dk, q, k, qw, kw, dq_weight=dw[0], dk_weight=dw[1])
    def value():
        y = binding.rotary_forward(q, k, qw, kw)
        return float((y[0].double() * dq.double()).sum() + (y[1].double() * dk.double()).sum())
    step = 2.0 ** -6
    for grad, leaf in ((got[0], q), (got[1], k), (dw[0][0], qw), (dw[1][0], kw)):
        flat, g = leaf.view(-1), grad.reshape(-1)
        for i in range(0, flat.numel(), 5):
            old = float(flat[i])
            flat[i] = old + step
            up = value()
            flat[i] = old - step
            down = value()
            flat[i] = old
            assert abs((up - down) / (2 * step) - float(g[i])) <= 5e-3 * max(1.0, float(grad.abs().max()))


def test_nothing_to_do():
    w = torch.ones(64, device="cuda")
    for b, t, h, hk in ((0, 5, 2, 1), (2, 0, 2, 1), (2, 5, 0, 0), (2, 5, 0, 3), (2, 5, 3, 0)):
        x = draw(b, t, h, hk, 64)
        y = binding.rotary_forward(*x[:4])
        assert y[0].shape == x[0].shape and y[1].shape == x[1].shape
        if b:
            dw = torch.full((2, 2, 64), float("nan"), device="cuda")
            binding.rotary_backward(x[4], x[5], x[0], x[1], w, w, dq_weight=dw[0], dk_weight=dw[1])
            assert (dw[0] == 0).all() if not (t and h) else torch.isfinite(dw[0]).all()
            assert (dw[1] == 0).all() if not (t and hk) else torch.isfinite(dw[1]).all()


def test_strides_beyond_32_bits():
    """Sequences that lie 2^31 elements apart."""
    q, k, qw, kw, dq, dk = draw(2, 3, 2, 1, 64)
    big = torch.empty(2 ** 31 + 4096, dtype=torch.bfloat16, device="cuda")
    far = big.as_strided((2, 3, 2, 64), (2 ** 31, 128, 64, 1))
    far.copy_(q)
    y = binding.rotary_forward(far, k, qw, kw)
    assert torch.equal(y[0], binding.rotary_forward(q, k, qw, kw)[0])


def test_refusals():
    q, k, qw, kw, dq, dk = draw(4, 6, 2, 2, 64)
    for bad in (dict(q=q.half()), dict(k=k.float()), dict(k=k[:2]), dict(k=k[:, :3]), dict(k=k[..., :32]), dict(q=q[0]), dict(q_weight=qw[:32]), dict(q_weight=qw.bfloat16()),
                dict(positions=torch.zeros(6, device="cuda")), dict(positions=torch.zeros(5, dtype=torch.int64, device="cuda")),
                dict(positions=torch.zeros(6, 4, dtype=torch.int64, device="cuda").t()), dict(lens=torch.zeros(4, dtype=torch.int64, device="cuda")),
                dict(lens=torch.zeros(3, dtype=torch.int32, device="cuda")), dict(q_out=k[:2]), dict(q=q.transpose(2, 3).contiguous().transpose(2, 3)),
                dict(k_weight=kw.cpu())):
        kw2 = dict(q=q, k=k, q_weight=qw, k_weight=kw) | bad
        with pytest.raises(ValueError):
            binding.rotary_forward(**kw2)
    for bad in (dict(rotary_dim=4), dict(rotary_dim=72), dict(rotary_dim=-8), dict(eps=-1.0), dict(eps=float("nan")), dict(base=0.0), dict(base=float("inf"))):
        with pytest.raises(binding.CdgrabError):
            binding.rotary_forward(q, k, qw, kw, **bad)
    for d in (4, 12, 264):
        with pytest.raises(binding.CdgrabError):
            binding.rotary_forward(*(torch.zeros(1, 2, 1, d, device="cuda") for _ in range(2)))
    wide = torch.zeros(4, 6, 2, 68, dtype=torch.bfloat16, device="cuda")
    for bad in (wide[..., 1:65], wide[..., :64]):           # a start and strides that are no multiples of 16 bytes
        with pytest.raises(binding.CdgrabError):
            binding.rotary_forward(bad, k)
    with pytest.raises(binding.CdgrabError):
        binding.rotary_forward(q[:, :1].expand(4, 6, 2, 64), k)      # tokens on top of each other
    for bad in (dict(dq_weight=torch.empty(3, 64, device="cuda")), dict(dq_weight=torch.empty(4, 32, device="cuda")), dict(dq=dq[:2]), dict(dk=None),
                dict(dq_weight=torch.empty(4, 64, device="cuda"), dk_weight=torch.empty(4, 128, device="cuda")[:, :64])):
        kw2 = dict(dq=dq, dk=dk, q=q, k=k) | bad
        with pytest.raises(ValueError):
            binding.rotary_backward(**kw2)
