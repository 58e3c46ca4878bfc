"""The norms and the rotation over the whole range of their types: sizes whose squares or products leave 32 bits while the
results do not."""
import pytest
import torch

import model_operators_ref as ref
from operators_ref import assert_within
from paper_2302_00845_b200 import binding
from test_rotary_gpu import draw

pytestmark = pytest.mark.gpu


def sized(x, *factors):
    """Token i's heads times factors[i]."""
    y = x.clone()
    for i, f in enumerate(factors):
        y[:, i] = (y[:, i].double() * f).to(x.dtype)
    return y


@pytest.mark.parametrize("dtype", ["f32", "bf16"])
@pytest.mark.parametrize("interleaved", [False, True])
@pytest.mark.parametrize("eps", [0.0, 1e-6])
def test_heads_of_any_size(dtype, interleaved, eps):
    """Squares beyond 32 bits on either side: without epsilon each head comes out as it would at size one."""
    sizes = (1.0, 1e15, 1e19, 1e25, 1e36) + ((1e-15, 1e-19, 1e-22, 1e-30) if eps == 0.0 else ())
    q, k, qw, kw, dq, dk = draw(2, len(sizes), 3, 2, 80, dtype)
    q, k = sized(q, *sizes), sized(k, *sizes[::-1])
    for got, x, w, name in zip(binding.rotary_forward(q, k, qw, kw, interleaved=interleaved, eps=eps), (q, k), (qw, kw), "qk"):
        assert_within(got, *ref.rotary(x, w, None, 10000.0, 80, interleaved, eps, None), name)


# of the input and of the gradient: their product, its sum, the squares, or the third power of the norm leave 32 bits
@pytest.mark.parametrize("size,gradient,eps", [(1.0, 1.0, 0.0), (1e15, 1e25, 1e-6), (1e18, 1e20, 1e-6), (1e15, 1e-12, 1e-6), (1e25, 1e3, 1e-6),
                                               (1e25, 1e30, 0.0), (1e-20, 1e-28, 0.0), (1e-12, 1e-15, 0.0), (1e-18, 1e-5, 0.0), (1e-3, 1e34, 1e-6),
                                               (1e-8, 1e-25, 1e-12), (0.0, 1e-10, 1e-6), (1e-25, 1e8, 1e-6)])
@pytest.mark.parametrize("dtype,interleaved,d", [("f32", False, 64), ("f32", True, 80), ("bf16", False, 128), ("bf16", True, 40)])
def test_gradients_of_any_size(size, gradient, eps, dtype, interleaved, d):
    m = 2
    q, k, qw, kw, dq, dk = draw(m, 5, 3, 2, d, dtype)
    one = (1.0, 1.0, 1.0, 1.0)
    # one token of each worker, among others of ordinary size; the weights' sums get them apart
    q, k = sized(q, *one, size), sized(k, *one, size)
    dq, dk = sized(dq, *one, gradient), sized(dk, *one, gradient)
    buf = torch.full((m, 2 * d), float("nan"), device="cuda")
    for part in (slice(None), slice(4, 5)):
        x = [v[:, part] for v in (dq, dk, q, k)]
        pos = torch.arange(5, device="cuda")[part]
        got = binding.rotary_backward(*x, qw, kw, dq_weight=buf[:, :d], dk_weight=buf[:, d:], positions=pos, eps=eps, interleaved=interleaved)
        for i, w in enumerate((qw, kw)):
            (dx, bound), (dw, wbound) = ref.rotary(x[2 + i], w, pos, 10000.0, d, interleaved, eps, None, dy=x[i], m=m, grad_dtype=torch.float32)
            assert_within(got[i], dx, bound, "d" + "qk"[i])
            assert_within(buf[:, i * d:(i + 1) * d], dw, wbound, "dw " + "qk"[i])


def test_a_heads_results_do_not_depend_on_its_neighbours():
    """Heads of other sizes beside it, which take more care, leave a head's bits as they are."""
    q, k, qw, kw, dq, dk = draw(1, 9, 4, 2, 64)
    a = binding.rotary_forward(q, k, qw, kw) + binding.rotary_backward(dq, dk, q, k, qw, kw)
    q2, k2 = q.clone(), k.clone()
    q2[:, 1::2] *= 1e30
    k2[:, :, 1] *= 1e-30
    b = binding.rotary_forward(q2, k2, qw, kw) + binding.rotary_backward(dq, dk, q2, k2, qw, kw)
    for x, y in zip(a[::2], b[::2]):
        assert torch.equal(x[:, ::2], y[:, ::2])
    for x, y in zip(a[1::2], b[1::2]):
        assert torch.equal(x[:, :, 0], y[:, :, 0])


@pytest.mark.parametrize("dtype,d,h,hk,interleaved", [("bf16", 8, 5, 2, False), ("bf16", 64, 40, 3, True), ("f32", 80, 5, 3, False), ("f32", 256, 2, 1, True),
                                                      ("bf16", 128, 16, 4, False), ("bf16", 248, 3, 2, False)])
@pytest.mark.parametrize("t", [9, 900])
def test_sizes_scattered_over_heads(dtype, d, h, hk, interleaved, t):
    """Heads of ordinary size first, then some of others among them, in sequences of several lengths; in place the same bits."""
    m = 2
    q, k, qw, kw, dq, dk = draw(m, t, h, hk, d, dtype)
    g = torch.Generator(device="cuda").manual_seed(t + d)
    for x, dx in ((q, dq), (k, dk)):
        size = torch.tensor([1.0, 1.0, 1.0, 1e-22, 1e24, 1e5], device="cuda")[torch.randint(0, 6, x.shape[:3], generator=g, device="cuda")]
        size[:, :t // 2] = 1.0
        x.copy_((x.double() * size[..., None]).to(x.dtype))
        dx.copy_((dx.double() * size[..., None].clamp(max=1e20)).to(x.dtype))
    lens = torch.tensor([t, t - 3], dtype=torch.int32, device="cuda")
    opts = dict(eps=0.0, lens=lens, interleaved=interleaved)
    y = binding.rotary_forward(q, k, qw, kw, **opts)
    buf = torch.full((m, 2 * d), float("nan"), device="cuda")
    dx = binding.rotary_backward(dq, dk, q, k, qw, kw, dq_weight=buf[:, :d], dk_weight=buf[:, d:], **opts)
    for i, (x, w, gr) in enumerate(((q, qw, dq), (k, kw, dk))):
        args = (x, w, None, 10000.0, d, interleaved, 0.0, lens)
        assert_within(y[i], *ref.rotary(*args), "qk"[i])
        (val, bound), (dw, wbound) = ref.rotary(*args, dy=gr, m=m, grad_dtype=torch.float32)
        assert_within(dx[i], val, bound, "d" + "qk"[i])
        assert_within(buf[:, i * d:(i + 1) * d], dw, wbound, "dw " + "qk"[i])
    a, b = q.clone(), k.clone()
    binding.rotary_forward(a, b, qw, kw, q_out=a, k_out=b, **opts)
    assert torch.equal(a, y[0]) and torch.equal(b, y[1])
    again = torch.empty_like(buf)
    for first in (True, False):            # over the gradients, over the inputs
        a, b = (dq.clone(), dk.clone()) if first else (q.clone(), k.clone())
        binding.rotary_backward(*((a, b, q, k) if first else (dq, dk, a, b)), qw, kw, dq_weight=again[:, :d], dk_weight=again[:, d:], q_out=a, k_out=b, **opts)
        assert torch.equal(a, dx[0]) and torch.equal(b, dx[1]) and torch.equal(again, buf)
