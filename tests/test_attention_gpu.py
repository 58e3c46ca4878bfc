"""Attention, forward and backward, against the formulas in 64 bits."""
import math

import pytest
import torch

import operators_ref as ref
from paper_2302_00845_b200 import binding

pytestmark = pytest.mark.gpu


def draw(b, tq, tk, h, hk, d, seed=0, packed=False):
    g = torch.Generator(device="cuda").manual_seed(seed * 7 + b + 3 * tq + 5 * tk + d)
    r = lambda *s: torch.randn(*s, generator=g, device="cuda").to(torch.bfloat16)  # noqa: E731
    if packed:
        qkv = r(b, tq, h + 2 * hk, d)
        return qkv[:, :, :h], qkv[:, :, h:h + hk], qkv[:, :, h + hk:], r(b, tq, h, d)
    return r(b, tq, h, d), r(b, tk, hk, d), r(b, tk, hk, d), r(b, tq, h, d)


def check(q, k, v, do, causal=False, scale=None, q_lens=None, kv_lens=None, **kw):
    lens = [None if t is None else torch.tensor(t, dtype=torch.int32, device="cuda") for t in (q_lens, kv_lens)]
    o, lse = binding.attention_forward(q, k, v, causal, scale, *lens, out=kw.get("out"))
    grads = binding.attention_backward(do, q, k, v, o, lse, causal, scale, *lens, dq=kw.get("dq"), dk=kw.get("dk"),
                                       dv=kw.get("dv"))
    assert binding.operators_status() == binding.OK
    want = ref.attention(q, k, v, causal, q.shape[3] ** -0.5 if scale is None else scale, q_lens, kv_lens, do)
    for name, got in zip(("o", "lse", "dq", "dk", "dv"), (o, lse) + tuple(grads)):
        ref.assert_within(got, *want[name], name)
    return (o, lse) + tuple(grads)


@pytest.mark.parametrize("causal", [False, True])
@pytest.mark.parametrize("t", [1, 2, 7, 16, 31, 64, 65, 127, 128, 129, 255, 256, 257, 385, 640])
def test_lengths(t, causal):
    check(*draw(2, t, t, 2, 2, 64), causal=causal)


@pytest.mark.parametrize("causal", [False, True])
@pytest.mark.parametrize("d", [8, 16, 24, 32, 40, 56, 64, 72, 80, 96, 104, 120, 128])
def test_head_dims(d, causal):
    check(*draw(1, 200, 200, 2, 1, d), causal=causal)


@pytest.mark.parametrize("causal", [False, True])
@pytest.mark.parametrize("tq,tk", [(1, 300), (300, 1), (130, 520), (520, 130), (257, 256), (128, 129), (1, 1), (3, 1000)])
@pytest.mark.parametrize("d", [64, 128])
def test_unequal_lengths(tq, tk, d, causal):
    """Causal with more queries than keys leaves the first rows empty."""
    out = check(*draw(2, tq, tk, 2, 2, d), causal=causal)
    if causal and tq > tk:
        assert (out[0][:, :tq - tk] == 0).all() and (out[1][:, :, :tq - tk] == -math.inf).all()
        assert (out[2][:, :tq - tk] == 0).all()


@pytest.mark.parametrize("h,hk", [(1, 1), (3, 3), (4, 1), (6, 2), (12, 12), (8, 4)])
def test_shared_heads(h, hk):
    check(*draw(2, 150, 150, h, hk, 64), causal=True)


@pytest.mark.parametrize("d", [32, 64, 128])
def test_packed_projection_and_packed_gradient(d):
    b, t, h, hk = 3, 201, 4, 2
    q, k, v, do = draw(b, t, t, h, hk, d, packed=True)
    grad = torch.full((b, t, h + 2 * hk + 1, d), 3.0, dtype=torch.bfloat16, device="cuda")
    out = torch.full((b, t, h + 1, d), 3.0, dtype=torch.bfloat16, device="cuda")
    check(q, k, v, do, causal=True, out=out[:, :, :h], dq=grad[:, :, :h], dk=grad[:, :, h:h + hk],
          dv=grad[:, :, h + hk:h + 2 * hk])
    assert (grad[:, :, -1] == 3).all() and (out[:, :, -1] == 3).all()


def test_other_orders():
    """[batch][head][token] tensors, and a batch of one that is a slice of a longer buffer."""
    q, k, v, do = (t.permute(0, 2, 1, 3).contiguous().permute(0, 2, 1, 3) for t in draw(2, 140, 140, 3, 3, 64))
    check(q, k, v, do, causal=True)
    q, k, v, do = draw(4, 140, 140, 3, 3, 64)
    check(q[2:3, 5:], k[2:3], v[2:3, :], do[2:3, 5:], causal=True)
    k1 = k[:1].expand(4, -1, -1, -1)          # keys shared by the batch
    check(q, k1, v, do)


@pytest.mark.parametrize("causal", [False, True])
@pytest.mark.parametrize("d", [64, 128])
def test_lengths_in_use(d, causal):
    """Padded sequences: empty ones, one token, ends inside and on the edge of a tile; NaN and infinity past the ends."""
    tq, tk = 300, 333
    ql, kl = [300, 0, 1, 128, 129, 200, 17, 256], [333, 333, 1, 0, 128, 256, 301, 255]
    q, k, v, do = draw(len(ql), tq, tk, 2, 1, d)
    for b, (a, c) in enumerate(zip(ql, kl)):
        q[b, a:], do[b, a:] = math.nan, math.inf
        k[b, c:], v[b, c:] = math.inf, math.nan
    out = check(q, k, v, do, causal=causal, q_lens=ql, kv_lens=kl)
    for b, (a, c) in enumerate(zip(ql, kl)):
        assert (out[0][b, a:] == 0).all() and (out[2][b, a:] == 0).all()
        assert (out[3][b, c:] == 0).all() and (out[4][b, c:] == 0).all()


@pytest.mark.parametrize("causal", [False, True])
@pytest.mark.parametrize("tq,tk,h,hk,d", [(2500, 2500, 1, 1, 64), (2300, 2300, 4, 1, 128), (64, 4100, 2, 1, 128), (4100, 100, 1, 1, 64),
                                          (1, 3000, 2, 2, 64)])
def test_long_and_few(tq, tk, h, hk, d, causal):
    """Few tiles of rows and a long other axis: the loop is dealt out over several blocks and joined."""
    check(*draw(1, tq, tk, h, hk, d), causal=causal)


def test_long_and_few_padded():
    q, k, v, do = draw(2, 1500, 1700, 2, 1, 64)
    ql, kl = [1500, 130], [700, 1653]
    for b in range(2):
        q[b, ql[b]:], do[b, ql[b]:], k[b, kl[b]:], v[b, kl[b]:] = math.nan, math.nan, math.inf, math.nan
    check(q, k, v, do, causal=True, q_lens=ql, kv_lens=kl)
    check(q, k, v, do, q_lens=ql, kv_lens=kl)


@pytest.mark.parametrize("causal", [False, True])
@pytest.mark.parametrize("tq,tk,d", [(520, 520, 64), (400, 700, 128), (700, 300, 64)])
def test_more_blocks_than_multiprocessors(tq, tk, d, causal):
    """Every SM takes several blocks of rows, of unequal lengths and some empty, one after another."""
    b, h = 9, 12
    ql, kl = [tq - 71 * i for i in range(b)], [tk - 30 * ((3 * i) % b) for i in range(b)]
    ql = [max(0, t) for t in ql]
    args = draw(b, tq, tk, h, h // 2, d)
    check(*args, causal=causal)
    check(*args, causal=causal, q_lens=ql, kv_lens=kl)


def test_only_some_lengths_given():
    q, k, v, do = draw(2, 100, 260, 2, 2, 64)
    check(q, k, v, do, kv_lens=[70, 260])
    check(q, k, v, do, q_lens=[70, 100], causal=True)


def test_lengths_out_of_range_are_clamped():
    q, k, v, do = draw(2, 100, 100, 1, 1, 64)
    a = check(q, k, v, do)
    lens = torch.tensor([500, -3], dtype=torch.int32, device="cuda")
    o, _ = binding.attention_forward(q, k, v, kv_lens=lens)
    assert torch.equal(o[0], a[0][0]) and (o[1] == 0).all()


@pytest.mark.parametrize("scale", [0.0, 0.02, 1.0, -0.3])
def test_scales(scale):
    check(*draw(1, 160, 160, 2, 2, 64), scale=scale, causal=True)


def test_large_scores():
    """Scores of several hundred: one key takes nearly all of each row, the maximum moves by large steps."""
    q, k, v, do = draw(1, 300, 300, 1, 1, 64)
    q, k = q * 8, k * 8
    o, lse = binding.attention_forward(q, k, v, causal=True)
    want = ref.attention(q, k, v, True, 0.125)
    ref.assert_within(o, *want["o"], "o")
    ref.assert_within(lse, *want["lse"], "lse")


def test_rising_and_falling_scores():
    """Keys in order of their score, up and down: the running maximum changes at every key or only once."""
    q, k, v, do = draw(1, 140, 500, 1, 1, 64)
    q = torch.full_like(q, 1.0)
    ramp = torch.linspace(-8, 8, 500, device="cuda").to(torch.bfloat16)
    for r in (ramp, ramp.flip(0)):
        check(q, r[None, :, None, None].expand(1, 500, 1, 64).contiguous(), v, do)


def test_nothing_to_do():
    q, k, v, do = draw(2, 5, 0, 2, 2, 64)
    o, lse = binding.attention_forward(q, k, v)
    assert (o == 0).all() and (lse == -math.inf).all()
    dq, dk, dv = binding.attention_backward(do, q, k, v, o, lse)
    assert (dq == 0).all() and dk.shape == k.shape
    q, k, v, do = draw(2, 0, 5, 2, 2, 64)
    o, lse = binding.attention_forward(q, k, v)
    dq, dk, dv = binding.attention_backward(do, q, k, v, o, lse)
    assert (dk == 0).all() and (dv == 0).all()
    q, k, v, do = draw(0, 5, 5, 2, 2, 64)
    o, lse = binding.attention_forward(q, k, v)
    binding.attention_backward(do, q, k, v, o, lse)


def test_offsets_past_32_bits():
    """Token strides that put the last sequence beyond 2^31 elements."""
    b, t, h, d = 3, 70, 1, 64
    base = torch.empty(2 * (1 << 30) + (1 << 20), dtype=torch.bfloat16, device="cuda")
    q, k, v, do = draw(b, t, t, h, h, d)
    far = base.as_strided((b, t, h, d), (1 << 30, 64, 64, 1))
    for src in (q, k, v, do):
        far.copy_(src)
        args = [far if s is src else s for s in (q, k, v, do)]
        check(*args, causal=True)
    o = binding.attention_forward(q, k, v, True, out=far)[0]
    assert torch.equal(o, binding.attention_forward(q, k, v, True)[0])


def test_gradient_against_differences():
    """Central differences of the definition in 64 bits along random directions; the kernel's gradient may be
    off by its own bound along the same direction."""
    b, t, h, hk, d = 1, 70, 2, 1, 32
    q, k, v, do = draw(b, t, t, h, hk, d, seed=3)
    o, lse = binding.attention_forward(q, k, v, True)
    grads = binding.attention_backward(do, q, k, v, o, lse, True)
    want = ref.attention(q, k, v, True, d ** -0.5, do=do)
    gen = torch.Generator(device="cuda").manual_seed(1)

    def loss(*qkv):
        return float((ref.attention(*qkv, True, d ** -0.5)["o"][0] * do.double()).sum())

    step = 1e-4
    for i, (grad, name) in enumerate(zip(grads, ("dq", "dk", "dv"))):
        way = torch.randn(grad.shape, generator=gen, device="cuda", dtype=torch.float64)
        at = [t.double() for t in (q, k, v)]
        up, dn = list(at), list(at)
        up[i], dn[i] = at[i] + step * way, at[i] - step * way
        slope = (loss(*up) - loss(*dn)) / (2 * step)
        assert abs(slope - float((grad.double() * way).sum())) <= float((want[name][1] * way.abs()).sum()) + 1e-4 * abs(slope)


def test_same_bits_every_time_and_on_another_stream():
    q, k, v, do = draw(2, 500, 500, 4, 2, 64)
    first = check(q, k, v, do, causal=True)
    s = torch.cuda.Stream()
    s.wait_stream(torch.cuda.current_stream())
    for _ in range(3):
        o, lse = binding.attention_forward(q, k, v, True, stream=s)
        got = binding.attention_backward(do, q, k, v, o, lse, True, stream=s)
        s.synchronize()
        for a, b in zip((o, lse) + tuple(got), first):
            assert torch.equal(a, b)


def test_refusals():
    q, k, v, do = draw(2, 20, 20, 4, 2, 64)
    o, lse = binding.attention_forward(q, k, v)
    for bad in (lambda: binding.attention_forward(q.float(), k, v),
                lambda: binding.attention_forward(q, k[:, :10], v),
                lambda: binding.attention_forward(q, k, v[:, :, :, :32]),
                lambda: binding.attention_forward(q.transpose(2, 3), k, v),
                lambda: binding.attention_forward(q, k, v, q_lens=torch.zeros(2, device="cuda")),
                lambda: binding.attention_forward(q, k, v, kv_lens=torch.zeros(3, dtype=torch.int32, device="cuda")),
                lambda: binding.attention_forward(q, k.cpu(), v),
                lambda: binding.attention_backward(do[:, :10], q, k, v, o, lse),
                lambda: binding.attention_backward(do, q, k, v, o, lse[:, :2])):
        with pytest.raises(ValueError):
            bad()
    odd = torch.zeros(2, 20, 4, 20, dtype=torch.bfloat16, device="cuda")       # head_dim 20
    wide = torch.zeros(2, 20, 4, 136, dtype=torch.bfloat16, device="cuda")     # head_dim 136
    off = torch.zeros(2, 20, 4, 72, dtype=torch.bfloat16, device="cuda")[..., 4:68]   # 8 bytes off
    step = torch.zeros(2, 20, 4, 68, dtype=torch.bfloat16, device="cuda")[..., :64]   # strides of 68
    for t in (odd, wide, off, step):
        with pytest.raises(binding.CdgrabError):
            binding.attention_forward(t, t, t)
    with pytest.raises(binding.CdgrabError):
        binding.attention_forward(q[:, :, :3], k, v)        # 3 heads over 2
    with pytest.raises(binding.CdgrabError):
        binding.attention_forward(q, k, v, scale=math.nan)
    with pytest.raises(binding.CdgrabError):                # outputs of a batch on top of each other
        binding.attention_forward(q, k, v, out=torch.empty_like(q[:1]).expand(2, -1, -1, -1))
