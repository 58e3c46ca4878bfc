"""What the binding of embedding, dropout and the rotation does with streams and graphs, and a run of them together with
attention as a model uses them."""
import pytest
import torch

import model_operators_ref as ref
from paper_2302_00845_b200 import binding
from test_operators_binding_gpu import late

pytestmark = pytest.mark.gpu


def draws(seed):
    gen = torch.Generator(device="cuda").manual_seed(seed)
    r = lambda *s: torch.randn(*s, generator=gen, device="cuda")  # noqa: E731
    t = lambda v, *s: torch.randint(v, s, generator=gen, device="cuda")  # noqa: E731
    return r, t


def test_inputs_given_up_after_a_call_on_another_stream():
    r, t = draws(3)
    tokens, table, dy = t(5000, 4, 500), r(5000, 264), r(2000, 264)
    want = binding.embedding_forward(tokens, table)
    assert torch.equal(late(lambda s, *a: binding.embedding_forward(*a, stream=s), tokens, table), want)
    buf = torch.empty(4, 5000, 264, device="cuda")
    binding.embedding_backward(dy, tokens, buf)
    other = torch.empty_like(buf)
    late(lambda s, *a: binding.embedding_backward(*a, other, stream=s), dy, tokens)
    assert torch.equal(other, buf)
    x, res, step = r(500, 768), r(500, 768), torch.tensor([7], dtype=torch.int64, device="cuda")
    want = binding.dropout_forward(x, 0.2, 5, 1, step, residual=res)
    assert torch.equal(late(lambda s, a, b, c: binding.dropout_forward(a, 0.2, 5, 1, c, residual=b, stream=s), x, res, step), want)
    want = binding.dropout_backward(x, 0.2, 5, 1, step)
    assert torch.equal(late(lambda s, a, c: binding.dropout_backward(a, 0.2, 5, 1, c, stream=s), x, step), want)
    q, k, dq, dk = (r(4, 300, h, 64).bfloat16() for h in (4, 2, 4, 2))
    qw, kw, pos = r(64), r(64), t(100_000, 4, 300)
    lens = torch.tensor([300, 20, 299, 0], dtype=torch.int32, device="cuda")
    fwd = lambda s, *a: binding.rotary_forward(*a[:4], positions=a[4], lens=a[5], stream=s)  # noqa: E731
    for got, want in zip(late(fwd, q, k, qw, kw, pos, lens), fwd(None, q, k, qw, kw, pos, lens)):
        assert torch.equal(got, want)
    dw, dw2 = torch.empty(2, 2, 64, device="cuda"), torch.empty(2, 2, 64, device="cuda")
    bwd = lambda to: lambda s, *a: binding.rotary_backward(*a[:6], positions=a[6], lens=a[7], dq_weight=to[0], dk_weight=to[1], stream=s)  # noqa: E731
    want = bwd(dw)(None, dq, dk, q, k, qw, kw, pos, lens)
    for got, val in zip(late(bwd(dw2), dq, dk, q, k, qw, kw, pos, lens), want):
        assert torch.equal(got, val)
    assert torch.equal(dw, dw2)


def test_captured_calls_run_on_what_the_buffers_hold():
    r, t = draws(9)
    tokens, table, dy = t(3000, 3, 400), r(3000, 100), r(1200, 100).bfloat16()
    buf, tied = torch.empty(3, 3000, 100, device="cuda"), torch.empty(3, 3000, 100, device="cuda", dtype=torch.bfloat16)
    x, step = r(700, 96), torch.zeros(1, dtype=torch.int64, device="cuda")
    q, k, dq, dk = (r(3, 200, h, 80).bfloat16() for h in (4, 2, 4, 2))
    qw, kw, dw = r(80), r(80), torch.empty(2, 3, 80, device="cuda")

    def calls():
        tied.fill_(0.25)
        out = (binding.embedding_forward(tokens, table), binding.embedding_backward(dy, tokens, buf),
               binding.embedding_backward(dy, tokens, tied, accumulate=True), binding.dropout_forward(x, 0.3, 5, 1, step),
               binding.dropout_backward(x, 0.3, 5, 1, step), dw)
        return out + tuple(binding.rotary_forward(q, k, qw, kw)) + tuple(
            binding.rotary_backward(dq, dk, q, k, qw, kw, dq_weight=dw[0], dk_weight=dw[1]))

    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    with torch.cuda.stream(side):
        calls()
    torch.cuda.synchronize()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        out = calls()
    for n in range(3):
        for v in (table, dy, x, q, k, dq, dk, qw, kw):
            v.copy_(r(*v.shape))
        tokens.copy_(t(3000, 3, 400))
        tokens[n % 3, 100:] = n                    # another length of the longest run each time
        step.fill_(n)
        graph.replay()
        got = [v.clone() for v in out]
        for a, c in zip(got, calls()):
            assert torch.equal(a, c)
        assert binding.operators_status() == binding.OK


def test_two_streams_at_once():
    """Calls that overlap have scratch of their own."""
    r, t = draws(5)
    sets = []
    for _ in range(2):
        tokens, dy = t(50, 2, 3000), r(6000, 256)
        q, k, dq, dk = (r(2, 500, h, 64).bfloat16() for h in (4, 2, 4, 2))
        buf, dw = torch.empty(2, 50, 256, device="cuda"), torch.empty(2, 2, 64, device="cuda")
        sets.append((tokens, dy, q, k, dq, dk, buf, dw))

    def call(z, **kw):
        tokens, dy, q, k, dq, dk, buf, dw = z
        return [binding.embedding_backward(dy, tokens, buf, **kw), *binding.rotary_backward(dq, dk, q, k, dq_weight=dw[0], dk_weight=dw[1], **kw), dw]
    want = [[v.clone() for v in call(z)] for z in sets]
    streams = [torch.cuda.Stream(), torch.cuda.Stream()]
    torch.cuda.synchronize()
    for _ in range(5):
        out = [call(z, stream=s) for z, s in zip(sets, streams)]
        torch.cuda.synchronize()
        for got, val in zip(out, want):
            assert all(torch.equal(a, c) for a, c in zip(got, val))


def test_checks_are_made_for_every_shape():
    """Checks that are kept belong to sizes, strides and types; calls of other ones are checked anew."""
    r, _ = draws(1)
    q, k, w = r(2, 5, 3, 64), r(2, 5, 1, 64), r(64)
    first = binding.rotary_forward(q, k, w, w)
    for _ in range(2):
        with pytest.raises(ValueError):
            binding.rotary_forward(q, k[:, :4], w, w)
        with pytest.raises(ValueError):
            binding.rotary_forward(q, k, w[:32], w)
        with pytest.raises(binding.CdgrabError):
            binding.rotary_forward(q, k, w, w, rotary_dim=12)
        assert all(torch.equal(a, c) for a, c in zip(first, binding.rotary_forward(q, k, w, w)))
    half = binding.rotary_forward(q, k, w, w, rotary_dim=32)
    assert not torch.equal(half[0], first[0])
    assert all(torch.equal(a, c) for a, c in zip(first, binding.rotary_forward(q.clone(), k.clone(), w.clone(), w.clone())))


def test_a_layer_from_tokens_to_gradients():
    """Lookup, norms and rotation, attention, dropout onto the lookup, and back: every worker's gradients against automatic
    differentiation in 64 bits of the same layer with the same mask."""
    m, t, vocab, h, hk, d, p = 3, 65, 40, 4, 2, 32, 0.25
    width = h * d
    r, rint = draws(11)
    tokens = rint(vocab, m, t)
    table, w_qkv = r(vocab, width), r((h + 2 * hk) * d, width) * width ** -0.5
    qw, kw = 1 + 0.1 * r(d), 1 + 0.1 * r(d)
    dy = r(m * t, width)
    # forward, 16-bit products, the residual stream in 32
    x = binding.embedding_forward(tokens, table, 2.0)
    qkv = (x.bfloat16() @ w_qkv.bfloat16().T).view(m, t, h + 2 * hk, d)
    q, k, v = qkv[:, :, :h], qkv[:, :, h:h + hk], qkv[:, :, h + hk:]
    q2, k2 = binding.rotary_forward(q, k, qw, kw)
    o, lse = binding.attention_forward(q2, k2, v, causal=True)
    y = binding.dropout_forward(o.view(m * t, width), p, 7, 3, 1, residual=x)
    # and back
    do = binding.dropout_backward(dy, p, 7, 3, 1, dtype=torch.bfloat16)
    dqkv, grads = torch.empty_like(qkv), torch.full((m, vocab * width + 2 * d), float("nan"), device="cuda")
    dq, dk = torch.empty_like(q, memory_format=torch.contiguous_format), torch.empty_like(k, memory_format=torch.contiguous_format)
    binding.attention_backward(do.view(m, t, h, d), q2, k2, v, o, lse, causal=True, dq=dq, dk=dk, dv=dqkv[:, :, h + hk:])
    binding.rotary_backward(dq, dk, q, k, qw, kw, dq_weight=grads[:, -2 * d:-d], dk_weight=grads[:, -d:], q_out=dqkv[:, :, :h], k_out=dqkv[:, :, h:h + hk])
    dx = dy + (dqkv.view(m * t, -1) @ w_qkv.bfloat16()).float()
    dtable = grads[:, :vocab * width].view(m, vocab, width)
    binding.embedding_backward(dx, tokens, dtable, 2.0)
    assert binding.operators_status() == binding.OK
    keep = torch.from_numpy(ref.keep(range(m * t * width), p, 7, 3, 1)).view(m, t, width).cuda()
    limit = int(65536 * p + 0.5)
    for i in range(m):
        tab, a, b = (z.double().requires_grad_(True) for z in (table, qw, kw))
        xs = 2.0 * tab[tokens[i]]
        z = (xs @ w_qkv.double().T).view(t, h + 2 * hk, d)
        def turned(u, w):
            n = u / torch.sqrt(u.square().mean(-1, keepdim=True) + 1e-6) * w
            angle = torch.arange(t, device="cuda").double()[:, None] * 10000.0 ** (-2.0 * torch.arange(d // 2, device="cuda").double() / d)
            c, s = torch.cos(angle)[:, None], torch.sin(angle)[:, None]
            e, f = n[..., :d // 2], n[..., d // 2:]
            return torch.cat((e * c - f * s, e * s + f * c), -1)
        qq, kk, vv = turned(z[:, :h], a), turned(z[:, h:h + hk], b).repeat_interleave(h // hk, 1), z[:, h + hk:].repeat_interleave(h // hk, 1)
        s = torch.einsum("ihd,jhd->hij", qq, kk) * d ** -0.5
        s = s.masked_fill(torch.triu(torch.ones(t, t, dtype=torch.bool, device="cuda"), 1), float("-inf"))
        oo = torch.einsum("hij,jhd->ihd", torch.softmax(s, -1), vv).reshape(t, width)
        out = xs + torch.where(keep[i], oo * (65536 / (65536 - limit)), 0.0)
        out.backward(dy.view(m, t, width)[i].double())
        # products with operands of 16 bits, each rounded by up to 2^-8 and mostly independently, about eight deep: 1 % of the norm
        for got, want in ((y.view(m, t, width)[i], out.detach()), (dtable[i], tab.grad), (grads[i, -2 * d:-d], a.grad), (grads[i, -d:], b.grad)):
            assert float((got.double() - want).norm()) <= 3e-2 * float(want.norm())


def test_other_device_is_refused():
    with pytest.raises(ValueError):
        binding.dropout_forward(torch.zeros(4, 8), 0.1, 0)
    with pytest.raises(ValueError):
        binding.embedding_backward(torch.zeros(4, 8, device="cuda"), torch.zeros(4, dtype=torch.int64), torch.zeros(9, 8, device="cuda"))
    with pytest.raises(ValueError):
        binding.rotary_forward(torch.zeros(1, 2, 1, 8, device="cuda"), torch.zeros(1, 2, 1, 8))


def test_numbers_beyond_their_bits_are_refused():
    """Not taken modulo a power of two, as the boundary would."""
    t, table = torch.zeros(4, dtype=torch.int64, device="cuda"), torch.zeros(9, 8, device="cuda")
    for padding in (2 ** 63, -2 ** 63 - 1, 2 ** 64 - 1):
        with pytest.raises(ValueError):
            binding.embedding_forward(t, table, padding=padding)
        with pytest.raises(ValueError):
            binding.embedding_backward(torch.zeros(4, 8, device="cuda"), t, table, padding=padding)
    q = torch.zeros(1, 2, 1, 64, device="cuda")
    for rotary_dim in (2 ** 32 + 64, -2 ** 32):
        with pytest.raises(ValueError):
            binding.rotary_forward(q, q, rotary_dim=rotary_dim)


def test_keys_shared_over_the_batch():
    """Inputs may be broadcast, outputs not."""
    r, _ = draws(2)
    q, k = r(3, 20, 4, 64), r(1, 20, 2, 64)
    shared = k.expand(3, 20, 2, 64)
    got, want = binding.rotary_forward(q, shared), binding.rotary_forward(q, shared.contiguous())
    assert all(torch.equal(a, c) for a, c in zip(got, want))
    dq, dk, dw, dw2 = r(3, 20, 4, 64), r(3, 20, 2, 64), torch.empty(3, 64, device="cuda"), torch.empty(3, 64, device="cuda")
    got = binding.rotary_backward(dq, dk, q, shared, dk_weight=dw)
    want = binding.rotary_backward(dq, dk, q, shared.contiguous(), dk_weight=dw2)
    assert all(torch.equal(a, c) for a, c in zip(got, want)) and torch.equal(dw, dw2)
    with pytest.raises(binding.CdgrabError):
        binding.rotary_forward(q, shared, k_out=torch.empty_like(k).expand(3, 20, 2, 64))
