"""What the training operators' binding does with its arguments: sizes beyond 32 bits, tensors of other streams."""
import pytest
import torch

from paper_2302_00845_b200 import binding

pytestmark = pytest.mark.gpu


def test_numbers_beyond_32_bits_are_refused():
    """Not taken modulo 2^32, as the boundary would."""
    g = torch.randn(8, 16, device="cuda")
    for steps in (2 ** 32 + 5, -2 ** 32 + 5):
        with pytest.raises(ValueError):
            binding.orthogonalise(g, steps=steps)
    wide = torch.zeros(1, 2 ** 32 + 64, dtype=torch.bfloat16, device="cuda")     # 8 GB
    with pytest.raises(ValueError):
        binding.orthogonalise(wide, out=wide)
    stats = torch.zeros(1, device="cuda")
    with pytest.raises(ValueError):
        binding.layer_norm_forward(wide, out=wide)
    with pytest.raises(ValueError):
        binding.layer_norm_backward(wide, wide, None, stats, stats, dx=wide)


def late(call, *tensors):
    """call(stream, *copies) on a stream that has 20 ms of other work to do first, with copies of the tensors that are
    given up, and their memory asked for again and overwritten, before it gets there."""
    copies = [t.clone() for t in tensors]
    s = torch.cuda.Stream()
    s.wait_stream(torch.cuda.current_stream())
    with torch.cuda.stream(s):
        torch.cuda._sleep(40_000_000)
    out = call(s, *copies)
    del copies
    again = [torch.full_like(t, 7) for t in tensors for _ in range(3)]
    torch.cuda.synchronize()
    del again
    assert binding.operators_status() == binding.OK
    return out


def test_inputs_given_up_after_a_call_on_another_stream():
    gen = torch.Generator(device="cuda").manual_seed(3)
    r = lambda *s: torch.randn(*s, generator=gen, device="cuda")  # noqa: E731
    x, dy, w, b = r(512, 1000), r(512, 1000), r(1000), r(1000)
    want = binding.layer_norm_forward(x, w, b)
    for got, val in zip(late(lambda s, *t: binding.layer_norm_forward(*t, stream=s), x, w, b), want):
        assert torch.equal(got, val)
    grads = torch.empty(4, 1000, device="cuda")
    dx = binding.layer_norm_backward(dy, x, w, *want[1:], grads)
    grads2 = torch.empty_like(grads)
    assert torch.equal(late(lambda s, *t: binding.layer_norm_backward(*t, grads2, stream=s), dy, x, w, *want[1:]), dx)
    assert torch.equal(grads2, grads)
    q, k, v, do = (r(2, 600, h, 64).bfloat16() for h in (4, 2, 2, 4))
    lens = torch.tensor([600, 333], dtype=torch.int32, device="cuda")
    want = binding.attention_forward(q, k, v, True, None, lens, lens)
    fwd = lambda s, *t: binding.attention_forward(*t[:3], True, None, *t[3:], stream=s)  # noqa: E731
    for got, val in zip(late(fwd, q, k, v, lens, lens), want):
        assert torch.equal(got, val)
    grads = binding.attention_backward(do, q, k, v, *want, True, None, lens, lens)
    bwd = lambda s, *t: binding.attention_backward(*t[:6], True, None, *t[6:], stream=s)  # noqa: E731
    for got, val in zip(late(bwd, do, q, k, v, *want, lens, lens), grads):
        assert torch.equal(got, val)
    g = r(300, 700)
    assert torch.equal(late(lambda s, t: binding.orthogonalise(t, stream=s), g), binding.orthogonalise(g))


def test_captured_calls_run_on_what_the_buffers_hold():
    """Every operator captured once and replayed on other data in the same buffers, and as it is called directly."""
    gen = torch.Generator(device="cuda").manual_seed(9)
    r = lambda *s: torch.randn(*s, generator=gen, device="cuda")  # noqa: E731
    x, dy, w, b = r(300, 768).bfloat16(), r(300, 768).bfloat16(), r(768), r(768)
    grads = torch.empty(3, 2 * 768, device="cuda")
    q, k, v, do = (r(2, 700, h, 64).bfloat16() for h in (4, 2, 2, 4))
    g1, g2, g3 = r(3, 100, 200), r(650, 2600), r(4, 1000, 2600)      # one block; a cluster for a tile; many tiles

    def calls():
        y, mean, rstd = binding.layer_norm_forward(x, w, b)
        dx = binding.layer_norm_backward(dy, x, w, mean, rstd, grads[:, :768], grads[:, 768:])
        o, lse = binding.attention_forward(q, k, v, causal=True)
        back = binding.attention_backward(do, q, k, v, o, lse, causal=True)
        return (y, mean, rstd, dx, grads, o, lse) + tuple(back) + tuple(binding.orthogonalise(g) for g in (g1, g2, g3))

    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    with torch.cuda.stream(side):
        calls()
    torch.cuda.synchronize()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        out = calls()
    for _ in range(3):
        for t in (x, dy, w, b, q, k, v, do, g1, g2, g3):
            t.copy_(r(*t.shape))
        graph.replay()
        got = [t.clone() for t in out]
        for a, c in zip(got, calls()):
            assert torch.equal(a, c)
        assert binding.operators_status() == binding.OK
