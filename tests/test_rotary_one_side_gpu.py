"""The backward rotation of queries alone or of keys alone, over many tokens: the side that is not there takes no time."""
import pytest
import torch

from paper_2302_00845_b200 import binding
from test_rotary_gpu import draw

pytestmark = pytest.mark.gpu


def microseconds(call, n=10):
    """The shortest of n passes of a captured call."""
    call()
    torch.cuda.synchronize()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        call()
    best = float("inf")
    for _ in range(n):
        a, b = torch.cuda.Event(enable_timing=True), torch.cuda.Event(enable_timing=True)
        a.record()
        graph.replay()
        b.record()
        b.synchronize()
        best = min(best, 1e3 * a.elapsed_time(b))
    return best


@pytest.mark.parametrize("m", [1, 2])
def test_an_absent_side_takes_no_time(m):
    q, k, qw, kw, dq, dk = draw(4, 4096, 16, 4, 128)
    none_q, none_k = q[:, :, :0], k[:, :, :0]
    both, one = torch.empty(2, m, 128, device="cuda"), torch.full((2, m, 128), float("nan"), device="cuda")
    dx = binding.rotary_backward(dq, dk, q, k, qw, kw, dq_weight=both[0], dk_weight=both[1])
    all_of_it = microseconds(lambda: binding.rotary_backward(dq, dk, q, k, qw, kw, dq_weight=both[0], dk_weight=both[1]))
    calls = (lambda: binding.rotary_backward(dq, None, q, None, qw, dq_weight=one[0], dk_weight=one[1]),
             lambda: binding.rotary_backward(dq, none_k, q, none_k, qw, kw, dq_weight=one[0], dk_weight=one[1]),
             lambda: binding.rotary_backward(none_q, dk, none_q, k, qw, kw, dq_weight=one[0], dk_weight=one[1]))
    for i, call in enumerate(calls):
        one.fill_(float("nan"))
        got, side = call(), i // 2
        assert torch.equal(got[side], dx[side])
        assert (one[1 - side] == 0).all()
        # (fewer blocks share the sums when the other side is there: their order, but nothing else, may differ)
        assert float((one[side] - both[side]).abs().max()) <= 1e-3 * float(both[side].abs().max())
        assert microseconds(call) <= 1.5 * all_of_it
