"""What the rotation writes past a sequence's length when the weights are no numbers."""
import pytest
import torch

from paper_2302_00845_b200 import binding
from test_rotary_gpu import draw

pytestmark = pytest.mark.gpu


@pytest.mark.parametrize("dtype,interleaved", [("f32", True), ("bf16", False)])
@pytest.mark.parametrize("bad", [float("nan"), float("inf")])
def test_past_a_length_there_are_zeros_whatever_the_weights_are(dtype, interleaved, bad):
    q, k, qw, kw, dq, dk = draw(3, 12, 3, 2, 64, dtype)
    qw[5], kw[63] = bad, bad
    lens = torch.tensor([12, 7, 0], dtype=torch.int32, device="cuda")
    y = binding.rotary_forward(q, k, qw, kw, lens=lens, interleaved=interleaved)
    dx = binding.rotary_backward(dq, dk, q, k, qw, kw, lens=lens, interleaved=interleaved)
    for v in (*y, *dx):
        assert not torch.isfinite(v[0]).all()
        assert (v[1, 7:] == 0).all() and (v[2] == 0).all()
