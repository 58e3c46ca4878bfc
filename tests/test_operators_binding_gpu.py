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
