"""What operators_status says when two things were reported since it was last read."""
import pytest
import torch

from paper_2302_00845_b200 import binding

pytestmark = pytest.mark.gpu


def test_a_token_outside_the_vocabulary_is_not_lost_behind_an_expired_wait():
    g = torch.randn(1, 650, 2600, generator=torch.Generator(device="cuda").manual_seed(1), device="cuda")
    tokens, table = torch.tensor([3, 99], device="cuda"), torch.ones(10, 8, device="cuda")
    binding.orthogonalise(g)
    binding.operators_status()
    try:
        for first in (True, False):            # whichever came first
            if first:
                binding.embedding_forward(tokens, table)
            binding.operators_wait_limit(1)    # (the wait is given up: nothing else goes wrong)
            binding.orthogonalise(g)
            binding.operators_wait_limit(0)
            if not first:
                binding.embedding_forward(tokens, table)
            assert binding.operators_status() == binding.ERR_TIMEOUT
            assert binding.operators_status() == binding.ERR_INVALID
            assert binding.operators_status() == binding.OK
    finally:
        binding.operators_wait_limit(0)
        binding.operators_status()
