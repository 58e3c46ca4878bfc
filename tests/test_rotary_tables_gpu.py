"""Calls that take turns with different bases and widths, as layers with two kinds of rotation do."""
import time

import pytest
import torch

from paper_2302_00845_b200 import binding
from test_rotary_gpu import draw

pytestmark = pytest.mark.gpu
KINDS = [(10000.0, 128), (500_000.0, 128), (10000.0, 64), (1_000_000.0, 32)]


def test_the_same_bits_in_any_order():
    q, k, qw, kw, dq, dk = draw(1, 40, 2, 1, 128, "f32")
    def call(base, rot):
        return binding.rotary_forward(q, k, qw, kw, base=base, rotary_dim=rot) + binding.rotary_backward(dq, dk, q, k, qw, kw, base=base, rotary_dim=rot)
    more = KINDS + [(b, r) for b in (100.0, 0.5) for r in (0, 8, 96)]            # more than are kept at once
    want = {}
    for kind in more:
        call(7.0, 128)
        want[kind] = call(*kind)
    for _ in range(3):
        for kinds in (KINDS, more, more[::-1]):
            for kind in kinds:
                assert all(torch.equal(a, c) for a, c in zip(call(*kind), want[kind]))


def test_taking_turns_costs_no_more():
    q, k, *_ = draw(1, 1, 2, 1, 128)
    out, out_k = torch.empty_like(q), torch.empty_like(k)

    def host(kinds):
        best = float("inf")
        for _ in range(20):
            torch.cuda.synchronize()
            start = time.perf_counter()
            for i in range(100):
                base, rot = kinds[i % len(kinds)]
                binding.rotary_forward(q, k, base=base, rotary_dim=rot, q_out=out, k_out=out_k)
            best = min(best, time.perf_counter() - start)
        return best
    host(KINDS)
    assert host(KINDS) <= 1.5 * host(KINDS[:1])
