"""The training operators' bounded waits run out: the kernels end, the status says so, the context stays usable.

A limit of one cycle lets a wait last as long as the hardware suspends it (some 8000 cycles), so that what is
waited for longer, such as the end of a loop over 32 tiles, is given up.  Nothing is made to fail but the waiting."""
import pytest
import torch

from paper_2302_00845_b200 import binding

pytestmark = pytest.mark.gpu


@pytest.fixture
def short_waits():
    binding.operators_status()
    yield lambda: binding.operators_wait_limit(1)
    binding.operators_wait_limit(0)
    torch.cuda.synchronize()
    binding.operators_status()


@pytest.mark.parametrize("b,t,h,hk,d", [(4, 4096, 12, 12, 64), (4, 4096, 8, 2, 128), (1, 4096, 2, 1, 64), (1, 4096, 1, 1, 128)])
def test_attention(short_waits, b, t, h, hk, d):
    """Many blocks of rows to a CTA, and few that are shared by clusters."""
    g = torch.Generator(device="cuda").manual_seed(d)
    r = lambda n: torch.randn(b, t, n, d, generator=g, device="cuda").to(torch.bfloat16)  # noqa: E731
    q, k, v, do = r(h), r(hk), r(hk), r(h)
    o, lse = binding.attention_forward(q, k, v)
    want = (o, lse) + binding.attention_backward(do, q, k, v, o, lse)
    assert binding.operators_status() == binding.OK
    short_waits()
    if b > 1:                # (a single block of rows to a CTA: nothing in the forward pass waits for long)
        binding.attention_forward(q, k, v)
        assert binding.operators_status() == binding.ERR_TIMEOUT
    binding.attention_backward(do, q, k, v, o, lse)
    assert binding.operators_status() == binding.ERR_TIMEOUT
    assert binding.operators_status() == binding.OK          # read and cleared
    binding.operators_wait_limit(0)
    o, lse = binding.attention_forward(q, k, v)
    got = (o, lse) + binding.attention_backward(do, q, k, v, o, lse)
    assert binding.operators_status() == binding.OK
    for a, c in zip(got, want):
        assert torch.equal(a, c)


@pytest.mark.parametrize("batch,rows,cols", [(1, 650, 2600), (1, 300, 900), (1, 1030, 640), (6, 600, 180), (4, 1500, 2600)])
def test_orthogonalise(short_waits, batch, rows, cols):
    """Clusters of four and of two, most of whose blocks have no tile in two products of three; no clusters; several
    tiles to a block."""
    g = torch.randn(batch, rows, cols, generator=torch.Generator(device="cuda").manual_seed(rows), device="cuda")
    want = binding.orthogonalise(g)
    assert binding.operators_status() == binding.OK
    short_waits()
    for _ in range(3):
        binding.orthogonalise(g)
        assert binding.operators_status() == binding.ERR_TIMEOUT
    binding.operators_wait_limit(0)
    assert torch.equal(binding.orthogonalise(g), want)
    assert binding.operators_status() == binding.OK


def test_a_long_loop_is_no_expired_wait():
    """262,144 tiles of queries and heads share one key head: the loop over them, in a cluster of eight, takes longer than
    the limit for short loops, and nothing is wrong.  (With the default limit it would take ten million tiles.)"""
    t, h, d = 262144, 128, 8
    g = torch.Generator(device="cuda").manual_seed(1)
    r = lambda n, heads: torch.randn(1, n, heads, d, generator=g, device="cuda").to(torch.bfloat16)  # noqa: E731
    q, k, v, do = r(t, h), r(128, 1), r(128, 1), r(t, h)
    o, lse = binding.attention_forward(q, k, v)
    want = binding.attention_backward(do, q, k, v, o, lse)
    assert binding.operators_status() == binding.OK
    try:
        binding.operators_wait_limit(30_000_000)
        got = binding.attention_backward(do, q, k, v, o, lse)
        assert binding.operators_status() == binding.OK
    finally:
        binding.operators_wait_limit(0)
    for a, c in zip(got, want):
        assert torch.equal(a, c)
