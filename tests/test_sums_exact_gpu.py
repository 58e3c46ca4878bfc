"""Sums over many rows of small whole numbers, which 32 bits hold exactly: one row lost or taken twice shows at any length."""
import pytest
import torch

from paper_2302_00845_b200 import binding

pytestmark = pytest.mark.gpu


def whole(seed, *shape, lo=1, hi=4):
    """Whole numbers from lo on, below hi."""
    return torch.randint(lo, hi, shape, generator=torch.Generator(device="cuda").manual_seed(seed), device="cuda")


def sums(dy, tokens, m, vocab):
    """[m][vocab][cols] in whole numbers"""
    t = tokens.reshape(m, -1).long()
    key = (t + vocab * torch.arange(m, device=t.device)[:, None]).reshape(-1)
    return torch.zeros(m * vocab, dy.shape[1], dtype=torch.int64, device=dy.device).index_add_(0, key, dy).view(m, vocab, -1)


def check(tokens, m, vocab, cols, dtype=torch.float32):
    dy = whole(tokens.numel() + cols, tokens.numel(), cols)
    want = sums(dy, tokens, m, vocab)
    assert int(want.max()) < 2 ** 24
    for accumulate in (False, True):
        buf = torch.full((m, vocab, cols), 5.0, device="cuda")
        binding.embedding_backward(dy.to(dtype), tokens, buf, accumulate=accumulate)
        seen = torch.zeros(m, vocab, dtype=torch.bool, device="cuda").scatter_(1, tokens.reshape(m, -1).long(), True)
        before = 5 if accumulate else 0
        assert torch.equal(buf, torch.where(seen[:, :, None], want + before, before).float())


# around one, two, three and four windows of 16, the parts of eight windows that the join takes, and steps of its search
@pytest.mark.parametrize("length", [15, 16, 17, 31, 32, 33, 47, 48, 49, 63, 64, 65, 127, 128, 129, 143, 144, 145, 511, 512, 513, 529, 5000, 40000, 100_003])
@pytest.mark.parametrize("cols", [300, 33])
def test_one_token_throughout(length, cols):
    for lead in (0, 1, 2, 8, 14, 15, 16, 17, 18, 30, 31, 32, 33):
        if lead < length:
            t = torch.full((1, length), 7, device="cuda")
            t[0, :lead] = torch.arange(lead, device="cuda") % 7
            check(t, 1, 50, cols, torch.bfloat16 if lead % 2 else torch.float32)


@pytest.mark.parametrize("run", list(range(1, 36)) + [46, 47, 48, 49, 50, 62, 63, 64, 65, 66, 79, 80, 81, 95, 96, 97, 112])
def test_runs_of_every_length_from_every_start(run):
    """Windows are 16 positions: runs within one, over a boundary, over a whole window, and longer; each from 32 starts, with
    single tokens or with other runs before and after."""
    alone, beside = [], []
    for start in range(32):
        after = 160 - run - start
        alone.append(torch.cat((torch.arange(start), torch.full((run,), 40), torch.arange(41, 41 + after))))
        beside.append(torch.cat((torch.full((start,), 39), torch.full((run,), 40), torch.full((min(after, run),), 41),
                                 torch.full((after - min(after, run),), 42))))
    check(torch.stack(alone).cuda(), 32, 201, 12)
    check(torch.stack(beside).cuda(), 32, 201, 12)


def test_runs_side_by_side():
    """Every token of a sequence in a run of its own, of lengths from 1 to 120, in an order that mixes the runs."""
    lengths = [1 + i * 37 % 120 for i in range(120)]
    t = torch.cat([torch.full((n,), i) for i, n in enumerate(lengths)])
    for seed in range(4):
        p = torch.randperm(t.numel(), generator=torch.Generator().manual_seed(seed))
        check(t[p].view(1, -1).cuda(), 1, 120, 40)
        check(torch.stack((t[p], t, t.flip(0))).cuda().int(), 3, 120, 40, torch.bfloat16)


@pytest.mark.parametrize("m,length", [(1, 70_000), (1, 140_001), (3, 8191), (1, 32_767), (1, 32_768), (1, 32_769), (64, 513)])
def test_long_lists_of_tokens(m, length):
    t = whole(length, m, length, lo=0, hi=300)
    t[:, ::3] = 11
    check(t, m, 300, 40)


# one head of one token to a block, and many; a cluster to a side, and blocks of their own with a second launch
@pytest.mark.parametrize("b,t,h,hk,m", [(1, 1, 1, 1, 1), (1, 5000, 1, 1, 1), (4, 4096, 4, 1, 2), (3, 357, 6, 2, 3), (64, 33, 3, 2, 16), (2, 1, 300, 7, 1),
                                        (1, 20_000, 2, 3, 1), (300, 2, 1, 5, 300)])
@pytest.mark.parametrize("dtype,d", [(torch.float32, 80), (torch.bfloat16, 64)])
def test_weights_of_the_rotation(b, t, h, hk, m, dtype, d):
    """Heads of plus and minus one have a root mean square of one.  It comes from an inverse root that may be two units off, so that a sum
    below 2^20 is within 2^-2 of its whole number; without rotation nothing else is rounded."""
    grads = torch.full((2, m, d), float("nan"), device="cuda")
    x, dy, want = [], [], []
    for i, heads in enumerate((h, hk)):
        sign = 2 * whole(i, b, t, heads, d, lo=0, hi=2) - 1
        g = whole(5 + i, b, t, heads, d)
        x.append(sign.to(dtype))
        dy.append((g * sign).to(dtype))              # (g n is positive: nothing that is lost is made up for elsewhere)
        want.append(g.view(m, -1, d).sum(1))
    assert int(torch.stack(want).max()) < 2 ** 20
    binding.rotary_backward(*dy, *x, dq_weight=grads[0], dk_weight=grads[1], rotary_dim=0, eps=0.0)
    for i in range(2):
        assert torch.equal(grads[i].round().long(), want[i])
