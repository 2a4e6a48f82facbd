"""Sums of what rejections leave, held in 64 bits: a draw that sums in 32 bits of eight weights would miss."""
import math

import pytest
import torch

import sparse_plain as P
import test_gpu_sampled as S

pytestmark = pytest.mark.gpu


@pytest.mark.parametrize("place", [0, 1, 3])
@pytest.mark.parametrize("children", [2, 5])
def test_many_small_weights_beside_large_ones(children, place):
    """4096 tokens, every fourth of the first half with the weight 1, all others with 0.9 2^-24, which 32 bits drop beside a 1; 1024
    tokens of weight 1 behind them.  The random number lies between where a sum without the small weights and one with them
    ends the first 4096.  Weights of 1 are exact and the small ones, of all 1.9e-4, are off by 2^-23 of themselves: sums in 64 bits by
    less than 1e-10, so the token is that of 64 bits or a neighbour (5e-8 apart)."""
    V, M, small = 8192, children + 1, 0.9 * 2.0 ** -24
    logits, q = torch.full((M, V), -60.0), torch.full((M, V), -math.inf)
    logits[0, :4096] = math.log(small)
    logits[0, place:2048:4] = 0.0
    logits[0, 4096:5120] = 0.0
    tokens = torch.zeros(M, dtype=torch.int32)
    tokens[1:] = 6000 + torch.arange(children)
    q[0, 6000:6000 + children] = 0.0
    q[0, 7000] = 0.0                             # (no child's: something is left of q)
    large, less = 512 + 1024.0, 512.0
    more = less + 3584 * math.exp(logits[0, 4000].double().item())
    between = 0.5 * (less / large + more / (large + more - less))
    u = torch.full((M,), 0.99)
    u[0] = between
    assert less / large < u[0].double().item() < more / (large + more - less)
    want = P.accept(logits, tokens, [-1] + [0] * children, u, 1.0, q)
    assert want[0] == 1 and 2048 <= want[1] < 4096
    got = S._gpu((logits, tokens, [-1] + [0] * children, u, q, None))
    assert got[0] == 1 and abs(got[1] - want[1]) <= 1, (got[:2], want)


@pytest.mark.parametrize("gap", [2.0, 5.0, 7.0, 7.6, 9.0, 14.0])
def test_what_is_left_of_the_draft_around_a_thousandth(gap):
    """After two rejections exp(-gap) of the draft's probability, and some more, is left: what follows from a difference, or is summed up."""
    V, M = 4100, 6
    for seed in range(4):
        g = torch.Generator().manual_seed(seed)
        logits, q = torch.randn(M, V, generator=g), torch.full((M, V), -40.0)
        tokens = torch.tensor([0, 11, 4098, 17, 2000, 4099], dtype=torch.int32)
        q[0, tokens[1:3].long()] = 0.0
        q[0, tokens[3:].long()], q[0, 100:110] = -gap, -gap - 1.0
        logits[0, tokens[1:].long()] = -30.0
        u = torch.full((M,), 0.9)
        u[0] = 0.1 + 0.25 * seed
        want = S._check((logits, tokens, [-1] + [0] * 5, u, q, None))
        assert want[0] == 1
        logits[0, 17] = 0.0                      # the third may be accepted
        u[3] = 0.2
        S._check((logits, tokens, [-1] + [0] * 5, u, q, None))
