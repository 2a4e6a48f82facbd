"""Selection where scores are below zero and some blocks score infinity: every kernel that picks, against the plain 64-bit form."""
import math

import pytest
import torch

import sparse_plain as P
import test_gpu_sparse as T
from paper_2505_23219_amd import binding as B

pytestmark = pytest.mark.gpu


def _check(M, nh, nkv, d, n, count, sinks, recent, mixed=False):
    g = T._gen(M + n + d)
    k = torch.randn(nkv, n * 64, d, generator=g)
    # (rows of a block nearly alike, so that its bounds have the signs of its keys)
    k = (0.05 * k + torch.randn(nkv, n, 1, d, generator=g).expand(nkv, n, 64, d).reshape(k.shape) if mixed else k + 3).half()
    kd = k.cuda()
    hi, lo, unit = P.bounds(k, n)
    keep = count - sinks - recent
    order = sinks + torch.randperm(n - sinks - recent, generator=g)
    for scale in (1.0, 2.0):                     # either parity of every score's exponent
        q = torch.randn(M, nh, d, generator=g)
        q = (scale * (q if mixed else -q.abs())).half()
        clean = P.scores(q, (hi, lo, unit))
        assert (clean < 0).any() and (clean > 0).any() if mixed else (clean < 0).all()
        for infinite in sorted({0, 1, max(keep - 1, 0), keep, keep + 3, keep + 80}):
            infinite = min(infinite, len(order) - 1)
            bad, kb = unit.clone(), kd.clone()
            for i, b in enumerate(order[:infinite].tolist()):
                bad[:, b] = math.inf
                kb[:, 64 * b + i % 64, i % d] = (math.nan, math.inf, -math.inf)[i % 3]
            score = P.scores(q, (hi, lo, bad))
            bounds = B.BlockBounds(nkv, d, n * 64)
            B.ghd_block_bounds(bounds, kb, 0, n)
            got = B.ghd_block_select(q.cuda(), bounds, n * 64, count, sinks=sinks, recent=recent)
            want = P.words(P.select(score, count, sinks, recent))
            assert torch.equal(got.cpu(), want), (scale, infinite, (got.cpu() != want).sum().item())


# one launch for up to 128 blocks, or 512 of many picks; a workgroup a pick, with its scores in registers or not; eight picks a workgroup
@pytest.mark.parametrize("M,nh,nkv,d,n,count,sinks,recent", [
    (1, 2, 1, 64, 6, 1, 0, 0), (6, 4, 2, 64, 14, 5, 1, 1), (9, 2, 2, 128, 128, 20, 0, 2), (128, 8, 8, 64, 300, 9, 1, 1),
    (3, 4, 2, 128, 200, 6, 0, 0), (2, 2, 2, 64, 1500, 70, 1, 2), (1, 1, 1, 64, 4500, 33, 0, 1), (128, 8, 8, 64, 600, 5, 0, 0),
    (128, 8, 8, 64, 1200, 30, 2, 2)])
def test_scores_below_zero(M, nh, nkv, d, n, count, sinks, recent):
    _check(M, nh, nkv, d, n, count, sinks, recent)


@pytest.mark.parametrize("M,nh,nkv,d,n,count", [(7, 2, 2, 64, 100, 90), (5, 1, 1, 128, 700, 690), (128, 8, 8, 64, 520, 500)])
def test_scores_of_both_signs(M, nh, nkv, d, n, count):
    """Picks that go down to the scores below zero."""
    _check(M, nh, nkv, d, n, count, 0, 0, mixed=True)


@pytest.mark.parametrize("M,nkv,n", [(3, 2, 100), (128, 8, 300), (2, 1, 700), (1, 1, 4300), (128, 8, 700)])
def test_bounds_that_were_never_given(M, nkv, n):
    """Blocks whose bounds hold anything: which of them a token reads says nothing, but it reads `count` blocks."""
    g, d = T._gen(n), 64
    bounds = B.BlockBounds(nkv, d, n * 64)
    bounds.data.copy_(torch.randint(0, 256, (bounds.data.numel(),), dtype=torch.uint8, generator=g))
    units = bounds.data[nkv * n * 2 * d:].view(torch.int32)
    odd = torch.tensor([0xff800000, 0xffffffff, 0x7fffffff, 0x7f800000, 0xff7fffff, 0x80000000]).int()
    units[::3] = odd[torch.randint(0, 6, (len(units[::3]),), generator=g)].cuda()
    q = torch.randn(M, nkv, d, generator=g).half().cuda()
    for count in (1, 2, 20, n - 1):
        sel = B.ghd_block_select(q, bounds, n * 64, count, sinks=1, recent=0).cpu()
        bits = torch.stack([sel[:, i // 64] >> (i % 64) & 1 for i in range(M)])
        assert (bits.sum(2) == count).all() and (bits[:, :, 0] == 1).all()
