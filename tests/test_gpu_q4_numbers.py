"""Numbers at the ends of what the 4-bit operators take."""
import numpy as np
import pytest
import torch

from paper_2505_23219_amd import binding as B

import q4_plain as P

pytestmark = pytest.mark.gpu


@pytest.mark.parametrize("M,kv_len", [(1, 0), (3, 40), (20, 700), (64, 0)])
def test_a_scale_that_is_no_number_gives_none(M, kv_len):
    """As the formula does, for every row that sees a key; the others are zeros."""
    nh, nkv, d = 4, 2, 64
    cache = B.KvQ4(1, nkv, d, -(-(kv_len + M) // 32) * 32)
    rows = torch.randn(kv_len + M, nkv, d, device="cuda").half()
    B.ghd_kv_append_q4(cache, 0, rows, rows, 0)
    q = torch.randn(M, nh, d, device="cuda").half()
    see = np.eye(M, dtype=bool)
    see[::2] = False
    got = B.ghd_masked_attention_q4(q, cache, 0, torch.from_numpy(P.mask_words(see)).cuda(), kv_len, scale=float("nan"))
    sees = torch.from_numpy(see.any(1) | (kv_len > 0)).cuda()
    assert torch.isnan(got[sees]).all() and (got[~sees] == 0).all()


@pytest.mark.parametrize("M", [1, 20, 64, 100])
@pytest.mark.parametrize("group", [32, 64, 128])
def test_zero_points_of_eight_bits(M, group):
    """Zero points may lie outside of the codes; a code less any of them is exact."""
    rng = np.random.default_rng([M, group])
    N, K = 70, 392
    G = -(-K // group)
    codes = rng.integers(0, 256, (N, K // 2), dtype=np.uint8)
    scales = (rng.uniform(0.2, 1.0, (N, G)) * 0.01).astype(np.float16)
    zeros = rng.integers(0, 256, (N, G), dtype=np.uint8)
    zeros[0], zeros[1] = 255, 0
    x = rng.standard_normal((M, K)).astype(np.float16)
    Wq = B.ghd_pack_weight_q4(*(torch.from_numpy(t).cuda() for t in (codes, scales, zeros)), group)
    got = B.ghd_linear_q4(torch.from_numpy(x).cuda(), Wq, N, group).cpu().numpy()
    want, tol = P.linear(x, P.unpack_weight(codes, scales, zeros, K, group), False)
    assert (np.abs(got - want) <= tol).all()
