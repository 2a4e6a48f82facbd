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
