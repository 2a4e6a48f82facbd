"""The 4-bit operators at sizes whose offsets, or whose launches, pass 32 bits."""
import ctypes as C
import math

import numpy as np
import pytest
import torch

from paper_2505_23219_amd import binding as B

import q4_plain as P

pytestmark = pytest.mark.gpu


@pytest.fixture(autouse=True)
def room():
    torch.cuda.empty_cache()
    yield
    torch.cuda.empty_cache()


def _enough(gib):
    free = torch.cuda.mem_get_info()[0]
    if free < gib << 30:
        pytest.skip("%d GiB of memory are free, %d are needed" % (free >> 30, gib))


def test_packing_the_largest_matrices():
    """2^20 rows of 257 units of 128 columns: more workgroups than one launch has."""
    N, K, group = 1 << 20, 32776, 128
    _enough(40)
    torch.manual_seed(0)
    codes = torch.zeros((N, K // 2), dtype=torch.uint8, device="cuda")
    scales = torch.ones((N, -(-K // group)), dtype=torch.float16, device="cuda")
    some = [0, (1 << 23) // 257 * 16 - 16, (1 << 23) // 257 * 16, N // 2, N - 32]      # (the second launch's first tile among them)
    for n in some:
        codes[n:n + 32] = torch.randint(0, 256, (32, K // 2), dtype=torch.uint8, device="cuda")
        scales[n:n + 32] = torch.rand(32, scales.shape[1], device="cuda").half()
    packed = B.ghd_pack_weight_q4(codes, scales, None, group).view(N // 16, -1)
    for n in some + [n + 32 for n in some[:-1]]:
        alone = B.ghd_pack_weight_q4(codes[n:n + 32].contiguous(), scales[n:n + 32].contiguous(), None, group).view(2, -1)
        assert torch.equal(packed[n // 16:n // 16 + 2], alone), n
    x = torch.randn(3, K, device="cuda").half()
    y = B.ghd_linear_q4(x, packed.view(-1), N, group)
    want, tol = P.linear(x.cpu().numpy(), P.unpack_weight(codes[-32:].cpu().numpy(), scales[-32:].cpu().numpy(), None, K, group), False)
    assert (np.abs(y[:, -32:].cpu().numpy() - want) <= tol).all()


def test_reading_back_more_than_one_launch():
    """48 layers - all the same cache - of 32 heads and 43691 octets of rows."""
    L, nkv, d, rows = 48, 32, 64, 349528
    _enough(150)
    torch.manual_seed(0)
    cache = B.KvQ4(1, nkv, d, -(-rows // 32) * 32)
    x = torch.randn(rows, nkv, d, device="cuda").half()
    B.ghd_kv_append_q4(cache, 0, x, x.flip(0).contiguous(), 0)
    want = [t[0] for t in B.ghd_kv_read_q4(cache, 0, rows)]
    many = B.KvQ4.__new__(B.KvQ4)
    many.L, many.nkv, many.d, many.capacity, many.k, many.v = L, nkv, d, cache.capacity, cache.k, cache.v
    many.kv = (B.KV * L)(*[cache.kv[0]] * L)
    many.layers = [C.byref(kv) for kv in many.kv]
    out = [torch.empty((L, rows, nkv, d), dtype=torch.float16, device="cuda") for _ in range(2)]
    for t in out:
        t[0], t[-1] = 7, 7
    B.ghd_kv_read_q4(many, 0, rows, *out)
    for t, w in zip(out, want):
        for layer in (0, 23, 46, 47):
            assert torch.equal(t[layer], w), layer
