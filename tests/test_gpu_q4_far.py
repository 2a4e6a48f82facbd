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


@pytest.mark.parametrize("d", [64, 128])
def test_heads_beyond_4_gib(d):
    """The last head's rows begin above 2^32 bytes."""
    nkv, nh, cap, M, kv = 640 // d, 1280 // d, 1 << 24, 6, 50
    _enough(20)
    n = B.lib().ghd_kv_q4_bytes(nkv, cap, d)
    assert n // nkv * (nkv - 1) > 1 << 32
    rng = np.random.default_rng(d)
    cache = B.KvQ4.__new__(B.KvQ4)
    cache.L, cache.nkv, cache.d, cache.capacity = 1, nkv, d, cap
    cache.k, cache.v = (torch.empty((1, n), dtype=torch.uint8, device="cuda") for _ in range(2))
    cache.kv = (B.KV * 1)(B.KV(cache.k.data_ptr(), cache.v.data_ptr()))
    cache.layers = [C.byref(cache.kv[0])]
    k, v = (rng.standard_normal((kv + M, nkv, d)).astype(np.float16) for _ in range(2))
    q = rng.standard_normal((M, nh, d)).astype(np.float16)
    parent = np.arange(-1, M - 1, dtype=np.int32)
    kt, vt, qt, pt = (torch.from_numpy(t).cuda() for t in (k, v, q, parent))
    B.ghd_kv_append_q4(cache, 0, kt, vt, 0)
    got = B.ghd_tree_attention_q4(qt, cache, 0, pt, kv).cpu().numpy().astype(np.float64)
    want, tol = P.attention(q, P.held(k), P.held(v), P.sees_of_parent(parent), kv, 1 / math.sqrt(d))
    assert (np.abs(got - want) <= tol).all()
    # rows far behind in every head
    at = cap - 40
    B.ghd_kv_append_q4(cache, 0, kt[:40], vt[:40], at)
    B.ghd_commit_path_q4(cache, torch.tensor([3, 0, 0, 11, 39], dtype=torch.int32, device="cuda"), 40, at)
    order = [0, 11, 39] + list(range(3, 40))
    for got, x in zip(B.ghd_kv_read_q4(cache, at, 40), (k, v)):
        assert np.array_equal(got[0].cpu().numpy(), P.held(x[:40])[order])
    # the first rows are as they were
    for got, x in zip(B.ghd_kv_read_q4(cache, 0, kv + M), (k, v)):
        assert np.array_equal(got[0].cpu().numpy(), P.held(x))
