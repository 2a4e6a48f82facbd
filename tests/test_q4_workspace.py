"""Workspace sizes of the 4-bit operators: what is made for the widest tree over the longest context does for
every call before it."""
import ctypes as C
import random

import pytest

from paper_2505_23219_amd import binding as B

HEADS = [(1, 1), (4, 4), (20, 4), (32, 8), (32, 32), (40, 40), (40, 8), (64, 1), (64, 2), (32, 1), (129, 129), (256, 256), (256, 8),
         (6, 3), (100, 100), (17, 1)]
FAKE = 0x10000


def _lengths(rng, n):
    return sorted({0, 1, 31, 32, 200, 6393, 8192, 58328, 65536, (1 << 24) - 128} | {int(2 ** rng.uniform(0, 24)) - 1 for _ in range(n)})


def _own(M, kv_len, nh, nkv, d):
    out = (C.c_int64 * 4)()
    B.lib().ghd_debug_q4_attention(M, kv_len, nh, nkv, d, out)
    return out[3]


@pytest.mark.parametrize("d", [64, 128])
@pytest.mark.parametrize("nh,nkv", HEADS)
def test_attention_sizes_never_fall_and_hold_every_call(nh, nkv, d):
    rng = random.Random(nh * 1000 + nkv + d)
    size = B.lib().ghd_attention_q4_workspace_bytes
    lengths = _lengths(rng, 60)
    before = None
    for M in sorted({1, 2, 3, 8, 15, 16, 17, 32, 33, 37, 48, 64, 65, 96, 97, 128} | {rng.randint(1, 128) for _ in range(6)}):
        row = [size(M, kv, nh, nkv, d) for kv in lengths]
        assert row == sorted(row), M
        assert before is None or all(a <= b for a, b in zip(before, row)), M
        assert all(_own(M, kv, nh, nkv, d) <= n for kv, n in zip(lengths, row)), M
        before = row
    assert before[-1] < 9 << 20


def test_a_call_takes_what_was_made_for_a_longer_one():
    """Two contexts on the way to a longer one; only the workspace of their own cut would be refused a byte less."""
    kv = (B.KV * 1)(B.KV(FAKE, FAKE))
    for M, nh, nkv, short, long in ((37, 20, 4, 58328, 65536), (8, 32, 8, 6393, 8192)):
        n, own = B.lib().ghd_attention_q4_workspace_bytes(M, long, nh, nkv, 128), _own(M, short, nh, nkv, 128)
        assert own <= n
        assert B.lib().ghd_tree_attention_q4(FAKE, FAKE, kv, FAKE, M, short, nh, nkv, 128, 1 << 17, 0.1, FAKE, own - 1,
                                             None) == B.GHD_ERR_WORKSPACE


@pytest.mark.parametrize("N,K", [(4096, 11008), (4096, 4096), (1003, 1288), (22016, 4096), (32000, 5120), (16, 65536), (5120, 13824),
                                 (640, 13824), (1, 8), (33, 8192), (1 << 20, 64)])
def test_linear_sizes_never_fall_with_rows(N, K):
    sizes = [B.lib().ghd_linear_q4_workspace_bytes(M, N, K) for M in range(1, 129)]
    assert sizes == sorted(sizes)
    assert sizes[0] >= 256
