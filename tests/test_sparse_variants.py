"""Every variant of the sparse attention's kernels: the cases take them all, and each is right, with an odd value, too."""
import ctypes as C
import itertools
import math

import pytest
import torch

import sparse_plain as P
from paper_2505_23219_amd import binding as B

# (M, nh, nkv, d, kv_len): tiles of rows in a block 1, 2, 4, 8; one or more parts; one or more blocks of rows
CASES = [(1, 1, 1, 64, 0), (1, 32, 1, 64, 0), (1, 1, 1, 64, 130), (17, 1, 1, 64, 130), (17, 256, 256, 64, 700), (3, 32, 1, 64, 0),
         (17, 64, 64, 64, 1500), (65, 1, 1, 64, 0), (64, 256, 256, 64, 130), (65, 64, 2, 64, 0), (40, 33, 33, 64, 1500), (65, 24, 3, 64, 0),
         (33, 256, 128, 64, 0), (33, 32, 1, 64, 0), (65, 32, 1, 64, 0), (128, 40, 40, 64, 4096),
         (1, 1, 1, 128, 0), (1, 32, 1, 128, 0), (1, 1, 1, 128, 130), (17, 1, 1, 128, 130), (17, 256, 256, 128, 700), (3, 32, 1, 128, 0),
         (17, 33, 33, 128, 1500), (65, 1, 1, 128, 0), (64, 256, 256, 128, 5), (33, 32, 1, 128, 0), (17, 51, 17, 128, 1500),
         (97, 3, 3, 128, 130), (65, 256, 256, 128, 0), (65, 160, 5, 128, 0), (65, 32, 1, 128, 0), (128, 40, 40, 128, 8000)]


def _cut(M, nh, nkv, d, kv_len):
    out = (C.c_int64 * 4)()
    B.lib().ghd_debug_sparse_attention(M, kv_len, nh, nkv, d, out)
    return list(out)


def test_the_cases_take_every_variant():
    taken = {(c[3], cut[0], cut[2] > 1) for c in CASES for cut in [_cut(*c)]}
    assert taken == set(itertools.product((64, 128), (1, 2, 4, 8), (False, True)))
    assert {(c[3], cut[0], cut[1] > 1) for c in CASES for cut in [_cut(*c)]} == taken       # one or more blocks of rows


def test_workspaces_hold_any_smaller_call():
    for nh, nkv, d in ((32, 32, 128), (32, 8, 128), (20, 4, 64), (40, 1, 64), (256, 256, 128), (1, 1, 64)):
        for M, kv in itertools.product((1, 5, 16, 33, 64, 65, 128), (0, 63, 64, 777, 4096, 70000, 131072, 1 << 21)):
            room = B.ghd_sparse_attention_workspace_bytes(M, kv, nh, nkv, d)
            for m, k in itertools.product((1, 3, 16, 17, 40, 64, 128), (0, 1, 64, 700, 4096, 65600, 131072, 1 << 21)):
                if m <= M and k <= kv:
                    assert _cut(m, nh, nkv, d, k)[3] <= room, (nh, nkv, d, M, kv, m, k)


def test_lists_hold_what_a_part_reads():
    for nkv, rep, M in itertools.product((1, 2, 7, 40, 256), (1, 2, 5), (1, 16, 64, 128)):
        if nkv * rep > 256:
            continue
        for kv in (0, 65535, 65600, 131072, 1 << 20, (1 << 21) - 1, 1 << 21):
            most, splits = kv // 64 + -(-(kv % 64 + M) // 64), _cut(M, nkv * rep, nkv, 128, kv)[2]
            assert -(-most // splits) <= 1024


def test_no_half_of_a_block_lies_behind_the_rows():
    """The first key of every half block that a wavefront reads is there, and none that holds a row is left out."""
    f = B.lib().ghd_debug_sparse_halves
    for M in range(1, 129):
        for kv_len in list(range(0, 200)) + [700, 2047, 1 << 20]:
            n, total = kv_len // 64, kv_len + M
            tail = -(-(total - 64 * n) // 64)
            for count in (1, tail, tail + 3):            # a part that ends with the last block
                halves = f(count, n + tail - 1, total)
                last = (n + tail - 1) * 64 + (halves - 1) % 2 * 32
                assert last < total <= last + 32 and (halves + 1) // 2 == count
            for last in range(max(0, n - 2), n + tail - 1):          # and one that ends before
                assert f(5, last, total) == 10
    assert f(0, 0, 5) == 0


def test_many_query_heads_fit_what_a_launch_holds():
    """Blocks and parts are 16 bits each, tiles of rows 2^13 at the most."""
    for nkv, rep in ((1, 1024), (2, 512), (40, 8), (204, 5), (256, 4), (256, 1)):
        for M, kv_len in itertools.product((1, 16, 17, 128), (0, 64, 5000, 1 << 21)):
            for d in (64, 128):
                room = B.ghd_sparse_attention_workspace_bytes(M, kv_len, nkv * rep, nkv, d)
                rows, blocks, splits, need = _cut(M, nkv * rep, nkv, d, kv_len)
                assert 0 < need <= room and blocks < 1 << 16 and splits < 1 << 16
                assert rows * blocks * 16 >= M * rep > rows * (blocks - 1) * 16


@pytest.mark.gpu
@pytest.mark.parametrize("M,nh,nkv,d,kv_len", CASES)
def test_variants(M, nh, nkv, d, kv_len):
    import test_gpu_sparse as T
    n = kv_len // 64
    sel = T._selection(nkv, M, n, min(3, n), M + n, pool=7)
    T._check(M, nh, nkv, d, kv_len, sel, "random", seed=M)
    T._check(M, nh, nkv, d, kv_len, sel, "sparse", seed=M + 1, layout="tokens")


@pytest.mark.gpu
@pytest.mark.parametrize("M,nh,nkv,d,kv_len", [c for c in CASES if c[0] > 1 and c[1] < 200])
def test_variants_with_an_odd_value(M, nh, nkv, d, kv_len):
    """A value that is infinite reaches the tokens that see its row; the others are as they were, to twice the rounding."""
    import test_gpu_sparse as T
    n, rep = kv_len // 64, nh // nkv
    sel = T._selection(nkv, M, n, min(3, n), M + n, pool=7)
    rows = -(-(kv_len + M) // 8) * 8
    _, v, kd, vd = T._cache(nkv, rows, d, M)
    q = torch.randn(M, nh, d, generator=T._gen(M)).half().cuda()
    rel, see = T._relation("random", M, M)
    words = P.words(sel).cuda()
    clean = B.ghd_sparse_attention(q, kd, vd, words, kv_len, **rel).cpu()
    head, block = nkv - 1, int(sel[nkv - 1].any(0).nonzero()[0]) if n else -1
    row, seen = (block * 64 + 37, sel[head, :, block]) if n else (kv_len + M // 2, see[:, M // 2])
    vd[head, d - 3, row] = math.inf
    got = B.ghd_sparse_attention(q, kd, vd, words, kv_len, **rel).cpu()
    mine, was = got[:, head * rep:], clean[:, head * rep:]
    assert torch.equal(got[:, :head * rep], clean[:, :head * rep])
    assert not torch.isfinite(mine[seen][:, :, d - 3]).any()
    mine[seen, :, d - 3] = was[seen, :, d - 3] = 0
    assert ((mine - was).abs() <= 2.0 ** -10 * (was.abs() + v.abs().max() * 0.1)).all()
