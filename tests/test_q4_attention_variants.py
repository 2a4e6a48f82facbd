"""Every variant of the 4-bit attention's kernels, chosen by the sizes as a caller's: blocks of one to four tiles of 16
rows, a head's keys whole and in parts, wavefronts that take one tile of keys, two (of a ring of two) and more.

Results are compared with 64 bits over the rows that the cache holds, with the bound of q4_plain.attention."""
import ctypes as C
import math
import zlib

import numpy as np
import pytest
import torch

from paper_2505_23219_amd import binding as B

import q4_plain as P

# M, nh, nkv, kv_len
CASES = [(1, 1, 1, 0), (1, 1, 1, 300), (3, 4, 1, 150), (1, 8, 2, 700), (2, 3, 1, 1000), (1, 2, 2, 16384), (5, 6, 3, 16391), (1, 6, 6, 12000),
         (1, 40, 40, 16384),
         (8, 5, 1, 0), (17, 1, 1, 300), (33, 1, 1, 300), (17, 32, 32, 700), (65, 12, 12, 700), (17, 1, 1, 1000), (33, 2, 2, 16384),
         (37, 20, 4, 777), (37, 40, 40, 1500), (17, 32, 32, 4096),
         (33, 129, 129, 0), (33, 200, 100, 0), (33, 129, 129, 300), (33, 200, 100, 500), (33, 6, 6, 16384), (65, 32, 32, 1500),
         (33, 24, 24, 4000), (65, 32, 32, 2000),
         (49, 129, 129, 0), (49, 200, 100, 0), (60, 129, 129, 200), (100, 96, 96, 200), (49, 200, 100, 500), (8, 24, 3, 40000),
         (49, 40, 40, 6000), (128, 24, 3, 3000), (128, 40, 40, 8192)]
NAN_CASES = [(8, 5, 1, 3), (33, 200, 100, 40), (49, 200, 100, 40), (60, 129, 129, 200), (33, 6, 6, 16384), (65, 32, 32, 1500),
             (128, 24, 3, 3000), (5, 6, 3, 16391)]


def _cut(M, nh, nkv, kv_len, d):
    """(tiles of a block, parts of a head's keys, turns of a wavefront)"""
    out = (C.c_int64 * 4)()
    B.lib().ghd_debug_q4_attention(M, kv_len, nh, nkv, d, out)
    rows, _, parts, _ = out
    tiles = -(-(-(-(kv_len + M) // 32)) // parts)
    return rows, parts, -(-tiles // (4 if rows == 1 else 8))


@pytest.mark.parametrize("d", [64, 128])
def test_the_cases_take_every_variant(d):
    cuts = {c: _cut(*c, d) for c in CASES}
    for rows in (1, 2, 3, 4):
        for parts in (False, True):
            turns = {t for r, p, t in cuts.values() if (r, p > 1) == (rows, parts)}
            assert turns and max(turns) > 2 and (parts or min(turns) == 1), (rows, parts, turns)
    assert {1, 2} <= {t for r, p, t in cuts.values() if r == 1 and p > 1}
    assert any(p > 256 // c[2] for c, (r, p, _) in cuts.items() if r == 1)           # three times as many parts
    # a last block without rows in its last tile
    assert any(r == rows and -(-c[0] * (c[1] // c[2]) // 16) % r for rows in (2, 3) for c, (r, _, _) in cuts.items())
    nan = {(r, p > 1) for r, p, _ in (_cut(*c, d) for c in NAN_CASES)}
    assert nan >= {(1, True), (2, False), (3, False), (3, True), (4, False), (4, True)}


def _rows(rng, *shape):
    spread = np.exp(0.5 * rng.standard_normal(shape[-2:], np.float32))
    return (rng.standard_normal(shape, np.float32) * spread + 0.5).astype(np.float16)


def _exact(q, k, v, see, kv_len, scale):
    """q4_plain.attention, a head at a time."""
    M, nh, d = q.shape
    T, rep = k.shape[0], nh // k.shape[1]
    out, tol = np.zeros((M, nh, d)), np.zeros((M, nh, d))
    on = np.concatenate([np.ones((M, kv_len), bool), see], 1)
    any_key = on.any(1)
    for h in range(nh):
        kh, vh, x = (t.astype(np.float64) for t in (k[:, h // rep], v[:, h // rep], q[:, h]))
        s = np.where(on, x @ kh.T * scale, -np.inf)
        ds = (d + 4) * 2.0 ** -24 * np.where(on, np.abs(x) @ np.abs(kh).T, 0).max(1, initial=0)[:, None] * abs(scale)
        e = np.exp(s - np.where(any_key, s.max(1), 0)[:, None])
        n = np.where(any_key, e.sum(1), 1)[:, None]
        y, size = e / n @ vh, e / n @ np.abs(vh)
        t = (2.0 ** -11 + 2.0 ** -21 + 4 * ds + T * 2.0 ** -23) * (size + np.abs(y)) + 2.0 ** -25 * (on @ np.abs(vh)) / n \
            + 2.0 ** -11 * np.abs(y) + 2.0 ** -25
        out[:, h], tol[:, h] = y, t * any_key[:, None]
    return out, tol


def _tree(rng, M):
    return np.array([-1] + [rng.integers(max(0, i - 6), i) for i in range(1, M)], np.int32)


def _relation(rng, M):
    see = rng.random((M, M)) < 0.3
    see[::3] = False                                     # with nothing committed these rows see no key
    return see


def _cache(rng, T, nkv, d, spoil=None):
    cache = B.KvQ4(1, nkv, d, -(-T // 32) * 32 + 32)
    cache.k.fill_(0xFF)
    cache.v.fill_(0xFF)
    k, v = _rows(rng, T, nkv, d), _rows(rng, T, nkv, d)
    if spoil:
        spoil(k, v)
    B.ghd_kv_append_q4(cache, 0, torch.from_numpy(k).cuda(), torch.from_numpy(v).cuda(), 0)
    return cache


def _seed(*key):
    return np.random.default_rng([zlib.crc32(str(key).encode())])


@pytest.mark.gpu
@pytest.mark.parametrize("d", [64, 128])
@pytest.mark.parametrize("M,nh,nkv,kv_len", CASES)
def test_against_64_bits(M, nh, nkv, kv_len, d):
    """Over a workspace that holds anything, with the same bits every time."""
    print("q4 attention variant", M, nh, nkv, kv_len, d, _cut(M, nh, nkv, kv_len, d), flush=True)
    rng, scale = _seed(M, nh, nkv, kv_len, d), 1 / math.sqrt(d)
    cache = _cache(rng, kv_len + M, nkv, d)
    k, v = (t[0].cpu().numpy() for t in B.ghd_kv_read_q4(cache, 0, kv_len + M))
    q = rng.standard_normal((M, nh, d), np.float32).astype(np.float16)
    parent, see = _tree(rng, M), _relation(rng, M)
    n = B.ghd_attention_q4_workspace_bytes(M, kv_len, nh, nkv, d)
    for call, on, relation in ((B.ghd_tree_attention_q4, P.sees_of_parent(parent), parent),
                               (B.ghd_masked_attention_q4, see, P.mask_words(see))):
        args = torch.from_numpy(q).cuda(), cache, 0, torch.from_numpy(relation).cuda(), kv_len
        got = call(*args, scale=scale, ws=B.workspace(n).fill_(0xFF))
        for byte in (0, 0x7F):
            assert torch.equal(got, call(*args, scale=scale, ws=B.workspace(n).fill_(byte)))
        want, tol = _exact(q, k, v, on, kv_len, scale)
        err = np.abs(got.cpu().numpy().astype(np.float64) - want)
        assert (err <= tol).all(), (call.__name__, err.max(), np.unravel_index(np.argmax(err - tol), err.shape))


@pytest.mark.gpu
@pytest.mark.parametrize("d", [64, 128])
@pytest.mark.parametrize("where,value", [("k", np.nan), ("v", np.nan), ("v", np.inf)])
@pytest.mark.parametrize("M,nh,nkv,kv_len", NAN_CASES)
def test_nan_reaches_the_rows_that_see_it(M, nh, nkv, kv_len, where, value, d):
    print("q4 attention nan", M, nh, nkv, kv_len, d, where, value, _cut(M, nh, nkv, kv_len, d), flush=True)
    bad, head, rep = M // 2, nkv - 1, nh // nkv
    outs = []

    def spoil(k, v):
        (k if where == "k" else v)[kv_len + bad, head, d - 5] = value

    for s in (None, spoil):
        rng = _seed(M, nh, nkv, kv_len, d)
        cache = _cache(rng, kv_len + M, nkv, d, s)
        see = np.tril(rng.random((M, M)) < 0.4) | np.eye(M, dtype=bool)
        q = torch.from_numpy(rng.standard_normal((M, nh, d), np.float32).astype(np.float16)).cuda()
        outs.append(B.ghd_masked_attention_q4(q, cache, 0, torch.from_numpy(P.mask_words(see)).cuda(), kv_len).cpu().numpy())
    hit = np.zeros((M, nh, d), bool)
    hit[see[:, bad], head * rep:] = True
    if where == "v":
        hit[..., :d - 32] = False                        # the last group of channels
    assert np.isfinite(outs[0]).all() and np.isnan(outs[1][hit]).all()
    assert np.array_equal(outs[1][~hit], outs[0][~hit])
