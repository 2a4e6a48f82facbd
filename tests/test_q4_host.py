"""Host-side checks of the 4-bit entry points, which need no GPU."""
import os

import pytest

from paper_2505_23219_amd import binding as B

FAKE = 0x10000


@pytest.fixture(scope="module")
def lib():
    if not os.path.exists(B.LIB_PATH):
        from paper_2505_23219_amd.build import build
        build()
    return B.lib()


def _refuses(call, code, **kw):
    assert call(**kw) == code, kw


def test_sizes(lib):
    assert lib.ghd_weight_q4_bytes(16, 128, 128) == 1024 + 64
    assert lib.ghd_weight_q4_bytes(17, 136, 32) == 2 * 2 * (1024 + 256)
    assert lib.ghd_weight_q4_bytes(22016, 4096, 64) == 22016 * 4096 // 2 + 22016 * 64 * 4
    for bad in ((0, 128, 128), (16, 0, 128), (16, 12, 32), (16, 128, 48), (16, 65544, 32), ((1 << 20) + 1, 128, 32)):
        assert lib.ghd_weight_q4_bytes(*bad) == 0
    assert lib.ghd_kv_q4_bytes(8, 64, 128) == 8 * 64 * (64 + 16)
    assert lib.ghd_kv_q4_bytes(3, 1 << 24, 64) == 3 * (1 << 24) * 40
    for bad in ((0, 64, 128), (257, 64, 128), (8, 0, 128), (8, 40, 128), (8, 64, 96), (8, (1 << 24) + 32, 64)):
        assert lib.ghd_kv_q4_bytes(*bad) == 0
    assert lib.ghd_linear_q4_workspace_bytes(0, 64, 64) == 0 and lib.ghd_linear_q4_workspace_bytes(129, 64, 64) == 0
    assert lib.ghd_linear_q4_workspace_bytes(1, 64, 64) > 0
    assert lib.ghd_attention_q4_workspace_bytes(1, 0, 4, 2, 64) > 0
    for bad in ((0, 0, 4, 2, 64), (129, 0, 4, 2, 64), (1, -1, 4, 2, 64), (1, 0, 4, 3, 64), (1, 0, 4, 0, 64), (1, 0, 4, 2, 96)):
        assert lib.ghd_attention_q4_workspace_bytes(*bad) == 0


def test_linear_and_packing_refuse_bad_arguments(lib):
    def linear(y=FAKE, x=FAKE, W=FAKE, M=16, N=64, K=64, group=32, ldx=64, ldy=64, flags=0, ws=FAKE, n=1 << 30):
        return lib.ghd_linear_q4(y, x, W, M, N, K, group, ldx, ldy, flags, ws, n, None)

    for name in ("y", "x", "W"):
        _refuses(linear, B.GHD_ERR_NULL, **{name: None})
        _refuses(linear, B.GHD_ERR_ALIGN, **{name: FAKE + 8})
    for kw in ({"M": 0}, {"M": 129}, {"N": 0}, {"K": 60, "ldx": 64}, {"group": 16}, {"group": 0}, {"flags": 2}, {"ldx": 56}, {"ldy": 63}):
        _refuses(linear, B.GHD_ERR_SHAPE, **kw)
    _refuses(linear, B.GHD_ERR_ALIGN, ldx=68)
    _refuses(linear, B.GHD_ERR_ALIGN, ws=FAKE + 8)
    _refuses(linear, B.GHD_ERR_WORKSPACE, ws=None)
    _refuses(linear, B.GHD_ERR_WORKSPACE, n=16)

    def pack(dst=FAKE, codes=FAKE, scales=FAKE, zeros=FAKE, N=16, K=64, group=32):
        return lib.ghd_pack_weight_q4(dst, codes, scales, zeros, N, K, group, None)

    for name in ("dst", "codes", "scales"):
        _refuses(pack, B.GHD_ERR_NULL, **{name: None})
    for kw in ({"N": 0}, {"K": 4}, {"K": 70}, {"group": 256}):
        _refuses(pack, B.GHD_ERR_SHAPE, **kw)
    _refuses(pack, B.GHD_ERR_ALIGN, dst=FAKE + 4)
    _refuses(pack, B.GHD_ERR_ALIGN, scales=FAKE + 1)


def test_cache_calls_refuse_bad_arguments(lib):
    kv = (B.KV * 2)(B.KV(FAKE, FAKE), B.KV(FAKE, FAKE))
    half = (B.KV * 2)(B.KV(FAKE, FAKE), B.KV(FAKE, None))
    odd = (B.KV * 2)(B.KV(FAKE, FAKE + 8), B.KV(FAKE, FAKE))

    def append(kv=kv, k=FAKE, v=FAKE, q=FAKE, qo=FAKE, parent=FAKE, M=8, kv_len=10, nh=4, nkv=2, d=64, cap=64, lk=128, lv=128,
               lq=256, lqo=256, base=10000.0):
        return lib.ghd_kv_append_q4(kv, k, v, q, qo, parent, M, kv_len, nh, nkv, d, cap, lk, lv, lq, lqo, base, None)

    for kw in ({"kv": None}, {"k": None}, {"v": None}, {"qo": None}, {"kv": (B.KV * 1)(B.KV(None, FAKE))}):
        _refuses(append, B.GHD_ERR_NULL, **kw)
    for kw in ({"M": 0}, {"M": 129, "cap": 1024}, {"kv_len": -1}, {"nkv": 0}, {"nh": 0}, {"nh": 257}, {"d": 96}, {"lk": 126}, {"lv": 0},
               {"lq": 254}, {"lqo": 254}, {"base": -1.0}, {"base": 0.0}, {"base": float("nan")}):
        _refuses(append, B.GHD_ERR_SHAPE, **kw)
    for kw in ({"cap": 0}, {"cap": 48}, {"kv_len": 57}, {"cap": 1 << 25}):
        _refuses(append, B.GHD_ERR_CAPACITY, **kw)
    for kw in ({"kv": odd}, {"k": FAKE + 2}, {"v": FAKE + 2}, {"q": FAKE + 2}, {"qo": FAKE + 2}, {"parent": FAKE + 2}, {"lk": 129},
               {"lv": 129}, {"lq": 257}, {"lqo": 257}):
        _refuses(append, B.GHD_ERR_ALIGN, **kw)

    def commit(kv=kv, L=2, nkv=2, d=64, cap=64, res=FAKE, M=8, kv_len=10):
        return lib.ghd_commit_path_q4(kv, L, nkv, d, cap, res, M, kv_len, None)

    for kw in ({"kv": None}, {"res": None}, {"kv": half}):
        _refuses(commit, B.GHD_ERR_NULL, **kw)
    for kw in ({"L": 0}, {"L": 49}, {"M": 0}, {"M": 129}, {"kv_len": -1}, {"nkv": 0}, {"d": 32}):
        _refuses(commit, B.GHD_ERR_SHAPE, **kw)
    for kw in ({"cap": 40}, {"kv_len": 57}):
        _refuses(commit, B.GHD_ERR_CAPACITY, **kw)
    for kw in ({"kv": odd}, {"res": FAKE + 1}):
        _refuses(commit, B.GHD_ERR_ALIGN, **kw)

    def read(k=FAKE, v=FAKE, kv=kv, L=2, nkv=2, d=64, cap=64, row0=0, rows=64):
        return lib.ghd_kv_read_q4(k, v, kv, L, nkv, d, cap, row0, rows, None)

    for kw in ({"kv": None}, {"k": None}, {"v": None}, {"kv": half}):
        _refuses(read, B.GHD_ERR_NULL, **kw)
    for kw in ({"L": 0}, {"L": 49}, {"row0": -1}, {"rows": 0}, {"d": 256}):
        _refuses(read, B.GHD_ERR_SHAPE, **kw)
    for kw in ({"row0": 1}, {"rows": 65}):
        _refuses(read, B.GHD_ERR_CAPACITY, **kw)
    for kw in ({"kv": odd}, {"k": FAKE + 8}, {"v": FAKE + 8}):
        _refuses(read, B.GHD_ERR_ALIGN, **kw)


@pytest.mark.parametrize("name", ["ghd_tree_attention_q4", "ghd_masked_attention_q4"])
def test_attention_refuses_bad_arguments(lib, name):
    kv = (B.KV * 1)(B.KV(FAKE, FAKE))

    def call(out=FAKE, q=FAKE, kv=kv, rel=FAKE, M=8, kv_len=10, nh=4, nkv=2, d=64, cap=64, ws=FAKE, n=1 << 30):
        return getattr(lib, name)(out, q, kv, rel, M, kv_len, nh, nkv, d, cap, 0.125, ws, n, None)

    for kw in ({"out": None}, {"q": None}, {"kv": None}, {"rel": None}, {"kv": (B.KV * 1)(B.KV(FAKE, None))}):
        _refuses(call, B.GHD_ERR_NULL, **kw)
    for kw in ({"M": 0}, {"M": 129}, {"kv_len": -1}, {"nh": 0}, {"nh": 258}, {"nkv": 0}, {"nkv": 3}, {"nh": 2, "nkv": 4}, {"d": 80}):
        _refuses(call, B.GHD_ERR_SHAPE, **kw)
    for kw in ({"cap": 33}, {"kv_len": 57}):
        _refuses(call, B.GHD_ERR_CAPACITY, **kw)
    for kw in ({"out": FAKE + 8}, {"q": FAKE + 8}, {"rel": FAKE + 2}, {"ws": FAKE + 8}, {"kv": (B.KV * 1)(B.KV(FAKE + 4, FAKE))}):
        _refuses(call, B.GHD_ERR_ALIGN, **kw)
    _refuses(call, B.GHD_ERR_WORKSPACE, ws=None)
    _refuses(call, B.GHD_ERR_WORKSPACE, n=0)


def test_linear_refuses_rows_too_far_apart(lib):
    """x is read at 32-bit byte offsets: rows at most 2^23 apart, 2^30 numbers in all."""
    def linear(M, K, ldx):
        return lib.ghd_linear_q4(FAKE, FAKE, FAKE, M, 64, K, 32, ldx, 64, 0, FAKE, 0, None)

    assert linear(1, 64, (1 << 23) + 8) == B.GHD_ERR_SHAPE
    assert linear(128, 64, 1 << 23) == B.GHD_ERR_WORKSPACE          # (127 * 2^23 < 2^30: only the workspace is too small)
    assert linear(128, 65536, 1 << 23) == B.GHD_ERR_WORKSPACE
