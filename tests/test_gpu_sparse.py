"""Block bounds, block selection and sparse attention against plain 64-bit forms."""
import math

import pytest
import torch

import sparse_plain as P
from paper_2505_23219_amd import binding as B, workloads as wl

pytestmark = pytest.mark.gpu


def _gen(seed):
    return torch.Generator().manual_seed(seed)


def _cache(nkv, rows, d, seed, layout="heads"):
    """Keys and values on the CPU, and on the GPU as the calls take them; rows of a passage of 64 are alike."""
    g = _gen(seed)
    k = torch.randn(nkv, rows, d, generator=g)
    k += torch.randn(nkv, -(-rows // 64), 1, d, generator=g).repeat_interleave(64, dim=1)[:, :rows].reshape(nkv, rows, d) \
        if rows else 0
    k = (k * torch.exp(0.5 * torch.randn(nkv, 1, d, generator=g))).half()
    v = torch.randn(nkv, d, rows, generator=g).half()
    kd = k.cuda() if layout == "heads" else k.cuda().transpose(0, 1).contiguous().transpose(0, 1)
    return k, v, kd, v.cuda()


def _bounds(k, kd, n, rows):
    nkv, _, d = k.shape
    b = B.BlockBounds(nkv, d, rows)
    B.ghd_block_bounds(b, kd, 0, n)
    return b


# ---- bounds ------------------------------------------------------------------------------
@pytest.mark.parametrize("nkv,d,rows,layout", [(1, 64, 64, "heads"), (3, 128, 200, "heads"), (8, 128, 1024, "tokens"),
                                               (5, 64, 719, "tokens"), (1, 128, 63, "heads")])
def test_bounds(nkv, d, rows, layout):
    k, _, kd, _ = _cache(nkv, rows, d, rows, layout)
    n = rows // 64
    b = _bounds(k, kd, n, rows)
    hi, lo = B.ghd_block_bounds_read(b, 0, n)
    want = P.read(P.bounds(k, n))
    assert torch.equal(hi.cpu().double(), want[0]) and torch.equal(lo.cpu().double(), want[1])
    if n:                                        # they are bounds, but for the codes' end at 127
        x = k[:, :n * 64].view(nkv, n, 64, d).float()
        s = P.bounds(k, n)[2].float()[..., None]
        assert (hi.cpu() >= x.amax(2) - s).all() and (lo.cpu() <= x.amin(2) + s).all()


def test_bounds_of_odd_numbers():
    d, n = 64, 9
    k = torch.randn(1, n * 64, d, generator=_gen(5)).half()
    k[0, 0:64] = 0
    k[0, 64:128] = -k[0, 64:128].abs() - 1                  # no channel reaches 0
    k[0, 130, 3] = math.inf
    k[0, 200, 63] = math.nan
    k[0, 256:320] = 2.0 ** -24 * torch.randint(-3, 4, (64, d), generator=_gen(6)).half()
    k[0, 320:384] = 65504.0
    k[0, 384:448] = -0.0
    k[0, 450, 7] = -math.inf
    k[0, 512:576] = torch.where(k[0, 512:576] > 0, 127.9, -127.9).half()
    b = _bounds(k, k.cuda(), n, n * 64)
    hi, lo = B.ghd_block_bounds_read(b, 0, n)
    want = P.read(P.bounds(k, n))
    assert torch.equal(hi.cpu().double(), want[0]) and torch.equal(lo.cpu().double(), want[1])
    assert torch.isinf(hi[0, [2, 3, 7]]).all() and torch.isfinite(hi[0, [0, 1, 4, 5, 6, 8]]).all()


def test_bounds_of_a_range_leave_the_others():
    k, _, kd, _ = _cache(4, 640, 128, 1)
    b = _bounds(k, kd, 10, 640)
    before = b.data.clone()
    kd[:, 64 * 3:64 * 5] *= 2
    B.ghd_block_bounds(b, kd, 3, 2)
    B.ghd_block_bounds(b, kd, 7, 0)
    want = _bounds(kd.cpu(), kd, 10, 640)
    assert torch.equal(b.data, want.data) and not torch.equal(b.data, before)


# ---- selection ---------------------------------------------------------------------------
def _check_select(q, k, kd, kv_len, count, sinks, recent, **kw):
    n = kv_len // 64
    b = _bounds(k, kd, n, kd.shape[1])
    got = B.ghd_block_select(q.cuda(), b, kv_len, count, sinks=sinks, recent=recent, **kw)
    want = P.words(P.select(P.scores(q, P.bounds(k, n)), count, sinks, recent))
    assert torch.equal(got.cpu(), want)
    return got


@pytest.mark.parametrize("M,nh,nkv,d,kv_len,count,sinks,recent", [
    (1, 8, 8, 128, 64, 1, 0, 0), (1, 8, 2, 128, 2000, 9, 1, 2), (5, 20, 4, 64, 1931, 7, 0, 1), (16, 4, 4, 64, 4095, 31, 2, 2),
    (17, 6, 3, 128, 1100, 5, 0, 0), (64, 2, 2, 128, 1300, 3, 1, 1), (65, 4, 1, 64, 700, 10, 1, 1), (128, 2, 2, 64, 1000, 6, 3, 3),
    (3, 16, 1, 128, 17000, 64, 1, 1), (2, 2, 2, 64, 33000, 300, 1, 1), (4, 4, 4, 128, 640, 10, 1, 1), (4, 4, 4, 128, 640, 50, 20, 20),
    (6, 2, 1, 64, 50000, 40, 1, 1), (9, 2, 1, 64, 100000, 70, 1, 2), (70, 1, 1, 64, 140000, 20, 0, 1), (2, 2, 1, 64, 330000, 100, 1, 1),
    (2, 4, 2, 128, 700, 0, 0, 0), (2, 4, 2, 128, 700, 4, 4, 0), (2, 4, 2, 64, 700, 4, 0, 4), (1, 256, 1, 64, 300, 2, 0, 0)])
def test_select(M, nh, nkv, d, kv_len, count, sinks, recent):
    k, _, kd, _ = _cache(nkv, kv_len + M, d, kv_len + M)
    q = torch.randn(M, nh, d, generator=_gen(M)).half()
    _check_select(q, k, kd, kv_len, count, sinks, recent)


@pytest.mark.parametrize("M,nh,nkv,d,kv_len,count,sinks,recent", [
    (128, 8, 8, 64, 64 * 128, 5, 1, 1), (128, 8, 8, 64, 64 * 129, 9, 0, 0), (127, 9, 9, 64, 64 * 512, 40, 2, 1), (128, 8, 8, 128, 64 * 513, 33, 1, 2),
    (100, 22, 11, 64, 64 * 1100 + 5, 17, 0, 0), (128, 8, 8, 64, 64 * 2048, 60, 1, 1), (128, 8, 8, 64, 64 * 2049, 60, 1, 1),
    (20, 104, 104, 64, 64 * 130, 7, 1, 1), (16, 4, 4, 64, 64 * 129, 128, 0, 0), (128, 17, 17, 64, 64 * 100, 3, 0, 1)])
def test_select_of_many_picks(M, nh, nkv, d, kv_len, count, sinks, recent):
    """1024 picks and more, and few of them, on either side of what one launch and one workgroup take."""
    test_select(M, nh, nkv, d, kv_len, count, sinks, recent)


@pytest.mark.parametrize("M,n", [(128, 200), (128, 600), (128, 1200)])
def test_many_picks_of_equal_blocks(M, n):
    some = torch.randn(2, 64, 64, generator=_gen(2)).half()
    k = some[torch.arange(n) * 7 % 2].reshape(1, n * 64, 64).repeat(8, 1, 1)
    q = torch.randn(M, 8, 64, generator=_gen(9)).half()
    for count in (1, 130, n - 1):
        _check_select(q, k, k.cuda(), n * 64, count, 1, 0)


@pytest.mark.parametrize("M,n", [(3, 300), (3, 700), (9, 900), (6, 1500), (1, 5000)])
@pytest.mark.parametrize("kinds", [1, 2, 5])
def test_select_takes_the_lowest_of_equal_blocks(kinds, M, n):
    d = 64
    some = torch.randn(kinds, 64, d, generator=_gen(kinds)).half()
    k = some[torch.arange(n) * 7 % kinds].reshape(1, n * 64, d).repeat(2, 1, 1)
    q = torch.randn(M, 2, d, generator=_gen(9)).half()
    for count in (1, 2, 257, n - 1):
        _check_select(q, k, k.cuda(), n * 64, count, 1, 0)


def test_select_with_numbers_that_are_none():
    k, _, _, _ = _cache(2, 900, 64, 4)
    k[0, 100, 3], k[0, 700, 5], k[1, 320, 0] = math.nan, math.inf, -math.inf
    q = torch.randn(6, 4, 64, generator=_gen(2)).half()
    q[0, 0, 3], q[1, 2, 0], q[2] = math.nan, math.inf, 0.0
    q[3] = q[3] * 1e-7
    q[4, 0] = 65504.0
    for count in (1, 2, 3, 6):
        _check_select(q, k, k.cuda(), 896, count, 0, 0)


def test_select_writes_all_of_its_words_and_no_others():
    k, _, kd, _ = _cache(2, 800, 64, 4)
    q = torch.randn(70, 2, 64, generator=_gen(2)).half()
    want = _check_select(q, k, kd, 770, 4, 1, 1)
    room = torch.full((want.numel() + 2,), -1, dtype=torch.int64, device="cuda")
    ws = torch.full((B.ghd_block_select_workspace_bytes(70, 770, 2),), 255, dtype=torch.uint8, device="cuda")
    got = B.ghd_block_select(q.cuda(), _bounds(k, kd, 12, 800), 770, 4, sel=room[1:-1].view(want.shape), ws=ws)
    assert torch.equal(got, want) and room[0] == -1 and room[-1] == -1
    empty = B.ghd_block_select(q.cuda(), _bounds(k, kd, 12, 800), 63, 4)
    assert empty.shape == (2, 2, 0)


# ---- attention ---------------------------------------------------------------------------
def _tolerance(size, want, q, k, v, scale, keys):
    """Probabilities are rounded to fp16 (2^-11, against a sum that is at least 1; what is below 2^-14 by at most 2^-25), their sum is
    that of the rounded ones, the result is rounded to fp16.  A score of d products in 32 bits is off by at most d 2^-24 of the
    sum of their sizes, and the exponential by a few units in the last place."""
    d = q.shape[2]
    terms = (q.double().abs().amax((0, 1)) * k.double().nan_to_num(0, 0, 0).abs().amax((0, 1))).sum().item() * abs(scale)
    by_score = 2 * (d * 2.0 ** -24 * terms + 2.0 ** -21)
    small = keys * 2.0 ** -25 * v.double().nan_to_num(0, 0, 0).abs().max().item()
    return (2 * 2.0 ** -11 + by_score) * size + 2.0 ** -11 * want.abs() + small + 2.0 ** -24


def _selection(nkv, M, n, count, seed, pool=None):
    g = _gen(seed)
    sel = torch.zeros((nkv, M, n), dtype=torch.bool)
    for h in range(nkv):
        of = torch.randperm(n, generator=g)[:pool or n]
        for i in range(M):
            sel[h, i, of[torch.randperm(len(of), generator=g)[:count]]] = True
    return sel


def _relation(kind, M, seed):
    """(arguments for the call, which drafted tokens a token sees)"""
    if kind in ("chain", "random", "star"):
        parent = {"chain": wl.tree_chain, "star": wl.tree_star}.get(kind, lambda m: wl.tree_random(m, 5, seed))(M).tolist()
        return {"parent": torch.tensor(parent, dtype=torch.int32, device="cuda")}, P.ancestors(parent)
    see = torch.rand((M, M), generator=_gen(seed)) < {"none": 0.0, "sparse": 0.3, "all": 2.0}[kind]
    if kind == "sparse":
        see[::3] = False
    return {"mask": P.mask_words(see).cuda()}, see


def _check(M, nh, nkv, d, kv_len, sel, kind, layout="heads", scale=None, pad=0, seed=0, spoil=True, **kw):
    rows = -(-(kv_len + M + pad) // 8) * 8
    k, v, kd, vd = _cache(nkv, rows, d, seed + kv_len + M, layout)
    q = torch.randn(M, nh, d, generator=_gen(seed + 1)).half()
    if spoil:                                    # rows that are not there hold anything
        kd[:, kv_len + M:] = math.nan
        vd[:, :, kv_len + M:] = math.nan
    rel, see = _relation(kind, M, seed)
    scale = d ** -0.5 if scale is None else scale
    want, size = P.attend(q, k, v, sel, see, kv_len, scale)
    got = B.ghd_sparse_attention(q.cuda(), kd, vd, P.words(sel).cuda(), kv_len, scale=scale, **rel, **kw)
    off = (got.cpu().double() - want).abs()
    tol = _tolerance(size, want, q, k[:, :kv_len + M], v[:, :, :kv_len + M], scale, kv_len + M)
    assert (off <= tol).all(), ((off / tol).max().item(), (off > tol).nonzero()[:3].tolist())
    return got, want


@pytest.mark.parametrize("M,nh,nkv,d,kv_len,count,kind,layout", [
    (1, 1, 1, 64, 0, 0, "chain", "heads"), (1, 2, 2, 128, 1, 0, "chain", "heads"), (1, 8, 2, 128, 63, 0, "chain", "tokens"),
    (1, 4, 4, 128, 64, 1, "chain", "heads"), (1, 32, 8, 128, 4099, 11, "chain", "heads"), (3, 4, 2, 64, 130, 1, "random", "heads"),
    (7, 20, 4, 64, 777, 5, "sparse", "tokens"), (16, 4, 4, 128, 1000, 4, "random", "heads"), (17, 2, 2, 64, 960, 3, "star", "heads"),
    (37, 10, 2, 64, 777, 5, "sparse", "tokens"), (64, 2, 2, 128, 2051, 9, "random", "heads"), (65, 3, 3, 64, 650, 2, "chain", "heads"),
    (100, 4, 2, 128, 901, 6, "all", "heads"), (128, 2, 2, 128, 1501, 8, "chain", "tokens"), (128, 4, 1, 64, 320, 2, "random", "heads"),
    (5, 16, 1, 128, 513, 2, "random", "heads"), (2, 256, 2, 64, 200, 1, "chain", "heads"), (33, 40, 8, 128, 333, 2, "random", "heads")])
def test_attention(M, nh, nkv, d, kv_len, count, kind, layout):
    n = kv_len // 64
    _check(M, nh, nkv, d, kv_len, _selection(nkv, M, n, min(count, n), M + n), kind, layout)


@pytest.mark.parametrize("M,nh,nkv,d,kv_len", [(16, 320, 40, 128, 333), (3, 312, 39, 64, 200), (1, 1024, 1, 128, 150), (5, 1024, 256, 64, 130),
                                               (128, 1024, 2, 64, 70)])
def test_many_query_heads(M, nh, nkv, d, kv_len):
    """Tokens of all heads together, 40 key heads of eight and a row of 1024 heads among them."""
    n = kv_len // 64
    _check(M, nh, nkv, d, kv_len, _selection(nkv, M, n, min(2, n), M), "random", "tokens")
    k, _, kd, _ = _cache(nkv, kv_len + M, d, kv_len)
    _check_select(torch.randn(M, nh, d, generator=_gen(M)).half(), k, kd, kv_len, 1, 0, 0)


def test_nothing_selected_and_nothing_seen():
    sel = torch.zeros((2, 9, 4), dtype=torch.bool)
    sel[1, 2, 3] = sel[0, 4, 0] = True
    got, want = _check(9, 2, 2, 64, 256, sel, "none")
    assert (got[:, 0][[0, 1, 2, 3, 5, 6, 7, 8]] == 0).all() and (want[4, 0] != 0).any()
    _check(9, 2, 2, 64, 256, sel, "sparse")
    _check(9, 4, 2, 128, 270, torch.zeros((2, 9, 4), dtype=torch.bool), "none")


@pytest.mark.parametrize("kind", ["none", "sparse"])
def test_nothing_committed(kind):
    _check(21, 4, 2, 128, 0, torch.zeros((2, 21, 0), dtype=torch.bool), kind)


@pytest.mark.parametrize("scale", [0.0, -0.1, 0.5, 1e-30])
def test_scales(scale):
    _check(6, 4, 2, 64, 400, _selection(2, 6, 6, 3, 1), "random", scale=scale)


@pytest.mark.parametrize("M,rep,d,kv_len", [(1, 1, 64, 700), (7, 4, 128, 700), (40, 1, 64, 1500), (100, 1, 128, 300), (128, 2, 64, 300)])
@pytest.mark.parametrize("scale", [None, -3.0, 1e9])
def test_the_largest_scores(M, rep, d, kv_len, scale):
    """Queries and keys of 60000 with any signs: scores differ by 2^30 and more, so a row has the value of its best key, bit for bit."""
    nkv, g = 2, _gen(M + d)
    sign = lambda *n: (torch.randint(2, n, generator=g) * 2 - 1).half()
    rows, n = -(-(kv_len + M) // 8) * 8, kv_len // 64
    k, v = 60000 * sign(nkv, rows, d), torch.randn(nkv, d, rows, generator=g).half()
    q = 60000 * sign(M, nkv * rep, d)
    at = torch.randperm(kv_len, generator=g)[:M * rep].view(M, rep)
    for h in range(nkv):                         # the key of a row's own signs, or of the opposite ones
        k[h, at.view(-1)] = (q[:, h * rep:(h + 1) * rep].reshape(M * rep, d) * (-1 if scale is not None and scale < 0 else 1))
    sel = torch.full((nkv, -(-M // 64), n), -1, dtype=torch.int64, device="cuda")
    rel, _ = _relation("none", M, 1)
    got = B.ghd_sparse_attention(q.cuda(), k.cuda(), v.cuda(), sel, kv_len, scale=scale, **rel).cpu()
    for h in range(nkv):
        assert torch.equal(got[:, h * rep:(h + 1) * rep], v[h][:, at].permute(1, 2, 0))


def test_all_blocks_are_all_of_the_attention():
    for M, kv_len in ((1, 700), (24, 1000), (128, 200)):
        nh, d = 8, 128
        k, v, kd, vd = _cache(nh, -(-(kv_len + M) // 8) * 8, d, 3)
        q = torch.randn(M, nh, d, generator=_gen(4)).half().cuda()
        parent = torch.from_numpy(wl.tree_random(M, 6, 1)).cuda()
        sel = torch.full((nh, -(-M // 64), kv_len // 64), -1, dtype=torch.int64, device="cuda")
        got = B.ghd_sparse_attention(q, kd, vd, sel, kv_len, parent=parent)
        full = B.ghd_tree_attention(q, kd, vd, parent, kv_len)
        # both round probabilities and results: 2^-11 of sums of p |v| twice, and of the results
        bound = 2 * (2 * 2.0 ** -11 * vd.abs().max() + 2.0 ** -11 * full.abs())
        assert ((got - full).abs() <= bound).all()


def test_bits_of_no_token_say_nothing():
    q = torch.randn(5, 2, 64, generator=_gen(4)).half().cuda()
    _, _, kd, vd = _cache(2, 648, 64, 3)
    sel, parent = P.words(_selection(2, 5, 10, 2, 1)).cuda(), torch.from_numpy(wl.tree_chain(5)).cuda()
    want = B.ghd_sparse_attention(q, kd, vd, sel, 640, parent=parent)
    assert torch.equal(B.ghd_sparse_attention(q, kd, vd, sel | -32, 640, parent=parent), want)


@pytest.mark.parametrize("M,rep,d", [(1, 4, 128), (9, 1, 64), (40, 2, 128), (70, 1, 128)])
@pytest.mark.parametrize("bad", [math.nan, math.inf])
def test_a_bad_row_reaches_who_sees_it(M, rep, d, bad):
    """An infinity or NaN in a value or key of a block, of the rows behind the blocks, or of a drafted row."""
    nkv, kv_len, n = 2, 700, 10
    k, v, kd, vd = _cache(nkv, 776, d, 3)
    q = torch.randn(M, nkv * rep, d, generator=_gen(4)).half().cuda()
    sel = _selection(nkv, M, n, 3, 1, pool=6)
    rel, see = _relation("random", M, 1)
    clean = B.ghd_sparse_attention(q, kd, vd, P.words(sel).cuda(), kv_len, **rel)
    for row, seen_by in ((5 * 64 + 9, sel[:, :, 5]), (660, torch.ones(nkv, M, dtype=torch.bool)),
                         (kv_len + M // 2, see[:, M // 2].expand(nkv, M))):
        for of_keys in (False, True):
            kb, vb = kd.clone(), vd.clone()
            if of_keys:
                kb[1, row, 5] = bad
            else:
                vb[1, 5, row] = bad
            got = B.ghd_sparse_attention(q, kb, vb, P.words(sel).cuda(), kv_len, **rel).cpu()
            for i in range(M):
                mine, other = got[i, rep:], clean[i, rep:].cpu()
                assert torch.equal(got[i, :rep], clean[i, :rep].cpu())       # the other key head
                if not seen_by[1, i]:
                    # (the values are taken one by one then, in another order: twice what that rounds)
                    assert ((mine - other).abs() <= 2.0 ** -10 * (other.abs() + 0.05)).all()
                elif of_keys:
                    # (an infinite key of a negative product has the probability 0)
                    assert not torch.isfinite(mine).all() or bad == math.inf
                else:
                    assert not torch.isfinite(mine[:, 5]).any()
                    keep = [c for c in range(d) if c != 5]
                    assert ((mine - other).abs() <= 2.0 ** -10 * (other.abs() + 0.05))[:, keep].all()


def test_a_token_whose_queries_are_none():
    """An infinity or NaN among a token's queries is that token's alone, bit for bit."""
    for M, rep, d in ((3, 2, 64), (24, 1, 128), (60, 1, 128), (100, 1, 64), (128, 2, 128)):
        _, _, kd, vd = _cache(2, 840, d, 3)
        q = torch.randn(M, 2 * rep, d, generator=_gen(4)).half().cuda()
        sel, (rel, _) = P.words(_selection(2, M, 10, 3, 1, pool=6)).cuda(), _relation("random", M, 1)
        want = B.ghd_sparse_attention(q, kd, vd, sel, 700, **rel)
        q[M // 2, 1, 5], q[M - 1, 0, 7] = math.nan, math.inf
        got = B.ghd_sparse_attention(q, kd, vd, sel, 700, **rel)
        same = torch.ones(M, 2 * rep, dtype=torch.bool)
        same[M // 2, 1] = same[M - 1, 0] = False
        assert torch.equal(got[same], want[same]) and torch.isnan(got[M // 2, 1]).all()


def test_in_place_over_any_workspace_and_behind_it():
    M, nh, nkv, d, kv_len = 12, 8, 2, 128, 3000
    _, _, kd, vd = _cache(nkv, 3016, d, 3)
    q = torch.randn(M, nh, d, generator=_gen(4)).half().cuda()
    sel, parent = P.words(_selection(nkv, M, 46, 9, 1)).cuda(), torch.from_numpy(wl.tree_random(M, 4, 2)).cuda()
    want = B.ghd_sparse_attention(q, kd, vd, sel, kv_len, parent=parent)
    need = B.ghd_sparse_attention_workspace_bytes(M, kv_len, nh, nkv, d)
    room = torch.full((need + 512,), 255, dtype=torch.uint8, device="cuda")
    mine = q.clone()
    got = B.ghd_sparse_attention(mine, kd, vd, sel, kv_len, parent=parent, ws=room[256:256 + need], out=mine)
    assert got is mine and torch.equal(got, want) and (room[:256] == 255).all() and (room[256 + need:] == 255).all()


def test_side_streams_and_graphs():
    """Calls on other streams, captured and replayed with changed inputs, two graphs over one workspace."""
    M, nh, nkv, d, kv_len = 20, 8, 4, 64, 2500
    _, _, kd, vd = _cache(nkv, 2560, d, 3)
    q, parent = torch.randn(M, nh, d, generator=_gen(4)).half().cuda(), torch.from_numpy(wl.tree_random(M, 4, 2)).cuda()
    bounds = B.BlockBounds(nkv, d, 2560)
    ws = B.workspace(max(B.ghd_block_select_workspace_bytes(M, kv_len, nkv), B.ghd_sparse_attention_workspace_bytes(M, kv_len, nh, nkv, d)))
    sel, out = torch.empty((nkv, 1, 39), dtype=torch.int64, device="cuda"), torch.empty_like(q)

    def step(count):
        B.ghd_block_bounds(bounds, kd, 0, 39)
        B.ghd_block_select(q, bounds, kv_len, count, sel=sel, ws=ws)
        B.ghd_sparse_attention(q, kd, vd, sel, kv_len, parent=parent, ws=ws, out=out)
    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    with torch.cuda.stream(side):
        step(5)
    torch.cuda.synchronize()
    graphs = []
    for count in (5, 9):
        g = torch.cuda.CUDAGraph()
        with torch.cuda.graph(g):
            step(count)
        graphs.append((g, count))
    for turn in range(4):
        q.copy_(torch.randn(M, nh, d, generator=_gen(40 + turn)).half())
        kd[:, 64 * turn:64 * turn + 64] *= 1.5
        for g, count in graphs:
            g.replay()
            torch.cuda.synchronize()
            got, picked = out.clone(), sel.clone()
            step(count)
            assert torch.equal(got, out) and torch.equal(picked, sel)


def test_offsets_beyond_four_gib():
    """Heads 5 GiB apart in both caches."""
    nkv, d, M, kv_len, apart = 3, 128, 4, 1000, (5 << 30) // 2
    k, v, _, _ = _cache(nkv, 1008, d, 3)
    store = torch.zeros(2 * apart + 1008 * d, dtype=torch.float16, device="cuda")
    kd, vd = store.as_strided((nkv, 1008, d), (apart, d, 1)), store.as_strided((nkv, d, 1008), (apart, 1008, 1))
    q, parent = torch.randn(M, 6, d, generator=_gen(4)).half().cuda(), torch.from_numpy(wl.tree_chain(M)).cuda()
    sel = P.words(_selection(nkv, M, 15, 4, 1)).cuda()
    kd.copy_(k.cuda())
    far_bounds, near = B.BlockBounds(nkv, d, 1008), _bounds(k, k.cuda(), 15, 1008)
    B.ghd_block_bounds(far_bounds, kd, 0, 15)
    assert torch.equal(far_bounds.data, near.data)
    want = B.ghd_sparse_attention(q, k.cuda(), v.cuda(), sel, kv_len, parent=parent)
    assert torch.equal(B.ghd_sparse_attention(q, kd, v.cuda(), sel, kv_len, parent=parent), want)
    vd.copy_(v.cuda())
    assert torch.equal(B.ghd_sparse_attention(q, k.cuda(), vd, sel, kv_len, parent=parent), want)


def test_a_long_context():
    """2^21 committed rows, one head; what is read is checked against the same rows side by side."""
    kv_len, d, M = 1 << 21, 64, 2
    kd = torch.randn(1, kv_len + 8, d, generator=torch.Generator("cuda").manual_seed(1), device="cuda").half()
    vd = torch.randn(1, d, kv_len + 8, generator=torch.Generator("cuda").manual_seed(2), device="cuda").half()
    bounds, n = B.BlockBounds(1, d, kv_len + 8), kv_len // 64
    B.ghd_block_bounds(bounds, kd, 0, n)
    q = torch.randn(M, 4, d, generator=_gen(4)).half().cuda()
    sel = B.ghd_block_select(q, bounds, kv_len, 50)
    assert ((sel[0, 0] & 1).sum() == 50) and ((sel[0, 0] >> 1 & 1).sum() == 50)
    b = P.bounds(kd[:, :64 * 300].cpu(), 300)
    some = B.ghd_block_select(q, bounds, 64 * 300, 50)
    assert torch.equal(some.cpu(), P.words(P.select(P.scores(q.cpu(), b), 50, 1, 1)))
    parent = torch.from_numpy(wl.tree_chain(M)).cuda()
    got = B.ghd_sparse_attention(q, kd, vd, sel, kv_len, parent=parent)
    at = sel[0, 0].nonzero()[:, 0]
    rows = torch.cat([(at[:, None] * 64 + torch.arange(64, device="cuda")).reshape(-1), torch.arange(kv_len, kv_len + M, device="cuda")])
    want, size = P.attend(q.cpu(), kd[:, rows].cpu(), vd[:, :, rows].cpu(),
                          torch.stack([sel[0, 0][at] >> i & 1 for i in range(M)])[None].bool().cpu(), P.ancestors([-1, 0]),
                          len(at) * 64, d ** -0.5)
    off = (got.cpu().double() - want).abs()
    assert (off <= _tolerance(size, want, q.cpu(), kd[:, rows].cpu(), vd[:, :, rows].cpu(), d ** -0.5, len(rows))).all()


def test_the_same_twice():
    _, _, kd, vd = _cache(8, 4160, 128, 3)
    q, parent = torch.randn(64, 32, 128, generator=_gen(4)).half().cuda(), torch.from_numpy(wl.tree_random(64, 4, 2)).cuda()
    bounds = B.BlockBounds(8, 128, 4160)
    B.ghd_block_bounds(bounds, kd, 0, 64)
    first = None
    for _ in range(5):
        sel = B.ghd_block_select(q, bounds, 4096, 12)
        out = B.ghd_sparse_attention(q, kd, vd, sel, 4096, parent=parent)
        if first is not None:
            assert torch.equal(sel, first[0]) and torch.equal(out, first[1])
        first = (sel, out)
