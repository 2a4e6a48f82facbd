"""Plain numpy forms of the 4-bit formats and operators, in 64 bits except where a format says
which fp16 or fp32 number is stored.  Written from the formulas in include/ghd.h."""
import numpy as np

GROUP = 32


def quantise(x):
    """x fp16 [..., d] -> (codes [..., d], lo, s fp16 [..., d / 32]): the IEEE operations of the format."""
    g = x.reshape(x.shape[:-1] + (-1, GROUP)).astype(np.float32)
    finite = np.isfinite(g).all(-1)
    gz = np.where(finite[..., None], g, np.float32(0))
    lo = gz.min(-1)
    s = ((gz.max(-1) - lo) / np.float32(15)).astype(np.float16)
    over = lo + np.float32(15) * s.astype(np.float32) >= 65520
    s = np.where(over, (s.view(np.uint16) - over.astype(np.uint16)).view(np.float16), s)
    sf = s.astype(np.float32)[..., None]
    code = np.where(sf > 0, (gz - lo[..., None]) / np.where(sf > 0, sf, np.float32(1)), 0)
    code = np.clip(np.rint(code), 0, 15).astype(np.int64)
    s = np.where(finite, s, np.float16(np.nan))
    return code.reshape(x.shape), lo.astype(np.float16), s


def values(code, lo, s):
    """What codes stand for: fp16(lo + code * s), rounded once (64 bits hold the sum exactly)."""
    g = code.reshape(code.shape[:-1] + (-1, GROUP)).astype(np.float64)
    v = lo.astype(np.float64)[..., None] + g * s.astype(np.float64)[..., None]
    return v.astype(np.float16).reshape(code.shape)


def held(x):
    return values(*quantise(x))


def depths(parent):
    out = [0] * len(parent)
    for i in range(1, len(parent)):
        out[i] = out[parent[i]] + 1
    return np.array(out)


def sees_of_parent(parent):
    M = len(parent)
    see = np.zeros((M, M), bool)
    for i in range(M):
        j = i
        while j >= 0:
            see[i, j] = True
            j = parent[j]
    return see


def mask_words(see):
    out = np.zeros((see.shape[0], 2), np.uint64)
    for i, row in enumerate(see):
        for j in np.nonzero(row)[0]:
            out[i, j // 64] |= np.uint64(1) << np.uint64(j % 64)
    return out.view(np.int64)


def turn(x, pos, base):
    """x [M, heads, d] in 64 bits, turned at pos [M]."""
    x, d = x.astype(np.float64), x.shape[-1]
    ang = np.asarray(pos, np.float64)[:, None, None] * base ** (-2.0 * np.arange(d // 2) / d)
    a, b = x[..., :d // 2], x[..., d // 2:]
    return np.concatenate([a * np.cos(ang) - b * np.sin(ang), b * np.cos(ang) + a * np.sin(ang)], -1)


def attention(q, k, v, see, kv_len, scale):
    """q [M, nh, d], k and v [T, nkv, d], see [M, M] -> (out, bound) [M, nh, d]: the result in 64 bits, and
    how far fp16 probabilities, 32-bit sums and an fp16 result may be from it."""
    q, k, v = (t.astype(np.float64) for t in (q, k, v))
    M, nh, d = q.shape
    rep, T = nh // k.shape[1], k.shape[0]
    out, tol = np.zeros((M, nh, d)), np.zeros((M, nh, d))
    all_see = np.concatenate([np.ones((M, kv_len), bool), see], 1)
    for h in range(nh):
        kh, vh = k[:, h // rep], v[:, h // rep]
        for i in range(M):
            on = all_see[i]
            if not on.any():
                continue
            s = kh[on] @ q[i, h] * scale
            # a sum of d products in 32 bits, and its product with the scale
            ds = (d + 4) * 2.0 ** -24 * (np.abs(kh[on]) @ np.abs(q[i, h])).max() * abs(scale)
            e = np.exp(s - s.max())
            p = e / e.sum()
            out[i, h] = p @ vh[on]
            size = p @ np.abs(vh[on])
            # probabilities: rounded to fp16 (2^-11 of each, 2^-25 of the largest below fp16's normal range), their
            # exponent off by 2 ds and the exponential's own 2^-21, sums of T terms in 32 bits; the result rounded to fp16
            tol[i, h] = (2.0 ** -11 + 2.0 ** -21 + 4 * ds + T * 2.0 ** -23) * (size + np.abs(out[i, h])) \
                + 2.0 ** -25 * np.abs(vh[on]).sum(0) / e.sum() + 2.0 ** -11 * np.abs(out[i, h]) + 2.0 ** -25
    return out, tol


def unpack_weight(codes, scales, zeros, K, group):
    """codes uint8 [N, K / 2] -> W [N, K] in 64 bits."""
    c = np.empty((codes.shape[0], K))
    c[:, 0::2], c[:, 1::2] = codes & 15, codes >> 4
    z = np.full(scales.shape, 8.0) if zeros is None else zeros.astype(np.float64)
    at = np.arange(K) // group
    return (c - z[:, at]) * scales.astype(np.float64)[:, at]


def linear(x, W, out16):
    """-> (y, bound): sums of K products in 32 bits, at most one rounding for every eight products of a chain
    and 64 more where scales are applied and chains meet, then the result's own rounding."""
    x = x.astype(np.float64)
    y, size = x @ W.T, np.abs(x) @ np.abs(W).T
    tol = (x.shape[1] / 8 + 64) * 2.0 ** -24 * size
    if out16:
        tol = tol + 2.0 ** -11 * np.abs(y) + 2.0 ** -25
    return y, tol
