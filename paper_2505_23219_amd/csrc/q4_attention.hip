// Attention of the drafted tokens over a 4-bit cache.
//
// out[i, h] = softmax over the keys that node i sees of (scale q . K^) applied to V^, where K^ and V^ are the fp16
// numbers that the codes stand for (q4.h).  A key head's query rows - M nodes by nh / nkv heads - are the columns of
// S^T = K^ q^T and O^T = V^T P^T, so softmax statistics are a lane's own and the probabilities come out as the operand of
// the second product.  Running maximum and sum are kept in 32 bits; probabilities are rounded to fp16, relative to a maximum
// that lags by up to 2^8 (fp16 holds that as exactly, and sums are rescaled seldom).
//
// A wavefront takes 32 keys at a time by itself, codes straight into operand registers, and the wavefronts' states meet in LDS at
// the end.  Up to 16 query rows what counts is that the cache streams: a ring of two tiles a wavefront.  Above, blocks of two to
// four tiles of rows share a key's conversion, which takes longer than its products with one.  (Before, a wavefront had 16 rows,
// and operands converted by turns came through LDS with a barrier for every 32 keys: 64 rows of 32 heads over 2112 keys 16.0 us a
// call, this way 14.4; 128 of 40 over 8320 42.7 and 40.8; 37 of 20 heads of 64 channels, on 4 key heads, over 814 10.4 and 7.7.)
#include "q4.h"
#include "attention_impl.h"

namespace ghd {

typedef uint32_t word2 __attribute__((ext_vector_type(2)));
typedef uint32_t word4 __attribute__((ext_vector_type(4)));

// the lane's number, counted anew: nothing is kept in registers for it meanwhile
__device__ __forceinline__ int q4_lane()
{
    uint32_t zero = 0;
    asm volatile("" : "+s"(zero));
    return __builtin_amdgcn_mbcnt_hi(~0u, __builtin_amdgcn_mbcnt_lo(~0u, zero));
}

// does a node see any drafted key? (bits from M on say nothing)
__device__ __forceinline__ bool q4_sees(const uint64_t* mask, int node, int M)
{
    const uint64_t lo = M >= 64 ? ~0ull : (1ull << M) - 1, hi = M >= 128 ? ~0ull : M > 64 ? (1ull << (M - 64)) - 1 : 0;
    return (mask[2 * node] & lo) | (mask[2 * node + 1] & hi);
}

// The masks of all nodes to LDS.  Parents are asked for when a workgroup begins, their sets worked out by its first wavefront; the
// workgroup's barrier is the caller's.
struct Q4Masks {
    int up0, up1;
    bool needed;
    __device__ __forceinline__ Q4Masks(const Q4Attn& a, bool reaches, int wave, int lane) : up0(0), up1(0), needed(reaches)
    {
        if (reaches && !a.mask && wave == 0) {
            up0 = a.parent[min(lane, a.M - 1)];
            up1 = a.parent[min(lane + 64, a.M - 1)];
        }
    }
    __device__ __forceinline__ void store(const Q4Attn& a, int wave, int lane, uint64_t* s_mask) const
    {
        if (!needed) return;
        if (a.mask) {
            for (int e = threadIdx.x; e < 2 * a.M; e += blockDim.x) {
                const int left = a.M - 64 * (e & 1);               // bits of this word that mean something
                s_mask[e] = left >= 64 ? a.mask[e] : left <= 0 ? 0 : a.mask[e] & ((1ull << left) - 1);
            }
        } else if (wave == 0) {
            store_masks(tree_nodes<2, true>(up0, up1, a.M, lane), a.M, lane, s_mask);
        }
    }
};

// A head's tiles, of keys or of values.  Tiles at scalar offsets (below 2^31: 2^19 tiles of 2560 bytes), a lane's share at a 32-bit
// one: as pointers these are a pair of registers for every load.
struct Q4Head {
    __amdgpu_buffer_rsrc_t rows;
    __device__ __forceinline__ Q4Head(const char* base, int head, int tiles, int d)
        : rows(__builtin_amdgcn_make_buffer_rsrc((void*)(base + q4_tile_at(head, 0, tiles, d)), 0, tiles * q4_tile_bytes(d), 0x00027000))
    {
    }
    __device__ __forceinline__ half2_ get1(uint32_t tile, uint32_t at) const
    {
        return __builtin_bit_cast(half2_, __builtin_amdgcn_raw_buffer_load_b32(rows, at, tile, 0));
    }
    __device__ __forceinline__ word2 get2(uint32_t tile, uint32_t at) const
    {
        return __builtin_bit_cast(word2, __builtin_amdgcn_raw_buffer_load_b64(rows, at, tile, 0));
    }
    __device__ __forceinline__ word4 get4(uint32_t tile, uint32_t at) const
    {
        return __builtin_bit_cast(word4, __builtin_amdgcn_raw_buffer_load_b128(rows, at, tile, 0));
    }
};

// 16 keys of a tile (half h), as a lane (g, col) has them: operand row r is key 8 (r / 4) + 4 h + r % 4, so that a lane's 8
// scores of a column are those of keys 8 g .. 8 g + 7, the probabilities it holds in the second product.  Its channels, D / 4
// from g D / 4 on, are the k-steps' in turn.
template <int D>
struct Q4RawK {
    uint32_t w[D / 32];
    half2_ m;
    __device__ __forceinline__ void load(const Q4Head& head, uint32_t tile, int h, int col, int g)
    {
        const uint32_t key = 8u * (col >> 2) + (col & 3);          // of half 0
        if constexpr (D == 128) {
            const word4 v = head.get4(tile + h * 256, key * 64u + g * 16u);
#pragma unroll
            for (int s = 0; s < 4; ++s) w[s] = v[s];
            m = head.get1(tile + h * 64 + q4_codes_bytes(D), key * 16u + g * 4u);
        } else {
            const word2 v = head.get2(tile + h * 128, key * 32u + g * 8u);
            w[0] = v[0];
            w[1] = v[1];
            m = head.get1(tile + h * 32 + q4_codes_bytes(D), key * 8u + (g >> 1) * 4u);
        }
    }
    __device__ __forceinline__ half8 operand(const Q4Bits& bits, int s) const
    {
        return q4_values(bits, w[s], pair_of(m[0]), pair_of(m[1]));
    }
};

struct Q4Pairs {
    half2_ lo[4], s[4];                // of a lane's 8 keys
    __device__ __forceinline__ void set(half8 l, half8 sc)
    {
#pragma unroll
        for (int e = 0; e < 4; ++e) {
            lo[e] = (half2_){l[2 * e], l[2 * e + 1]};
            s[e] = (half2_){sc[2 * e], sc[2 * e + 1]};
        }
    }
};

// Values of rows that are not there may be anything, and 0 times anything is no 0: they count as 0.  So does what reads as NaN
// (a NaN was appended), which only reaches the rows that see it (q4_tile's `nan`); returned: which of the 8 keys those are.
__device__ __forceinline__ uint32_t q4_clean(half8& lo, half8& s, int key0, int total)
{
    word4 l = __builtin_bit_cast(word4, lo), c = __builtin_bit_cast(word4, s);
    const int there = total - key0;                            // so many of the 8 keys, from the first on
    uint32_t bad = 0;
#pragma unroll
    for (int p = 0; p < 4; ++p) {
        const uint32_t in = (there > 2 * p ? 0xffffu : 0u) | (there > 2 * p + 1 ? 0xffff0000u : 0u);
        // an exponent of all ones, plus one, carries into the sign
        const uint32_t odd = (((l[p] & 0x7c007c00u) + 0x04000400u) | ((c[p] & 0x7c007c00u) + 0x04000400u)) & 0x80008000u & in;
        const uint32_t keep = in & ~((odd >> 15) * 0xffffu);
        l[p] &= keep;
        c[p] &= keep;
        bad |= (odd >> 15 & 1u) << 2 * p | odd >> 31 << (2 * p + 1);
    }
    lo = __builtin_bit_cast(half8, l);
    s = __builtin_bit_cast(half8, c);
    return bad;
}

// scores to powers of two; above 0, so that minus infinity, the score of a key that is not seen, stays that (a NaN stays one, too)
__device__ __forceinline__ float q4_power(float scale) { return __builtin_elementwise_maximum(fabsf(scale) * 1.4426950408889634f, 1e-37f); }

// A row tile's state over the keys so far.
template <int D>
struct Q4State {
    floatx4 o[D / 16], l;              // l: the sum of the (rounded) probabilities, by a product with ones; four times the same
    float m;
    __device__ __forceinline__ Q4State() : l((floatx4){0.f, 0.f, 0.f, 0.f}), m(-INFINITY)
    {
#pragma unroll
        for (int ct = 0; ct < D / 16; ++ct) o[ct] = (floatx4){0.f, 0.f, 0.f, 0.f};
    }
    // Scores (of this lane's 8 keys) to probabilities: the highest, a new maximum if that is far above the old one, powers.  c, what
    // makes powers of two of scores, is above 0.
    __device__ __forceinline__ float highest(const floatx4 (&s)[2], float c) const
    {
        // (of the maximum that NaN passes through: fmaxf first takes every score through an instruction that quiets NaN)
        float top = s[0][0];
#pragma unroll
        for (int e = 1; e < 8; ++e) top = __builtin_elementwise_maximum(top, s[e >> 2][e & 3]);
        return max_over_groups(top) * c;
    }
    __device__ __forceinline__ void raise(float top)
    {
        const float now = fmaxf(m, top), r = m == now ? 1.f : __builtin_amdgcn_exp2f(m - now);
        l *= r;
#pragma unroll
        for (int ct = 0; ct < D / 16; ++ct) o[ct] *= r;
        m = now;
    }
    __device__ __forceinline__ half8 powers(const floatx4 (&s)[2], float c)
    {
        const float off = m == -INFINITY ? 0.f : -m;
        half2_ p[4];
#pragma unroll
        for (int e = 0; e < 4; ++e) {
            floatx2 x;
#pragma unroll
            for (int u = 0; u < 2; ++u) x[u] = __builtin_amdgcn_exp2f(fmaf(s[e >> 1][2 * (e & 1) + u], c, off));
            p[e] = __builtin_convertvector(x, half2_);
        }
        const half8 all = join(p[0], p[1], p[2], p[3]);
        const half_t one = (half_t)1.f;
        l = __builtin_amdgcn_mfma_f32_16x16x32_f16((half8){one, one, one, one, one, one, one, one}, all, l, 0, 0, 0);
        return all;
    }
};

// What a wavefront hands over of a row: maximum, sum, and the groups of channels that are NaN, a bit each (as a float's bits).
typedef floatx4 Q4Row;
__device__ __forceinline__ Q4Row q4_row(float m, float l, uint32_t nan, int shift)
{
    return (Q4Row){m, l, __builtin_bit_cast(float, nan >> shift), 0.f};
}

__device__ __forceinline__ uint32_t or_over_groups(uint32_t x)
{
    const int lane = q4_lane();
    x |= (uint32_t)__builtin_amdgcn_ds_bpermute(4 * (lane ^ 16), (int)x);
    return x | (uint32_t)__builtin_amdgcn_ds_bpermute(4 * (lane ^ 32), (int)x);
}

// A row's part of the sum over the wavefronts: how much each wavefront's counts, the highest maximum, the sum, and the groups of
// channels that are NaN.
template <int W>
struct Q4Meet {
    float f[W], m, l;
    uint32_t nan;
    template <class Rows>
    __device__ __forceinline__ Q4Meet(const Rows& rows, int row) : m(-INFINITY), l(0.f), nan(0)
    {
        Q4Row x[W];
#pragma unroll
        for (int w = 0; w < W; ++w) {
            x[w] = rows[w][row];
            m = fmaxf(m, x[w][0]);
            const float bits = x[w][2];                            // (of an element in place, the cast takes the first one's)
            nan |= __builtin_bit_cast(uint32_t, bits);
        }
        const float off = m == -INFINITY ? 0.f : m;
#pragma unroll
        for (int w = 0; w < W; ++w) {
            f[w] = __builtin_amdgcn_exp2f(x[w][0] - off);
            l += x[w][1] * f[w];
        }
    }
    __device__ __forceinline__ floatx4 spoil(floatx4 o, int group) const
    {
        return nan >> group & 1 ? (floatx4){NAN, NAN, NAN, NAN} : o;
    }
};

// How a launch is divided: a head's rows in blocks, its keys in parts of `per` or one more tiles (the first `rem`).
struct Q4Parts {
    int splits, blocks, per, rem;
};
// What the first loads need comes in the twelve words that the hardware puts into scalar registers before a kernel starts; the
// argument block, host memory, is 0.6 us away.
// rows: kv_len (below 2^24) << 8 | M; heads: nkv - 1 | rep - 1 << 8 | splits (up to 768) << 16; tiles: up to 2^19 | rem << 20 |
// whether `relation` is masks << 31
#define Q4_FIRST const char *k, const char *v, const half_t *q, const void *relation, uint32_t rows, uint32_t heads, uint32_t tiles, int per
__device__ __forceinline__ void q4_rows_and_heads(Q4Attn& a, uint32_t rows, uint32_t heads)
{
    a.M = rows & 255;
    a.kv_len = rows >> 8;
    a.nkv = (heads & 255) + 1;
    a.rep = (heads >> 8 & 255) + 1;
    a.nh = a.nkv * a.rep;
    a.inv_rep = q4_inverse(a.rep);
}
__device__ __forceinline__ void q4_first(Q4Attn& a, Q4Parts& parts, Q4_FIRST)
{
    q4_rows_and_heads(a, rows, heads);
    a.k = k;
    a.v = v;
    a.q = q;
    a.tiles = tiles & 0xfffff;
    a.mask = tiles >> 31 ? (const uint64_t*)relation : nullptr;
    a.parent = tiles >> 31 ? nullptr : (const int32_t*)relation;
    parts.splits = heads >> 16;
    parts.per = per;
    parts.rem = tiles >> 20 & 1023;
}
static uint32_t q4_rows_word(const Q4Attn& a) { return (uint32_t)a.kv_len << 8 | a.M; }
static uint32_t q4_heads_word(const Q4Attn& a, const Q4Parts& c) { return (a.nkv - 1) | (a.rep - 1) << 8 | (uint32_t)c.splits << 16; }
static uint32_t q4_tiles_word(const Q4Attn& a, const Q4Parts& c) { return a.tiles | c.rem << 20 | (a.mask ? 1u << 31 : 0u); }
static const void* q4_relation(const Q4Attn& a) { return a.mask ? (const void*)a.mask : a.parent; }

struct Q4Item {
    int head, block, split, R, total, t0, t1;
    __device__ __forceinline__ Q4Item(const Q4Attn& a, const Q4Parts& c, int head, int block, int split)
        : head(head), block(block), split(split), R(a.M * a.rep), total(a.kv_len + a.M), t0(split * c.per + min(split, c.rem)),
          t1(t0 + c.per + (split < c.rem ? 1 : 0))
    {
    }
    __device__ __forceinline__ int unit(const Q4Parts& c) const { return (head * c.blocks + block) * c.splits + split; }
};

// the node of a row
__device__ __forceinline__ int q4_node(const Q4Attn& a, int row) { return q4_over(row, a.inv_rep); }

// operand s of a row; zeros where there is no row
template <int D>
__device__ __forceinline__ half8 q4_query(const Q4Attn& a, const Q4Item& it, int row, int g, int s)
{
    const int node = q4_node(a, row);
    const uint32_t at = (node * a.nh + it.head * a.rep + row - node * a.rep) * D + g * (D / 4);     // (below 2^22)
    half8 q = {0, 0, 0, 0, 0, 0, 0, 0};
    if (row < it.R) q = *(const half8*)(a.q + at + 8 * s);
    return a.scale < 0.f ? -q : q;
}

// the four channels of tile ct of a row, the sums divided by l; a row that sees no key gives zeros
template <int D>
__device__ __forceinline__ void q4_out(const Q4Attn& a, int head, int row, int ct, int g, floatx4 o, float l)
{
    const int node = q4_node(a, row);
    const bool none = a.kv_len == 0 && a.mask && !q4_sees(a.mask, node, a.M);
    const float r = 1.f / l;
    half4 y;
#pragma unroll
    for (int e = 0; e < 4; ++e) y[e] = none ? (half_t)0.f : (half_t)(o[e] * r);
    *(half4*)(a.out + (uint32_t)((node * a.nh + head * a.rep + row - node * a.rep) * D + ct * 16 + 4 * g)) = y;
}

// ---- up to 16 rows -----------------------------------------------------------------------
// Bound: the bytes (1 row of 32 heads, on 8 key heads, over 65537 keys 20.5 us with the rows in the 256 MB cache, 23.0 from HBM,
// 3.6 TB/s of a copy's 4.75, the second launch among them); over few keys the way from queries and masks to the states' meeting
// (6 us).
constexpr int kQ4KeyWaves = 4;

// a tile of 32 keys, as a wavefront has it on its way
template <int D>
struct Q4Tile {
    Q4RawK<D> k[2];
    word4 v[D / 64];
    half8 lo, s;                       // of the lane's 8 keys and group col % (D / 32): the four (two) lanes side by side have all
    __device__ __forceinline__ void load_k(const Q4Head& keys, uint32_t at, int col, int g)
    {
#pragma unroll
        for (int h = 0; h < 2; ++h) k[h].load(keys, at, h, col, g);
    }
    __device__ __forceinline__ void load_v(const Q4Head& values, uint32_t at, int col, int g)
    {
#pragma unroll
        for (int i = 0; i < D / 64; ++i) v[i] = values.get4(at + i * 1024, (g * 16 + col) * 16u);
        const uint32_t m = col % (D / 32) * 128u + g * 16u;
        lo = __builtin_bit_cast(half8, values.get4(at + q4_codes_bytes(D), m));
        s = __builtin_bit_cast(half8, values.get4(at + q4_codes_bytes(D) + 64, m));
    }
};

// x of the lane that has group i, among the lanes side by side that have all
template <int D, int I>
__device__ __forceinline__ half8 q4_of_group(half8 x)
{
    constexpr int kCtrl = D == 128 ? I * 0x55 : I ? 0xF5 : 0xA0;
    word4 w = __builtin_bit_cast(word4, x);
#pragma unroll
    for (int e = 0; e < 4; ++e) w[e] = (uint32_t)__builtin_amdgcn_mov_dpp((int)w[e], kCtrl, 0xf, 0xf, true);
    return __builtin_bit_cast(half8, w);
}

// Products of 32 keys with RT tiles of rows, whose operands are in registers (q) or in LDS (at q_lds, as the MFMA takes them), and
// the codes of tile `next` requested in their place.  One piece of code for all tiles: what a launch runs once costs as much to
// fetch as to run.
template <int D, int RT, class Query>
__device__ __forceinline__ void q4_tile(const Q4Attn& a, const Q4Item& it, const Q4Bits& bits, Q4State<D> (&st)[RT], const Query& query,
                                        Q4Tile<D>& t, float c, int tile, int row0, int lane, const uint64_t* s_mask, const Q4Head& keys,
                                        const Q4Head& values, uint32_t next, uint32_t& nan)
{
    constexpr int KS = D / 32;
    const int col = lane & 15, g = lane >> 4;
    floatx4 s[RT][2];
#pragma unroll
    for (int r = 0; r < RT; ++r) s[r][0] = s[r][1] = (floatx4){0.f, 0.f, 0.f, 0.f};
#pragma unroll
    for (int k = 0; k < KS; ++k) {
        half8 x[RT];
#pragma unroll
        for (int r = 0; r < RT; ++r) x[r] = query(r, k);
#pragma unroll
        for (int h = 0; h < 2; ++h) {
            const half8 y = t.k[h].operand(bits, k);
#pragma unroll
            for (int r = 0; r < RT; ++r) s[r][h] = __builtin_amdgcn_mfma_f32_16x16x32_f16(y, x[r], s[r][h], 0, 0, 0);
        }
    }
    pin_order();
    t.load_k(keys, next, col, g);
    pin_order();
    auto sees = [&](int lane, int r) {
        const int row = row0 + r * 16 + (lane & 15);
        return seen_keys((const uint32_t*)(s_mask + 2 * (row < it.R ? q4_node(a, row) : 0)), tile * kQ4Tile + 8 * (lane >> 4), a.kv_len,
                         it.total);
    };
    uint32_t bad = 0;
    if ((tile + 1) * kQ4Tile > a.kv_len) {                         // into the drafted rows
        const int here = q4_lane();
#pragma unroll
        for (int r = 0; r < RT; ++r) {
            const uint32_t see = sees(here, r);
#pragma unroll
            for (int e = 0; e < 8; ++e)
                if (!(see >> e & 1)) s[r][e >> 2][e & 3] = -INFINITY;
        }
        bad = q4_clean(t.lo, t.s, tile * kQ4Tile + 8 * (here >> 4), it.total);
    }
    half8 p[RT];
    float top[RT];
    bool more = false;
#pragma unroll
    for (int r = 0; r < RT; ++r) {
        top[r] = st[r].highest(s[r], c);
        more = more || top[r] > st[r].m + 8.f;
    }
    if (__ballot(more))
#pragma unroll
        for (int r = 0; r < RT; ++r) st[r].raise(top[r]);
#pragma unroll
    for (int r = 0; r < RT; ++r) p[r] = st[r].powers(s[r], c);
    auto group = [&](auto I) {
        constexpr int i = decltype(I)::value;
        Q4Pairs m;
        m.set(q4_of_group<D, i>(t.lo), q4_of_group<D, i>(t.s));
#pragma unroll
        for (int e = 0; e < 2; ++e) {
            const int ct = 2 * i + e;
            const half8 y = q4_values(bits, t.v[ct / 4][ct % 4], m.lo, m.s);
#pragma unroll
            for (int r = 0; r < RT; ++r) st[r].o[ct] = __builtin_amdgcn_mfma_f32_16x16x32_f16(y, p[r], st[r].o[ct], 0, 0, 0);
        }
    };
    group(std::integral_constant<int, 0>());
    group(std::integral_constant<int, 1>());
    if constexpr (D == 128) {
        group(std::integral_constant<int, 2>());
        group(std::integral_constant<int, 3>());
    }
    pin_order();
    t.load_v(values, next, col, g);
    pin_order();
    if (__builtin_expect(__ballot(bad != 0) != 0, 0)) {
        const int here = q4_lane();
#pragma unroll 1
        for (int r = 0; r < RT; ++r) {
            const uint32_t see = sees(here, r);
#pragma unroll 1
            for (int i = 0; i < KS; ++i)                           // (the lane that has group i of the same keys)
                if (see & (uint32_t)__builtin_amdgcn_ds_bpermute(4 * ((here & ~(KS - 1)) + i), (int)bad)) nan |= 1u << (r * KS + i);
        }
    }
}

template <int D>
__global__ __launch_bounds__(kQ4KeyWaves * 64, 3) void k_q4_attention_keys(Q4_FIRST, Q4Attn a, Q4Parts parts)
{
    q4_first(a, parts, k, v, q, relation, rows, heads, tiles, per);
    constexpr int CT = D / 16;
    __shared__ uint64_t s_mask[2 * GHD_MAX_M];
    __shared__ floatx4 s_o[kQ4KeyWaves][CT][64];
    __shared__ Q4Row s_ml[kQ4KeyWaves][16];
    const int lane = threadIdx.x & 63, wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
    const Q4Item it(a, parts, blockIdx.y, 0, blockIdx.x);
    const int t0 = it.t0, t1 = it.t1;
    const bool reaches = t1 * kQ4Tile > a.kv_len;                  // into the drafted rows
    const Q4Masks masks(a, reaches, wave, lane);
    const Q4Head keys(a.k, it.head, a.tiles, D), values(a.v, it.head, a.tiles, D);
    auto at = [&](int tile) { return (uint32_t)min(tile, t1 - 1) * q4_tile_bytes(D); };
    Q4Tile<D> tile[2];
#pragma unroll
    for (int i = 0; i < 2; ++i) {
        tile[i].load_k(keys, at(t0 + wave + i * kQ4KeyWaves), lane & 15, lane >> 4);
        tile[i].load_v(values, at(t0 + wave + i * kQ4KeyWaves), lane & 15, lane >> 4);
    }
    half8 x[D / 32];
#pragma unroll
    for (int s = 0; s < D / 32; ++s) x[s] = q4_query<D>(a, it, lane & 15, lane >> 4, s);
    masks.store(a, wave, lane, s_mask);
    if (reaches) __syncthreads();
    const Q4Bits bits;
    const float c = q4_power(a.scale);
    Q4State<D> st[1];
    uint32_t nan = 0;                  // a bit for every group of channels of a row: it has seen one there
    int t = t0 + wave;
    // (two tiles in turn: a copy of the one on its way would have to wait for it)
    auto query = [&](int, int k) { return x[k]; };
    for (; t < t1; t += 2 * kQ4KeyWaves) {
        q4_tile<D, 1>(a, it, bits, st, query, tile[0], c, t, 0, lane, s_mask, keys, values, at(t + 2 * kQ4KeyWaves), nan);
        if (t + kQ4KeyWaves >= t1) break;
        q4_tile<D, 1>(a, it, bits, st, query, tile[1], c, t + kQ4KeyWaves, 0, lane, s_mask, keys, values, at(t + 3 * kQ4KeyWaves), nan);
    }
    // the wavefronts' states meet in LDS; each finishes its share of the channel tiles
    const int here = q4_lane(), col = here & 15, g = here >> 4;
    nan = or_over_groups(nan);
    if (g == 0) s_ml[wave][col] = q4_row(st[0].m, st[0].l[0], nan, 0);
#pragma unroll
    for (int ct = 0; ct < CT; ++ct) s_o[wave][ct][here] = st[0].o[ct];
    __syncthreads();
    const Q4Meet<kQ4KeyWaves> all(s_ml, col);
    if (parts.splits > 1 && wave == 0 && g == 0) ((floatx2*)a.ml_part)[(size_t)it.unit(parts) * 16 + col] = (floatx2){all.m, all.l};
#pragma unroll
    for (int j = 0; j < CT / kQ4KeyWaves; ++j) {
        const int ct = wave * (CT / kQ4KeyWaves) + j;
        floatx4 o = {0.f, 0.f, 0.f, 0.f};
#pragma unroll
        for (int w = 0; w < kQ4KeyWaves; ++w) o += s_o[w][ct][here] * all.f[w];
        o = all.spoil(o, ct / 2);
        if (parts.splits > 1) ((floatx4*)a.o_part)[((size_t)it.unit(parts) * CT + ct) * 64 + here] = o;
        else if (col < it.R) q4_out<D>(a, it.head, col, ct, g, o, all.l);
    }
}

// ---- more rows ---------------------------------------------------------------------------
// Blocks of RT tiles of 16 rows, queries as operands in LDS.
// Bound, over many keys, by the issue of vector instructions: 32 keys by four tiles of rows take 2640 cycles of a wavefront when two
// share a SIMD, of them 240 instructions for the conversion and 62 for the softmax of each tile (exponentials, at a quarter of
// the rate, are half of those) at 4 cycles, and 68 products, which keep the issue for 10 cycles each (measured: 17 cycles for
// a product alone, 32 for 8 packed instructions, 42 for both).  128 rows of 40 heads over 8320 keys: 41 us, 0.53 PFLOP/s.
// Over few keys by what comes one after another, in cycles of 64 rows of 32 heads: 5000 until queries are there, 1600 for the
// ancestors' masks meanwhile, 3500 for the first keys (whose instructions are fetched, too), 4700 until the states have met.
// Four wavefronts a workgroup and two of those on a compute unit: 64 rows of 32 heads over 2112 keys 19.6 us instead of 15.2.
// Queries in registers: 32 rows over 224 keys 9.9 instead of 8.6 us (all wavefronts read all of them).
constexpr int kQ4RowWaves = 8;

template <int D, int RT>
__global__ __launch_bounds__(kQ4RowWaves * 64, 2) void k_q4_attention_rows(Q4_FIRST, Q4Attn a, Q4Parts parts)
{
    q4_first(a, parts, k, v, q, relation, rows, heads, tiles, per);
    constexpr int CT = D / 16, KS = D / 32, W = kQ4RowWaves, kFrags = RT * CT, kRound = kFrags < 16 ? kFrags : 16;
    __shared__ uint64_t s_mask[2 * GHD_MAX_M];
    __shared__ Q4Row s_ml[W][RT * 16];
    extern __shared__ __attribute__((aligned(16))) char lds[];
    const int lane = threadIdx.x & 63, wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
    // 8 xcds by blocks, by parts in eights: the blocks of a part of a head's keys share an L2
    const int item = blockIdx.y * 8 + (blockIdx.x & 7);
    if (item >= a.nkv * parts.splits) return;
    const int head = __builtin_amdgcn_readfirstlane(q4_over(item, q4_inverse(parts.splits)));
    const Q4Item it(a, parts, head, blockIdx.x >> 3, item - head * parts.splits);
    const int t0 = it.t0, t1 = it.t1;
    const Q4Masks masks(a, t1 * kQ4Tile > a.kv_len, wave, lane);
    const Q4Head keys(a.k, it.head, a.tiles, D), values(a.v, it.head, a.tiles, D);
    auto tile_at = [&](int tile) { return (uint32_t)min(tile, t1 - 1) * q4_tile_bytes(D); };
    Q4Tile<D> tile;
    tile.load_k(keys, tile_at(t0 + wave), lane & 15, lane >> 4);
    tile.load_v(values, tile_at(t0 + wave), lane & 15, lane >> 4);
    const int row0 = it.block * RT * 16;
    constexpr int kMine = (RT * KS + W - 1) / W;                   // operands of q that a wavefront brings
    half8 x[kMine];
#pragma unroll
    for (int f = 0; f < kMine; ++f) {
        const int frag = min(f * W + wave, RT * KS - 1);
        x[f] = q4_query<D>(a, it, row0 + frag / KS * 16 + (lane & 15), lane >> 4, frag % KS);
    }
    masks.store(a, wave, lane, s_mask);
#pragma unroll
    for (int f = 0; f < kMine; ++f)
        if (f * W + wave < RT * KS) *(half8*)(lds + (f * W + wave) * 1024 + lane * 16) = x[f];
    __syncthreads();
    const Q4Bits bits;
    const float c = q4_power(a.scale);
    Q4State<D> st[RT];
    uint32_t nan = 0;                  // a bit for every group of channels of a row of each tile: it has seen one there
    auto query = [&](int r, int k) { return *(const half8*)(lds + (r * KS + k) * 1024 + lane * 16); };
    for (int t = t0 + wave; t < t1; t += W)
        q4_tile<D, RT>(a, it, bits, st, query, tile, c, t, row0, lane, s_mask, keys, values, tile_at(t + W), nan);
    // The wavefronts' states meet in LDS, as many fragments at a time as fit, each added up by one wavefront.
    const int at = q4_lane(), col = at & 15, g = at >> 4;
    nan = or_over_groups(nan);
    if (g == 0)
#pragma unroll
        for (int r = 0; r < RT; ++r) s_ml[wave][r * 16 + col] = q4_row(st[r].m, st[r].l[0], nan, r * KS);
    const size_t unit = (size_t)it.unit(parts) * RT;
    floatx4* part = (floatx4*)lds + at;                            // [wave][fragment][64]
#pragma unroll
    for (int f0 = 0; f0 < kFrags; f0 += kRound) {
        __syncthreads();
#pragma unroll
        for (int f = f0; f < std::min(f0 + kRound, kFrags); ++f) part[(wave * kRound + f - f0) * 64] = st[f / CT].o[f % CT];
        __syncthreads();
#pragma unroll 2
        for (int e = wave; e < kRound && f0 + e < kFrags; e += W) {
            const int f = f0 + e, r = f / CT, ct = f % CT, row = row0 + r * 16 + col;
            const Q4Meet<W> all(s_ml, r * 16 + col);
            floatx4 o = {0.f, 0.f, 0.f, 0.f};
#pragma unroll
            for (int w = 0; w < W; ++w) o += part[(w * kRound + e) * 64] * all.f[w];
            o = all.spoil(o, ct / 2);
            if (parts.splits > 1) {
                ((floatx4*)a.o_part)[((unit + r) * CT + ct) * 64 + at] = o;
                if (ct == 0 && g == 0) ((floatx2*)a.ml_part)[(unit + r) * 16 + col] = (floatx2){all.m, all.l};
            } else if (row < it.R) {
                q4_out<D>(a, it.head, row, ct, g, o, all.l);
            }
        }
    }
}

// ---- parts of a head's keys to its rows ----------------------------------------------------
// Four wavefronts take the parts of one fragment - 16 channels by 16 rows - in turn, eight requests at a time.
template <int D>
__global__ __launch_bounds__(256) void k_q4_join(const float* o_part, const float* ml_part, half_t* out, uint32_t rows, uint32_t heads,
                                                 int row_tiles, int blocks, Q4Attn a)
{
    q4_rows_and_heads(a, rows, heads);
    a.out = out;
    constexpr int CT = D / 16, kAt = 8;
    __shared__ floatx4 s_o[4][64];
    __shared__ floatx2 s_ml[4][16];
    const int lane = threadIdx.x & 63, wave = threadIdx.x >> 6, col = lane & 15, g = lane >> 4;
    const int ct = blockIdx.x, rt = blockIdx.y, hb = blockIdx.z, splits = heads >> 16;
    const int head = q4_over(hb, q4_inverse(blocks)), block = hb - head * blocks, row = (block * row_tiles + rt) * 16 + col;
    if ((block * row_tiles + rt) * 16 >= a.M * a.rep) return;
    float m = -INFINITY, l = 0.f;
    floatx4 o = {0.f, 0.f, 0.f, 0.f};
    for (int p0 = wave; p0 < splits; p0 += 4 * kAt) {
        floatx2 ml[kAt];
        floatx4 v[kAt];
        float top = m;
#pragma unroll
        for (int j = 0; j < kAt; ++j) {
            const size_t unit = ((size_t)hb * splits + min(p0 + 4 * j, splits - 1)) * row_tiles + rt;
            ml[j] = ((const floatx2*)ml_part)[unit * 16 + col];
            v[j] = ((const floatx4*)o_part)[(unit * CT + ct) * 64 + lane];
        }
#pragma unroll
        for (int j = 0; j < kAt; ++j)
            if (p0 + 4 * j < splits) top = fmaxf(top, ml[j][0]);
        const float off = top == -INFINITY ? 0.f : top, r = __builtin_amdgcn_exp2f(m - off);
        l *= r;
        o *= r;
#pragma unroll
        for (int j = 0; j < kAt; ++j)
            if (p0 + 4 * j < splits) {
                const float f = __builtin_amdgcn_exp2f(ml[j][0] - off);
                l += ml[j][1] * f;
                o += v[j] * f;
            }
        m = top;
    }
    s_o[wave][lane] = o;
    if (g == 0) s_ml[wave][col] = (floatx2){m, l};
    __syncthreads();
    if (wave != 0 || row >= a.M * a.rep) return;
    float top = -INFINITY;
#pragma unroll
    for (int w = 0; w < 4; ++w) top = fmaxf(top, s_ml[w][col][0]);
    const float off = top == -INFINITY ? 0.f : top;
    l = 0.f;
    o = (floatx4){0.f, 0.f, 0.f, 0.f};
#pragma unroll
    for (int w = 0; w < 4; ++w) {
        const float f = __builtin_amdgcn_exp2f(s_ml[w][col][0] - off);
        l += s_ml[w][col][1] * f;
        o += s_o[w][lane] * f;
    }
    q4_out<D>(a, head, row, ct, g, o, l);
}

// ---- how a call is divided -----------------------------------------------------------------
struct Q4AttnCut {
    int rows, blocks, splits;    // tiles of 16 rows in a block, blocks, parts of the keys
};

// Up to 16 rows parts cost a launch that joins them (3 us): none where a workgroup is through sooner than that (8 tokens of 8 heads
// over 308 keys: 1 part 7.4 us a call, 2 9.4), else as many as make 256 workgroups, one a compute unit, and three times as many
// where each then has long to go (1 token of 40 heads over 32000: 6 parts 48.9, 12 44.7, 19 43.7).
static int q4_key_splits(int ntiles, int nkv)
{
    const int turns = ceil_div(ntiles, kQ4KeyWaves), splits = ntiles / (256 / nkv) > 64 ? 768 / nkv : 256 / nkv;
    return turns <= 6 ? 1 : std::max(1, std::min(splits, turns));
}

// Above, what is estimated to be fastest of blocks of 2, 3 and 4 tiles of rows and of parts that fill the compute units once: a turn
// of the wavefronts takes 2.0, 2.4 or 2.8 us, so the larger a block the better where keys are many, and getting to the first and
// from the last 7, 9 or 10.4 (with 64 channels .6 of the one, 5.5, 6.5 and 7.2 of the other), so the smaller the better where
// they are few.  64 rows of 32 heads, the kernel alone: over 512 keys blocks of 2 9.8, of 4 12.8; over 8256 22.0 and 22.2; 128
// rows of 40 heads over 8320 64 and 41.
static Q4AttnCut q4_attn_cut(int M, int kv_len, int nh, int nkv, int d)
{
    const int rt = ceil_div(M * (nh / nkv), 16), ntiles = ceil_div(kv_len + M, kQ4Tile);
    if (rt == 1) return {1, 1, q4_key_splits(ntiles, nkv)};
    Q4AttnCut best = {};
    float least = 0.f;
    for (int most = 2; most <= 4; ++most) {
        const int blocks = ceil_div(rt, most), rows = ceil_div(rt, blocks), items = nkv * blocks;
        if (rows != most) continue;
        const float turn = d == 128 ? 1.2f + 0.4f * rows : 0.72f + 0.24f * rows, rest = d == 128 ? 3.6f + 1.7f * rows : 3.8f + 0.85f * rows;
        for (int splits = 1; splits == 1 || (splits * items <= 256 && splits <= ntiles); splits += 1 + splits / 8) {
            const int turns = ceil_div(ceil_div(ntiles, splits), kQ4RowWaves), rounds = ceil_div(items * splits, 256);
            float us = rounds * (rest + turns * turn);
            if (splits > 1) us += 3.5f + 0.35e-6f * 64.f * d * splits * items * rows;
            if (least == 0.f || us < least) {
                least = us;
                best = {rows, blocks, splits};
            }
        }
    }
    return best;
}

static size_t q4_attn_units(const Q4AttnCut& c, int nkv) { return (size_t)nkv * c.blocks * c.splits * c.rows; }

static size_t q4_units_bytes(size_t units, int d) { return align_up(units * 16 * d * 4, 256) + align_up(units * 128, 256); }

static size_t q4_attn_bytes(const Q4AttnCut& c, int nkv, int d) { return c.splits == 1 ? 256 : q4_units_bytes(q4_attn_units(c, nkv), d); }

// The most that a call of up to M tokens over up to kv_len rows takes, whatever its cut: what a caller makes once for its widest tree
// and longest context does for every step on the way there.
size_t q4_attention_bytes(int M, int kv_len, int nh, int nkv, int d)
{
    const int rep = nh / nkv, ntiles = ceil_div(kv_len + M, kQ4Tile), rt = ceil_div(M * rep, 16);
    size_t units = 0;
    if (rep <= 16 && q4_key_splits(ntiles, nkv) > 1) units = (size_t)nkv * q4_key_splits(ntiles, nkv);
    // blocks of 2 to 4 tiles: at most 256 workgroups where there are parts, a part has a tile, and blocks end up to a tile behind the rows
    if (rt > 1 && ntiles > 1 && nkv <= 128)
        units = std::max(units, (size_t)std::min<int64_t>(256 * 4, (int64_t)nkv * (rt + (rt + 1) / 2 - 1) * ntiles));
    return units ? q4_units_bytes(units, d) : 256;
}

void q4_attention_on_host(int M, int kv_len, int nh, int nkv, int d, int64_t* out4)
{
    const Q4AttnCut c = q4_attn_cut(M, kv_len, nh, nkv, d);
    out4[0] = c.rows;
    out4[1] = c.blocks;
    out4[2] = c.splits;
    out4[3] = q4_attn_bytes(c, nkv, d);
}

template <int D, int RT>
static ghd_status q4_rows_of(const Q4Attn& a, const Q4Parts& c, hipStream_t st)
{
    const size_t lds = (size_t)kQ4RowWaves * std::min(RT * (D / 16), 16) * 1024;
    const ghd_status s = launch_resident_checked((const void*)k_q4_attention_rows<D, RT>, kQ4RowWaves * 64, lds, nullptr);
    if (s) return s;
    hipLaunchKernelGGL((k_q4_attention_rows<D, RT>), dim3(8 * c.blocks, ceil_div(a.nkv * c.splits, 8)), dim3(kQ4RowWaves * 64), lds, st, a.k,
                       a.v, a.q, q4_relation(a), q4_rows_word(a), q4_heads_word(a, c), q4_tiles_word(a, c), c.per, a, c);
    return check_launch();
}

template <int D>
static ghd_status q4_attention_of(const Q4Attn& a, const Q4AttnCut& c, hipStream_t st)
{
    const int ntiles = ceil_div(a.kv_len + a.M, kQ4Tile);
    const Q4Parts p = {c.splits, c.blocks, ntiles / c.splits, ntiles % c.splits};
    ghd_status s;
    if (c.rows == 1) {
        hipLaunchKernelGGL(k_q4_attention_keys<D>, dim3(c.splits, a.nkv), dim3(kQ4KeyWaves * 64), 0, st, a.k, a.v, a.q, q4_relation(a),
                           q4_rows_word(a), q4_heads_word(a, p), q4_tiles_word(a, p), p.per, a, p);
        s = check_launch();
    } else {
        s = c.rows == 2 ? q4_rows_of<D, 2>(a, p, st) : c.rows == 3 ? q4_rows_of<D, 3>(a, p, st) : q4_rows_of<D, 4>(a, p, st);
    }
    if (s || c.splits == 1) return s;
    hipLaunchKernelGGL(k_q4_join<D>, dim3(D / 16, c.rows, a.nkv * c.blocks), dim3(256), 0, st, a.o_part, a.ml_part, a.out,
                       q4_rows_word(a), q4_heads_word(a, p), c.rows, c.blocks, a);
    return check_launch();
}

ghd_status launch_q4_attention(Q4Attn a, int d, void* ws, size_t ws_bytes, hipStream_t st)
{
    const Q4AttnCut c = q4_attn_cut(a.M, a.kv_len, a.nh, a.nkv, d);
    if (ws_bytes < q4_attn_bytes(c, a.nkv, d)) return GHD_ERR_WORKSPACE;
    a.rep = a.nh / a.nkv;
    a.inv_rep = 1.f / (float)a.rep;
    a.o_part = (float*)ws;
    a.ml_part = (float*)((char*)ws + align_up(q4_attn_units(c, a.nkv) * 16 * d * 4, 256));
    return d == 128 ? q4_attention_of<128>(a, c, st) : q4_attention_of<64>(a, c, st);
}

}  // namespace ghd
