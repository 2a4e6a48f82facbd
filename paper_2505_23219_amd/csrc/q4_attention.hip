// Attention of the drafted tokens over a 4-bit cache.
//
// out[i, h] = softmax over the keys that node i sees of (scale q . K^) applied to V^, where K^ and V^ are the fp16
// numbers that the codes stand for (q4.h).  A key head's query rows - M nodes by nh / nkv heads - are the columns of
// S^T = K^ q^T and O^T = V^T P^T, so softmax statistics are a lane's own and the probabilities come out as the operand of
// the second product.  Running maximum and sum are kept in 32 bits; probabilities are rounded to fp16, relative to a maximum
// that lags by up to 2^8 (fp16 holds that as exactly, and sums are rescaled seldom).
//
// Up to 16 query rows a wavefront takes 32 keys at a time by itself, codes straight into operand registers: what counts is
// that the cache streams.  Above, the wavefronts of a workgroup have 16 rows each and share the conversion of the codes, which
// takes longer than the products of 16 rows: each converts a piece of the keys to come into LDS, as operands.
#include "q4.h"
#include "attention_impl.h"

namespace ghd {

typedef uint32_t word2 __attribute__((ext_vector_type(2)));
typedef uint32_t word4 __attribute__((ext_vector_type(4)));

// the bits of a node's mask for the 32 keys from `base` on, counted from the first drafted row; keys
// before that are committed, and seen
__device__ __forceinline__ uint32_t q4_mask32(uint64_t lo, uint64_t hi, int base)
{
    if (base <= -32) return ~0u;
    if (base < 0) return (uint32_t)(lo << -base) | ((1u << -base) - 1u);
    if (base >= 128) return 0;
    if (base >= 64) return (uint32_t)(hi >> (base - 64));
    return (uint32_t)(base ? lo >> base | hi << (64 - base) : lo);
}

// does a node see any drafted key? (bits from M on say nothing)
__device__ __forceinline__ bool q4_sees(const uint64_t* mask, int node, int M)
{
    const uint64_t lo = M >= 64 ? ~0ull : (1ull << M) - 1, hi = M >= 128 ? ~0ull : M > 64 ? (1ull << (M - 64)) - 1 : 0;
    return (mask[2 * node] & lo) | (mask[2 * node + 1] & hi);
}

// The masks of all nodes to LDS; the workgroup's barrier is the caller's.
__device__ __forceinline__ void q4_masks(const Q4Attn& a, uint64_t* s_mask)
{
    const int tid = threadIdx.x, lane = tid & 63;
    if (a.mask) {
        for (int e = tid; e < 2 * a.M; e += blockDim.x) {
            const int left = a.M - 64 * (e & 1);                   // bits of this word that mean something
            s_mask[e] = left >= 64 ? a.mask[e] : left <= 0 ? 0 : a.mask[e] & ((1ull << left) - 1);
        }
    } else if (tid < 64) {
        store_masks(tree_nodes<2, true>(a.parent[min(lane, a.M - 1)], a.parent[min(lane + 64, a.M - 1)], a.M, lane), a.M, lane, s_mask);
    }
}

// 16 keys of a tile (half h), as a lane (g, col) has them: operand row r is key 8 (r / 4) + 4 h + r % 4, so that a lane's 8
// scores of a column are those of keys 8 g .. 8 g + 7, the probabilities it holds in the second product.  Its channels, D / 4
// from g D / 4 on, are the k-steps' in turn.
template <int D>
struct Q4RawK {
    uint32_t w[D / 32];
    half2_ m;
    __device__ __forceinline__ void load(const char* tile, int h, int col, int g)
    {
        const int key = 8 * (col >> 2) + 4 * h + (col & 3);
        if constexpr (D == 128) {
            const word4 v = *(const word4*)(tile + key * 64 + g * 16);
#pragma unroll
            for (int s = 0; s < 4; ++s) w[s] = v[s];
            m = *(const half2_*)(tile + q4_codes_bytes(D) + (key * 4 + g) * 4);
        } else {
            const word2 v = *(const word2*)(tile + key * 32 + g * 8);
            w[0] = v[0];
            w[1] = v[1];
            m = *(const half2_*)(tile + q4_codes_bytes(D) + (key * 2 + (g >> 1)) * 4);
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
// (a NaN was appended), which only reaches the rows that see it (q4_poison); returned: which of the 8 keys those are.
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
    // scores (of this lane's 8 keys) to probabilities; c, what makes powers of two of them, is not negative
    template <bool MASKED>
    __device__ __forceinline__ half8 probabilities(const floatx4 (&s)[2], float c, uint32_t see)
    {
        float top = -INFINITY;
#pragma unroll
        for (int e = 0; e < 8; ++e) {
            const float v = s[e >> 2][e & 3];
            top = fmaxf(top, MASKED && !(see >> e & 1) ? -INFINITY : v);
        }
        top = max_over_groups(top);
        top = top == -INFINITY ? top : top * c;
        if (__ballot(top > m + 8.f)) {
            const float now = fmaxf(m, top), r = m == now ? 1.f : __builtin_amdgcn_exp2f(m - now);
            l *= r;
#pragma unroll
            for (int ct = 0; ct < D / 16; ++ct) o[ct] *= r;
            m = now;
        }
        const float off = m == -INFINITY ? 0.f : -m;
        half2_ p[4];
#pragma unroll
        for (int e = 0; e < 4; ++e) {
            floatx2 x;
#pragma unroll
            for (int u = 0; u < 2; ++u) {
                x[u] = __builtin_amdgcn_exp2f(fmaf(s[e >> 1][2 * (e & 1) + u], c, off));
                if (MASKED && !(see >> (2 * e + u) & 1)) x[u] = 0.f;
            }
            p[e] = __builtin_convertvector(x, half2_);
        }
        const half8 all = join(p[0], p[1], p[2], p[3]);
        const half_t one = (half_t)1.f;
        l = __builtin_amdgcn_mfma_f32_16x16x32_f16((half8){one, one, one, one, one, one, one, one}, all, l, 0, 0, 0);
        return all;
    }
    // NaN in the channels of group i for rows that see one of the keys with a NaN there: how many they see is a product of ones
    __device__ __forceinline__ void poison(int i, uint32_t bad, uint32_t see)
    {
        half8 b, v;
#pragma unroll
        for (int e = 0; e < 8; ++e) {
            b[e] = bad >> e & 1 ? (half_t)1.f : (half_t)0.f;
            v[e] = see >> e & 1 ? (half_t)1.f : (half_t)0.f;
        }
        const floatx4 n = __builtin_amdgcn_mfma_f32_16x16x32_f16(b, v, (floatx4){0.f, 0.f, 0.f, 0.f}, 0, 0, 0);
#pragma unroll
        for (int e = 0; e < 4; ++e)
            if (n[e] > 0.f) o[2 * i][e] = o[2 * i + 1][e] = NAN;
    }
};

// What a launch works on: a head's rows in blocks, its keys in parts.
struct Q4Item {
    int head, block, split, rep, R, total;
    __device__ __forceinline__ Q4Item(const Q4Attn& a, int splits, int blocks)
    {
        split = blockIdx.x % splits;
        block = blockIdx.x / splits % blocks;
        head = blockIdx.x / splits / blocks;
        rep = a.nh / a.nkv;
        R = a.M * rep;
        total = a.kv_len + a.M;
    }
};

template <int D>
__device__ __forceinline__ void q4_queries(const Q4Attn& a, const Q4Item& it, int row, int g, half8 (&q)[D / 32])
{
    const int node = row / it.rep;
    const half_t* p = a.q + ((size_t)node * a.nh + it.head * it.rep + row - node * it.rep) * D + g * (D / 4);
#pragma unroll
    for (int s = 0; s < D / 32; ++s) {
        q[s] = (half8){0, 0, 0, 0, 0, 0, 0, 0};
        if (row < it.R) q[s] = *(const half8*)(p + 8 * s);
        if (a.scale < 0.f) q[s] = -q[s];
    }
}

// the four channels of tile ct of a row, the sums divided by l; a row that sees no key gives zeros
template <int D>
__device__ __forceinline__ void q4_out(const Q4Attn& a, int head, int rep, int row, int ct, int g, floatx4 o, float l)
{
    const int node = row / rep;
    const bool none = a.kv_len == 0 && a.mask && !q4_sees(a.mask, node, a.M);
    const float r = 1.f / l;
    half4 y;
#pragma unroll
    for (int e = 0; e < 4; ++e) y[e] = none ? (half_t)0.f : (half_t)(o[e] * r);
    *(half4*)(a.out + ((size_t)node * a.nh + head * rep + row - node * rep) * D + ct * 16 + 4 * g) = y;
}

// ---- up to 16 rows -----------------------------------------------------------------------
constexpr int kQ4KeyWaves = 4;

// a tile of 32 keys, as a wavefront has it on its way
template <int D>
struct Q4Tile {
    Q4RawK<D> k[2];
    word4 v[D / 64];
    half8 lo, s;                       // of the lane's 8 keys and group col % (D / 32): the four (two) lanes side by side have all
    __device__ __forceinline__ void load(const char* kt, const char* vt, int col, int g)
    {
#pragma unroll
        for (int h = 0; h < 2; ++h) k[h].load(kt, h, col, g);
#pragma unroll
        for (int i = 0; i < D / 64; ++i) v[i] = *(const word4*)(vt + ((i * 4 + g) * 16 + col) * 16);
        const char* m = vt + q4_codes_bytes(D) + col % (D / 32) * 128 + g * 16;
        lo = *(const half8*)m;
        s = *(const half8*)(m + 64);
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

template <int D, bool MASKED>
__device__ __forceinline__ void q4_tile(const Q4Attn& a, const Q4Bits& bits, Q4State<D>& st, const half8 (&q)[D / 32], Q4Tile<D>& t,
                                        float c, int tile, int total, int g, const uint64_t* mask)
{
    floatx4 s[2];
#pragma unroll
    for (int h = 0; h < 2; ++h) {
        s[h] = (floatx4){0.f, 0.f, 0.f, 0.f};
#pragma unroll
        for (int k = 0; k < D / 32; ++k) s[h] = __builtin_amdgcn_mfma_f32_16x16x32_f16(t.k[h].operand(bits, k), q[k], s[h], 0, 0, 0);
    }
    uint32_t see = 0, bad = 0;
    if constexpr (MASKED) {
        see = q4_mask32(mask[0], mask[1], tile * kQ4Tile - a.kv_len) >> 8 * g & 255u;
        bad = q4_clean(t.lo, t.s, tile * kQ4Tile + 8 * g, total);
    }
    const half8 p = st.template probabilities<MASKED>(s, c, see);
    auto group = [&](auto I) {
        constexpr int i = decltype(I)::value;
        Q4Pairs m;
        m.set(q4_of_group<D, i>(t.lo), q4_of_group<D, i>(t.s));
#pragma unroll
        for (int e = 0; e < 2; ++e) {
            const int ct = 2 * i + e;
            st.o[ct] = __builtin_amdgcn_mfma_f32_16x16x32_f16(q4_values(bits, t.v[ct / 4][ct % 4], m.lo, m.s), p, st.o[ct], 0, 0, 0);
        }
        if constexpr (MASKED) {
            constexpr int kCtrl = D == 128 ? i * 0x55 : i ? 0xF5 : 0xA0;
            const uint32_t b = (uint32_t)__builtin_amdgcn_mov_dpp((int)bad, kCtrl, 0xf, 0xf, true);
            if (__ballot(b != 0)) st.poison(i, b, see);
        }
    };
    group(std::integral_constant<int, 0>());
    group(std::integral_constant<int, 1>());
    if constexpr (D == 128) {
        group(std::integral_constant<int, 2>());
        group(std::integral_constant<int, 3>());
    }
}

template <int D>
__global__ __launch_bounds__(kQ4KeyWaves * 64, 3) void k_q4_attention_keys(const Q4Attn a, int splits)
{
    constexpr int CT = D / 16;
    __shared__ uint64_t s_mask[2 * GHD_MAX_M];
    __shared__ floatx4 s_o[kQ4KeyWaves][CT][64];
    __shared__ floatx2 s_ml[kQ4KeyWaves][16];
    const int lane = threadIdx.x & 63, wave = threadIdx.x >> 6, col = lane & 15, g = lane >> 4;
    const Q4Item it(a, splits, 1);
    const int ntiles = (it.total + kQ4Tile - 1) / kQ4Tile, plain = a.kv_len / kQ4Tile;     // tiles whose keys all see
    const int t0 = (int)((int64_t)ntiles * it.split / splits), t1 = (int)((int64_t)ntiles * (it.split + 1) / splits);
    const char* kh = a.k + q4_tile_at(it.head, 0, a.tiles, D);
    const char* vh = a.v + q4_tile_at(it.head, 0, a.tiles, D);
    auto load = [&](Q4Tile<D>& t, int tile) {
        const size_t at = (size_t)min(tile, t1 - 1) * q4_tile_bytes(D);
        t.load(kh + at, vh + at, col, g);
    };
    Q4Tile<D> tile[2];
    load(tile[0], t0 + wave);
    half8 q[D / 32];
    q4_queries<D>(a, it, col, g, q);
    if (t1 > plain) {
        q4_masks(a, s_mask);
        __syncthreads();
    }
    const Q4Bits bits;
    const float c = fabsf(a.scale) * 1.4426950408889634f;
    Q4State<D> st;
    const int t_plain = min(t1, plain);
    int t = t0 + wave;
    // (two tiles in turn: a copy of the one on its way would have to wait for it)
    for (; t < t_plain; t += 2 * kQ4KeyWaves) {
        load(tile[1], t + kQ4KeyWaves);
        q4_tile<D, false>(a, bits, st, q, tile[0], c, t, it.total, g, nullptr);
        if (t + kQ4KeyWaves >= t_plain) {
            tile[0] = tile[1];
            t += kQ4KeyWaves;
            break;
        }
        load(tile[0], t + 2 * kQ4KeyWaves);
        q4_tile<D, false>(a, bits, st, q, tile[1], c, t + kQ4KeyWaves, it.total, g, nullptr);
    }
    const uint64_t* mask = s_mask + 2 * (col < it.R ? col / it.rep : 0);
    for (; t < t1; t += kQ4KeyWaves) {                       // the few that reach into the drafted rows
        q4_tile<D, true>(a, bits, st, q, tile[0], c, t, it.total, g, mask);
        load(tile[0], t + kQ4KeyWaves);
    }
    // the wavefronts' states meet in LDS; each finishes its share of the channel tiles
    if (g == 0) s_ml[wave][col] = (floatx2){st.m, st.l[0]};
#pragma unroll
    for (int ct = 0; ct < CT; ++ct) s_o[wave][ct][lane] = st.o[ct];
    __syncthreads();
    float m = -INFINITY, l = 0.f, f[kQ4KeyWaves];
#pragma unroll
    for (int w = 0; w < kQ4KeyWaves; ++w) m = fmaxf(m, s_ml[w][col][0]);
    const float off = m == -INFINITY ? 0.f : m;
#pragma unroll
    for (int w = 0; w < kQ4KeyWaves; ++w) {
        f[w] = __builtin_amdgcn_exp2f(s_ml[w][col][0] - off);
        l += s_ml[w][col][1] * f[w];
    }
    if (splits > 1 && wave == 0 && g == 0) ((floatx2*)a.ml_part)[(size_t)blockIdx.x * 16 + col] = (floatx2){m, l};
#pragma unroll
    for (int j = 0; j < CT / kQ4KeyWaves; ++j) {
        const int ct = wave * (CT / kQ4KeyWaves) + j;
        floatx4 o = {0.f, 0.f, 0.f, 0.f};
#pragma unroll
        for (int w = 0; w < kQ4KeyWaves; ++w) o += s_o[w][ct][lane] * f[w];
        if (splits > 1) ((floatx4*)a.o_part)[((size_t)blockIdx.x * CT + ct) * 64 + lane] = o;
        else if (col < it.R) q4_out<D>(a, it.head, it.rep, col, ct, g, o, l);
    }
}

// ---- more rows ---------------------------------------------------------------------------
// KG groups of NR wavefronts of 16 rows; the groups take stages of the keys in turn and meet at the end.  A stage is 32 keys (64 for
// eight wavefronts), a group has two buffers of it in LDS, as operands; a stage's pieces - 16 keys of K, or 64 channels of 32
// keys of V - are converted by a wavefront each.  Codes of the stage after the next are requested before a stage's products,
// converted after the next one's.  One barrier a stage.
// Bound: neither pipe: in 128 rows of 40 heads over 8320 keys (43 us) products take 22% of the time, other vector instructions 38%
// and LDS 26%, one much behind the other.  Four wavefronts on a SIMD, so 128 registers (three: 52 us).  Taken back: 32 rows a
// wavefront, which reads LDS half as often (45 to 62 us), four groups for 64 rows (18.5 us a call over 2112 keys of 32 heads,
// two 17.5, one 18.4), two for 128.
template <int D, int NR, int KG>
__global__ __launch_bounds__(NR * KG * 64, 4) void k_q4_attention_rows(const Q4Attn a, int splits, int blocks)
{
    constexpr int CT = D / 16, KS = D / 32, TS = NR == 8 ? 2 : 1;             // tiles a stage
    constexpr int kKPieces = 2 * TS, kVPieces = D / 64 * TS, kPieces = kKPieces + kVPieces;
    constexpr int kTileFrags = 2 * KS + CT, kBuf = TS * kTileFrags * 1024;
    __shared__ uint64_t s_mask[2 * GHD_MAX_M];
    __shared__ uint8_t s_bad[KG][2][TS][KS][4];
    extern __shared__ __attribute__((aligned(16))) char lds[];
    const int lane = threadIdx.x & 63, col = lane & 15, g = lane >> 4;
    const int kg = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6) / NR, wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6) % NR;
    const Q4Item it(a, splits, blocks);
    const int ntiles = (it.total + kQ4Tile - 1) / kQ4Tile, nstages = (ntiles + TS - 1) / TS;
    const int s0 = (int)((int64_t)nstages * it.split / splits), s1 = (int)((int64_t)nstages * (it.split + 1) / splits);
    const char* kh = a.k + q4_tile_at(it.head, 0, a.tiles, D);
    const char* vh = a.v + q4_tile_at(it.head, 0, a.tiles, D);
    // A piece as it is requested, the same way for both kinds (a choice between requests ends in copies, which wait for them):
    // codes; of K the row's (lo, scale), twice, of V lo and scale of group col % 2 of two.
    static_assert(kPieces <= NR, "a piece a wavefront");
    const bool of_k = wave < kKPieces;
    const int vp = wave - kKPieces, part = of_k ? wave % 2 : vp % (D / 64), of_tile = of_k ? wave / 2 : vp / (D / 64);
    const char* piece_head = of_k ? kh : vh;
    const int key = 8 * (col >> 2) + 4 * part + (col & 3);                    // (of K)
    const int off_codes = of_k ? key * (D / 2) + (D == 128 ? g : g >> 1) * 16 : ((part * 4 + g) * 16 + col) * 16;
    const int off_lo = q4_codes_bytes(D) + (of_k ? key * (D / 8) & ~15 : (2 * part + (col & 1)) * 128 + g * 16);
    const int off_scale = of_k ? off_lo : off_lo + 64;
    word4 raw[3];
    auto load = [&](int stage) {
        const char* at = piece_head + (size_t)min(min(stage, s1 - 1) * TS + of_tile, ntiles - 1) * q4_tile_bytes(D);
        raw[0] = *(const word4*)(at + off_codes);
        raw[1] = *(const word4*)(at + off_lo);
        raw[2] = *(const word4*)(at + off_scale);
    };
    const Q4Bits bits;
    auto reaches = [&](int stage) { return (stage + 1) * TS * kQ4Tile > a.kv_len; };      // into the drafted rows
    auto convert = [&](int stage, int buf) {
        char* to = lds + (kg * 2 + buf) * kBuf + of_tile * kTileFrags * 1024 + lane * 16;
        if (of_k) {
            uint32_t m = raw[1][0];
#pragma unroll
            for (int e = 1; e < 4; ++e)
                if ((D == 128 ? g : (key & 1) * 2 + (g >> 1)) == e) m = raw[1][e];
            const half2_ ms = __builtin_bit_cast(half2_, m);
#pragma unroll
            for (int s = 0; s < KS; ++s) {
                const uint32_t w = D == 128 ? raw[0][s] : g & 1 ? raw[0][(2 + s) & 3] : raw[0][s];
                *(half8*)(to + (part * KS + s) * 1024) = q4_values(bits, w, pair_of(ms[0]), pair_of(ms[1]));
            }
        } else if (vp < kVPieces) {
            half8 lo = __builtin_bit_cast(half8, raw[1]), sc = __builtin_bit_cast(half8, raw[2]);
            if (reaches(stage)) {
                const uint32_t bad = q4_clean(lo, sc, (stage * TS + of_tile) * kQ4Tile + 8 * g, it.total);
                if (col < 2) s_bad[kg][buf][of_tile][2 * part + col][g] = (uint8_t)bad;
            }
#pragma unroll
            for (int u = 0; u < 2; ++u) {
                Q4Pairs m;
                if (u == 0) m.set(q4_of_group<64, 0>(lo), q4_of_group<64, 0>(sc));
                else m.set(q4_of_group<64, 1>(lo), q4_of_group<64, 1>(sc));
#pragma unroll
                for (int x = 0; x < 2; ++x)
                    *(half8*)(to + (2 * KS + 4 * part + 2 * u + x) * 1024) = q4_values(bits, raw[0][2 * u + x], m.lo, m.s);
            }
        }
    };
    load(s0 + kg);
    const int row0 = it.block * NR * 16 + wave * 16, row = row0 + col;
    half8 q[KS];
    q4_queries<D>(a, it, row, g, q);
    if (s1 * TS * kQ4Tile > a.kv_len) q4_masks(a, s_mask);
    convert(s0 + kg, 0);
    load(s0 + kg + KG);
    __syncthreads();
    const float c = fabsf(a.scale) * 1.4426950408889634f;
    const uint64_t* mask = s_mask + 2 * (row < it.R ? row / it.rep : 0);
    Q4State<D> st;
    auto work = [&](auto MASKED, int stage) {
        constexpr bool masked = decltype(MASKED)::value;
        const int buf = (stage - s0) / KG & 1;
        if (row0 < it.R && stage < s1) {
#pragma unroll
            for (int tile = 0; tile < TS; ++tile) {
                const char* base = lds + (kg * 2 + buf) * kBuf + tile * kTileFrags * 1024 + lane * 16;
                floatx4 s[2];
#pragma unroll
                for (int h = 0; h < 2; ++h) {
                    s[h] = (floatx4){0.f, 0.f, 0.f, 0.f};
#pragma unroll
                    for (int k = 0; k < KS; ++k)
                        s[h] = __builtin_amdgcn_mfma_f32_16x16x32_f16(*(const half8*)(base + (h * KS + k) * 1024), q[k], s[h], 0, 0, 0);
                }
                uint32_t see = 0;
                if (masked) see = q4_mask32(mask[0], mask[1], (stage * TS + tile) * kQ4Tile - a.kv_len) >> 8 * g & 255u;
                const half8 p = st.template probabilities<masked>(s, c, see);
#pragma unroll
                for (int ct = 0; ct < CT; ++ct)
                    st.o[ct] = __builtin_amdgcn_mfma_f32_16x16x32_f16(*(const half8*)(base + (2 * KS + ct) * 1024), p, st.o[ct], 0, 0, 0);
                if (masked && reaches(stage))
#pragma unroll
                    for (int i = 0; i < KS; ++i) {
                        const uint32_t bad = s_bad[kg][buf][tile][i][g];
                        if (__ballot(bad != 0)) st.poison(i, bad, see);
                    }
            }
        }
        if (stage + KG < s1) {
            convert(stage + KG, buf ^ 1);
            load(stage + 2 * KG);
        }
        __syncthreads();
    };
    // (first of a turn of the groups; up to s_plain all rows see all keys of all the groups' stages)
    const int s_plain = min(s1, a.kv_len / (TS * kQ4Tile)) - KG + 1;
    int first = s0;
    for (; first < s_plain; first += KG) work(std::false_type(), first + kg);
    for (; first < s1; first += KG) work(std::true_type(), first + kg);
    if constexpr (KG > 1) {
        // the groups' states meet in LDS (behind the loop's last barrier nothing there is read any more)
        constexpr int kShare = CT * 1024 + 256;
        char* mine = lds + ((kg - 1) * NR + wave) * kShare;
        if (kg > 0) {
#pragma unroll
            for (int ct = 0; ct < CT; ++ct) ((floatx4*)mine)[ct * 64 + lane] = st.o[ct];
            if (g == 0) ((floatx2*)(mine + CT * 1024))[col] = (floatx2){st.m, st.l[0]};
        }
        __syncthreads();
        if (kg > 0) return;
#pragma unroll
        for (int k = 1; k < KG; ++k) {
            const char* other = lds + ((k - 1) * NR + wave) * kShare;
            const floatx2 ml = ((const floatx2*)(other + CT * 1024))[col];
            const float m = fmaxf(st.m, ml[0]), off = m == -INFINITY ? 0.f : m;
            const float f0 = __builtin_amdgcn_exp2f(st.m - off), f1 = __builtin_amdgcn_exp2f(ml[0] - off);
            st.m = m;
            st.l[0] = st.l[0] * f0 + ml[1] * f1;
#pragma unroll
            for (int ct = 0; ct < CT; ++ct) st.o[ct] = st.o[ct] * f0 + ((const floatx4*)other)[ct * 64 + lane] * f1;
        }
    }
    if (splits > 1) {
        const size_t unit = (size_t)blockIdx.x * NR + wave;
        if (g == 0) ((floatx2*)a.ml_part)[unit * 16 + col] = (floatx2){st.m, st.l[0]};
#pragma unroll
        for (int ct = 0; ct < CT; ++ct) ((floatx4*)a.o_part)[(unit * CT + ct) * 64 + lane] = st.o[ct];
        return;
    }
    if (row < it.R)
#pragma unroll
        for (int ct = 0; ct < CT; ++ct) q4_out<D>(a, it.head, it.rep, row, ct, g, st.o[ct], st.l[0]);
}

// ---- parts of a head's keys to its rows ----------------------------------------------------
// Four wavefronts take the parts of one fragment - 16 channels by 16 rows - in turn, eight requests at a time.
template <int D>
__global__ __launch_bounds__(256) void k_q4_join(const Q4Attn a, int splits, int blocks, int row_tiles)
{
    constexpr int CT = D / 16, kAt = 8;
    __shared__ floatx4 s_o[4][64];
    __shared__ floatx2 s_ml[4][16];
    const int lane = threadIdx.x & 63, wave = threadIdx.x >> 6, col = lane & 15, g = lane >> 4;
    const int ct = blockIdx.x % CT, rt = blockIdx.x / CT % row_tiles, hb = blockIdx.x / CT / row_tiles;
    const int block = hb % blocks, head = hb / blocks, rep = a.nh / a.nkv, row = (block * row_tiles + rt) * 16 + col;
    if ((block * row_tiles + rt) * 16 >= a.M * rep) return;
    float m = -INFINITY, l = 0.f;
    floatx4 o = {0.f, 0.f, 0.f, 0.f};
    for (int p0 = wave; p0 < splits; p0 += 4 * kAt) {
        floatx2 ml[kAt];
        floatx4 v[kAt];
        float top = m;
#pragma unroll
        for (int j = 0; j < kAt; ++j) {
            const size_t unit = ((size_t)hb * splits + min(p0 + 4 * j, splits - 1)) * row_tiles + rt;
            ml[j] = ((const floatx2*)a.ml_part)[unit * 16 + col];
            v[j] = ((const floatx4*)a.o_part)[(unit * CT + ct) * 64 + lane];
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
    if (wave != 0 || row >= a.M * rep) return;
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
    q4_out<D>(a, head, rep, row, ct, g, o, l);
}

// ---- how a call is divided -----------------------------------------------------------------
struct Q4AttnCut {
    int rows, blocks, splits;    // wavefronts of 16 rows in a workgroup, blocks of rows, parts of the keys
};
// Parts of the keys cost a launch that joins them (3 us) and what they write: as many as make 256 workgroups, one a compute unit
// (64 rows of 32 heads over 2112 keys: 2, 4, 8 parts 24.8, 19.7, 17.5 us), and where each then has long to go twice as many or,
// of the wavefronts that wait for the cache most, three times (128 rows of 40 heads over 8320 keys: 6 parts 48.4, 12 45.5;
// 1 token of 40 heads over 32000: 6 48.9, 12 44.7, 19 43.7).  No parts where a workgroup is through sooner than a second launch
// (8 tokens of 8 heads over 308 keys: 1 part 7.4, 2 9.4).
static Q4AttnCut q4_attn_cut(int M, int kv_len, int nh, int nkv)
{
    Q4AttnCut c;
    const int rt = ceil_div(M * (nh / nkv), 16), ntiles = ceil_div(kv_len + M, kQ4Tile);
    c.rows = rt <= 1 ? 1 : rt <= 4 ? 4 : 8;
    c.blocks = ceil_div(rt, c.rows);
    // what a workgroup takes at a time, in tiles, and after how many of those a part more pays
    const int step = c.rows == 1 ? kQ4KeyWaves : c.rows == 8 ? 2 : 1, turns = ceil_div(ntiles, step), items = nkv * c.blocks;
    const int far = c.rows == 1 ? 64 : 16;
    c.splits = 256 / std::min(items, 256);
    if (ntiles / c.splits > far) c.splits = (c.rows == 1 ? 768 : 512) / std::min(items, 512);
    c.splits = std::max(1, std::min(c.splits, turns <= (c.rows == 1 ? 6 : 4) ? 1 : c.rows == 1 ? turns : (turns + 1) / 2));
    return c;
}

static size_t q4_attn_units(const Q4AttnCut& c, int nkv) { return (size_t)nkv * c.blocks * c.splits * c.rows; }

size_t q4_attention_bytes(int M, int kv_len, int nh, int nkv, int d)
{
    const Q4AttnCut c = q4_attn_cut(M, kv_len, nh, nkv);
    if (c.splits == 1) return 256;
    const size_t units = q4_attn_units(c, nkv);
    return align_up(units * 16 * d * 4, 256) + align_up(units * 128, 256);
}

template <int D, int NR, int KG>
static ghd_status q4_rows_of(const Q4Attn& a, const Q4AttnCut& c, hipStream_t st)
{
    const size_t lds = (size_t)KG * 2 * (NR == 8 ? 2 : 1) * (D / 8) * 1024;
    const ghd_status s = launch_resident_checked((const void*)k_q4_attention_rows<D, NR, KG>, NR * KG * 64, lds, nullptr);
    if (s) return s;
    hipLaunchKernelGGL((k_q4_attention_rows<D, NR, KG>), dim3(a.nkv * c.blocks * c.splits), dim3(NR * KG * 64), lds, st, a, c.splits, c.blocks);
    return check_launch();
}

template <int D>
static ghd_status q4_attention_of(const Q4Attn& a, const Q4AttnCut& c, hipStream_t st)
{
    ghd_status s;
    if (c.rows == 1) {
        hipLaunchKernelGGL(k_q4_attention_keys<D>, dim3(a.nkv * c.splits), dim3(kQ4KeyWaves * 64), 0, st, a, c.splits);
        s = check_launch();
    } else if (c.rows == 4) {
        s = q4_rows_of<D, 4, 2>(a, c, st);
    } else {
        s = q4_rows_of<D, 8, 1>(a, c, st);
    }
    if (s || c.splits == 1) return s;
    hipLaunchKernelGGL(k_q4_join<D>, dim3(a.nkv * c.blocks * c.rows * (D / 16)), dim3(256), 0, st, a, c.splits, c.blocks, c.rows);
    return check_launch();
}

ghd_status launch_q4_attention(Q4Attn a, int d, void* ws, hipStream_t st)
{
    const Q4AttnCut c = q4_attn_cut(a.M, a.kv_len, a.nh, a.nkv);
    a.o_part = (float*)ws;
    a.ml_part = (float*)((char*)ws + align_up(q4_attn_units(c, a.nkv) * 16 * d * 4, 256));
    return d == 128 ? q4_attention_of<128>(a, c, st) : q4_attention_of<64>(a, c, st);
}

}  // namespace ghd
