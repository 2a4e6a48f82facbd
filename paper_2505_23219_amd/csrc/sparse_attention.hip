// Attention of the drafted tokens over the blocks that each has selected, the committed rows behind the last whole block, and the
// drafted rows that it sees.
//
// A key head's query rows - M tokens by nh / nkv heads - are the columns of S^T = K q^T and O^T = V^T P^T, so softmax statistics are a
// lane's own and probabilities come out as the operand of the second product.  Maximum and sum run along in 32 bits; probabilities
// are rounded to fp16 relative to a maximum that lags by up to 2^8 (fp16 holds that as exactly, and sums are rescaled seldom).
// A workgroup has a block of rows and reads what any of them has selected; a row that has not selected a block has the score minus
// infinity there.
#include "sparse.h"
#include "attention_impl.h"
#include "wave.h"

namespace ghd {

typedef uint32_t uint4_ __attribute__((ext_vector_type(4)));

// How a launch is divided: rows in `blocks` blocks, what a block of rows reads in `splits` parts.
struct SparseCut {
    int rows, blocks, splits;                    // rows: tiles of 16 in a block
    float inv_splits;                            // (a kernel's)
};

// What the first loads need comes in the first words of the arguments, which the hardware puts into scalar registers before a kernel
// starts; the argument block, host memory, is 0.6 us away.
// rows: kv_len (up to 2^21) | whether `relation` is masks << 31; heads: M | nkv - 1 << 8 | rep - 1 << 16; parts: splits | blocks << 16
#define SPARSE_FIRST const uint64_t *sel, const half_t *q, const void *relation, uint32_t rows, uint32_t heads, uint32_t parts, float inv_rep, \
                     float inv_splits
__device__ __forceinline__ void sparse_first(SparseArgs& a, SparseCut& cut, SPARSE_FIRST)
{
    a.sel = sel;
    a.q = q;
    a.mask = rows >> 31 ? (const uint64_t*)relation : nullptr;
    a.parent = rows >> 31 ? nullptr : (const int32_t*)relation;
    a.kv_len = rows & 0x7fffffff;
    a.n = a.kv_len / kBlock;
    a.M = heads & 255;
    a.nkv = (heads >> 8 & 255) + 1;
    a.rep = (heads >> 16) + 1;
    a.nh = a.nkv * a.rep;
    a.inv_rep = inv_rep;
    cut.splits = parts & 0xffff;
    cut.blocks = parts >> 16;
    cut.inv_splits = inv_splits;
}
static uint32_t sparse_heads(const SparseArgs& a) { return (uint32_t)a.M | (a.nkv - 1) << 8 | (a.rep - 1) << 16; }
static uint32_t sparse_parts(const SparseCut& c) { return (uint32_t)c.splits | (uint32_t)c.blocks << 16; }
// x / n of whole numbers, x below 2^20, by 1 / n: half a unit above x the quotient is at least 1 / (2 n) from a whole number, and
// what is rounded in it is less than x / n 2^-22
__device__ __forceinline__ int over(int x, float inv) { return (int)(((float)x + 0.5f) * inv); }

constexpr int kList = 1024;                      // blocks of a workgroup's list: the host divides a head's so that they fit
template <bool WIDE>
struct SparseList {
    uint64_t bits[WIDE ? 2 : 1][kList];          // a bit for each of the workgroup's tokens
    int32_t block[kList];
    int32_t part[8];
};

// What a workgroup reads: the blocks that its tokens i0 .. i1 (at most 64, or with WIDE all 128) have selected, then the `tail` that
// all read.  Words of the selection are asked for when a workgroup begins; every workgroup of a row block puts the blocks in the same order,
// a thread's one behind the other, and takes its share.
template <int THREADS, bool WIDE>
struct SparseScan {
    static constexpr int kKept = 4;              // blocks of a thread whose words stay in registers
    struct Word {
        uint64_t x, y;
        __device__ __forceinline__ bool some() const { return (x | (WIDE ? y : 0)) != 0; }
    };
    const uint64_t *lo, *hi;
    uint64_t keep, keep_hi;
    Word word[kKept];
    int n, shift;
    bool apart;                                  // (WIDE) the second word is one of its own
    __device__ __forceinline__ SparseScan(const SparseArgs& a, int head, int i0, int i1) : n(a.n), shift(i0 & 63), apart(i1 - i0 >= 64)
    {
        const int words = (a.M + 63) / 64, more = i1 - i0;
        lo = a.sel + ((size_t)head * words + (i0 >> 6)) * n;
        hi = i1 >> 6 != i0 >> 6 ? lo + n : nullptr;      // (then shift is not 0, or the tokens are all 65 to 128 of them)
        keep = more >= 63 ? ~0ull : (1ull << (more + 1)) - 1;
        keep_hi = more >= 127 ? ~0ull : more >= 64 ? (1ull << (more - 63)) - 1 : 0;
#pragma unroll
        for (int j = 0; j < kKept; ++j) word[j] = {0, 0};
        if (n == 0) return;
        // (all requests before the first is waited for)
#pragma unroll
        for (int j = 0; j < kKept; ++j) word[j].x = lo[min((int)threadIdx.x + j * THREADS, n - 1)];
        if (hi)
#pragma unroll
            for (int j = 0; j < kKept; ++j) word[j].y = hi[min((int)threadIdx.x + j * THREADS, n - 1)];
    }
    // the tokens' bits of two words as they lie
    __device__ __forceinline__ Word tokens(uint64_t x, uint64_t y) const
    {
        if (WIDE && apart) return {x & keep, y & keep_hi};
        return {(x >> shift | (hi ? y << (64 - shift) : 0)) & keep, 0};
    }
    __device__ __forceinline__ Word at(int b) const { return tokens(lo[b], hi ? hi[b] : 0); }
    // shares of `splits` to the list; returns how many blocks this one has, and how many come before the tail's in all
    __device__ __forceinline__ int list(SparseList<WIDE>& s, int tail, int split, int splits, int& before_tail)
    {
        const int tid = threadIdx.x, lane = tid & 63, wave = tid >> 6;
        int mine = 0;
#pragma unroll
        for (int j = 0; j < kKept; ++j) {
            word[j] = tid + j * THREADS < n ? tokens(word[j].x, word[j].y) : Word{0, 0};
            mine += word[j].some();
        }
        for (int b = tid + kKept * THREADS; b < n; b += THREADS) mine += at(b).some();
        int before = running_sum(mine);
        if (lane == 63) s.part[wave] = before;
        __syncthreads();
        before -= mine;
        int all = 0;
#pragma unroll
        for (int w = 0; w < THREADS / 64; ++w) {
            const int c = s.part[w];
            if (w < wave) before += c;
            all += c;
        }
        const int total = all + tail, first = (int)((int64_t)total * split / splits), end = (int)((int64_t)total * (split + 1) / splits);
        auto put = [&](int b, const Word& w) {
            if (!w.some()) return;
            if (before >= first && before < end) {
                s.bits[0][before - first] = w.x;
                if constexpr (WIDE) s.bits[1][before - first] = w.y;
                s.block[before - first] = b;
            }
            ++before;
        };
        if (mine != 0 && before < end && before + mine > first) {
#pragma unroll
            for (int j = 0; j < kKept; ++j) put(tid + j * THREADS, word[j]);
            for (int b = tid + kKept * THREADS; b < n; b += THREADS) put(b, at(b));
        }
        if (tid < tail && all + tid >= first && all + tid < end) s.block[all + tid - first] = n + tid;
        before_tail = all - first;
        return end - first;
    }
};

// 32 keys as a wavefront's operands: operand row r of half h is key 8 (r / 4) + 4 h + r % 4, so that a lane's 8 scores of a column
// are those of keys 8 g .. 8 g + 7, the probabilities it holds in the second product.  A unit's rows lie at a uniform address, a
// lane's share at a 32-bit offset.
template <int D>
struct SparseUnit {
    half8 k[2][D / 32], v[D / 16];
    // (there: how many of the unit's keys there are, one at least; others are read as the last of them)
    __device__ __forceinline__ void load_k(const SparseArgs& a, int head, int key0, int there, int lane)
    {
        const int key = 8 * ((lane & 15) >> 2) + (lane & 3);
        const char* base = (const char*)(a.k + head * a.k_head + key0 * a.k_tok);
        if (there >= 32) {
            const uint32_t at = (uint32_t)key * (uint32_t)(2 * a.k_tok) + (lane >> 4) * 16;
#pragma unroll
            for (int h = 0; h < 2; ++h)
#pragma unroll
                for (int s = 0; s < D / 32; ++s) k[h][s] = *(const half8*)(base + h * 8 * a.k_tok + s * 64 + at);
        } else {
#pragma unroll
            for (int h = 0; h < 2; ++h) {
                const uint32_t at = (uint32_t)min(key + 4 * h, there - 1) * (uint32_t)(2 * a.k_tok) + (lane >> 4) * 16;
#pragma unroll
                for (int s = 0; s < D / 32; ++s) k[h][s] = *(const half8*)(base + s * 64 + at);
            }
        }
    }
    __device__ __forceinline__ void load_v(const SparseArgs& a, int head, int key0, int there, int lane)
    {
        const char* base = (const char*)(a.v + head * a.v_head + key0);
        const uint32_t at = (uint32_t)(lane & 15) * (uint32_t)(2 * a.v_ch) + min(8 * (lane >> 4), (there - 1) & ~7) * 2;
#pragma unroll
        for (int ct = 0; ct < D / 16; ++ct) v[ct] = *(const half8*)(base + (int64_t)ct * 32 * a.v_ch + at);
    }
    // Rows that are not there may hold anything, and 0 times anything is no 0
    __device__ __forceinline__ void clean(int there, int lane)
    {
        const int mine = there - 8 * (lane >> 4);
#pragma unroll
        for (int ct = 0; ct < D / 16; ++ct) {
            uint4_ w = __builtin_bit_cast(uint4_, v[ct]);
#pragma unroll
            for (int p = 0; p < 4; ++p) w[p] &= (mine > 2 * p ? 0xffffu : 0u) | (mine > 2 * p + 1 ? 0xffff0000u : 0u);
            v[ct] = __builtin_bit_cast(half8, w);
        }
    }
};

// A row tile's state over the keys so far.
template <int D>
struct SparseState {
    floatx4 o[D / 16];
    float m, l;                        // l: the sum of the lane's own rounded probabilities
    __device__ __forceinline__ void clear()
    {
        m = -INFINITY;
        l = 0.f;
#pragma unroll
        for (int ct = 0; ct < D / 16; ++ct) o[ct] = (floatx4){0.f, 0.f, 0.f, 0.f};
    }
    // scores (of the lane's 8 keys, c makes powers of two of them) to probabilities
    __device__ __forceinline__ half8 powers(const floatx4 (&s)[2], float c)
    {
        // (of the maximum that NaN passes through: fmaxf first takes every score through an instruction that quiets NaN)
        float top = s[0][0];
#pragma unroll
        for (int e = 1; e < 8; ++e) top = __builtin_elementwise_maximum(top, s[e >> 2][e & 3]);
        top = max_over_groups(top) * c;
        // (m is minus infinity until a key is seen; m + 8 then is, too)
        if (__ballot(top > m + 8.f)) {
            const float now = top > m + 8.f ? top : m, r = m == now ? 1.f : fast_exp2(m - now);
            l *= r;
#pragma unroll
            for (int ct = 0; ct < D / 16; ++ct) o[ct] *= r;
            m = now;
        }
        // (products are rounded as the maximum was, so none passes it by more than 8: with one rounding for both, scores of 2^28 and more
        // would be off from their maximum by so much that a power overflows)
        const float off = m == -INFINITY ? 0.f : m;
        half2_ p[4];
#pragma unroll
        for (int e = 0; e < 4; ++e) {
#pragma clang fp contract(off)
            floatx2 x;
#pragma unroll
            for (int u = 0; u < 2; ++u) x[u] = fast_exp2(s[e >> 1][2 * (e & 1) + u] * c - off);
            p[e] = __builtin_convertvector(x, half2_);
        }
        const half8 all = {p[0][0], p[0][1], p[1][0], p[1][1], p[2][0], p[2][1], p[3][0], p[3][1]};
        const half_t one = (half_t)1.f;
#pragma unroll
        for (int e = 0; e < 4; ++e) l = __builtin_amdgcn_fdot2(p[e], (half2_){one, one}, l, false);
        return all;
    }
};

// The values that a row sees, one by one: for units that hold an infinity or NaN, which times the probability 0 is no 0.
template <int D>
__device__ __forceinline__ void values_one_by_one(const SparseArgs& a, int head, SparseState<D>& st, half8 p, uint32_t see, int key0, int lane)
{
    const int col = lane & 15, g = lane >> 4, total = a.kv_len + a.M;
#pragma unroll 1
    for (int key = 0; key < 32; ++key) {
        const int from = col + 16 * (key >> 3);
        float mine = 0.f;
#pragma unroll
        for (int e = 0; e < 8; ++e) mine = (key & 7) == e ? (float)p[e] : mine;
        const float pk = __shfl(mine, from);
        if (__shfl((int)see, from) >> (key & 7) & 1) {
            const half_t* vp = a.v + head * a.v_head + min(key0 + key, total - 1) + (int64_t)(4 * g) * a.v_ch;
#pragma unroll
            for (int ct = 0; ct < D / 16; ++ct) {
#pragma unroll
                for (int e = 0; e < 4; ++e) st.o[ct][e] += pk * (float)vp[(int64_t)(ct * 16 + e) * a.v_ch];
                __builtin_amdgcn_sched_barrier(0);
            }
        }
    }
}
// Has a row met such a value?  (Its sum of probabilities is finite then; otherwise it is the scores that are not.)
template <int D, int RT>
__device__ __forceinline__ bool not_finite(const SparseState<D> (&st)[RT])
{
    bool odd = false;
#pragma unroll
    for (int r = 0; r < RT; ++r) {
        bool mine = false;
#pragma unroll
        for (int ct = 0; ct < D / 16; ++ct)
#pragma unroll
            for (int e = 0; e < 4; ++e) mine = mine || !(fabsf(st[r].o[ct][e]) < INFINITY);
        odd = odd || (mine && fabsf(sum_over_groups(st[r].l)) < INFINITY);
    }
    return odd;
}

// Which token a column is, and which of a workgroup's tokens a tile of rows has.
__device__ __forceinline__ int token_of(const SparseArgs& a, int row) { return min(over(row, a.inv_rep), a.M - 1); }
__device__ __forceinline__ uint64_t tile_tokens(const SparseArgs& a, int row0, int i0)
{
    const int from = over(row0, a.inv_rep) - i0, to = token_of(a, row0 + 15) - i0;
    return from > to ? 0 : (to - from >= 63 ? ~0ull : (1ull << (to - from + 1)) - 1) << from;
}
__device__ __forceinline__ uint64_t uniform64(uint64_t x)
{
    return (uint64_t)(uint32_t)__builtin_amdgcn_readfirstlane((int)(x >> 32)) << 32 | (uint32_t)__builtin_amdgcn_readfirstlane((int)x);
}
// a row's share of q as an operand; where there is no row, the last one's
template <int D>
__device__ __forceinline__ half8 sparse_query(const SparseArgs& a, int head, int row, int s, int g)
{
    row = min(row, a.M * a.rep - 1);
    const int token = over(row, a.inv_rep);
    const half8 x = *(const half8*)(a.q + ((size_t)token * a.nh + head * a.rep + row - token * a.rep) * D + s * 32 + g * 8);
    return a.scale < 0.f ? -x : x;
}
// scores to powers of two; above 0, so that minus infinity stays that
__device__ __forceinline__ float sparse_power(float scale) { return fmaxf(fabsf(scale) * 1.4426950408889634f, 1e-37f); }

// a row's output from the sums and their divisor; a row that sees no key gives zeros
__device__ __forceinline__ void sparse_out(const SparseArgs& a, int head, int row, int d, int ct, int g, floatx4 o, float l)
{
    const int token = over(row, a.inv_rep);
    const float r = 1.f / l;
    half4 y;
#pragma unroll
    for (int e = 0; e < 4; ++e) y[e] = l == 0.f ? (half_t)0.f : (half_t)(o[e] * r);
    *(half4*)(a.out + ((size_t)token * a.nh + head * a.rep + row - token * a.rep) * d + ct * 16 + 4 * g) = y;
}

template <int D, int RT>
struct SparseShape {
    static constexpr int kWaves = RT == 1 ? 4 : 8, kThreads = kWaves * 64, CT = D / 16, KS = D / 32, kFrags = RT * CT,
                         kRound = kFrags < 16 ? kFrags : 16;           // fragments that meet at a time
    static constexpr size_t kLds = (size_t)kWaves * kRound * 1024;      // queries first, states at the end
};

// Up to 32 rows: a wavefront takes every fourth (eighth) half block of the list by itself, keys and values straight to registers, the next
// half block's asked for before this one's products; wavefronts meet in LDS at the end.  Bound: few bytes for so many compute units - what
// comes before the first key and behind the last product.  One token, 32 heads on 8, 64 blocks of 128 channels, 17 MB: 11.2 us,
// with arguments from memory 0.5 us more, and with 512 workgroups instead of 256.
template <int D, int RT>
__global__ __launch_bounds__(RT == 1 ? 256 : 512, RT == 1 ? 3 : 2) void k_sparse_attention(SPARSE_FIRST, SparseArgs a, SparseCut cut)
{
    sparse_first(a, cut, sel, q, relation, rows, heads, parts, inv_rep, inv_splits);
    typedef SparseShape<D, RT> S;
    constexpr int CT = S::CT, KS = S::KS, W = S::kWaves;
    __shared__ SparseList<false> list;
    __shared__ uint64_t s_mask[2 * GHD_MAX_M];
    __shared__ floatx2 s_ml[W][RT * 16];
    extern __shared__ __attribute__((aligned(16))) char lds[];
    const int lane = threadIdx.x & 63, wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6), g = lane >> 4, col = lane & 15;
    // 8 XCDs by blocks, by parts in eights: the row blocks of a part of a head's keys share an L2
    const int item = blockIdx.y * 8 + (blockIdx.x & 7);
    if (item >= a.nkv * cut.splits) return;
    const int block = blockIdx.x >> 3, head = __builtin_amdgcn_readfirstlane(over(item, cut.inv_splits)), split = item - head * cut.splits;
    const int row0 = block * RT * 16, R = a.M * a.rep, i0 = over(row0, a.inv_rep), i1 = token_of(a, row0 + RT * 16 - 1);
    const int total = a.kv_len + a.M, tail = (total - a.n * kBlock + kBlock - 1) / kBlock;
    SparseScan<S::kThreads, false> scan(a, head, i0, i1);
    constexpr int kMine = (RT * KS + W - 1) / W;                   // operands of q that a wavefront brings
    half8 x[kMine];
#pragma unroll
    for (int f = 0; f < kMine; ++f) {
        const int frag = min(f * W + wave, RT * KS - 1);
        x[f] = sparse_query<D>(a, head, row0 + frag / KS * 16 + col, frag % KS, g);
    }
    int up0 = 0, up1 = 0;
    if (wave == 0 && a.parent) {
        up0 = a.parent[min(lane, a.M - 1)];
        up1 = a.parent[min(lane + 64, a.M - 1)];
    }
    int before_tail;
    const int count = scan.list(list, tail, split, cut.splits, before_tail);
    if (before_tail < count) {                                     // it has some of the rows behind the blocks
        if (!a.parent)
            for (int e = threadIdx.x; e < 2 * a.M; e += S::kThreads) s_mask[e] = a.mask[e];
        else if (wave == 0)
            store_masks(tree_nodes<2, true>(up0, up1, a.M, lane), a.M, lane, s_mask);
    }
#pragma unroll
    for (int f = 0; f < kMine; ++f)
        if (f * W + wave < RT * KS) *(half8*)(lds + (f * W + wave) * 1024 + lane * 16) = x[f];
    __syncthreads();
    auto query = [&](int r, int s) { return *(const half8*)(lds + (r * KS + s) * 1024 + lane * 16); };
    const float c = sparse_power(a.scale);
    uint32_t tokens = 0;                                           // of a lane's columns, 8 bits each
    auto token = [&](int r) { return (int)(tokens >> 8 * r & 255); };
    uint64_t tile_bits[RT];
#pragma unroll
    for (int r = 0; r < RT; ++r) {
        tokens |= (uint32_t)token_of(a, row0 + r * 16 + col) << 8 * r;
        tile_bits[r] = tile_tokens(a, row0 + r * 16, i0);
    }
    SparseState<D> st[RT];
    const int units = sparse_halves(count, list.block[max(count - 1, 0)], total);
    auto key_of = [&](int u) { return __builtin_amdgcn_readfirstlane(list.block[u >> 1]) * kBlock + (u & 1) * 32; };
    // One pass over the wavefront's units.  PLAIN: every row meets all of a unit's values, those that it does not see with
    // the probability 0; an infinity or NaN there is no 0 then.  Otherwise a row takes the values that it sees one by one.
    auto pass = [&](auto plain) {
#pragma unroll
        for (int r = 0; r < RT; ++r) st[r].clear();
        int u = wave;
        if (u >= units) return;
        SparseUnit<D> unit;
        int key0 = key_of(u);
        unit.load_k(a, head, key0, min(32, total - key0), lane);
        unit.load_v(a, head, key0, min(32, total - key0), lane);
        for (;;) {
            const int next = u + W < units ? u + W : u, next0 = key_of(next), there = total - key0;
            const int next_there = min(32, total - next0);
            const bool rest = key0 >= a.n * kBlock;                // behind the blocks
            const uint64_t bits = rest ? ~0ull : uniform64(list.bits[0][u >> 1]);
            if (there < 32) unit.clean(there, lane);
#pragma unroll
            for (int r = 0; r < RT; ++r) {
                const bool met = (bits & tile_bits[r]) != 0;
                half8 p;
                uint32_t see = 0;
                if (met) {
                    floatx4 s[2];
#pragma unroll
                    for (int h = 0; h < 2; ++h) {
                        s[h] = (floatx4){0.f, 0.f, 0.f, 0.f};
#pragma unroll
                        for (int ks = 0; ks < KS; ++ks)
                            s[h] = __builtin_amdgcn_mfma_f32_16x16x32_f16(unit.k[h][ks], query(r, ks), s[h], 0, 0, 0);
                    }
                    see = rest ? seen_keys((const uint32_t*)(s_mask + 2 * token(r)), key0 + g * 8, a.kv_len, total)
                               : bits >> (token(r) - i0) & 1 ? 0xffu : 0u;
                    if (rest || (bits & tile_bits[r]) != tile_bits[r])
#pragma unroll
                        for (int e = 0; e < 8; ++e) s[e >> 2][e & 3] = see >> e & 1 ? s[e >> 2][e & 3] : -INFINITY;
                    p = st[r].powers(s, c);
                }
                if (r == RT - 1) unit.load_k(a, head, next0, next_there, lane);
                if (!met) continue;
                if constexpr (decltype(plain)::value) {
#pragma unroll
                    for (int ct = 0; ct < CT; ++ct) st[r].o[ct] = __builtin_amdgcn_mfma_f32_16x16x32_f16(unit.v[ct], p, st[r].o[ct], 0, 0, 0);
                } else {
                    values_one_by_one<D>(a, head, st[r], p, see, key0, lane);
                }
            }
            if (next == u) break;
            unit.load_v(a, head, next0, next_there, lane);
            u = next;
            key0 = next0;
        }
    };
    pass(std::true_type{});
    if (__builtin_expect(__ballot(not_finite<D, RT>(st)) != 0, 0)) pass(std::false_type{});
    // the wavefronts' states meet in LDS, some fragments at a time, each added up by one wavefront
#pragma unroll
    for (int r = 0; r < RT; ++r) {
        const float l = sum_over_groups(st[r].l);
        if (g == 0) s_ml[wave][r * 16 + col] = (floatx2){st[r].m, l};
    }
    const size_t unit0 = (((size_t)head * cut.blocks + block) * cut.splits + split) * RT;
    floatx4* const part = (floatx4*)lds + lane;                    // [wave][fragment][64]
#pragma unroll
    for (int f0 = 0; f0 < S::kFrags; f0 += S::kRound) {
        __syncthreads();
#pragma unroll
        for (int f = f0; f < f0 + S::kRound && f < S::kFrags; ++f) part[(wave * S::kRound + f - f0) * 64] = st[f / CT].o[f % CT];
        __syncthreads();
#pragma unroll 2
        for (int e = wave; e < S::kRound && f0 + e < S::kFrags; e += W) {
            const int f = f0 + e, r = f / CT, ct = f % CT, row = row0 + r * 16 + col;
            float m = -INFINITY, l = 0.f;
            floatx2 ml[W];
            floatx4 o = {0.f, 0.f, 0.f, 0.f};
#pragma unroll
            for (int w = 0; w < W; ++w) {
                ml[w] = s_ml[w][r * 16 + col];
                m = fmaxf(m, ml[w][0]);
            }
            const float off = m == -INFINITY ? 0.f : m;
#pragma unroll
            for (int w = 0; w < W; ++w) {
                const float by = fast_exp2(ml[w][0] - off);
                l += ml[w][1] * by;
                o += part[(w * S::kRound + e) * 64] * by;
            }
            if (row >= R) continue;
            if (cut.splits > 1) {
                ((floatx4*)a.o_part)[((unit0 + r) * CT + ct) * 64 + lane] = o;
                if (ct == 0 && g == 0) ((floatx2*)a.ml_part)[(unit0 + r) * 16 + col] = (floatx2){m, l};
            } else {
                sparse_out(a, head, row, D, ct, g, o, l);
            }
        }
    }
}

// ---- more rows ----------------------------------------------------------------------------
// Wavefronts that read keys by themselves read them once for each tile or two of rows, so above 32 rows a block of keys is read once for all rows
// of a workgroup: straight to LDS, four blocks of 64 keys on their way, while eight wavefronts - four groups of rows, each RT tiles of
// 16, by halves of a block - take their operands from there.
constexpr int kStages = 4;
template <int D>
struct StagedShape {
    static constexpr int kHalf = 128 * D, kStage = 2 * kHalf;     // bytes of a block's keys (as many of values), and of both
    static constexpr int kPieces = D / 64;                         // KiB of each that a wavefront brings
    static constexpr size_t kLds = kStages * kStage;
};

// A KiB of the LDS is 4 (or 8) rows of K or 8 channels of V^T; the 16-byte pieces of a row lie in an order of their own (piece p of row r in place
// p ^ f(r)), so that the 16 rows that an operand takes the same piece of are spread over all banks.
template <int D>
struct StagedBlock {
    uint32_t k_row, k_piece, v_ch, v_piece;                        // what the lane brings
    uint32_t k_at, v_at;                                           // where it finds its operands, but for the k-step's piece
    __device__ __forceinline__ StagedBlock(int wave, int lane)
    {
        constexpr int kLanes = D / 8, kRows = 64 / kLanes;         // lanes of a row, rows of a KiB
        const int col = lane & 15;
        k_row = wave * StagedShape<D>::kPieces * kRows + lane / kLanes;
        k_piece = lane % kLanes;
        v_ch = wave * StagedShape<D>::kPieces * 8 + lane / 8;
        v_piece = lane % 8;
        k_at = (uint32_t)((col >> 2) * 8 + (col & 3)) * (D * 2);
        v_at = StagedShape<D>::kHalf + (uint32_t)col * 128;
    }
    // f of a row of K: the column that has it, by twos where a row is 128 bytes
    __device__ __forceinline__ static uint32_t k_turn(uint32_t key)
    {
        const uint32_t col = (key & 3) | (key >> 3 & 3) << 2;
        return D == 128 ? col : col >> 1;
    }
    __device__ __forceinline__ void request(const SparseArgs& a, int head, int block, int wave, uint32_t lds) const
    {
        constexpr int kRows = 512 / D, kPieces = StagedShape<D>::kPieces;
        const int there = a.kv_len + a.M - block * kBlock;         // rows of the block, and behind it
        const auto k = (GLOBAL const char*)gp(a.k + head * a.k_head + (int64_t)block * kBlock * a.k_tok);
        const auto v = (GLOBAL const char*)gp(a.v + head * a.v_head + (int64_t)block * kBlock);
#pragma unroll
        for (int i = 0; i < kPieces; ++i) {
            const uint32_t key = k_row + i * kRows;
            to_lds(k, (uint32_t)min((int)key, there - 1) * (uint32_t)(2 * a.k_tok) + (k_piece ^ k_turn(key)) * 16, lds + (wave * kPieces + i) * 1024);
        }
#pragma unroll
        for (int i = 0; i < kPieces; ++i) {
            const uint32_t ch = v_ch + i * 8;
            to_lds(v, ch * (uint32_t)(2 * a.v_ch) + min((v_piece ^ (ch >> 1 & 7)) * 16, (uint32_t)((there - 1) >> 3) * 16),
                   lds + StagedShape<D>::kHalf + (wave * kPieces + i) * 1024);
        }
    }
    __device__ __forceinline__ half8 key(const char* at, int half, int h, int s, int lane) const
    {
        const uint32_t col = lane & 15, turn = D == 128 ? col : col >> 1;
        return *(const half8*)(at + k_at + (half * 32 + h * 4) * (D * 2) + ((s * 4 + (lane >> 4)) ^ turn) * 16);
    }
    __device__ __forceinline__ half8 value(const char* at, int half, int ct, int lane) const
    {
        return *(const half8*)(at + v_at + ct * 2048 + ((half * 4 + (lane >> 4)) ^ (lane & 15) >> 1) * 16);
    }
};

// Bound: the loads, but by what is not known.  64 tokens, 32 heads, lists of up to 48 blocks: 19.3 us, without the products 19.7 of 23.3 (of an
// earlier state); 128 tokens, 40 heads, up to 96 blocks: 42.5 us, without them 42.4 of 47.7: a workgroup's 17 blocks of 32 KB come at
// 13 GB/s, with 96 KB on their way, where attn_staged (attention_impl.h) has twice that inside its step's launch.  All 131 blocks of those tokens
// take 52.8 us with the join, 3.2 TB/s; ghd_tree_attention's 49.4.  Loads past the L2: 46.2 of 48.3, but 23.8 against 22.9 for the tree,
// so none has them; 256 rows in four wavefronts of 512 registers: 63.
template <int D, int RT>
__global__ __launch_bounds__(512, 2) void k_sparse_staged(SPARSE_FIRST, SparseArgs a, SparseCut cut)
{
    sparse_first(a, cut, sel, q, relation, rows, heads, parts, inv_rep, inv_splits);
    constexpr int CT = D / 16, KS = D / 32, W = 8, kLoads = 2 * StagedShape<D>::kPieces;
    constexpr bool WIDE = RT > 1;
    __shared__ SparseList<WIDE> list;
    __shared__ uint64_t s_mask[2 * GHD_MAX_M];
    __shared__ floatx2 s_ml[W][RT * 16];
    extern __shared__ __attribute__((aligned(16))) char lds[];
    const uint32_t lds0 = (uint32_t)(uintptr_t)(__attribute__((address_space(3))) char*)lds;
    const int lane = threadIdx.x & 63, wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6), g = lane >> 4, col = lane & 15;
    const int item = blockIdx.y * 8 + (blockIdx.x & 7);
    if (item >= a.nkv * cut.splits) return;
    const int block = blockIdx.x >> 3, head = __builtin_amdgcn_readfirstlane(over(item, cut.inv_splits)), split = item - head * cut.splits;
    const int row0 = block * RT * 64, R = a.M * a.rep, i0 = over(row0, a.inv_rep), i1 = token_of(a, row0 + RT * 64 - 1);
    const int total = a.kv_len + a.M, tail = (total - a.n * kBlock + kBlock - 1) / kBlock;
    const int group = wave >> 1, half = wave & 1, my_row = row0 + group * RT * 16;
    SparseScan<512, WIDE> scan(a, head, i0, i1);
    half8 ask[RT][KS];
#pragma unroll
    for (int r = 0; r < RT; ++r)
#pragma unroll
        for (int s = 0; s < KS; ++s) ask[r][s] = sparse_query<D>(a, head, my_row + r * 16 + col, s, g);
    int up0 = 0, up1 = 0;
    if (wave == 0 && a.parent) {
        up0 = a.parent[min(lane, a.M - 1)];
        up1 = a.parent[min(lane + 64, a.M - 1)];
    }
    int before_tail;
    const int count = scan.list(list, tail, split, cut.splits, before_tail);
    __syncthreads();
    const StagedBlock<D> staged(wave, lane);
    auto request = [&](int i) {
        staged.request(a, head, __builtin_amdgcn_readfirstlane(list.block[i]), wave, lds0 + (uint32_t)(i & (kStages - 1)) * StagedShape<D>::kStage);
    };
    // (the queries are there before that: otherwise they are waited for together with all of these)
#pragma unroll
    for (int r = 0; r < RT; ++r)
#pragma unroll
        for (int s = 0; s < KS; ++s) asm volatile("" : "+v"(ask[r][s]));
    for (int i = 0; i < min(count, kStages - 1); ++i) request(i);
    if (before_tail < count) {
        if (!a.parent)
            for (int e = threadIdx.x; e < 2 * a.M; e += 512) s_mask[e] = a.mask[e];
        else if (wave == 0)
            store_masks(tree_nodes<2, true>(up0, up1, a.M, lane), a.M, lane, s_mask);
    }
    const float c = sparse_power(a.scale);
    // (128 tokens are in two words: of a group of 32 rows in one of them)
    const bool second = over(my_row, a.inv_rep) - i0 >= 64;
    const int base = i0 + (second ? 64 : 0);
    int token[RT];
    uint64_t tile_bits[RT];
#pragma unroll
    for (int r = 0; r < RT; ++r) {
        token[r] = token_of(a, my_row + r * 16 + col);
        tile_bits[r] = my_row + r * 16 < R ? tile_tokens(a, my_row + r * 16, base) : 0;
    }
    SparseState<D> st[RT];
    auto pass = [&](auto plain) {
#pragma unroll
        for (int r = 0; r < RT; ++r) st[r].clear();
        for (int i = 0; i < count; ++i) {
            // a barrier a block: it is there for everybody, and everybody is done with the one before, whose place is requested into
            const int young = min(count - 1 - i, kStages - 2);
            if (young == 2) wait_loads<2 * kLoads>();
            else if (young == 1) wait_loads<kLoads>();
            else wait_loads<0>();
            pin_order();
            barrier_lds();
            if (i + kStages - 1 < count) request(i + kStages - 1);
            const int at = __builtin_amdgcn_readfirstlane(list.block[i]), key0 = at * kBlock + half * 32, there = total - key0;
            const bool rest = at >= a.n;
            const uint64_t bits = rest ? ~0ull : uniform64(list.bits[WIDE && second][i]);
            uint64_t mine = 0;
#pragma unroll
            for (int r = 0; r < RT; ++r) mine |= tile_bits[r];
            if (there <= 0 || (bits & mine) == 0) continue;
            const char* const buf = lds + (i & (kStages - 1)) * StagedShape<D>::kStage;
            half8 k[2][KS], v[CT];
#pragma unroll
            for (int h = 0; h < 2; ++h)
#pragma unroll
                for (int s = 0; s < KS; ++s) k[h][s] = staged.key(buf, half, h, s, lane);
            __builtin_amdgcn_sched_barrier(0);
            half8 p[RT];
            uint32_t see[RT];
#pragma unroll
            for (int r = 0; r < RT; ++r) {
                floatx4 s[2];
#pragma unroll
                for (int h = 0; h < 2; ++h) {
                    s[h] = (floatx4){0.f, 0.f, 0.f, 0.f};
#pragma unroll
                    for (int ks = 0; ks < KS; ++ks) s[h] = __builtin_amdgcn_mfma_f32_16x16x32_f16(k[h][ks], ask[r][ks], s[h], 0, 0, 0);
                }
                if (r == 0) {
#pragma unroll
                    for (int ct = 0; ct < CT; ++ct) v[ct] = staged.value(buf, half, ct, lane);
                }
                see[r] = rest ? seen_keys((const uint32_t*)(s_mask + 2 * token[r]), key0 + g * 8, a.kv_len, total)
                              : bits >> (max(token[r] - base, 0) & 63) & 1 ? 0xffu : 0u;
                if (rest || (bits & tile_bits[r]) != tile_bits[r])
#pragma unroll
                    for (int e = 0; e < 8; ++e) s[e >> 2][e & 3] = see[r] >> e & 1 ? s[e >> 2][e & 3] : -INFINITY;
                p[r] = st[r].powers(s, c);
            }
            if (there < 32) {
                // rows that are not there may hold anything, and 0 times anything is no 0
                const int some = there - 8 * g;
#pragma unroll
                for (int ct = 0; ct < CT; ++ct) {
                    uint4_ w = __builtin_bit_cast(uint4_, v[ct]);
#pragma unroll
                    for (int e = 0; e < 4; ++e) w[e] &= (some > 2 * e ? 0xffffu : 0u) | (some > 2 * e + 1 ? 0xffff0000u : 0u);
                    v[ct] = __builtin_bit_cast(half8, w);
                }
            }
#pragma unroll
            for (int r = 0; r < RT; ++r) {
                if constexpr (decltype(plain)::value) {
#pragma unroll
                    for (int ct = 0; ct < CT; ++ct) st[r].o[ct] = __builtin_amdgcn_mfma_f32_16x16x32_f16(v[ct], p[r], st[r].o[ct], 0, 0, 0);
                } else {
                    values_one_by_one<D>(a, head, st[r], p[r], see[r], key0, lane);
                }
            }
        }
    };
    pass(std::true_type{});
    if (__builtin_expect(__syncthreads_or(not_finite<D, RT>(st)), 0)) {
        for (int i = 0; i < min(count, kStages - 1); ++i) request(i);
        pass(std::false_type{});
    }
    // the two wavefronts of a group meet in LDS, each adds up half of the fragments
#pragma unroll
    for (int r = 0; r < RT; ++r) {
        const float l = sum_over_groups(st[r].l);
        if (g == 0) s_ml[wave][r * 16 + col] = (floatx2){st[r].m, l};
    }
    __syncthreads();
    floatx4* const part = (floatx4*)lds + lane;                    // [wave][fragment][64]
#pragma unroll
    for (int f = 0; f < RT * CT; ++f) part[(wave * RT * CT + f) * 64] = st[f / CT].o[f % CT];
    __syncthreads();
    const size_t unit0 = (((size_t)head * cut.blocks + block) * cut.splits + split) * (RT * 4) + group * RT;
#pragma unroll 2
    for (int f = half; f < RT * CT; f += 2) {
        const int r = f / CT, ct = f % CT, row = my_row + r * 16 + col;
        const floatx2 x = s_ml[wave & ~1][r * 16 + col], y = s_ml[wave | 1][r * 16 + col];
        const float m = fmaxf(x[0], y[0]), off = m == -INFINITY ? 0.f : m, bx = fast_exp2(x[0] - off), by = fast_exp2(y[0] - off);
        const float l = x[1] * bx + y[1] * by;
        const floatx4 o = part[((wave & ~1) * RT * CT + f) * 64] * bx + part[((wave | 1) * RT * CT + f) * 64] * by;
        if (row >= R) continue;
        if (cut.splits > 1) {
            ((floatx4*)a.o_part)[((unit0 + r) * CT + ct) * 64 + lane] = o;
            if (ct == 0 && g == 0) ((floatx2*)a.ml_part)[(unit0 + r) * 16 + col] = (floatx2){m, l};
        } else {
            sparse_out(a, head, row, D, ct, g, o, l);
        }
    }
}

// Parts to rows: four wavefronts take the parts of a fragment, 16 channels by 16 rows, in turn, eight requests at a time.
// Bound: a launch and a round of loads: 4 us; 128 tokens of 40 heads in 6 parts of 8 tiles 6.8 us.
template <int D>
__global__ __launch_bounds__(256) void k_sparse_join(const float* o_part, const float* ml_part, half_t* out, uint32_t heads, uint32_t parts, int rows,
                                                     float inv_rep)
{
    SparseArgs a = {};
    SparseCut cut = {};
    sparse_first(a, cut, nullptr, nullptr, nullptr, 0, heads, parts, inv_rep, 0.f);
    a.out = out;
    cut.rows = rows;
    constexpr int CT = D / 16, kAt = 8;
    __shared__ floatx4 s_o[4][64];
    __shared__ floatx2 s_ml[4][16];
    const int lane = threadIdx.x & 63, wave = threadIdx.x >> 6, g = lane >> 4, col = lane & 15;
    const int ct = blockIdx.x % CT, rt = blockIdx.x / CT, block = blockIdx.y, head = blockIdx.z, row = (block * cut.rows + rt) * 16 + col;
    if ((block * cut.rows + rt) * 16 >= a.M * a.rep) return;
    const bool is = row < a.M * a.rep;                             // (no part has written the others)
    const size_t unit0 = ((size_t)head * cut.blocks + block) * cut.splits;
    float m = -INFINITY, l = 0.f;
    floatx4 o = {0.f, 0.f, 0.f, 0.f};
    for (int p0 = wave; p0 < cut.splits; p0 += 4 * kAt) {
        floatx2 ml[kAt];
        floatx4 v[kAt];
        float top = m;
#pragma unroll
        for (int j = 0; j < kAt; ++j) {
            const int part = p0 + 4 * j;
            const size_t unit = (unit0 + min(part, cut.splits - 1)) * cut.rows + rt;
            ml[j] = (floatx2){-INFINITY, 0.f};
            v[j] = (floatx4){0.f, 0.f, 0.f, 0.f};
            if (is && part < cut.splits) {
                ml[j] = ((const floatx2*)ml_part)[unit * 16 + col];
                v[j] = ((const floatx4*)o_part)[(unit * CT + ct) * 64 + lane];
            }
        }
#pragma unroll
        for (int j = 0; j < kAt; ++j) top = fmaxf(top, ml[j][0]);
        const float off = top == -INFINITY ? 0.f : top, r = fast_exp2(m - off);
        l *= r;
        o *= r;
#pragma unroll
        for (int j = 0; j < kAt; ++j) {
            const float by = fast_exp2(ml[j][0] - off);
            l += ml[j][1] * by;
            o += v[j] * by;
        }
        m = top;
    }
    s_o[wave][lane] = o;
    if (g == 0) s_ml[wave][col] = (floatx2){m, l};
    __syncthreads();
    if (wave != 0 || !is) return;
    float top = -INFINITY;
#pragma unroll
    for (int w = 0; w < 4; ++w) top = fmaxf(top, s_ml[w][col][0]);
    const float off = top == -INFINITY ? 0.f : top;
    l = 0.f;
    o = (floatx4){0.f, 0.f, 0.f, 0.f};
#pragma unroll
    for (int w = 0; w < 4; ++w) {
        const float by = fast_exp2(s_ml[w][col][0] - off);
        l += s_ml[w][col][1] * by;
        o += s_o[w][lane] * by;
    }
    sparse_out(a, head, row, D, ct, g, o, l);
}

// What is estimated to be fastest of blocks of 1, 2 (wavefronts by themselves), 4 and 8 tiles of rows (through LDS) and of parts
// that make 128 or 256 workgroups, in us: a launch takes `fixed`, every round of the workgroups on an XCD's 32 compute units `round` and for
// each block of keys of a part `block`, a second launch `join` and what it reads and writes.  Fitted to 2178 calls (1 to 128 tokens, 2 to 40
// key heads, 777 to 16384 rows; off by 5% in the mean); the fastest of a call's cuts is missed by 1.2% in the mean, 23% at
// the most.  A token's blocks are on the device: a row block is taken to read 64, which is what decides between the cuts best.
static SparseCut sparse_cut(int M, int kv_len, int nh, int nkv, int d)
{
    static const struct {
        int rows;
        float fixed, round, block, join, mb;
    } kinds[2][4] = {{{1, 4.5f, 0.f, .48f, 3.1f, 1.f}, {2, 2.6f, 3.7f, .48f, 2.9f, .83f}, {4, 7.5f, .6f, .78f, 1.f, .53f}, {8, 4.f, 3.2f, 1.18f, 2.6f, .61f}},
                     {{1, 3.9f, 0.f, .95f, 3.7f, .83f}, {2, 2.9f, 4.f, .98f, 2.8f, .75f}, {4, 5.4f, 3.3f, 1.08f, 1.f, .62f}, {8, 7.f, 2.6f, 1.5f, 3.f, .49f}}};
    const int tiles = ceil_div(M * (nh / nkv), 16), n = kv_len / kBlock;
    const int most = n + ceil_div(kv_len + M - n * kBlock, kBlock);      // blocks that a row can read
    SparseCut best = {};
    float least = 0.f;
    for (const auto& k : kinds[d == 128]) {
        if (k.rows == 1 ? tiles > 4 : k.rows >= 2 * tiles) continue;
        const int blocks = ceil_div(tiles, k.rows), items = nkv * blocks;
        for (int wgs = 128; wgs <= 256; wgs += 128) {
            const int splits = std::max(ceil_div(most, kList), std::min(most, std::max(1, wgs / items)));
            const int on_xcd = ceil_div(nkv * splits, 8) * blocks;
            // (of workgroups of one tile, four wavefronts, a compute unit has several)
            const float rounds = k.rows == 1 ? std::max(1.f, on_xcd / 32.f) : (float)ceil_div(on_xcd, 32);
            float us = k.fixed + rounds * (k.round + ceil_div(std::min(most, 64), splits) * k.block);
            if (splits > 1) us += k.join + k.mb * 64e-6f * items * splits * k.rows * d;
            if (least == 0.f || us < least) {
                least = us;
                best = {k.rows, blocks, splits, 1.f / splits};
            }
        }
    }
    return best;
}

static size_t sparse_units(const SparseCut& c, int nkv) { return c.splits == 1 ? 0 : (size_t)nkv * c.blocks * c.splits * c.rows; }
static size_t sparse_o_bytes(size_t units, int d) { return align_up(units * 16 * d * 4, 256); }
static size_t sparse_bytes(size_t units, int d) { return std::max<size_t>(256, sparse_o_bytes(units, d) + align_up(units * 128, 256)); }

// The most that a call of up to M tokens over up to kv_len rows takes, whatever its cut: parts are at most 256 workgroups of eight
// tiles of rows and a part reads a block, or as many as a list's length makes of them; blocks end up to seven tiles behind the rows.
size_t sparse_attention_bytes(int M, int kv_len, int nh, int nkv, int d)
{
    const size_t tiles = ceil_div(M * (nh / nkv), 16) + 7, most = kv_len / kBlock + 1 + ceil_div(M, kBlock);
    return sparse_bytes(std::max(std::min<size_t>(2048, nkv * tiles * most), most > kList ? nkv * tiles * ((most + kList - 1) / kList) : 0), d);
}

void sparse_attention_on_host(int M, int kv_len, int nh, int nkv, int d, int64_t* out4)
{
    const SparseCut c = sparse_cut(M, kv_len, nh, nkv, d);
    out4[0] = c.rows;
    out4[1] = c.blocks;
    out4[2] = c.splits;
    out4[3] = sparse_bytes(sparse_units(c, nkv), d);
}

template <int D, int RT, bool STAGED>
static ghd_status sparse_rows(const SparseArgs& a, const SparseCut& c, hipStream_t st)
{
    void (*const kernel)(SPARSE_FIRST, SparseArgs, SparseCut) = STAGED ? k_sparse_staged<D, RT> : k_sparse_attention<D, RT>;
    const int threads = STAGED ? 512 : SparseShape<D, RT>::kThreads;
    const size_t lds = STAGED ? StagedShape<D>::kLds : SparseShape<D, RT>::kLds;
    const ghd_status s = launch_resident_checked((const void*)kernel, threads, lds, nullptr);
    if (s) return s;
    hipLaunchKernelGGL(kernel, dim3(8 * c.blocks, ceil_div(a.nkv * c.splits, 8)), dim3(threads), lds, st, a.sel, a.q,
                       a.mask ? (const void*)a.mask : (const void*)a.parent, (uint32_t)a.kv_len | (a.mask ? 1u << 31 : 0u),
                       sparse_heads(a), sparse_parts(c),
                       a.inv_rep, c.inv_splits, a, c);
    return check_launch();
}

template <int D>
static ghd_status sparse_of(const SparseArgs& a, const SparseCut& c, hipStream_t st)
{
    const ghd_status s = c.rows == 1   ? sparse_rows<D, 1, false>(a, c, st)
                         : c.rows == 2 ? sparse_rows<D, 2, false>(a, c, st)
                         : c.rows == 4 ? sparse_rows<D, 1, true>(a, c, st)
                                       : sparse_rows<D, 2, true>(a, c, st);
    if (s || c.splits == 1) return s;
    hipLaunchKernelGGL(k_sparse_join<D>, dim3(c.rows * (D / 16), c.blocks, a.nkv), dim3(256), 0, st, a.o_part, a.ml_part, a.out, sparse_heads(a),
                       sparse_parts(c), c.rows, a.inv_rep);
    return check_launch();
}

ghd_status launch_sparse_attention(SparseArgs a, int d, void* ws, size_t ws_bytes, hipStream_t st)
{
    const SparseCut c = sparse_cut(a.M, a.kv_len, a.nh, a.nkv, d);
    if (ws_bytes < sparse_bytes(sparse_units(c, a.nkv), d)) return GHD_ERR_WORKSPACE;
    a.rep = a.nh / a.nkv;
    a.inv_rep = 1.f / (float)a.rep;
    a.n = a.kv_len / kBlock;
    a.o_part = (float*)ws;
    a.ml_part = (float*)((char*)ws + sparse_o_bytes(sparse_units(c, a.nkv), d));
    return d == 128 ? sparse_of<128>(a, c, st) : sparse_of<64>(a, c, st);
}

}  // namespace ghd
