// Bounds of blocks of keys, and which blocks each drafted token reads (sparse.h has the layout, include/ghd.h the rules).
#include "sparse.h"
#include "wave.h"

namespace ghd {

typedef int32_t int4_ __attribute__((ext_vector_type(4)));
typedef uint32_t uint4_ __attribute__((ext_vector_type(4)));

// 2^(floor(log2 a) - 6) of a positive fp16 number, and one over it
__device__ __forceinline__ float unit_below(half_t a) { return __uint_as_float((__float_as_uint((float)a) & 0x7f800000u) - (6u << 23)); }
__device__ __forceinline__ float one_over_power(float p) { return __uint_as_float((254u << 23) - __float_as_uint(p)); }
__device__ __forceinline__ int code_of(float x) { return (int)fminf(fmaxf(x, -127.f), 127.f); }

// ---- bounds ------------------------------------------------------------------------------
// A wavefront has a block: 16-byte loads, so many rows at a time as fit, all requested at once.  Bound: the bytes of
// K: 256 blocks of 32 heads of 128 channels, 134 MB, 28.9 us (4.6 TB/s).  A single block of 8 heads: 3.6 us, a launch's time.
template <int D>
__global__ __launch_bounds__(256) void k_block_bounds(Bounds to, const half_t* __restrict__ k, int first, int n, int nkv, int64_t k_head,
                                                      int64_t k_tok)
{
    constexpr int kLanes = D / 8, kRows = 64 / kLanes, kLoads = kBlock / kRows;    // lanes of a row, rows of a load
    const int lane = threadIdx.x & 63, item = blockIdx.x * 4 + (threadIdx.x >> 6);
    if (item >= n * nkv) return;
    const int head = item / n, block = first + item - head * n;
    const half_t* p = k + head * k_head + ((int64_t)block * kBlock + lane / kLanes) * k_tok + lane % kLanes * 8;
    half8 x[kLoads];
#pragma unroll
    for (int i = 0; i < kLoads; ++i) x[i] = *(const half8*)(p + (int64_t)i * kRows * k_tok);
    half8 hi = x[0], lo = x[0];
    uint32_t odd = 0;
#pragma unroll
    for (int i = 0; i < kLoads; ++i) {
        hi = __builtin_elementwise_max(hi, x[i]);
        lo = __builtin_elementwise_min(lo, x[i]);
        const uint4_ w = __builtin_bit_cast(uint4_, x[i]);
        // (an exponent of all ones, plus one, carries into the sign)
#pragma unroll
        for (int e = 0; e < 4; ++e) odd |= (w[e] & 0x7c007c00u) + 0x04000400u;
    }
    // lanes of the same channels meet, then all lanes, for the largest number of the block
#pragma unroll
    for (int off = kLanes; off < 64; off *= 2) {
        uint4_ h = __builtin_bit_cast(uint4_, hi), l = __builtin_bit_cast(uint4_, lo);
#pragma unroll
        for (int e = 0; e < 4; ++e) {
            h[e] = (uint32_t)__shfl_xor((int)h[e], off);
            l[e] = (uint32_t)__shfl_xor((int)l[e], off);
        }
        hi = __builtin_elementwise_max(hi, __builtin_bit_cast(half8, h));
        lo = __builtin_elementwise_min(lo, __builtin_bit_cast(half8, l));
    }
    float a = 0.f;
#pragma unroll
    for (int e = 0; e < 8; ++e) a = fmaxf(a, fmaxf(fabsf((float)hi[e]), fabsf((float)lo[e])));
#pragma unroll
    for (int off = 1; off < kLanes; off *= 2) a = fmaxf(a, __shfl_xor(a, off));
    const bool finite = __ballot((odd & 0x80008000u) != 0) == 0;
    const float unit = !finite ? INFINITY : a > 0.f ? unit_below((half_t)a) : 0.f;
    const float inv = finite && a > 0.f ? one_over_power(unit) : 0.f;
    const size_t at = (size_t)head * to.blocks + block;
    if (lane == 0) to.units[at] = unit;
    if (lane >= 2 * kLanes) return;
    const bool low = lane >= kLanes;
    uint32_t code[2] = {0, 0};
#pragma unroll
    for (int e = 0; e < 8; ++e) {
        // (of a block that is not finite a code may be anything: inv * NaN is no number, and is replaced)
        const float v = (low ? (float)lo[e] : (float)hi[e]) * inv;
        const int c = finite ? code_of(low ? floorf(v) : ceilf(v)) : 0;
        code[e / 4] |= (uint32_t)(c & 255) << 8 * (e % 4);
    }
    *(uint2*)(to.codes + at * 2 * D + lane * 8) = make_uint2(code[0], code[1]);
}

// What the codes stand for; of a block that is not finite plus and minus infinity.
__global__ __launch_bounds__(256) void k_block_bounds_read(float* __restrict__ hi, float* __restrict__ lo, Bounds from, int first, int n, int nkv,
                                                           int d)
{
    const int64_t i = (int64_t)blockIdx.x * 256 + threadIdx.x;             // four channels of a block's bounds
    const int per = d / 4;
    if (i >= (int64_t)nkv * n * per) return;
    const int64_t row = i / per;
    const int c = (int)(i - row * per) * 4, head = (int)(row / n);
    const size_t at = (size_t)head * from.blocks + first + (row - (int64_t)head * n);
    const float unit = from.units[at];
    const bool finite = unit < INFINITY;
    const char4 h = *(const char4*)(from.codes + at * 2 * d + c), l = *(const char4*)(from.codes + at * 2 * d + d + c);
    auto up = [&](int x) { return finite ? (float)x * unit : INFINITY; };
    auto down = [&](int x) { return finite ? (float)x * unit : -INFINITY; };
    ((floatx4*)hi)[i] = (floatx4){up(h.x), up(h.y), up(h.z), up(h.w)};
    ((floatx4*)lo)[i] = (floatx4){down(l.x), down(l.y), down(l.z), down(l.w)};
}

// ---- scores ------------------------------------------------------------------------------
// The order of the scores as the order of unsigned numbers (-0 as 0); 0 is no score.
__device__ __forceinline__ uint32_t score_key(float t)
{
    const uint32_t b = __float_as_uint(t + 0.0f);
    return b ^ ((uint32_t)((int32_t)b >> 31) | 0x80000000u);
}

__device__ __forceinline__ uint32_t max_over_four(uint32_t x)
{
    // (rows of 16 lanes, then halves, exchanged with themselves: each lane has one of both in either register)
    const auto a = __builtin_amdgcn_permlane16_swap(x, x, false, false);
    x = max((uint32_t)a[0], (uint32_t)a[1]);
    const auto b = __builtin_amdgcn_permlane32_swap(x, x, false, false);
    return max((uint32_t)b[0], (uint32_t)b[1]);
}

// 16 channels' codes, those above zero (which meet HI) and those below (which meet LO), by pairs in fp16: a number times the two
// factors of 1 / unit is exact (or so far below a half that it does not matter), and 1536 more is rounded to a whole number,
// ties to even, whose low byte is the code.
__device__ __forceinline__ void query_codes(const half8 (&x)[2], half2_ first, half2_ second, int4_& above, int4_& below)
{
    const half2_ zero = {0, 0}, most = {127, 127}, round = {1536, 1536};
#pragma unroll
    for (int w = 0; w < 4; ++w) {
        uint32_t up[2], down[2];
#pragma unroll
        for (int e = 0; e < 2; ++e) {
            const int at = w % 2 * 4 + 2 * e;
            const half2_ v = (half2_){x[w / 2][at], x[w / 2][at + 1]} * first * second;
            up[e] = __builtin_bit_cast(uint32_t, __builtin_elementwise_min(__builtin_elementwise_max(v, zero), most) + round);
            down[e] = __builtin_bit_cast(uint32_t, __builtin_elementwise_max(__builtin_elementwise_min(v, zero), -most) + round);
        }
        above[w] = (int32_t)__builtin_amdgcn_perm(up[1], up[0], 0x06040200u);
        below[w] = (int32_t)__builtin_amdgcn_perm(down[1], down[0], 0x06040200u);
    }
}

// What the first loads need, in the arguments that are in scalar registers when a kernel starts (see SAMPLE_FIRST).
#define SELECT_FIRST const half_t *q, char *codes, float *units, int blocks, int M, int nkv, int rep, int n
__device__ __forceinline__ void select_first(SelectArgs& a, SELECT_FIRST)
{
    a.q = q;
    a.bounds = {codes, units, blocks};
    a.M = M;
    a.nkv = nkv;
    a.rep = rep;
    a.n = n;
}

// Blocks are the rows of the product, 16 tokens of one query head its columns.  A wavefront keeps the codes of TILES tiles of 16 blocks in
// registers (tiles `step` blocks apart) and goes through the query heads.  to(b, keys): blocks b .. b + 3 of the lane's token.
template <int D, int TILES, class Store>
__device__ __forceinline__ void block_scores(const SelectArgs& a, int head, int m, int b0, int step, int lane, const Store& to)
{
    constexpr int KS = 2 * D / 64;               // k-steps: the first half of them HI, the second LO
    const int g = lane >> 4, col = lane & 15;
    half8 x[KS / 2][2];
    const half_t* q = a.q + ((size_t)min(m, a.M - 1) * a.nkv + head) * a.rep * D + g * 16;
    auto ask_for = [&]() {
#pragma unroll
        for (int s = 0; s < KS / 2; ++s)
#pragma unroll
            for (int e = 0; e < 2; ++e) x[s][e] = *(const half8*)(q + s * 64 + e * 8);
    };
    ask_for();
    const size_t row0 = (size_t)head * a.bounds.blocks;
    int4_ code[TILES][KS];
#pragma unroll
    for (int t = 0; t < TILES; ++t)
#pragma unroll
        for (int s = 0; s < KS; ++s)
            code[t][s] = *(const int4_*)(a.bounds.codes + (row0 + min(b0 + t * step + col, a.n - 1)) * 2 * D + s * 64 + g * 16);
    floatx4 unit[TILES], best[TILES];
#pragma unroll
    for (int t = 0; t < TILES; ++t) {
        best[t] = (floatx4){-INFINITY, -INFINITY, -INFINITY, -INFINITY};
#pragma unroll
        for (int r = 0; r < 4; ++r) unit[t][r] = a.bounds.units[row0 + min(b0 + t * step + 4 * g + r, a.n - 1)];
    }
    for (int h = 0; h < a.rep; ++h) {
        typedef uint16_t ushort2_ __attribute__((ext_vector_type(2)));
        ushort2_ size = {0, 0};
#pragma unroll
        for (int s = 0; s < KS / 2; ++s)
#pragma unroll
            for (int e = 0; e < 2; ++e) {
                const uint4_ w = __builtin_bit_cast(uint4_, x[s][e]) & 0x7fff7fffu;
#pragma unroll
                for (int i = 0; i < 4; ++i) size = __builtin_elementwise_max(size, __builtin_bit_cast(ushort2_, (uint32_t)w[i]));
            }
        const uint32_t top = max_over_four(max((uint32_t)size[0], (uint32_t)size[1]));
        // (a head that holds an infinity or NaN, or only zeros, scores 0 everywhere)
        const bool some = top > 0 && top < 0x7c00u;
        const float step = some ? unit_below(__builtin_bit_cast(half_t, (uint16_t)top)) : 0.f;
        // 1 / step is 2^-9 to 2^30: two factors, each an fp16 number
        const int up = some ? 127 - (int)(__float_as_uint(step) >> 23) : 0, half = up >> 1;
        const half_t f1 = __builtin_bit_cast(half_t, (uint16_t)((half + 15) << 10)), f2 = __builtin_bit_cast(half_t, (uint16_t)((up - half + 15) << 10));
        int4_ ask[KS];
#pragma unroll
        for (int s = 0; s < KS / 2; ++s) {
            query_codes(x[s], (half2_){f1, f1}, (half2_){f2, f2}, ask[s], ask[KS / 2 + s]);
            if (!some) ask[s] = ask[KS / 2 + s] = (int4_){0, 0, 0, 0};
        }
        if (h + 1 < a.rep) {
            q += D;
            ask_for();
        }
#pragma unroll
        for (int t = 0; t < TILES; ++t) {
            int4_ sum = {0, 0, 0, 0};
#pragma unroll
            for (int s = 0; s < KS; ++s) sum = __builtin_amdgcn_mfma_i32_16x16x64_i8(code[t][s], ask[s], sum, 0, 0, 0);
#pragma unroll
            for (int r = 0; r < 4; ++r) best[t][r] = fmaxf(best[t][r], (float)sum[r] * step);
        }
    }
#pragma unroll
    for (int t = 0; t < TILES; ++t) {
        uint4_ key;
#pragma unroll
        for (int r = 0; r < 4; ++r) key[r] = score_key(unit[t][r] < INFINITY ? best[t][r] * unit[t][r] : INFINITY);
        to(b0 + t * step + 4 * g, key);
    }
}

// Bound: reading codes where tokens are few (8 heads of 2047 blocks, 4.3 MB: 6.1 us, half of it before the first of them is there), else the
// quantising of queries, which every wavefront does for itself.
template <int D, int TILES>
__global__ __launch_bounds__(256) void k_block_scores(SELECT_FIRST, SelectArgs a)
{
    select_first(a, q, codes, units, blocks, M, nkv, rep, n);
    const int lane = threadIdx.x & 63, wave = threadIdx.x >> 6, b0 = (blockIdx.x * 4 + wave) * TILES * 16, head = blockIdx.y, m = blockIdx.z * 16 + (lane & 15);
    if (b0 >= a.n) return;
    if (a.zero && blockIdx.z == 0 && lane < TILES * 16 && b0 + lane < a.n)       // the picks set bits
        for (int w = 0; w < (a.M + 63) / 64; ++w) a.sel[((size_t)head * ((a.M + 63) / 64) + w) * a.n + b0 + lane] = 0;
    const int n4 = (a.n + 3) & ~3;
    uint32_t* keys = a.keys + ((size_t)head * a.M + m) * n4;
    block_scores<D, TILES>(a, head, m, b0, 16, lane, [&](int b, uint4_ key) {
        if (m < a.M && b < n4) *(uint4_*)(keys + b) = key;
    });
}

// ---- picks -------------------------------------------------------------------------------
// A team of wavefronts has a token and a key head: one wavefront, of eight in a workgroup, or all of a workgroup's.  The range of the keys is
// cut in 256 steps and the step counted out in which the `keep` best end (scores lie close together: by their leading bits nearly
// all would fall in a few); what is above is taken, and what is in it ranked, or, if it is much, cut again.  Of more
// equal keys than are ranked the first are taken in order.
template <int TEAM>
struct PickShared {
    static constexpr int kWaves = TEAM / 64, kRanked = TEAM < 256 ? TEAM : 256;
    uint32_t hist[256], low[kWaves], high[kWaves], step, need, in, n, key[kRanked];
    int at[kRanked];
};
template <int TEAM>
__device__ __forceinline__ void team_sync()
{
    if constexpr (TEAM == 64) {
        __builtin_amdgcn_fence(__ATOMIC_ACQ_REL, "wavefront");
        __builtin_amdgcn_wave_barrier();
    } else {
        __syncthreads();
    }
}

// KEPT: keys that a thread keeps in registers, all of them; 0: they are read again each time.  take(b): block b is taken.
template <int TEAM, int KEPT, class Take>
__device__ __forceinline__ void pick_blocks(const SelectArgs& a, PickShared<TEAM>& s, const uint32_t* keys, int tid, const Take& take)
{
    typedef PickShared<TEAM> S;
    const int lane = tid & 63, wave = tid >> 6;
    uint32_t kept[KEPT ? KEPT : 1];
    if constexpr (KEPT > 0) {
#pragma unroll
        for (int i = 0; i < KEPT; ++i) kept[i] = a.lo + i * TEAM + tid < a.hi ? keys[a.lo + i * TEAM + tid] : 0;
    }
    // (0 is no score)
    auto each = [&](auto f) {
        if constexpr (KEPT > 0) {
#pragma unroll
            for (int i = 0; i < KEPT; ++i)
                if (kept[i] != 0) f(kept[i], a.lo + i * TEAM + tid);
        } else {
            for (int b = a.lo + tid; b < a.hi; b += TEAM) f(keys[b], b);
        }
    };
    for (int b = tid; b < a.lo + (a.n - a.hi); b += TEAM) take(b < a.lo ? b : a.hi + b - a.lo);
    if (a.keep <= 0) return;
    uint32_t low = ~0u, high = 0;
    each([&](uint32_t key, int) {
        low = min(low, key);
        high = max(high, key);
    });
    low = ~wave_highest(~low);
    high = wave_highest(high);
    for (int i = tid; i < 256; i += TEAM) s.hist[i] = 0;
    if (tid == 0) s.n = 0;
    if constexpr (TEAM > 64) {
        if (lane == 0) {
            s.low[wave] = low;
            s.high[wave] = high;
        }
    }
    team_sync<TEAM>();
    if constexpr (TEAM > 64) {
#pragma unroll
        for (int w = 0; w < S::kWaves; ++w) {
            low = min(low, s.low[w]);
            high = max(high, s.high[w]);
        }
    }
    uint32_t need = a.keep, in;                  // of the keys from low to high, of which there are `in`
    int shift = pick_shift(low, high);
    for (;;) {
        each([&](uint32_t key, int) {
            if (key >= low && key <= high) atomicAdd(&s.hist[(key - low) >> shift], 1u);
        });
        team_sync<TEAM>();
        if (tid < 64) {                          // steps from the highest on: lane l has 255 - 4 l .. 252 - 4 l
            uint32_t c[4], sum = 0;
#pragma unroll
            for (int e = 0; e < 4; ++e) sum += c[e] = s.hist[255 - 4 * tid - e];
            uint32_t before = running_sum(sum);
            before -= sum;
#pragma unroll
            for (int e = 0; e < 4; ++e) {
                if (before < need && before + c[e] >= need) {
                    s.step = 255 - 4 * tid - e;
                    s.need = need - before;
                    s.in = c[e];
                }
                before += c[e];
            }
        }
        team_sync<TEAM>();
        const uint32_t from = low + (s.step << shift), to = pick_step_end(from, high, shift);
        each([&](uint32_t key, int b) {
            if (key > to && key <= high) take(b);
        });
        low = from;
        high = to;
        need = s.need;
        in = s.in;
        if (in == need || in <= S::kRanked || shift == 0) break;
        shift = max(0, shift - 8);
        for (int i = tid; i < 256; i += TEAM) s.hist[i] = 0;   // (read last before it was synchronised)
        team_sync<TEAM>();
    }
    if (in == need) {
        each([&](uint32_t key, int b) {
            if (key >= low && key <= high) take(b);
        });
        return;
    }
    if (in <= S::kRanked) {
        // (as many as were counted, unless another call writes to this workspace meanwhile: then nothing is taken that is no block)
        each([&](uint32_t key, int b) {
            if (key < low || key > high) return;
            const uint32_t to = atomicAdd(&s.n, 1u);
            if (to >= S::kRanked) return;
            s.key[to] = key;
            s.at[to] = b;
        });
        team_sync<TEAM>();
        in = min(in, s.n);
        if (tid >= (int)in) return;
        const uint32_t key = s.key[tid];
        const int at = s.at[tid];
        uint32_t rank = 0;
        for (uint32_t j = 0; j < in; ++j) rank += s.key[j] > key || (s.key[j] == key && s.at[j] < at);
        if (rank < need) take(at);
        return;
    }
    // equal keys, more than are needed: the first, in order
    for (int b0 = a.lo; b0 < a.hi && need > 0; b0 += TEAM) {
        const int b = b0 + tid;
        const bool is = b < a.hi && keys[b] == low;
        const uint64_t with = __ballot(is);
        uint32_t before = __popcll(with & ((1ull << lane) - 1)), all = __popcll(with);
        if constexpr (TEAM > 64) {
            if (lane == 0) s.low[wave] = all;
            __syncthreads();
            all = 0;
            for (int w = 0; w < S::kWaves; ++w) {
                if (w < wave) before += s.low[w];
                all += s.low[w];
            }
            __syncthreads();
        }
        if (is && before < need) take(b);
        need -= min(need, all);
    }
}

// Eight tokens' bits, a byte of the blocks' words: from LDS to their place; the last tokens' workgroup writes what is left of the words, too.
__device__ __forceinline__ void store_eight(const SelectArgs& a, int head, int m0, const uint32_t* s_bits, int tid)
{
    uint64_t* words = a.sel + ((size_t)head * ((a.M + 63) / 64) + m0 / 64) * a.n;
    uint8_t* to = (uint8_t*)words + m0 % 64 / 8;
    const int left = m0 + 8 >= a.M ? 8 - m0 % 64 / 8 : 1;          // bytes of a word that are this workgroup's
    for (int b = tid; b < a.n; b += 512) {
        const uint8_t x = (uint8_t)(s_bits[b >> 2] >> 8 * (b & 3));
        if (left == 8) {
            words[b] = x;
        } else {
            to[(size_t)8 * b] = x;
            for (int i = 1; i < left; ++i) to[(size_t)8 * b + i] = 0;
        }
    }
}

// Scores and picks of few blocks in one launch: a workgroup has eight tokens of a head, whose scores stay in LDS.  Bound: what follows one
// another - codes' way from the L2, the product, three or four rounds of a pick.  64 tokens of 32 heads over 512 blocks: 12.9 us (14.1 with
// arguments from memory and maxima by shuffles, 16.4 with heads spread over the XCDs).
constexpr int kFewBlocks = 512;
template <int D>
__global__ __launch_bounds__(512) void k_block_few(SELECT_FIRST, SelectArgs a)
{
    select_first(a, q, codes, units, blocks, M, nkv, rep, n);
    __shared__ PickShared<64> s[8];
    __shared__ __attribute__((aligned(16))) uint32_t s_key[8][kFewBlocks + 4];
    __shared__ uint32_t s_bits[kFewBlocks / 4];
    const int tid = threadIdx.x, lane = tid & 63, wave = __builtin_amdgcn_readfirstlane(tid >> 6), head = blockIdx.x, m0 = blockIdx.y * 8, m = m0 + wave;
    if (tid < kFewBlocks / 4) s_bits[tid] = 0;
    auto keep = [&](int b, uint4_ key) {
        if ((lane & 15) < 8) *(uint4_*)(s_key[lane & 7] + b) = key;
    };
    // (all of a wavefront's tiles are asked for at once: by two, that took 0.2 us more)
    if (a.n > 128) block_scores<D, kFewBlocks / 128>(a, head, m0 + (lane & 7), wave * 16, 128, lane, keep);
    else if (wave * 16 < a.n) block_scores<D, 1>(a, head, m0 + (lane & 7), wave * 16, 128, lane, keep);
    __syncthreads();
    if (m < a.M) pick_blocks<64, kFewBlocks / 64>(a, s[wave], s_key[wave], lane, [&](int b) { atomicOr(&s_bits[b >> 2], 1u << (8 * (b & 3) + wave)); });
    __syncthreads();
    store_eight(a, head, m0, s_bits, tid);
}

// A workgroup has eight tokens, a wavefront each; their bits meet in LDS and leave as bytes of the words.
constexpr int kPickBytes = 2048;                 // blocks
template <int KEPT>
__global__ __launch_bounds__(512) void k_block_pick_eight(SelectArgs a)
{
    __shared__ PickShared<64> s[8];
    __shared__ uint32_t s_bits[kPickBytes / 4];
    const int tid = threadIdx.x, wave = __builtin_amdgcn_readfirstlane(tid >> 6), m0 = blockIdx.x * 8, m = m0 + wave, head = blockIdx.y;
    for (int i = tid; i < (a.n + 3) / 4; i += 512) s_bits[i] = 0;
    __syncthreads();
    if (m < a.M)
        pick_blocks<64, KEPT>(a, s[wave], a.keys + ((size_t)head * a.M + m) * ((a.n + 3) & ~3), tid & 63,
                              [&](int b) { atomicOr(&s_bits[b >> 2], 1u << (8 * (b & 3) + wave)); });
    __syncthreads();
    store_eight(a, head, m0, s_bits, tid);
}

// A workgroup has a token; the words are zeros before (k_block_scores).  Bound: what follows one another.  8 heads' picks among 2047 blocks: 5.2 us.
template <int KEPT>
__global__ __launch_bounds__(1024) void k_block_pick(SelectArgs a)
{
    __shared__ PickShared<1024> s;
    const int m = blockIdx.x, head = blockIdx.y;
    uint64_t* sel = a.sel + ((size_t)head * ((a.M + 63) / 64) + m / 64) * a.n;
    const uint64_t bit = 1ull << (m % 64);
    pick_blocks<1024, KEPT>(a, s, a.keys + ((size_t)head * a.M + m) * ((a.n + 3) & ~3), threadIdx.x,
                            [&](int b) { atomicOr((unsigned long long*)(sel + b), (unsigned long long)bit); });
}

ghd_status launch_block_bounds(Bounds to, const half_t* k, int first, int n, int nkv, int d, int64_t k_head, int64_t k_tok, hipStream_t st)
{
    if (n == 0) return GHD_OK;
    const dim3 grid(ceil_div(n * nkv, 4));
    if (d == 128) hipLaunchKernelGGL(k_block_bounds<128>, grid, dim3(256), 0, st, to, k, first, n, nkv, k_head, k_tok);
    else hipLaunchKernelGGL(k_block_bounds<64>, grid, dim3(256), 0, st, to, k, first, n, nkv, k_head, k_tok);
    return check_launch();
}

ghd_status launch_block_bounds_read(float* hi, float* lo, Bounds from, int first, int n, int nkv, int d, hipStream_t st)
{
    if (n == 0) return GHD_OK;
    // (at most 256 heads of 2^15 blocks of 32 pieces: 2^20 workgroups)
    const int64_t pieces = (int64_t)nkv * n * (d / 4);
    hipLaunchKernelGGL(k_block_bounds_read, dim3((uint32_t)((pieces + 255) / 256)), dim3(256), 0, st, hi, lo, from, first, n, nkv, d);
    return check_launch();
}

ghd_status launch_block_select(SelectArgs a, int d, hipStream_t st)
{
    if (a.n == 0) return GHD_OK;
    // One launch takes up to 128 blocks, or 512 where there are so many picks that they fill the GPU anyhow, if it is one round of workgroups.
    // In a graph, us, against two launches: 1 token, 8 heads of 4, 128 blocks 9.2 | 9.2, 512 blocks 13.4 | 9.2; 64 tokens, 32 heads, 128 blocks
    // 7.8 | 10.2, 512 blocks 11.6 | 14.5; 128 tokens, 32 heads of 4, 512 blocks 28.4 | 24.  Without a graph a launch costs the host 3 us.
    const bool many = a.M * a.nkv >= 1024;
    if (a.n <= kFewBlocks && a.nkv * ceil_div(a.M, 8) <= 256 && (a.n <= 128 || many)) {
        const dim3 teams(a.nkv, ceil_div(a.M, 8));                  // (a head's tokens on one XCD, where its codes are)
        if (d == 128) hipLaunchKernelGGL(k_block_few<128>, teams, dim3(512), 0, st, a.q, a.bounds.codes, a.bounds.units, a.bounds.blocks, a.M, a.nkv, a.rep, a.n, a);
        else hipLaunchKernelGGL(k_block_few<64>, teams, dim3(512), 0, st, a.q, a.bounds.codes, a.bounds.units, a.bounds.blocks, a.M, a.nkv, a.rep, a.n, a);
        return check_launch();
    }
    // A wavefront has 64 blocks, or 16 where there would be fewer than four wavefronts for each compute unit: 1 token, 8 heads of 4, 1000
    // blocks 9.2 us, with 64 11.7; 128 tokens 17.0, with 16 21.6.
    const int tiles = ceil_div(a.M, 16), per = (int64_t)ceil_div(a.n, 64) * a.nkv * tiles >= 1024 ? 4 : 1;
    const dim3 grid(ceil_div(a.n, 64 * per), a.nkv, tiles);
    // eight tokens' picks in a workgroup, or one's: 64 tokens, 32 heads, 1000 blocks 20.1 us | 27.7; 64 tokens, 8 heads of 4, 2000 blocks
    // 21.3 | 16.1, 8 tokens 16.6 | 9.8
    const bool eight = a.n <= kPickBytes && many;
    a.zero = !eight;
    if (d == 128) {
        if (per == 4) hipLaunchKernelGGL((k_block_scores<128, 4>), grid, dim3(256), 0, st, a.q, a.bounds.codes, a.bounds.units, a.bounds.blocks, a.M, a.nkv, a.rep, a.n, a);
        else hipLaunchKernelGGL((k_block_scores<128, 1>), grid, dim3(256), 0, st, a.q, a.bounds.codes, a.bounds.units, a.bounds.blocks, a.M, a.nkv, a.rep, a.n, a);
    } else {
        if (per == 4) hipLaunchKernelGGL((k_block_scores<64, 4>), grid, dim3(256), 0, st, a.q, a.bounds.codes, a.bounds.units, a.bounds.blocks, a.M, a.nkv, a.rep, a.n, a);
        else hipLaunchKernelGGL((k_block_scores<64, 1>), grid, dim3(256), 0, st, a.q, a.bounds.codes, a.bounds.units, a.bounds.blocks, a.M, a.nkv, a.rep, a.n, a);
    }
    const ghd_status s = check_launch();
    if (s) return s;
    const int range = a.hi - a.lo;
    if (eight) {
        const dim3 teams(ceil_div(a.M, 8), a.nkv);
        if (range <= 64 * 16) hipLaunchKernelGGL(k_block_pick_eight<16>, teams, dim3(512), 0, st, a);
        else hipLaunchKernelGGL(k_block_pick_eight<32>, teams, dim3(512), 0, st, a);
    } else if (range <= 1024 * 4) {
        hipLaunchKernelGGL(k_block_pick<4>, dim3(a.M, a.nkv), dim3(1024), 0, st, a);
    } else {
        hipLaunchKernelGGL(k_block_pick<0>, dim3(a.M, a.nkv), dim3(1024), 0, st, a);
    }
    return check_launch();
}

}  // namespace ghd
