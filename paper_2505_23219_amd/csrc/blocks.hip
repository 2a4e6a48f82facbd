// Bounds of blocks of keys, and which blocks each drafted token reads (sparse.h has the layout, include/ghd.h the rules).
#include "sparse.h"

namespace ghd {

typedef int32_t int4_ __attribute__((ext_vector_type(4)));
typedef uint32_t uint4_ __attribute__((ext_vector_type(4)));

// 2^(floor(log2 a) - 6) of a positive fp16 number, and one over it
__device__ __forceinline__ float unit_below(half_t a) { return __uint_as_float((__float_as_uint((float)a) & 0x7f800000u) - (6u << 23)); }
__device__ __forceinline__ float one_over_power(float p) { return __uint_as_float((254u << 23) - __float_as_uint(p)); }
__device__ __forceinline__ int code_of(float x) { return (int)fminf(fmaxf(x, -127.f), 127.f); }

// ---- bounds ------------------------------------------------------------------------------
// A wavefront has a block: 16-byte loads, so many rows at a time as fit, all requested at once.  Bound: the bytes of K.
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
    x = max(x, (uint32_t)__shfl_xor((int)x, 16));
    return max(x, (uint32_t)__shfl_xor((int)x, 32));
}

// 16 channels' codes: those above zero (which meet HI) and those below (which meet LO)
__device__ __forceinline__ void query_codes(const half8 (&x)[2], float inv, int4_& above, int4_& below)
{
#pragma unroll
    for (int w = 0; w < 4; ++w) {
        uint32_t p = 0, n = 0;
#pragma unroll
        for (int e = 0; e < 4; ++e) {
            const int c = code_of(rintf((float)x[w / 2][w % 2 * 4 + e] * inv));
            p |= (uint32_t)max(c, 0) << 8 * e;
            n |= (uint32_t)(min(c, 0) & 255) << 8 * e;
        }
        above[w] = (int32_t)p;
        below[w] = (int32_t)n;
    }
}

constexpr int kScoreTiles = 4;                   // of 16 blocks: a wavefront's

// Blocks are the rows of the product, 16 tokens of one query head its columns.  A wavefront keeps the codes of 64 blocks in registers
// and goes through the query heads.  Bound: over long contexts the bytes of the codes.
template <int D>
__global__ __launch_bounds__(256) void k_block_scores(SelectArgs a)
{
    constexpr int KS = 2 * D / 64;               // k-steps: the first half of them HI, the second LO
    const int lane = threadIdx.x & 63, wave = threadIdx.x >> 6, g = lane >> 4, col = lane & 15;
    const int b0 = (blockIdx.x * 4 + wave) * kScoreTiles * 16, head = blockIdx.y, m = blockIdx.z * 16 + col;
    if (b0 >= a.n) return;
    const size_t row0 = (size_t)head * a.bounds.blocks;
    int4_ code[kScoreTiles][KS];
#pragma unroll
    for (int t = 0; t < kScoreTiles; ++t)
#pragma unroll
        for (int s = 0; s < KS; ++s)
            code[t][s] = *(const int4_*)(a.bounds.codes + (row0 + min(b0 + t * 16 + col, a.n - 1)) * 2 * D + s * 64 + g * 16);
    floatx4 unit[kScoreTiles], best[kScoreTiles];
#pragma unroll
    for (int t = 0; t < kScoreTiles; ++t) {
        best[t] = (floatx4){-INFINITY, -INFINITY, -INFINITY, -INFINITY};
#pragma unroll
        for (int r = 0; r < 4; ++r) unit[t][r] = a.bounds.units[row0 + min(b0 + t * 16 + 4 * g + r, a.n - 1)];
    }
    if (blockIdx.z == 0 && b0 + lane < a.n)      // the picks set bits
        for (int w = 0; w < (a.M + 63) / 64; ++w) a.sel[((size_t)head * ((a.M + 63) / 64) + w) * a.n + b0 + lane] = 0;
    const half_t* q = a.q + ((size_t)min(m, a.M - 1) * a.nkv + head) * a.rep * D + g * 16;
    for (int h = 0; h < a.rep; ++h, q += D) {
        half8 x[KS / 2][2];
        uint32_t top = 0;
#pragma unroll
        for (int s = 0; s < KS / 2; ++s)
#pragma unroll
            for (int e = 0; e < 2; ++e) {
                x[s][e] = *(const half8*)(q + s * 64 + e * 8);
                const uint4_ w = __builtin_bit_cast(uint4_, x[s][e]) & 0x7fff7fffu;
#pragma unroll
                for (int i = 0; i < 4; ++i) top = max(top, max(w[i] & 0xffffu, w[i] >> 16));
            }
        top = max_over_four(top);
        // (a head that holds an infinity or NaN, or only zeros, scores 0 everywhere)
        const bool some = top > 0 && top < 0x7c00u;
        const float step = some ? unit_below(__builtin_bit_cast(half_t, (uint16_t)top)) : 0.f, inv = some ? one_over_power(step) : 0.f;
        int4_ ask[KS];
#pragma unroll
        for (int s = 0; s < KS / 2; ++s) {
            query_codes(x[s], inv, ask[s], ask[KS / 2 + s]);
            if (!some) ask[s] = ask[KS / 2 + s] = (int4_){0, 0, 0, 0};
        }
#pragma unroll
        for (int t = 0; t < kScoreTiles; ++t) {
            int4_ sum = {0, 0, 0, 0};
#pragma unroll
            for (int s = 0; s < KS; ++s) sum = __builtin_amdgcn_mfma_i32_16x16x64_i8(code[t][s], ask[s], sum, 0, 0, 0);
#pragma unroll
            for (int r = 0; r < 4; ++r) best[t][r] = fmaxf(best[t][r], (float)sum[r] * step);
        }
    }
    if (m >= a.M) return;
    const int n4 = (a.n + 3) & ~3;
    uint32_t* to = a.keys + ((size_t)head * a.M + m) * n4;
#pragma unroll
    for (int t = 0; t < kScoreTiles; ++t) {
        const int b = b0 + t * 16 + 4 * g;
        if (b >= n4) continue;
        uint4_ key;
#pragma unroll
        for (int r = 0; r < 4; ++r) key[r] = score_key(unit[t][r] < INFINITY ? best[t][r] * unit[t][r] : INFINITY);
        *(uint4_*)(to + b) = key;
    }
}

// ---- picks -------------------------------------------------------------------------------
// A workgroup has a token and a key head: the lowest key of the `keep` best is found 8 bits at a time, then what is above it is
// taken and of those equal to it the first.
__global__ __launch_bounds__(256) void k_block_pick(SelectArgs a)
{
    __shared__ uint32_t s_hist[256], s_bin, s_need, s_same;
    const int tid = threadIdx.x, m = blockIdx.x, head = blockIdx.y;
    const uint32_t* keys = a.keys + ((size_t)head * a.M + m) * ((a.n + 3) & ~3);
    uint64_t* sel = a.sel + ((size_t)head * ((a.M + 63) / 64) + m / 64) * a.n;
    const uint64_t bit = 1ull << (m % 64);
    auto take = [&](int b) { atomicOr((unsigned long long*)(sel + b), (unsigned long long)bit); };
    for (int b = tid; b < a.lo + (a.n - a.hi); b += 256) take(b < a.lo ? b : a.hi + b - a.lo);
    if (a.keep <= 0) return;
    uint32_t prefix = 0, known = 0, need = a.keep;
    for (int shift = 24; shift >= 0; shift -= 8) {
        s_hist[tid] = 0;
        __syncthreads();
        for (int b = a.lo + tid; b < a.hi; b += 256) {
            const uint32_t key = keys[b];
            if ((key & known) == prefix) atomicAdd(&s_hist[key >> shift & 255], 1u);
        }
        __syncthreads();
        if (tid < 64) {                          // bins from the highest on: lane l has 255 - 4 l .. 252 - 4 l
            uint32_t c[4], sum = 0;
#pragma unroll
            for (int e = 0; e < 4; ++e) sum += c[e] = s_hist[255 - 4 * tid - e];
            uint32_t before = sum;
            for (int off = 1; off < 64; off *= 2) {
                const uint32_t o = (uint32_t)__shfl_up((int)before, off);
                if (tid >= off) before += o;
            }
            before -= sum;
#pragma unroll
            for (int e = 0; e < 4; ++e) {
                if (before < need && before + c[e] >= need) {
                    s_bin = 255 - 4 * tid - e;
                    s_need = need - before;
                    s_same = c[e];
                }
                before += c[e];
            }
        }
        __syncthreads();
        prefix |= s_bin << shift;
        known |= 255u << shift;
        need = s_need;
    }
    const uint32_t same = s_same;
    for (int b = a.lo + tid; b < a.hi; b += 256) {
        const uint32_t key = keys[b];
        if (key > prefix || (same == need && key == prefix)) take(b);
    }
    if (same == need) return;
    // more of them than are needed: the first, in order
    uint32_t* s_count = s_hist;                  // (read last before a barrier)
    for (int b0 = a.lo; b0 < a.hi && need > 0; b0 += 256) {
        const int b = b0 + tid;
        const bool is = b < a.hi && keys[b] == prefix;
        const uint64_t with = __ballot(is);
        if ((tid & 63) == 0) s_count[tid >> 6] = __popcll(with);
        __syncthreads();
        uint32_t before = __popcll(with & ((1ull << (tid & 63)) - 1)), all = 0;
        for (int w = 0; w < 4; ++w) {
            if (w < tid >> 6) before += s_count[w];
            all += s_count[w];
        }
        if (is && before < need) take(b);
        need -= min(need, all);
        __syncthreads();
    }
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

ghd_status launch_block_select(const SelectArgs& a, int d, hipStream_t st)
{
    if (a.n == 0) return GHD_OK;
    const dim3 grid(ceil_div(a.n, 4 * kScoreTiles * 16), a.nkv, ceil_div(a.M, 16));
    if (d == 128) hipLaunchKernelGGL(k_block_scores<128>, grid, dim3(256), 0, st, a);
    else hipLaunchKernelGGL(k_block_scores<64>, grid, dim3(256), 0, st, a);
    const ghd_status s = check_launch();
    if (s) return s;
    hipLaunchKernelGGL(k_block_pick, dim3(a.M, a.nkv), dim3(256), 0, st, a);
    return check_launch();
}

}  // namespace ghd
