// Linear layer over 4-bit weights with group scales, 1 to 128 rows.
//
// y[m, n] = sum over groups of scale[n, group] * (sum over the group's k of x[m, k] (code[n, k] - zero[n, group])).  The inner
// sums are products of fp16 numbers with whole numbers below 256, exact, summed in 32 bits by the MFMA; the scale is applied to
// them in 32 bits, so nothing is rounded to fewer bits before the result.  x is the A operand and W the B operand: a lane's
// operand, its column of the result, and with them scale and zero point, all belong to one row of W.
#include "q4.h"

namespace ghd {

constexpr int kQ4LinWaves = 8;
typedef uint32_t word4 __attribute__((ext_vector_type(4)));

template <int MT, int R, int G>
__global__ __launch_bounds__(kQ4LinWaves * 64) void k_q4_linear(const Q4Linear a, int ntiles, int nunits)
{
    constexpr int kUnitBytes = 1024 + 64 * G, kSteps = 4 / G;      // k-steps that share a scale
    extern __shared__ __attribute__((aligned(16))) char lds[];
    const int lane = threadIdx.x & 63, wave = threadIdx.x >> 6, r = lane & 15, g = lane >> 4;
    const int tile0 = blockIdx.x * R;
    floatx4 acc[R][MT];
#pragma unroll
    for (int t = 0; t < R; ++t)
#pragma unroll
        for (int mt = 0; mt < MT; ++mt) acc[t][mt] = (floatx4){0.f, 0.f, 0.f, 0.f};
    for (int u = wave; u < nunits; u += kQ4LinWaves) {
        half8 x[4][MT];
#pragma unroll
        for (int mt = 0; mt < MT; ++mt) {
            const int m = mt * 16 + r;
#pragma unroll
            for (int s = 0; s < 4; ++s) {
                const int k = u * kQ4Unit + 32 * s + 8 * g;
                x[s][mt] = (half8){0, 0, 0, 0, 0, 0, 0, 0};
                if (m < a.M && k < a.K) x[s][mt] = *(const half8*)(a.x + (size_t)m * a.ldx + k);
            }
        }
#pragma unroll
        for (int t = 0; t < R; ++t) {
            const int tile = min(tile0 + t, ntiles - 1);
            const char* unit = a.W + ((size_t)tile * nunits + u) * kUnitBytes;
            const word4 w = *(const word4*)(unit + lane * 16);
            const half2_* meta = (const half2_*)(unit + 1024) + r * G;
#pragma unroll
            for (int q = 0; q < G; ++q) {
                const half2_ sz = meta[q];
                floatx4 sum[MT];
#pragma unroll
                for (int mt = 0; mt < MT; ++mt) sum[mt] = (floatx4){0.f, 0.f, 0.f, 0.f};
#pragma unroll
                for (int s = q * kSteps; s < (q + 1) * kSteps; ++s) {
                    const half8 b = q4_codes(w[s], pair_of(sz[1]));
#pragma unroll
                    for (int mt = 0; mt < MT; ++mt)
                        sum[mt] = __builtin_amdgcn_mfma_f32_16x16x32_f16(x[s][mt], b, sum[mt], 0, 0, 0);
                }
#pragma unroll
                for (int mt = 0; mt < MT; ++mt) acc[t][mt] += sum[mt] * (float)sz[0];
            }
        }
    }
    // The wavefronts' sums meet in LDS, eight fragments at a time, each added up by one wavefront in a fixed order.
    floatx4* part = (floatx4*)lds;                                 // [fragment][wave][64]
    constexpr int kFrags = R * MT;
#pragma unroll
    for (int f0 = 0; f0 < kFrags; f0 += kQ4LinWaves) {
        if (f0) __syncthreads();
#pragma unroll
        for (int f = f0; f < f0 + kQ4LinWaves && f < kFrags; ++f)
            part[((f - f0) * kQ4LinWaves + wave) * 64 + lane] = acc[f / MT][f % MT];
        __syncthreads();
        const int f = f0 + wave;
        if (f < kFrags) {
            floatx4 y = part[wave * kQ4LinWaves * 64 + lane];
#pragma unroll
            for (int w = 1; w < kQ4LinWaves; ++w) y += part[(wave * kQ4LinWaves + w) * 64 + lane];
            const int n = (tile0 + f / MT) * 16 + r, m0 = f % MT * 16 + 4 * g;
#pragma unroll
            for (int e = 0; e < 4; ++e) {
                if (n >= a.N || m0 + e >= a.M) continue;
                const int64_t at = (int64_t)(m0 + e) * a.ldy + n;
                if (a.out16) ((half_t*)a.y)[at] = (half_t)y[e];
                else ((float*)a.y)[at] = y[e];
            }
        }
    }
}

size_t q4_linear_bytes(int, int, int) { return 256; }

template <int MT, int R, int G>
static void q4_linear_of(const Q4Linear& a, hipStream_t st)
{
    const int ntiles = ceil_div(a.N, 16), nunits = ceil_div(a.K, kQ4Unit), frags = std::min(R * MT, kQ4LinWaves);
    hipLaunchKernelGGL((k_q4_linear<MT, R, G>), dim3(ceil_div(ntiles, R)), dim3(kQ4LinWaves * 64),
                       (size_t)frags * kQ4LinWaves * 1024, st, a, ntiles, nunits);
}

template <int MT, int R>
static void q4_linear_group(const Q4Linear& a, hipStream_t st)
{
    if (a.group == 128) q4_linear_of<MT, R, 1>(a, st);
    else if (a.group == 64) q4_linear_of<MT, R, 2>(a, st);
    else q4_linear_of<MT, R, 4>(a, st);
}

template <int MT>
static void q4_linear_rows(const Q4Linear& a, hipStream_t st)
{
    constexpr int kWide = MT <= 2 ? 4 : MT <= 4 ? 2 : 1;
    if (ceil_div(a.N, 16) >= 1024) q4_linear_group<MT, kWide>(a, st);
    else q4_linear_group<MT, 1>(a, st);
}

ghd_status launch_q4_linear(Q4Linear a, void*, hipStream_t st)
{
    if (a.M <= 16) q4_linear_rows<1>(a, st);
    else if (a.M <= 32) q4_linear_rows<2>(a, st);
    else if (a.M <= 64) q4_linear_rows<4>(a, st);
    else q4_linear_rows<8>(a, st);
    return check_launch();
}

// ---- packing -----------------------------------------------------------------------------
// One thread a word of codes; the first 16 of a unit's 256 also write a row's scales and zero points.
__global__ __launch_bounds__(256) void k_q4_pack(char* dst, const uint8_t* codes, const half_t* scales, const uint8_t* zeros,
                                                 int N, int K, int group, int nunits)
{
    const int tile = blockIdx.x / nunits, unit = blockIdx.x % nunits, per = kQ4Unit / group, groups = (K + group - 1) / group;
    char* at = dst + (size_t)blockIdx.x * q4_unit_bytes(group);
    const int lane = threadIdx.x >> 2, s = threadIdx.x & 3, n = tile * 16 + (lane & 15);
    const int k = unit * kQ4Unit + 32 * s + 8 * (lane >> 4);
    uint32_t word = 0;
    if (n < N && k < K) {
        const uint8_t* src = codes + (size_t)n * (K / 2) + k / 2;
#pragma unroll
        for (int p = 0; p < 4; ++p) word |= (uint32_t)(src[p] & 15) << 4 * p | (uint32_t)(src[p] >> 4) << (16 + 4 * p);
    }
    ((uint32_t*)at)[threadIdx.x] = word;
    if ((int)threadIdx.x < 16 * per) {
        const int row = threadIdx.x / per, i = threadIdx.x % per, q = unit * per + i;
        half2_ m = {0, (half_t)-1032.f};
        if (tile * 16 + row < N && q < groups) {
            const size_t e = (size_t)(tile * 16 + row) * groups + q;
            m[0] = scales[e];
            if (zeros) m[1] = (half_t)(-1024.f - (float)zeros[e]);
        }
        ((half2_*)(at + 1024))[threadIdx.x] = m;
    }
}

ghd_status launch_q4_pack(void* dst, const void* codes, const void* scales, const void* zeros, int N, int K, int group,
                          hipStream_t st)
{
    const int nunits = ceil_div(K, kQ4Unit);
    hipLaunchKernelGGL(k_q4_pack, dim3(ceil_div(N, 16) * nunits), dim3(256), 0, st, (char*)dst, (const uint8_t*)codes,
                       (const half_t*)scales, (const uint8_t*)zeros, N, K, group, nunits);
    return check_launch();
}

}  // namespace ghd
