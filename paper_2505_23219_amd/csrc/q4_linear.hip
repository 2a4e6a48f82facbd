// Linear layer over 4-bit weights with group scales, 1 to 128 rows.
//
// y[m, n] = sum over groups of scale[n, group] * (sum over the group's k of x[m, k] (code[n, k] - zero[n, group])).  The inner
// sums are products of fp16 numbers with whole numbers below 256, exact, summed in 32 bits by the MFMA; the scale is applied to
// them in 32 bits, so nothing is rounded to fewer bits before the result.  x is the A operand and W the B operand: a lane's
// operand, its column of the result, and with them scale and zero point, all belong to one row of W.
#include "q4.h"
#include "attention_impl.h"

namespace ghd {

constexpr int kQ4LinWaves = 8;
typedef uint32_t word4 __attribute__((ext_vector_type(4)));

// rows m0 .. m0 + 3 of column n
__device__ __forceinline__ void q4_store(const Q4Linear& a, int n, int m0, floatx4 y)
{
    if (n >= a.N) return;
#pragma unroll
    for (int e = 0; e < 4; ++e) {
        if (m0 + e >= a.M) break;
        const int64_t at = (int64_t)(m0 + e) * a.ldy + n;
        if (a.out16) ((half_t*)a.y)[at] = (half_t)y[e];
        else ((float*)a.y)[at] = y[e];
    }
}

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
            q4_store(a, (tile0 + f / MT) * 16 + r, f % MT * 16 + 4 * g, y);
        }
    }
}

// Above 16 rows x is most of what a compute unit reads, so the wavefronts of a workgroup share it: each has RW tiles of
// its own, and all the same columns, whose x lies in LDS as MFMA operands (1 KiB a k-step and 16 rows, lane after lane, loaded
// without passing through registers).  A ring of kRing units, one barrier a unit; weights are requested kRing - 1 units ahead.
constexpr int kQ4RowWaves = 4, kRing = 3;

template <int MT, int RW, int G>
__global__ __launch_bounds__(kQ4RowWaves * 64, 2) void k_q4_linear_rows(const Q4Linear a, int ntiles, int nunits, int splits)
{
    constexpr int kUnitBytes = 1024 + 64 * G, kSteps = 4 / G, kBuf = MT * 4096;
    constexpr int kLoads = MT + 2 * RW;                            // a wavefront's requests for one unit
    extern __shared__ __attribute__((aligned(16))) char lds[];
    const uint32_t lds0 = (uint32_t)(uintptr_t)(__attribute__((address_space(3))) char*)lds;
    const int lane = threadIdx.x & 63, wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6), r = lane & 15, g = lane >> 4;
    const int split = blockIdx.x % splits, tile0 = (blockIdx.x / splits * kQ4RowWaves + wave) * RW;
    const int u0 = nunits * split / splits, u1 = nunits * (split + 1) / splits;
    // x through a buffer resource: what lies behind its last row is not read.  A wavefront requests k-step `wave` of every row
    // tile, lane (g, r) row r, columns 8 g .. + 7.
    const __amdgpu_buffer_rsrc_t xbuf =
        __builtin_amdgcn_make_buffer_rsrc((void*)a.x, 0, (int)(((a.M - 1) * a.ldx + a.K) * 2), 0x00027000);
    const int xlane = r * (int)a.ldx * 2 + 16 * g, xtile = 16 * (int)a.ldx * 2;
    GLOBAL const char* wtile[RW];
#pragma unroll
    for (int t = 0; t < RW; ++t) wtile[t] = gp(a.W + (size_t)min(tile0 + t, ntiles - 1) * nunits * kUnitBytes);
    struct Unit {
        word4 w[RW];
        half2_ meta[RW][G];
    } ring[kRing];
    auto request = [&](int u, int slot) {
#pragma unroll
        for (int i = 0; i < MT; ++i)
            __builtin_amdgcn_raw_ptr_buffer_load_lds(xbuf, (LdsPtr)(uintptr_t)(lds0 + slot * kBuf + (i * 4 + wave) * 1024), 16, xlane,
                                                     i * xtile + u * (kQ4Unit * 2) + wave * 64, 0, 0);
#pragma unroll
        for (int t = 0; t < RW; ++t) {
            GLOBAL const char* p = wtile[t] + (size_t)u * kUnitBytes;
            ring[slot].w[t] = *(GLOBAL const word4*)(p + lane * 16);
            if constexpr (G == 1) ring[slot].meta[t][0] = *(GLOBAL const half2_*)(p + 1024 + r * 4);
            else if constexpr (G == 2) {
                const half4 m = *(GLOBAL const half4*)(p + 1024 + r * 8);
                ring[slot].meta[t][0] = (half2_){m[0], m[1]};
                ring[slot].meta[t][1] = (half2_){m[2], m[3]};
            } else {
                const half8 m = *(GLOBAL const half8*)(p + 1024 + r * 16);
#pragma unroll
                for (int q = 0; q < 4; ++q) ring[slot].meta[t][q] = (half2_){m[2 * q], m[2 * q + 1]};
            }
        }
        pin_order();
    };
    floatx4 acc[RW][MT];
#pragma unroll
    for (int t = 0; t < RW; ++t)
#pragma unroll
        for (int mt = 0; mt < MT; ++mt) acc[t][mt] = (floatx4){0.f, 0.f, 0.f, 0.f};
#pragma unroll
    for (int p = 0; p < kRing - 1; ++p) request(min(u0 + p, u1 - 1), p);
    for (int u = u0; u < u1; u += kRing) {
#pragma unroll
        for (int p = 0; p < kRing; ++p) {
            const int unit = u + p;
            if (unit >= u1) break;
            wait_loads<(kRing - 2) * kLoads>();
            barrier_lds();
            if ((unit + 1) * kQ4Unit > a.K) {                      // the last unit, where it is not whole
                for (int c = threadIdx.x; c < MT * 256; c += kQ4RowWaves * 64)
                    if (unit * kQ4Unit + (c >> 6) % 4 * 32 + ((c & 63) >> 4) * 8 >= a.K)
                        *(half8*)(lds + p * kBuf + c * 16) = (half8){0, 0, 0, 0, 0, 0, 0, 0};
                barrier_lds();
            }
            request(min(unit + kRing - 1, u1 - 1), (p + kRing - 1) % kRing);
            const half8* xs = (const half8*)(lds + p * kBuf) + lane;
#pragma unroll
            for (int q = 0; q < G; ++q) {
                floatx4 sum[RW][MT];
#pragma unroll
                for (int s = q * kSteps; s < (q + 1) * kSteps; ++s) {
                    half8 b[RW];
#pragma unroll
                    for (int t = 0; t < RW; ++t) b[t] = q4_codes(ring[p].w[t][s], pair_of(ring[p].meta[t][q][1]));
#pragma unroll
                    for (int mt = 0; mt < MT; ++mt) {
                        const half8 x = xs[(mt * 4 + s) * 64];
#pragma unroll
                        for (int t = 0; t < RW; ++t)
                            sum[t][mt] = __builtin_amdgcn_mfma_f32_16x16x32_f16(
                                x, b[t], s == q * kSteps ? (floatx4){0.f, 0.f, 0.f, 0.f} : sum[t][mt], 0, 0, 0);
                    }
                }
#pragma unroll
                for (int t = 0; t < RW; ++t)
#pragma unroll
                    for (int mt = 0; mt < MT; ++mt) acc[t][mt] += sum[t][mt] * (float)ring[p].meta[t][q][0];
            }
        }
    }
#pragma unroll
    for (int t = 0; t < RW; ++t) {
        if (tile0 + t >= ntiles) break;
#pragma unroll
        for (int mt = 0; mt < MT; ++mt) {
            if (splits > 1) {
                ((floatx4*)a.part)[(((size_t)split * ntiles + tile0 + t) * MT + mt) * 64 + lane] = acc[t][mt];
            } else {
                q4_store(a, (tile0 + t) * 16 + r, mt * 16 + 4 * g, acc[t][mt]);
            }
        }
    }
}

// Sums of the parts of k, in their order.  A wavefront takes one fragment.
__global__ __launch_bounds__(256) void k_q4_linear_sum(const Q4Linear a, int frags, int mts, int splits)
{
    const int lane = threadIdx.x & 63, f = blockIdx.x * 4 + (threadIdx.x >> 6);
    if (f >= frags) return;
    floatx4 y = ((const floatx4*)a.part)[(size_t)f * 64 + lane];
    for (int s = 1; s < splits; ++s) y += ((const floatx4*)a.part)[((size_t)s * frags + f) * 64 + lane];
    q4_store(a, f / mts * 16 + (lane & 15), f % mts * 16 + 4 * (lane >> 4), y);
}

struct Q4Cut {
    int mt, rw, splits;      // rw 0: the kernel of up to 16 rows
};

static Q4Cut q4_cut(int M, int N, int K)
{
    const int ntiles = ceil_div(N, 16), nunits = ceil_div(K, kQ4Unit), rt = ceil_div(M, 16);
    Q4Cut c = {rt <= 4 ? rt : rt <= 6 ? 6 : 8, 0, 1};
    if (rt == 1) return c;
    c.rw = 2;
    const int blocks = ceil_div(ntiles, c.rw * kQ4RowWaves);
    c.splits = std::max(1, std::min(nunits / 4, 256 / blocks));
    return c;
}

size_t q4_linear_bytes(int M, int N, int K)
{
    const Q4Cut c = q4_cut(M, N, K);
    return c.splits == 1 ? 256 : align_up((size_t)c.splits * ceil_div(N, 16) * c.mt * 1024, 256);
}

template <int MT, int RW, int G>
static ghd_status q4_rows_of(const Q4Linear& a, const Q4Cut& c, hipStream_t st)
{
    const int ntiles = ceil_div(a.N, 16), nunits = ceil_div(a.K, kQ4Unit);
    const size_t lds = (size_t)kRing * MT * 4096;
    const ghd_status s = launch_resident_checked((const void*)k_q4_linear_rows<MT, RW, G>, kQ4RowWaves * 64, lds, nullptr);
    if (s) return s;
    hipLaunchKernelGGL((k_q4_linear_rows<MT, RW, G>), dim3(ceil_div(ntiles, RW * kQ4RowWaves) * c.splits), dim3(kQ4RowWaves * 64),
                       lds, st, a, ntiles, nunits, c.splits);
    if (c.splits > 1)
        hipLaunchKernelGGL(k_q4_linear_sum, dim3(ceil_div(ntiles * MT, 4)), dim3(256), 0, st, a, ntiles * MT, MT, c.splits);
    return check_launch();
}

template <int MT, int RW>
static ghd_status q4_rows_group(const Q4Linear& a, const Q4Cut& c, hipStream_t st)
{
    if (a.group == 128) return q4_rows_of<MT, RW, 1>(a, c, st);
    if (a.group == 64) return q4_rows_of<MT, RW, 2>(a, c, st);
    return q4_rows_of<MT, RW, 4>(a, c, st);
}

template <int R, int G>
static void q4_linear_of(const Q4Linear& a, hipStream_t st)
{
    const int ntiles = ceil_div(a.N, 16), nunits = ceil_div(a.K, kQ4Unit);
    hipLaunchKernelGGL((k_q4_linear<1, R, G>), dim3(ceil_div(ntiles, R)), dim3(kQ4LinWaves * 64),
                       (size_t)std::min(R, kQ4LinWaves) * kQ4LinWaves * 1024, st, a, ntiles, nunits);
}

template <int R>
static void q4_linear_group(const Q4Linear& a, hipStream_t st)
{
    if (a.group == 128) q4_linear_of<R, 1>(a, st);
    else if (a.group == 64) q4_linear_of<R, 2>(a, st);
    else q4_linear_of<R, 4>(a, st);
}

static ghd_status q4_linear_cut(Q4Linear a, const Q4Cut& c, void* ws, hipStream_t st)
{
    a.part = (float*)ws;
    if (c.rw == 0) {
        if (ceil_div(a.N, 16) >= 1024) q4_linear_group<4>(a, st);
        else q4_linear_group<1>(a, st);
        return check_launch();
    }
    switch (c.mt) {
    case 2: return q4_rows_group<2, 2>(a, c, st);
    case 3: return q4_rows_group<3, 2>(a, c, st);
    case 4: return q4_rows_group<4, 2>(a, c, st);
    case 6: return q4_rows_group<6, 2>(a, c, st);
    default: return q4_rows_group<8, 2>(a, c, st);
    }
}

ghd_status launch_q4_linear(const Q4Linear& a, void* ws, hipStream_t st)
{
    return q4_linear_cut(a, q4_cut(a.M, a.N, a.K), ws, st);
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
