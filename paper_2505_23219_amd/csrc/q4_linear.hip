// Linear layer over 4-bit weights with group scales, 1 to 128 rows.
//
// y[m, n] = sum over groups of scale[n, group] * (sum over the group's k of x[m, k] (code[n, k] - zero[n, group])).  The inner
// sums are products of fp16 numbers with whole numbers below 256, exact, summed in 32 bits by the MFMA; the scale is applied to
// them in 32 bits, so nothing is rounded to fewer bits before the result.  x is the A operand and W the B operand: a lane's
// operand, its column of the result, and with them scale and zero point, all belong to one row of W.
//
// A workgroup has R tiles of 16 rows of W by a range of units of 128 columns, which its eight wavefronts take in turn, each
// by itself: no barrier until their sums meet in LDS.  (Wavefronts that share x, with a barrier every few units, wait for each
// other: [4096, 4096] at 64 rows 12.1 us, 9.5 this way.)  x comes through LDS, where it is loaded without
// passing through registers, into a ring of the wavefront's own, half a unit a slot.  A request is 8 rows by 128 bytes, 8 lanes
// a line of the cache: with 16 rows by 64 bytes and the rows in neighbouring lanes, as the MFMA takes them, a compute unit
// reads 36 bytes/ns instead of 121.  LDS takes a request lane after lane; so that operands are read without bank conflicts the
// 16-byte pieces of row r of the 8 lie in the order piece ^ r.  Above 64 rows there are two groups of rows in workgroups of
// their own, on the same XCD, whose L2 has the weights for the second.
// Bound: at one row the bytes ([22016, 4096] 11.3 us with weights in the 256 MB cache, 13.0 from HBM, 3.6 TB/s); for small matrices
// the launch (3 to 4 us).
// Every workgroup begins somewhere else in its range (`turn`): rows of x are often a power of two apart, a unit's 256 bytes of
// all of them then lie in one channel of the L2, and all workgroups would ask that one at a time.
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

// What the first loads need comes in the twelve words that the hardware puts into scalar registers before a kernel starts; the
// argument block, host memory, is 0.6 us away.  cut: M | (groups of rows - 1) << 8 | log2 of the parts of k << 9.
struct Q4Launch {
    int ntiles, nunits, log_splits, splits, log_groups, row_groups;
};
#define Q4_LINEAR_FIRST const char *W, const half_t *x_rows, float *parts, void *out, int ldx, uint32_t cut, int K, int ntiles
__device__ __forceinline__ Q4Launch q4_linear_first(Q4Linear& a, Q4_LINEAR_FIRST)
{
    a.W = W;
    a.x = x_rows;
    a.part = parts;
    a.y = out;
    a.ldx = ldx;
    a.M = cut & 255;
    a.K = K;
    Q4Launch c;
    c.ntiles = ntiles;
    c.nunits = (K + kQ4Unit - 1) / kQ4Unit;
    c.log_splits = cut >> 9;
    c.splits = 1 << c.log_splits;
    c.log_groups = cut >> 8 & 1;
    c.row_groups = 1 << c.log_groups;
    return c;
}
// Where a workgroup begins in its range of n units: x modulo n, of x below 2^15 or anything.
__device__ __forceinline__ int q4_turn(int x, int n)
{
    const int at = x & 0x7fff;
    return __builtin_amdgcn_readfirstlane(at - q4_over(at, q4_inverse(n)) * n);
}

// x comes through a buffer resource that ends with the last number of its last row, and a request for what lies behind is dropped.
// Of the two offsets that a request has the check counts the lane's and may leave out the scalar one, so all of where a request
// goes is in the lane's: an addition for each (16 rows of [22016, 4096] 12.2 us, with scalar offsets 12.1).  A wavefront's lanes
// take 16 bytes each of 8 rows by 64 columns.
__host__ __device__ __forceinline__ int q4_x_bytes(int M, int K, int ldx) { return ((M - 1) * ldx + K) * 2; }
__host__ __device__ __forceinline__ int q4_x_lane(int lane, int ldx) { return (lane >> 3) * ldx * 2 + ((lane & 7) ^ (lane >> 3)) * 16; }
__host__ __device__ __forceinline__ int q4_x_first(int row, int col, int ldx) { return row * (ldx * 2) + col * 2; }

template <int MT, int R, int G>
__global__ __launch_bounds__(kQ4LinWaves * 64) void k_q4_linear(Q4_LINEAR_FIRST, Q4Linear a)
{
    const Q4Launch c = q4_linear_first(a, W, x_rows, parts, out, ldx, cut, K, ntiles);
    constexpr int kUnitBytes = 1024 + 64 * G, kHalf = MT * 2048;
    extern __shared__ __attribute__((aligned(16))) char lds[];
    const uint32_t lds0 = (uint32_t)(uintptr_t)(__attribute__((address_space(3))) char*)lds;
    const int lane = threadIdx.x & 63, wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6), r = lane & 15, g = lane >> 4;
    // workgroup (q row_groups + rows) 8 + xcd: item 8 q + xcd, one of the groups of rows
    const int q8 = blockIdx.x >> 3, rows = q8 & (c.row_groups - 1), item = (q8 >> c.log_groups) * 8 + (blockIdx.x & 7);
    if (item >> c.log_splits >= (c.ntiles + R - 1) / R) return;
    const int mrow0 = rows * MT * 16, M = min(a.M - mrow0, MT * 16);
    const int split = item & (c.splits - 1), tile0 = (item >> c.log_splits) * R;
    const int u0 = c.nunits * split >> c.log_splits, n = (c.nunits * (split + 1) >> c.log_splits) - u0;
    const int turn = q4_turn(q8 >> c.log_groups, n), mine = (n - wave + kQ4LinWaves - 1) / kQ4LinWaves;     // this wavefront's units
    const __amdgpu_buffer_rsrc_t xbuf =
        __builtin_amdgcn_make_buffer_rsrc((void*)(a.x + (int64_t)mrow0 * a.ldx), 0, q4_x_bytes(M, a.K, (int)a.ldx), 0x00027000);
    const int xlane = q4_x_lane(lane, (int)a.ldx);
    const int tile_bytes = c.nunits * kUnitBytes;
    GLOBAL const char* wbase = gp(a.W + (size_t)tile0 * tile_bytes);
    const int last = min(R, c.ntiles - tile0) - 1;                 // (tiles that are not there: the last one again)
    auto unit_of = [&](int i) {                                    // of this wavefront's (one that is not there: another)
        const int at = min(max(min(i, mine - 1), 0) * kQ4LinWaves + wave, n - 1) + turn;
        return u0 + (at >= n ? at - n : at);
    };
    auto request_x = [&](int j) {                                  // half j % 2 of unit j / 2
        const int u = unit_of(j >> 1);
        const uint32_t to = lds0 + (wave * 2 + (j & 1)) * kHalf;
#pragma unroll
        for (int m = 0; m < 2 * MT; ++m)
            __builtin_amdgcn_raw_ptr_buffer_load_lds(xbuf, (LdsPtr)(uintptr_t)(to + m * 1024), 16,
                                                     xlane + q4_x_first(8 * m, u * kQ4Unit + (j & 1) * 64, (int)a.ldx), 0, 0, 0);
        pin_order();
    };
    struct {
        word4 w;
        half2_ meta[G];
    } held[R];
    auto request_w = [&](int i, int t) {
        GLOBAL const char* p = wbase + (uint32_t)(min(t, last) * tile_bytes + unit_of(i) * kUnitBytes);
        held[t].w = *(GLOBAL const word4*)(p + lane * 16);
        if constexpr (G == 1) held[t].meta[0] = *(GLOBAL const half2_*)(p + 1024 + r * 4);
        else if constexpr (G == 2) {
            const half4 m = *(GLOBAL const half4*)(p + 1024 + r * 8);
            held[t].meta[0] = (half2_){m[0], m[1]};
            held[t].meta[1] = (half2_){m[2], m[3]};
        } else {
            const half8 m = *(GLOBAL const half8*)(p + 1024 + r * 16);
#pragma unroll
            for (int q = 0; q < 4; ++q) held[t].meta[q] = (half2_){m[2 * q], m[2 * q + 1]};
        }
        pin_order();
    };
    const Q4Bits bits;
    floatx4 acc[R][MT];
#pragma unroll
    for (int t = 0; t < R; ++t)
#pragma unroll
        for (int mt = 0; mt < MT; ++mt) acc[t][mt] = (floatx4){0.f, 0.f, 0.f, 0.f};
    request_x(0);
#pragma unroll
    for (int t = 0; t < R; ++t) request_w(0, t);
    for (int i = 0; i < mine; ++i) {
#pragma unroll
        for (int h = 0; h < 2; ++h) {
            request_x(2 * i + h + 1);
            // x of this half is there when no more is under way than was asked for after it: the next half's, and before
            // an even half the unit's weights
            if (h == 0) wait_loads<2 * MT + 2 * R>();
            else wait_loads<2 * MT>();
            pin_order();
            const int k0 = unit_of(i) * kQ4Unit + h * 64;
            // row r, columns 32 s + 8 g .. + 7: piece 4 s + g
            const char* xr = lds + (wave * 2 + h) * kHalf + (r >> 3) * 1024 + (r & 7) * 128;
            half8 x[2][MT];
#pragma unroll
            for (int s = 0; s < 2; ++s)
#pragma unroll
                for (int m = 0; m < MT; ++m) x[s][m] = *(const half8*)(xr + m * 2048 + ((4 * s + g) ^ (r & 7)) * 16);
            if (k0 + 64 > a.K)                                     // columns from K on are whatever lies behind the row
#pragma unroll
                for (int s = 0; s < 2; ++s)
#pragma unroll
                    for (int m = 0; m < MT; ++m)
                        if (k0 + 32 * s + 8 * g >= a.K) x[s][m] = (half8){0, 0, 0, 0, 0, 0, 0, 0};
#pragma unroll
            for (int t = 0; t < R; ++t) {
                floatx4 sum[MT];
#pragma unroll
                for (int s = 0; s < 2; ++s) {
                    constexpr int kPer = G == 4 ? 1 : 2;           // k-steps of a half that share a scale
                    const int k = 2 * h + s, q = k * G / 4;
                    const half8 b = q4_codes(bits, held[t].w[k], pair_of(held[t].meta[q][1]));
#pragma unroll
                    for (int m = 0; m < MT; ++m)
                        sum[m] = __builtin_amdgcn_mfma_f32_16x16x32_f16(x[s][m], b, s % kPer == 0 ? (floatx4){0.f, 0.f, 0.f, 0.f} : sum[m],
                                                                        0, 0, 0);
                    if (s % kPer == kPer - 1)
#pragma unroll
                        for (int m = 0; m < MT; ++m) acc[t][m] += sum[m] * (float)held[t].meta[q][0];
                }
                if (h == 1) request_w(i + 1, t);
            }
        }
    }
    wait_loads<0>();                                               // of x: none may land in LDS from here on
    // The wavefronts' sums meet in LDS, as many fragments at a time as fit, each added up by one wavefront in a fixed order.
    constexpr int kFrags = R * MT, kRound = std::min(kFrags, 4 * MT);
    floatx4* part = (floatx4*)lds;                                 // [wave][fragment][64]
#pragma unroll
    for (int f0 = 0; f0 < kFrags; f0 += kRound) {
        __syncthreads();
#pragma unroll
        for (int f = f0; f < std::min(f0 + kRound, kFrags); ++f) part[(wave * kRound + f - f0) * 64 + lane] = acc[f / MT][f % MT];
        __syncthreads();
        for (int e = wave; e < kRound; e += kQ4LinWaves) {
            floatx4 y = part[e * 64 + lane];
#pragma unroll
            for (int w = 1; w < kQ4LinWaves; ++w) y += part[(w * kRound + e) * 64 + lane];
            const int f = f0 + e, tile = tile0 + f / MT;
            if (f >= kFrags || tile >= c.ntiles) continue;
            if (c.splits > 1)
                ((floatx4*)a.part)[((((size_t)split * c.ntiles + tile) * c.row_groups + rows) * MT + f % MT) * 64 + lane] = y;
            else
                q4_store(a, tile * 16 + r, mrow0 + f % MT * 16 + 4 * g, y);
        }
    }
}

// Where a workgroup's share of W is large, what it reads of x again and again outweighs barriers: here 16 wavefronts share it.
// Four groups of wavefronts have RW tiles each; four shares of every group take the units of the workgroup's k range in turn, x
// and weights of the next four requested while four are worked on, one barrier every four; the shares' sums meet in LDS.  (Two
// shares of twice the registers, operands read ahead: [22016, 4096] at 64 rows 24.4 us, 21.8 with four; a finer ring, half
// a unit a barrier: 25.8; two shares with three turns under way instead of one: 23.2 and 22.3; weights requested a whole turn ahead
// instead of half of one 21.7 and 22.5, but with groups of 32 and 64 more registers than there are.)
// Bound: [32000, 5120] at 128 rows takes 54 to 56 us, from HBM as from the 256 MB cache (which three such matrices pass).  Of an earlier
// 58 it would have taken 27 with neither weights nor x to fetch, 33 with x alone, 50 with weights alone: their way into a compute
// unit, at 2 TB/s of the card's 4.75, with more of them under way no faster.  [4096, 11008] at 64 rows, 13.8 us (16.2 from HBM): a
// launch of 10, 4 of them before the first and behind the last product, and one that adds up.
constexpr int kQ4Groups = 4, kQ4Shares = 4, kQ4RowThreads = kQ4Groups * kQ4Shares * 64;

template <int MT, int RW, int G>
__global__ __launch_bounds__(kQ4RowThreads) void k_q4_linear_shared(Q4_LINEAR_FIRST, Q4Linear a)
{
    const Q4Launch c = q4_linear_first(a, W, x_rows, parts, out, ldx, cut, K, ntiles);
    constexpr int kUnitBytes = 1024 + 64 * G, kBuf = MT * 4096, KH = kQ4Shares;
    // k-steps summed up before the scale is applied; row tiles whose sums are under way (what the registers hold)
    constexpr int kSteps = G == 2 && MT * RW == 8 ? 1 : 4 / G, kAt = kSteps == 1 && MT > 3 ? 2 : MT;
    // workgroup (q row_groups + rows) 8 + xcd: item 8 q + xcd, one of the groups of rows
    const int q8 = blockIdx.x >> 3, rows = q8 & (c.row_groups - 1), item = (q8 >> c.log_groups) * 8 + (blockIdx.x & 7);
    if (item >> c.log_splits >= (c.ntiles + kQ4Groups * RW - 1) / (kQ4Groups * RW)) return;
    const int mrow0 = rows * MT * 16, M = min(a.M - mrow0, MT * 16);
    extern __shared__ __attribute__((aligned(16))) char lds[];
    const uint32_t lds0 = (uint32_t)(uintptr_t)(__attribute__((address_space(3))) char*)lds;
    const int lane = threadIdx.x & 63, wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6), r = lane & 15, g = lane >> 4;
    const int share = wave / kQ4Groups, grp = wave % kQ4Groups;
    const int split = item & (c.splits - 1), tile0 = ((item >> c.log_splits) * kQ4Groups + grp) * RW;
    const int u0 = c.nunits * split >> c.log_splits, n = (c.nunits * (split + 1) >> c.log_splits) - u0;
    const int turn = q4_turn(q8 >> c.log_groups, n);
    // the turn of four with the unit that K does not fill
    const int short_turn = a.K % kQ4Unit != 0 && u0 + n == c.nunits ? (turn == n - 1 ? 0 : n - 1 - turn) / KH : -1;
    // A wavefront requests 8 rows (the first or last of 16: grp / 2) by 64 columns (grp % 2) of every row tile of its share's unit.
    const __amdgpu_buffer_rsrc_t xbuf =
        __builtin_amdgcn_make_buffer_rsrc((void*)(a.x + (int64_t)mrow0 * a.ldx), 0, q4_x_bytes(M, a.K, (int)a.ldx), 0x00027000);
    const int xlane = q4_x_lane(lane, (int)a.ldx) + q4_x_first(grp / 2 * 8, grp % 2 * 64, (int)a.ldx);
    GLOBAL const char* wtile[RW];
#pragma unroll
    for (int t = 0; t < RW; ++t) wtile[t] = gp(a.W + (size_t)min(tile0 + t, c.ntiles - 1) * c.nunits * kUnitBytes);
    struct Unit {
        word4 w[RW];
        half2_ meta[RW][G];
    } ring[2];
    // this share's unit of turn i (one that is not there: the last one again)
    auto unit_of = [&](int i) {
        const int at = min(KH * i + share, n - 1) + turn;
        return u0 + (at >= n ? at - n : at);
    };
    auto request_x = [&](int i, int from, int to) {                // of row tiles [from, to)
        const int u = unit_of(i);
#pragma unroll
        for (int m = from; m < to; ++m)
            __builtin_amdgcn_raw_ptr_buffer_load_lds(xbuf, (LdsPtr)(uintptr_t)(lds0 + ((i & 1) * KH + share) * kBuf + (m * 4 + grp) * 1024),
                                                     16, xlane + q4_x_first(m * 16, u * kQ4Unit, (int)a.ldx), 0, 0, 0);
        pin_order();
    };
    auto request_w = [&](int i, int slot) {
        const int u = unit_of(i);
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
    const Q4Bits bits;
    floatx4 acc[RW][MT];
#pragma unroll
    for (int t = 0; t < RW; ++t)
#pragma unroll
        for (int mt = 0; mt < MT; ++mt) acc[t][mt] = (floatx4){0.f, 0.f, 0.f, 0.f};
    request_x(0, 0, MT);
    request_w(0, 0);
    for (int i0 = 0; KH * i0 < n; i0 += 2) {
#pragma unroll
        for (int p = 0; p < 2; ++p) {
            const int i = i0 + p;
            if (KH * i >= n) break;
            wait_loads<0>();
            barrier_lds();
            const int unit = unit_of(i);
            if (i == short_turn) {
                // columns from K on: whatever lay there, so they are made zero
                for (int e = threadIdx.x & 255; e < MT * 256; e += 256)
                    if (unit * kQ4Unit + (e >> 6) % 2 * 64 + ((e & 7) ^ (e >> 3 & 7)) * 8 >= a.K)
                        *(half8*)(lds + (p * KH + share) * kBuf + e * 16) = (half8){0, 0, 0, 0, 0, 0, 0, 0};
                barrier_lds();
            }
            if (KH * i + share >= n) continue;                     // the last turn may not have a unit for every share
            // row r, columns 32 s + 8 g .. + 7: of 64 columns piece s % 2 * 4 + g
            const char* xbase = lds + (p * KH + share) * kBuf + (r >> 3) * 2048 + (r & 7) * 128;
            const char* xs[2] = {xbase + (g ^ (r & 7)) * 16, xbase + ((4 + g) ^ (r & 7)) * 16};
            floatx4 sum[RW][MT];
#pragma unroll
            for (int s = 0; s < 4; ++s) {
                // (requests are spread: the compute unit takes one every 16 cycles, and products would wait behind all)
                pin_order();
                if (s == 0) request_x(i + 1, 0, MT / 2);
                if (s == 1) request_x(i + 1, MT / 2, MT);
                if (s == 2) request_w(i + 1, p ^ 1);
                half8 x[MT], b[RW];
#pragma unroll
                for (int m = 0; m < MT; ++m) x[m] = *(const half8*)(xs[s % 2] + m * 4096 + s / 2 * 1024);
#pragma unroll
                for (int t = 0; t < RW; ++t) b[t] = q4_codes(bits, ring[p].w[t][s], pair_of(ring[p].meta[t][s * G / 4][1]));
#pragma unroll
                for (int m0 = 0; m0 < MT; m0 += kAt) {
                    if (m0) pin_order();
#pragma unroll
                    for (int m = m0; m < m0 + kAt; ++m)
#pragma unroll
                        for (int t = 0; t < RW; ++t)
                            sum[t][m] = __builtin_amdgcn_mfma_f32_16x16x32_f16(
                                x[m], b[t], s % kSteps == 0 ? (floatx4){0.f, 0.f, 0.f, 0.f} : sum[t][m], 0, 0, 0);
                    if (s % kSteps == kSteps - 1)
#pragma unroll
                        for (int t = 0; t < RW; ++t)
#pragma unroll
                            for (int m = m0; m < m0 + kAt; ++m) acc[t][m] += sum[t][m] * (float)ring[p].meta[t][s * G / 4][0];
                }
            }
        }
    }
    wait_loads<0>();                                               // of x: none may land in LDS from here on
    __syncthreads();
    // The shares' sums meet in LDS, added up in their order, every KH-th fragment by one of them.
    constexpr int kFrags = RW * MT, kMine = (kFrags + KH - 1) / KH, kShare = kQ4Groups * kFrags * 64;
    floatx4* sums = (floatx4*)lds + (size_t)grp * (kFrags * 64) + lane;
#pragma unroll
    for (int f = 0; f < kFrags; ++f) sums[share * kShare + f * 64] = acc[f / MT][f % MT];
    __syncthreads();
    floatx4 y[kMine];
#pragma unroll
    for (int j = 0; j < kMine; ++j) {
        const int f = min(j * KH + share, kFrags - 1);
        y[j] = sums[f * 64];
#pragma unroll
        for (int h = 1; h < KH; ++h) y[j] += sums[h * kShare + f * 64];
    }
    if (c.splits > 1) {
#pragma unroll
        for (int j = 0; j < kMine; ++j) {
            const int f = j * KH + share, tile = tile0 + f / MT;
            if (f < kFrags && tile < c.ntiles)
                ((floatx4*)a.part)[((((size_t)split * c.ntiles + tile) * c.row_groups + rows) * MT + f % MT) * 64 + lane] = y[j];
        }
        return;
    }
    // rows of y side by side, so that a wavefront stores 64 neighbours
    constexpr int kCols = kQ4Groups * RW * 16, kRow = kCols + 4;
    float* ys = (float*)lds;
    __syncthreads();
#pragma unroll
    for (int j = 0; j < kMine; ++j) {
        const int f = j * KH + share;
        if (f >= kFrags) break;
#pragma unroll
        for (int e = 0; e < 4; ++e) ys[(f % MT * 16 + 4 * g + e) * kRow + (grp * RW + f / MT) * 16 + r] = y[j][e];
    }
    __syncthreads();
    const int n0 = item * kCols;
    for (int m = wave; m < M; m += KH * kQ4Groups)
#pragma unroll
        for (int col = 0; col < kCols; col += 64) {
            const int n = n0 + col + lane;
            if (n >= a.N) break;
            const float v = ys[m * kRow + col + lane];
            if (a.out16) ((half_t*)a.y)[(int64_t)(mrow0 + m) * a.ldy + n] = (half_t)v;
            else ((float*)a.y)[(int64_t)(mrow0 + m) * a.ldy + n] = v;
        }
}

// Sums of the parts of k, in their order.  A wavefront takes one fragment.  cut: M | parts << 8 | (fp16 results) << 16.
__global__ __launch_bounds__(256) void k_q4_linear_sum(const floatx4* part, void* out, int N, int ntiles, int64_t ldy, uint32_t cut)
{
    const int lane = threadIdx.x & 63, tile = blockIdx.x * 4 + (threadIdx.x >> 6), mt = blockIdx.y, mts = gridDim.y, splits = cut >> 8 & 255;
    if (tile >= ntiles) return;
    Q4Linear a = {};
    a.y = out;
    a.M = cut & 255;
    a.N = N;
    a.ldy = ldy;
    a.out16 = cut >> 16;
    const floatx4* p = part + ((size_t)tile * mts + mt) * 64 + lane;
    const size_t step = (size_t)ntiles * mts * 64;
    floatx4 y = {0.f, 0.f, 0.f, 0.f};
    for (int s0 = 0; s0 < splits; s0 += 8) {          // eight requests at a time
        floatx4 v[8];
#pragma unroll
        for (int s = 0; s < 8; ++s) v[s] = p[min(s0 + s, splits - 1) * step];
#pragma unroll
        for (int s = 0; s < 8; ++s)
            if (s0 + s < splits) y += v[s];
    }
    q4_store(a, tile * 16 + (lane & 15), mt * 16 + 4 * (lane >> 4), y);
}

struct Q4Cut {
    bool shared;                 // which of the two kernels
    int mt, tiles, splits;       // row tiles of a workgroup, tiles of W (of a wavefront, where x is shared), parts of k
};

static int q4_row_groups(int M, int mt) { return ceil_div(M, mt * 16); }

// us that a unit of 128 columns takes a workgroup, 256 of them at work, by its row tiles (less one) and tiles of W; 0: a kernel that
// there is not, as others are faster.  Fitted, with the constants in q4_cut, to 2000 calls: 1 to 128 rows, 1024 to 32000 by 1024
// to 11008, every cut; the choice is 1.6% slower than the fastest cut on average, 18% at most.
static float q4_unit_us(bool shared, int mt, int tiles)
{
    static const float own[4][4] = {{.060f, .098f, .172f, .331f}, {.109f, .151f, .247f}, {.163f, .208f, .322f}, {.205f, .256f}};
    static const float with[4][2] = {{}, {0.f, .406f}, {0.f, .485f}, {.353f, .566f}};
    return shared ? with[mt - 1][tiles - 1] : own[mt - 1][tiles == 8 ? 3 : tiles / 2];
}

// The cut that is estimated to be fastest: rounds of 256 workgroups, and with k in parts a launch more that adds up what the
// parts wrote.
static Q4Cut q4_cut(int M, int N, int K)
{
    const int ntiles = ceil_div(N, 16), nunits = ceil_div(K, kQ4Unit), rt = ceil_div(M, 16);
    const int mt = rt <= 4 ? rt : (rt + 1) / 2, groups = q4_row_groups(M, mt);
    Q4Cut best = {};
    float least = 0.f;
    for (int shared = 0; shared < 2; ++shared)
        for (int tiles = 1; tiles <= (shared ? 2 : 8); tiles *= 2) {
            const float unit_us = q4_unit_us(shared, mt, tiles);
            if (unit_us == 0.f) continue;
            const int blocks = ceil_div(ntiles, shared ? tiles * kQ4Groups : tiles) * groups, turn = shared ? kQ4Shares : kQ4LinWaves;
            for (int splits = 1; splits <= 32 && (splits == 1 || splits * turn <= nunits); splits *= 2) {
                const int units = ceil_div(ceil_div(nunits, splits), turn) * turn, rounds = ceil_div(blocks * splits, 256);
                float us = rounds * ((shared ? 2.25f : 1.12f) + units * unit_us);
                if (splits > 1) us += 2.5f + 0.62e-6f * 1024.f * splits * ntiles * groups * mt;
                if (least == 0.f || us < least) {
                    least = us;
                    best = {shared != 0, mt, tiles, splits};
                }
            }
        }
    return best;
}

static size_t q4_cut_bytes(const Q4Cut& c, int M, int N)
{
    return c.splits == 1 ? 256 : align_up((size_t)c.splits * ceil_div(N, 16) * q4_row_groups(M, c.mt) * c.mt * 1024, 256);
}

// The most that a call of up to M rows takes, whatever its cut.
size_t q4_linear_bytes(int M, int N, int K)
{
    size_t most = 0;
    for (int m = std::min(M, 16); m <= M; m = m < M ? std::min(m + 16, M) : m + 1) most = std::max(most, q4_cut_bytes(q4_cut(m, N, K), m, N));
    return most;
}

static ghd_status q4_linear_start(const Q4Linear& a, const Q4Cut& c,
                                  void (*kernel)(const char*, const half_t*, float*, void*, int, uint32_t, int, int, Q4Linear), int threads,
                                  int tiles, size_t lds, hipStream_t st)
{
    const int groups = q4_row_groups(a.M, c.mt), ntiles = ceil_div(a.N, 16);
    const ghd_status s = launch_resident_checked((const void*)kernel, threads, lds, nullptr);
    if (s) return s;
    const uint32_t cut = a.M | (groups - 1) << 8 | __builtin_ctz(c.splits) << 9;
    hipLaunchKernelGGL(kernel, dim3(ceil_div(ceil_div(ntiles, tiles) * c.splits, 8) * 8 * groups), dim3(threads), lds, st, a.W, a.x, a.part, a.y,
                       (int)a.ldx, cut, a.K, ntiles, a);
    if (c.splits > 1)
        hipLaunchKernelGGL(k_q4_linear_sum, dim3(ceil_div(ntiles, 4), groups * c.mt), dim3(256), 0, st, (const floatx4*)a.part, a.y, a.N, ntiles,
                           a.ldy, a.M | c.splits << 8 | (a.out16 ? 1u << 16 : 0u));
    return check_launch();
}

template <int MT, int R, int G>
static ghd_status q4_linear_of(const Q4Linear& a, const Q4Cut& c, hipStream_t st)
{
    return q4_linear_start(a, c, k_q4_linear<MT, R, G>, kQ4LinWaves * 64, R, (size_t)kQ4LinWaves * MT * 4096, st);
}
template <int MT, int RW, int G>
static ghd_status q4_shared_of(const Q4Linear& a, const Q4Cut& c, hipStream_t st)
{
    return q4_linear_start(a, c, k_q4_linear_shared<MT, RW, G>, kQ4RowThreads, RW * kQ4Groups,
                           (size_t)kQ4Shares * MT * std::max(2 * 4096, kQ4Groups * RW * 1024), st);
}

template <int MT, int R>
static ghd_status q4_linear_group(const Q4Linear& a, const Q4Cut& c, hipStream_t st)
{
    if (a.group == 128) return q4_linear_of<MT, R, 1>(a, c, st);
    if (a.group == 64) return q4_linear_of<MT, R, 2>(a, c, st);
    return q4_linear_of<MT, R, 4>(a, c, st);
}
template <int MT, int RW>
static ghd_status q4_shared_group(const Q4Linear& a, const Q4Cut& c, hipStream_t st)
{
    if (a.group == 128) return q4_shared_of<MT, RW, 1>(a, c, st);
    if (a.group == 64) return q4_shared_of<MT, RW, 2>(a, c, st);
    return q4_shared_of<MT, RW, 4>(a, c, st);
}

template <int MT>
static ghd_status q4_linear_tiles(const Q4Linear& a, const Q4Cut& c, hipStream_t st)
{
    if constexpr (MT == 4)
        if (c.shared && c.tiles == 1) return q4_shared_group<MT, 1>(a, c, st);
    if constexpr (MT > 1)
        if (c.shared) return q4_shared_group<MT, 2>(a, c, st);
    if (c.tiles == 1) return q4_linear_group<MT, 1>(a, c, st);
    if constexpr (MT < 4)
        if (c.tiles == 4) return q4_linear_group<MT, 4>(a, c, st);
    if constexpr (MT == 1)
        if (c.tiles == 8) return q4_linear_group<MT, 8>(a, c, st);
    return q4_linear_group<MT, 2>(a, c, st);
}

// Do rows of a and of b share a byte?  (Rows of one may lie between those of the other: halves of one wide buffer.)
struct Q4Rows {
    uintptr_t at;
    int64_t step, bytes;
    int n;
};
static bool q4_meet(Q4Rows a, Q4Rows b)
{
    while (a.n > 0 && b.n > 0) {
        if (a.at + a.bytes <= b.at) a.at += a.step, --a.n;
        else if (b.at + b.bytes <= a.at) b.at += b.step, --b.n;
        else return true;
    }
    return false;
}

// Workgroups that are done write y while others still read x and W, so y must lie beside both.
bool q4_linear_meets(const Q4Linear& a)
{
    const int size = a.out16 ? 2 : 4;
    const Q4Rows y = {(uintptr_t)a.y, a.ldy * size, (int64_t)a.N * size, a.M};
    return q4_meet(y, {(uintptr_t)a.x, a.ldx * 2, a.K * 2, a.M}) || q4_meet(y, {(uintptr_t)a.W, 0, (int64_t)q4_weight_bytes(a.N, a.K, a.group), 1});
}

ghd_status launch_q4_linear(Q4Linear a, void* ws, size_t ws_bytes, hipStream_t st)
{
    const Q4Cut c = q4_cut(a.M, a.N, a.K);
    if (ws_bytes < q4_cut_bytes(c, a.M, a.N)) return GHD_ERR_WORKSPACE;
    if (q4_linear_meets(a)) return GHD_ERR_SHAPE;
    a.part = (float*)ws;
    switch (c.mt) {
    case 1: return q4_linear_tiles<1>(a, c, st);
    case 2: return q4_linear_tiles<2>(a, c, st);
    case 3: return q4_linear_tiles<3>(a, c, st);
    default: return q4_linear_tiles<4>(a, c, st);
    }
}

// Which bytes behind x the requests of a call that the hardware lets through end at most, and how many numbers of x they bring.
void q4_x_on_host(int M, int N, int K, int ldx, int64_t* out2)
{
    const Q4Cut c = q4_cut(M, N, K);
    out2[0] = out2[1] = 0;
    for (int mrow0 = 0; mrow0 < M; mrow0 += c.mt * 16) {
        const int rows = std::min(M - mrow0, c.mt * 16), bytes = q4_x_bytes(rows, K, ldx);
        for (int u = 0; u < ceil_div(K, kQ4Unit); ++u)
            for (int half = 0; half < 2; ++half)
                for (int row = 0; row < c.mt * 16; row += 8)
                    for (int lane = 0; lane < 64; ++lane) {
                        const int at = q4_x_lane(lane, ldx) + q4_x_first(row, u * kQ4Unit + half * 64, ldx);
                        if (at >= bytes) continue;
                        out2[0] = std::max<int64_t>(out2[0], (int64_t)mrow0 * ldx * 2 + at + 16);
                        const int col = u * kQ4Unit + half * 64 + ((lane & 7) ^ (lane >> 3)) * 8;
                        if (row + (lane >> 3) < rows && col < K) out2[1] += 8;
                    }
    }
}

// ---- packing -----------------------------------------------------------------------------
// One thread a word of codes; the first 16 of a unit's 256 also write a row's scales and zero points.
__global__ __launch_bounds__(256) void k_q4_pack(char* dst, const uint8_t* codes, const half_t* scales, const uint8_t* zeros,
                                                 int N, int K, int group, int nunits, int tile0)
{
    const int tile = tile0 + blockIdx.x / nunits, unit = blockIdx.x % nunits, per = kQ4Unit / group, groups = (K + group - 1) / group;
    char* at = dst + ((size_t)tile * nunits + unit) * q4_unit_bytes(group);
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
    const int nunits = ceil_div(K, kQ4Unit), ntiles = ceil_div(N, 16), most = kQ4MostGroups / nunits;
    for (int tile0 = 0; tile0 < ntiles; tile0 += most) {
        hipLaunchKernelGGL(k_q4_pack, dim3(std::min(most, ntiles - tile0) * nunits), dim3(256), 0, st, (char*)dst, (const uint8_t*)codes,
                           (const half_t*)scales, (const uint8_t*)zeros, N, K, group, nunits, tile0);
        const ghd_status s = check_launch();
        if (s) return s;
    }
    return GHD_OK;
}

}  // namespace ghd
