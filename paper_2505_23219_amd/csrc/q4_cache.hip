// Rows into, inside and out of a 4-bit cache: append (with the rotary turn of keys and queries on the way),
// commit of an accepted path, reading back.
//
// A group x of 32 channels is held as lo = min x, s = fp16((max x - lo) / 15) and codes rint((x - lo) / s).  All of it is
// IEEE arithmetic in the order written here, so that the codes are the same wherever they are worked out.
//
// Everything here works on octets: 8 cache rows of a head, whose V codes share words (a channel's 8 keys, see q4.h).  A
// wavefront has an octet of a head to itself, so a word that a call changes in part is read and written back by one thread.
#include "q4.h"
#include "attention_impl.h"

namespace ghd {

typedef uint32_t word4 __attribute__((ext_vector_type(4)));

template <int CTRL>
__device__ __forceinline__ uint32_t dpp(uint32_t x)
{
    return (uint32_t)__builtin_amdgcn_update_dpp(0, (int)x, CTRL, 0xf, 0xf, true);
}
constexpr int kXor1 = 0xB1, kXor2 = 0x4E, kMirror8 = 0x141, kMirror16 = 0x140;   // exchanges inside 16 lanes

// over 16 lanes (each has two of a group's 32 channels)
template <class Op>
__device__ __forceinline__ uint32_t over16(uint32_t x, Op op)
{
    x = op(x, dpp<kXor1>(x));
    x = op(x, dpp<kXor2>(x));
    x = op(x, dpp<kMirror8>(x));
    return op(x, dpp<kMirror16>(x));
}

struct Group {
    half_t lo, s;
    uint32_t c0, c1;       // this lane's two codes
};

// x: this lane's two channels of a group that 16 lanes hold
__device__ __forceinline__ Group quantise(half2_ x)
{
#pragma clang fp contract(off)
    const uint32_t bits = __builtin_bit_cast(uint32_t, x);
    // (min x, min -x) of the two channels, then of the 16 lanes
    const half2_ m = {x[0] < x[1] ? x[0] : x[1], x[0] < x[1] ? -x[1] : -x[0]};
    const half2_ r = __builtin_bit_cast(half2_, over16(__builtin_bit_cast(uint32_t, m), [](uint32_t a, uint32_t b) {
        return __builtin_bit_cast(uint32_t, __builtin_elementwise_min(__builtin_bit_cast(half2_, a), __builtin_bit_cast(half2_, b)));
    }));
    const bool odd = (bits & 0x7c00u) == 0x7c00u || (bits & 0x7c000000u) == 0x7c000000u;
    const uint32_t bad = over16((uint32_t)odd, [](uint32_t a, uint32_t b) { return a | b; });
    Group g;
    g.lo = r[0];
    const float lo = (float)r[0];
    g.s = (half_t)((-(float)r[1] - lo) / 15.f);
    // rounded up, the scale of the widest ranges would make the largest code stand for more than fp16 holds
    if (lo + 15.f * (float)g.s >= 65520.f)
        g.s = __builtin_bit_cast(half_t, (uint16_t)(__builtin_bit_cast(uint16_t, g.s) - 1));
    const float s = (float)g.s;
    auto code = [&](half_t v) { return s > 0.f ? (uint32_t)fminf(fmaxf(rintf(((float)v - lo) / s), 0.f), 15.f) : 0u; };
    g.c0 = code(x[0]);
    g.c1 = code(x[1]);
    if (bad) {             // a group with an infinity or NaN in it reads as NaN
        g.s = __builtin_bit_cast(half_t, (uint16_t)0x7e00);
        g.c0 = g.c1 = 0;
    }
    return g;
}

// ---- append ------------------------------------------------------------------------------
// Bound: for a tree's rows latency (one launch, rows read, reduced over lanes and written); for a prompt the bytes.
// Rows are read 4 bytes a lane, two channels and, of keys and queries, the two they turn with half a row
// away; 16 lanes hold a group.  A wavefront has one octet and a run of heads, whose cosines it works out once: heads
// 0 .. nkv - 1 are keys and values, nkv .. nkv + nq - 1 queries.
template <int D>
__global__ __launch_bounds__(256) void k_q4_append(const Q4Append a, int chunks, int per_chunk, int units)
{
    const int lane = threadIdx.x & 63, unit = blockIdx.x * 4 + (threadIdx.x >> 6);
    if (unit >= units) return;
    const int octet = a.kv_len / 8 + unit / chunks, head0 = unit % chunks * per_chunk;
    const int head1 = min(head0 + per_chunk, a.nkv + a.nq);
    const int row0 = octet * 8 - a.kv_len;                    // input row of the octet's first key (may be negative)
    constexpr int kLanes = D / 4, kSets = 64 / kLanes, kRows = 8 / kSets;   // lanes a row of turned pairs; rows a lane
    const int i = lane % kLanes, set = lane / kLanes;         // channels 2 i, 2 i + 1 and D / 2 further
    float cs[kRows][2], sn[kRows][2];
    const bool turn = a.rope_base > 0.f;
    if (turn) {
        int up0 = 0, up1 = 0;
        if (a.parent) {
            up0 = a.parent[min(lane, a.M - 1)];
            up1 = a.parent[min(lane + 64, a.M - 1)];
        }
        const TreeNodes<2> t = tree_nodes<2, false>(up0, up1, a.parent ? a.M : 0, lane);
#pragma unroll
        for (int j = 0; j < kRows; ++j) {
            const int row = row0 + set * kRows + j, in = min(max(row, 0), a.M - 1);
            const int depth = t.depth(a.parent ? in : 0);
            const int at = a.kv_len + (a.parent ? depth : in);
#pragma unroll
            for (int e = 0; e < 2; ++e) {
                const double freq = exp2(-2.0 / D * log2((double)a.rope_base) * (2 * i + e));
                double s, c;
                sincos((double)at * freq, &s, &c);
                cs[j][e] = (float)c;
                sn[j][e] = (float)s;
            }
        }
    }
    auto rotate = [&](half2_& lo, half2_& hi, int j) {
#pragma clang fp contract(off)
#pragma unroll
        for (int e = 0; e < 2; ++e) {
            const float x = (float)lo[e], y = (float)hi[e];
            lo[e] = (half_t)(x * cs[j][e] - y * sn[j][e]);
            hi[e] = (half_t)(y * cs[j][e] + x * sn[j][e]);
        }
    };
    for (int head = head0; head < head1; ++head) {
        if (head >= a.nkv) {                                  // a query head
            const int h = head - a.nkv;
#pragma unroll
            for (int j = 0; j < kRows; ++j) {
                const int row = row0 + set * kRows + j;
                if (row < 0 || row >= a.M) continue;
                const half_t* src = a.q + (size_t)row * a.ld_q + h * D + 2 * i;
                half_t* dst = a.q_out + (size_t)row * a.ld_qo + h * D + 2 * i;
                half2_ lo = *(const half2_*)src, hi = *(const half2_*)(src + D / 2);
                rotate(lo, hi, j);
                *(half2_*)dst = lo;
                *(half2_*)(dst + D / 2) = hi;
            }
            continue;
        }
        const size_t tile = q4_tile_at(head, octet / 4, a.tiles, D);
        const int in_tile = octet % 4 * 8;
        {   // keys
            char* kt = a.k + tile;
            half2_ x[kRows][2];
#pragma unroll
            for (int j = 0; j < kRows; ++j) {
                const int row = min(max(row0 + set * kRows + j, 0), a.M - 1);
                const half_t* src = a.kx + (size_t)row * a.ld_k + head * D + 2 * i;
                x[j][0] = *(const half2_*)src;
                x[j][1] = *(const half2_*)(src + D / 2);
            }
#pragma unroll
            for (int j = 0; j < kRows; ++j) {
                const int row = row0 + set * kRows + j, key = in_tile + set * kRows + j;
                const bool in = row >= 0 && row < a.M;
                if (turn) rotate(x[j][0], x[j][1], j);
#pragma unroll
                for (int u = 0; u < 2; ++u) {
                    const Group g = quantise(x[j][u]);
                    uint32_t w = (g.c0 | g.c1 << 16) << 4 * (i & 3);      // a word: four lanes
                    w |= dpp<kXor1>(w);
                    w |= dpp<kXor2>(w);
                    const int c = 2 * i + u * (D / 2);
                    if (in && (i & 3) == 0) *(uint32_t*)(kt + key * (D / 2) + c / 2) = w;
                    if (in && (i & 15) == 0)
                        *(half2_*)(kt + q4_codes_bytes(D) + (key * (D / 32) + c / 32) * 4) = (half2_){g.lo, g.s};
                }
            }
        }
        {   // values: 64 lanes hold a row of 128 channels, or two halves of the octet of 64
            char* vt = a.v + tile;
            constexpr int kHalves = 128 / D, kKeys = 8 / kHalves;
            const int c = 2 * (lane % (D / 2)), k0 = lane / (D / 2) * kKeys;
            half2_ x[kKeys];
#pragma unroll
            for (int j = 0; j < kKeys; ++j) {
                const int row = min(max(row0 + k0 + j, 0), a.M - 1);
                x[j] = *(const half2_*)(a.vx + (size_t)row * a.ld_v + head * D + c);
            }
            uint32_t w0 = 0, w1 = 0, held = 0;                // words of channels c, c + 1; bits of rows that are held already
            half_t* meta = (half_t*)(vt + q4_codes_bytes(D)) + c / 32 * 64;
#pragma unroll
            for (int j = 0; j < kKeys; ++j) {
                const int k = k0 + j, row = row0 + k, at = 4 * (k / 2) + 16 * (k % 2);
                const Group g = quantise(x[j]);
                if (row >= 0 && row < a.M) {
                    w0 |= g.c0 << at;
                    w1 |= g.c1 << at;
                    if ((lane & 15) == 0) {
                        meta[in_tile + k] = g.lo;
                        meta[32 + in_tile + k] = g.s;
                    }
                } else {
                    held |= 15u << at;
                }
            }
            if constexpr (kHalves == 2) {
                w0 |= (uint32_t)__shfl_xor((int)w0, 32);
                w1 |= (uint32_t)__shfl_xor((int)w1, 32);
                held |= (uint32_t)__shfl_xor((int)held, 32);
            }
            if (k0 == 0) {
                uint32_t* p0 = (uint32_t*)vt + q4_v_word(c, octet % 4);
                uint32_t* p1 = (uint32_t*)vt + q4_v_word(c + 1, octet % 4);
                if (held) {
                    w0 |= *p0 & held;
                    w1 |= *p1 & held;
                }
                *p0 = w0;
                *p1 = w1;
            }
        }
    }
}

ghd_status launch_q4_append(const Q4Append& a, int d, hipStream_t st)
{
    const int octets = (a.kv_len + a.M - 1) / 8 - a.kv_len / 8 + 1, heads = a.nkv + a.nq;
    // one head a wavefront where that is at most 4096 wavefronts; above that, runs of heads, which share cosines
    const int per = (int)std::min<int64_t>(heads, std::max<int64_t>(1, (int64_t)octets * heads / 4096));
    const int chunks = ceil_div(heads, per), units = octets * chunks;
    const dim3 grid(ceil_div(units, 4));
    if (d == 128) hipLaunchKernelGGL(k_q4_append<128>, grid, dim3(256), 0, st, a, chunks, per, units);
    else hipLaunchKernelGGL(k_q4_append<64>, grid, dim3(256), 0, st, a, chunks, per, units);
    return check_launch();
}

// ---- commit ------------------------------------------------------------------------------
struct Q4Layers {
    char *k[kQ4MaxLayers], *v[kQ4MaxLayers];
};

// One wavefront a (layer, head, K or V).  The path's rows are taken eight at a time, all read before the first is written;
// rows come from behind where they go (path[j] >= j), so a later eight's are still as they were.
// Bound: latency, two trips to memory one behind the other.
template <int D>
__global__ __launch_bounds__(256) void k_q4_commit(const Q4Layers a, int L, int nkv, int tiles, int kv_len, int M,
                                                   const int32_t* res)
{
    const int lane = threadIdx.x & 63, unit = blockIdx.x * 4 + (threadIdx.x >> 6);
    if (unit >= L * nkv * 2) return;
    const bool is_v = unit & 1;
    const int head = unit / 2 % nkv, layer = unit / 2 / nkv;
    const int len = min(max(res[0], 0), M);
    char* base = (is_v ? a.v[layer] : a.k[layer]) + q4_tile_at(head, 0, tiles, D);
    constexpr int kBatch = 8;
    for (int j0 = 0; j0 < len; j0 += kBatch) {
        const int n = min(kBatch, len - j0);
        const int mine = min(max(res[2 + j0 + min(lane & 7, n - 1)], 0), M - 1);    // lane j: where the batch's row j comes from
        if (__ballot(mine != j0 + min(lane & 7, n - 1)) == 0) continue;             // all where they belong
        if (!is_v) {
            constexpr int kWords = D / 8;                // of codes; D / 32 of (lo, scale) follow
            uint32_t got[kBatch];
            const int w = min(lane, kWords + D / 32 - 1);
            auto at = [&](int row) {
                char* t = base + (size_t)(row >> 5) * q4_tile_bytes(D);
                row &= 31;
                return (uint32_t*)(w < kWords ? t + row * (D / 2) + w * 4 : t + q4_codes_bytes(D) + (row * (D / 32) + w - kWords) * 4);
            };
#pragma unroll
            for (int j = 0; j < kBatch; ++j)
                if (j < n) got[j] = *at(kv_len + __builtin_amdgcn_readlane(mine, j));
#pragma unroll
            for (int j = 0; j < kBatch; ++j)
                if (j < n && lane < kWords + D / 32) *at(kv_len + j0 + j) = got[j];
            continue;
        }
        // the words of the one or two octets that the batch goes to, of up to two channels a lane
        const int to = kv_len + j0, o0 = to >> 3, o1 = (to + n - 1) >> 3;
        constexpr int kCh = D / 64;
        auto word = [&](int octet, int u) {
            return (uint32_t*)(base + (size_t)(octet >> 2) * q4_tile_bytes(D)) + q4_v_word(lane + 64 * u, octet & 3);
        };
        uint32_t src[kBatch][kCh], dst[2][kCh];
#pragma unroll
        for (int u = 0; u < kCh; ++u) {
            dst[0][u] = *word(o0, u);
            dst[1][u] = *word(o1, u);
#pragma unroll
            for (int j = 0; j < kBatch; ++j)
                if (j < n) src[j][u] = *word((kv_len + __builtin_amdgcn_readlane(mine, j)) >> 3, u);
        }
        // lo and scale: lane (row of the batch, group, which)
        constexpr int kMeta = D / 32 * 2;
        const int mj = lane / kMeta, part = lane % kMeta;
        auto meta = [&](int row) {
            return (half_t*)(base + (size_t)(row >> 5) * q4_tile_bytes(D) + q4_codes_bytes(D)) + part * 32 + (row & 31);
        };
        const int from = __shfl(mine, mj & 7);
        half_t held = 0;
        if (mj < n) held = *meta(kv_len + from);
#pragma unroll
        for (int j = 0; j < kBatch; ++j) {
            if (j >= n) break;
            const int r = (kv_len + __builtin_amdgcn_readlane(mine, j)) & 7, t = to + j;
            const int sr = 4 * (r / 2) + 16 * (r % 2), sl = 4 * ((t & 7) / 2) + 16 * (t & 1);
            const bool second = (t >> 3) != o0;
#pragma unroll
            for (int u = 0; u < kCh; ++u) {
                const uint32_t code = (src[j][u] >> sr & 15u) << sl, keep = ~(15u << sl);
                if (second) dst[1][u] = (dst[1][u] & keep) | code;
                else dst[0][u] = (dst[0][u] & keep) | code;
            }
        }
#pragma unroll
        for (int u = 0; u < kCh; ++u) {
            *word(o0, u) = dst[0][u];
            if (o1 != o0) *word(o1, u) = dst[1][u];
        }
        if (mj < n) *meta(to + mj) = held;
    }
}

static Q4Layers layers_of(void* const* k, void* const* v, int L)
{
    Q4Layers a = {};
    for (int l = 0; l < L; ++l) {
        a.k[l] = (char*)k[l];
        a.v[l] = (char*)v[l];
    }
    return a;
}

ghd_status launch_q4_commit(void* const* k, void* const* v, int L, int nkv, int d, int cap, int kv_len, int M,
                            const int32_t* res, hipStream_t st)
{
    const Q4Layers a = layers_of(k, v, L);
    const dim3 grid(ceil_div(L * nkv * 2, 4));
    if (d == 128) hipLaunchKernelGGL(k_q4_commit<128>, grid, dim3(256), 0, st, a, L, nkv, cap / kQ4Tile, kv_len, M, res);
    else hipLaunchKernelGGL(k_q4_commit<64>, grid, dim3(256), 0, st, a, L, nkv, cap / kQ4Tile, kv_len, M, res);
    return check_launch();
}

// ---- reading back ------------------------------------------------------------------------
// A wavefront reads one octet of a (layer, head), K and V, and writes rows of fp16.  Bound: the bytes written.
template <int D>
__global__ __launch_bounds__(256) void k_q4_read(const Q4Layers a, int nkv, int tiles, int octets, int row0, int rows,
                                                 half_t* ko, half_t* vo, int64_t units)
{
    const int lane = threadIdx.x & 63;
    const int64_t unit = (int64_t)blockIdx.x * 4 + (threadIdx.x >> 6);
    if (unit >= units) return;
    const int head = unit % nkv, octet = row0 / 8 + (int)(unit / nkv % octets), layer = (int)(unit / nkv / octets);
    const size_t tile = q4_tile_at(head, octet / 4, tiles, D);
    const int in_tile = octet % 4 * 8, first = octet * 8 - row0;         // output row of the octet's first key
    const size_t out0 = (size_t)layer * rows * nkv * D + (size_t)head * D;
    const int64_t step = (int64_t)nkv * D;
    const char* kt = a.k[layer] + tile;
    const Q4Bits bits;
#pragma unroll
    for (int u = 0; u < D / 64; ++u) {                                   // 8 rows of D / 8 words
        const int e = lane + 64 * u, key = e / (D / 8), w = e % (D / 8), row = first + key;
        const uint32_t word = *(const uint32_t*)(kt + (in_tile + key) * (D / 2) + w * 4);
        const half2_ m = *(const half2_*)(kt + q4_codes_bytes(D) + ((in_tile + key) * (D / 32) + w / 4) * 4);
        if (row >= 0 && row < rows)
            *(half8*)(ko + out0 + row * step + w * 8) = q4_values(bits, word, pair_of(m[0]), pair_of(m[1]));
    }
    const char* vt = a.v[layer] + tile;
    constexpr int kHalves = 128 / D, kKeys = 8 / kHalves;
    const int c = 2 * (lane % (D / 2)), k0 = lane / (D / 2) * kKeys;
    const half_t* meta = (const half_t*)(vt + q4_codes_bytes(D)) + c / 32 * 64 + in_tile;
    const half8 lo = *(const half8*)meta, s = *(const half8*)(meta + 32);
    half2_ l2[4], s2[4];
#pragma unroll
    for (int p = 0; p < 4; ++p) {
        l2[p] = (half2_){lo[2 * p], lo[2 * p + 1]};
        s2[p] = (half2_){s[2 * p], s[2 * p + 1]};
    }
    const half8 x0 = q4_values(bits, ((const uint32_t*)vt)[q4_v_word(c, octet % 4)], l2, s2);
    const half8 x1 = q4_values(bits, ((const uint32_t*)vt)[q4_v_word(c + 1, octet % 4)], l2, s2);
#pragma unroll
    for (int j = 0; j < 8; ++j) {
        const int row = first + j;
        if (j / kKeys == k0 / kKeys && row >= 0 && row < rows)
            *(half2_*)(vo + out0 + row * step + c) = (half2_){x0[j], x1[j]};
    }
}

ghd_status launch_q4_read(void* const* k, void* const* v, int L, int nkv, int d, int cap, int row0, int rows, half_t* ko,
                          half_t* vo, hipStream_t st)
{
    const Q4Layers a = layers_of(k, v, L);
    const int octets = (row0 + rows - 1) / 8 - row0 / 8 + 1;
    const int64_t units = (int64_t)L * nkv * octets;
    const dim3 grid((uint32_t)((units + 3) / 4));
    if (d == 128)
        hipLaunchKernelGGL(k_q4_read<128>, grid, dim3(256), 0, st, a, nkv, cap / kQ4Tile, octets, row0, rows, ko, vo, units);
    else
        hipLaunchKernelGGL(k_q4_read<64>, grid, dim3(256), 0, st, a, nkv, cap / kQ4Tile, octets, row0, rows, ko, vo, units);
    return check_launch();
}

}  // namespace ghd
