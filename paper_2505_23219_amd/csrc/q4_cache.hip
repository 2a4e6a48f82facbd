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
typedef word4 word4_at4 __attribute__((aligned(4)));       // rows of the caller's may begin at any word

template <int CTRL>
__device__ __forceinline__ uint32_t dpp(uint32_t x)
{
    return (uint32_t)__builtin_amdgcn_update_dpp(0, (int)x, CTRL, 0xf, 0xf, true);
}
constexpr int kXor1 = 0xB1, kXor2 = 0x4E, kXor8 = 0x128;   // exchanges inside 4, 4 and 16 lanes (the last turns 16 by 8)

struct Group {
    half_t lo, s;
    uint32_t codes;        // of this lane's 8 channels, as a word of q4.h
};

// x: this lane's 8 channels of a group that four lanes side by side hold
__device__ __forceinline__ Group quantise(half8 x)
{
#pragma clang fp contract(off)
    const word4 bits = __builtin_bit_cast(word4, x);
    half2_ least = {x[0], x[1]}, most = least;
    uint32_t odd = 0;      // an infinity or NaN: an exponent of all ones, plus one, carries into the sign
#pragma unroll
    for (int p = 0; p < 4; ++p) {
        const half2_ v = {x[2 * p], x[2 * p + 1]};
        least = __builtin_elementwise_min(least, v);
        most = __builtin_elementwise_max(most, v);
        odd |= (bits[p] & 0x7c007c00u) + 0x04000400u;
    }
    odd &= 0x80008000u;
    // (min x, min -x), of the lane, then of the four
    half2_ m = {__builtin_elementwise_min(least[0], least[1]), -__builtin_elementwise_max(most[0], most[1])};
    m = __builtin_elementwise_min(m, __builtin_bit_cast(half2_, dpp<kXor1>(__builtin_bit_cast(uint32_t, m))));
    m = __builtin_elementwise_min(m, __builtin_bit_cast(half2_, dpp<kXor2>(__builtin_bit_cast(uint32_t, m))));
    odd |= dpp<kXor1>(odd);
    odd |= dpp<kXor2>(odd);
    Group g;
    g.lo = m[0];
    const float lo = (float)m[0];
    g.s = (half_t)((-(float)m[1] - lo) / 15.f);
    // rounded up, the scale of the widest ranges would make the largest code stand for more than fp16 holds
    if (lo + 15.f * (float)g.s >= 65520.f)
        g.s = __builtin_bit_cast(half_t, (uint16_t)(__builtin_bit_cast(uint16_t, g.s) - 1));
    const float s = (float)g.s;
    // (x - lo) / s by a reciprocal, which is off by less than 1e-5; where a quotient is that near to the middle of two codes for any
    // lane, by divisions (a division is ten instructions, and there are 16 a lane and row)
    float code[8];
    const float r = __builtin_amdgcn_rcpf(s);
    bool near = false;
#pragma unroll
    for (int j = 0; j < 8; ++j) {
        const float t = ((float)x[j] - lo) * r;
        code[j] = rintf(t);
        near = near || fabsf(t - code[j]) > 0.49998f;
    }
    if (__ballot(near && s > 0.f))
#pragma unroll
        for (int j = 0; j < 8; ++j) code[j] = rintf(((float)x[j] - lo) / s);
    g.codes = 0;
#pragma unroll
    for (int j = 0; j < 8; ++j) g.codes |= (uint32_t)fminf(code[j], 15.f) << (4 * (j / 2) + 16 * (j % 2));
    if (!(s > 0.f)) g.codes = 0;
    if (odd) {             // a group with an infinity or NaN in it reads as NaN
        g.s = __builtin_bit_cast(half_t, (uint16_t)0x7e00);
        g.codes = 0;
    }
    return g;
}

// A word of every lane (key k = lane / 8) has 8 channels; afterwards lane 8 c + i has channel c's 8 keys.  Key bit 0 changes
// places with the half a code is in, bit 1 with its lowest and bit 2 with its next place among four.
__device__ __forceinline__ uint32_t keys_of_channel(uint32_t w, int lane)
{
    uint32_t other = dpp<kXor8>(w);
    w = lane & 8 ? other >> 16 | (w & 0xffff0000u) : (w & 0xffffu) | other << 16;
    other = (uint32_t)__shfl_xor((int)w, 16);
    w = lane & 16 ? (other >> 4 & 0x0f0f0f0fu) | (w & 0xf0f0f0f0u) : (w & 0x0f0f0f0fu) | (other & 0x0f0f0f0fu) << 4;
    other = (uint32_t)__shfl_xor((int)w, 32);
    return lane & 32 ? (other >> 8 & 0x00ff00ffu) | (w & 0xff00ff00u) : (w & 0x00ff00ffu) | (other & 0x00ff00ffu) << 8;
}

// ---- append ------------------------------------------------------------------------------
// A wavefront takes the octet of a head (of two heads of 64 channels) at a time: lane 8 k + i has of key k channels 8 i .. + 7 and
// those half a row further, which turn with them: two 16-byte requests, and a word of K codes, each.  The workgroup's
// four wavefronts have one octet, whose cosines and sines, worked out in 64 bits, they share through LDS (worked out by every
// wavefront for itself the smallest call took 9 us, 4096 rows of 32 + 8 heads 47).
// Bound: for a tree's rows latency - parents, cosines, rows, one behind the other (64 rows of 32 heads and 32 key heads 7 us); for a
// prompt the bytes (4096 rows of 32 and 8 heads 23 us for 89 MB, 3.9 TB/s; a copy reaches 4.75).
template <int D>
__global__ __launch_bounds__(256) void k_q4_append(const Q4Append a, int chunks, int per_chunk)
{
    constexpr int kHeads = 128 / D, kHalf = D / 2;
    __shared__ float2 s_turn[8][kHalf];
    const int tid = threadIdx.x, lane = tid & 63, wave = tid >> 6, key = lane >> 3;
    const int i = D == 128 ? lane & 7 : lane & 3, second = D == 128 ? 0 : lane >> 2 & 1;     // (the second of two heads)
    const int octet = a.kv_len / 8 + blockIdx.x / chunks, row0 = octet * 8 - a.kv_len;       // row0: input row of the first key
    const int kv_items = (a.nkv + kHeads - 1) / kHeads, items = kv_items + (a.nq + kHeads - 1) / kHeads;
    const int first = blockIdx.x % chunks * per_chunk, end = min(first + per_chunk, items);
    const int row = row0 + key, row_in = min(max(row, 0), a.M - 1);
    const bool in = row >= 0 && row < a.M;
    struct Rows {
        half8 x[2], v[2];
    };
    auto load = [&](Rows& r, int item) {
        item = min(item, end - 1);
        const bool is_q = item >= kv_items;
        const int head = min((is_q ? item - kv_items : item) * kHeads + second, (is_q ? a.nq : a.nkv) - 1);
        const half_t* x = (is_q ? a.q + (int64_t)row_in * a.ld_q : a.kx + (int64_t)row_in * a.ld_k) + head * D + 8 * i;
        r.x[0] = __builtin_bit_cast(half8, *(const word4_at4*)x);
        r.x[1] = __builtin_bit_cast(half8, *(const word4_at4*)(x + kHalf));
        if (!is_q) {
            const half_t* v = a.vx + (int64_t)row_in * a.ld_v + head * D + 8 * i;
            r.v[0] = __builtin_bit_cast(half8, *(const word4_at4*)v);
            r.v[1] = __builtin_bit_cast(half8, *(const word4_at4*)(v + kHalf));
        }
    };
    Rows r;
    load(r, first + wave);
    const bool turn = a.rope_base > 0.f;
    float2 cs[8];
    if (turn) {
        int depth = 0;
        if (a.parent) {
            const TreeNodes<2> t =
                tree_nodes<2, false>(a.parent[min(lane, a.M - 1)], a.parent[min(lane + 64, a.M - 1)], a.M, lane);
            depth = t.depth(min(max(row0 + (lane & 7), 0), a.M - 1));          // lane k: of the octet's key k
        }
        // entry (key, j) by thread; a wavefront's entries are of one key, or of two
#pragma unroll
        for (int e = tid; e < 8 * kHalf; e += 256) {
            const int k = e / kHalf, j = e % kHalf, from = row0 + k;
            const int at = a.kv_len + (a.parent ? __shfl(depth, k) : from);
            if (from < 0 || from >= a.M) continue;
            double s, c;
            sincos((double)at * exp2(a.log2_step * j), &s, &c);
            s_turn[k][j] = make_float2((float)c, (float)s);
        }
        __syncthreads();
#pragma unroll
        for (int j = 0; j < 8; ++j) cs[j] = s_turn[key][8 * i + j];
    }
    auto rotate = [&](Rows& w) {
#pragma clang fp contract(off)
#pragma unroll
        for (int j = 0; j < 8; ++j) {
            const float x = (float)w.x[0][j], y = (float)w.x[1][j];
            w.x[0][j] = (half_t)(x * cs[j].x - y * cs[j].y);
            w.x[1][j] = (half_t)(y * cs[j].x + x * cs[j].y);
        }
    };
    auto store = [&](Rows& w, int item) {
        const bool is_q = item >= kv_items;
        const int head = (is_q ? item - kv_items : item) * kHeads + second;
        if (turn) rotate(w);
        if (is_q) {
            if (!in || head >= a.nq) return;
            half_t* to = a.q_out + (int64_t)row * a.ld_qo + head * D + 8 * i;
            *(word4_at4*)to = __builtin_bit_cast(word4, w.x[0]);
            *(word4_at4*)(to + kHalf) = __builtin_bit_cast(word4, w.x[1]);
            return;
        }
        const bool there = head < a.nkv;
        const size_t tile = q4_tile_at(min(head, a.nkv - 1), octet / 4, a.tiles, D);
        const int in_tile = octet % 4 * 8;
        char *kt = a.k + tile, *vt = a.v + tile;
        half_t* meta = (half_t*)(vt + q4_codes_bytes(D));
        uint32_t held = 0;                                       // codes of rows that are not this call's
#pragma unroll
        for (int k = 0; k < 8; ++k)
            if (row0 + k < 0 || row0 + k >= a.M) held |= 15u << (4 * (k / 2) + 16 * (k % 2));
#pragma unroll
        for (int u = 0; u < 2; ++u) {
            const int c = u * kHalf + 8 * i;
            const Group gk = quantise(w.x[u]);
            if (in && there) {
                *(uint32_t*)(kt + (in_tile + key) * (D / 2) + c / 2) = gk.codes;
                if ((i & 3) == 0) *(half2_*)(kt + q4_codes_bytes(D) + ((in_tile + key) * (D / 32) + c / 32) * 4) = (half2_){gk.lo, gk.s};
            }
            const Group gv = quantise(w.v[u]);
            if (in && there && (i & 3) == 0) {
                meta[c / 32 * 64 + in_tile + key] = gv.lo;
                meta[c / 32 * 64 + 32 + in_tile + key] = gv.s;
            }
            uint32_t word = keys_of_channel(gv.codes, lane);     // now of channel u kHalf + 8 i + key
            uint32_t* to = (uint32_t*)vt + q4_v_word(c + key, octet % 4);
            if (there) {
                if (held) word = (word & ~held) | (*to & held);
                *to = word;
            }
        }
    };
    // (two in turn: a copy of the one on its way would have to wait for it)
    Rows next;
    for (int item = first + wave; item < end; item += 8) {
        load(next, item + 4);
        store(r, item);
        if (item + 4 >= end) break;
        load(r, item + 8);
        store(next, item + 4);
    }
}

ghd_status launch_q4_append(Q4Append a, int d, hipStream_t st)
{
    a.log2_step = -2.0 / d * log2((double)(a.rope_base > 0.f ? a.rope_base : 1.f));
    const int heads = 128 / d, octets = (a.kv_len + a.M - 1) / 8 - a.kv_len / 8 + 1;
    const int items = ceil_div(a.nkv, heads) + ceil_div(a.nq, heads);
    // an item a wavefront where that is at most 1024 workgroups; above that runs of them, which share cosines
    const int per = (int)std::min<int64_t>(align_up(items, 4), 4 * std::max<int64_t>(1, (int64_t)octets * items / 4096));
    const int chunks = ceil_div(items, per);
    const dim3 grid(octets * chunks);
    if (d == 128) hipLaunchKernelGGL(k_q4_append<128>, grid, dim3(256), 0, st, a, chunks, per);
    else hipLaunchKernelGGL(k_q4_append<64>, grid, dim3(256), 0, st, a, chunks, per);
    return check_launch();
}

// ---- commit ------------------------------------------------------------------------------
struct Q4Layers {
    char *k[kQ4MaxLayers], *v[kQ4MaxLayers];
};

// One wavefront a (layer, head, K or V).  The path's rows are taken eight at a time, all read before the first is written;
// rows come from behind where they go (path[j] >= j), so a later eight's are still as they were.
// Bound: latency, two trips to memory one behind the other: 4 rows of 32 heads in 32 layers 4.8 us.
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
// A wavefront reads one octet of a (layer, head), K and V, and writes rows of fp16.  Bound: the bytes written (64 rows of 32
// heads in 32 layers, 34 MB, 10.5 us), for fewer a launch (3.2 us).
template <int D>
__global__ __launch_bounds__(256) void k_q4_read(const Q4Layers a, int nkv, int tiles, int octets, int row0, int rows,
                                                 half_t* ko, half_t* vo, int64_t unit0, int64_t units)
{
    const int lane = threadIdx.x & 63;
    const int64_t unit = unit0 + blockIdx.x * 4 + (threadIdx.x >> 6);
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
    for (int64_t unit0 = 0; unit0 < units; unit0 += 4 * kQ4MostGroups) {
        const dim3 grid((uint32_t)std::min<int64_t>(kQ4MostGroups, (units - unit0 + 3) / 4));
        if (d == 128)
            hipLaunchKernelGGL(k_q4_read<128>, grid, dim3(256), 0, st, a, nkv, cap / kQ4Tile, octets, row0, rows, ko, vo, unit0, units);
        else
            hipLaunchKernelGGL(k_q4_read<64>, grid, dim3(256), 0, st, a, nkv, cap / kQ4Tile, octets, row0, rows, ko, vo, unit0, units);
        const ghd_status s = check_launch();
        if (s) return s;
    }
    return GHD_OK;
}

}  // namespace ghd
