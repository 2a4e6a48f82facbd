// Attention of the drafted tokens over a 4-bit cache.
//
// out[i, h] = softmax over the keys that node i sees of (scale q . K^) applied to V^, where K^ and V^ are the fp16
// numbers that the codes stand for (q4.h).  A key head's query rows - M nodes by nh / nkv heads - are the columns of
// S^T = K^ q^T and O^T = V^T P^T, so softmax statistics are a lane's own and the probabilities come out as the operand of
// the second product.  A wavefront takes 32 keys at a time by itself: 32 bytes of codes a lane, turned into fp16 operands in
// registers; running maximum and sum in 32 bits, probabilities rounded to fp16 (they are at most 1).
#include "q4.h"
#include "attention_impl.h"

namespace ghd {

constexpr int kQ4Waves = 4;

typedef uint32_t word2 __attribute__((ext_vector_type(2)));
typedef uint32_t word4 __attribute__((ext_vector_type(4)));

// the bits of a node's mask for the 32 keys from `base` on, counted from the first drafted row; keys
// before that are committed, and seen
__device__ __forceinline__ uint32_t q4_mask32(uint64_t lo, uint64_t hi, int base)
{
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

template <int D, int MT>
__global__ __launch_bounds__(kQ4Waves * 64) void k_q4_attention(const Q4Attn a, int splits, int blocks)
{
    constexpr int CT = D / 16, KS = D / 32;
    __shared__ uint64_t s_mask[2 * GHD_MAX_M];
    extern __shared__ __attribute__((aligned(16))) char lds[];
    const int lane = threadIdx.x & 63, wave = threadIdx.x >> 6, col = lane & 15, g = lane >> 4;
    const int split = blockIdx.x % splits, block = blockIdx.x / splits % blocks, head = blockIdx.x / splits / blocks;
    const int rep = a.nh / a.nkv, R = a.M * rep, total = a.kv_len + a.M;
    const int ntiles = (total + kQ4Tile - 1) / kQ4Tile;
    const int t0 = (int)((int64_t)ntiles * split / splits), t1 = (int)((int64_t)ntiles * (split + 1) / splits);
    if (t1 * kQ4Tile > a.kv_len) {                     // masks are looked at
        if (a.mask) {
            if ((int)threadIdx.x < 2 * a.M) {
                const int w = threadIdx.x & 1, left = a.M - 64 * w;      // bits of this word that mean something
                const uint64_t m = a.mask[threadIdx.x];
                s_mask[threadIdx.x] = left >= 64 ? m : left <= 0 ? 0 : m & ((1ull << left) - 1);
            }
        } else if (threadIdx.x < 64) {
            store_masks(tree_nodes<2, true>(a.parent[min(lane, a.M - 1)], a.parent[min(lane + 64, a.M - 1)], a.M, lane),
                        a.M, lane, s_mask);
        }
        __syncthreads();
    }
    half8 q[KS][MT];
    int node[MT];
#pragma unroll
    for (int mt = 0; mt < MT; ++mt) {
        const int row = block * 16 * MT + mt * 16 + col;
        const bool in = row < R;
        node[mt] = in ? row / rep : 0;
        const half_t* qr = a.q + ((size_t)node[mt] * a.nh + head * rep + (in ? row - node[mt] * rep : 0)) * D + g * (D / 4);
#pragma unroll
        for (int s = 0; s < KS; ++s) {
            q[s][mt] = (half8){0, 0, 0, 0, 0, 0, 0, 0};
            if (in) q[s][mt] = *(const half8*)(qr + 8 * s);
        }
    }
    const Q4Bits bits;
    const float c = a.scale * 1.4426950408889634f;
    floatx4 o[CT][MT];
    float m[MT], l[MT];
#pragma unroll
    for (int mt = 0; mt < MT; ++mt) {
        m[mt] = -INFINITY;
        l[mt] = 0.f;
#pragma unroll
        for (int ct = 0; ct < CT; ++ct) o[ct][mt] = (floatx4){0.f, 0.f, 0.f, 0.f};
    }
    const char* kh = a.k + q4_tile_at(head, 0, a.tiles, D);
    const char* vh = a.v + q4_tile_at(head, 0, a.tiles, D);
    for (int t = t0 + wave; t < t1; t += kQ4Waves) {
        const char* kt = kh + (size_t)t * q4_tile_bytes(D);
        const char* vt = vh + (size_t)t * q4_tile_bytes(D);
        // K: operand row r of half h is key 8 (r / 4) + 4 h + r % 4, so that a lane's 8 scores of a column are
        // those of keys 8 g .. 8 g + 7, the probabilities it holds in the second product
        uint32_t kw[2][KS];
        half2_ km[2];
#pragma unroll
        for (int h = 0; h < 2; ++h) {
            const int key = 8 * (col >> 2) + 4 * h + (col & 3);
            if constexpr (D == 128) {
                const word4 w = *(const word4*)(kt + key * 64 + g * 16);
#pragma unroll
                for (int s = 0; s < KS; ++s) kw[h][s] = w[s];
                km[h] = *(const half2_*)(kt + q4_codes_bytes(D) + (key * 4 + g) * 4);
            } else {
                const word2 w = *(const word2*)(kt + key * 32 + g * 8);
#pragma unroll
                for (int s = 0; s < KS; ++s) kw[h][s] = w[s];
                km[h] = *(const half2_*)(kt + q4_codes_bytes(D) + (key * 2 + (g >> 1)) * 4);
            }
        }
        word4 vw[CT / 4];
        half8 vlo[CT / 2], vs[CT / 2];
#pragma unroll
        for (int i = 0; i < CT / 4; ++i) vw[i] = *(const word4*)(vt + ((i * 4 + g) * 16 + col) * 16);
#pragma unroll
        for (int i = 0; i < CT / 2; ++i) {
            vlo[i] = *(const half8*)(vt + q4_codes_bytes(D) + i * 128 + g * 16);
            vs[i] = *(const half8*)(vt + q4_codes_bytes(D) + i * 128 + 64 + g * 16);
        }
        floatx4 s[2][MT];
#pragma unroll
        for (int h = 0; h < 2; ++h) {
#pragma unroll
            for (int mt = 0; mt < MT; ++mt) s[h][mt] = (floatx4){0.f, 0.f, 0.f, 0.f};
#pragma unroll
            for (int k = 0; k < KS; ++k) {
                const half8 ka = q4_values(bits, kw[h][k], pair_of(km[h][0]), pair_of(km[h][1]));
#pragma unroll
                for (int mt = 0; mt < MT; ++mt)
                    s[h][mt] = __builtin_amdgcn_mfma_f32_16x16x32_f16(ka, q[k][mt], s[h][mt], 0, 0, 0);
            }
        }
        const int base = t * kQ4Tile - a.kv_len;
        const bool masked = base + kQ4Tile > 0;
        uint32_t see[MT];
        uint32_t nan_keys = 0;       // keys of this lane (bit 8 i + key) whose lo or scale of group i is no number
        if (masked) {
#pragma unroll
            for (int mt = 0; mt < MT; ++mt)
                see[mt] = q4_mask32(s_mask[2 * node[mt]], s_mask[2 * node[mt] + 1], base) >> 8 * g & 255u;
            // Values of rows that are not there may be anything, and 0 times anything is no 0: they count as 0, and so
            // does what reads as NaN (a NaN was appended), which only reaches the rows that see it, below.
#pragma unroll
            for (int i = 0; i < CT / 2; ++i)
#pragma unroll
                for (int e = 0; e < 8; ++e) {
                    const bool there = t * kQ4Tile + 8 * g + e < total;
                    const bool number = (__builtin_bit_cast(uint16_t, (half_t)vlo[i][e]) & 0x7c00u) != 0x7c00u &&
                                        (__builtin_bit_cast(uint16_t, (half_t)vs[i][e]) & 0x7c00u) != 0x7c00u;
                    if (there && !number) nan_keys |= 1u << (8 * i + e);
                    if (!there || !number) vlo[i][e] = vs[i][e] = 0;
                }
        }
        half8 p[MT];
#pragma unroll
        for (int mt = 0; mt < MT; ++mt) {
            float v[8], top = -INFINITY;
#pragma unroll
            for (int e = 0; e < 8; ++e) {
                v[e] = s[e >> 2][mt][e & 3] * c;
                if (masked && !(see[mt] >> e & 1)) v[e] = -INFINITY;
                top = fmaxf(top, v[e]);
            }
            top = max_over_groups(top);
            if (top > m[mt]) {       // (the same in the four lanes of a column)
                const float r = __builtin_amdgcn_exp2f(m[mt] - top);
                l[mt] *= r;
#pragma unroll
                for (int ct = 0; ct < CT; ++ct) o[ct][mt] *= r;
                m[mt] = top;
            }
            const float off = m[mt] == -INFINITY ? 0.f : m[mt];
#pragma unroll
            for (int e = 0; e < 8; ++e) {
                const float x = __builtin_amdgcn_exp2f(v[e] - off);
                l[mt] += x;
                p[mt][e] = (half_t)x;
            }
        }
#pragma unroll
        for (int ct = 0; ct < CT; ++ct) {
            half2_ lo[4], sc[4];
#pragma unroll
            for (int e = 0; e < 4; ++e) {
                lo[e] = (half2_){vlo[ct / 2][2 * e], vlo[ct / 2][2 * e + 1]};
                sc[e] = (half2_){vs[ct / 2][2 * e], vs[ct / 2][2 * e + 1]};
            }
            const half8 va = q4_values(bits, vw[ct / 4][ct % 4], lo, sc);
#pragma unroll
            for (int mt = 0; mt < MT; ++mt)
                o[ct][mt] = __builtin_amdgcn_mfma_f32_16x16x32_f16(va, p[mt], o[ct][mt], 0, 0, 0);
        }
        if (masked && __ballot(nan_keys != 0)) {
            // how many keys with a NaN in this channel's group a row sees: a product of ones
#pragma unroll
            for (int i = 0; i < CT / 2; ++i) {
                half8 bad;
#pragma unroll
                for (int e = 0; e < 8; ++e) bad[e] = nan_keys >> (8 * i + e) & 1 ? (half_t)1.f : (half_t)0.f;
#pragma unroll
                for (int mt = 0; mt < MT; ++mt) {
                    half8 sees;
#pragma unroll
                    for (int e = 0; e < 8; ++e) sees[e] = see[mt] >> e & 1 ? (half_t)1.f : (half_t)0.f;
                    const floatx4 n = __builtin_amdgcn_mfma_f32_16x16x32_f16(bad, sees, (floatx4){0.f, 0.f, 0.f, 0.f}, 0, 0, 0);
#pragma unroll
                    for (int e = 0; e < 4; ++e)
                        if (n[e] > 0.f) o[2 * i][mt][e] = o[2 * i + 1][mt][e] = NAN;
                }
            }
        }
    }
#pragma unroll
    for (int mt = 0; mt < MT; ++mt) l[mt] = sum_over_groups(l[mt]);
    // The wavefronts' states meet in LDS, one after the other into the first one's registers.
    floatx4* so = (floatx4*)lds;                                // [CT][MT][64]
    float* sm = (float*)(lds + (size_t)CT * MT * 64 * 16);      // [MT][16][2]
    for (int w = 1; w < kQ4Waves; ++w) {
        __syncthreads();
        if (wave == w) {
#pragma unroll
            for (int mt = 0; mt < MT; ++mt) {
                if (g == 0) {
                    sm[(mt * 16 + col) * 2] = m[mt];
                    sm[(mt * 16 + col) * 2 + 1] = l[mt];
                }
#pragma unroll
                for (int ct = 0; ct < CT; ++ct) so[(ct * MT + mt) * 64 + lane] = o[ct][mt];
            }
        }
        __syncthreads();
        if (wave == 0) {
#pragma unroll
            for (int mt = 0; mt < MT; ++mt) {
                const float mo = sm[(mt * 16 + col) * 2], lo = sm[(mt * 16 + col) * 2 + 1];
                const float mn = fmaxf(m[mt], mo), off = mn == -INFINITY ? 0.f : mn;
                const float f0 = __builtin_amdgcn_exp2f(m[mt] - off), f1 = __builtin_amdgcn_exp2f(mo - off);
                m[mt] = mn;
                l[mt] = l[mt] * f0 + lo * f1;
#pragma unroll
                for (int ct = 0; ct < CT; ++ct) o[ct][mt] = o[ct][mt] * f0 + so[(ct * MT + mt) * 64 + lane] * f1;
            }
        }
    }
    if (wave != 0) return;
    if (splits > 1) {
        const size_t unit = blockIdx.x;
        floatx4* po = (floatx4*)a.o_part + unit * (CT * MT * 64);
        float* pm = a.ml_part + unit * (MT * 32);
#pragma unroll
        for (int mt = 0; mt < MT; ++mt) {
            if (g == 0) {
                pm[(mt * 16 + col) * 2] = m[mt];
                pm[(mt * 16 + col) * 2 + 1] = l[mt];
            }
#pragma unroll
            for (int ct = 0; ct < CT; ++ct) po[(ct * MT + mt) * 64 + lane] = o[ct][mt];
        }
        return;
    }
#pragma unroll
    for (int mt = 0; mt < MT; ++mt) {
        const int row = block * 16 * MT + mt * 16 + col;
        if (row >= R) continue;
        // a row that sees no key gives zeros
        const bool none = a.kv_len == 0 && a.mask && !q4_sees(a.mask, node[mt], a.M);
        const float r = 1.f / l[mt];
        half_t* dst = a.out + ((size_t)node[mt] * a.nh + head * rep + row - node[mt] * rep) * D + 4 * g;
#pragma unroll
        for (int ct = 0; ct < CT; ++ct) {
            half4 y;
#pragma unroll
            for (int e = 0; e < 4; ++e) y[e] = none ? (half_t)0.f : (half_t)(o[ct][mt][e] * r);
            *(half4*)(dst + ct * 16) = y;
        }
    }
}

// Parts of a head's keys to its rows.  A wavefront takes one fragment of 16 channels by 16 rows.
template <int D, int MT>
__global__ __launch_bounds__(256) void k_q4_join(const Q4Attn a, int splits, int blocks, int items)
{
    constexpr int CT = D / 16;
    const int lane = threadIdx.x & 63, item = blockIdx.x * 4 + (threadIdx.x >> 6), col = lane & 15, g = lane >> 4;
    if (item >= items) return;
    const int frag = item % (CT * MT), hb = item / (CT * MT), mt = frag % MT, ct = frag / MT;
    const int block = hb % blocks, head = hb / blocks;
    const size_t unit0 = (size_t)hb * splits;
    float m = -INFINITY;
    for (int s = 0; s < splits; ++s) m = fmaxf(m, a.ml_part[(unit0 + s) * (MT * 32) + (mt * 16 + col) * 2]);
    const float off = m == -INFINITY ? 0.f : m;
    float l = 0.f;
    floatx4 o = {0.f, 0.f, 0.f, 0.f};
    for (int s = 0; s < splits; ++s) {
        const float* pm = a.ml_part + (unit0 + s) * (MT * 32) + (mt * 16 + col) * 2;
        const float f = __builtin_amdgcn_exp2f(pm[0] - off);
        l += pm[1] * f;
        o += ((const floatx4*)a.o_part)[(unit0 + s) * (CT * MT * 64) + frag * 64 + lane] * f;
    }
    const int rep = a.nh / a.nkv, row = block * 16 * MT + mt * 16 + col;
    if (row >= a.M * rep) return;
    const int node = row / rep;
    const bool none = a.kv_len == 0 && a.mask && !q4_sees(a.mask, node, a.M);
    half4 y;
#pragma unroll
    for (int e = 0; e < 4; ++e) y[e] = none ? (half_t)0.f : (half_t)(o[e] / l);
    *(half4*)(a.out + ((size_t)node * a.nh + head * rep + row - node * rep) * D + ct * 16 + 4 * g) = y;
}

struct Q4AttnCut {
    int mt, blocks, splits;
};
static Q4AttnCut q4_attn_cut(int M, int kv_len, int nh, int nkv)
{
    Q4AttnCut c;
    const int R = M * (nh / nkv), rt = ceil_div(R, 16), ntiles = ceil_div(kv_len + M, kQ4Tile);
    c.mt = rt <= 1 ? 1 : 2;
    c.blocks = ceil_div(rt, c.mt);
    const int items = nkv * c.blocks;
    c.splits = std::max(1, std::min(ceil_div(ntiles, kQ4Waves), 512 / items));
    return c;
}

size_t q4_attention_bytes(int M, int kv_len, int nh, int nkv, int d)
{
    const Q4AttnCut c = q4_attn_cut(M, kv_len, nh, nkv);
    if (c.splits == 1) return 256;
    const size_t units = (size_t)nkv * c.blocks * c.splits;
    return align_up(units * c.mt * 16 * d * 4, 256) + align_up(units * c.mt * 32 * 4, 256);
}

template <int D, int MT>
static ghd_status q4_attention_of(const Q4Attn& a, const Q4AttnCut& c, hipStream_t st)
{
    const size_t lds = (size_t)(D / 16) * MT * 64 * 16 + MT * 128;
    hipLaunchKernelGGL((k_q4_attention<D, MT>), dim3(a.nkv * c.blocks * c.splits), dim3(kQ4Waves * 64), lds, st, a, c.splits,
                       c.blocks);
    if (c.splits > 1) {
        const int items = a.nkv * c.blocks * (D / 16) * MT;
        hipLaunchKernelGGL((k_q4_join<D, MT>), dim3(ceil_div(items, 4)), dim3(256), 0, st, a, c.splits, c.blocks, items);
    }
    return check_launch();
}

ghd_status launch_q4_attention(Q4Attn a, int d, void* ws, hipStream_t st)
{
    const Q4AttnCut c = q4_attn_cut(a.M, a.kv_len, a.nh, a.nkv);
    const size_t units = (size_t)a.nkv * c.blocks * c.splits;
    a.o_part = (float*)ws;
    a.ml_part = (float*)((char*)ws + align_up(units * c.mt * 16 * d * 4, 256));
    if (d == 128) return c.mt == 1 ? q4_attention_of<128, 1>(a, c, st) : q4_attention_of<128, 2>(a, c, st);
    return c.mt == 1 ? q4_attention_of<64, 1>(a, c, st) : q4_attention_of<64, 2>(a, c, st);
}

}  // namespace ghd
