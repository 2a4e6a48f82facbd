// The 4-bit formats of weights and cache: layouts, what a code stands for, and the launches.
//
// Eight codes lie in a 32-bit word: of pair p = 0..3 the first at bits 4p, the second at bits 16 + 4p.
// So one AND leaves a pair in the low bits of both halves of a word, and an OR of fp16's 1024.0 makes
// fp16 numbers of it: 1024 + c exactly (pairs 0 and 2), 1024 + 16 c (1 and 3).
#pragma once
#include "common.h"

namespace ghd {

// ---- cache -----------------------------------------------------------------------------
// A head's rows lie in tiles of 32, one behind the other.  A K tile: 32 rows of d / 2 bytes of codes (word w
// of a row holds channels 8w .. 8w + 7), then 32 rows of d / 32 (lo, scale) pairs.  A V tile: the MFMA
// operand of V^T as a wavefront's lanes take it with 16-byte loads: word ((c / 64 * 4 + t / 8) * 16 +
// c % 16) * 4 + c / 16 % 4 holds keys t - t % 8 .. + 7 of channel c; then, for every 32 channels, the lo of the 32
// keys and their scales.
constexpr int kQ4Tile = 32;                      // rows of a tile
constexpr int kQ4Group = 32;                     // channels that share lo and scale
__host__ __device__ constexpr int q4_tile_bytes(int d) { return 20 * d; }       // 16 d of codes, 4 d of lo and scale
__host__ __device__ constexpr int q4_codes_bytes(int d) { return 16 * d; }
static inline size_t q4_cache_bytes(int nkv, int cap, int d)
{
    return (size_t)nkv * (cap / kQ4Tile) * q4_tile_bytes(d);
}
// byte offset of a head's tile
__device__ __forceinline__ size_t q4_tile_at(int head, int tile, int tiles, int d)
{
    return ((size_t)head * tiles + tile) * q4_tile_bytes(d);
}
__device__ __forceinline__ int q4_v_word(int c, int octet) { return ((c / 64 * 4 + octet) * 16 + c % 16) * 4 + c / 16 % 4; }

// ---- weights ---------------------------------------------------------------------------
// Unit: 16 rows (a tile) by 128 columns: 1 KiB of codes, 16 bytes a lane of the MFMA operand (word s of lane
// (g, r): row r, columns 32 s + 8 g .. + 7), then for every row and each of its 128 / group groups (scale fp16,
// -(1024 + zero) fp16).  A tile's units lie one behind the other.
constexpr int kQ4Unit = 128;
__host__ __device__ constexpr int q4_unit_bytes(int group) { return 1024 + 64 * (kQ4Unit / group); }
static inline size_t q4_weight_bytes(int N, int K, int group)
{
    return (size_t)ceil_div(N, 16) * ceil_div(K, kQ4Unit) * q4_unit_bytes(group);
}

#ifdef __HIPCC__
// 1 / x, in a scalar register
__device__ __forceinline__ float q4_inverse(int x)
{
    return __builtin_bit_cast(float, __builtin_amdgcn_readfirstlane(__builtin_bit_cast(int, __builtin_amdgcn_rcpf((float)x))));
}

// x / n of an x below 2^15 and an n up to 2^10, by 1 / n: half a unit above x the quotient is at least 1 / 2048 from a whole number,
// and what is rounded in it is less than x / n 2^-22
__device__ __forceinline__ int q4_over(int x, float inv) { return (int)(((float)x + 0.5f) * inv); }

// ---- codes to numbers --------------------------------------------------------------------
// Masks and 1024.0 are kept in registers: as literals they make an AND and an OR of 8 bytes each out of one instruction.
struct Q4Bits {
    uint32_t low, high, k1024;
    __device__ __forceinline__ Q4Bits() : low(0x000f000fu), high(0x00f000f0u), k1024(0x64006400u)
    {
        asm("" : "+s"(low), "+s"(high), "+v"(k1024));
    }
    __device__ __forceinline__ half2_ operator()(uint32_t word, uint32_t mask) const
    {
        return __builtin_bit_cast(half2_, (word & mask) | k1024);
    }
};
__device__ __forceinline__ half2_ pair_of(half_t x) { return (half2_){x, x}; }
__device__ __forceinline__ half8 join(half2_ a, half2_ b, half2_ c, half2_ d)
{
    return (half8){a[0], a[1], b[0], b[1], c[0], c[1], d[0], d[1]};
}
// the codes of a word, less a zero point, exactly: off = -(1024 + zero) (fp16 holds whole numbers up to 2048)
__device__ __forceinline__ half8 q4_codes(const Q4Bits& bits, uint32_t w, half2_ off)
{
    const half2_ off16 = off + pair_of((half_t)960.f);         // -(64 + zero)
    const half2_ sixteenth = pair_of((half_t)0.0625f);
    const uint32_t v = w >> 8;
    return join(bits(w, bits.low) + off, __builtin_elementwise_fma(bits(w, bits.high), sixteenth, off16),
                bits(v, bits.low) + off, __builtin_elementwise_fma(bits(v, bits.high), sixteenth, off16));
}
// fp16(lo + code * scale) of the codes of a word, pair by pair
__device__ __forceinline__ half8 q4_values(const Q4Bits& bits, uint32_t w, const half2_ lo[4], const half2_ scale[4])
{
    const half8 c = q4_codes(bits, w, pair_of((half_t)-1024.f));
    half2_ r[4];
#pragma unroll
    for (int p = 0; p < 4; ++p)
        r[p] = __builtin_elementwise_fma((half2_){c[2 * p], c[2 * p + 1]}, scale[p], lo[p]);
    return join(r[0], r[1], r[2], r[3]);
}
__device__ __forceinline__ half8 q4_values(const Q4Bits& bits, uint32_t w, half2_ lo, half2_ scale)
{
    const half2_ l[4] = {lo, lo, lo, lo}, s[4] = {scale, scale, scale, scale};
    return q4_values(bits, w, l, s);
}
#endif

// ---- launches --------------------------------------------------------------------------
struct Q4Append {
    char *k, *v;                     // one layer's cache
    const half_t *kx, *vx, *q;       // rows [M][heads][d]; q may be null
    half_t* q_out;
    const int32_t* parent;           // null: consecutive positions
    int64_t ld_k, ld_v, ld_q, ld_qo;
    int M, kv_len, nkv, nq, tiles;   // nq: query heads to be turned (0 without q)
    float rope_base;                 // 0: rows as they are
    double log2_step;                // of the angles of neighbouring channels (the launch's)
};
ghd_status launch_q4_append(Q4Append a, int d, hipStream_t st);
ghd_status launch_q4_commit(void* const* k, void* const* v, int L, int nkv, int d, int cap, int kv_len, int M,
                            const int32_t* res, hipStream_t st);
ghd_status launch_q4_read(void* const* k, void* const* v, int L, int nkv, int d, int cap, int row0, int rows, half_t* ko,
                          half_t* vo, hipStream_t st);
constexpr int kQ4MaxLayers = 48;
constexpr int kQ4MostGroups = 1 << 23;           // workgroups of 256 in a launch, which has below 2^32 threads along an axis

struct Q4Attn {
    half_t* out;
    const half_t* q;
    const char *k, *v;
    const int32_t* parent;           // one of the two is null
    const uint64_t* mask;
    float *o_part, *ml_part;
    int M, kv_len, nh, nkv, tiles;   // tiles: of the whole cache, a head
    float scale;
    int rep;                         // query heads of a key head, and 1 / rep (the launch fills these in)
    float inv_rep;
};
size_t q4_attention_bytes(int M, int kv_len, int nh, int nkv, int d);
void q4_attention_on_host(int M, int kv_len, int nh, int nkv, int d, int64_t* out4);
ghd_status launch_q4_attention(Q4Attn a, int d, void* ws, size_t ws_bytes, hipStream_t st);     // GHD_ERR_WORKSPACE: too small

struct Q4Linear {
    void* y;
    const half_t* x;
    const char* W;
    float* part;
    int M, N, K, group;
    int64_t ldx, ldy;
    bool out16;
};
size_t q4_linear_bytes(int M, int N, int K);
bool q4_linear_meets(const Q4Linear& a);
void q4_x_on_host(int M, int N, int K, int ldx, int64_t* out2);
ghd_status launch_q4_linear(Q4Linear a, void* ws, size_t ws_bytes, hipStream_t st);              // the same
ghd_status launch_q4_pack(void* dst, const void* codes, const void* scales, const void* zeros, int N, int K, int group,
                          hipStream_t st);

}  // namespace ghd
