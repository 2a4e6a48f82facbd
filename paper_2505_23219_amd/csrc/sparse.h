// Attention over blocks of the committed cache that each drafted token selects: layouts and launches.
//
// A block is 64 committed rows.  Its bounds: for every channel the largest and the smallest key as whole numbers HI and LO,
// within -127 .. 127, of a unit that is a power of two; HI rounded up and LO down, so q.k <= sum_c (q > 0 ? q HI : q LO) unit, but
// for what ends at 127.
// Scores are whole numbers times powers of two, exact in 32 bits: the order of the blocks does not depend on how they are summed.
#pragma once
#include "common.h"

namespace ghd {

constexpr int kBlock = 64;                       // rows of a block
constexpr int kSparseMaxRows = 1 << 21;          // committed rows of a call

// Bounds of one layer: HI then LO of every channel, a byte each, [nkv][blocks][2 d]; behind them the units, float [nkv][blocks]
// (0: all keys are zeros; infinity: one is not finite).
static inline size_t bounds_units_at(int nkv, int d, int blocks) { return (size_t)nkv * blocks * 2 * d; }
static inline size_t bounds_bytes(int nkv, int d, int blocks) { return bounds_units_at(nkv, d, blocks) + (size_t)nkv * blocks * 4; }

struct Bounds {
    char* codes;
    float* units;
    int blocks;                      // of a head, as laid out
};
static inline Bounds bounds_of(void* p, int nkv, int d, int blocks)
{
    return {(char*)p, (float*)((char*)p + bounds_units_at(nkv, d, blocks)), blocks};
}

ghd_status launch_block_bounds(Bounds to, const half_t* k, int first, int n, int nkv, int d, int64_t k_head, int64_t k_tok, hipStream_t st);
ghd_status launch_block_bounds_read(float* hi, float* lo, Bounds from, int first, int n, int nkv, int d, hipStream_t st);

struct SelectArgs {
    uint64_t* sel;                   // [nkv][words][n]
    const half_t* q;
    Bounds bounds;
    uint32_t* keys;                  // workspace: [nkv][M][n rounded up to 4]
    int M, nkv, rep, n;
    bool zero;                       // (the launch's) the words have to be zeros when the picks begin
    int lo, hi, keep;                // blocks [0, lo) and [hi, n) are taken, and `keep` of those between
};
// A pick cuts the keys from low to high into at most 256 steps of 2^shift keys.
__host__ __device__ static inline int pick_shift(uint32_t low, uint32_t high)
{
    const int bits = 32 - __builtin_clz((high - low) | 1);
    return bits > 8 ? bits - 8 : 0;
}
// The last key of the step that begins at `from`: the highest step ends at `high`.  (Where infinite scores meet ones below zero a step is 2^24
// keys, and the highest may reach beyond 32 bits.)
__host__ __device__ static inline uint32_t pick_step_end(uint32_t from, uint32_t high, int shift)
{
    return (high - from) >> shift ? from + ((1u << shift) - 1) : high;
}
static inline size_t select_bytes(int M, int n, int nkv) { return align_up((size_t)nkv * M * ((n + 3) & ~3) * 4, 256) + 256; }
ghd_status launch_block_select(SelectArgs a, int d, hipStream_t st);

struct SparseArgs {
    half_t* out;
    const half_t *q, *k, *v;
    const uint64_t* sel;             // [nkv][ceil(M / 64)][n]
    const int32_t* parent;           // one of the two is null
    const uint64_t* mask;
    int64_t k_head, k_tok, v_head, v_ch;
    float *o_part, *ml_part;
    int M, kv_len, nh, nkv, rep, n;
    float scale, inv_rep;            // (rep, 1 / rep, n and the workspace's parts are the launch's)
};
size_t sparse_attention_bytes(int M, int kv_len, int nh, int nkv, int d);
// Halves of the `count` blocks of a list that hold rows: the last block may end in its first half (`total` rows are there, and a block's
// first).
__host__ __device__ static inline int sparse_halves(int count, int last_block, int total)
{
    return 2 * count - (count > 0 && last_block * kBlock + kBlock / 2 >= total);
}
void sparse_attention_on_host(int M, int kv_len, int nh, int nkv, int d, int64_t* out4);
ghd_status launch_sparse_attention(SparseArgs a, int d, void* ws, size_t ws_bytes, hipStream_t st);    // GHD_ERR_WORKSPACE: too small

struct SampleArgs {
    const float *logits, *q_logits, *u;
    const int32_t *tokens, *parent, *q_row;
    int32_t* res;
    int M, V, q_rows;
    float temperature, q_temperature;
};
size_t accept_sampled_bytes(int M, int V, bool drafts);   // drafts: they have probabilities
ghd_status launch_accept_sampled(const SampleArgs& a, void* ws, hipStream_t st);

}  // namespace ghd
