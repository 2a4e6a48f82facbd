// Host side of the sparse attention's and the sampled acceptance's entry points (include/ghd.h): argument checks and launches.
#include "sparse.h"

#include <math.h>

namespace ghd {

static inline bool at16(const void* p) { return ((uintptr_t)p & 15) == 0; }
static inline bool at_word(const void* p, size_t n) { return ((uintptr_t)p & (n - 1)) == 0; }

// do two ranges of memory share a byte?
static inline bool meet(const void* a, size_t na, const void* b, size_t nb)
{
    return a && b && na && nb && (uintptr_t)a < (uintptr_t)b + nb && (uintptr_t)b < (uintptr_t)a + na;
}

static bool heads_ok(int nh, int nkv, int d)
{
    return nh >= 1 && nh <= 1024 && nkv >= 1 && nkv <= 256 && nh % nkv == 0 && (d == 64 || d == 128);
}
static bool rows_ok(int M, int kv_len) { return M >= 1 && M <= GHD_MAX_M && kv_len >= 0 && kv_len <= kSparseMaxRows; }

// a cache's layout of bounds
static ghd_status check_bounds(int nkv, int d, int capacity)
{
    if (nkv < 1 || nkv > 256 || (d != 64 && d != 128)) return GHD_ERR_SHAPE;
    if (capacity < 1 || capacity > (1 << 24)) return GHD_ERR_CAPACITY;
    return GHD_OK;
}
static ghd_status check_range(int block0, int blocks, int capacity)
{
    if (block0 < 0 || blocks < 0 || blocks > kSparseMaxRows / kBlock) return GHD_ERR_SHAPE;
    return (int64_t)block0 + blocks > capacity / kBlock ? GHD_ERR_CAPACITY : GHD_OK;
}

// bytes from a cache's first number to behind the last that rows [0, rows) hold
static size_t k_bytes(int nkv, int64_t rows, int d, int64_t head, int64_t tok) { return 2 * (size_t)((nkv - 1) * head + (rows - 1) * tok + d); }
static size_t v_bytes(int nkv, int64_t rows, int d, int64_t head, int64_t ch) { return 2 * (size_t)((nkv - 1) * head + (d - 1) * ch + rows); }

}  // namespace ghd

using namespace ghd;

extern "C" {

size_t ghd_block_bounds_bytes(int nkv, int capacity, int d)
{
    return check_bounds(nkv, d, capacity) ? 0 : bounds_bytes(nkv, d, capacity / kBlock);
}

ghd_status ghd_block_bounds(void* bounds, const void* k_cache, int block0, int blocks, int nkv, int d, int capacity, int64_t k_stride_head,
                            int64_t k_stride_tok, void* stream)
{
    if (!bounds || !k_cache) return GHD_ERR_NULL;
    ghd_status s = check_bounds(nkv, d, capacity);
    if (!s) s = check_range(block0, blocks, capacity);
    if (s) return s;
    if (k_stride_tok < d || k_stride_head < 0) return GHD_ERR_SHAPE;
    if (!at16(bounds) || !at16(k_cache) || k_stride_tok % 8 != 0 || k_stride_head % 8 != 0) return GHD_ERR_ALIGN;
    if (blocks == 0) return GHD_OK;
    if (meet(bounds, bounds_bytes(nkv, d, capacity / kBlock), k_cache,
             k_bytes(nkv, ((int64_t)block0 + blocks) * kBlock, d, k_stride_head, k_stride_tok)))
        return GHD_ERR_SHAPE;
    return launch_block_bounds(bounds_of(bounds, nkv, d, capacity / kBlock), (const half_t*)k_cache, block0, blocks, nkv, d, k_stride_head,
                               k_stride_tok, (hipStream_t)stream);
}

ghd_status ghd_block_bounds_read(float* hi, float* lo, const void* bounds, int block0, int blocks, int nkv, int d, int capacity, void* stream)
{
    if (!bounds || (blocks > 0 && (!hi || !lo))) return GHD_ERR_NULL;
    ghd_status s = check_bounds(nkv, d, capacity);
    if (!s) s = check_range(block0, blocks, capacity);
    if (s || blocks == 0) return s;
    if (!at16(hi) || !at16(lo) || !at16(bounds)) return GHD_ERR_ALIGN;
    const size_t n = (size_t)nkv * blocks * d * 4, held = bounds_bytes(nkv, d, capacity / kBlock);
    if (meet(hi, n, lo, n) || meet(hi, n, bounds, held) || meet(lo, n, bounds, held)) return GHD_ERR_SHAPE;
    // (the kernel only reads through it)
    return launch_block_bounds_read(hi, lo, bounds_of(const_cast<void*>(bounds), nkv, d, capacity / kBlock), block0, blocks, nkv, d,
                                    (hipStream_t)stream);
}

size_t ghd_block_select_workspace_bytes(int M, int kv_len, int nkv)
{
    if (!rows_ok(M, kv_len) || nkv < 1 || nkv > 256) return 0;
    return select_bytes(M, kv_len / kBlock, nkv);
}

ghd_status ghd_block_select(uint64_t* sel_dev, const void* q, const void* bounds, int M, int kv_len, int nh, int nkv, int d, int capacity,
                            int count, int sinks, int recent, void* ws, size_t ws_bytes, void* stream)
{
    const int n = kv_len / kBlock;
    if (!q || !bounds || (!sel_dev && n > 0)) return GHD_ERR_NULL;
    if (!rows_ok(M, kv_len) || !heads_ok(nh, nkv, d)) return GHD_ERR_SHAPE;
    ghd_status s = check_bounds(nkv, d, capacity);
    if (s) return s;
    if (count < 0 || sinks < 0 || recent < 0 || (int64_t)sinks + recent > count) return GHD_ERR_SHAPE;
    if (n > capacity / kBlock) return GHD_ERR_CAPACITY;
    if (!at16(q) || !at16(bounds) || !at_word(sel_dev, 8)) return GHD_ERR_ALIGN;
    if (n == 0) return GHD_OK;
    if (!ws) return GHD_ERR_WORKSPACE;
    if (!at16(ws)) return GHD_ERR_ALIGN;
    if (ws_bytes < select_bytes(M, n, nkv)) return GHD_ERR_WORKSPACE;
    const size_t held = (size_t)nkv * ceil_div(M, 64) * n * 8, q_bytes = (size_t)M * nh * d * 2, used = select_bytes(M, n, nkv);
    const size_t b_bytes = bounds_bytes(nkv, d, capacity / kBlock);
    if (meet(sel_dev, held, q, q_bytes) || meet(sel_dev, held, bounds, b_bytes) || meet(sel_dev, held, ws, used) || meet(ws, used, q, q_bytes) ||
        meet(ws, used, bounds, b_bytes))
        return GHD_ERR_SHAPE;
    SelectArgs a = {};
    a.sel = sel_dev;
    a.q = (const half_t*)q;
    a.bounds = bounds_of(const_cast<void*>(bounds), nkv, d, capacity / kBlock);
    a.keys = (uint32_t*)ws;
    a.M = M;
    a.nkv = nkv;
    a.rep = nh / nkv;
    a.n = n;
    a.lo = sinks < n ? sinks : n;
    a.hi = n - recent > a.lo ? n - recent : a.lo;
    const int all = count < n ? count : n;
    a.keep = all - a.lo - (n - a.hi);
    return launch_block_select(a, d, (hipStream_t)stream);
}

size_t ghd_sparse_attention_workspace_bytes(int M, int kv_len, int nh, int nkv, int d)
{
    return rows_ok(M, kv_len) && heads_ok(nh, nkv, d) ? sparse_attention_bytes(M, kv_len, nh, nkv, d) : 0;
}

ghd_status ghd_sparse_attention(void* out, const void* q, const void* k_cache, const void* v_cache, const uint64_t* sel_dev,
                                const int32_t* parent_dev, const uint64_t* mask_dev, int M, int kv_len, int nh, int nkv, int d,
                                int64_t k_stride_head, int64_t k_stride_tok, int64_t v_stride_head, int64_t v_stride_ch, float scale,
                                void* ws, size_t ws_bytes, void* stream)
{
    const int n = kv_len / kBlock;
    if (!out || !q || !k_cache || !v_cache || (!sel_dev && n > 0) || (!parent_dev && !mask_dev)) return GHD_ERR_NULL;
    if (!rows_ok(M, kv_len) || !heads_ok(nh, nkv, d) || (parent_dev && mask_dev) || !(fabsf(scale) <= 1e20f)) return GHD_ERR_SHAPE;
    // (a block's rows and a head's channels are read at 32-bit offsets)
    if (k_stride_tok < d || k_stride_head < 0 || v_stride_head < 0 || k_stride_tok > (1 << 24) || v_stride_ch > (1 << 22)) return GHD_ERR_SHAPE;
    const int64_t rows = (int64_t)kv_len + M;
    if (v_stride_ch < rows) return GHD_ERR_CAPACITY;
    if (!at16(out) || !at16(q) || !at16(k_cache) || !at16(v_cache) || k_stride_tok % 8 != 0 || k_stride_head % 8 != 0 ||
        v_stride_ch % 8 != 0 || v_stride_head % 8 != 0 || !at_word(sel_dev, 8) || !at_word(mask_dev, 8) || !at_word(parent_dev, 4))
        return GHD_ERR_ALIGN;
    if (!ws) return GHD_ERR_WORKSPACE;
    if (!at16(ws)) return GHD_ERR_ALIGN;
    // neither what is written nor the workspace meets what is read (out may be q: a workgroup writes the rows that it has read)
    int64_t cut[4];
    sparse_attention_on_host(M, kv_len, nh, nkv, d, cut);
    const size_t held = (size_t)M * nh * d * 2, used = cut[3] < (int64_t)ws_bytes ? cut[3] : ws_bytes;
    const struct {
        const void* p;
        size_t n;
    } read[] = {{q, held}, {k_cache, k_bytes(nkv, rows, d, k_stride_head, k_stride_tok)}, {v_cache, v_bytes(nkv, rows, d, v_stride_head, v_stride_ch)},
                {sel_dev, (size_t)nkv * ceil_div(M, 64) * n * 8}, {parent_dev, (size_t)M * 4}, {mask_dev, (size_t)M * 16}};
    for (const auto& r : read)
        if ((r.p != out && meet(out, held, r.p, r.n)) || meet(ws, used, r.p, r.n)) return GHD_ERR_SHAPE;
    if (meet(out, held, ws, used) || out == k_cache || out == v_cache || out == (const void*)sel_dev || out == (const void*)parent_dev ||
        out == (const void*)mask_dev)
        return GHD_ERR_SHAPE;
    SparseArgs a = {};
    a.out = (half_t*)out;
    a.q = (const half_t*)q;
    a.k = (const half_t*)k_cache;
    a.v = (const half_t*)v_cache;
    a.sel = sel_dev;
    a.parent = parent_dev;
    a.mask = mask_dev;
    a.k_head = k_stride_head;
    a.k_tok = k_stride_tok;
    a.v_head = v_stride_head;
    a.v_ch = v_stride_ch;
    a.M = M;
    a.kv_len = kv_len;
    a.nh = nh;
    a.nkv = nkv;
    a.scale = scale;
    return launch_sparse_attention(a, d, ws, ws_bytes, (hipStream_t)stream);
}

size_t ghd_accept_sampled_workspace_bytes(int M, int V)
{
    return M < 1 || M > GHD_MAX_M || V < 1 || V > 262144 ? 0 : accept_sampled_bytes(M, V, true);
}

size_t ghd_accept_sampled_undrawn_workspace_bytes(int M, int V)
{
    return M < 1 || M > GHD_MAX_M || V < 1 || V > 262144 ? 0 : accept_sampled_bytes(M, V, false);
}

ghd_status ghd_accept_sampled(const float* logits, const int32_t* tokens_dev, const int32_t* parent_dev, const float* u_dev,
                              const float* q_logits, const int32_t* q_row_dev, int q_rows, int M, int V, float temperature,
                              float q_temperature, int32_t* res_dev, void* ws, size_t ws_bytes, void* stream)
{
    if (!logits || !tokens_dev || !parent_dev || !u_dev || !res_dev) return GHD_ERR_NULL;
    if (M < 1 || M > GHD_MAX_M || V < 1 || V > 262144) return GHD_ERR_SHAPE;
    if (!(temperature > 0.f) || !isfinite(temperature)) return GHD_ERR_SHAPE;
    if (q_logits) {
        if (!(q_temperature > 0.f) || !isfinite(q_temperature) || q_rows < (q_row_dev ? 1 : M) || q_rows > GHD_MAX_M) return GHD_ERR_SHAPE;
    } else if (q_row_dev) {
        return GHD_ERR_NULL;
    }
    if (!at_word(logits, 4) || !at_word(q_logits, 4) || !at_word(tokens_dev, 4) || !at_word(parent_dev, 4) || !at_word(u_dev, 4) ||
        !at_word(q_row_dev, 4) || !at_word(res_dev, 4))
        return GHD_ERR_ALIGN;
    const size_t used = accept_sampled_bytes(M, V, q_logits != nullptr), row = (size_t)V * 4, ints = (size_t)M * 4;
    if (!ws || ws_bytes < used) return GHD_ERR_WORKSPACE;
    if (!at16(ws)) return GHD_ERR_ALIGN;
    // (the result is written when all else has been read: it may lie where an input is)
    if (meet(ws, used, res_dev, ints + 8) || meet(ws, used, logits, M * row) || meet(ws, used, q_logits, q_rows * row) || meet(ws, used, tokens_dev, ints) ||
        meet(ws, used, parent_dev, ints) || meet(ws, used, u_dev, ints) || meet(ws, used, q_row_dev, ints))
        return GHD_ERR_SHAPE;
    SampleArgs a = {};
    a.logits = logits;
    a.q_logits = q_logits;
    a.u = u_dev;
    a.tokens = tokens_dev;
    a.parent = parent_dev;
    a.q_row = q_row_dev;
    a.res = res_dev;
    a.M = M;
    a.V = V;
    a.q_rows = q_rows;
    a.temperature = temperature;
    a.q_temperature = q_temperature;
    return launch_accept_sampled(a, ws, (hipStream_t)stream);
}

/* Test support (not part of the documented ABI): out4 = {tiles of 16 rows in a block of an attention call, blocks of a key head, parts of
 * what a block reads, bytes of workspace that it needs}. */
void ghd_debug_sparse_attention(int M, int kv_len, int nh, int nkv, int d, int64_t* out4)
{
    sparse_attention_on_host(M, kv_len, nh, nkv, d, out4);
}

/* Halves of blocks that a list of `count` blocks, the last of them `last_block`, gives the wavefronts. */
int ghd_debug_sparse_halves(int count, int last_block, int total) { return sparse_halves(count, last_block, total); }

/* How a pick cuts a range of keys, and the last key of a step of it. */
int ghd_debug_pick_shift(uint32_t low, uint32_t high) { return pick_shift(low, high); }
uint32_t ghd_debug_pick_step_end(uint32_t from, uint32_t high, int shift) { return pick_step_end(from, high, shift); }

}  // extern "C"
