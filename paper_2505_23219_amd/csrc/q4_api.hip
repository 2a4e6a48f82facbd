// Host side of the 4-bit entry points (include/ghd.h): argument checks and launches.
#include "q4.h"

namespace ghd {

static inline bool aligned_to(const void* p, size_t n) { return ((uintptr_t)p & (n - 1)) == 0; }

// a 4-bit cache's sizes, and rows [0, rows) inside it
static ghd_status check_cache(int nkv, int d, int cap, int64_t rows)
{
    if (nkv < 1 || nkv > 256 || (d != 64 && d != 128)) return GHD_ERR_SHAPE;
    if (cap < 1 || cap > (1 << 24) || cap % kQ4Tile != 0 || rows > cap) return GHD_ERR_CAPACITY;
    return GHD_OK;
}

static ghd_status check_layers(const ghd_kv* kv, int L)
{
    for (int l = 0; l < L; ++l) {
        if (!kv[l].k || !kv[l].v) return GHD_ERR_NULL;
        if (!aligned_to(kv[l].k, 16) || !aligned_to(kv[l].v, 16)) return GHD_ERR_ALIGN;
    }
    return GHD_OK;
}

static bool weight_shape_ok(int N, int K, int group)
{
    if (N < 1 || N > (1 << 20) || K < 8 || K > 65536 || K % 8 != 0) return false;
    return group == 32 || group == 64 || group == 128;
}

static Q4Linear linear_args(void* y, const void* x, const void* Wq, int M, int N, int K, int group, int64_t ldx, int64_t ldy, uint32_t flags)
{
    Q4Linear a = {};
    a.y = y;
    a.x = (const half_t*)x;
    a.W = (const char*)Wq;
    a.M = M;
    a.N = N;
    a.K = K;
    a.group = group;
    a.ldx = ldx;
    a.ldy = ldy;
    a.out16 = flags == GHD_OUT_F16;
    return a;
}

static ghd_status attention_q4(void* out, const void* q, const ghd_kv* kv, const int32_t* parent, const uint64_t* mask, int M,
                               int kv_len, int nh, int nkv, int d, int cap, float scale, void* ws, size_t ws_bytes,
                               void* stream)
{
    if (!out || !q || !kv || (!parent && !mask)) return GHD_ERR_NULL;
    ghd_status s = check_layers(kv, 1);
    if (s == GHD_ERR_NULL) return s;
    if (M < 1 || M > GHD_MAX_M || kv_len < 0 || nh < 1 || nh > 256 || nkv < 1 || nh % nkv != 0) return GHD_ERR_SHAPE;
    ghd_status c = check_cache(nkv, d, cap, (int64_t)kv_len + M);
    if (c) return c;
    if (s) return s;
    if (!aligned_to(out, 16) || !aligned_to(q, 16) || !aligned_to(mask, 8) || !aligned_to(parent, 4)) return GHD_ERR_ALIGN;
    if (!ws) return GHD_ERR_WORKSPACE;
    if (!aligned_to(ws, 16)) return GHD_ERR_ALIGN;
    Q4Attn a = {};
    a.out = (half_t*)out;
    a.q = (const half_t*)q;
    a.k = (const char*)kv->k;
    a.v = (const char*)kv->v;
    a.parent = parent;
    a.mask = mask;
    a.M = M;
    a.kv_len = kv_len;
    a.nh = nh;
    a.nkv = nkv;
    a.tiles = cap / kQ4Tile;
    a.scale = scale;
    return launch_q4_attention(a, d, ws, ws_bytes, (hipStream_t)stream);
}

}  // namespace ghd

using namespace ghd;

extern "C" {

size_t ghd_weight_q4_bytes(int N, int K, int group) { return weight_shape_ok(N, K, group) ? q4_weight_bytes(N, K, group) : 0; }

ghd_status ghd_pack_weight_q4(void* dst, const void* codes, const void* scales, const void* zeros, int N, int K, int group,
                              void* stream)
{
    if (!dst || !codes || !scales) return GHD_ERR_NULL;
    if (!weight_shape_ok(N, K, group)) return GHD_ERR_SHAPE;
    if (!aligned_to(dst, 16) || !aligned_to(scales, 2)) return GHD_ERR_ALIGN;
    return launch_q4_pack(dst, codes, scales, zeros, N, K, group, (hipStream_t)stream);
}

size_t ghd_linear_q4_workspace_bytes(int M, int N, int K)
{
    if (M < 1 || M > GHD_MAX_M || !weight_shape_ok(N, K, 128)) return 0;
    return q4_linear_bytes(M, N, K);
}

ghd_status ghd_linear_q4(void* y, const void* x, const void* Wq, int M, int N, int K, int group, int64_t ldx, int64_t ldy,
                         uint32_t flags, void* ws, size_t ws_bytes, void* stream)
{
    if (!y || !x || !Wq) return GHD_ERR_NULL;
    if (M < 1 || M > GHD_MAX_M || !weight_shape_ok(N, K, group) || flags > GHD_OUT_F16) return GHD_ERR_SHAPE;
    // x is read at 32-bit byte offsets: 128 rows so far apart end below 2^31
    if (ldx < K || ldy < N || ldx > (1 << 23)) return GHD_ERR_SHAPE;
    if (!aligned_to(x, 16) || !aligned_to(Wq, 16) || !aligned_to(y, 16) || ldx % 8 != 0) return GHD_ERR_ALIGN;
    if (!ws) return GHD_ERR_WORKSPACE;
    if (!aligned_to(ws, 16)) return GHD_ERR_ALIGN;
    const Q4Linear a = linear_args(y, x, Wq, M, N, K, group, ldx, ldy, flags);
    return launch_q4_linear(a, ws, ws_bytes, (hipStream_t)stream);
}

size_t ghd_kv_q4_bytes(int nkv, int capacity, int d)
{
    return check_cache(nkv, d, capacity, 0) ? 0 : q4_cache_bytes(nkv, capacity, d);
}

ghd_status ghd_kv_append_q4(const ghd_kv* kv, const void* k, const void* v, const void* q, void* q_out,
                            const int32_t* parent_dev, int M, int kv_len, int nh, int nkv, int d, int capacity, int64_t ld_k,
                            int64_t ld_v, int64_t ld_q, int64_t ld_q_out, float rope_base, void* stream)
{
    if (!kv || !k || !v || (q && !q_out)) return GHD_ERR_NULL;
    ghd_status s = check_layers(kv, 1);
    if (s == GHD_ERR_NULL) return s;
    if (M < 1 || (parent_dev && M > GHD_MAX_M) || kv_len < 0 || !(rope_base >= 0.f) || rope_base > 1e30f) return GHD_ERR_SHAPE;
    ghd_status c = check_cache(nkv, d, capacity, (int64_t)kv_len + M);
    if (c) return c;
    if (ld_k < (int64_t)nkv * d || ld_v < (int64_t)nkv * d) return GHD_ERR_SHAPE;
    if (q && (rope_base == 0.f || nh < 1 || nh > 256 || ld_q < (int64_t)nh * d || ld_q_out < (int64_t)nh * d))
        return GHD_ERR_SHAPE;
    if (s) return s;
    if (!aligned_to(k, 4) || !aligned_to(v, 4) || !aligned_to(parent_dev, 4) || ld_k % 2 != 0 || ld_v % 2 != 0)
        return GHD_ERR_ALIGN;
    if (q && (!aligned_to(q, 4) || !aligned_to(q_out, 4) || ld_q % 2 != 0 || ld_q_out % 2 != 0)) return GHD_ERR_ALIGN;
    Q4Append a = {};
    a.k = (char*)kv->k;
    a.v = (char*)kv->v;
    a.kx = (const half_t*)k;
    a.vx = (const half_t*)v;
    a.q = (const half_t*)q;
    a.q_out = (half_t*)q_out;
    a.parent = parent_dev;
    a.ld_k = ld_k;
    a.ld_v = ld_v;
    a.ld_q = ld_q;
    a.ld_qo = ld_q_out;
    a.M = M;
    a.kv_len = kv_len;
    a.nkv = nkv;
    a.nq = q ? nh : 0;
    a.tiles = capacity / kQ4Tile;
    a.rope_base = rope_base;
    return launch_q4_append(a, d, (hipStream_t)stream);
}

size_t ghd_attention_q4_workspace_bytes(int M, int kv_len, int nh, int nkv, int d)
{
    if (M < 1 || M > GHD_MAX_M || kv_len < 0 || kv_len > (1 << 24) || nh < 1 || nh > 256 || nkv < 1 || nh % nkv != 0 ||
        (d != 64 && d != 128))
        return 0;
    return q4_attention_bytes(M, kv_len, nh, nkv, d);
}

ghd_status ghd_tree_attention_q4(void* out, const void* q, const ghd_kv* kv, const int32_t* parent_dev, int M, int kv_len,
                                 int nh, int nkv, int d, int capacity, float scale, void* ws, size_t ws_bytes, void* stream)
{
    if (!parent_dev) return GHD_ERR_NULL;
    return attention_q4(out, q, kv, parent_dev, nullptr, M, kv_len, nh, nkv, d, capacity, scale, ws, ws_bytes, stream);
}

ghd_status ghd_masked_attention_q4(void* out, const void* q, const ghd_kv* kv, const uint64_t* mask_dev, int M, int kv_len,
                                   int nh, int nkv, int d, int capacity, float scale, void* ws, size_t ws_bytes, void* stream)
{
    if (!mask_dev) return GHD_ERR_NULL;
    return attention_q4(out, q, kv, nullptr, mask_dev, M, kv_len, nh, nkv, d, capacity, scale, ws, ws_bytes, stream);
}

static ghd_status check_stack(const ghd_kv* kv_host, int L, int nkv, int d, int capacity, int64_t rows, void** k, void** v)
{
    if (L < 1 || L > kQ4MaxLayers) return GHD_ERR_SHAPE;
    ghd_status s = check_layers(kv_host, L);
    if (s == GHD_ERR_NULL) return s;
    ghd_status c = check_cache(nkv, d, capacity, rows);
    if (c) return c;
    for (int l = 0; l < L; ++l) {
        k[l] = kv_host[l].k;
        v[l] = kv_host[l].v;
    }
    return s;
}

ghd_status ghd_commit_path_q4(const ghd_kv* kv_host, int L, int nkv, int d, int capacity, const int32_t* res_dev, int M,
                              int kv_len, void* stream)
{
    if (!kv_host || !res_dev) return GHD_ERR_NULL;
    if (M < 1 || M > GHD_MAX_M || kv_len < 0) return GHD_ERR_SHAPE;
    void *k[kQ4MaxLayers], *v[kQ4MaxLayers];
    ghd_status s = check_stack(kv_host, L, nkv, d, capacity, (int64_t)kv_len + M, k, v);
    if (s) return s;
    if (!aligned_to(res_dev, 4)) return GHD_ERR_ALIGN;
    return launch_q4_commit(k, v, L, nkv, d, capacity, kv_len, M, res_dev, (hipStream_t)stream);
}

ghd_status ghd_kv_read_q4(void* k_out, void* v_out, const ghd_kv* kv_host, int L, int nkv, int d, int capacity, int row0,
                          int rows, void* stream)
{
    if (!kv_host || !k_out || !v_out) return GHD_ERR_NULL;
    if (row0 < 0 || rows < 1) return GHD_ERR_SHAPE;
    void *k[kQ4MaxLayers], *v[kQ4MaxLayers];
    ghd_status s = check_stack(kv_host, L, nkv, d, capacity, (int64_t)row0 + rows, k, v);
    if (s) return s;
    if (!aligned_to(k_out, 16) || !aligned_to(v_out, 16)) return GHD_ERR_ALIGN;
    return launch_q4_read(k, v, L, nkv, d, capacity, row0, rows, (half_t*)k_out, (half_t*)v_out, (hipStream_t)stream);
}

/* Test support (not part of the documented ABI): the host's rules and the kernels' arithmetic. */
/* out2 = {bytes from the beginning of x to the end of the last that a call reads, numbers of x that it reads}. */
void ghd_debug_q4_x(int M, int N, int K, int ldx, int64_t* out2) { q4_x_on_host(M, N, K, ldx, out2); }

/* out4 = {tiles of 16 rows in a block, blocks of a key head, parts of its keys, bytes of workspace} of an attention call. */
void ghd_debug_q4_attention(int M, int kv_len, int nh, int nkv, int d, int64_t* out4)
{
    q4_attention_on_host(M, kv_len, nh, nkv, d, out4);
}

/* Would y of a linear call meet x or Wq? */
int ghd_debug_q4_linear_meets(void* y, const void* x, const void* Wq, int M, int N, int K, int group, int64_t ldx, int64_t ldy, uint32_t flags)
{
    return q4_linear_meets(linear_args(y, x, Wq, M, N, K, group, ldx, ldy, flags));
}

}  // extern "C"
