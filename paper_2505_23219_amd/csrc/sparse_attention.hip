// Attention of the drafted tokens over the blocks that each has selected, the committed rows behind the last whole block, and the
// drafted rows that it sees.
//
// A key head's query rows - M tokens by nh / nkv heads - are the columns of S^T = K q^T and O^T = V^T P^T, so softmax statistics are a
// lane's own and probabilities come out as the operand of the second product.  Maximum and sum run along in 32 bits; probabilities
// are rounded to fp16 relative to a maximum that lags by up to 2^8 (fp16 holds that as exactly, and sums are rescaled seldom).
// A workgroup has a block of rows and reads what any of them has selected; a row that has not selected a block has the score minus
// infinity there.
#include "sparse.h"
#include "attention_impl.h"

namespace ghd {

typedef uint32_t uint4_ __attribute__((ext_vector_type(4)));

constexpr int kSparseWaves = 4, kSparseThreads = kSparseWaves * 64;
constexpr int kList = 1024;                      // blocks of a workgroup's list: the host divides a head's so that they fit

// How a launch is divided: rows in `blocks` blocks, what a block of rows reads in `splits` parts.
struct SparseCut {
    int rows, blocks, splits;                    // rows: tiles of 16 in a block
};

// The blocks that tokens i0 .. i1 (at most 64 of them) have selected, then the `tail` that all read: [lo, hi) of them, in order, to the
// list, with a bit for each of the tokens.  Returns how many.
struct SparseList {
    uint64_t bits[kList];
    int32_t block[kList];
    int32_t part[kSparseWaves];
};
__device__ __forceinline__ int sparse_list(const SparseArgs& a, SparseList& s, int head, int i0, int i1, int tail, int split, int splits)
{
    const int tid = threadIdx.x, lane = tid & 63, wave = tid >> 6, words = (a.M + 63) / 64, n = a.n;
    const int w0 = i0 >> 6, w1 = i1 >> 6, shift = i0 & 63;
    const uint64_t keep = i1 - i0 >= 63 ? ~0ull : (1ull << (i1 - i0 + 1)) - 1;
    const uint64_t* sel = a.sel + (size_t)head * words * n;
    auto bits_of = [&](int b) {
        uint64_t x = sel[(size_t)w0 * n + b] >> shift;
        if (w1 != w0) x |= sel[(size_t)w1 * n + b] << (64 - shift);      // (w1 != w0: shift is not 0)
        return x & keep;
    };
    // how many there are: a thread counts neighbours
    const int per = (n + kSparseThreads - 1) / kSparseThreads, b0 = min(tid * per, n), b1 = min(b0 + per, n);
    int mine = 0;
    for (int b = b0; b < b1; ++b) mine += bits_of(b) != 0;
    int before = mine;
    for (int off = 1; off < 64; off *= 2) {
        const int o = __shfl_up(before, off);
        if (lane >= off) before += o;
    }
    if (lane == 63) s.part[wave] = before;
    __syncthreads();
    before -= mine;
    int all = 0;
    for (int w = 0; w < kSparseWaves; ++w) {
        if (w < wave) before += s.part[w];
        all += s.part[w];
    }
    const int total = all + tail, lo = (int)((int64_t)total * split / splits), hi = (int)((int64_t)total * (split + 1) / splits);
    if (before < hi && before + mine > lo)
        for (int b = b0; b < b1; ++b) {
            const uint64_t x = bits_of(b);
            if (x == 0) continue;
            if (before >= lo && before < hi) {
                s.bits[before - lo] = x;
                s.block[before - lo] = b;
            }
            ++before;
        }
    if (tid < tail && all + tid >= lo && all + tid < hi) {
        s.bits[all + tid - lo] = 0;
        s.block[all + tid - lo] = n + tid;
    }
    __syncthreads();
    return hi - lo;
}

// 32 keys, as a wavefront's operands: operand row r of half h is key 8 (r / 4) + 4 h + r % 4, so that a lane's 8 scores of a column
// are those of keys 8 g .. 8 g + 7, the probabilities it holds in the second product.
template <int D>
struct SparseUnit {
    half8 k[2][D / 32], v[D / 16];
    __device__ __forceinline__ void load(const SparseArgs& a, int head, int key0, int lane)
    {
        const int g = lane >> 4, col = lane & 15, total = a.kv_len + a.M;
        const half_t* kp = a.k + head * a.k_head + g * 8;
#pragma unroll
        for (int h = 0; h < 2; ++h)
#pragma unroll
            for (int s = 0; s < D / 32; ++s)
                k[h][s] = *(const half8*)(kp + (int64_t)min(key0 + 8 * (col >> 2) + 4 * h + (col & 3), total - 1) * a.k_tok + s * 32);
        const half_t* vp = a.v + head * a.v_head + min(key0 + 8 * g, (total - 1) & ~7);
#pragma unroll
        for (int ct = 0; ct < D / 16; ++ct) v[ct] = *(const half8*)(vp + (int64_t)(ct * 16 + col) * a.v_ch);
        if (key0 + 32 <= total) return;
        // rows that are not there may hold anything, and 0 times anything is no 0
        const int there = total - key0 - 8 * g;
#pragma unroll
        for (int ct = 0; ct < D / 16; ++ct) {
            uint4_ w = __builtin_bit_cast(uint4_, v[ct]);
#pragma unroll
            for (int p = 0; p < 4; ++p) w[p] &= (there > 2 * p ? 0xffffu : 0u) | (there > 2 * p + 1 ? 0xffff0000u : 0u);
            v[ct] = __builtin_bit_cast(half8, w);
        }
    }
};

// A row tile's state over the keys so far.
template <int D>
struct SparseState {
    floatx4 o[D / 16], l;              // l: the sum of the rounded probabilities, by a product with ones; four times the same
    float m;
    __device__ __forceinline__ void clear()
    {
        m = -INFINITY;
        l = (floatx4){0.f, 0.f, 0.f, 0.f};
#pragma unroll
        for (int ct = 0; ct < D / 16; ++ct) o[ct] = (floatx4){0.f, 0.f, 0.f, 0.f};
    }
    // scores (of the lane's 8 keys, c makes powers of two of them) to probabilities
    __device__ __forceinline__ half8 powers(const floatx4 (&s)[2], float c)
    {
        float top = s[0][0];
#pragma unroll
        for (int e = 1; e < 8; ++e) top = __builtin_elementwise_maximum(top, s[e >> 2][e & 3]);
        top = max_over_groups(top) * c;
        if (__ballot(top > m + 8.f || m == -INFINITY)) {
            const float now = top > m + 8.f || m == -INFINITY ? fmaxf(m, top) : m, r = m == now ? 1.f : fast_exp2(m - now);
            l *= r;
#pragma unroll
            for (int ct = 0; ct < D / 16; ++ct) o[ct] *= r;
            m = now;
        }
        const float off = m == -INFINITY ? 0.f : -m;
        half8 p;
#pragma unroll
        for (int e = 0; e < 8; ++e) p[e] = (half_t)fast_exp2(fmaf(s[e >> 2][e & 3], c, off));
        const half_t one = (half_t)1.f;
        l = __builtin_amdgcn_mfma_f32_16x16x32_f16((half8){one, one, one, one, one, one, one, one}, p, l, 0, 0, 0);
        return p;
    }
};

// The rows of a workgroup, and which of a unit's keys a row sees.
struct SparseRows {
    int row0, R, i0;
    __device__ __forceinline__ int token(const SparseArgs& a, int r, int col) const { return min((row0 + r * 16 + col) / a.rep, a.M - 1); }
    // a bit for each of the lane's 8 keys
    __device__ __forceinline__ uint32_t sees(const SparseArgs& a, const SparseList& list, const uint64_t* s_mask, int entry, int key0, int r,
                                             int lane) const
    {
        const int i = token(a, r, lane & 15);
        if (list.block[entry] < a.n) return list.bits[entry] >> (i - i0) & 1 ? 0xffu : 0u;
        return seen_keys((const uint32_t*)(s_mask + 2 * i), key0 + (lane >> 4) * 8, a.kv_len, a.kv_len + a.M);
    }
};

// One unit into the states.  PLAIN: every row meets all of the unit's values, those that it does not see with the
// probability 0; an infinity or NaN there is no 0 then.  Otherwise a row takes the values it sees, one by one.
template <int D, int RT, bool PLAIN>
__device__ __forceinline__ void sparse_unit(const SparseArgs& a, const SparseList& list, const uint64_t* s_mask, const SparseRows& rows, int head,
                                            const half8* s_q, SparseState<D> (&st)[RT], const SparseUnit<D>& u, int entry, int key0, float c,
                                            int lane)
{
#pragma unroll
    for (int r = 0; r < RT; ++r) {
        floatx4 s[2];
#pragma unroll
        for (int h = 0; h < 2; ++h) {
            s[h] = (floatx4){0.f, 0.f, 0.f, 0.f};
#pragma unroll
            for (int ks = 0; ks < D / 32; ++ks)
                s[h] = __builtin_amdgcn_mfma_f32_16x16x32_f16(u.k[h][ks], s_q[(r * (D / 32) + ks) * 64 + lane], s[h], 0, 0, 0);
        }
        const uint32_t see = rows.sees(a, list, s_mask, entry, key0, r, lane);
#pragma unroll
        for (int e = 0; e < 8; ++e) s[e >> 2][e & 3] = see >> e & 1 ? s[e >> 2][e & 3] : -INFINITY;
        const half8 p = st[r].powers(s, c);
        if constexpr (PLAIN) {
#pragma unroll
            for (int ct = 0; ct < D / 16; ++ct) st[r].o[ct] = __builtin_amdgcn_mfma_f32_16x16x32_f16(u.v[ct], p, st[r].o[ct], 0, 0, 0);
        } else {
            const int col = lane & 15, g = lane >> 4, total = a.kv_len + a.M;
            for (int key = 0; key < 32; ++key) {
                const int from = col + 16 * (key >> 3);
                float mine = 0.f;
#pragma unroll
                for (int e = 0; e < 8; ++e) mine = (key & 7) == e ? (float)p[e] : mine;
                const float pk = __shfl(mine, from);
                const bool seen = __shfl((int)see, from) >> (key & 7) & 1;
                if (!seen) continue;
                const half_t* vp = a.v + head * a.v_head + min(key0 + key, total - 1) + (int64_t)(4 * g) * a.v_ch;
#pragma unroll
                for (int ct = 0; ct < D / 16; ++ct)
#pragma unroll
                    for (int e = 0; e < 4; ++e) st[r].o[ct][e] += pk * (float)vp[(int64_t)(ct * 16 + e) * a.v_ch];
            }
        }
    }
}

// a row's output from the sums and their divisor; a row that sees no key gives zeros
__device__ __forceinline__ void sparse_out(const SparseArgs& a, int head, int row, int d, int ct, int g, floatx4 o, float l)
{
    const int token = row / a.rep;
    const float r = 1.f / l;
    half4 y;
#pragma unroll
    for (int e = 0; e < 4; ++e) y[e] = l == 0.f ? (half_t)0.f : (half_t)(o[e] * r);
    *(half4*)(a.out + ((size_t)token * a.nh + head * a.rep + row - token * a.rep) * d + ct * 16 + 4 * g) = y;
}

template <int D, int RT>
__global__ __launch_bounds__(kSparseThreads) void k_sparse_attention(SparseArgs a, SparseCut cut)
{
    constexpr int CT = D / 16, KS = D / 32, kRound = 8;
    __shared__ SparseList list;
    __shared__ uint64_t s_mask[2 * GHD_MAX_M];
    __shared__ half8 s_q[RT * KS * 64];
    __shared__ floatx2 s_ml[kSparseWaves][RT * 16];
    __shared__ floatx4 s_o[kSparseWaves][kRound][64];
    const int lane = threadIdx.x & 63, wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6), g = lane >> 4, col = lane & 15;
    const int split = blockIdx.x, block = blockIdx.y, head = blockIdx.z;
    SparseRows rows;
    rows.row0 = block * RT * 16;
    rows.R = a.M * a.rep;
    rows.i0 = rows.row0 / a.rep;
    const int tail0 = a.n * kBlock, tail = (a.kv_len + a.M - tail0 + kBlock - 1) / kBlock;
    if (wave == 0 && a.parent)
        store_masks(tree_nodes<2, true>(a.parent[min(lane, a.M - 1)], a.parent[min(lane + 64, a.M - 1)], a.M, lane), a.M, lane, s_mask);
    if (!a.parent)
        for (int e = threadIdx.x; e < 2 * a.M; e += kSparseThreads) s_mask[e] = a.mask[e];
    for (int f = wave; f < RT * KS; f += kSparseWaves) {
        const int row = rows.row0 + f / KS * 16 + col, token = row / a.rep;
        half8 x = {0, 0, 0, 0, 0, 0, 0, 0};
        if (row < rows.R) x = *(const half8*)(a.q + ((size_t)token * a.nh + head * a.rep + row - token * a.rep) * D + f % KS * 32 + g * 8);
        s_q[f * 64 + lane] = a.scale < 0.f ? -x : x;
    }
    const int count = sparse_list(a, list, head, rows.i0, min((rows.row0 + RT * 16 - 1) / a.rep, a.M - 1), tail, split, cut.splits);
    // scores to powers of two; above 0, so that minus infinity stays that
    const float c = fmaxf(fabsf(a.scale) * 1.4426950408889634f, 1e-37f);
    SparseState<D> st[RT];
#pragma unroll
    for (int r = 0; r < RT; ++r) st[r].clear();
    auto key_of = [&](int u) { return list.block[u >> 1] * kBlock + (u & 1) * 32; };
    auto pass = [&](auto plain) {
        for (int u = wave; u < 2 * count; u += kSparseWaves) {
            const int key0 = key_of(u);
            if (key0 >= a.kv_len + a.M) continue;
            SparseUnit<D> unit;
            unit.load(a, head, key0, lane);
            sparse_unit<D, RT, decltype(plain)::value>(a, list, s_mask, rows, head, s_q, st, unit, u >> 1, key0, c, lane);
        }
    };
    pass(std::true_type{});
    bool odd = false;
#pragma unroll
    for (int r = 0; r < RT; ++r)
#pragma unroll
        for (int ct = 0; ct < CT; ++ct)
#pragma unroll
            for (int e = 0; e < 4; ++e) odd = odd || !(fabsf(st[r].o[ct][e]) < INFINITY);
    if (__ballot(odd)) {
#pragma unroll
        for (int r = 0; r < RT; ++r) st[r].clear();
        pass(std::false_type{});
    }
    // the wavefronts' states meet in LDS, some fragments at a time
    if (g == 0)
#pragma unroll
        for (int r = 0; r < RT; ++r) s_ml[wave][r * 16 + col] = (floatx2){st[r].m, st[r].l[0]};
    const size_t unit = (((size_t)head * cut.blocks + block) * cut.splits + split) * RT;
#pragma unroll
    for (int f0 = 0; f0 < RT * CT; f0 += kRound) {
        __syncthreads();
#pragma unroll
        for (int f = 0; f < kRound && f0 + f < RT * CT; ++f) s_o[wave][f][lane] = st[(f0 + f) / CT].o[(f0 + f) % CT];
        __syncthreads();
        for (int f = f0 + wave; f < f0 + kRound && f < RT * CT; f += kSparseWaves) {
            const int r = f / CT, ct = f % CT, row = rows.row0 + r * 16 + col;
            float m = -INFINITY, l = 0.f;
            floatx4 o = {0.f, 0.f, 0.f, 0.f};
            for (int w = 0; w < kSparseWaves; ++w) m = fmaxf(m, s_ml[w][r * 16 + col][0]);
            for (int w = 0; w < kSparseWaves; ++w) {
                const floatx2 ml = s_ml[w][r * 16 + col];
                const float by = fast_exp2(ml[0] - (m == -INFINITY ? 0.f : m));
                l += ml[1] * by;
                o += s_o[w][f - f0][lane] * by;
            }
            if (cut.splits > 1) {
                ((floatx4*)a.o_part)[((unit + r) * CT + ct) * 64 + lane] = o;
                if (ct == 0 && g == 0) ((floatx2*)a.ml_part)[(unit + r) * 16 + col] = (floatx2){m, l};
            } else if (row < rows.R) {
                sparse_out(a, head, row, D, ct, g, o, l);
            }
        }
    }
}

// Parts to rows: a wavefront has a fragment, 16 channels by 16 rows, and its parts in order.
template <int D>
__global__ __launch_bounds__(256) void k_sparse_join(SparseArgs a, SparseCut cut)
{
    constexpr int CT = D / 16;
    const int lane = threadIdx.x & 63, f = blockIdx.x * 4 + (threadIdx.x >> 6), g = lane >> 4, col = lane & 15;
    const int ct = f % CT, rt = f / CT, head = blockIdx.z, block = blockIdx.y, row = (block * cut.rows + rt) * 16 + col;
    if (rt >= cut.rows) return;
    const size_t unit0 = ((size_t)head * cut.blocks + block) * cut.splits;
    float m = -INFINITY, l = 0.f;
    floatx4 o = {0.f, 0.f, 0.f, 0.f};
    for (int p = 0; p < cut.splits; ++p) {
        const size_t unit = (unit0 + p) * cut.rows + rt;
        const floatx2 ml = ((const floatx2*)a.ml_part)[unit * 16 + col];
        const floatx4 v = ((const floatx4*)a.o_part)[(unit * CT + ct) * 64 + lane];
        const float now = fmaxf(m, ml[0]), off = now == -INFINITY ? 0.f : now, was = fast_exp2(m - off), by = fast_exp2(ml[0] - off);
        l = l * was + ml[1] * by;
        o = o * was + v * by;
        m = now;
    }
    if (row < a.M * a.rep) sparse_out(a, head, row, D, ct, g, o, l);
}

static SparseCut sparse_cut(int M, int kv_len, int nh, int nkv, int d)
{
    const int tiles = ceil_div(M * (nh / nkv), 16), rows = tiles == 1 ? 1 : 2, blocks = ceil_div(tiles, rows), n = kv_len / kBlock;
    const int most = n + ceil_div(kv_len + M - n * kBlock, kBlock);      // blocks that a row can read
    const int splits = std::max(ceil_div(most, kList), std::min(most, std::max(1, 512 / (nkv * blocks))));
    return {rows, blocks, splits};
}

static size_t sparse_units(const SparseCut& c, int nkv) { return c.splits == 1 ? 0 : (size_t)nkv * c.blocks * c.splits * c.rows; }
static size_t sparse_o_bytes(size_t units, int d) { return align_up(units * 16 * d * 4, 256); }
static size_t sparse_bytes(size_t units, int d) { return std::max<size_t>(256, sparse_o_bytes(units, d) + align_up(units * 128, 256)); }

// The most that a call of up to M tokens over up to kv_len rows takes, whatever its cut: parts are at most 512 workgroups of two
// tiles of rows and a part reads a block, or as many as a list's length makes of them.
size_t sparse_attention_bytes(int M, int kv_len, int nh, int nkv, int d)
{
    const size_t tiles = ceil_div(M * (nh / nkv), 16) + 1, most = kv_len / kBlock + 1 + ceil_div(M, kBlock);
    return sparse_bytes(std::max(std::min<size_t>(1024, nkv * tiles * most), most > kList ? nkv * tiles * ((most + kList - 1) / kList) : 0), d);
}

template <int D>
static ghd_status sparse_of(const SparseArgs& a, const SparseCut& c, hipStream_t st)
{
    const dim3 grid(c.splits, c.blocks, a.nkv);
    if (c.rows == 1) hipLaunchKernelGGL((k_sparse_attention<D, 1>), grid, dim3(kSparseThreads), 0, st, a, c);
    else hipLaunchKernelGGL((k_sparse_attention<D, 2>), grid, dim3(kSparseThreads), 0, st, a, c);
    const ghd_status s = check_launch();
    if (s || c.splits == 1) return s;
    hipLaunchKernelGGL(k_sparse_join<D>, dim3(ceil_div(c.rows * (D / 16), 4), c.blocks, a.nkv), dim3(256), 0, st, a, c);
    return check_launch();
}

ghd_status launch_sparse_attention(SparseArgs a, int d, void* ws, size_t ws_bytes, hipStream_t st)
{
    const SparseCut c = sparse_cut(a.M, a.kv_len, a.nh, a.nkv, d);
    if (ws_bytes < sparse_bytes(sparse_units(c, a.nkv), d)) return GHD_ERR_WORKSPACE;
    a.rep = a.nh / a.nkv;
    a.n = a.kv_len / kBlock;
    a.o_part = (float*)ws;
    a.ml_part = (float*)((char*)ws + sparse_o_bytes(sparse_units(c, a.nkv), d));
    return d == 128 ? sparse_of<128>(a, c, st) : sparse_of<64>(a, c, st);
}

}  // namespace ghd
