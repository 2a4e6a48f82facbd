// Acceptance of drafted tokens against the target's probabilities from given random numbers (include/ghd.h has the rule).
//
// Every node is judged at once as if the walk came there: k_sample_rows leaves maxima and sums of softmax weights of the rows' segments,
// k_sample_nodes which child of each node is accepted, or which token is drawn there; its last workgroup goes from the root down.
// Where drafts have probabilities, k_sample_first tries every node's first child, which takes no more than the rows' sums; that leaves
// few nodes that the walk can come to, and of those k_sample_rest sums up what a first rejection leaves, over the segments again,
// and keeps the weights where there may be others.
//
// Weights exp((l - m) / T) have arguments in 64 bits and 24 bits themselves, and so has what rejections leave of each; sums are 64 bits.  So a sum over a row is off by some
// 2^-24 / sqrt(V) of its largest terms, by random roundings of single weights, and what 64 bits would accept or draw is
// what is accepted or drawn but where a random number lies as close to a border: of 17500 calls over 32000 to 131072 tokens two drew
// another token, a neighbour.
#include "sparse.h"
#include "wave.h"

#include <type_traits>

namespace ghd {

constexpr int kSegment = 4096;                   // logits of a row that a workgroup takes
constexpr int kRowThreads = 256, kPerThread = kSegment / kRowThreads;
constexpr int kNodeThreads = 512, kNodeWaves = kNodeThreads / 64, kSide = kSegment / kNodeThreads;
constexpr int kMaxSegments = 64;                 // of the largest vocabulary, 262144
constexpr int kAtOnce = 8;                       // segments whose kept weights a node's workgroup asks for
constexpr double kLog2e = 1.4426950408889634;

// Softmax weights of a row: 2^((l - m) c), c = log2 e / T.  NaN and minus infinity have none; where the maximum is
// infinity only such logits have one.
struct Weights {
    double c, from;
    float top;
    __device__ __forceinline__ Weights(float m, double c) : c(c), from((double)m), top(m) {}
    // (The difference is exact, or all but: l c - m c in one instruction is off by 2^-53 of m c, which at a temperature of 1e-15 is
    // no small exponent.  fmax takes the number of a number and NaN; 2^-1100 is 0.)
    __device__ __forceinline__ double exponent(float l) const { return fmax(((double)l - from) * c, -1100.0); }
    __device__ __forceinline__ double operator()(float l) const
    {
        if (!(fabsf(top) < INFINITY)) return top > 0.f && l == top ? 1.0 : 0.0;
        const double x = exponent(l), n = rint(x);
        return ldexp((double)__builtin_amdgcn_exp2f((float)(x - n)), (int)n);
    }
    // in 32 bits' range
    __device__ __forceinline__ float low(float l) const
    {
        if (!(fabsf(top) < INFINITY)) return top > 0.f && l == top ? 1.f : 0.f;
        const double x = exponent(l), n = rint(x);
        return ldexpf(__builtin_amdgcn_exp2f((float)(x - n)), (int)n);
    }
};

// What the first loads need comes in the first twelve words of the arguments, which the hardware puts into scalar registers before a
// kernel starts; the argument block, host memory, is 0.6 us away.
#define SAMPLE_FIRST(FIFTH) const float *logits, const int32_t *tokens, const int32_t *parent, const float *u, FIFTH, int M, int V
__device__ __forceinline__ void sample_first(SampleArgs& a, const float* logits, const int32_t* tokens, const int32_t* parent, const float* u, int M, int V)
{
    a.logits = logits;
    a.tokens = tokens;
    a.parent = parent;
    a.u = u;
    a.M = M;
    a.V = V;
}

struct Segment {
    double sum;                                  // of weights against the segment's maximum
    float top, unused;
};
struct Rest {
    double p, q;                                 // what the first rejection leaves: sums of max(p - q, 0) and q without the token
};
struct First {
    double one, one_q;                           // one over the sums of the target's and the draft's row, 0 where those are
    float top, top_q;                            // their maxima
    int child, accepted;                         // the first child whose token is in the vocabulary, or GHD_MAX_M
    int reached;                                 // k_sample_rest's, where it is not accepted: whether the walk can come to the node
    int more;                                    // whether there is a second such child
};

// Node c as a child: asked for before it is known whose child it is.
struct Child {
    int c, parent, token;
    __device__ __forceinline__ Child(const SampleArgs& a, int c) : c(c), parent(a.parent[min(c, a.M - 1)]), token(a.tokens[min(c, a.M - 1)]) {}
    __device__ __forceinline__ bool of(const SampleArgs& a, int node) const { return c > node && c < a.M && parent == node; }
};
__device__ __forceinline__ bool in_vocabulary(const SampleArgs& a, int t) { return t >= 0 && t < a.V; }
__device__ __forceinline__ double u_of(float u) { return u > 0.f ? (double)u : 0.0; }
__device__ __forceinline__ int draft_row(const SampleArgs& a, int node)
{
    return a.q_row ? min(max(a.q_row[node], 0), a.q_rows - 1) : node;
}

// A row's maximum and one over its sum, from its segments' (a lane has one); 0 where no token has a weight.
struct RowSum {
    float top, mine;                             // mine: the lane's segment's
    double one, part;                            // part: the lane's segment's sum against the row's maximum
    __device__ __forceinline__ RowSum(const Segment* seg, int segments, int lane, double c)
    {
        Segment s = {0.0, -INFINITY, 0.f};
        if (lane < segments) s = seg[lane];
        mine = s.top;
        top = wave_highest(s.top);
        part = s.sum * Weights(top, c)(s.top);
        double sum = wave_sum(part);
        asm volatile("" : "+v"(top), "+v"(sum));     // (known to be uniform they cost k_sample_nodes' loop of rejections 106 spilled registers)
        one = sum > 0.0 ? 1.0 / sum : 0.0;
    }
};

// Target rows (blockIdx.y < M), without the tokens of the node's children where drafts have no probabilities; draft rows.
// Bound: the bytes of the logits: 256 rows of 131072 24.2 us (5.5 TB/s, some of it out of the 256 MB cache); 64 rows of 32000, 8 MB, 5.4 us.
__global__ __launch_bounds__(kRowThreads) void k_sample_rows(SAMPLE_FIRST(const float* q_logits), SampleArgs a, Segment* __restrict__ seg,
                                                             uint32_t* __restrict__ arrived)
{
    sample_first(a, logits, tokens, parent, u, M, V);
    a.q_logits = q_logits;
    __shared__ uint32_t s_out[kSegment / 32];
    __shared__ double s_sum[kRowThreads / 64];
    __shared__ float s_top[kRowThreads / 64];
    const int tid = threadIdx.x, y = blockIdx.y, lo = blockIdx.x * kSegment, segments = gridDim.x;
    if (y == 0 && blockIdx.x == 0 && tid == 0) *arrived = 0;
    const bool target = y < a.M;
    const float* row = (target ? a.logits + (size_t)y * a.V : a.q_logits + (size_t)(y - a.M) * a.V) + lo;
    const int n = min(a.V - lo, kSegment);
    const double c = kLog2e / (double)(target ? a.temperature : a.q_temperature);
    const Child child(a, tid);
    float l[kPerThread];
    // four neighbours a load where the row allows it
    const bool wide = ((uintptr_t)row & 15) == 0 && n == kSegment;
    if (wide) {
#pragma unroll
        for (int i = 0; i < kPerThread / 4; ++i) {
            const floatx4 v = ((const floatx4*)row)[i * kRowThreads + tid];
#pragma unroll
            for (int e = 0; e < 4; ++e) l[4 * i + e] = v[e];
        }
    } else {
#pragma unroll
        for (int i = 0; i < kPerThread; ++i) {
            const int t = (i / 4 * kRowThreads + tid) * 4 + i % 4;
            l[i] = t < n ? row[t] : -INFINITY;
        }
    }
    if (target && !a.q_logits) {
        if (tid < kSegment / 32) s_out[tid] = 0;
        __syncthreads();
        bool any = false;
        if (tid < GHD_MAX_M && child.of(a, y)) {
            const int t = child.token;
            any = t >= lo && t < lo + kSegment;
            if (any) atomicOr(&s_out[(t - lo) >> 5], 1u << ((t - lo) & 31));
        }
        if (__syncthreads_or(any))
#pragma unroll
            for (int i = 0; i < kPerThread; ++i) {
                const int t = (i / 4 * kRowThreads + tid) * 4 + i % 4;
                if (s_out[t >> 5] >> (t & 31) & 1) l[i] = -INFINITY;
            }
    }
    float top = -INFINITY;
#pragma unroll
    for (int i = 0; i < kPerThread; ++i) top = fmaxf(top, l[i]);
    top = wave_highest(top);
    if ((tid & 63) == 0) s_top[tid >> 6] = top;
    __syncthreads();
#pragma unroll
    for (int w = 0; w < kRowThreads / 64; ++w) top = fmaxf(top, s_top[w]);
    const Weights weight(top, c);
    double sum = 0.0;
#pragma unroll
    for (int i = 0; i < kPerThread; ++i) sum += (double)weight.low(l[i]);
    sum = running_sum(sum);
    if ((tid & 63) == 63) s_sum[tid >> 6] = sum;
    __syncthreads();
    if (tid == 0) {
        sum = 0.0;
        for (int w = 0; w < kRowThreads / 64; ++w) sum += s_sum[w];
        seg[(size_t)y * segments + blockIdx.x] = {sum, top, 0.f};
    }
}

// A wavefront a node: its rows' sums, and whether its first child is accepted.  Bound: three loads that follow one another, 3.7 us.
__global__ __launch_bounds__(64) void k_sample_first(SAMPLE_FIRST(const Segment* __restrict__ seg), SampleArgs a, int segments, First* __restrict__ out)
{
    sample_first(a, logits, tokens, parent, u, M, V);
    const int lane = threadIdx.x, node = blockIdx.x, qr = draft_row(a, node);
    const Child low(a, lane), high(a, lane + 64);
    const double c = kLog2e / (double)a.temperature, cq = kLog2e / (double)a.q_temperature;
    const uint64_t in_low = __ballot(low.of(a, node) && in_vocabulary(a, low.token)), in_high = __ballot(high.of(a, node) && in_vocabulary(a, high.token));
    const int at = in_low ? (int)__builtin_ctzll(in_low) : in_high ? (int)__builtin_ctzll(in_high) : 0;
    const int x = __shfl(in_low ? low.token : high.token, at), child = in_low ? at : in_high ? at + 64 : GHD_MAX_M;
    float lp = 0.f, lq = 0.f, number = 0.f;
    if (child < GHD_MAX_M) {
        lp = a.logits[(size_t)node * a.V + x];
        lq = a.q_logits[(size_t)qr * a.V + x];
        number = a.u[child];
    }
    const RowSum p(seg + (size_t)node * segments, segments, lane, c), q(seg + (size_t)(a.M + qr) * segments, segments, lane, cq);
    if (lane != 0) return;
    const double px = Weights(p.top, c)(lp) * p.one, qx = Weights(q.top, cq)(lq) * q.one;
    out[node] = {p.one, q.one, p.top, q.top, child, child < GHD_MAX_M && u_of(number) * qx < px, 0, __popcll(in_low) + __popcll(in_high) > 1};
}

// Can the walk come to a node?  By what its ancestors' first children are: accepted, no other child of theirs is tried, rejected, not
// they.  All threads of a workgroup (128 or more), pointers doubled.
struct Reach {
    int up[GHD_MAX_M], lost[GHD_MAX_M];
};
__device__ __forceinline__ bool can_be_reached(const SampleArgs& a, const First* first, int node, Reach& s)
{
    const int i = threadIdx.x;
    int up = -1, lost = 0;
    if (i < a.M) {
        const int p = a.parent[i];
        if (p >= 0 && p < i) {
            up = p;
            lost = (first[p].child == i) != (first[p].accepted != 0);
        } else {
            lost = i != 0;
        }
    }
    while (__syncthreads_or(up >= 0)) {
        if (i < GHD_MAX_M) {
            s.up[i] = up;
            s.lost[i] = lost;
        }
        __syncthreads();
        if (up >= 0) {
            lost |= s.lost[up];
            up = s.up[up];
        }
    }
    if (i < GHD_MAX_M) s.lost[i] = lost;
    __syncthreads();
    return s.lost[node] == 0;
}

// Kept weights: [node][segment][target, draft][kSegment]
__host__ __device__ __forceinline__ size_t kept_at(int node, int segments, int segment) { return ((size_t)node * segments + segment) * 2 * kSegment; }

// What is left of a segment when the first child of a node is rejected: then beta is 1.  Where there are other children, the weights against
// the rows' maxima are kept, 0 for the rejected token: another rejection goes over all of them in one workgroup.
// Bound: a launch's time (64 nodes of 32000: 3.1 us).  A chain of 128 nodes, 131072 tokens: 8.0 us, of which the exponentials, one node's in 32
// workgroups, are half at most: every rejected node's 32 workgroups first work out whether the walk can come there, and rows are asked for
// behind that.
__global__ __launch_bounds__(kRowThreads) void k_sample_rest(SampleArgs a, First* firsts, Rest* __restrict__ rest, float* __restrict__ kept)
{
    __shared__ Reach s_reach;
    __shared__ double s_sum[2][kRowThreads / 64];
    const int tid = threadIdx.x, lane = tid & 63, node = blockIdx.y, lo = blockIdx.x * kSegment, segments = gridDim.x;
    const First first = firsts[node];
    if (first.accepted || (first.child == GHD_MAX_M && blockIdx.x != 0)) return;
    const bool reached = can_be_reached(a, firsts, node, s_reach);
    if (blockIdx.x == 0 && tid == 0) firsts[node].reached = reached;
    if (first.child == GHD_MAX_M || !reached) return;
    const int x = a.tokens[first.child], qr = draft_row(a, node);
    const float *row = a.logits + (size_t)node * a.V, *q_row = a.q_logits + (size_t)qr * a.V;
    const int n = min(a.V - lo, kSegment);
    float lp[kPerThread], lq[kPerThread];
#pragma unroll
    for (int i = 0; i < kPerThread; ++i) {
        const int t = lo + min(i * kRowThreads + tid, n - 1);
        lp[i] = row[t];
        lq[i] = q_row[t];
    }
    const Weights wp(first.top, kLog2e / (double)a.temperature), wq(first.top_q, kLog2e / (double)a.q_temperature);
    double s = 0.0, r = 0.0;
    float* const keep = kept + kept_at(node, segments, blockIdx.x) + tid;
#pragma unroll
    for (int i = 0; i < kPerThread; ++i) {
        const int t = i * kRowThreads + tid;
        const bool is = t < n && lo + t != x;
        const double pw = is ? wp(lp[i]) : 0.0, qw = is ? wq(lq[i]) : 0.0, qt = qw * first.one_q;
        s += fmax(pw * first.one - qt, 0.0);
        r += qt;
        if (first.more) {
            keep[i * kRowThreads] = (float)pw;
            keep[kSegment + i * kRowThreads] = (float)qw;
        }
    }
    s = running_sum(s);
    r = running_sum(r);
    if (lane == 63) {
        s_sum[0][tid >> 6] = s;
        s_sum[1][tid >> 6] = r;
    }
    __syncthreads();
    if (tid == 0) {
        Rest all = {0.0, 0.0};
        for (int w = 0; w < kRowThreads / 64; ++w) {
            all.p += s_sum[0][w];
            all.q += s_sum[1][w];
        }
        rest[(size_t)node * segments + blockIdx.x] = all;
    }
}

// What a node's workgroup shares.
struct NodeShared {
    int child[GHD_MAX_M], token[GHD_MAX_M], kids, taken, final, place[kNodeWaves], last[kNodeWaves];
    double u0, u[GHD_MAX_M], weight[GHD_MAX_M], part[2][kNodeWaves], sums[kMaxSegments][kNodeWaves], p[GHD_MAX_M], q[GHD_MAX_M];
    uint32_t out[kMaxSegments * kSegment / 32];  // a bit for each token that has been rejected
    __device__ __forceinline__ bool rejected(int t) const { return out[t >> 5] >> (t & 31) & 1; }
};

// The token at which the running sum of weights passes u[0] of all.  part: what the lane's segment has in all (each wavefront has
// them all); weight(t): a token's.  Called by all threads; thread 0 has the result, -1 where no token has a weight.
template <class Weight>
__device__ __forceinline__ int draw_from_segments(const SampleArgs& a, NodeShared& s, double part, int segments, const Weight& weight)
{
    const int tid = threadIdx.x, lane = tid & 63, wave = tid >> 6;
    const double upto = running_sum(part);
    const double goal = s.u0 * lane_of(upto, 63);
    const uint64_t over = __ballot(part > 0.0 && upto > goal), some = __ballot(part > 0.0);
    if (some == 0) return -1;
    const int at = __builtin_amdgcn_readfirstlane(over ? (int)__builtin_ctzll(over) : 63 - (int)__builtin_clzll(some));
    // a thread has some neighbours of it
    double w[kSide], sum = 0.0;
#pragma unroll
    for (int e = 0; e < kSide; ++e) {
        const int t = at * kSegment + tid * kSide + e;
        w[e] = t < a.V ? weight(t) : 0.0;
        sum += w[e];
    }
    const double run = running_sum(sum);
    __syncthreads();
    if (lane == 63) s.part[0][wave] = run;
    __syncthreads();
    double before = (at > 0 ? lane_of(upto, max(at - 1, 0)) : 0.0) + run - sum;
    for (int v = 0; v < wave; ++v) before += s.part[0][v];
    // the first that passes, or the last that has a weight (the segment's own sum was larger by a rounding)
    int first = 0x7fffffff, last = -1;
#pragma unroll
    for (int e = 0; e < kSide; ++e) {
        before += w[e];
        if (!(w[e] > 0.0)) continue;
        last = at * kSegment + tid * kSide + e;
        if (before > goal && first == 0x7fffffff) first = last;
    }
    first = -wave_highest(-first);
    last = wave_highest(last);
    if (lane == 0) {
        s.place[wave] = first;
        s.last[wave] = last;
    }
    __syncthreads();
    for (int v = 0; v < kNodeWaves; ++v) {
        first = min(first, s.place[v]);
        last = max(last, s.last[v]);
    }
    return first != 0x7fffffff ? first : last;
}

// A node's result - the accepted child or -1, and the token drawn where there is none - and, from the workgroup that is last to have
// one, the walk.  Results and their count are atomics of the device's scope, which pass the XCDs' own caches; a workgroup counts itself when
// its result has been acknowledged.  (A launch of its own for the walk: 3 us of the host and as much of the GPU.)
__device__ __forceinline__ void node_is_done(const SampleArgs& a, NodeShared& s, uint64_t* nodes, uint32_t* arrived, int node, int taken, int token)
{
    const int tid = threadIdx.x;
    __syncthreads();                             // (all of it is done with the inputs, where the result may be written)
    if (tid == 0) {
        __hip_atomic_store(nodes + node, (uint64_t)(uint32_t)token << 32 | (uint32_t)taken, __ATOMIC_RELAXED, __HIP_MEMORY_SCOPE_AGENT);
        asm volatile("s_waitcnt vmcnt(0)" ::: "memory");
        s.final = __hip_atomic_fetch_add(arrived, 1u, __ATOMIC_RELAXED, __HIP_MEMORY_SCOPE_AGENT) == (uint32_t)a.M - 1;
    }
    __syncthreads();
    if (!s.final) return;
    if (tid < a.M) {
        const uint64_t r = __hip_atomic_load(nodes + tid, __ATOMIC_RELAXED, __HIP_MEMORY_SCOPE_AGENT);
        s.child[tid] = (int)(uint32_t)r;
        s.token[tid] = (int)(r >> 32);
    }
    __syncthreads();
    if (tid != 0) return;
    int at = 0, len = 1;
    a.res[2] = 0;
    // (a child comes after its node and is one of the tree's: at most M steps, whatever nodes hold that the walk does not come to)
    for (; s.child[at] > at && s.child[at] < a.M; ++len) {
        at = s.child[at];
        a.res[2 + len] = at;
    }
    a.res[0] = len;
    a.res[1] = s.token[at];
}

// One workgroup a node.  DRAFTS: they have probabilities.  Bound: what follows one another.  64 nodes, 32000 tokens: 8.0 us, with draft
// probabilities 6.7 where no second child is rejected.  Each that is takes a pass over the kept weights: 2 us at 8000 tokens,
// 3.9 at 32000 (256 KB), 9.2 at 131072 (1 MB), read and summed up by one compute unit.  In registers up to 32768 tokens'
// weights took 10% less of many rejections, and 15% more at 8000 tokens.
template <bool DRAFTS>
__global__ __launch_bounds__(kNodeThreads) void k_sample_nodes(SAMPLE_FIRST(const Segment* __restrict__ seg), SampleArgs a, const First* __restrict__ firsts,
                                                               const Rest* __restrict__ rest, float* kept, int segments, uint64_t* nodes, uint32_t* arrived)
{
    sample_first(a, logits, tokens, parent, u, M, V);
    __shared__ NodeShared s;
    const int tid = threadIdx.x, lane = tid & 63, wave = tid >> 6, node = blockIdx.x;
    if constexpr (DRAFTS) {
        if (firsts[node].accepted) return node_is_done(a, s, nodes, arrived, node, firsts[node].child, -1);
        if (!firsts[node].reached) return node_is_done(a, s, nodes, arrived, node, -1, -1);
    }
    const float* row = a.logits + (size_t)node * a.V;
    const double c = kLog2e / (double)a.temperature;
    // children, in order
    if (wave == 0) {
        const Child some[2] = {Child(a, lane), Child(a, lane + 64)};
        const float u[2] = {a.u[min(lane, a.M - 1)], a.u[min(lane + 64, a.M - 1)]};
        int n = 0;
#pragma unroll
        for (int h = 0; h < 2; ++h) {
            const bool is = some[h].of(a, node);
            const uint64_t with = __ballot(is);
            if (is) {
                const int k = n + __popcll(with & ((1ull << lane) - 1));
                s.child[k] = some[h].c;
                s.token[k] = some[h].token;
                s.u[k] = u_of(u[h]);
            }
            n += __popcll(with);
        }
        if (lane == 0) {
            s.kids = n;
            s.u0 = u_of(u[0]);
        }
    }
    for (int i = tid; i < (a.V + 31) / 32; i += kNodeThreads) s.out[i] = 0;
    const RowSum p(seg + (size_t)node * segments, segments, lane, c);
    __syncthreads();
    const int kids = s.kids;
    auto twice = [&](int k) {                    // whether child k's token was an earlier child's
        bool is = false;
        for (int j = 0; j < k; ++j) is = is || s.token[j] == s.token[k];
        return is;
    };
    auto finish = [&](int taken, int token) { node_is_done(a, s, nodes, arrived, node, taken, token); };

    if constexpr (!DRAFTS) {
        // A child is accepted if u (what is left) < its weight.  What is left before a child: the tokens that no child has, and the
        // weights of this child and those after it.
        if (wave == 0) {
            float top = p.top;
            for (int k = lane; k < kids; k += 64)
                if (in_vocabulary(a, s.token[k])) top = fmaxf(top, row[s.token[k]]);
            top = wave_highest(top);
            const Weights weight(top, c);
            const double others = p.one > 0.0 ? weight(p.top) / p.one : 0.0;
            for (int k = lane; k < kids; k += 64)
                s.weight[k] = in_vocabulary(a, s.token[k]) && !twice(k) ? weight(row[s.token[k]]) : 0.0;
            __builtin_amdgcn_fence(__ATOMIC_ACQ_REL, "wavefront");
            int first = GHD_MAX_M;
            for (int k = lane; k < kids; k += 64) {
                double left = others;
                for (int j = kids - 1; j >= k; --j) left += s.weight[j];
                if (s.u[k] * left < s.weight[k]) first = min(first, k);
            }
            first = -wave_highest(-first);
            if (lane == 0) s.taken = first < GHD_MAX_M ? s.child[first] : -1;
        }
        __syncthreads();
        if (s.taken >= 0) return finish(s.taken, -1);
        if (tid < kids && in_vocabulary(a, s.token[tid])) atomicOr(&s.out[s.token[tid] >> 5], 1u << (s.token[tid] & 31));
        __syncthreads();
        const Weights weight(p.top, c);
        const int token = draw_from_segments(a, s, p.part, segments, [&](int t) { return s.rejected(t) ? 0.0 : weight(row[t]); });
        return finish(-1, token);
    } else {
        const Weights wp(p.top, c);
        if (kids == 0) {
            const int token = draw_from_segments(a, s, p.part, segments, [&](int t) { return wp(row[t]); });
            return finish(-1, token);
        }
        // After some rejections what is left is alpha (p - beta q)+ of the tokens not rejected, and what is left of q its other tokens:
        // two sums over the row for each rejection.
        const int qr = draft_row(a, node);
        const float* q_row = a.q_logits + (size_t)qr * a.V;
        const double cq = kLog2e / (double)a.q_temperature;
        const First q = firsts[node];
        const Weights wq(q.top_q, cq);
        auto p_of = [&](int t) { return wp(row[t]) * p.one; };
        auto q_of = [&](int t) { return wq(q_row[t]) * q.one_q; };
        // the children's own, nothing of a token that an earlier child has
        if (tid < kids) {
            const int x = s.token[tid];
            const bool is = in_vocabulary(a, x) && !twice(tid);
            s.p[tid] = is ? p_of(x) : 0.0;
            s.q[tid] = is ? q_of(x) : 0.0;
        }
        __syncthreads();
        // Weights in 32 bits, 0 of what was rejected, are there if a second child is; where less is left than
        // those show, they are worked out anew each time, in 64 bits' range.  In units of the target's weights what is left of a token is p - by q; `by` in two parts.
        float* const w = kept + kept_at(node, segments, 0);
        struct Left {
            float high, low;
            __device__ __forceinline__ Left(double by) : high((float)by), low((float)(by - (double)high)) {}
            __device__ __forceinline__ float operator()(float pw, float qw) const { return fmaxf(fmaf(-low, qw, fmaf(-high, qw, pw)), 0.f); }
        };
        // to(v, left, left_q): a thread's share of segment v, two times four neighbours of either row, q's if it is to be summed; eight segments are
        // asked for at a time
        auto over_kept = [&](double by, bool sum_q_too, auto to) {
            const Left left(by);
            for (int v0 = 0; v0 < segments; v0 += kAtOnce) {
                floatx4 has[kAtOnce][4];
                const floatx4* from = (const floatx4*)(w + kept_at(0, segments, v0)) + tid;
#pragma unroll
                for (int i = 0; i < kAtOnce; ++i) {
                    if (v0 + i >= segments) continue;
#pragma unroll
                    for (int f = 0; f < 4; ++f) has[i][f] = from[i * (2 * kSegment / 4) + f * kNodeThreads];
                }
                __builtin_amdgcn_sched_barrier(0);
#pragma unroll
                for (int i = 0; i < kAtOnce; ++i) {
                    if (v0 + i >= segments) continue;
                    double sum = 0.0, sum_q = 0.0;
#pragma unroll
                    for (int e = 0; e < kSide; ++e) sum += (double)left(has[i][e / 4][e % 4], has[i][2 + e / 4][e % 4]);
                    if (sum_q_too)
#pragma unroll
                        for (int e = 0; e < kSide; ++e) sum_q += (double)has[i][2 + e / 4][e % 4];
                    to(v0 + i, sum, sum_q);
                }
            }
        };
        bool shows = q.more;
        double alpha = 1.0, beta = 0.0, rest_q = q.one_q > 0.0 ? 1.0 : 0.0;
        Rest first = {0.0, 0.0};                 // the lane's segment's, of what the first rejection leaves
        int tried = 0, k = 0;
        for (; k < kids; ++k) {
            const int x = s.token[k];
            if (!in_vocabulary(a, x)) continue;
            const double px = fmax(alpha * (s.p[k] - beta * s.q[k]), 0.0), qx = rest_q > 0.0 ? s.q[k] / rest_q : 0.0;
            if (s.u[k] * qx < px) break;
            __syncthreads();                     // (the last round's bits and sums have been read)
            if (tid == 0) {
                s.out[x >> 5] |= 1u << (x & 31);
                if (q.more) w[kept_at(0, segments, x / kSegment) + x % kSegment] = w[kept_at(0, segments, x / kSegment) + kSegment + x % kSegment] = 0.f;
            }
            __syncthreads();
            const double next = rest_q > 0.0 ? beta + 1.0 / (alpha * rest_q) : beta;
            double all, all_q;
            if (tried++ == 0 && rest_q > 0.0) {
                if (lane < segments) first = rest[(size_t)node * segments + lane];
                all = wave_sum(first.p);
                all_q = wave_sum(first.q);
                asm volatile("" : "+v"(all), "+v"(all_q));
            } else {
                // What is left of q follows from what was: off by 2^-53 of the whole for each rejection, 2^-36 of a thousandth at the most.  Where less
                // is left it is summed up.
                const double without = rest_q - s.q[k];
                const bool follows = without > 1e-3;
                for (;;) {
                    double sp = 0.0, sq = 0.0;
                    if (shows) {
                        over_kept(next * q.one_q / p.one, !follows, [&](int, double left, double left_q) {
                            sp += left;
                            sq += left_q;
                        });
                        sp *= p.one;
                        sq *= q.one_q;
                    } else {
                        for (int t = tid; t < a.V; t += kNodeThreads) {
                            if (s.rejected(t)) continue;
                            const double qt = q_of(t);
                            sp += fmax(p_of(t) - next * qt, 0.0);
                            sq += qt;
                        }
                    }
                    sp = running_sum(sp);
                    if (!follows) sq = running_sum(sq);
                    if (lane == 63) {
                        s.part[0][wave] = sp;
                        s.part[1][wave] = sq;
                    }
                    __syncthreads();
                    all = all_q = 0.0;
                    for (int v = 0; v < kNodeWaves; ++v) {
                        all += s.part[0][v];
                        all_q += s.part[1][v];
                    }
                    if (follows) all_q = without;
                    if (!shows || (all > 1e-25 && all_q > 1e-25)) break;
                    shows = false;
                    __syncthreads();
                }
            }
            if (all > 0.0) {
                alpha = 1.0 / all;
                beta = next;
            }
            rest_q = all_q;
        }
        if (k < kids) return finish(s.child[k], -1);
        auto left_of = [&](int t) { return s.rejected(t) ? 0.0 : fmax(p_of(t) - beta * q_of(t), 0.0); };
        // sums of segments: none rejected, or one, they are there
        double part = 0.0;
        if (tried == 0 || beta == 0.0) {
            part = p.part * p.one;
        } else if (tried == 1) {
            part = first.p;
        } else if (shows) {
            const double by = beta * q.one_q / p.one;
            over_kept(by, false, [&](int v, double left, double) {
                const double sum = running_sum(left);
                if (lane == 63) s.sums[v][wave] = sum;
            });
            __syncthreads();
            if (lane < segments)
                for (int i = 0; i < kNodeWaves; ++i) part += s.sums[lane][i];
            const Left left(by);
            return finish(-1, draw_from_segments(a, s, part, segments, [&](int t) {
                const float* at = w + kept_at(0, segments, t / kSegment) + t % kSegment;
                return (double)left(at[0], at[kSegment]);
            }));
        } else {
            for (int v = 0; v < segments; ++v) {
                double w = 0.0;
                for (int t = v * kSegment + tid; t < min((v + 1) * kSegment, a.V); t += kNodeThreads) w += left_of(t);
                w = running_sum(w);
                __syncthreads();
                if (lane == 63) s.part[0][wave] = w;
                __syncthreads();
                if (v == lane)
                    for (int i = 0; i < kNodeWaves; ++i) part += s.part[0][i];
            }
        }
        return finish(-1, draw_from_segments(a, s, part, segments, left_of));
    }
}

static int sample_segments(int V) { return ceil_div(V, kSegment); }
static size_t sample_rest_at(int V) { return align_up((size_t)2 * GHD_MAX_M * sample_segments(V) * sizeof(Segment), 256); }
static size_t sample_first_at(int V) { return sample_rest_at(V) + align_up((size_t)GHD_MAX_M * sample_segments(V) * sizeof(Rest), 256); }
static size_t sample_nodes_at(int V) { return sample_first_at(V) + align_up(GHD_MAX_M * sizeof(First), 256); }

static size_t sample_kept_at(int V) { return sample_nodes_at(V) + align_up(GHD_MAX_M * 8 + 4, 256); }

// (without draft probabilities nothing is kept: 0.4 MB instead of 269 MB for 128 nodes of 262144)
size_t accept_sampled_bytes(int M, int V, bool drafts) { return sample_kept_at(V) + (drafts ? kept_at(M, sample_segments(V), 0) * 4 : 0); }

ghd_status launch_accept_sampled(const SampleArgs& a, void* ws, hipStream_t st)
{
    static_assert(kNodeThreads * kSide == kSegment && kSide == 8 && kMaxSegments == 64, "a segment's tokens are dealt evenly, a lane has a segment of a row");
    Segment* seg = (Segment*)ws;
    Rest* rest = (Rest*)((char*)ws + sample_rest_at(a.V));
    First* firsts = (First*)((char*)ws + sample_first_at(a.V));
    uint64_t* nodes = (uint64_t*)((char*)ws + sample_nodes_at(a.V));
    uint32_t* arrived = (uint32_t*)(nodes + GHD_MAX_M);
    const int segments = sample_segments(a.V);
    hipLaunchKernelGGL(k_sample_rows, dim3(segments, a.M + (a.q_logits ? a.q_rows : 0)), dim3(kRowThreads), 0, st, a.logits,
                       a.tokens, a.parent, a.u, a.q_logits, a.M, a.V, a, seg, arrived);
    ghd_status s = check_launch();
    if (s) return s;
    if (a.q_logits) {
        hipLaunchKernelGGL(k_sample_first, dim3(a.M), dim3(64), 0, st, a.logits, a.tokens, a.parent, a.u, (const Segment*)seg, a.M, a.V, a, segments,
                           firsts);
        if ((s = check_launch())) return s;
        float* kept = (float*)((char*)ws + sample_kept_at(a.V));
        hipLaunchKernelGGL(k_sample_rest, dim3(segments, a.M), dim3(kRowThreads), 0, st, a, firsts, rest, kept);
        if ((s = check_launch())) return s;
        hipLaunchKernelGGL(k_sample_nodes<true>, dim3(a.M), dim3(kNodeThreads), 0, st, a.logits, a.tokens,
                           a.parent, a.u, (const Segment*)seg, a.M, a.V, a, (const First*)firsts, (const Rest*)rest, kept, segments, nodes,
                           arrived);
    } else {
        hipLaunchKernelGGL(k_sample_nodes<false>, dim3(a.M), dim3(kNodeThreads), 0, st, a.logits, a.tokens, a.parent, a.u, (const Segment*)seg, a.M,
                           a.V, a, (const First*)nullptr,
                           (const Rest*)nullptr, (float*)nullptr, segments, nodes, arrived);
    }
    return check_launch();
}

}  // namespace ghd
