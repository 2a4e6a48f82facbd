// Acceptance of drafted tokens against the target's probabilities from given random numbers (include/ghd.h has the rule).
//
// Every node is judged at once as if the walk came there: k_sample_rows leaves maxima and sums of softmax weights of the rows' segments,
// k_sample_nodes which child of each node is accepted, or which token is drawn there, and k_sample_walk goes from the root down.
//
// Weights exp((l - m) / T) have arguments in 64 bits and 24 bits themselves; sums are 64 bits.  So a sum over a row is off by some
// 2^-24 / sqrt(V) of its largest terms, by random roundings of single weights, and what 64 bits would accept or draw is
// what is accepted or drawn but where a random number lies as close to a border.
#include "sparse.h"

namespace ghd {

constexpr int kSegment = 4096;                   // logits of a row that a workgroup takes
constexpr int kRowThreads = 256, kPerThread = kSegment / kRowThreads;
constexpr int kNodeThreads = 1024, kNodeWaves = kNodeThreads / 64;
constexpr int kMaxSegments = 64;                 // of the largest vocabulary, 262144

// 2^x for x <= 0 in 64 bits' range
__device__ __forceinline__ double power_of(double x)
{
    const double n = rint(x);
    return ldexp((double)__builtin_amdgcn_exp2f((float)(x - n)), (int)fmax(n, -2000.0));
}
// The weight of a logit against a maximum, c = log2 e / T.  NaN and minus infinity have none; where the maximum is infinity only such
// logits have one.
__device__ __forceinline__ double weight_of(float l, float m, double c)
{
    if (!(l > -INFINITY)) return 0.0;
    if (l == m) return 1.0;
    if (m == INFINITY) return 0.0;
    return power_of(((double)l - (double)m) * c);
}

struct Segment {
    double sum;                                  // of weights against the segment's maximum
    float top;
    int last;                                    // of the tokens that have a weight; -1: none has
};
struct NodeResult {
    int taken, token;                            // accepted child or -1, and the token drawn where there is none
};

__device__ __forceinline__ double wave_sum(double x)
{
    for (int off = 32; off > 0; off >>= 1) x += __shfl_xor(x, off);
    return x;
}
__device__ __forceinline__ float wave_max_of(float x)
{
    for (int off = 32; off > 0; off >>= 1) x = fmaxf(x, __shfl_xor(x, off));
    return x;
}
__device__ __forceinline__ int wave_max_of(int x)
{
    for (int off = 32; off > 0; off >>= 1) x = max(x, __shfl_xor(x, off));
    return x;
}

// child c's parent, if c is one of the tree's nodes
__device__ __forceinline__ bool child_of(const SampleArgs& a, int c, int node) { return c > node && c < a.M && a.parent[c] == node; }

// Target rows (blockIdx.y < M) without the tokens of the node's children, where drafts have no probabilities; draft rows.
__global__ __launch_bounds__(kRowThreads) void k_sample_rows(SampleArgs a, Segment* __restrict__ seg)
{
    __shared__ uint32_t s_out[kSegment / 32];
    __shared__ double s_sum[kRowThreads / 64];
    __shared__ float s_top[kRowThreads / 64];
    __shared__ int s_last[kRowThreads / 64];
    const int tid = threadIdx.x, y = blockIdx.y, lo = blockIdx.x * kSegment, segments = gridDim.x;
    const bool target = y < a.M;
    const float* row = target ? a.logits + (size_t)y * a.V : a.q_logits + (size_t)(y - a.M) * a.V;
    const double c = 1.4426950408889634 / (double)(target ? a.temperature : a.q_temperature);
    float l[kPerThread];
#pragma unroll
    for (int i = 0; i < kPerThread; ++i) {
        const int t = lo + i * kRowThreads + tid;
        l[i] = t < a.V ? row[t] : -INFINITY;
    }
    if (target && !a.q_logits) {
        if (tid < kSegment / 32) s_out[tid] = 0;
        __syncthreads();
        if (tid < GHD_MAX_M && child_of(a, tid, y)) {
            const int t = a.tokens[tid];
            if (t >= lo && t < lo + kSegment) atomicOr(&s_out[(t - lo) >> 5], 1u << ((t - lo) & 31));
        }
        __syncthreads();
#pragma unroll
        for (int i = 0; i < kPerThread; ++i) {
            const int t = i * kRowThreads + tid;
            if (s_out[t >> 5] >> (t & 31) & 1) l[i] = -INFINITY;
        }
    }
    float top = -INFINITY;
#pragma unroll
    for (int i = 0; i < kPerThread; ++i) top = fmaxf(top, l[i]);
    top = wave_max_of(top);
    if ((tid & 63) == 0) s_top[tid >> 6] = top;
    __syncthreads();
#pragma unroll
    for (int w = 0; w < kRowThreads / 64; ++w) top = fmaxf(top, s_top[w]);
    double sum = 0.0;
    int last = -1;
#pragma unroll
    for (int i = 0; i < kPerThread; ++i) {
        const double x = weight_of(l[i], top, c);
        sum += x;
        if (x > 0.0) last = lo + i * kRowThreads + tid;
    }
    sum = wave_sum(sum);
    last = wave_max_of(last);
    if ((tid & 63) == 0) {
        s_sum[tid >> 6] = sum;
        s_last[tid >> 6] = last;
    }
    __syncthreads();
    if (tid == 0) {
        Segment s = {0.0, top, -1};
        for (int w = 0; w < kRowThreads / 64; ++w) {
            s.sum += s_sum[w];
            s.last = max(s.last, s_last[w]);
        }
        seg[(size_t)y * segments + blockIdx.x] = s;
    }
}

// What a workgroup knows of a row: its maximum and, before every segment, the sum of weights against that
struct Row {
    float top;
    double sum, at[kMaxSegments];                // at: a segment's factor, then the sum before it
};

__device__ __forceinline__ double u_of(float u) { return u > 0.f ? (double)u : 0.0; }

// One workgroup a node.
__global__ __launch_bounds__(kNodeThreads) void k_sample_nodes(SampleArgs a, const Segment* __restrict__ seg, int segments,
                                                               NodeResult* __restrict__ out)
{
    __shared__ int s_child[GHD_MAX_M], s_token[GHD_MAX_M];
    __shared__ double s_weight[GHD_MAX_M], s_part[3][kNodeWaves];
    __shared__ int s_kids, s_taken, s_last[kNodeWaves];
    __shared__ float s_top;
    __shared__ uint32_t s_out[kSegment / 32];
    const int tid = threadIdx.x, lane = tid & 63, wave = tid >> 6, node = blockIdx.x;
    const float* row = a.logits + (size_t)node * a.V;
    const Segment* mine = seg + (size_t)node * segments;
    const double c = 1.4426950408889634 / (double)a.temperature;
    // children, in order
    if (wave == 0) {
        int n = 0;
        for (int h = 0; h < GHD_MAX_M / 64; ++h) {
            const bool is = child_of(a, h * 64 + lane, node);
            const uint64_t with = __ballot(is);
            if (is) {
                const int k = n + __popcll(with & ((1ull << lane) - 1));
                s_child[k] = h * 64 + lane;
                s_token[k] = a.tokens[h * 64 + lane];
            }
            n += __popcll(with);
        }
        if (lane == 0) {
            s_kids = n;
            s_taken = -1;
        }
    }
    __syncthreads();
    const int kids = s_kids;
    auto there = [&](int t) { return t >= 0 && t < a.V; };

    if (!a.q_logits || kids == 0) {
        // Drafts without probabilities: a child is accepted if u (what is left) < its weight.  What is left before a child: the
        // tokens that no child has, and the weights of this child and those after it.
        if (wave == 0) {
            float top = -INFINITY;
            for (int s = lane; s < segments; s += 64) top = fmaxf(top, mine[s].top);
            for (int k = lane; k < kids; k += 64)
                if (there(s_token[k])) top = fmaxf(top, row[s_token[k]]);
            top = wave_max_of(top);
            double rest = 0.0;
            for (int s = lane; s < segments; s += 64) rest += mine[s].sum * weight_of(mine[s].top, top, c);
            rest = wave_sum(rest);
            for (int k = lane; k < kids; k += 64) {
                double w = there(s_token[k]) ? weight_of(row[s_token[k]], top, c) : 0.0;
                for (int j = 0; j < k; ++j)
                    if (s_token[j] == s_token[k]) w = 0.0;     // it was rejected before
                s_weight[k] = w;
            }
            __builtin_amdgcn_fence(__ATOMIC_ACQ_REL, "wavefront");
            int first = GHD_MAX_M;
            for (int k = lane; k < kids; k += 64) {
                double left = rest;
                for (int j = kids - 1; j >= k; --j) left += s_weight[j];
                if (u_of(a.u[s_child[k]]) * left < s_weight[k]) first = min(first, k);
            }
            first = -wave_max_of(-first);
            if (lane == 0) {
                s_top = top;
                s_part[0][0] = rest;
                s_taken = first < GHD_MAX_M ? s_child[first] : -1;
            }
        }
        __syncthreads();
        if (s_taken >= 0) {
            if (tid == 0) out[node] = {s_taken, -1};
            return;
        }
        // the segment in which the sum passes u, then the place
        const double goal = u_of(a.u[0]) * s_part[0][0];
        __shared__ int s_seg;
        __shared__ double s_before;
        if (tid == 0) {
            double sum = 0.0;
            int at = -1;
            s_seg = -1;
            for (int s = 0; s < segments; ++s) {
                const double w = mine[s].sum * weight_of(mine[s].top, s_top, c);
                if (w > 0.0) {
                    at = s;
                    s_before = sum;
                    if (sum + w > goal) break;
                }
                sum += w;
            }
            s_seg = at;
        }
        if (tid < kSegment / 32) s_out[tid] = 0;
        __syncthreads();
        if (s_seg < 0) {                         // no token has a weight
            if (tid == 0) out[node] = {-1, -1};
            return;
        }
        const int lo = s_seg * kSegment;
        const float top = mine[s_seg].top;
        const double factor = weight_of(top, s_top, c);
        if (tid < kids && s_token[tid] >= lo && s_token[tid] < lo + kSegment)
            atomicOr(&s_out[(s_token[tid] - lo) >> 5], 1u << ((s_token[tid] - lo) & 31));
        __syncthreads();
        // a thread has four neighbours
        double w[4], sum = 0.0;
#pragma unroll
        for (int e = 0; e < 4; ++e) {
            const int j = tid * 4 + e, t = lo + j;
            w[e] = t < a.V && !(s_out[j >> 5] >> (j & 31) & 1) ? weight_of(row[t], top, c) * factor : 0.0;
            sum += w[e];
        }
        double upto = sum;
        for (int off = 1; off < 64; off *= 2) {
            const double o = __shfl_up(upto, off);
            if (lane >= off) upto += o;
        }
        if (lane == 63) s_part[1][wave] = upto;
        __syncthreads();
        double before = s_before + upto - sum;
        for (int v = 0; v < wave; ++v) before += s_part[1][v];
        int place = 0x7fffffff;
#pragma unroll
        for (int e = 0; e < 4; ++e) {
            before += w[e];
            if (w[e] > 0.0 && before > goal && place == 0x7fffffff) place = lo + tid * 4 + e;
        }
        place = -wave_max_of(-place);
        if (lane == 0) s_last[wave] = place;
        __syncthreads();
        if (tid == 0) {
            for (int v = 0; v < kNodeWaves; ++v) place = min(place, s_last[v]);
            out[node] = {-1, place == 0x7fffffff ? mine[s_seg].last : place};
        }
        return;
    }

    // Drafts from probabilities: after some rejections what is left is alpha (p - beta q)+ of the tokens not rejected, and what is left of
    // q its other tokens; one sum over the row for each rejection.
    const int qr = a.q_row ? min(max(a.q_row[node], 0), a.q_rows - 1) : node;
    const float* q_row = a.q_logits + (size_t)qr * a.V;
    const Segment* drafts = seg + (size_t)(a.M + qr) * segments;
    const double cq = 1.4426950408889634 / (double)a.q_temperature;
    float top = -INFINITY, top_q = -INFINITY;
    for (int s = 0; s < segments; ++s) {
        top = fmaxf(top, mine[s].top);
        top_q = fmaxf(top_q, drafts[s].top);
    }
    double sum = 0.0, sum_q = 0.0;
    for (int s = 0; s < segments; ++s) {
        sum += mine[s].sum * weight_of(mine[s].top, top, c);
        sum_q += drafts[s].sum * weight_of(drafts[s].top, top_q, cq);
    }
    const double one = sum > 0.0 ? 1.0 / sum : 0.0, one_q = sum_q > 0.0 ? 1.0 / sum_q : 0.0;
    auto p_of = [&](int t) { return weight_of(row[t], top, c) * one; };
    auto q_of = [&](int t) { return weight_of(q_row[t], top_q, cq) * one_q; };
    // tokens of a wavefront: neighbours, so that sums over wavefronts are sums up to a token
    const int per = (a.V + kNodeThreads - 1) / kNodeThreads * 64, from = min(wave * per, a.V), to = min(from + per, a.V);
    double alpha = 1.0, beta = 0.0, rest_q = sum_q > 0.0 ? 1.0 : 0.0, part = 0.0;
    auto rejected = [&](int t, int k) {
        bool is = false;
        for (int j = 0; j < k; ++j) is = is || s_token[j] == t;
        return is;
    };
    int k = 0;
    for (; k < kids; ++k) {
        const int x = s_token[k];
        if (!there(x)) continue;
        const bool gone = rejected(x, k);
        const double px = gone ? 0.0 : fmax(alpha * (p_of(x) - beta * q_of(x)), 0.0), qx = gone || !(rest_q > 0.0) ? 0.0 : q_of(x) / rest_q;
        if (u_of(a.u[s_child[k]]) * qx < px) break;
        const double next = rest_q > 0.0 ? beta + 1.0 / (alpha * rest_q) : beta;
        double s = 0.0, r = 0.0;
        for (int t = from + lane; t < to; t += 64) {
            if (rejected(t, k + 1)) continue;
            const double q = q_of(t);
            s += fmax(p_of(t) - next * q, 0.0);
            r += q;
        }
        s = wave_sum(s);
        r = wave_sum(r);
        __syncthreads();                         // (the last round's sums have been read)
        if (lane == 0) {
            s_part[0][wave] = s;
            s_part[1][wave] = r;
        }
        __syncthreads();
        double all = 0.0, all_q = 0.0;
        for (int v = 0; v < kNodeWaves; ++v) {
            all += s_part[0][v];
            all_q += s_part[1][v];
        }
        if (all > 0.0) {
            alpha = 1.0 / all;
            beta = next;
        }
        rest_q = all_q;
    }
    if (k < kids) {
        if (tid == 0) out[node] = {s_child[k], -1};
        return;
    }
    // the draw
    auto left_of = [&](int t) { return rejected(t, kids) ? 0.0 : fmax(p_of(t) - beta * q_of(t), 0.0); };
    int last = -1;
    for (int t = from + lane; t < to; t += 64) {
        const double w = left_of(t);
        part += w;
        if (w > 0.0) last = t;
    }
    part = wave_sum(part);
    last = wave_max_of(last);
    __syncthreads();
    if (lane == 0) {
        s_part[2][wave] = part;
        s_last[wave] = last;
    }
    __syncthreads();
    double total = 0.0, before = 0.0;
    int at = -1, end = -1;
    for (int v = 0; v < kNodeWaves; ++v) {
        total += s_part[2][v];
        end = max(end, s_last[v]);
    }
    const double goal = u_of(a.u[0]) * total;
    double so_far = 0.0;
    for (int v = 0; v < kNodeWaves; ++v) {
        if (at < 0 && so_far + s_part[2][v] > goal) {
            at = v;
            before = so_far;
        }
        so_far += s_part[2][v];
    }
    if (at < 0) {
        if (tid == 0) out[node] = {-1, end};
        return;
    }
    if (wave != at) return;
    for (int t0 = from; t0 < to; t0 += 64) {
        const double w = t0 + lane < to ? left_of(t0 + lane) : 0.0;
        double upto = w;
        for (int off = 1; off < 64; off *= 2) {
            const double o = __shfl_up(upto, off);
            if (lane >= off) upto += o;
        }
        const uint64_t over = __ballot(w > 0.0 && before + upto > goal);
        if (over) {
            if (lane == 0) out[node] = {-1, t0 + (int)__builtin_ctzll(over)};
            return;
        }
        before += __shfl(upto, 63);
    }
    if (lane == 0) out[node] = {-1, last};       // (the wavefront's own sum was larger by a rounding)
}

__global__ __launch_bounds__(GHD_MAX_M) void k_sample_walk(const NodeResult* __restrict__ nodes, int M, int32_t* __restrict__ res)
{
    __shared__ NodeResult s_node[GHD_MAX_M];
    const int tid = threadIdx.x;
    if (tid < M) s_node[tid] = nodes[tid];
    __syncthreads();
    if (tid != 0) return;
    int node = 0, len = 1;
    res[2] = 0;
    for (; s_node[node].taken > node; ++len) {   // (a child comes after its node: at most M steps)
        node = s_node[node].taken;
        res[2 + len] = node;
    }
    res[0] = len;
    res[1] = s_node[node].token;
}

static int sample_segments(int V) { return ceil_div(V, kSegment); }
static size_t sample_nodes_at(int V) { return align_up((size_t)2 * GHD_MAX_M * sample_segments(V) * sizeof(Segment), 256); }

size_t accept_sampled_bytes(int M, int V) { return sample_nodes_at(V) + align_up(GHD_MAX_M * sizeof(NodeResult), 256); }

ghd_status launch_accept_sampled(const SampleArgs& a, void* ws, hipStream_t st)
{
    static_assert(kNodeThreads * 4 == kSegment, "a thread has four tokens of a segment");
    Segment* seg = (Segment*)ws;
    NodeResult* nodes = (NodeResult*)((char*)ws + sample_nodes_at(a.V));
    const int segments = sample_segments(a.V);
    hipLaunchKernelGGL(k_sample_rows, dim3(segments, a.M + (a.q_logits ? a.q_rows : 0)), dim3(kRowThreads), 0, st, a, seg);
    ghd_status s = check_launch();
    if (s) return s;
    hipLaunchKernelGGL(k_sample_nodes, dim3(a.M), dim3(kNodeThreads), 0, st, a, (const Segment*)seg, segments, nodes);
    s = check_launch();
    if (s) return s;
    hipLaunchKernelGGL(k_sample_walk, dim3(1), dim3(GHD_MAX_M), 0, st, (const NodeResult*)nodes, a.M, a.res);
    return check_launch();
}

}  // namespace ghd
