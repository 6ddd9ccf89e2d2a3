// qnn_route_topk() and qnn_expert_plan(): which experts a token goes to, and the tokens each expert gets.
//
// route_topk_kernel: one warp owns one token; lane l holds NV neighbouring experts from l * NV on.  Scores are compared as
// 32-bit keys whose unsigned order is the order of the floats, so the warp's best expert is one integer maximum over the
// lanes and the lowest index among equals one integer minimum: ties go to the lowest index by construction.  The choice
// uses the score itself (the logit where softmax scores carry no bias: the same order without rounding).  Groups that are
// whole lanes, a power of two of them, find their two best with a few shuffles; other splits go through shared memory.
// The kernel is bound by its instructions, not by the logits' bytes: 32768 tokens, 8 of 256 experts in 16 groups, sigmoid
// with a bias, 30 us, 930 instructions a token.
//
// expert plan: a stable counting sort of the slots (token * top + choice) by expert.  Ranks come from ordered per-warp
// counts, never from the order in which atomics land, so the plan is the same on every run.  262144 slots over 256
// experts: 4 us to count, 11 to place.
#include "block_common.cuh"
#include "block_internal.h"

namespace qnn {
namespace {

constexpr int kRouteWarps = 8;
constexpr uint32_t kFull = 0xffffffffu;

struct RouteArgs {
    const void *logits;
    const float *bias;
    float *weights;
    int32_t *ids;
    int64_t t, ld;
    int e, k, sigmoid, groups, top_groups, two, renorm;
    int group_size;
    int vec, bias_vec;     // rows of logits, and the bias, are aligned for 16-byte loads
    uint32_t group_magic;  // expert / group_size = (expert * magic) >> 20 for experts below 1024
    float scale;
};

// Key whose unsigned order is the float order; 0 for an expert that cannot be chosen (-inf or NaN).
__device__ __forceinline__ uint32_t order_key(float v)
{
    const uint32_t b = __float_as_uint(v + 0.f);  // -0 becomes +0
    if (!(v > -INFINITY)) return 0u;
    return b & 0x80000000u ? ~b : b | 0x80000000u;
}

// exp(v - top); where the largest logit is infinite, the infinite ones share the weight
__device__ __forceinline__ float exp_from(float v, float top)
{
    const float e = expf(v - (top == INFINITY ? 0.f : top));
    return top == INFINITY ? (v == INFINITY ? 1.f : 0.f) : e;
}

// The sum is rounded by itself, so that a score is the same wherever it is computed.
__device__ __forceinline__ float sigmoid_of(float v) { return __frcp_rn(__fadd_rn(1.f, expf(-v))); }

__device__ __forceinline__ float score_of(float v, int sigmoid, float top)
{
    if (sigmoid) return v > -INFINITY ? sigmoid_of(v) : 0.f;
    return v > -INFINITY ? exp_from(v, top) : 0.f;
}

// Below this, sums of scores lose their leading bits to underflow (exp(-69)).
constexpr float kLeastScore = 1e-30f;

// NV (a multiple of four) neighbouring logits.
template <typename T, int NV>
__device__ __forceinline__ void load_run(const T *p, float (&x)[NV])
{
    if constexpr (sizeof(T) == 4) {
#pragma unroll
        for (int i = 0; i + 4 <= NV; i += 4) {
            const float4 q = *reinterpret_cast<const float4 *>(p + i);
            x[i] = q.x; x[i + 1] = q.y; x[i + 2] = q.z; x[i + 3] = q.w;
        }
    } else {
#pragma unroll
        for (int i = 0; i + 4 <= NV; i += 4) {
            const uint2 q = *reinterpret_cast<const uint2 *>(p + i);
            const float2 f = unpack2<T>(q.x), h = unpack2<T>(q.y);
            x[i] = f.x; x[i + 1] = f.y; x[i + 2] = h.x; x[i + 3] = h.y;
        }
    }
}

// This lane's share of the chosen scores where all of them underflow (a bias may choose any expert): that of exp(logit), for
// sigmoid scores as well (exp(l) / (1 + exp(l)), the divisor 1 there), taken from the largest of them.  0 where none is chosen.
__device__ __noinline__ float tiny_share(float l)
{
    float m = l;
#pragma unroll
    for (int o = 16; o > 0; o >>= 1) m = fmaxf(m, __shfl_xor_sync(kFull, m, o));
    const float w = l > -INFINITY ? exp_from(l, m) : 0.f;
    float s = w;
#pragma unroll
    for (int o = 16; o > 0; o >>= 1) s += __shfl_xor_sync(kFull, s, o);
    return s > 0.f ? w / s : 0.f;
}

template <typename T, int NV>
__global__ void __launch_bounds__(kRouteWarps * 32) route_topk_kernel(const RouteArgs a)
{
    __shared__ uint2 candidates[kRouteWarps][64];  // key and expert
    extern __shared__ float sm_scores[];  // one row of group_size * groups scores a warp (grouped calls only)
    const int lane = threadIdx.x & 31;
    const int64_t token = static_cast<int64_t>(blockIdx.x) * kRouteWarps + (threadIdx.x >> 5);
    pdl_begin();
    if (token >= a.t) return;
    const T *row = static_cast<const T *>(a.logits) + token * a.ld;
    const int e0 = lane * NV;  // this lane's first expert

    float x[NV];
    if (NV >= 4 && a.vec && e0 + NV <= a.e) {
        load_run<T, NV>(row + e0, x);
    } else {
#pragma unroll
        for (int i = 0; i < NV; ++i) x[i] = e0 + i < a.e ? to_f32<T>(row[e0 + i]) : -INFINITY;
    }
    float top = 0.f, total = 1.f;
    if (!a.sigmoid) {
        top = -INFINITY;
#pragma unroll
        for (int i = 0; i < NV; ++i) top = fmaxf(top, x[i]);  // fmaxf drops NaN
#pragma unroll
        for (int o = 16; o > 0; o >>= 1) top = fmaxf(top, __shfl_xor_sync(kFull, top, o));
        if (!a.renorm || a.bias) {
            total = 0.f;
#pragma unroll
            for (int i = 0; i < NV; ++i) total += score_of(x[i], 0, top);
#pragma unroll
            for (int o = 16; o > 0; o >>= 1) total += __shfl_xor_sync(kFull, total, o);
            total = total > 0.f ? total : 1.f;
        }
    }
    // what the choice goes by
    const bool scored = a.sigmoid || a.bias;
    uint32_t key[NV];
    float of[NV], bias[NV];  // what groups go by
    if (NV >= 4 && a.bias && a.bias_vec && e0 + NV <= a.e) {
        load_run<float, NV>(a.bias + e0, bias);
    } else {
#pragma unroll
        for (int i = 0; i < NV; ++i) bias[i] = a.bias && e0 + i < a.e ? a.bias[e0 + i] : 0.f;
    }
    // Straight-line loops, the mode outside: a closed expert's logit counts as 0 here (its key is 0 below), which also keeps
    // the exponential and the reciprocal off their slow paths for infinities.
    float c[NV];
#pragma unroll
    for (int i = 0; i < NV; ++i) c[i] = x[i];
    if (a.sigmoid) {
#pragma unroll
        for (int i = 0; i < NV; ++i) c[i] = __fadd_rn(sigmoid_of(x[i] > -INFINITY ? x[i] : 0.f), bias[i]);
    } else if (a.bias) {
#pragma unroll
        for (int i = 0; i < NV; ++i) c[i] = score_of(x[i], 0, top) / total + bias[i];
    }
#pragma unroll
    for (int i = 0; i < NV; ++i) key[i] = x[i] > -INFINITY ? order_key(c[i]) : 0u;
    if (a.groups > 1) {
#pragma unroll
        for (int i = 0; i < NV; ++i) of[i] = key[i] == 0u ? -INFINITY : c[i];
        // Keys of this lane's group: `mine` while there is one in it to choose, then `far`.  Both find the group's two best
        // first; where the choice goes by logits, the sum is that of their softmax numerators.  A sum that would underflow (of
        // a group that lies 69 or more below the row's largest logit) is compared by its logarithm, which keeps its order;
        // these groups come after all of the others.
        uint32_t mine = 0u, far = 0u;
        auto rank_group = [&](float best, float second) {
            if (!a.two) {
                mine = order_key(best);
            } else if (scored) {
                mine = order_key(second > -INFINITY ? best + second : best);
            } else if (best > -INFINITY) {
                const float sum = exp_from(best, top) + score_of(second, 0, top);
                if (sum >= kLeastScore) mine = order_key(sum);
                else far = order_key(best + log1pf(expf(second - best)));
            }
        };
        int group;
        const int width = a.group_size / NV;  // lanes a group
        const bool lanes = a.group_size % NV == 0 && (width & (width - 1)) == 0;
        if (lanes) {
            float best = of[0], second = -INFINITY;
#pragma unroll
            for (int i = 1; i < NV; ++i) {
                second = fmaxf(second, fminf(best, of[i]));
                best = fmaxf(best, of[i]);
            }
            for (int o = 1; o < width; o <<= 1) {
                const float b = __shfl_xor_sync(kFull, best, o), s = __shfl_xor_sync(kFull, second, o);
                second = fmaxf(fmaxf(second, s), fminf(best, b));
                best = fmaxf(best, b);
            }
            group = lane / width;
            if (group < a.groups) rank_group(best, second);
        } else {
            float *sc = sm_scores + (threadIdx.x >> 5) * a.e;
#pragma unroll
            for (int i = 0; i < NV; ++i)
                if (e0 + i < a.e) sc[e0 + i] = of[i];
            __syncwarp();
            group = lane;
            if (lane < a.groups) {
                float best = -INFINITY, second = -INFINITY;
                int j = lane % a.group_size;  // a start of its own a lane: fewer bank conflicts
                for (int n = 0; n < a.group_size; ++n) {
                    const float v = sc[lane * a.group_size + j];
                    second = fmaxf(second, fminf(best, v));
                    best = fmaxf(best, v);
                    j = j + 1 == a.group_size ? 0 : j + 1;
                }
                rank_group(best, second);
            }
        }
        uint32_t keep = 0u;
        for (int n = 0; n < a.top_groups; ++n) {
            uint32_t top_key = __reduce_max_sync(kFull, mine);
            if (top_key == 0u) {  // (a second time round both are 0)
                mine = far;
                far = 0u;
                top_key = __reduce_max_sync(kFull, mine);
                if (top_key == 0u) break;
            }
            const uint32_t g = __reduce_min_sync(kFull, mine == top_key ? static_cast<uint32_t>(group) : kFull);
            keep |= 1u << g;
            if (static_cast<uint32_t>(group) == g) mine = 0u;
        }
        if (lanes) {
            if (!((keep >> (group & 31)) & 1) || group >= a.groups)
#pragma unroll
                for (int i = 0; i < NV; ++i) key[i] = 0u;
        } else {
#pragma unroll
            for (int i = 0; i < NV; ++i) {
                const uint32_t g = (static_cast<uint32_t>(e0 + i) * a.group_magic) >> 20;
                if (!((keep >> (g & 31)) & 1)) key[i] = 0u;
            }
        }
    }
    // The k best, one warp maximum each; lane j keeps choice j.  Few keys can be among them: at least k are as large as the
    // k-th largest of the lanes' maxima, so only keys from there on are candidates, about a dozen of 256.  They are moved
    // together, at most two to a lane, which makes a step a few instructions instead of a search through NV keys.
    int id = -1;
    uint32_t best = key[0];
#pragma unroll
    for (int i = 1; i < NV; ++i) best = max(best, key[i]);
    uint32_t floor_key = 1u;  // the k-th largest maximum; 1 (any open expert) where there are fewer, or few experts in all
    if (a.groups == 1 || a.top_groups * a.group_size > 64) {
        uint32_t least = best;
        for (int j = 0; j < a.k; ++j) {
            const uint32_t top_key = __reduce_max_sync(kFull, least);
            if (top_key == 0u) {
                floor_key = 1u;
                break;
            }
            floor_key = top_key;
            // one lane a step: equal maxima count one by one
            const uint32_t who = __ballot_sync(kFull, least == top_key);
            if (lane == __ffs(who) - 1) least = 0u;
        }
    }
    int count = 0;
#pragma unroll
    for (int i = 0; i < NV; ++i) count += key[i] >= floor_key;
    int before = count;  // lanes in order, so candidates lie in the order of their experts
#pragma unroll
    for (int o = 1; o < 32; o <<= 1) {
        const int v = __shfl_up_sync(kFull, before, o);
        if (lane >= o) before += v;
    }
    const int all = __shfl_sync(kFull, before, 31);
    if (all <= 64) {
        uint2 *mine = candidates[threadIdx.x >> 5];
        int at = before - count;
#pragma unroll
        for (int i = 0; i < NV; ++i)
            if (key[i] >= floor_key) mine[at++] = make_uint2(key[i], e0 + i);
        __syncwarp();
        uint2 c0 = lane < all ? mine[lane] : make_uint2(0u, kFull), c1 = lane + 32 < all ? mine[lane + 32] : make_uint2(0u, kFull);
        for (int j = 0; j < a.k; ++j) {
            const uint32_t top_key = __reduce_max_sync(kFull, max(c0.x, c1.x));
            if (top_key == 0u) break;
            // the lower expert of the two where both are equal: c0 comes first
            const uint32_t e = __reduce_min_sync(kFull, c0.x == top_key ? c0.y : c1.x == top_key ? c1.y : kFull);
            if (lane == j) id = static_cast<int>(e);
            if (c0.y == e) c0.x = 0u;
            if (c1.y == e) c1.x = 0u;
        }
    } else {  // many equal scores
        for (int j = 0; j < a.k; ++j) {
            uint32_t lane_best = key[0];
            int at = 0;
#pragma unroll
            for (int i = 1; i < NV; ++i)
                if (key[i] > lane_best) {
                    lane_best = key[i];
                    at = i;
                }
            const uint32_t top_key = __reduce_max_sync(kFull, lane_best);
            if (top_key == 0u) break;
            // lanes hold neighbours in order, so the lowest lane has the lowest index
            const int owner = __ffs(__ballot_sync(kFull, lane_best == top_key)) - 1;
            const int e = __shfl_sync(kFull, e0 + at, owner);
            if (lane == j) id = e;
#pragma unroll
            for (int i = 0; i < NV; ++i)
                if (e == e0 + i) key[i] = 0u;
        }
    }
    float w = 0.f;
    if (id >= 0) {
        w = score_of(to_f32<T>(row[id]), a.sigmoid, top);
        if (!a.sigmoid && !a.renorm) w /= total;
    }
    if (a.renorm) {
        float s = w;
#pragma unroll
        for (int o = 16; o > 0; o >>= 1) s += __shfl_xor_sync(kFull, s, o);
        if (s >= kLeastScore) w /= s;
        else if (top < INFINITY) w = tiny_share(id >= 0 ? to_f32<T>(row[id]) : -INFINITY);
    }
    if (lane < a.k) {
        a.weights[token * a.k + lane] = w * a.scale;
        a.ids[token * a.k + lane] = id;
    }
}

// ---------------------------------------------------------------- plan

constexpr int kPlanThreads = 512;
constexpr int kPlanWarps = kPlanThreads / 32;
constexpr int kPlanChunk = 2048;  // slots a block

int plan_blocks(int64_t slots, int64_t *chunk)
{
    int64_t c = kPlanChunk;
    while ((slots + c - 1) / c > 128) c *= 2;
    *chunk = c;
    return static_cast<int>(slots ? (slots + c - 1) / c : 1);
}

__device__ __forceinline__ int expert_of(const int32_t *ids, int64_t slot, int64_t end, int experts)
{
    if (slot >= end) return -1;
    const int e = ids[slot];
    return e >= 0 && e < experts ? e : -1;
}

__global__ void __launch_bounds__(kPlanThreads) plan_count_kernel(const int32_t *ids, int64_t slots, int64_t chunk,
                                                                  int experts, int32_t *counts)
{
    extern __shared__ int32_t sm_plan[];
    for (int e = threadIdx.x; e < experts; e += kPlanThreads) sm_plan[e] = 0;
    __syncthreads();
    pdl_begin();
    const int64_t begin = blockIdx.x * chunk, end = begin + chunk < slots ? begin + chunk : slots;
    for (int64_t s = begin + threadIdx.x; s < end; s += kPlanThreads) {
        const int e = expert_of(ids, s, end, experts);
        if (e >= 0) atomicAdd(&sm_plan[e], 1);
    }
    __syncthreads();
    for (int e = threadIdx.x; e < experts; e += kPlanThreads) counts[e * gridDim.x + blockIdx.x] = sm_plan[e];
}

// counts: plan_count_kernel's [expert][block], or NULL when one block holds all slots.
__global__ void __launch_bounds__(kPlanThreads) plan_place_kernel(const int32_t *ids, int64_t slots, int64_t chunk,
                                                                  int experts, const int32_t *counts, int32_t *offsets,
                                                                  int32_t *order, int32_t *position)
{
    extern __shared__ int32_t sm_plan[];  // [warps][experts] counts, then [experts] starts and totals
    __shared__ int32_t part[32];
    int32_t *start = sm_plan + kPlanWarps * experts, *totals = start + experts;
    const int lane = threadIdx.x & 31, warp = threadIdx.x >> 5;
    for (int i = threadIdx.x; i < kPlanWarps * experts; i += kPlanThreads) sm_plan[i] = 0;
    __syncthreads();
    pdl_begin();
    const int64_t begin = blockIdx.x * chunk, end = begin + chunk < slots ? begin + chunk : slots;
    const int64_t span = chunk / kPlanWarps;  // a multiple of 32
    const int64_t wb = begin + warp * span, we = wb + span < end ? wb + span : end;
    int32_t *mine = sm_plan + warp * experts;
    int held[4];  // the warp's first 128 slots stay in registers for the second pass
#pragma unroll
    for (int i = 0; i < 4; ++i) held[i] = expert_of(ids, wb + i * 32 + lane, we, experts);
#pragma unroll
    for (int i = 0; i < 4; ++i)
        if (held[i] >= 0) atomicAdd(&mine[held[i]], 1);
    for (int64_t s = wb + 128 + lane; s < we; s += 32) {
        const int e = expert_of(ids, s, we, experts);
        if (e >= 0) atomicAdd(&mine[e], 1);
    }
    __syncthreads();
    if (counts) {
        // a warp an expert: its slots over all blocks (at most 128), and over the blocks before this one
        const int blocks = gridDim.x, rounds = (experts + kPlanWarps - 1) / kPlanWarps;
        // every block starts at another expert: all of them at the same rows at once would queue at one L2 slice
        const int first = static_cast<int>(blockIdx.x) % rounds;
#pragma unroll 8
        for (int n = 0; n < rounds; ++n) {
            const int turn = first + n < rounds ? first + n : first + n - rounds;
            const int e = turn * kPlanWarps + warp;
            if (e >= experts) continue;
            int all = 0, before = 0;
#pragma unroll
            for (int i = 0; i < 4; ++i) {
                const int b = i * 32 + lane;
                const int c = b < blocks ? counts[e * blocks + b] : 0;
                all += c;
                before += b < static_cast<int>(blockIdx.x) ? c : 0;
            }
            all = __reduce_add_sync(kFull, all);
            before = __reduce_add_sync(kFull, before);
            if (lane == 0) {
                totals[e] = all;
                start[e] = before;
            }
        }
        __syncthreads();
    }
    // exclusive counts over the warps; exclusive scan of the totals over the experts
    int32_t running = 0;
    for (int base = 0; base < experts; base += kPlanThreads) {
        const int e = base + threadIdx.x;
        int32_t total = 0, before = 0;
        if (e < experts) {
            int32_t own = 0;
            for (int w = 0; w < kPlanWarps; ++w) {
                const int32_t c = sm_plan[w * experts + e];
                sm_plan[w * experts + e] = own;
                own += c;
            }
            total = counts ? totals[e] : own;
            before = counts ? start[e] : 0;
        }
        int32_t inc = total;
#pragma unroll
        for (int o = 1; o < 32; o <<= 1) {
            const int32_t v = __shfl_up_sync(kFull, inc, o);
            if (lane >= o) inc += v;
        }
        if (lane == 31) part[warp] = inc;
        __syncthreads();
        int32_t lower = running, all = running;
        for (int w = 0; w < kPlanWarps; ++w) {
            lower += w < warp ? part[w] : 0;
            all += part[w];
        }
        if (e < experts) {
            start[e] = lower + inc - total + before;
            if (blockIdx.x == 0) offsets[e] = lower + inc - total;
        }
        running = all;
        __syncthreads();
    }
    if (blockIdx.x == 0 && threadIdx.x == 0) offsets[experts] = running;
    // ranks: 32 slots at a time in order, equal experts by lane
    auto rank32 = [&](int64_t s, int e) {
        const uint32_t same = __match_any_sync(kFull, e);
        const int below = __popc(same & ((1u << lane) - 1u));
        const int32_t base = e >= 0 ? mine[e] : 0;
        __syncwarp();
        if (e >= 0 && below == 0) mine[e] = base + __popc(same);
        __syncwarp();
        if (s < we) {
            const int32_t at = e >= 0 ? start[e] + base + below : -1;
            position[s] = at;
            if (at >= 0) order[at] = static_cast<int32_t>(s);
        }
    };
#pragma unroll
    for (int i = 0; i < 4; ++i) rank32(wb + i * 32 + lane, held[i]);
    for (int64_t s0 = wb + 128; s0 < we; s0 += 32) rank32(s0 + lane, expert_of(ids, s0 + lane, we, experts));
    // the places after the last planned slot
    const int64_t from = begin > running ? begin : running;
    for (int64_t s = from + threadIdx.x; s < end; s += kPlanThreads) order[s] = -1;
}

template <typename T>
cudaError_t launch_route_type(const RouteArgs &a, cudaStream_t stream)
{
    const unsigned grid = static_cast<unsigned>((a.t + kRouteWarps - 1) / kRouteWarps);
    const int threads = kRouteWarps * 32;
    const size_t smem = a.groups > 1 ? sizeof(float) * kRouteWarps * a.e : 0;  // at most 32 KB
    const int nv = (a.e + 31) / 32;
    if (nv <= 1) return launch_pdl(route_topk_kernel<T, 1>, dim3(grid), threads, smem, stream, 1, a);
    if (nv <= 2) return launch_pdl(route_topk_kernel<T, 2>, dim3(grid), threads, smem, stream, 1, a);
    if (nv <= 4) return launch_pdl(route_topk_kernel<T, 4>, dim3(grid), threads, smem, stream, 1, a);
    if (nv <= 8) return launch_pdl(route_topk_kernel<T, 8>, dim3(grid), threads, smem, stream, 1, a);
    if (nv <= 16) return launch_pdl(route_topk_kernel<T, 16>, dim3(grid), threads, smem, stream, 1, a);
    return launch_pdl(route_topk_kernel<T, 32>, dim3(grid), threads, smem, stream, 1, a);
}

}  // namespace

cudaError_t launch_route_topk(const qnn_route_desc &d, const void *logits, const float *bias, float *weights,
                              int32_t *ids, cudaStream_t stream)
{
    if (d.t == 0) return cudaSuccess;
    RouteArgs a;
    a.logits = logits; a.bias = bias; a.weights = weights; a.ids = ids;
    a.t = d.t; a.ld = d.ld; a.e = d.experts; a.k = d.k; a.sigmoid = d.score == QNN_SCORE_SIGMOID;
    // limiting the choice to all groups limits nothing
    a.groups = d.top_groups < d.groups ? d.groups : 1;
    a.top_groups = d.top_groups; a.two = d.group_score == QNN_GROUP_TOP2; a.renorm = d.renormalise; a.scale = d.scale;
    a.group_size = d.experts / d.groups;
    a.group_magic = ((1u << 20) + a.group_size - 1) / a.group_size;
    const int64_t row_bytes = d.ld * (d.dtype == QNN_F32 ? 4 : 2);
    a.vec = reinterpret_cast<uintptr_t>(logits) % 16 == 0 && row_bytes % 16 == 0;
    a.bias_vec = reinterpret_cast<uintptr_t>(bias) % 16 == 0;
    if (d.dtype == QNN_F32) return launch_route_type<float>(a, stream);
    if (d.dtype == QNN_F16) return launch_route_type<__half>(a, stream);
    return launch_route_type<__nv_bfloat16>(a, stream);
}

size_t expert_plan_workspace(int64_t slots, int experts)
{
    int64_t chunk;
    const int nb = plan_blocks(slots, &chunk);
    return nb > 1 ? static_cast<size_t>(nb) * experts * sizeof(int32_t) : 0;
}

cudaError_t launch_expert_plan(const int32_t *ids, int64_t slots, int experts, int32_t *offsets, int32_t *order,
                               int32_t *position, void *workspace, cudaStream_t stream)
{
    int64_t chunk;
    const int nb = plan_blocks(slots, &chunk);
    int32_t *counts = nb > 1 ? static_cast<int32_t *>(workspace) : nullptr;
    const size_t smem = sizeof(int32_t) * (kPlanWarps + 2) * experts;
    // The limit counts static memory too: always the most that any number of experts takes, before anything is queued.
    cudaError_t e = raise_smem<plan_place_kernel>(sizeof(int32_t) * (kPlanWarps + 2) * 1024);
    if (e != cudaSuccess) return e;
    if (counts) {
        e = launch_pdl(plan_count_kernel, dim3(nb), kPlanThreads, sizeof(int32_t) * experts, stream, 1, ids, slots, chunk, experts, counts);
        if (e != cudaSuccess) return e;
    }
    return launch_pdl(plan_place_kernel, dim3(nb), kPlanThreads, smem, stream, 1, ids, slots, chunk, experts, counts, offsets,
                      order, position);
}

}  // namespace qnn
