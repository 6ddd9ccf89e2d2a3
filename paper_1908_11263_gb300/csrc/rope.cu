// Rotary positions, and keys and values on their way into a paged cache.
//
// A pair (a, b) of a head at position p becomes (a cos - b sin, a sin + b cos) with the angle p f_i.  The angle is kept in
// turns, as a 64-bit binary fraction: turns[i] = f_i / 2 pi * 2^64, so p * turns[i] modulo 2^64 is the exact phase of
// p times the stored frequency, at any position and either sign, and its upper 32 bits are the angle to 2^-32 of a turn.
// A 32-bit product p * f_i would be off by p * 2^-24 radians, a tenth of a turn at a million.
//
// A block takes a few tokens: it finds their places in the cache, computes the cosines of a token once for all of its
// heads (a quarter of a microsecond, against one for each head), then moves rows as 16-byte vectors: where pointers and strides
// are aligned for that, and both the head's elements and its pairs are multiples of 8.  All else goes element by element, what
// is only copied too (8192 tokens of 40 heads of 80: 81 us with 40 elements rotated, 29 with all of them).
// Bound by its instructions for prompts (20011 tokens of 20 heads of 96, two thirds rotated: 35 us, 4.4 TB/s, 0.65 of a
// copy's, issue slots 72 % busy, some 290 instructions for an item) and by the host for a decode step (5 us of 11).  float32,
// whose vectors spill under the bound of five blocks an SM: 8192 tokens of 40 heads of 128 64 us, 5.2 TB/s.
#include "attention.h"
#include "block_common.cuh"

namespace qnn {
namespace {

constexpr int kRopeThreads = 256;
// Tokens of a block at most.  (Two, four, eight, each after a flush of the L2: the prompt above 50, 40 and 40 us; 8354 tokens of
// 32 + 8 heads of 128 into the cache 54, 50 and 64.)
constexpr int kRopeTokens = 4;

struct Place {
    int64_t position;  // of the rotation
    int64_t k, v;      // elements into the cache; -1: not written
    int live;          // belongs to a sequence (or there are none)
};

// Largest s in [0, seqs] with offsets[s] <= r; -1 where there is none.
__device__ __forceinline__ int sequence_of(const int32_t *offsets, int seqs, int64_t r)
{
    int lo = -1, hi = seqs + 1;
    while (hi - lo > 1) {
        const int mid = (lo + hi) >> 1;
        if (offsets[mid] <= r) lo = mid;
        else hi = mid;
    }
    return lo;
}

__device__ Place place_of(const RotateArgs &a, int64_t r)
{
    Place p = {0, -1, -1, 1};
    if (a.seqs >= 0) {
        int s;
        int64_t position;
        if (a.offsets) {
            s = sequence_of(a.offsets, a.seqs, r);
            if (s < 0 || s >= a.seqs) {
                p.live = 0;
                return p;
            }
            position = static_cast<int64_t>(a.lengths[s]) - a.offsets[s + 1] + r;
        } else {
            s = static_cast<int>(r / a.each);
            position = static_cast<int64_t>(a.lengths[s]) - a.each + (r - s * a.each);
        }
        p.position = position;
        if (position >= 0 && position < static_cast<int64_t>(a.width) * a.page_size) {
            const int column = static_cast<int>(position) / a.page_size, row = static_cast<int>(position) - column * a.page_size;
            const int page = a.table[s * a.ldt + column];
            if (page >= 0 && page < a.pages) {
                p.k = page * a.k_page + row * a.k_row;
                p.v = page * a.v_page + row * a.v_row;
            }
        }
    }
    if (a.positions)
        p.position = a.wide ? static_cast<const int64_t *>(a.positions)[r] : static_cast<const int32_t *>(a.positions)[r];
    return p;
}

// Sixteen rotated elements of a head, as loaded from two vectors, and where they go.
template <typename T>
__device__ __forceinline__ void rotate16(Raw8<T> &r0, Raw8<T> &r1, T *y0, T *y1, const float2 *cs, bool interleaved)
{
    float u[8], w[8];
    r0.get(u);
    r1.get(w);
    if (interleaved) {
#pragma unroll
        for (int i = 0; i < 4; ++i) {
            const float2 c = cs[i], e = cs[4 + i];
            const float a = u[2 * i], b = u[2 * i + 1], f = w[2 * i], g = w[2 * i + 1];
            u[2 * i] = a * c.x - b * c.y;
            u[2 * i + 1] = a * c.y + b * c.x;
            w[2 * i] = f * e.x - g * e.y;
            w[2 * i + 1] = f * e.y + g * e.x;
        }
    } else {
#pragma unroll
        for (int i = 0; i < 8; ++i) {
            const float2 c = cs[i];
            const float a = u[i], b = w[i];
            u[i] = a * c.x - b * c.y;
            w[i] = a * c.y + b * c.x;
        }
    }
    r0.set(u);
    r1.set(w);
    r0.store(y0);
    r1.store(y1);
}

// A thread's way through the items of a block's tokens and heads, from `first` on, `step` apart.
struct Walk {
    int token, head, item;
    int per, heads, by_token, by_head, by_item;

    __device__ __forceinline__ Walk(int heads_, int per_, int first, int step) : per(per_), heads(heads_)
    {
        place(step);
        by_token = token;
        by_head = head;
        by_item = item;
        place(first);
    }
    __device__ __forceinline__ void place(int i)
    {
        const int w = i / per;
        item = i - w * per;
        token = w / heads;
        head = w - token * heads;
    }
    __device__ __forceinline__ void next()
    {
        item += by_item;
        head += by_head;
        token += by_token;
        if (item >= per) {
            item -= per;
            ++head;
        }
        if (head >= heads) {
            head -= heads;
            ++token;
        }
    }
};

// Cosines and sines of a block's tokens, once their places are known.
__device__ __forceinline__ void angles(const RotateArgs &a, const Place *places, int count, float2 *cs)
{
    for (int i = threadIdx.x; i < count * a.half; i += kRopeThreads) {
        const int token = i / a.half, pair = i - token * a.half;
        const uint64_t phase = static_cast<uint64_t>(places[token].position) * a.turns[pair];
        float s, c;
        sincospif(static_cast<float>(static_cast<int32_t>(phase >> 32)) * 0x1p-31f, &s, &c);
        cs[i] = make_float2(a.amplitude * c, a.amplitude * s);
    }
}

template <typename T, bool VEC>
__global__ void __launch_bounds__(kRopeThreads, 5) rope_kernel(const RotateArgs a, const int tokens)
{
    extern __shared__ __align__(16) float2 cs[];  // [tokens][half]
    __shared__ Place places[kRopeTokens];
    const int tid = threadIdx.x;
    pdl_begin();
    const int64_t first = static_cast<int64_t>(blockIdx.x) * tokens;
    const int count = static_cast<int>(a.t - first < tokens ? a.t - first : tokens);
    const int heads = a.heads + a.kv_heads, dim = 2 * a.half;  // rotated heads: the queries', then the keys'
    if (tid < count) places[tid] = place_of(a, first + tid);

    auto source = [&](const Walk &w) {
        return w.head < a.heads ? static_cast<const T *>(a.x) + (first + w.token) * a.ldx + w.head * a.hx
                                : static_cast<const T *>(a.k) + (first + w.token) * a.ldk + (w.head - a.heads) * a.hk;
    };
    auto target = [&](const Walk &w) -> T * {  // null: not written
        const Place &p = places[w.token];
        if (w.head < a.heads) return p.live ? static_cast<T *>(a.y) + (first + w.token) * a.ldy + w.head * a.hy : nullptr;
        return p.k >= 0 ? static_cast<T *>(a.k_pages) + p.k + (w.head - a.heads) * a.k_head : nullptr;
    };
    if constexpr (VEC) {
        // Items of 16 rotated or 8 copied elements, two a thread at a time; the first ones are on their way while the cosines are
        // computed.
        const int turned = a.half / 8, apart = a.interleaved ? 8 : a.half;
        auto begin = [&](int item) { return item < turned ? (a.interleaved ? 16 : 8) * item : dim + 8 * (item - turned); };
        auto load = [&](const Walk &w, Raw8<T> &r0, Raw8<T> &r1) {
            if (w.token >= count) return;
            const T *x = source(w) + begin(w.item);
            r0.load(x);
            if (w.item < turned) r1.load(x + apart);
        };
        auto finish = [&](const Walk &w, Raw8<T> &r0, Raw8<T> &r1) {
            if (w.token >= count) return;
            T *y = target(w);
            if (!y) return;
            y += begin(w.item);
            if (w.item < turned) rotate16<T>(r0, r1, y, y + apart, cs + w.token * a.half + 8 * w.item, a.interleaved);
            else r0.store(y);
        };
        Walk u(heads, turned + (a.d - dim) / 8, tid, 2 * kRopeThreads), v = u;
        v.place(tid + kRopeThreads);
        Raw8<T> u0, u1, v0, v1;
        load(u, u0, u1);
        load(v, v0, v1);
        __syncthreads();
        angles(a, places, count, cs);
        __syncthreads();
        while (u.token < count) {
            finish(u, u0, u1);
            finish(v, v0, v1);
            u.next();
            v.next();
            load(u, u0, u1);
            load(v, v0, v1);
        }
        if (a.kv_heads > 0) {  // values, two a thread at a time as well
            auto take = [&](const Walk &w, Raw8<T> &r) {
                if (w.token < count) r.load(static_cast<const T *>(a.v) + (first + w.token) * a.ldv + w.head * a.hv + 8 * w.item);
            };
            auto put = [&](const Walk &w, const Raw8<T> &r) {
                if (w.token < count && places[w.token].v >= 0)
                    r.store(static_cast<T *>(a.v_pages) + places[w.token].v + w.head * a.v_head + 8 * w.item);
            };
            Walk x(a.kv_heads, a.d / 8, tid, 2 * kRopeThreads), y = x;
            y.place(tid + kRopeThreads);
            while (x.token < count) {
                take(x, u0);
                take(y, v0);
                put(x, u0);
                put(y, v0);
                x.next();
                y.next();
            }
        }
    } else {
        __syncthreads();
        angles(a, places, count, cs);
        __syncthreads();
        for (Walk w(heads, a.d - a.half, tid, kRopeThreads); w.token < count; w.next()) {
            const T *x = source(w);
            T *y = target(w);
            if (!y) continue;
            if (w.item < a.half) {
                const float2 c = cs[w.token * a.half + w.item];
                const int at = a.interleaved ? 2 * w.item : w.item, to = a.interleaved ? at + 1 : at + a.half;
                const float p = to_f32<T>(x[at]), q = to_f32<T>(x[to]);
                y[at] = from_f32<T>(p * c.x - q * c.y);
                y[to] = from_f32<T>(p * c.y + q * c.x);
            } else {
                y[a.half + w.item] = x[a.half + w.item];
            }
        }
        if (a.kv_heads > 0)
            for (Walk w(a.kv_heads, a.d, tid, kRopeThreads); w.token < count; w.next()) {
                const Place p = places[w.token];
                if (p.v < 0) continue;
                static_cast<T *>(a.v_pages)[p.v + w.head * a.v_head + w.item] =
                    static_cast<const T *>(a.v)[(first + w.token) * a.ldv + w.head * a.hv + w.item];
            }
    }
}

template <typename T>
cudaError_t launch(const RotateArgs &a, cudaStream_t st)
{
    // four tokens a block once there are blocks enough for every SM
    const int tokens = a.t >= 8 * kRopeTokens * device_sm_count() ? kRopeTokens : 1;
    const unsigned grid = static_cast<unsigned>((a.t + tokens - 1) / tokens);
    const size_t smem = sizeof(float2) * tokens * (a.half > 0 ? a.half : 1);
    constexpr uintptr_t kStep = sizeof(T) == 2 ? 8 : 4;  // elements of 16 bytes
    auto ok = [](const void *p) { return reinterpret_cast<uintptr_t>(p) % 16 == 0; };
    bool vec = a.half % 8 == 0 && a.d % 8 == 0 && ok(a.x) && ok(a.y) && ok(a.k) && ok(a.v) && ok(a.k_pages) && ok(a.v_pages);
    for (const int64_t s : {a.ldx, a.hx, a.ldy, a.hy, a.ldk, a.hk, a.ldv, a.hv, a.k_page, a.k_head, a.k_row, a.v_page, a.v_head, a.v_row})
        vec = vec && s % static_cast<int64_t>(kStep) == 0;
    return vec ? launch_pdl(rope_kernel<T, true>, dim3(grid), kRopeThreads, smem, st, 1, a, tokens)
               : launch_pdl(rope_kernel<T, false>, dim3(grid), kRopeThreads, smem, st, 1, a, tokens);
}

}  // namespace

cudaError_t launch_rotate(const RotateArgs &a, int dtype, cudaStream_t st)
{
    if (a.t == 0) return cudaSuccess;
    if (dtype == QNN_F16) return launch<__half>(a, st);
    if (dtype == QNN_BF16) return launch<__nv_bfloat16>(a, st);
    return launch<float>(a, st);
}

}  // namespace qnn
