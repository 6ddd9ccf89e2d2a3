// Rotary positions, and keys and values on their way into a paged cache.
//
// A pair (a, b) of a head at position p becomes (a cos - b sin, a sin + b cos) with the angle p f_i.  The angle is kept in
// turns, as a 64-bit binary fraction: turns[i] = f_i / 2 pi * 2^64, so p * turns[i] modulo 2^64 is the exact phase of
// p times the stored frequency, at any position and either sign, and its upper 32 bits are the angle to 2^-32 of a turn.
// A 32-bit product p * f_i would be off by p * 2^-24 radians, a tenth of a turn at a million.
//
// A block takes a few tokens: it finds their places in the cache, computes the cosines of a token once for all of its
// heads (a quarter of a microsecond, against one for each head), then moves rows as 16-byte vectors.  Rows that are not
// aligned for that go element by element.
// Bound by HBM for prompts and by the launch for a decode step.
#include "attention.h"
#include "block_common.cuh"

namespace qnn {
namespace {

constexpr int kRopeThreads = 256;
constexpr int kRopeTokens = 4;  // of a block at most

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

// Sixteen rotated elements of a head: the vectors at x0 and x1, and where they go.
template <typename T>
__device__ __forceinline__ void rotate16(const T *x0, const T *x1, T *y0, T *y1, const float2 *cs, bool interleaved)
{
    Raw8<T> r0, r1;
    r0.load(x0);
    r1.load(x1);
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

template <typename T, bool VEC>
__global__ void __launch_bounds__(kRopeThreads) rope_kernel(const RotateArgs a, const int tokens)
{
    extern __shared__ float2 cs[];  // [tokens][half]
    __shared__ Place places[kRopeTokens];
    const int tid = threadIdx.x;
    pdl_begin();
    const int64_t first = static_cast<int64_t>(blockIdx.x) * tokens;
    const int count = static_cast<int>(a.t - first < tokens ? a.t - first : tokens);
    if (tid < count) places[tid] = place_of(a, first + tid);
    __syncthreads();
    for (int i = tid; i < count * a.half; i += kRopeThreads) {
        const int token = i / a.half, pair = i - token * a.half;
        const uint64_t phase = static_cast<uint64_t>(places[token].position) * a.turns[pair];
        float s, c;
        sincospif(static_cast<float>(static_cast<int32_t>(phase >> 32)) * 0x1p-31f, &s, &c);
        cs[i] = make_float2(a.amplitude * c, a.amplitude * s);
    }
    __syncthreads();

    // rotated heads: the queries', then the keys'
    const int heads = a.heads + a.kv_heads, dim = 2 * a.half;
    const int per = VEC ? a.half / 8 + (a.d - dim) / 8 : a.half + (a.d - dim);  // items of a head
    const int slots = kRopeThreads / per > 0 ? kRopeThreads / per : 1;
    const int step = slots == 1 ? kRopeThreads : per;  // items of a head a pass
    const int slot = slots == 1 ? 0 : tid / per, item0 = slots == 1 ? tid : tid - slot * per;
    if (slot < slots)
        for (int w = slot; w < count * heads; w += slots) {
            const int token = w / heads, head = w - token * heads;
            const Place p = places[token];
            const T *x;
            T *y;
            if (head < a.heads) {
                if (!p.live) continue;
                x = static_cast<const T *>(a.x) + (first + token) * a.ldx + head * a.hx;
                y = static_cast<T *>(a.y) + (first + token) * a.ldy + head * a.hy;
            } else {
                if (p.k < 0) continue;
                x = static_cast<const T *>(a.k) + (first + token) * a.ldk + (head - a.heads) * a.hk;
                y = static_cast<T *>(a.k_pages) + p.k + (head - a.heads) * a.k_head;
            }
            const float2 *c = cs + token * a.half;
            for (int item = item0; item < per; item += step) {
                if constexpr (VEC) {
                    if (item < a.half / 8) {
                        const int at = a.interleaved ? 16 * item : 8 * item, to = a.interleaved ? at + 8 : at + a.half;
                        rotate16<T>(x + at, x + to, y + at, y + to, c + 8 * item, a.interleaved);
                    } else {
                        const int at = dim + 8 * (item - a.half / 8);
                        Raw8<T> r;
                        r.load(x + at);
                        r.store(y + at);
                    }
                } else {
                    if (item < a.half) {
                        const int at = a.interleaved ? 2 * item : item, to = a.interleaved ? at + 1 : at + a.half;
                        const float u = to_f32<T>(x[at]), v = to_f32<T>(x[to]);
                        y[at] = from_f32<T>(u * c[item].x - v * c[item].y);
                        y[to] = from_f32<T>(u * c[item].y + v * c[item].x);
                    } else {
                        y[a.half + item] = x[a.half + item];
                    }
                }
            }
        }
    // values
    const int vper = VEC ? a.d / 8 : a.d;
    for (int i = tid; i < count * a.kv_heads * vper; i += kRopeThreads) {
        const int row = i / vper, at = i - row * vper, token = row / a.kv_heads, head = row - token * a.kv_heads;
        const Place p = places[token];
        if (p.v < 0) continue;
        const T *x = static_cast<const T *>(a.v) + (first + token) * a.ldv + head * a.hv;
        T *y = static_cast<T *>(a.v_pages) + p.v + head * a.v_head;
        if constexpr (VEC) {
            Raw8<T> r;
            r.load(x + 8 * at);
            r.store(y + 8 * at);
        } else {
            y[at] = x[at];
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
