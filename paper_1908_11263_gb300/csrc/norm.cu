// qnn_block_norm(): what stands between two blocks of a decoder, in one pass over the rows.
//
//   u = post_norm ? N(x) * post_w + post_b : x
//   r = residual + scale * gate * u
//   h = N(r) * pre_w + pre_b
//
// N divides by the root of the mean square (RMS) or subtracts the mean first (layer norm).  The kernel is bound by
// memory: x and the residual are read once, r and h written once.  One block owns one row and keeps it in registers
// as 32-bit values, so the second norm needs no second read; both statistics are block reductions.  h is computed from
// r before r is rounded to its own type: each output is rounded once.  The layer norm's variance is a second reduction
// over the centred values, not a difference of two sums that would cancel.
// Measured: 16384 x 8192 bf16 with a 32-bit residual, both norms and a gate, 248 us (6.5 TB/s); 8 x 4096 3.5 us.
#include "block_common.cuh"
#include "block_internal.h"
#include "device.cuh"

namespace qnn {
namespace {

struct NormArgs {
    const void *x, *residual, *gate, *post_w, *post_b, *pre_w, *pre_b;
    void *r, *h;
    int64_t ldx, ldres, ldr, ldh;
    int64_t rows_per_gate;  // rows that share one gate row
    int d, layer, post, param_f32;
    float scale, eps;
};

// Sum over the block.  Each reduction uses its own row of `part` (zeros past the block's warps), so one barrier a
// reduction is enough; every thread adds the warps' sums itself, in the same order.
__device__ __forceinline__ float block_sum(float v, float *part)
{
#pragma unroll
    for (int o = 16; o > 0; o >>= 1) v += __shfl_xor_sync(0xffffffffu, v, o);
    if (blockDim.x == 32) return v;
    if ((threadIdx.x & 31) == 0) part[threadIdx.x >> 5] = v;
    __syncthreads();
    float s = 0.f;
    for (int w = 0; w < static_cast<int>(blockDim.x >> 5); w += 4) {
        const float4 q = *reinterpret_cast<const float4 *>(part + w);
        s += (q.x + q.y) + (q.z + q.w);
    }
    return s;
}

template <typename T>
__device__ __forceinline__ void load4(const T *p, float *v)
{
    if constexpr (sizeof(T) == 4) {
        const float4 q = *reinterpret_cast<const float4 *>(p);
        v[0] = q.x; v[1] = q.y; v[2] = q.z; v[3] = q.w;
    } else {
        const uint2 q = *reinterpret_cast<const uint2 *>(p);
        const float2 a = unpack2<T>(q.x), b = unpack2<T>(q.y);
        v[0] = a.x; v[1] = a.y; v[2] = b.x; v[3] = b.y;
    }
}

template <typename T>
__device__ __forceinline__ void store4(T *p, const float *v)
{
    if constexpr (sizeof(T) == 4)
        *reinterpret_cast<float4 *>(p) = make_float4(v[0], v[1], v[2], v[3]);
    else
        *reinterpret_cast<uint2 *>(p) = make_uint2(pack2<T>(v[0], v[1]), pack2<T>(v[2], v[3]));
}

// A thread's values of a row, eight to an item.  VEC = 8: eight neighbours, one 16-byte access of 16-bit values.
// VEC = 4: two runs of four neighbours, a whole block's threads apart, for rows with a 32-bit tensor among them: its
// 16-byte accesses then cover whole sectors (two halves of 32 bytes a lane made each store a partial one).  VEC = 1:
// single elements a block's threads apart, so that neighbouring lanes touch neighbouring elements whatever the alignment.
// EXACT: rows are whole vectors.
template <int VEC, int ITEMS, bool EXACT = false>
struct Row {
    static __device__ __forceinline__ int at(int i, int j)
    {
        return ((i * 8 + j) / VEC * static_cast<int>(blockDim.x) + static_cast<int>(threadIdx.x)) * VEC + j % VEC;
    }

    template <typename T>
    static __device__ __forceinline__ void load(const T *p, int i, int d, float (&v)[8])
    {
#pragma unroll
        for (int h = 0; h < 8; h += VEC) {
            if (VEC > 1 && (EXACT ? at(i, h) : at(i, h + VEC - 1)) < d) {
                if constexpr (VEC == 8) {
                    Raw8<T> q;
                    q.load(p + at(i, 0));
                    q.get(v);
                } else {
                    load4(p + at(i, h), v + h);
                }
            } else {
#pragma unroll
                for (int j = h; j < h + VEC; ++j) v[j] = !EXACT && at(i, j) < d ? to_f32<T>(p[at(i, j)]) : 0.f;
            }
        }
    }

    template <typename T>
    static __device__ __forceinline__ void store(T *p, int i, int d, const float (&v)[8])
    {
#pragma unroll
        for (int h = 0; h < 8; h += VEC) {
            if (VEC > 1 && (EXACT ? at(i, h) : at(i, h + VEC - 1)) < d) {
                if constexpr (VEC == 8) {
                    Raw8<T> q;
                    q.set(v);
                    q.store(p + at(i, 0));
                } else {
                    store4(p + at(i, h), v + h);
                }
            } else if (!EXACT) {
#pragma unroll
                for (int j = h; j < h + VEC; ++j)
                    if (at(i, j) < d) p[at(i, j)] = from_f32<T>(v[j]);
            }
        }
    }

    // A parameter row, in the type of x or in 32 bits.
    template <typename T>
    static __device__ __forceinline__ void param(const void *p, int f32, int64_t off, int i, int d, float (&v)[8])
    {
        if (f32)
            load(static_cast<const float *>(p) + off, i, d, v);
        else
            load(static_cast<const T *>(p) + off, i, d, v);
    }

    // Scales v to unit root mean square (after removing the mean for layer norms).
    static __device__ __forceinline__ void normalise(float (&v)[ITEMS][8], const NormArgs &a, float (*part)[32])
    {
        const float inv_d = 1.f / static_cast<float>(a.d);
        float mean = 0.f;
        if (a.layer) {
            float s = 0.f;
#pragma unroll
            for (int i = 0; i < ITEMS; ++i)
#pragma unroll
                for (int j = 0; j < 8; ++j) s += v[i][j];
            mean = block_sum(s, part[0]) * inv_d;
        }
        float q = 0.f;
#pragma unroll
        for (int i = 0; i < ITEMS; ++i)
#pragma unroll
            for (int j = 0; j < 8; ++j) {
                if (a.layer && at(i, EXACT ? j / VEC * VEC : j) < a.d) v[i][j] -= mean;  // values past the row's end stay zero
                q = fmaf(v[i][j], v[i][j], q);
            }
        const float f = rsqrtf(block_sum(q, part[1]) * inv_d + a.eps);
#pragma unroll
        for (int i = 0; i < ITEMS; ++i)
#pragma unroll
            for (int j = 0; j < 8; ++j) v[i][j] *= f;
    }

    template <typename T>
    static __device__ __forceinline__ void affine(float (&v)[ITEMS][8], const void *w, const void *b, const NormArgs &a)
    {
#pragma unroll
        for (int i = 0; i < ITEMS; ++i) {
            float p[8];
            if (w) {
                param<T>(w, a.param_f32, 0, i, a.d, p);
#pragma unroll
                for (int j = 0; j < 8; ++j) v[i][j] *= p[j];
            }
            if (b) {
                param<T>(b, a.param_f32, 0, i, a.d, p);
#pragma unroll
                for (int j = 0; j < 8; ++j) v[i][j] += p[j];
            }
        }
    }
};

template <typename T, typename R, int VEC, int ITEMS>
__global__ void __launch_bounds__(1024) block_norm_kernel(const NormArgs a)
{
    __shared__ __align__(16) float part[4][32];
    using Q = Row<VEC, ITEMS>;
    if (threadIdx.x < 32)
#pragma unroll
        for (int i = 0; i < 4; ++i) part[i][threadIdx.x] = 0.f;
    __syncthreads();
    pdl_begin();
    const int64_t row = blockIdx.x;
    const T *x = static_cast<const T *>(a.x) + row * a.ldx;
    float v[ITEMS][8], res[ITEMS][8];
#pragma unroll
    for (int i = 0; i < ITEMS; ++i) Q::load(x, i, a.d, v[i]);
    if (a.residual) {
        const R *p = static_cast<const R *>(a.residual) + row * a.ldres;
#pragma unroll
        for (int i = 0; i < ITEMS; ++i) Q::load(p, i, a.d, res[i]);
    }
    if (a.post) {
        Q::normalise(v, a, part);
        Q::template affine<T>(v, a.post_w, a.post_b, a);
    }
    const int64_t gate_row = a.gate ? row / a.rows_per_gate : 0;
#pragma unroll
    for (int i = 0; i < ITEMS; ++i) {
        if (a.gate) {
            float g[8];
            Q::template param<T>(a.gate, a.param_f32, gate_row * a.d, i, a.d, g);
#pragma unroll
            for (int j = 0; j < 8; ++j) v[i][j] *= g[j];
        }
#pragma unroll
        for (int j = 0; j < 8; ++j) v[i][j] = a.residual ? fmaf(a.scale, v[i][j], res[i][j]) : a.scale * v[i][j];
    }
    if (a.r) {
        R *p = static_cast<R *>(a.r) + row * a.ldr;
#pragma unroll
        for (int i = 0; i < ITEMS; ++i) Q::store(p, i, a.d, v[i]);
    }
    if (a.h) {
        T *p = static_cast<T *>(a.h) + row * a.ldh;
        Q::normalise(v, a, part + 2);
        Q::template affine<T>(v, a.pre_w, a.pre_b, a);
#pragma unroll
        for (int i = 0; i < ITEMS; ++i) Q::store(p, i, a.d, v[i]);
    }
}

// The same over many rows: a block that stays on its SM and takes every gridDim-th row, fed by bulk copies `stages` rows
// ahead, so that the loads of the next rows run under the reductions of this one (with a block a row, every SM waits for
// its rows' loads, then for their reductions).  Rows are whole 16-byte vectors here.
// Weights and a gate in the type of x stay in registers from row to row, as packed words.
template <typename T, int VEC>
struct Held {
    uint32_t w[2][4];
    __device__ __forceinline__ void load(const void *p, int64_t off, int d)
    {
        const uint32_t *q = reinterpret_cast<const uint32_t *>(static_cast<const T *>(p) + off);
#pragma unroll
        for (int i = 0; i < 2; ++i)
#pragma unroll
            for (int h = 0; h < 8; h += VEC) {
                if (Row<VEC, 2>::at(i, h) >= d) {  // values past the row's end are zero and stay zero
                    for (int j = h / 2; j < (h + VEC) / 2; ++j) w[i][j] = 0u;
                    continue;
                }
                if constexpr (VEC == 8) {
                    const uint4 u = *reinterpret_cast<const uint4 *>(q + Row<VEC, 2>::at(i, 0) / 2);
                    w[i][0] = u.x; w[i][1] = u.y; w[i][2] = u.z; w[i][3] = u.w;
                } else {
                    const uint2 u = *reinterpret_cast<const uint2 *>(q + Row<VEC, 2>::at(i, h) / 2);
                    w[i][h / 2] = u.x; w[i][h / 2 + 1] = u.y;
                }
            }
    }
    __device__ __forceinline__ void scale(float (&v)[2][8]) const
    {
#pragma unroll
        for (int i = 0; i < 2; ++i)
#pragma unroll
            for (int j = 0; j < 4; ++j) {
                const float2 f = unpack2<T>(w[i][j]);
                v[i][2 * j] *= f.x;
                v[i][2 * j + 1] *= f.y;
            }
    }
};
template <int VEC>
struct Held<float, VEC> {  // 32-bit rows: read again for each row
    __device__ __forceinline__ void load(const void *, int64_t, int) {}
    __device__ __forceinline__ void scale(float (&)[2][8]) const {}
};

struct NormShared {
    float part[2][4][32];
    uint64_t full[8];
};
static_assert((sizeof(NormShared) + 127) / 128 * 128 == kNormStatic, "shared memory that norm_ring() reckons with");

template <typename T, typename R, int VEC>
__global__ void __launch_bounds__(1024) block_norm_stream_kernel(const NormArgs a, const NormRing s, int64_t t, int *status)
{
    extern __shared__ __align__(128) uint8_t ring[];
    __shared__ __align__(16) NormShared shared;
    auto &part = shared.part;
    uint64_t *full = shared.full;
    using Q = Row<VEC, kNormItems, true>;
    const uint32_t stage_bytes = s.x_bytes + s.res_bytes;
    if (threadIdx.x == 0) {
        for (int i = 0; i < s.stages; ++i) mbar_init(full + i, 1);
        fence_mbar_init();
    }
    if (threadIdx.x < 32)
#pragma unroll
        for (int i = 0; i < 8; ++i) part[i >> 2][i & 3][threadIdx.x] = 0.f;
    __syncthreads();
    pdl_begin();
    auto fetch = [&](int64_t row, int st) {
        uint8_t *dst = ring + st * stage_bytes;
        mbar_arrive_expect_tx(full + st, stage_bytes);
        if (s.res_bytes) bulk_g2s(dst + s.x_bytes, static_cast<const R *>(a.residual) + row * a.ldres, s.res_bytes, full + st);
        bulk_g2s(dst, static_cast<const T *>(a.x) + row * a.ldx, s.x_bytes, full + st);
    };
    if (threadIdx.x == 0)
        for (int i = 0; i < s.stages; ++i) {
            const int64_t row = blockIdx.x + static_cast<int64_t>(i) * gridDim.x;
            if (row < t) fetch(row, i);
        }
    const bool hold = sizeof(T) == 2 && !a.param_f32;
    const bool post_w = a.post && a.post_w;
    Held<T, VEC> hold_post, hold_gate, hold_pre;
    if (hold) {
        if (post_w) hold_post.load(a.post_w, 0, a.d);
        if (a.h && a.pre_w) hold_pre.load(a.pre_w, 0, a.d);
    }
    int64_t held_gate = -1;
    int st = 0, n = 0;
    uint32_t phase = 0;
    for (int64_t row = blockIdx.x; row < t; row += gridDim.x, ++n) {
        const int64_t gate_row = a.gate ? static_cast<int64_t>(static_cast<uint32_t>(row) / static_cast<uint32_t>(a.rows_per_gate)) : 0;
        if (hold && a.gate && gate_row != held_gate) {
            hold_gate.load(a.gate, gate_row * a.d, a.d);
            held_gate = gate_row;
        }
        // a thread that gives up goes on (the status word tells the caller), so that the block's barriers stay whole
        mbar_wait_warp(full + st, phase, status);
        const T *x = reinterpret_cast<const T *>(ring + st * stage_bytes);
        const R *res = reinterpret_cast<const R *>(ring + st * stage_bytes + s.x_bytes);
        float v[kNormItems][8];
#pragma unroll
        for (int i = 0; i < kNormItems; ++i) Q::load(x, i, a.d, v[i]);
        if (a.post) {
            Q::normalise(v, a, part[n & 1]);
            if (post_w && hold) hold_post.scale(v);
            Q::template affine<T>(v, hold ? nullptr : a.post_w, a.post_b, a);
        }
        if (a.gate && hold) hold_gate.scale(v);
#pragma unroll
        for (int i = 0; i < kNormItems; ++i) {
            float g[8];
            if (a.gate && !hold) {
                Q::template param<T>(a.gate, a.param_f32, gate_row * a.d, i, a.d, g);
#pragma unroll
                for (int j = 0; j < 8; ++j) v[i][j] *= g[j];
            }
            if (s.res_bytes) {
                Q::load(res, i, a.d, g);
#pragma unroll
                for (int j = 0; j < 8; ++j) v[i][j] = fmaf(a.scale, v[i][j], g[j]);
            } else {
#pragma unroll
                for (int j = 0; j < 8; ++j) v[i][j] *= a.scale;
            }
        }
        if (a.r) {
            R *p = static_cast<R *>(a.r) + row * a.ldr;
#pragma unroll
            for (int i = 0; i < kNormItems; ++i) Q::store(p, i, a.d, v[i]);
        }
        if (a.h)
            Q::normalise(v, a, part[n & 1] + 2);
        else
            __syncthreads();
        // every thread is past its reads of the stage: the reduction's barrier (or the one above) lies between
        const int64_t next = row + static_cast<int64_t>(s.stages) * gridDim.x;
        if (threadIdx.x == 0 && next < t) fetch(next, st);
        if (a.h) {
            if (a.pre_w && hold) hold_pre.scale(v);
            Q::template affine<T>(v, hold ? nullptr : a.pre_w, a.pre_b, a);
            T *p = static_cast<T *>(a.h) + row * a.ldh;
#pragma unroll
            for (int i = 0; i < kNormItems; ++i) Q::store(p, i, a.d, v[i]);
        }
        if (++st == s.stages) {
            st = 0;
            phase ^= 1;
        }
    }
}

template <typename T, typename R, int VEC>
cudaError_t launch_stream(const NormArgs &a, int64_t t, cudaStream_t stream, bool *taken)
{
    *taken = false;
    if (a.d % 8 || a.d > 8192 * kNormItems) return cudaSuccess;
    int *status = device_status_ptr();
    if (!status) return cudaErrorNotSupported;
    const NormRing s = norm_ring(a.d, a.d * sizeof(T), a.residual ? a.d * sizeof(R) : 0);
    const int blocks = s.per_sm * device_sm_count();
    // a few rows a block at least, or the ring does not pay for itself
    if (s.stages < 2 || t < 3ll * blocks) return cudaSuccess;
    const cudaError_t e = raise_smem<block_norm_stream_kernel<T, R, VEC>>(kNormRoom);
    if (e != cudaSuccess) return e;
    *taken = true;
    return launch_pdl(block_norm_stream_kernel<T, R, VEC>, dim3(blocks), s.threads, s.smem, stream, 1, a, s, t, status);
}

bool rows_aligned(const void *p, int64_t ld, int size)
{
    return reinterpret_cast<uintptr_t>(p) % 16 == 0 && (ld * size) % 16 == 0;
}

template <typename T, typename R, int VEC>
cudaError_t launch_items(const NormArgs &a, int64_t t, cudaStream_t stream)
{
    // Eight values a thread up to rows of 8192, the most threads and the shortest chain; longer rows take more.
    const int chunks = (a.d + 7) / 8;
    const int items = chunks <= 1024 ? 1 : chunks <= 2048 ? 2 : 4;
    const int threads = ((chunks + items - 1) / items + 31) / 32 * 32;
    const dim3 grid(static_cast<unsigned>(t));
    if (items == 1) return launch_pdl(block_norm_kernel<T, R, VEC, 1>, grid, threads, 0, stream, 1, a);
    if (items == 2) return launch_pdl(block_norm_kernel<T, R, VEC, 2>, grid, threads, 0, stream, 1, a);
    return launch_pdl(block_norm_kernel<T, R, VEC, 4>, grid, threads, 0, stream, 1, a);
}

template <typename T, typename R>
cudaError_t launch_vec(const NormArgs &a, int64_t t, cudaStream_t stream)
{
    const int sx = sizeof(T), sr = sizeof(R), sp = a.param_f32 ? 4 : sx;
    const bool vec = rows_aligned(a.x, a.ldx, sx) && rows_aligned(a.residual, a.residual ? a.ldres : 0, sr) &&
                     rows_aligned(a.r, a.r ? a.ldr : 0, sr) && rows_aligned(a.h, a.h ? a.ldh : 0, sx) &&
                     rows_aligned(a.gate, a.gate ? a.d : 0, sp) && rows_aligned(a.post_w, 0, sp) &&
                     rows_aligned(a.post_b, 0, sp) && rows_aligned(a.pre_w, 0, sp) && rows_aligned(a.pre_b, 0, sp);
    if (!vec) return launch_items<T, R, 1>(a, t, stream);
    constexpr int kVec = sizeof(R) == 4 ? 4 : 8;
    bool taken = false;
    const cudaError_t e = launch_stream<T, R, kVec>(a, t, stream, &taken);
    return e != cudaSuccess || taken ? e : launch_items<T, R, kVec>(a, t, stream);
}

}  // namespace

cudaError_t launch_block_norm(const qnn_norm_desc &d, const void *x, const void *residual, const void *gate,
                              const void *post_w, const void *post_b, const void *pre_w, const void *pre_b, void *r,
                              void *h, cudaStream_t stream)
{
    if (d.t == 0) return cudaSuccess;
    NormArgs a;
    a.x = x; a.residual = residual; a.gate = gate;
    a.post_w = d.post_norm ? post_w : nullptr;
    a.post_b = d.post_norm ? post_b : nullptr;
    a.pre_w = pre_w; a.pre_b = pre_b; a.r = r; a.h = h;
    a.ldx = d.ldx; a.ldres = d.ldres; a.ldr = d.ldr; a.ldh = d.ldh;
    a.rows_per_gate = gate ? d.t / d.gates : 1;
    a.d = d.d; a.layer = d.kind == QNN_NORM_LAYER; a.post = d.post_norm; a.param_f32 = d.param_dtype == QNN_F32;
    a.scale = d.scale; a.eps = d.eps;
    const bool wide = d.residual_dtype == QNN_F32;
    if (d.dtype == QNN_F16) return wide ? launch_vec<__half, float>(a, d.t, stream) : launch_vec<__half, __half>(a, d.t, stream);
    if (d.dtype == QNN_BF16)
        return wide ? launch_vec<__nv_bfloat16, float>(a, d.t, stream)
                    : launch_vec<__nv_bfloat16, __nv_bfloat16>(a, d.t, stream);
    return launch_vec<float, float>(a, d.t, stream);
}

}  // namespace qnn
