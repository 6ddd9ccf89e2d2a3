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
#include "block_common.cuh"
#include "block_internal.h"

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

// Sum over the block.  Each reduction uses its own row of `part`, so one barrier a reduction is enough.
__device__ __forceinline__ float block_sum(float v, float *part)
{
#pragma unroll
    for (int o = 16; o > 0; o >>= 1) v += __shfl_xor_sync(0xffffffffu, v, o);
    const int warps = blockDim.x >> 5;
    if (warps == 1) return v;
    if ((threadIdx.x & 31) == 0) part[threadIdx.x >> 5] = v;
    __syncthreads();
    float s = static_cast<int>(threadIdx.x & 31) < warps ? part[threadIdx.x & 31] : 0.f;
#pragma unroll
    for (int o = 16; o > 0; o >>= 1) s += __shfl_xor_sync(0xffffffffu, s, o);
    return s;
}

// A thread's values of a row.  VEC: chunks of 8 neighbours, chunk i at (i * threads + tid) * 8.  Otherwise
// value e of the thread is element e * threads + tid, so that neighbouring lanes touch neighbouring elements
// whatever the alignment.
template <bool VEC, int ITEMS>
struct Row {
    static __device__ __forceinline__ int at(int i, int j)
    {
        return VEC ? (i * static_cast<int>(blockDim.x) + static_cast<int>(threadIdx.x)) * 8 + j
                   : (i * 8 + j) * static_cast<int>(blockDim.x) + static_cast<int>(threadIdx.x);
    }

    template <typename T>
    static __device__ __forceinline__ void load(const T *p, int i, int d, float (&v)[8])
    {
        if (VEC && at(i, 7) < d) {
            Raw8<T> q;
            q.load(p + at(i, 0));
            q.get(v);
        } else {
#pragma unroll
            for (int j = 0; j < 8; ++j) v[j] = at(i, j) < d ? to_f32<T>(p[at(i, j)]) : 0.f;
        }
    }

    template <typename T>
    static __device__ __forceinline__ void store(T *p, int i, int d, const float (&v)[8])
    {
        if (VEC && at(i, 7) < d) {
            Raw8<T> q;
            q.set(v);
            q.store(p + at(i, 0));
        } else {
#pragma unroll
            for (int j = 0; j < 8; ++j)
                if (at(i, j) < d) p[at(i, j)] = from_f32<T>(v[j]);
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
            for (int j = 0; j < 8; ++j)
                if (at(i, j) < a.d) {
                    v[i][j] -= mean;
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

template <typename T, typename R, bool VEC, int ITEMS, int MAX_THREADS>
__global__ void __launch_bounds__(MAX_THREADS) block_norm_kernel(const NormArgs a)
{
    __shared__ float part[4][32];
    using Q = Row<VEC, ITEMS>;
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

bool rows_aligned(const void *p, int64_t ld, int size)
{
    return reinterpret_cast<uintptr_t>(p) % 16 == 0 && (ld * size) % 16 == 0;
}

template <typename T, typename R, bool VEC>
cudaError_t launch_items(const NormArgs &a, int64_t t, cudaStream_t stream)
{
    // Values a thread: few rows want many threads a row (latency), many rows want fewer and longer ones, which leave
    // more loads in flight for each barrier.  At most 1024 threads.
    const int chunks = (a.d + 7) / 8;
    int items = t > 2 * device_sm_count() ? (chunks >= 1024 ? 4 : chunks >= 256 ? 2 : 1) : 1;
    while (items < 4 && (chunks + items - 1) / items > 1024) items *= 2;
    const int threads = ((chunks + items - 1) / items + 31) / 32 * 32;
    const dim3 grid(static_cast<unsigned>(t));
    if (items == 1)
        block_norm_kernel<T, R, VEC, 1, 1024><<<grid, threads, 0, stream>>>(a);
    else if (items == 2)
        block_norm_kernel<T, R, VEC, 2, 1024><<<grid, threads, 0, stream>>>(a);
    else if (threads <= 512)
        block_norm_kernel<T, R, VEC, 4, 512><<<grid, threads, 0, stream>>>(a);
    else  // rows above 16384: 64 registers a thread are all there are
        block_norm_kernel<T, R, VEC, 4, 1024><<<grid, threads, 0, stream>>>(a);
    return cudaGetLastError();
}

template <typename T, typename R>
cudaError_t launch_vec(const NormArgs &a, int64_t t, cudaStream_t stream)
{
    const int sx = sizeof(T), sr = sizeof(R), sp = a.param_f32 ? 4 : sx;
    const bool vec = rows_aligned(a.x, a.ldx, sx) && rows_aligned(a.residual, a.residual ? a.ldres : 0, sr) &&
                     rows_aligned(a.r, a.r ? a.ldr : 0, sr) && rows_aligned(a.h, a.h ? a.ldh : 0, sx) &&
                     rows_aligned(a.gate, a.gate ? a.d : 0, sp) && rows_aligned(a.post_w, 0, sp) &&
                     rows_aligned(a.post_b, 0, sp) && rows_aligned(a.pre_w, 0, sp) && rows_aligned(a.pre_b, 0, sp);
    return vec ? launch_items<T, R, true>(a, t, stream) : launch_items<T, R, false>(a, t, stream);
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
