// Shared by the matrix-product kernels: the weight image qnn_matmul_prepare() writes, the arguments of a launch, the
// expansion of packed codes and the fused epilogue.
//
// Image.  Rows of the weight matrix are taken 32 at a time and columns 64 at a time; blocks follow one another along K,
// then along the rows, then along the experts, so that a kernel streams whole blocks with bulk copies.  A gated matrix
// (gate rows, then up rows) is interleaved eight by eight: rows 16 i .. 16 i + 7 of the image are gate channels 8 i ..,
// the next eight the same channels' up rows, so one thread or one pair of lanes meets both.
//   16-bit weights: 32 rows of 128 bytes, 16-byte chunk c of row r at chunk c ^ (r & 7): the 128-byte swizzle that
//     tcgen05.mma reads, so a block goes to shared memory as it is.
//   packed weights: codes biased to unsigned, in the order of the m16n8k16 A fragment: lane 4 g + t of a warp holds rows
//     g and g + 8 of each 16, columns 16 t .. 16 t + 15.  Within a 32-bit word the codes of a column pair sit 16 bits
//     apart, so one mask and one or expand two codes at once.
// After the blocks: one {scale, bias} pair of floats a row.
//
// Exactness.  A code of at most 8 bits is a whole number of at most 2^7 and exact in f16 and bf16, so the tensor cores
// multiply the codes themselves; the channel's scale is applied once, in 32 bits, in the epilogue.
#pragma once

#include "block_common.cuh"
#include "block_internal.h"
#include "device.cuh"

namespace qnn {

struct MatmulImage {
    int rows;        // image rows of one expert (multiple of 32)
    int mb, kb;      // blocks along the rows and along K
    uint32_t block_bytes;
    size_t param_off, bytes;
};

__host__ __device__ inline MatmulImage matmul_image(int experts, int m, int k, int bits, int gated)
{
    MatmulImage g;
    const int rows = gated ? (m + 7) / 8 * 16 : m;
    g.mb = (rows + 31) / 32;
    g.rows = g.mb * 32;
    g.kb = (k + 63) / 64;
    g.block_bytes = 32 * 64 * bits / 8;
    g.param_off = static_cast<size_t>(experts) * g.mb * g.kb * g.block_bytes;
    g.bytes = g.param_off + static_cast<size_t>(experts) * g.rows * sizeof(float2);
    return g;
}

// One product launch.  Plain product: plan == nullptr, rows = t.  Experts: places are the plan's sorted places, and
// `gather` says whether x has a row per token (order[place] / top) or per place.
struct MatmulArgs {
    const uint8_t *image;
    const float2 *params;      // [experts][image rows]
    const void *x;
    const void *residual;      // plain product only
    void *y;                   // T, or float when out_f32
    const int32_t *offsets;    // experts + 1 places, or null
    const int32_t *order;      // slot of each place (gather)
    int64_t ldx, ldres, ldy;
    int64_t rows;              // tokens of a plain product; slots of an experts' product
    int64_t x_rows;            // rows that x has
    int m, k, kb, mb, experts, top;
    int act, gated, out_f32, gather, zero_tail;
    int x_vec;                 // rows of x are 16-byte aligned
};

// ---------------------------------------------------------------- codes

template <typename T>
struct CodeConst;
template <>
struct CodeConst<__half> {
    static constexpr uint32_t kMagic = 0x64006400u;  // 1024 + v, v < 1024
    static constexpr uint32_t kMid4 = 0x64086408u, kMid2 = 0x64026402u, kMid8 = 0x64806480u;
};
template <>
struct CodeConst<__nv_bfloat16> {
    static constexpr uint32_t kMagic = 0x43004300u;  // 128 + v, v < 128
    static constexpr uint32_t kMid4 = 0x43084308u, kMid2 = 0x43024302u, kMid8 = 0u;
};

template <typename T>
__device__ __forceinline__ uint32_t sub2(uint32_t a, uint32_t b);
template <>
__device__ __forceinline__ uint32_t sub2<__half>(uint32_t a, uint32_t b)
{
    const __half2 r = __hsub2(*reinterpret_cast<__half2 *>(&a), *reinterpret_cast<__half2 *>(&b));
    return *reinterpret_cast<const uint32_t *>(&r);
}
template <>
__device__ __forceinline__ uint32_t sub2<__nv_bfloat16>(uint32_t a, uint32_t b)
{
    const __nv_bfloat162 r = __hsub2(*reinterpret_cast<__nv_bfloat162 *>(&a), *reinterpret_cast<__nv_bfloat162 *>(&b));
    return *reinterpret_cast<const uint32_t *>(&r);
}

// 16 biased codes of one row (BITS / 2 words) to 8 words of value pairs in column order.  All differences are exact.
template <typename T, int BITS>
__device__ __forceinline__ void expand16(const uint32_t *w, uint32_t (&v)[8])
{
    using C = CodeConst<T>;
    if constexpr (BITS == 8) {
#pragma unroll
        for (int i = 0; i < 8; ++i) {
            const uint32_t c = w[i >> 1] >> (8 * (i & 1));
            if constexpr (C::kMid8 != 0) {
                v[i] = sub2<T>((c & 0x00FF00FFu) | C::kMagic, C::kMid8);
            } else {
                // bf16 holds seven bits beside the leading one: the low seven from 128 + v, the top bit in what is
                // subtracted (128 where it is set, 256 where it is not)
                v[i] = sub2<T>((c & 0x007F007Fu) | C::kMagic, (c & 0x00800080u) ^ 0x43804380u);
            }
        }
    } else if constexpr (BITS == 4) {
#pragma unroll
        for (int i = 0; i < 8; ++i) v[i] = sub2<T>(((w[i >> 2] >> (4 * (i & 3))) & 0x000F000Fu) | C::kMagic, C::kMid4);
    } else {
#pragma unroll
        for (int i = 0; i < 8; ++i) v[i] = sub2<T>(((w[0] >> (2 * i)) & 0x00030003u) | C::kMagic, C::kMid2);
    }
}

// ---------------------------------------------------------------- epilogue

// 2^v and 1 / v on the special-function unit.
__device__ __forceinline__ float fast_exp2(float v)
{
    float e;
    asm("ex2.approx.ftz.f32 %0, %1;" : "=f"(e) : "f"(v));
    return e;
}
__device__ __forceinline__ float fast_rcp(float v)
{
    float r;
    asm("rcp.approx.ftz.f32 %0, %1;" : "=f"(r) : "f"(v));
    return r;
}

// v / (1 + 2^exponent).  Rounding the exponent leaves a relative error of about |exponent| 2^-24 in the power, far under
// the 2^-11 of a 16-bit output.
__device__ __forceinline__ float gated_by_sigmoid(float v, float exponent) { return v * fast_rcp(1.f + fast_exp2(exponent)); }

__device__ __forceinline__ float silu(float v) { return gated_by_sigmoid(v, -1.4426950408889634f * v); }

// v Phi(v) = max(v, 0) - |v| erfc(|v| / sqrt 2) / 2, erfc by formula 7.1.26 of Abramowitz and Stegun (error below 1.5e-7):
// no cancellation for negative v, and a third of the instructions of the erf that is accurate to the last bit.
__device__ __forceinline__ float gelu(float v)
{
    const float a = fabsf(v), t = fast_rcp(fmaf(0.3275911f * 0.70710678118654752f, a, 1.f));
    float p = fmaf(1.061405429f, t, -1.453152027f);
    p = fmaf(p, t, 1.421413741f);
    p = fmaf(p, t, -0.284496736f);
    p = fmaf(p, t, 0.254829592f) * t;
    const float e = fast_exp2(-0.72134752044448170f * v * v);  // exp(-v^2 / 2)
    const float h = 0.5f * a * p * e;
    return (v > 0.f ? v : v == v ? 0.f : v) - (e > 0.f ? h : 0.f);  // e is 0 for an infinite v
}

// 0.5 v (1 + tanh(u)) = v / (1 + exp(-2 u)), u = sqrt(2 / pi) (v + 0.044715 v^3)
__device__ __forceinline__ float gelu_tanh(float v)
{
    return gated_by_sigmoid(v, -2.f * 1.4426950408889634f * 0.79788456080286536f * v * fmaf(0.044715f * v, v, 1.f));
}

__device__ __forceinline__ float activate(float v, int act)
{
    switch (act) {
        case QNN_ACT_RELU: return v > 0.f ? v : v == v ? 0.f : v;
        case QNN_ACT_SILU: return silu(v);
        case QNN_ACT_GELU: return gelu(v);
        case QNN_ACT_GELU_TANH: return gelu_tanh(v);
        default: return v;
    }
}

// One output element: product row value(s) already scaled and biased.
template <typename T>
__device__ __forceinline__ void finish(const MatmulArgs &a, int64_t row, int64_t col, float v)
{
    if (a.residual) v += to_f32<T>(static_cast<const T *>(a.residual)[row * a.ldres + col]);
    if (a.out_f32)
        static_cast<float *>(a.y)[row * a.ldy + col] = v;
    else
        static_cast<T *>(a.y)[row * a.ldy + col] = from_f32<T>(v);
}

// tab[e] = tiles of `tile` places before expert e, tab[experts] = all of them.  A whole warp calls it.
__device__ __forceinline__ void expert_tiles(const int32_t *offsets, int experts, int tile, int *tab)
{
    const int lane = threadIdx.x & 31;
    int before = 0;
    for (int base = 0; base < experts; base += 32) {
        const int e = base + lane;
        const int n = e < experts ? (offsets[e + 1] - offsets[e] + tile - 1) / tile : 0;
        int inc = n;
#pragma unroll
        for (int o = 1; o < 32; o <<= 1) {
            const int v = __shfl_up_sync(0xffffffffu, inc, o);
            if (lane >= o) inc += v;
        }
        if (e < experts) tab[e] = before + inc - n;
        before += __shfl_sync(0xffffffffu, inc, 31);
    }
    if (lane == 0) tab[experts] = before;
}

// The expert of tile `u`: the last one whose first tile is at most u.
__device__ __forceinline__ int find_expert(const int *tab, int experts, int u)
{
    int lo = 0, hi = experts;
    while (hi - lo > 1) {
        const int mid = (lo + hi) >> 1;
        if (tab[mid] <= u) lo = mid;
        else hi = mid;
    }
    return lo;
}

}  // namespace qnn
