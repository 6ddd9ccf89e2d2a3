// The weight image of the matrix products (qnn_matmul_prepare) and the weighted sum over a token's experts that ends
// qnn_experts_combine.  The preparation is bound by its instructions, not by its bytes: a thread gathers the codes of a
// 16-byte vector one by one (8192 x 8192: 79 us with 16-bit weights, 70 INT-8, 66 INT-4 and INT-2, where the bytes of INT-4
// take 10).  It runs once, when a layer is set up.  The sum is bound by memory: 4099 x 4 rows of 2048 take 25 us.
#include "matmul.cuh"

namespace qnn {
namespace {

struct PrepArgs {
    const void *w;
    const float *scale, *bias;
    uint8_t *image;
    float2 *params;
    int experts, m, k, bits, gated, rows_src;
    MatmulImage g;
};

// Row of the caller's matrix behind an image row, or -1 for padding.
__device__ __forceinline__ int source_row(const PrepArgs &a, int row)
{
    if (!a.gated) return row < a.m ? row : -1;
    const int ch = (row >> 4) * 8 + (row & 7);
    if (ch >= a.m) return -1;
    return row & 8 ? a.m + ch : ch;
}

// Biased code of column k of a packed source row (padding: the code of zero).
template <int BITS>
__device__ __forceinline__ uint32_t code_at(const uint8_t *row, int k, int kmax)
{
    constexpr uint32_t kMask = (1u << BITS) - 1u, kMid = 1u << (BITS - 1);
    if (!row || k >= kmax) return kMid;
    constexpr int kPer = 8 / BITS;
    return ((row[k / kPer] >> (BITS * (k % kPer))) & kMask) ^ kMid;
}

// One 16-byte vector of the image a thread.
template <int BITS>
__global__ void matmul_prep_kernel(const PrepArgs a)
{
    constexpr int kVecs = 32 * 64 * BITS / 8 / 16;
    const int64_t total = static_cast<int64_t>(a.experts) * a.g.mb * a.g.kb * kVecs;
    for (int64_t i = static_cast<int64_t>(blockIdx.x) * blockDim.x + threadIdx.x; i < total;
         i += static_cast<int64_t>(gridDim.x) * blockDim.x) {
        const int v = static_cast<int>(i % kVecs);
        const int64_t block = i / kVecs;
        const int kb = static_cast<int>(block % a.g.kb);
        const int mb = static_cast<int>(block / a.g.kb % a.g.mb);
        const int64_t e = block / a.g.kb / a.g.mb;
        uint32_t out[4];
        if constexpr (BITS == 16) {
            const int r = v >> 3, c = (v & 7) ^ (r & 7);
            const int src = source_row(a, mb * 32 + r);
            const uint16_t *row = static_cast<const uint16_t *>(a.w) + (e * a.rows_src + (src < 0 ? 0 : src)) * a.k;
            uint16_t h[8];
#pragma unroll
            for (int j = 0; j < 8; ++j) {
                const int k = kb * 64 + c * 8 + j;
                h[j] = src >= 0 && k < a.k ? row[k] : 0;
            }
#pragma unroll
            for (int j = 0; j < 4; ++j) out[j] = h[2 * j] | static_cast<uint32_t>(h[2 * j + 1]) << 16;
        } else {
            constexpr int kRuns = 8 / BITS;  // runs of 16 codes in the vector
            constexpr int kWords = BITS / 2; // words of a run
#pragma unroll
            for (int s = 0; s < kRuns; ++s) {
                // run s of vector v: half-row index h (8 rows each, 4 of them) and the lane it belongs to
                const int h = BITS == 8 ? v >> 5 : BITS == 4 ? (v >> 5) * 2 + s : s;
                const int lane = v & 31;
                const int src = source_row(a, mb * 32 + h * 8 + (lane >> 2));
                const int k0 = kb * 64 + (lane & 3) * 16;
                const uint8_t *row = src < 0 ? nullptr
                                             : static_cast<const uint8_t *>(a.w) +
                                                   (e * a.rows_src + src) * (static_cast<int64_t>(a.k) * BITS / 8);
                uint32_t word[kWords];
#pragma unroll
                for (int q = 0; q < kWords; ++q) word[q] = 0;
#pragma unroll
                for (int p = 0; p < 8; ++p) {  // column pair p of the run
                    constexpr int kPairs = 16 / BITS;  // pairs a word
                    const int sh = BITS * (p % kPairs);
                    word[p / kPairs] |= code_at<BITS>(row, k0 + 2 * p, a.k) << sh;
                    word[p / kPairs] |= code_at<BITS>(row, k0 + 2 * p + 1, a.k) << (sh + 16);
                }
#pragma unroll
                for (int q = 0; q < kWords; ++q) out[s * kWords + q] = word[q];
            }
        }
        *reinterpret_cast<uint4 *>(a.image + i * 16) = make_uint4(out[0], out[1], out[2], out[3]);
    }
    const int64_t prows = static_cast<int64_t>(a.experts) * a.g.rows;
    for (int64_t i = static_cast<int64_t>(blockIdx.x) * blockDim.x + threadIdx.x; i < prows;
         i += static_cast<int64_t>(gridDim.x) * blockDim.x) {
        const int64_t e = i / a.g.rows;
        const int src = source_row(a, static_cast<int>(i % a.g.rows));
        float2 p = make_float2(0.f, 0.f);
        if (src >= 0) {
            p.x = a.scale ? a.scale[e * a.rows_src + src] : 1.f;
            p.y = a.bias ? a.bias[e * a.rows_src + src] : 0.f;
        }
        a.params[i] = p;
    }
}

// y[t] = residual[t] + sum over the token's experts of weight * z[place], in the order of the choices.
struct CombineArgs {
    const float *z, *weights;
    const int32_t *position;
    const void *residual;
    void *y;
    int64_t ldz, ldres, ldy, tokens;
    int m, top, vec;  // vec: four neighbours of y and the residual at once
};

template <typename T>
__global__ void combine_kernel(const CombineArgs a)
{
    const int64_t t = blockIdx.x;
    pdl_begin();
    for (int c = (blockIdx.y * blockDim.x + threadIdx.x) * 4; c < a.m; c += gridDim.y * blockDim.x * 4) {
        float4 s = make_float4(0.f, 0.f, 0.f, 0.f);
        for (int j0 = 0; j0 < a.top; j0 += 4) {  // four rows in flight
            float4 v[4];
            float w[4];
            int p[4];
#pragma unroll
            for (int i = 0; i < 4; ++i) {
                p[i] = j0 + i < a.top ? a.position[t * a.top + j0 + i] : -1;
                w[i] = j0 + i < a.top ? a.weights[t * a.top + j0 + i] : 0.f;
            }
#pragma unroll
            for (int i = 0; i < 4; ++i) {
                v[i] = make_float4(0.f, 0.f, 0.f, 0.f);
                if (p[i] >= 0)
                    v[i] = __ldcs(reinterpret_cast<const float4 *>(a.z + p[i] * a.ldz + c));
                else
                    w[i] = 0.f;  // whatever weight a left-out choice has
            }
#pragma unroll
            for (int i = 0; i < 4; ++i) {
                s.x = fmaf(w[i], v[i].x, s.x);
                s.y = fmaf(w[i], v[i].y, s.y);
                s.z = fmaf(w[i], v[i].z, s.z);
                s.w = fmaf(w[i], v[i].w, s.w);
            }
        }
        if (c + 4 <= a.m && a.vec) {
            if (a.residual) {
                const uint2 r = *reinterpret_cast<const uint2 *>(static_cast<const T *>(a.residual) + t * a.ldres + c);
                const float2 lo = unpack2<T>(r.x), hi = unpack2<T>(r.y);
                s.x += lo.x; s.y += lo.y; s.z += hi.x; s.w += hi.y;
            }
            *reinterpret_cast<uint2 *>(static_cast<T *>(a.y) + t * a.ldy + c) = make_uint2(pack2<T>(s.x, s.y), pack2<T>(s.z, s.w));
            continue;
        }
        const float q[4] = {s.x, s.y, s.z, s.w};
#pragma unroll
        for (int j = 0; j < 4; ++j)
            if (c + j < a.m) {
                float v = q[j];
                if (a.residual) v += to_f32<T>(static_cast<const T *>(a.residual)[t * a.ldres + c + j]);
                static_cast<T *>(a.y)[t * a.ldy + c + j] = from_f32<T>(v);
            }
    }
}

// Row i of dst: row i of src, or row order[i] / top (no row where order[i] is negative).  A warp a row, eight 16-byte
// loads of a lane in flight; VEC: rows are 16-byte aligned and whole vectors.
constexpr int kTakeWarps = 8;

template <bool VEC>
__global__ void __launch_bounds__(kTakeWarps * 32) take_rows_kernel(const uint16_t *src, int64_t lds, const int32_t *order, int top,
                                                                    uint16_t *dst, int64_t ldd, int64_t rows, int cols)
{
    pdl_begin();
    const int lane = threadIdx.x & 31;
    const int64_t row = static_cast<int64_t>(blockIdx.x) * kTakeWarps + (threadIdx.x >> 5);
    if (row >= rows) return;
    int64_t from = row;
    if (order) {
        const int slot = order[row];
        if (slot < 0) return;
        from = slot / top;
    }
    const uint16_t *p = src + from * lds;
    uint16_t *q = dst + row * ldd;
    if constexpr (VEC) {
        const int vecs = cols / 8;
        for (int c = lane; c < vecs; c += 256) {
            uint4 v[8];
#pragma unroll
            for (int i = 0; i < 8; ++i)
                if (c + i * 32 < vecs) v[i] = reinterpret_cast<const uint4 *>(p)[c + i * 32];
#pragma unroll
            for (int i = 0; i < 8; ++i)
                if (c + i * 32 < vecs) reinterpret_cast<uint4 *>(q)[c + i * 32] = v[i];
        }
    } else {
        for (int c = lane; c < cols; c += 256) {
            uint16_t v[8];
#pragma unroll
            for (int i = 0; i < 8; ++i)
                if (c + i * 32 < cols) v[i] = p[c + i * 32];
#pragma unroll
            for (int i = 0; i < 8; ++i)
                if (c + i * 32 < cols) q[c + i * 32] = v[i];
        }
    }
}

}  // namespace

cudaError_t launch_take_rows(const void *src, int64_t lds, const int32_t *order, int top, void *dst, int64_t ldd, int64_t rows,
                             int cols, cudaStream_t st)
{
    if (rows == 0) return cudaSuccess;
    const bool vec = reinterpret_cast<uintptr_t>(src) % 16 == 0 && lds % 8 == 0 && cols % 8 == 0;
    const unsigned grid = static_cast<unsigned>((rows + kTakeWarps - 1) / kTakeWarps);
    return vec ? launch_pdl(take_rows_kernel<true>, dim3(grid), kTakeWarps * 32, 0, st, 1, static_cast<const uint16_t *>(src), lds, order, top,
                            static_cast<uint16_t *>(dst), ldd, rows, cols)
               : launch_pdl(take_rows_kernel<false>, dim3(grid), kTakeWarps * 32, 0, st, 1, static_cast<const uint16_t *>(src), lds, order, top,
                            static_cast<uint16_t *>(dst), ldd, rows, cols);
}

cudaError_t launch_matmul_prep(const qnn_matmul_desc &d, const void *w, const float *scale, const float *bias,
                               void *image, cudaStream_t st)
{
    PrepArgs a;
    a.g = matmul_image(d.experts, d.m, d.k, d.bits, d.gated);
    a.w = w; a.scale = scale; a.bias = bias;
    a.image = static_cast<uint8_t *>(image);
    a.params = reinterpret_cast<float2 *>(a.image + a.g.param_off);
    a.experts = d.experts; a.m = d.m; a.k = d.k; a.bits = d.bits; a.gated = d.gated;
    a.rows_src = d.gated ? 2 * d.m : d.m;
    const size_t vecs = a.g.param_off / 16;
    const unsigned grid = static_cast<unsigned>(vecs / 256 + 1 < 65536 ? vecs / 256 + 1 : 65536);
    if (d.bits == 16) matmul_prep_kernel<16><<<grid, 256, 0, st>>>(a);
    else if (d.bits == 8) matmul_prep_kernel<8><<<grid, 256, 0, st>>>(a);
    else if (d.bits == 4) matmul_prep_kernel<4><<<grid, 256, 0, st>>>(a);
    else matmul_prep_kernel<2><<<grid, 256, 0, st>>>(a);
    return cudaGetLastError();
}

cudaError_t launch_combine(int dtype, const float *z, int64_t ldz, const float *weights, const int32_t *position,
                           int64_t tokens, int top, int m, const void *residual, int64_t ldres, void *y, int64_t ldy,
                           cudaStream_t st)
{
    if (tokens == 0) return cudaSuccess;
    const int vec = reinterpret_cast<uintptr_t>(y) % 8 == 0 && ldy % 4 == 0 &&
                    (!residual || (reinterpret_cast<uintptr_t>(residual) % 8 == 0 && ldres % 4 == 0));
    const CombineArgs a = {z, weights, position, residual, y, ldz, ldres, ldy, tokens, m, top, vec};
    const dim3 grid(static_cast<unsigned>(tokens), (m + 1023) / 1024);
    return dtype == QNN_F16 ? launch_pdl(combine_kernel<__half>, grid, 256, 0, st, 1, a)
                            : launch_pdl(combine_kernel<__nv_bfloat16>, grid, 256, 0, st, 1, a);
}

}  // namespace qnn
