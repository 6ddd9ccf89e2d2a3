// Matrix product for few rows of x: the weights are streamed once, straight into the fragments of mma.sync.
//
// One block owns 32 image rows and a tile of NT rows of x (8, 16 or 32); its warps split K, each taking whole 64-column
// blocks, and their partial sums are added in shared memory in a fixed order.  Nothing is staged: a lane's vector of
// packed codes is its A fragment, and x has so few rows that its fragments come from L2.  The product is bound by the
// weight bytes (or, for the narrowest codes, by expanding them), not by the tensor cores.
#include "matmul.cuh"

namespace qnn {
namespace {

constexpr int kStreamWarps = 8;

template <typename T>
__device__ __forceinline__ void mma16816(float (&c)[4], const uint32_t (&a)[4], uint32_t b0, uint32_t b1);
template <>
__device__ __forceinline__ void mma16816<__half>(float (&c)[4], const uint32_t (&a)[4], uint32_t b0, uint32_t b1)
{
    asm volatile("mma.sync.aligned.m16n8k16.row.col.f32.f16.f16.f32 {%0,%1,%2,%3}, {%4,%5,%6,%7}, {%8,%9}, {%0,%1,%2,%3};"
                 : "+f"(c[0]), "+f"(c[1]), "+f"(c[2]), "+f"(c[3])
                 : "r"(a[0]), "r"(a[1]), "r"(a[2]), "r"(a[3]), "r"(b0), "r"(b1));
}
template <>
__device__ __forceinline__ void mma16816<__nv_bfloat16>(float (&c)[4], const uint32_t (&a)[4], uint32_t b0, uint32_t b1)
{
    asm volatile("mma.sync.aligned.m16n8k16.row.col.f32.bf16.bf16.f32 {%0,%1,%2,%3}, {%4,%5,%6,%7}, {%8,%9}, {%0,%1,%2,%3};"
                 : "+f"(c[0]), "+f"(c[1]), "+f"(c[2]), "+f"(c[3])
                 : "r"(a[0]), "r"(a[1]), "r"(a[2]), "r"(a[3]), "r"(b0), "r"(b1));
}

// The raw words of one 32 x 64 block that a lane needs.
template <int BITS>
struct Lane {
    static constexpr int kVecs = BITS / 2;  // 16-byte vectors a lane: 8 for 16 bits, 4, 2, 1
    uint4 q[kVecs];
    __device__ __forceinline__ void load(const uint8_t *block, int lane)
    {
        const uint4 *p = reinterpret_cast<const uint4 *>(block);
#pragma unroll
        for (int i = 0; i < kVecs; ++i) {
            if constexpr (BITS == 16) {  // half-row i >> 1, chunk 2 t + (i & 1) of row g
                const int g = lane >> 2, c = 2 * (lane & 3) + (i & 1);
                q[i] = __ldg(p + ((i >> 1) * 8 + g) * 8 + (c ^ g));
            } else {
                q[i] = __ldg(p + i * 32 + lane);
            }
        }
    }
    // Value pairs of half-row h (rows 8 h + g), columns 16 t .. 16 t + 15.
    template <typename T>
    __device__ __forceinline__ void row(int h, uint32_t (&v)[8]) const
    {
        const uint32_t *w = reinterpret_cast<const uint32_t *>(q);
        if constexpr (BITS == 16) {
#pragma unroll
            for (int i = 0; i < 8; ++i) v[i] = w[h * 8 + i];
        } else {
            expand16<T, BITS>(w + h * (BITS / 2), v);
        }
    }
};

// 16 values of one row of x as 8 words, zeros past the row's end.
template <typename T>
__device__ __forceinline__ void load_x(const T *row, int k0, int k, int vec, uint32_t (&w)[8])
{
    if (row && vec && k0 + 16 <= k) {
        const uint4 a = *reinterpret_cast<const uint4 *>(row + k0), b = *reinterpret_cast<const uint4 *>(row + k0 + 8);
        w[0] = a.x; w[1] = a.y; w[2] = a.z; w[3] = a.w;
        w[4] = b.x; w[5] = b.y; w[6] = b.z; w[7] = b.w;
    } else {
        const uint16_t *p = reinterpret_cast<const uint16_t *>(row);
#pragma unroll
        for (int i = 0; i < 8; ++i) {
            const uint32_t lo = row && k0 + 2 * i < k ? p[k0 + 2 * i] : 0;
            const uint32_t hi = row && k0 + 2 * i + 1 < k ? p[k0 + 2 * i + 1] : 0;
            w[i] = lo | hi << 16;
        }
    }
}

template <typename T, int BITS, int NT>
__global__ void __launch_bounds__(kStreamWarps * 32) matmul_stream_kernel(const MatmulArgs a)
{
    __shared__ float part[kStreamWarps][32][NT + 1];
    constexpr int kN = NT / 8;
    const int lane = threadIdx.x & 31, warp = threadIdx.x >> 5, g = lane >> 2, t = lane & 3;
    const int mb = blockIdx.x;
    int expert = 0, count;
    int64_t first;
    if (a.offsets) {
        const ExpertTile tile = expert_tile(a.offsets, a.experts, NT, blockIdx.y);
        if (a.zero_tail) {  // rows that no expert fills
            const int chans = a.gated ? 16 : 32, c = mb * chans + threadIdx.x;
            if (threadIdx.x < chans && c < a.m)
                for (int64_t r = a.offsets[a.experts] + blockIdx.y; r < a.rows; r += gridDim.y)
                    static_cast<T *>(a.y)[r * a.ldy + c] = from_f32<T>(0.f);
        }
        if (tile.expert < 0) return;
        expert = tile.expert;
        first = tile.first;
        count = tile.count;
    } else {
        first = static_cast<int64_t>(blockIdx.y) * NT;
        count = static_cast<int>(a.rows - first < NT ? a.rows - first : NT);
    }
    const T *xrow[kN];
#pragma unroll
    for (int n = 0; n < kN; ++n) {
        const int r = n * 8 + g;
        xrow[n] = nullptr;
        if (r < count) {
            int64_t row = first + r;
            if (a.gather) row = a.order[row] / a.top;
            xrow[n] = static_cast<const T *>(a.x) + row * a.ldx;
        }
    }
    constexpr uint32_t kBlock = 32 * 64 * BITS / 8;
    const uint8_t *blocks = a.image + (static_cast<size_t>(expert) * a.mb + mb) * a.kb * kBlock;

    float acc[2][kN][4] = {};
    Lane<BITS> w;
    if (warp < a.kb) w.load(blocks + static_cast<size_t>(warp) * kBlock, lane);
    for (int kb = warp; kb < a.kb; kb += kStreamWarps) {
        uint32_t x[kN][8];
#pragma unroll
        for (int n = 0; n < kN; ++n) load_x(xrow[n], kb * 64 + t * 16, a.k, a.x_vec, x[n]);
        const Lane<BITS> cur = w;
        if (kb + kStreamWarps < a.kb) w.load(blocks + static_cast<size_t>(kb + kStreamWarps) * kBlock, lane);
#pragma unroll
        for (int j = 0; j < 2; ++j) {
            uint32_t lo[8], hi[8];
            cur.template row<T>(2 * j, lo);
            cur.template row<T>(2 * j + 1, hi);
#pragma unroll
            for (int s = 0; s < 4; ++s) {
                const uint32_t f[4] = {lo[2 * s], hi[2 * s], lo[2 * s + 1], hi[2 * s + 1]};
#pragma unroll
                for (int n = 0; n < kN; ++n) mma16816<T>(acc[j][n], f, x[n][2 * s], x[n][2 * s + 1]);
            }
        }
    }
#pragma unroll
    for (int j = 0; j < 2; ++j)
#pragma unroll
        for (int n = 0; n < kN; ++n)
#pragma unroll
            for (int i = 0; i < 4; ++i) part[warp][j * 16 + g + (i >> 1) * 8][n * 8 + 2 * t + (i & 1)] = acc[j][n][i];
    __syncthreads();

    const float2 *params = a.params + static_cast<int64_t>(expert) * a.mb * 32 + mb * 32;
    const int chans = a.gated ? 16 : 32;
    for (int i = threadIdx.x; i < chans * count; i += kStreamWarps * 32) {
        const int c = i % chans, n = i / chans;
        const int64_t col = static_cast<int64_t>(mb) * chans + c;
        if (col >= a.m) continue;
        const int r = a.gated ? (c >> 3) * 16 + (c & 7) : c;
        float s = 0.f, u = 0.f;
#pragma unroll
        for (int p = 0; p < kStreamWarps; ++p) s += part[p][r][n];
        float2 q = params[r];
        s = fmaf(s, q.x, q.y);
        s = activate(s, a.act);
        if (a.gated) {
#pragma unroll
            for (int p = 0; p < kStreamWarps; ++p) u += part[p][r + 8][n];
            q = params[r + 8];
            s *= fmaf(u, q.x, q.y);
        }
        finish<T>(a, first + n, col, s);
    }
}

template <typename T, int BITS>
cudaError_t launch_nt(const MatmulArgs &a, int nt, unsigned tiles, cudaStream_t st)
{
    const dim3 grid(a.mb, tiles);
    if (nt == 8) matmul_stream_kernel<T, BITS, 8><<<grid, kStreamWarps * 32, 0, st>>>(a);
    else if (nt == 16) matmul_stream_kernel<T, BITS, 16><<<grid, kStreamWarps * 32, 0, st>>>(a);
    else matmul_stream_kernel<T, BITS, 32><<<grid, kStreamWarps * 32, 0, st>>>(a);
    return cudaGetLastError();
}

template <typename T>
cudaError_t launch_bits(const MatmulArgs &a, int bits, int nt, unsigned tiles, cudaStream_t st)
{
    if (bits == 16) return launch_nt<T, 16>(a, nt, tiles, st);
    if (bits == 8) return launch_nt<T, 8>(a, nt, tiles, st);
    if (bits == 4) return launch_nt<T, 4>(a, nt, tiles, st);
    return launch_nt<T, 2>(a, nt, tiles, st);
}

}  // namespace

cudaError_t launch_matmul_stream(const MatmulArgs &a, int dtype, int bits, cudaStream_t st)
{
    // rows of x to a tile: all of them where they fit, for experts about what one expert gets
    const int64_t want = a.offsets ? (a.rows + a.experts - 1) / a.experts : a.rows;
    const int nt = want <= 8 ? 8 : want <= 16 ? 16 : 32;
    int64_t tiles = (a.rows + nt - 1) / nt;
    if (a.offsets) tiles += a.experts < a.rows ? a.experts : a.rows;  // each expert may end in a partial tile
    if (tiles == 0) return cudaSuccess;
    if (tiles > 65535) return cudaErrorInvalidConfiguration;
    return dtype == QNN_F16 ? launch_bits<__half>(a, bits, nt, static_cast<unsigned>(tiles), st)
                            : launch_bits<__nv_bfloat16>(a, bits, nt, static_cast<unsigned>(tiles), st);
}

}  // namespace qnn
