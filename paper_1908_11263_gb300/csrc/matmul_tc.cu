// Matrix product on the 5th-generation tensor cores, for more rows of x than the streaming kernel takes.
//
// A pair of CTAs (cluster of two, cta_group::2) owns a tile of 256 image rows x `nt` rows of x: the weights are the
// A operand (128 rows in each CTA's shared memory, M = 256), x is the B operand (half of the rows in each CTA), the
// 32-bit accumulators sit in tensor memory, two tiles deep, so one tile's epilogue runs under the next tile's MMAs.
// With the weights on the M side a thread of the epilogue owns one output channel: its scale and bias are two
// registers, and the number of rows of x can be any multiple of 16 up to 256.
//
// Warps: 0 loads (x by tiled TMA, or one four-row gather per lane where an expert picks its tokens; weight blocks by
// bulk copies), 1 issues the MMAs (first CTA of the pair), 2 hands complete stages of 16-bit weights on, 3 owns the
// tensor memory, 4-11 run the epilogue, 12-19 expand packed codes into the A operand (packed weights only).
// Every wait is bounded (mbar_wait_warp); a wait that gives up ends its role, and the kernel, with the status word set.
#include <cuda.h>

#include <cmath>
#include <mutex>
#include <type_traits>

#include "matmul.cuh"

namespace qnn {
namespace {

constexpr int kABytes = 128 * 128;  // A operand of one stage: 128 rows of 64 16-bit values
constexpr int kMaxStages = 8;
constexpr uint32_t kBarBytes = 8 * (3 * kMaxStages + 4) + 16;

struct TcShape {
    int nt, mt, stages;       // rows of x a tile, tiles along the image rows, pipeline stages
    uint32_t cols;            // tensor-memory columns (power of two)
    uint32_t off_x, off_raw, off_bar, off_tab, smem;
};

// ---------------------------------------------------------------- cluster and cta_group::2 forms

__device__ __forceinline__ uint32_t cluster_rank()
{
    uint32_t r;
    asm volatile("mov.u32 %0, %%cluster_ctarank;" : "=r"(r));
    return r;
}

__device__ __forceinline__ void cluster_sync()
{
    asm volatile("barrier.cluster.arrive.release.aligned;\n\tbarrier.cluster.wait.acquire.aligned;" ::: "memory");
}

// Arrives on the barrier at this address in the pair's first CTA.
__device__ __forceinline__ void mbar_arrive_leader(uint64_t *bar)
{
    asm volatile(
        "{\n\t.reg .b32 r;\n\t"
        "mapa.shared::cluster.u32 r, %0, 0;\n\t"
        "mbarrier.arrive.shared::cluster.b64 _, [r];\n\t}" ::"r"(smem_addr(bar))
        : "memory");
}

__device__ __forceinline__ void mma2_f16_warp(uint32_t d, uint64_t a, uint64_t b, uint32_t idesc, uint32_t accumulate)
{
    asm volatile(
        "{\n\t.reg .pred p, e;\n\t"
        "elect.sync _|e, 0xffffffff;\n\t"
        "setp.ne.b32 p, %4, 0;\n\t"
        "@e tcgen05.mma.cta_group::2.kind::f16 [%0], %1, %2, %3, p;\n\t}" ::"r"(d),
        "l"(a), "l"(b), "r"(idesc), "r"(accumulate)
        : "memory");
}

// Arrives on this barrier in both CTAs of the pair when the MMAs issued so far have completed.
__device__ __forceinline__ void mma2_commit_warp(uint64_t *bar)
{
    asm volatile(
        "{\n\t.reg .pred e;\n\t"
        "elect.sync _|e, 0xffffffff;\n\t"
        "@e tcgen05.commit.cta_group::2.mbarrier::arrive::one.shared::cluster.multicast::cluster.b64 [%0], %1;\n\t}" ::"r"(
            smem_addr(bar)),
        "h"(static_cast<uint16_t>(3))
        : "memory");
}

__device__ __forceinline__ void tma_tile(void *dst, const CUtensorMap *map, int x, int y, uint64_t *bar)
{
    asm volatile(
        "cp.async.bulk.tensor.2d.shared::cluster.global.tile.mbarrier::complete_tx::bytes [%0], [%1, {%2, %3}], [%4];" ::"r"(
            smem_addr(dst)),
        "l"(map), "r"(x), "r"(y), "r"(smem_addr(bar))
        : "memory");
}

// Four rows of the map (box one row high) to four consecutive rows of shared memory.
__device__ __forceinline__ void tma_gather4(void *dst, const CUtensorMap *map, int x, const int (&y)[4], uint64_t *bar)
{
    asm volatile(
        "cp.async.bulk.tensor.2d.shared::cluster.global.tile::gather4.mbarrier::complete_tx::bytes [%0], "
        "[%1, {%2, %3, %4, %5, %6}], [%7];" ::"r"(smem_addr(dst)),
        "l"(map), "r"(x), "r"(y[0]), "r"(y[1]), "r"(y[2]), "r"(y[3]), "r"(smem_addr(bar))
        : "memory");
}

// K-major operand in the 128-byte swizzle: rows of 128 bytes, groups of eight rows 1024 bytes apart.
__device__ __forceinline__ uint64_t desc_sw128(uint32_t saddr)
{
    return static_cast<uint64_t>((saddr >> 4) & 0x3FFFu) | static_cast<uint64_t>(1) << 16 |
           static_cast<uint64_t>(1024 >> 4) << 32 | static_cast<uint64_t>(1) << 46 | static_cast<uint64_t>(2) << 61;
}

// ---------------------------------------------------------------- epilogue

// Activation of an array, the choice outside the loop.
template <int N>
__device__ __forceinline__ void activate_all(float (&v)[N], int act)
{
    switch (act) {
        case QNN_ACT_RELU:
#pragma unroll
            for (int i = 0; i < N; ++i) v[i] = activate(v[i], QNN_ACT_RELU);
            break;
        case QNN_ACT_SILU:
#pragma unroll
            for (int i = 0; i < N; ++i) v[i] = activate(v[i], QNN_ACT_SILU);
            break;
        case QNN_ACT_GELU:
#pragma unroll
            for (int i = 0; i < N; ++i) v[i] = activate(v[i], QNN_ACT_GELU);
            break;
        case QNN_ACT_GELU_TANH:
#pragma unroll
            for (int i = 0; i < N; ++i) v[i] = activate(v[i], QNN_ACT_GELU_TANH);
            break;
        default: break;
    }
}

// N values of one channel to rows `step` elements apart, `n` of them at most.
template <typename T, int N>
__device__ __forceinline__ void store_rows(T *y, int64_t step, const float (&v)[N], int n)
{
    if (n >= N) {
#pragma unroll
        for (int i = 0; i < N; ++i) {
            *y = from_f32<T>(v[i]);
            y += step;
        }
    } else {
#pragma unroll
        for (int i = 0; i < N; ++i) {
            if (i < n) *y = from_f32<T>(v[i]);
            y += step;
        }
    }
}

// The residual of the same rows.
template <typename T, int N>
__device__ __forceinline__ void load_rows(const T *r, int64_t step, T (&v)[N], int n)
{
#pragma unroll
    for (int i = 0; i < N; ++i) {
        v[i] = i < n ? *r : from_f32<T>(0.f);
        r += step;
    }
}

// Sixteen rows of x (columns of the accumulator) from `row` on, `n` of them in use, of one image row.  Without a gate a
// lane finishes its own channel.  With one, a channel's gate and up rows are eight lanes apart: of each two rows of x the
// gate lane finishes the first and the up lane the second.
template <typename T, bool GATED>
__device__ __forceinline__ void finish16(const MatmulArgs &a, uint32_t src, float2 p, int64_t row, int n, int64_t ch,
                                         bool valid)
{
    constexpr int kN = GATED ? 8 : 16;
    const bool up = GATED && (threadIdx.x & 8);
    const int64_t rows = GATED ? 2 : 1;
    if (up) ++row;
    const int mine = !valid ? 0 : GATED ? (n + (up ? 0 : 1)) / 2 : n;  // rows that this lane finishes
    T res[kN];
    if (a.residual) load_rows(static_cast<const T *>(a.residual) + row * a.ldres + ch, rows * a.ldres, res, mine);
    uint32_t acc[16];
    __syncwarp();
    tmem_ld16(src, acc);
    tmem_wait_ld();
    float v[kN];
    if constexpr (GATED) {
        float u[kN];
#pragma unroll
        for (int i = 0; i < kN; ++i) {
            const float v0 = fmaf(__uint_as_float(acc[2 * i]), p.x, p.y), v1 = fmaf(__uint_as_float(acc[2 * i + 1]), p.x, p.y);
            const float other = __shfl_xor_sync(0xffffffffu, up ? v0 : v1, 8);
            v[i] = up ? other : v0;
            u[i] = up ? v1 : other;
        }
        activate_all(v, a.act);
#pragma unroll
        for (int i = 0; i < kN; ++i) v[i] *= u[i];
    } else {
#pragma unroll
        for (int i = 0; i < kN; ++i) v[i] = fmaf(__uint_as_float(acc[i]), p.x, p.y);
        activate_all(v, a.act);
    }
    if (a.residual)
#pragma unroll
        for (int i = 0; i < kN; ++i) v[i] += to_f32<T>(res[i]);
    if (a.out_f32)
        store_rows(static_cast<float *>(a.y) + row * a.ldy + ch, rows * a.ldy, v, mine);
    else
        store_rows(static_cast<T *>(a.y) + row * a.ldy + ch, rows * a.ldy, v, mine);
}

// ---------------------------------------------------------------- tiles

struct Tile {
    int expert, mtile, count;
    int64_t first;
};

// Tile `id`: tiles along the image rows first, then along the rows of x (of the experts one after another; `tab` holds
// the tiles before each expert).
__device__ __forceinline__ Tile tile_at(const MatmulArgs &a, const TcShape &s, const int *tab, int id)
{
    Tile t;
    t.mtile = id % s.mt;
    const int u = id / s.mt;
    t.expert = 0;
    if (a.offsets) {
        const int lo = find_expert(tab, a.experts, u);
        t.expert = lo;
        const int begin = a.offsets[lo], end = a.offsets[lo + 1];
        t.first = begin + static_cast<int64_t>(u - tab[lo]) * s.nt;
        t.count = min(s.nt, static_cast<int>(end - t.first));
    } else {
        t.first = static_cast<int64_t>(u) * s.nt;
        t.count = static_cast<int>(a.rows - t.first < s.nt ? a.rows - t.first : s.nt);
    }
    return t;
}

template <typename T, int BITS>
__global__ void __cluster_dims__(2, 1, 1) __launch_bounds__(BITS == 16 ? 384 : 640, 1)
    matmul_tc_kernel(const __grid_constant__ CUtensorMap xmap, const MatmulArgs a, const TcShape s, int *status)
{
    extern __shared__ __align__(1024) uint8_t smem[];
    constexpr bool kPacked = BITS != 16;
    constexpr uint32_t kBlock = 32 * 64 * BITS / 8;
    uint8_t *sm_a = smem, *sm_x = smem + s.off_x, *sm_raw = smem + s.off_raw;
    uint64_t *full = reinterpret_cast<uint64_t *>(smem + s.off_bar);
    uint64_t *ready = full + kMaxStages, *empty = ready + kMaxStages;
    uint64_t *acc_full = empty + kMaxStages, *acc_empty = acc_full + 2;
    uint32_t *slot = reinterpret_cast<uint32_t *>(acc_empty + 2);
    int *tab = reinterpret_cast<int *>(smem + s.off_tab);
    const int warp = threadIdx.x >> 5, lane = threadIdx.x & 31;
    const int rank = static_cast<int>(cluster_rank());
    const int pair = blockIdx.x >> 1, pairs = gridDim.x >> 1;
    const uint32_t x_bytes = s.nt / 2 * 128;

    if (threadIdx.x == 0) {
        for (int i = 0; i < s.stages; ++i) {
            mbar_init(full + i, 1);
            mbar_init(ready + i, kPacked ? 16 : 2);
            mbar_init(empty + i, 1);
        }
        for (int i = 0; i < 2; ++i) {
            mbar_init(acc_full + i, 1);
            mbar_init(acc_empty + i, 16);
        }
        fence_mbar_init();
    }
    pdl_begin();
    if (warp == 3) {
        asm volatile("tcgen05.alloc.cta_group::2.sync.aligned.shared::cta.b32 [%0], %1;" ::"r"(smem_addr(slot)), "r"(s.cols)
                     : "memory");
        asm volatile("tcgen05.relinquish_alloc_permit.cta_group::2.sync.aligned;" ::: "memory");
        if (a.offsets) expert_tiles(a.offsets, a.experts, s.nt, tab);
        tc_fence_before();
    }
    __syncthreads();
    cluster_sync();
    tc_fence_after();
    const uint32_t tmem = *slot;
    const int tiles = (a.offsets ? tab[a.experts] : static_cast<int>((a.rows + s.nt - 1) / s.nt)) * s.mt;

    if (a.zero_tail)  // rows that no expert fills
        for (int64_t r = a.offsets[a.experts] + blockIdx.x; r < a.rows; r += gridDim.x)
            for (int c = threadIdx.x; c < a.m; c += blockDim.x) static_cast<T *>(a.y)[r * a.ldy + c] = from_f32<T>(0.f);

    bool ok = true;
    if (warp == 0) {
        // ------------------------------------------------ loads
        int st = 0, uses = 0;
        uint32_t phase = 0;
        for (int id = pair; id < tiles && ok; id += pairs) {
            const Tile t = tile_at(a, s, tab, id);
            int rows[4] = {0, 0, 0, 0};
            const bool gathers = a.gather && lane < s.nt / 8;
            if (gathers)
#pragma unroll
                for (int i = 0; i < 4; ++i) {
                    const int r = rank * (s.nt / 2) + lane * 4 + i;
                    rows[i] = a.order[t.first + (r < t.count ? r : 0)] / a.top;  // rows past the count are not stored
                }
            const int mb = min((t.mtile * 2 + rank) * 4 + (lane & 3), a.mb - 1);  // rows past the image are not stored
            const uint8_t *src = a.image + (static_cast<size_t>(t.expert) * a.mb + mb) * a.kb * kBlock;
            for (int kb = 0; kb < a.kb; ++kb) {
                if (!mbar_wait_warp(empty + st, phase ^ 1, status)) {
                    ok = false;
                    break;
                }
                if (lane == 0) mbar_arrive_expect_tx(full + st, x_bytes + 4 * kBlock);
                __syncwarp();
                uint8_t *dst = kPacked ? sm_raw + st * 4 * kBlock : sm_a + st * kABytes;
                if (lane < 4) bulk_g2s(dst + lane * kBlock, src + static_cast<size_t>(kb) * kBlock, kBlock, full + st);
                if (gathers)
                    tma_gather4(sm_x + st * x_bytes + lane * 512, &xmap, kb * 64, rows, full + st);
                else if (!a.gather && lane == 4)
                    tma_tile(sm_x + st * x_bytes, &xmap, kb * 64, static_cast<int>(t.first) + rank * (s.nt / 2), full + st);
                __syncwarp();
                ++uses;
                if (++st == s.stages) {
                    st = 0;
                    phase ^= 1;
                }
            }
        }
        // copies still in flight land before the CTA may end
        for (int i = 0; i < min(uses, s.stages); ++i) {
            if (--st < 0) {
                st = s.stages - 1;
                phase ^= 1;
            }
            mbar_wait_warp(full + st, phase, status);
        }
    } else if (warp == 1 && rank == 0) {
        // ------------------------------------------------ MMAs
        constexpr uint32_t kFmt = std::is_same<T, __nv_bfloat16>::value ? 1u : 0u;
        const uint32_t idesc = (1u << 4) | (kFmt << 7) | (kFmt << 10) | (static_cast<uint32_t>(s.nt >> 3) << 17) | (16u << 24);
        int st = 0, it = 0;
        uint32_t phase = 0;
        for (int id = pair; id < tiles && ok; id += pairs, ++it) {
            const int buf = it & 1;
            if (!mbar_wait_warp(acc_empty + buf, ((it >> 1) & 1) ^ 1, status)) {
                ok = false;
                break;
            }
            tc_fence_after();
            const uint32_t d = tmem + buf * s.nt;
            for (int kb = 0; kb < a.kb; ++kb) {
                if (!mbar_wait_warp(ready + st, phase, status)) {
                    ok = false;
                    break;
                }
                tc_fence_after();
                const uint64_t da = desc_sw128(smem_addr(sm_a + st * kABytes));
                const uint64_t db = desc_sw128(smem_addr(sm_x + st * x_bytes));
#pragma unroll
                for (int k = 0; k < 4; ++k) mma2_f16_warp(d, da + 2 * k, db + 2 * k, idesc, kb | k);
                mma2_commit_warp(empty + st);
                if (++st == s.stages) {
                    st = 0;
                    phase ^= 1;
                }
            }
            if (ok) mma2_commit_warp(acc_full + buf);
        }
    } else if (warp == 2 && !kPacked) {
        // ------------------------------------------------ complete stages of 16-bit weights
        int st = 0;
        uint32_t phase = 0;
        for (int id = pair; id < tiles && ok; id += pairs)
            for (int kb = 0; kb < a.kb; ++kb) {
                if (!mbar_wait_warp(full + st, phase, status)) {
                    ok = false;
                    break;
                }
                if (lane == 0) mbar_arrive_leader(ready + st);
                __syncwarp();
                if (++st == s.stages) {
                    st = 0;
                    phase ^= 1;
                }
            }
    } else if (warp >= 4 && warp < 12) {
        // ------------------------------------------------ epilogue: two warps a quarter of the lanes
        const int quarter = warp & 3, half = (warp - 4) >> 2;
        int it = 0;
        for (int id = pair; id < tiles && ok; id += pairs, ++it) {
            const int buf = it & 1;
            const Tile t = tile_at(a, s, tab, id);
            const int row = t.mtile * 256 + rank * 128 + quarter * 32 + lane;  // image row
            const int ch = a.gated ? (row >> 4) * 8 + (row & 7) : row;
            const bool valid = ch < a.m;
            const float2 p = row < a.mb * 32 ? a.params[static_cast<int64_t>(t.expert) * a.mb * 32 + row] : make_float2(0.f, 0.f);
            if (!mbar_wait_warp(acc_full + buf, (it >> 1) & 1, status)) {
                ok = false;
                break;
            }
            tc_fence_after();
            const uint32_t src = tmem + buf * s.nt + (static_cast<uint32_t>(quarter * 32) << 16);
            for (int c = 16 * half; c < t.count; c += 32) {
                if (a.gated)
                    finish16<T, true>(a, src + c, p, t.first + c, t.count - c, ch, valid);
                else
                    finish16<T, false>(a, src + c, p, t.first + c, t.count - c, ch, valid);
            }
            __syncwarp();
            tc_fence_before();
            if (lane == 0) mbar_arrive_leader(acc_empty + buf);
            __syncwarp();
        }
    } else if (warp >= 12) {
        // ------------------------------------------------ packed codes to the A operand
        if constexpr (kPacked) {
            const int i = (warp - 12) >> 1, j = (warp - 12) & 1;  // 32-row block, its half
            const int g = lane >> 2, tt = lane & 3;
            int st = 0;
            uint32_t phase = 0;
            for (int id = pair; id < tiles && ok; id += pairs)
                for (int kb = 0; kb < a.kb; ++kb) {
                    if (!mbar_wait_warp(full + st, phase, status)) {
                        ok = false;
                        break;
                    }
                    const uint8_t *raw = sm_raw + st * 4 * kBlock + i * kBlock;
                    uint32_t w[BITS];  // two runs of 16 codes: rows g and g + 8 of the half
                    if constexpr (BITS == 8) {
#pragma unroll
                        for (int h = 0; h < 2; ++h)
                            *reinterpret_cast<uint4 *>(w + 4 * h) =
                                reinterpret_cast<const uint4 *>(raw)[(2 * j + h) * 32 + lane];
                    } else if constexpr (BITS == 4) {
                        *reinterpret_cast<uint4 *>(w) = reinterpret_cast<const uint4 *>(raw)[j * 32 + lane];
                    } else {
                        *reinterpret_cast<uint2 *>(w) = reinterpret_cast<const uint2 *>(raw)[lane * 2 + j];
                    }
#pragma unroll
                    for (int h = 0; h < 2; ++h) {
                        uint32_t v[8];
                        expand16<T, BITS>(w + h * (BITS / 2), v);
                        uint8_t *dst = sm_a + st * kABytes + (i * 32 + j * 16 + h * 8 + g) * 128;
                        *reinterpret_cast<uint4 *>(dst + ((2 * tt) ^ g) * 16) = make_uint4(v[0], v[1], v[2], v[3]);
                        *reinterpret_cast<uint4 *>(dst + ((2 * tt + 1) ^ g) * 16) = make_uint4(v[4], v[5], v[6], v[7]);
                    }
                    fence_proxy_async_smem();
                    __syncwarp();
                    if (lane == 0) mbar_arrive_leader(ready + st);
                    __syncwarp();
                    if (++st == s.stages) {
                        st = 0;
                        phase ^= 1;
                    }
                }
        }
    }
    __syncwarp();
    tc_fence_before();
    __syncthreads();
    cluster_sync();  // the pair's MMAs, copies and remote arrivals are done
    if (warp == 3) {
        tc_fence_after();
        asm volatile("tcgen05.dealloc.cta_group::2.sync.aligned.b32 %0, %1;" ::"r"(tmem), "r"(s.cols) : "memory");
    }
}

// ---------------------------------------------------------------- host

using EncodeTiled = CUresult (*)(CUtensorMap *, CUtensorMapDataType, cuuint32_t, void *, const cuuint64_t *, const cuuint64_t *,
                                 const cuuint32_t *, const cuuint32_t *, CUtensorMapInterleave, CUtensorMapSwizzle,
                                 CUtensorMapL2promotion, CUtensorMapFloatOOBfill);

EncodeTiled encode_tiled()
{
    static std::mutex mu;
    static EncodeTiled fn = nullptr;
    std::lock_guard<std::mutex> lock(mu);
    if (!fn) {
        void *p = nullptr;
        cudaDriverEntryPointQueryResult q;
        if (cudaGetDriverEntryPointByVersion("cuTensorMapEncodeTiled", &p, 12000, cudaEnableDefault, &q) == cudaSuccess &&
            q == cudaDriverEntryPointSuccess)
            fn = reinterpret_cast<EncodeTiled>(p);
    }
    return fn;
}

TcShape shape_of(const MatmulArgs &a, int bits, int nt)
{
    TcShape s;
    s.nt = nt;
    s.mt = (a.mb + 7) / 8;
    const uint32_t raw = bits == 16 ? 0 : 4 * (32 * 64 * bits / 8), x = nt / 2 * 128, stage = kABytes + x + raw;
    const uint32_t tab = (4 * (a.experts + 1) + 15) / 16 * 16;
    const uint32_t room = 227 * 1024 - kBarBytes - tab;
    s.stages = static_cast<int>(room / stage < kMaxStages ? room / stage : kMaxStages);
    s.off_x = s.stages * kABytes;
    s.off_raw = s.off_x + s.stages * x;
    s.off_bar = s.off_raw + s.stages * raw;
    s.off_tab = s.off_bar + kBarBytes;
    s.smem = s.off_tab + tab;
    s.cols = 32;
    while (s.cols < 2u * nt) s.cols *= 2;
    return s;
}

template <typename T, int BITS>
cudaError_t launch_tc(const CUtensorMap &map, const MatmulArgs &a, const TcShape &s, int64_t tiles, int *status, cudaStream_t st)
{
    static std::mutex mu;
    static unsigned raised = 0;  // devices whose shared-memory limit is raised
    int dev = 0;
    cudaError_t e = cudaGetDevice(&dev);
    if (e != cudaSuccess) return e;
    {
        std::lock_guard<std::mutex> lock(mu);
        if (dev >= 32 || !(raised >> dev & 1)) {
            e = cudaFuncSetAttribute(matmul_tc_kernel<T, BITS>, cudaFuncAttributeMaxDynamicSharedMemorySize, 227 * 1024);
            if (e != cudaSuccess) return e;
            if (dev < 32) raised |= 1u << dev;
        }
    }
    const int64_t pairs = device_sm_count() / 2;
    const unsigned grid = static_cast<unsigned>(2 * (tiles < pairs ? tiles : pairs));
    return launch_pdl(matmul_tc_kernel<T, BITS>, dim3(grid), BITS == 16 ? 384 : 640, s.smem, st, 1, map, a, s, status);
}

template <typename T>
cudaError_t launch_bits(const CUtensorMap &map, const MatmulArgs &a, const TcShape &s, int bits, int64_t tiles, int *status,
                        cudaStream_t st)
{
    if (bits == 16) return launch_tc<T, 16>(map, a, s, tiles, status, st);
    if (bits == 8) return launch_tc<T, 8>(map, a, s, tiles, status, st);
    if (bits == 4) return launch_tc<T, 4>(map, a, s, tiles, status, st);
    return launch_tc<T, 2>(map, a, s, tiles, status, st);
}

// Rows of x a tile.  A tile's MMAs take about 2 nt cycles for each 64 columns, but never less than the A operand takes to
// stage and read (kFloor), and a tile has a fixed cost (kFixed); the width with the least sum over the rounds of tiles
// that the CTA pairs make wins.
int choose_nt(const MatmulArgs &a)
{
    constexpr double kFloor = 220, kFixed = 3000;
    const int pairs = device_sm_count() / 2 > 0 ? device_sm_count() / 2 : 1;
    const int mt = (a.mb + 7) / 8;
    int best = 16;
    double cost = 0;
    for (int nt = 16; nt <= 256; nt += 16) {
        double tiles = static_cast<double>((a.rows + nt - 1) / nt);
        if (a.offsets) {  // every expert with rows ends in a partial tile: half a tile each
            const double live = a.experts < a.rows ? a.experts : static_cast<double>(a.rows);
            tiles = static_cast<double>(a.rows) / nt + 0.5 * live;
            if (tiles < live) tiles = live;
        }
        const double waves = std::ceil(tiles * mt / pairs);
        const double c = waves * (a.kb * (2.0 * nt > kFloor ? 2.0 * nt : kFloor) + kFixed);
        if (nt == 16 || c < cost) {
            cost = c;
            best = nt;
        }
    }
    return best;
}

}  // namespace

cudaError_t launch_matmul_tc(const MatmulArgs &a, int dtype, int bits, cudaStream_t st)
{
    if (a.rows == 0) return cudaSuccess;
    int *status = device_status_ptr();
    const EncodeTiled encode = encode_tiled();
    if (!status || !encode) return cudaErrorNotSupported;
    const int nt = choose_nt(a);
    const TcShape s = shape_of(a, bits, nt);
    int64_t u = (a.rows + nt - 1) / nt;
    if (a.offsets) u += a.experts < a.rows ? a.experts : a.rows;
    const int64_t tiles = u * s.mt;  // at most; experts' tiles are counted by the kernel
    if (tiles > 0x7fffffff / 2) return cudaErrorInvalidConfiguration;
    CUtensorMap map;
    const cuuint64_t dims[2] = {static_cast<cuuint64_t>(a.k), static_cast<cuuint64_t>(a.x_rows)};
    const cuuint64_t strides[1] = {static_cast<cuuint64_t>(a.ldx) * 2};
    const cuuint32_t box[2] = {64, a.gather ? 1u : static_cast<cuuint32_t>(nt / 2)}, unit[2] = {1, 1};
    if (encode(&map, dtype == QNN_F16 ? CU_TENSOR_MAP_DATA_TYPE_FLOAT16 : CU_TENSOR_MAP_DATA_TYPE_BFLOAT16, 2,
               const_cast<void *>(a.x), dims, strides, box, unit, CU_TENSOR_MAP_INTERLEAVE_NONE, CU_TENSOR_MAP_SWIZZLE_128B,
               CU_TENSOR_MAP_L2_PROMOTION_L2_256B, CU_TENSOR_MAP_FLOAT_OOB_FILL_NONE) != CUDA_SUCCESS)
        return cudaErrorInvalidValue;
    return dtype == QNN_F16 ? launch_bits<__half>(map, a, s, bits, tiles, status, st)
                            : launch_bits<__nv_bfloat16>(map, a, s, bits, tiles, status, st);
}

}  // namespace qnn
