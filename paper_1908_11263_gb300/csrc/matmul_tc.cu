// Matrix product on the 5th-generation tensor cores, for more rows of x than the streaming kernel takes.
//
// A pair of CTAs (cluster of two, cta_group::2) owns a tile of 256 image rows x `nt` rows of x: the weights are the
// A operand (128 rows in each CTA's shared memory, M = 256), x is the B operand (half of the rows in each CTA), the
// 32-bit accumulators sit in tensor memory, two tiles deep, so one tile's epilogue runs under the next tile's MMAs.
// With the weights on the M side a thread of the epilogue owns one output channel: its scale and bias are two
// registers, and the number of rows of x can be any multiple of 16 up to 256.
//
// Where the tiles fill half of the pairs at most, a cluster of several pairs takes one tile and splits its K; the other
// pairs write their sums into the first pair's shared memory, which adds them in order.
//
// Warps: 0 loads x and the weight blocks by tiled TMA, 1 issues the MMAs (first CTA of the pair), 2 hands
// complete stages of 16-bit weights on, 3 owns the tensor memory, 4-11 run the epilogue, 12-19 expand packed codes into
// the A operand, two groups on alternate stages.  Rows that an expert picks from x lie one after another before the
// launch: picking them inside it held the MMAs up (692 us with four-row TMA gathers, which take some 80 cycles each, 371
// with cp.async by two warps, for a product that takes 165 on rows in order and a copy that takes 27).
// Bound by the tensor pipe from about 500 rows of x on, with packed weights by the expansion, which every tile of x repeats
// and which hands a stage on in some 600 cycles where the MMAs take 512: 8192 x 4096 x 2 * 8192, gated silu, 533 us with
// 16-bit weights in ten calls in a row (2.06 PFLOP/s) and 556 in a hundred, where the power cap has set in; 734 INT-8, 644
// INT-4 and 616 INT-2 in a hundred.  Below 500 rows by the weights (64 x 8192 x 8192 16-bit 28 us) and, for small
// matrices, by its fixed cost of some 10 us.
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
    int ranks;                // pairs of a cluster that split K
    int group;                // tiles along the image rows that run side by side
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

// Arrives on the barrier at this address in the CTA of this rank (the pair's first).
__device__ __forceinline__ void mbar_arrive_at(uint64_t *bar, int rank)
{
    asm volatile(
        "{\n\t.reg .b32 r;\n\t"
        "mapa.shared::cluster.u32 r, %0, %1;\n\t"
        "mbarrier.arrive.shared::cluster.b64 _, [r];\n\t}" ::"r"(smem_addr(bar)),
        "r"(rank)
        : "memory");
}

// Stores a float at this shared-memory address of the CTA of this rank.
__device__ __forceinline__ void st_cluster(uint32_t at, int rank, float v)
{
    asm volatile("{\n\t.reg .b32 r;\n\tmapa.shared::cluster.u32 r, %0, %1;\n\tst.shared::cluster.f32 [r], %2;\n\t}" ::"r"(at),
                 "r"(rank), "f"(v)
                 : "memory");
}

// mbar_wait_warp with one look before the clock is read: the roles below wait once a stage, mostly for a phase that is
// complete or nearly so.
__device__ __forceinline__ bool wait_stage(uint64_t *bar, uint32_t parity, int *status)
{
    if (__all_sync(0xffffffffu, mbar_try_wait(bar, parity))) return true;
    return mbar_wait_warp(bar, parity, status);
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

// Arrives on this barrier in both CTAs of the pair (bits of `mask`) when the MMAs issued so far have completed.
__device__ __forceinline__ void mma2_commit_warp(uint64_t *bar, uint32_t mask)
{
    asm volatile(
        "{\n\t.reg .pred e;\n\t"
        "elect.sync _|e, 0xffffffff;\n\t"
        "@e tcgen05.commit.cta_group::2.mbarrier::arrive::one.shared::cluster.multicast::cluster.b64 [%0], %1;\n\t}" ::"r"(
            smem_addr(bar)),
        "h"(static_cast<uint16_t>(mask))
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

// Four 32-row blocks of the image, the same 64 columns, with one instruction: issuing a copy takes a warp some hundred
// cycles, and a copy for each block held a stage up to 600 cycles, whatever the MMAs took.
__device__ __forceinline__ void tma_blocks(void *dst, const CUtensorMap *map, int kb, int mb, uint64_t *bar)
{
    asm volatile(
        "cp.async.bulk.tensor.4d.shared::cluster.global.tile.mbarrier::complete_tx::bytes [%0], [%1, {%2, %2, %3, %4}], [%5];" ::"r"(
            smem_addr(dst)),
        "l"(map), "r"(0), "r"(kb), "r"(mb), "r"(smem_addr(bar))
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

// One lane's part of a tile's epilogue: sixteen rows of x (columns of the accumulator) at a time of one image row.  Without
// a gate a lane finishes its own channel.  With one, a channel's gate and up rows are eight lanes apart: of each two rows
// of x the gate lane finishes the first and the up lane the second.
// The residual of a chunk is loaded before the sums are waited for, that of the next chunk before this one is stored.
template <typename T, bool GATED>
struct Epilogue {
    static constexpr int kN = GATED ? 8 : 16, kRows = GATED ? 2 : 1;
    const MatmulArgs &a;
    float2 p;          // scale and bias
    int64_t row, ch;   // first row of the tile (of this lane's rows), channel
    int count;         // rows of the tile; none where the lane has no channel
    bool up;
    T res[kN];

    __device__ __forceinline__ Epilogue(const MatmulArgs &args, float2 params, int64_t first, int rows, int64_t channel)
        : a(args), p(params), row(first), ch(channel), count(channel < args.m ? rows : 0), up(GATED && (threadIdx.x & 8))
    {
        if (up) ++row;
    }
    // rows from column c on that this lane finishes
    __device__ __forceinline__ int mine(int c) const { return GATED ? (count - c + (up ? 0 : 1)) >> 1 : count - c; }

    __device__ __forceinline__ void fetch(int c)
    {
        if (a.residual)
            load_rows(static_cast<const T *>(a.residual) + (row + c) * a.ldres + ch, kRows * a.ldres, res, count ? mine(c) : 0);
    }

    // Finishes columns c .. c + 15 and fetches the residual of the chunk at `next`.  `others` sums of other pairs (one float
    // a lane and column, `step` floats apart) are added first.
    __device__ __forceinline__ void chunk(uint32_t src, int c, int next, const float *extra, int others, int step)
    {
        uint32_t acc[16];
        __syncwarp();
        tmem_ld16(src + c, acc);
        tmem_wait_ld();
        for (int o = 0; o < others; ++o)
#pragma unroll
            for (int i = 0; i < 16; ++i) acc[i] = __float_as_uint(__uint_as_float(acc[i]) + extra[o * step + (c + i) * 128]);
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
        if (a.residual) {
#pragma unroll
            for (int i = 0; i < kN; ++i) v[i] += to_f32<T>(res[i]);
            if (next < count) fetch(next);
        }
        const int n = count ? mine(c) : 0;
        if (a.out_f32)
            store_rows(static_cast<float *>(a.y) + (row + c) * a.ldy + ch, kRows * a.ldy, v, n);
        else
            store_rows(static_cast<T *>(a.y) + (row + c) * a.ldy + ch, kRows * a.ldy, v, n);
    }
};

// ---------------------------------------------------------------- tiles

struct Tile {
    int expert, mtile, count;
    int64_t first;
};

// Tile `id` of `us` tiles along the rows of x (of the experts one after another; `tab` holds the tiles before each
// expert): `group` tiles along the image rows, then along the rows of x, then the next group of image rows.  The pairs
// then work on about as many bytes of weights as of x at a time, and both stay in L2 while they are shared.
__device__ __forceinline__ Tile tile_at(const MatmulArgs &a, const TcShape &s, const int *tab, int us, int id)
{
    Tile t;
    const int block = id / (s.group * us), m0 = block * s.group, in = id - m0 * us;
    const int wide = min(s.group, s.mt - m0), u = in / wide;
    t.mtile = m0 + in - u * wide;
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

template <int BITS>
constexpr int kTcThreads = BITS == 16 ? 384 : 640;

template <typename T, int BITS>
__global__ void __launch_bounds__(kTcThreads<BITS>, 1)
    matmul_tc_kernel(const __grid_constant__ CUtensorMap xmap, const __grid_constant__ CUtensorMap wmap, const MatmulArgs a,
                     const TcShape s, int *status)
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
    const int cluster = static_cast<int>(cluster_rank());
    const int rank = cluster & 1, leader = cluster & ~1, split = cluster >> 1;  // CTA of the pair, its first CTA, share of K
    const int pair = blockIdx.x / (2 * s.ranks), pairs = gridDim.x / (2 * s.ranks);
    const uint32_t x_bytes = s.nt / 2 * 128;
    const int kb0 = a.kb * split / s.ranks, kb1 = a.kb * (split + 1) / s.ranks;  // this pair's 64-column blocks

    if (threadIdx.x == 0) {
        for (int i = 0; i < s.stages; ++i) {
            mbar_init(full + i, 1);
            mbar_init(ready + i, kPacked ? 8 : 2);
            mbar_init(empty + i, 1);
        }
        for (int i = 0; i < 2; ++i) {
            mbar_init(acc_full + i, 1);
            mbar_init(acc_empty + i, 16);
        }
        fence_mbar_init();
    }
    if (warp == 3) {
        asm volatile("tcgen05.alloc.cta_group::2.sync.aligned.shared::cta.b32 [%0], %1;" ::"r"(smem_addr(slot)), "r"(s.cols)
                     : "memory");
        asm volatile("tcgen05.relinquish_alloc_permit.cta_group::2.sync.aligned;" ::: "memory");
    }
    pdl_begin();
    if (warp == 3) {
        if (a.offsets) expert_tiles(a.offsets, a.experts, s.nt, tab);
        tc_fence_before();
    }
    __syncthreads();
    cluster_sync();
    tc_fence_after();
    const uint32_t tmem = *slot;
    const int us = a.offsets ? tab[a.experts] : static_cast<int>((a.rows + s.nt - 1) / s.nt), tiles = us * s.mt;

    if (a.zero_tail)  // rows that no expert fills
        for (int64_t r = a.offsets[a.experts] + blockIdx.x; r < a.rows; r += gridDim.x)
            for (int c = threadIdx.x; c < a.m; c += blockDim.x) static_cast<T *>(a.y)[r * a.ldy + c] = from_f32<T>(0.f);

    bool ok = true;
    int st = 0;          // stage, and the parity of its barriers' current phase
    uint32_t phase = 0;
    auto advance = [&]() {
        if (++st == s.stages) {
            st = 0;
            phase ^= 1;
        }
    };
    if (warp == 0) {
        // ------------------------------------------------ loads
        int uses = 0;
        for (int id = pair; id < tiles && ok; id += pairs) {
            const Tile t = tile_at(a, s, tab, us, id);
            const int mb = t.expert * a.mb + (t.mtile * 2 + rank) * 4;  // rows past the expert's are not stored
            for (int kb = kb0; kb < kb1; ++kb) {
                if (!wait_stage(empty + st, phase ^ 1, status)) {
                    ok = false;
                    break;
                }
                if (lane == 0) mbar_arrive_expect_tx(full + st, x_bytes + 4 * kBlock);
                __syncwarp();
                if (lane == 0)
                    tma_blocks(kPacked ? sm_raw + st * 4 * kBlock : sm_a + st * kABytes, &wmap, kb, mb, full + st);
                else if (lane == 1)
                    tma_tile(sm_x + st * x_bytes, &xmap, kb * 64, static_cast<int>(t.first) + rank * (s.nt / 2), full + st);
                __syncwarp();
                ++uses;
                advance();
            }
        }
        // copies still in flight land before the CTA may end
        for (int i = 0; i < min(uses, s.stages); ++i) {
            if (--st < 0) {
                st = s.stages - 1;
                phase ^= 1;
            }
            wait_stage(full + st, phase, status);
        }
    } else if (warp == 1 && rank == 0) {
        // ------------------------------------------------ MMAs
        constexpr uint32_t kFmt = std::is_same<T, __nv_bfloat16>::value ? 1u : 0u;
        const uint32_t idesc = (1u << 4) | (kFmt << 7) | (kFmt << 10) | (static_cast<uint32_t>(s.nt >> 3) << 17) | (16u << 24);
        const uint32_t both = 3u << leader;
        int it = 0;
        for (int id = pair; id < tiles && ok; id += pairs, ++it) {
            const int buf = it & 1;
            if (!wait_stage(acc_empty + buf, ((it >> 1) & 1) ^ 1, status)) {
                ok = false;
                break;
            }
            tc_fence_after();
            const uint32_t d = tmem + buf * s.nt;
            for (int kb = kb0; kb < kb1; ++kb) {
                if (!wait_stage(ready + st, phase, status)) {
                    ok = false;
                    break;
                }
                tc_fence_after();
                const uint64_t da = desc_sw128(smem_addr(sm_a + st * kABytes));
                const uint64_t db = desc_sw128(smem_addr(sm_x + st * x_bytes));
#pragma unroll
                for (int k = 0; k < 4; ++k) mma2_f16_warp(d, da + 2 * k, db + 2 * k, idesc, (kb - kb0) | k);
                mma2_commit_warp(empty + st, both);
                advance();
            }
            if (ok) mma2_commit_warp(acc_full + buf, both);
        }
    } else if (warp == 2 && !kPacked) {
        // ------------------------------------------------ complete stages of 16-bit weights
        for (int id = pair; id < tiles && ok; id += pairs)
            for (int kb = kb0; kb < kb1; ++kb) {
                if (!wait_stage(full + st, phase, status)) {
                    ok = false;
                    break;
                }
                if (lane == 0) mbar_arrive_at(ready + st, leader);
                __syncwarp();
                advance();
            }
    } else if (warp >= 4 && warp < 12) {
        // ------------------------------------------------ epilogue: two warps a quarter of the lanes
        const int quarter = warp & 3, half = (warp - 4) >> 2;
        int it = 0;
        for (int id = pair; id < tiles && ok; id += pairs, ++it) {
            const int buf = it & 1;
            const Tile t = tile_at(a, s, tab, us, id);
            const int row = t.mtile * 256 + rank * 128 + quarter * 32 + lane;  // image row
            const int ch = a.gated ? (row >> 4) * 8 + (row & 7) : row;
            const float2 p = row < a.mb * 32 ? a.params[static_cast<int64_t>(t.expert) * a.mb * 32 + row] : make_float2(0.f, 0.f);
            Epilogue<T, false> plain(a, p, t.first, t.count, ch);
            Epilogue<T, true> gated(a, p, t.first, t.count, ch);
            if (s.ranks == 1) {
                if (a.gated) gated.fetch(16 * half);
                else plain.fetch(16 * half);
            }
            if (!wait_stage(acc_full + buf, (it >> 1) & 1, status)) {
                ok = false;
                break;
            }
            tc_fence_after();
            if (s.ranks > 1) break;  // one tile a cluster: the sums of its pairs meet below
            const uint32_t src = tmem + buf * s.nt + (static_cast<uint32_t>(quarter * 32) << 16);
            for (int c = 16 * half; c < t.count; c += 32) {
                if (a.gated) gated.chunk(src, c, c + 32, nullptr, 0, 0);
                else plain.chunk(src, c, c + 32, nullptr, 0, 0);
            }
            __syncwarp();
            tc_fence_before();
            if (lane == 0) mbar_arrive_at(acc_empty + buf, leader);
            __syncwarp();
        }
    } else if (warp >= 12) {
        // ------------------------------------------------ packed codes to the A operand
        if constexpr (kPacked) {
            const int block = (warp - 12) & 3, group = (warp - 12) >> 2;  // 32-row block; stages taken by turns
            const int g = lane >> 2, tt = lane & 3;
            int turn = 0;
            for (int id = pair; id < tiles && ok; id += pairs)
                for (int kb = kb0; kb < kb1; ++kb, turn ^= 1) {
                    if (turn != group) {
                        advance();
                        continue;
                    }
                    // A barrier's parity tells two uses of a stage apart only for who knows that the one before is over, and
                    // with an odd number of stages that one was the other group's: its copies may still be in flight when a
                    // later stage's have landed.  So the stage is seen to be released first, as by the loader.  (The use
                    // before that was this group's own, and the MMAs, which go in order, have passed it: a group cannot be
                    // two uses behind.)
                    if (!wait_stage(empty + st, phase ^ 1, status) || !wait_stage(full + st, phase, status)) {
                        ok = false;
                        break;
                    }
                    const uint8_t *raw = sm_raw + st * 4 * kBlock + block * kBlock;
                    uint32_t w[2 * BITS];  // four runs of 16 codes: rows g, g + 8, g + 16, g + 24
#pragma unroll
                    for (int i = 0; i < BITS / 2; ++i)
                        *reinterpret_cast<uint4 *>(w + 4 * i) = reinterpret_cast<const uint4 *>(raw)[i * 32 + lane];
#pragma unroll
                    for (int h = 0; h < 4; ++h) {
                        uint32_t v[8];
                        expand16<T, BITS>(w + h * (BITS / 2), v);
                        uint8_t *dst = sm_a + st * kABytes + (block * 32 + h * 8 + g) * 128;
                        *reinterpret_cast<uint4 *>(dst + ((2 * tt) ^ g) * 16) = make_uint4(v[0], v[1], v[2], v[3]);
                        *reinterpret_cast<uint4 *>(dst + ((2 * tt + 1) ^ g) * 16) = make_uint4(v[4], v[5], v[6], v[7]);
                    }
                    fence_proxy_async_smem();
                    __syncwarp();
                    if (lane == 0) mbar_arrive_at(ready + st, leader);
                    __syncwarp();
                    advance();
                }
        }
    }
    __syncwarp();
    if (s.ranks > 1) {
        // The other pairs' sums go to the first pair's stages, which no copy or MMA uses any more: [pair - 1][column][lane].
        tc_fence_before();
        __syncthreads();
        cluster_sync();
        tc_fence_after();
        float *sums = reinterpret_cast<float *>(smem);
        const bool epilogue = warp >= 4 && warp < 12;
        const int quarter = warp & 3, half = (warp - 4) >> 2;
        const uint32_t src = tmem + (static_cast<uint32_t>(quarter * 32) << 16);
        const Tile t = tile_at(a, s, tab, us, pair);
        if (epilogue && split > 0)
            for (int c = 16 * half; c < t.count; c += 32) {
                uint32_t acc[16];
                tmem_ld16(src + c, acc);
                tmem_wait_ld();
                const uint32_t at = smem_addr(sums + ((split - 1) * s.nt + c) * 128 + quarter * 32 + lane);
#pragma unroll
                for (int i = 0; i < 16; ++i) st_cluster(at + i * 512, rank, __uint_as_float(acc[i]));
            }
        __syncwarp();
        cluster_sync();
        if (epilogue && split == 0) {
            const int row = t.mtile * 256 + rank * 128 + quarter * 32 + lane;
            const int ch = a.gated ? (row >> 4) * 8 + (row & 7) : row;
            const float2 p = row < a.mb * 32 ? a.params[row] : make_float2(0.f, 0.f);
            const float *extra = sums + quarter * 32 + lane;
            if (a.gated) {
                Epilogue<T, true> e(a, p, t.first, t.count, ch);
                e.fetch(16 * half);
                for (int c = 16 * half; c < t.count; c += 32) e.chunk(src, c, c + 32, extra, s.ranks - 1, s.nt * 128);
            } else {
                Epilogue<T, false> e(a, p, t.first, t.count, ch);
                e.fetch(16 * half);
                for (int c = 16 * half; c < t.count; c += 32) e.chunk(src, c, c + 32, extra, s.ranks - 1, s.nt * 128);
            }
        }
        __syncwarp();
    }
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

TcShape shape_of(const MatmulArgs &a, int bits, int nt, int ranks)
{
    TcShape s;
    s.nt = nt;
    s.ranks = ranks;
    s.mt = (a.mb + 7) / 8;
    // g tiles of weights (256 rows of `bits`) beside 76 / g tiles of x (nt rows of 16 bits): the fewest bytes at
    // g = sqrt(76 * 16 nt / (256 bits))
    s.group = static_cast<int>(std::sqrt(4.75 * nt / bits) + 0.5);
    if (s.group < 1) s.group = 1;
    if (s.group > s.mt) s.group = s.mt;
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
cudaError_t launch_tc(const CUtensorMap &map, const CUtensorMap &wmap, const MatmulArgs &a, const TcShape &s, int64_t tiles, int *status, cudaStream_t st)
{
    const cudaError_t e = raise_smem<matmul_tc_kernel<T, BITS>>(227 * 1024);
    if (e != cudaSuccess) return e;
    const int64_t pairs = device_sm_count() / 2;
    const unsigned grid = static_cast<unsigned>(s.ranks > 1 ? 2 * s.ranks * tiles : 2 * (tiles < pairs ? tiles : pairs));
    return launch_pdl(matmul_tc_kernel<T, BITS>, dim3(grid), kTcThreads<BITS>, s.smem, st, 2 * s.ranks, map, wmap, a, s, status);
}

template <typename T>
cudaError_t launch_bits(const CUtensorMap &map, const CUtensorMap &wmap, const MatmulArgs &a, const TcShape &s, int bits, int64_t tiles, int *status,
                        cudaStream_t st)
{
    if (bits == 16) return launch_tc<T, 16>(map, wmap, a, s, tiles, status, st);
    if (bits == 8) return launch_tc<T, 8>(map, wmap, a, s, tiles, status, st);
    if (bits == 4) return launch_tc<T, 4>(map, wmap, a, s, tiles, status, st);
    return launch_tc<T, 2>(map, wmap, a, s, tiles, status, st);
}

// Rows of x a tile, and pairs that split K.  A tile's MMAs take about 2 nt cycles for each 64 columns, but never less than
// a stage takes to be copied, expanded and handed on (kFloor), and a tile has a fixed cost (kFixed); a split adds the
// exchange of the sums.  The choice with the least sum over the rounds of tiles that the pairs make wins.
void choose(const MatmulArgs &a, int bits, int *nt_out, int *ranks_out)
{
    const double kFloor = 480, kFixed = 3000;
    const int pairs = device_sm_count() / 2 > 0 ? device_sm_count() / 2 : 1;
    const int mt = (a.mb + 7) / 8;
    double cost = 0;
    *nt_out = 0;
    for (int ranks = 1; ranks <= 4; ranks *= 2) {
        if (ranks > 1 && (a.offsets || a.kb < 4 * ranks)) break;
        for (int nt = 16; nt <= 256; nt += 16) {
            double tiles = static_cast<double>((a.rows + nt - 1) / nt);
            if (a.offsets) {  // every expert with rows ends in a partial tile: half a tile each
                const double live = a.experts < a.rows ? a.experts : static_cast<double>(a.rows);
                tiles = static_cast<double>(a.rows) / nt + 0.5 * live;
                if (tiles < live) tiles = live;
            }
            // clusters of eight CTAs leave some SMs of a GPC unused
            if (ranks > 1 && tiles * mt * ranks > (ranks == 4 ? 0.8 : 0.95) * pairs) continue;
            // the other pairs' sums have to fit the stages
            if (ranks > 1 && (ranks - 1) * nt * 512u > shape_of(a, bits, nt, ranks).off_bar) continue;
            const double waves = ranks > 1 ? 1 : std::ceil(tiles * mt / pairs);
            const double per_kb = 2.0 * nt > kFloor ? 2.0 * nt : kFloor;
            const double c = waves * ((a.kb + ranks - 1) / ranks * per_kb + kFixed) + (ranks > 1 ? 3000 + 20.0 * nt * (ranks - 1) : 0);
            if (*nt_out == 0 || c < cost) {
                cost = c;
                *nt_out = nt;
                *ranks_out = ranks;
            }
        }
    }
}

}  // namespace

cudaError_t launch_matmul_tc(const MatmulArgs &a, int dtype, int bits, cudaStream_t st)
{
    if (a.rows == 0) return cudaSuccess;
    int *status = device_status_ptr();
    const EncodeTiled encode = encode_tiled();
    if (!status || !encode) return cudaErrorNotSupported;
    int nt = 0, ranks = 1;
    choose(a, bits, &nt, &ranks);
    const TcShape s = shape_of(a, bits, nt, ranks);
    int64_t u = (a.rows + nt - 1) / nt;
    if (a.offsets) u += a.experts < a.rows ? a.experts : a.rows;
    const int64_t tiles = u * s.mt;  // at most; experts' tiles are counted by the kernel
    CUtensorMap map;
    const cuuint64_t dims[2] = {static_cast<cuuint64_t>(a.k), static_cast<cuuint64_t>(a.x_rows)};
    const cuuint64_t strides[1] = {static_cast<cuuint64_t>(a.ldx) * 2};
    const cuuint32_t box[2] = {64, static_cast<cuuint32_t>(nt / 2)}, unit[2] = {1, 1};
    if (encode(&map, dtype == QNN_F16 ? CU_TENSOR_MAP_DATA_TYPE_FLOAT16 : CU_TENSOR_MAP_DATA_TYPE_BFLOAT16, 2,
               const_cast<void *>(a.x), dims, strides, box, unit, CU_TENSOR_MAP_INTERLEAVE_NONE, CU_TENSOR_MAP_SWIZZLE_128B,
               CU_TENSOR_MAP_L2_PROMOTION_L2_256B, CU_TENSOR_MAP_FLOAT_OOB_FILL_NONE) != CUDA_SUCCESS)
        return cudaErrorInvalidValue;
    // the image as words: 128 of them, the rest of a block, the blocks along K, the 32-row groups of all experts
    CUtensorMap wmap;
    const cuuint64_t block = 32 * 64 * bits / 8;
    const cuuint64_t wdims[4] = {128, block / 512, static_cast<cuuint64_t>(a.kb), static_cast<cuuint64_t>(a.experts) * a.mb};
    const cuuint64_t wstrides[3] = {512, block, block * a.kb};
    const cuuint32_t wbox[4] = {128, static_cast<cuuint32_t>(block / 512), 1, 4}, wunit[4] = {1, 1, 1, 1};
    if (encode(&wmap, CU_TENSOR_MAP_DATA_TYPE_UINT32, 4, const_cast<uint8_t *>(a.image), wdims, wstrides, wbox, wunit,
               CU_TENSOR_MAP_INTERLEAVE_NONE, CU_TENSOR_MAP_SWIZZLE_NONE, CU_TENSOR_MAP_L2_PROMOTION_L2_256B,
               CU_TENSOR_MAP_FLOAT_OOB_FILL_NONE) != CUDA_SUCCESS)
        return cudaErrorInvalidValue;
    return dtype == QNN_F16 ? launch_bits<__half>(map, wmap, a, s, bits, tiles, status, st)
                            : launch_bits<__nv_bfloat16>(map, wmap, a, s, bits, tiles, status, st);
}

}  // namespace qnn
