// Attention of many rows on the 5th-generation tensor cores: prompts, chunks of them, cross attention.
//
// A tile is 256 rows of a sequence and key head (two halves of 128, the M of an MMA) over the keys that any of them sees, in
// units of 128.  The tiles' units, one tile after another, are shared evenly between the SMs, so causal, ragged and single
// long sequences load all of them alike; a tile that several share leaves parts (sum of 2^(z - m) v, m, sum of 2^(z - m))
// that a second launch joins in order.
//
// For each unit and half: S = Q K^T (A and B in shared memory, S in tensor memory); a thread a row takes S to registers,
// m = max, P = 2^(scale S - m), which replaces S in tensor memory as the A operand of O += P V.  Keys and values lie in
// shared memory as they come, rows of keys: for Q K^T that is K-major, for P V it is MN-major, so nothing is transposed.
// m is raised only where the maximum has grown by more than 2^8 (the weights stay below 2^8 then, and any m gives the same
// quotient), so that O, in tensor memory too, is rarely rescaled: conditional rescaling, a published refinement of the softmax
// in one pass.  P is rounded to the element type, off by half a step (2^-8
// of it for bf16, as the values are); its sum, m and O have 32 bits.
//
// Warps: 0-7 softmax and output, a group of four for each half; 8-11 load, each 32 keys of a unit, by tiled copies where all
// of them are there, else by cp.async, which takes rows from wherever their pages lie and fills with zeros what the cache does
// not have (past the length, in no page), whatever lies there; 12 and 13 issue the MMAs of a half each.  While the tensor
// cores work for one half, the other's softmax runs.
//
// A prompt of 8192 tokens, 32 heads on 8 key heads of 128: 470 us, 1.17 PFLOP/s (0.60 of a large product's).  Bound by what
// lies between the products: a unit's softmax takes some 2000 cycles beside the other warps' where its instructions alone take
// 900, a product starts 350 cycles after it is issued, P V and the next scores follow one another (P lies where S does).  A
// tile's output holds its half some 5000 cycles (heads of 128: a thread's own row).  With heads of 64 nothing is busy (16 * 448
// queries over up to 1500 keys, 16 heads: 65 us, tensor pipe 17 %, exponentials 22 %, issue slots 41 %): a unit takes
// more than 5000 cycles, and in which of its waits has not been measured.
#include <type_traits>

#include "attention.cuh"
#include "tensor_map.h"

namespace qnn {
namespace {

constexpr int kTcThreads = 512, kTcUnit = 128, kTcRows = 256, kLive = 8, kBins = 128;
// Of a tile beside its units, in units: filling the pipeline, output.  (A prompt of 8192 tokens 681 us with none, 537 with one,
// 470 with two and with four; 12 chunks over a cache 119, 117, 117 and 122.)
constexpr int kTileCost = 2;
constexpr long long kPassedLimit = 64 * kWaitLimitCycles;
constexpr float kRaise = 8.f;  // growth of the maximum (log2) that is left to the weights

template <int D>
struct TcRing {
    static constexpr int kStages = D == 64 ? 8 : 5;
    static constexpr uint32_t kHalf = 128 * 128;                // 128 rows of 64 elements
    static constexpr uint32_t kTile = kHalf * (D / 64);         // 128 rows of D
    static constexpr uint32_t kRing = 2 * kTile, kOut = kRing + kStages * kTile;
    // Room for the output on its way, where it does not cost a stage (a prompt of 8192 tokens, heads of 128: 497 us with four
    // stages, 461 with five).
    static constexpr bool kStaged = D == 64;
    static constexpr uint32_t kBars = kOut + (kStaged ? 2 * kHalf : 0);
    static constexpr uint32_t kSmem = kBars + kLive * 16 + kBins * 8 + 8 * (2 * kStages + 4 + 10 + 2 + kLive) + 16;
    // P beside S where tensor memory has room: the next scores then need not wait until P V has read the weights
    static constexpr bool kApart = D == 64;
    static constexpr uint32_t kPAt = kApart ? 256 : 0, kPStep = kApart ? 64 : 128, kOAt = kApart ? 384 : 256;
};
static_assert(TcRing<128>::kSmem <= 227 * 1024, "shared memory");

// ---------------------------------------------------------------- tensor memory

__device__ __forceinline__ void tmem_ld32(uint32_t taddr, float *v)
{
    asm volatile(
        "tcgen05.ld.sync.aligned.32x32b.x32.b32 "
        "{%0,%1,%2,%3,%4,%5,%6,%7,%8,%9,%10,%11,%12,%13,%14,%15,%16,%17,%18,%19,%20,%21,%22,%23,%24,%25,%26,%27,%28,%29,%30,%31}, [%32];"
        : "=f"(v[0]), "=f"(v[1]), "=f"(v[2]), "=f"(v[3]), "=f"(v[4]), "=f"(v[5]), "=f"(v[6]), "=f"(v[7]), "=f"(v[8]), "=f"(v[9]),
          "=f"(v[10]), "=f"(v[11]), "=f"(v[12]), "=f"(v[13]), "=f"(v[14]), "=f"(v[15]), "=f"(v[16]), "=f"(v[17]), "=f"(v[18]),
          "=f"(v[19]), "=f"(v[20]), "=f"(v[21]), "=f"(v[22]), "=f"(v[23]), "=f"(v[24]), "=f"(v[25]), "=f"(v[26]), "=f"(v[27]),
          "=f"(v[28]), "=f"(v[29]), "=f"(v[30]), "=f"(v[31])
        : "r"(taddr)
        : "memory");
}
__device__ __forceinline__ void tmem_st32(uint32_t taddr, const float *v)
{
    asm volatile(
        "tcgen05.st.sync.aligned.32x32b.x32.b32 [%0], "
        "{%1,%2,%3,%4,%5,%6,%7,%8,%9,%10,%11,%12,%13,%14,%15,%16,%17,%18,%19,%20,%21,%22,%23,%24,%25,%26,%27,%28,%29,%30,%31,%32};" ::"r"(
            taddr),
        "f"(v[0]), "f"(v[1]), "f"(v[2]), "f"(v[3]), "f"(v[4]), "f"(v[5]), "f"(v[6]), "f"(v[7]), "f"(v[8]), "f"(v[9]), "f"(v[10]),
        "f"(v[11]), "f"(v[12]), "f"(v[13]), "f"(v[14]), "f"(v[15]), "f"(v[16]), "f"(v[17]), "f"(v[18]), "f"(v[19]), "f"(v[20]),
        "f"(v[21]), "f"(v[22]), "f"(v[23]), "f"(v[24]), "f"(v[25]), "f"(v[26]), "f"(v[27]), "f"(v[28]), "f"(v[29]), "f"(v[30]),
        "f"(v[31])
        : "memory");
}

// D (+)= A B^T with A in tensor memory.
__device__ __forceinline__ void mma_f16_ts_warp(uint32_t d_tmem, uint32_t a_tmem, uint64_t b_desc, uint32_t idesc, uint32_t accumulate)
{
    asm volatile(
        "{\n\t.reg .pred p, e;\n\t"
        "elect.sync _|e, 0xffffffff;\n\t"
        "setp.ne.b32 p, %4, 0;\n\t"
        "@e tcgen05.mma.cta_group::1.kind::f16 [%0], [%1], %2, %3, p;\n\t}" ::"r"(d_tmem),
        "r"(a_tmem), "l"(b_desc), "r"(idesc), "r"(accumulate)
        : "memory");
}

// 128-byte swizzle, groups of eight rows 1024 bytes apart; `lbo`: bytes between blocks of 64 elements (MN-major operands).
__device__ __forceinline__ uint64_t swizzled(uint32_t saddr, uint32_t lbo)
{
    return static_cast<uint64_t>((saddr >> 4) & 0x3FFFu) | static_cast<uint64_t>(lbo >> 4) << 16 |
           static_cast<uint64_t>(1024 >> 4) << 32 | static_cast<uint64_t>(1) << 46 | static_cast<uint64_t>(2) << 61;
}

__device__ __forceinline__ bool wait_bar(uint64_t *bar, uint32_t parity, int *status)
{
    if (__all_sync(0xffffffffu, mbar_try_wait(bar, parity))) return true;
    return mbar_wait_warp(bar, parity, status);
}

// Arrives on the barrier (whose count includes it) once this thread's copies so far have landed.
__device__ __forceinline__ void copy_arrive(uint64_t *bar)
{
    asm volatile("cp.async.mbarrier.arrive.noinc.shared::cta.b64 [%0];" ::"r"(smem_addr(bar)) : "memory");
}

// More bytes to come for the barrier's phase; arrivals for a warp.
__device__ __forceinline__ void expect_bytes(uint64_t *bar, uint32_t bytes)
{
    asm volatile("mbarrier.expect_tx.relaxed.cta.shared::cta.b64 [%0], %1;" ::"r"(smem_addr(bar)), "r"(bytes) : "memory");
}
__device__ __forceinline__ void arrive_warp(uint64_t *bar)
{
    asm volatile("mbarrier.arrive.shared::cta.b64 _, [%0], 32;" ::"r"(smem_addr(bar)) : "memory");
}
// Box of a four-dimensional tensor.
__device__ __forceinline__ void tma_box(uint32_t dst, const CUtensorMap *map, int x, int y, int z, int w, uint64_t *bar)
{
    asm volatile(
        "cp.async.bulk.tensor.4d.shared::cluster.global.tile.mbarrier::complete_tx::bytes [%0], [%1, {%2, %3, %4, %5}], [%6];" ::"r"(dst),
        "l"(map), "r"(x), "r"(y), "r"(z), "r"(w), "r"(smem_addr(bar))
        : "memory");
}

// (x, y) * (s, s) + (c, c), (x, y) + (u, v)
__device__ __forceinline__ float2 fma2(float2 x, float2 s, float2 c)
{
    float2 r;
    asm("fma.rn.f32x2 %0, %1, %2, %3;"
        : "=l"(*reinterpret_cast<uint64_t *>(&r))
        : "l"(*reinterpret_cast<const uint64_t *>(&x)), "l"(*reinterpret_cast<const uint64_t *>(&s)),
          "l"(*reinterpret_cast<const uint64_t *>(&c)));
    return r;
}
__device__ __forceinline__ float2 add2(float2 x, float2 y)
{
    float2 r;
    asm("add.rn.f32x2 %0, %1, %2;"
        : "=l"(*reinterpret_cast<uint64_t *>(&r))
        : "l"(*reinterpret_cast<const uint64_t *>(&x)), "l"(*reinterpret_cast<const uint64_t *>(&y)));
    return r;
}

// ---------------------------------------------------------------- tiles

// The keys that the rows of a tile see, in units.
struct TileKeys {
    int first, units, lo, hi;
};
__device__ __forceinline__ int tile_count(const AttnArgs &a, const Sequence &q)
{
    const int rows = q.n * a.group;  // tokens times heads are below 2^31
    return rows > a.few ? (rows - 1) / kTcRows + 1 : 0;
}
__device__ __forceinline__ TileKeys tile_keys(const AttnArgs &a, const Sequence &q, int rt)
{
    const uint32_t r0 = static_cast<uint32_t>(rt) * kTcRows;
    const int last = static_cast<int>((r0 + kTcRows - 1) / static_cast<uint32_t>(a.group));
    TileKeys t;
    int x, y;
    keys_of(a, q, static_cast<int>(r0 / static_cast<uint32_t>(a.group)), t.lo, x);
    keys_of(a, q, last < q.n - 1 ? last : q.n - 1, y, t.hi);
    if (x > t.hi) t.hi = x;
    t.first = t.lo / kTcUnit;
    t.units = (t.hi + kTcUnit - 1) / kTcUnit - t.first;
    if (t.units < 1) t.units = 1;
    return t;
}

// A place in the order of units.
struct TcCursor {
    Sequence q;
    TileKeys w;
    int s, rt, h, pos, tiles;  // pos: in the tile's kTileCost + units

    __device__ __forceinline__ void open(const AttnArgs &a)
    {
        q = sequence(a, s);
        tiles = tile_count(a, q);
    }
    __device__ __forceinline__ int rows(const AttnArgs &a) const  // of the tile
    {
        const int left = q.n * a.group - rt * kTcRows;
        return left < kTcRows ? left : kTcRows;
    }
    __device__ __forceinline__ void next_tile(const AttnArgs &a)
    {
        pos = 0;
        if (++h < a.kv_heads) return;
        h = 0;
        if (++rt >= tiles) {
            rt = 0;
            do {
                if (++s >= a.seqs) return;
                open(a);
            } while (tiles == 0);
        }
        w = tile_keys(a, q, rt);
    }
};

// What a share has of the tile it is at: units begin .. begin + count.
struct Segment {
    int begin, count;
    bool whole, last;  // with the first, the last unit
};
__device__ __forceinline__ Segment take(const TcCursor &at, int64_t &left)
{
    const int room = at.w.units + kTileCost - at.pos, n = static_cast<int>(room < left ? room : left);
    left -= n;
    Segment g;
    g.begin = max(0, at.pos - kTileCost);
    const int end = max(0, at.pos + n - kTileCost);
    g.count = end - g.begin;
    g.whole = g.begin == 0;
    g.last = end == at.w.units;
    return g;
}

__device__ __forceinline__ int64_t warp_scan(int64_t v)  // inclusive
{
    const int lane = threadIdx.x & 31;
#pragma unroll
    for (int d = 1; d < 32; d *= 2) {
        const int64_t o = __shfl_up_sync(0xffffffffu, v, d);
        if (lane >= d) v += o;
    }
    return v;
}

// Units (with the tiles' own cost) of the sequences s0 + lane (those below s1) for one key head; all lanes of a warp.
__device__ __noinline__ int64_t sequence_units(const AttnArgs &a, int s0, int s1)
{
    const int lane = threadIdx.x & 31, s = s0 + lane;
    Sequence q = {0, 0, 0, 0};
    int tiles = 0;
    if (s < s1) {
        q = sequence(a, s);
        tiles = tile_count(a, q);
    }
    int64_t sum = 0;
    if (tiles <= 4)
#pragma unroll 1
        for (int rt = 0; rt < tiles; ++rt) sum += tile_keys(a, q, rt).units + kTileCost;
    for (uint32_t many = __ballot_sync(0xffffffffu, tiles > 4); many; many &= many - 1) {
        const int from = __ffs(many) - 1;
        Sequence o;
        o.first = 0;
        o.n = __shfl_sync(0xffffffffu, q.n, from);
        o.keys = __shfl_sync(0xffffffffu, q.keys, from);
        o.at = __shfl_sync(0xffffffffu, q.at, from);
        const int t = __shfl_sync(0xffffffffu, tiles, from);
        int64_t part = 0;
#pragma unroll 1
        for (int rt = lane; rt < t; rt += 32) part += tile_keys(a, o, rt).units + kTileCost;
#pragma unroll
        for (int d = 16; d; d >>= 1) part += __shfl_xor_sync(0xffffffffu, part, d);
        if (lane == from) sum = part;
    }
    return sum;
}

// Where a block's share begins.
struct Start {
    int64_t x0, x1, total, u0, u1;  // share; all units; those of the tile with the first, without the tile's own cost
    int s, rt, h, pos;
};

// Called by all threads: units in bins of sequences, the share, and (first warp) the place of its first unit.
__device__ void find_start(const AttnArgs &a, int64_t *bins, Start *out)
{
    const int warp = threadIdx.x >> 5, lane = threadIdx.x & 31;
    const int chunks = (a.seqs + 31) / 32, per = (chunks + kBins - 1) / kBins, used = (chunks + per - 1) / per;
    for (int b = warp; b < used; b += kTcThreads / 32) {
        int64_t sum = 0;
        for (int c = b * per; c < (b + 1) * per && c < chunks; ++c) sum += sequence_units(a, c * 32, a.seqs);
        sum = __shfl_sync(0xffffffffu, warp_scan(sum), 31);
        if (lane == 0) bins[b] = sum * a.kv_heads;
    }
    __syncthreads();
    if (warp == 0) {
        int64_t mine[kBins / 32], sum = 0;
#pragma unroll
        for (int i = 0; i < kBins / 32; ++i) {
            const int b = lane * (kBins / 32) + i;
            mine[i] = b < used ? bins[b] : 0;
            sum += mine[i];
        }
        const int64_t end = warp_scan(sum), total = __shfl_sync(0xffffffffu, end, 31);
        const int64_t x0 = total * blockIdx.x / gridDim.x, x1 = total * (blockIdx.x + 1) / gridDim.x;
        int64_t before = end - sum;
        int bin = -1;
        int64_t at = 0;
#pragma unroll
        for (int i = 0; i < kBins / 32; ++i) {
            if (before <= x0 && x0 < before + mine[i]) {
                bin = lane * (kBins / 32) + i;
                at = before;
            }
            before += mine[i];
        }
        Start st = {x0, x1, total, 0, 0, 0, 0, 0, 0};
        if (total > 0) {
            const int who = __ffs(__ballot_sync(0xffffffffu, bin >= 0)) - 1;
            bin = __shfl_sync(0xffffffffu, bin, who);
            at = __shfl_sync(0xffffffffu, at, who);
            // the sequence
            for (int c = bin * per;; ++c) {
                const int64_t n = sequence_units(a, c * 32, a.seqs) * a.kv_heads, e = at + warp_scan(n);
                const uint32_t hit = __ballot_sync(0xffffffffu, e - n <= x0 && x0 < e);
                if (hit) {
                    st.s = c * 32 + __ffs(hit) - 1;
                    at = __shfl_sync(0xffffffffu, e - n, __ffs(hit) - 1);
                    break;
                }
                at = __shfl_sync(0xffffffffu, e, 31);
                if ((c + 1) * 32 >= a.seqs) break;  // not reached: the bin holds the unit
            }
            // the row tile
            const Sequence q = sequence(a, st.s);
            const int tiles = tile_count(a, q);
            for (int r0 = 0; r0 < tiles; r0 += 32) {
                const int units = r0 + lane < tiles ? tile_keys(a, q, r0 + lane).units + kTileCost : 0;
                const int64_t n = static_cast<int64_t>(units) * a.kv_heads, e = at + warp_scan(n);
                const uint32_t hit = __ballot_sync(0xffffffffu, e - n <= x0 && x0 < e);
                if (hit) {
                    const int l = __ffs(hit) - 1, each = __shfl_sync(0xffffffffu, units, l);
                    at = __shfl_sync(0xffffffffu, e - n, l);
                    st.rt = r0 + l;
                    st.h = static_cast<int>((x0 - at) / each);
                    st.pos = static_cast<int>(x0 - at - static_cast<int64_t>(st.h) * each);
                    st.u0 = x0 - st.pos + kTileCost;
                    st.u1 = x0 - st.pos + each;
                    break;
                }
                at = __shfl_sync(0xffffffffu, e, 31);
            }
        }
        if (lane == 0) *out = st;
    }
    __syncthreads();
}

// ---------------------------------------------------------------- parts of shared tiles

struct TcRecord {
    int64_t x0, u0, u1, total;  // as in Start
    int s, h, rt, pad;
};
struct TcParts {
    float *sums, *stats;  // [2 * blocks][D][256], [2 * blocks][2][256]: m, then l
    TcRecord *records;    // [blocks]
};
template <int D>
__device__ __forceinline__ TcParts tc_parts(float *p, int blocks)
{
    TcParts s;
    s.sums = p;
    s.stats = p + static_cast<int64_t>(2 * blocks) * kTcRows * D;
    s.records = reinterpret_cast<TcRecord *>(s.stats + 2 * blocks * 2 * kTcRows);
    return s;
}

// ---------------------------------------------------------------- the kernel

template <typename T, int D>
__global__ void __launch_bounds__(kTcThreads, 1)
    attention_tc_kernel(const __grid_constant__ CUtensorMap q_map, const __grid_constant__ CUtensorMap k_map,
                        const __grid_constant__ CUtensorMap v_map, const AttnArgs a, int *status)
{
    using R = TcRing<D>;
    extern __shared__ __align__(1024) uint8_t smem[];
    uint32_t *live = reinterpret_cast<uint32_t *>(smem + R::kBars);  // [kLive][4]: keys of a unit that are in the cache
    int64_t *bins = reinterpret_cast<int64_t *>(live + kLive * 4);
    uint64_t *full = reinterpret_cast<uint64_t *>(bins + kBins), *empty = full + R::kStages;
    uint64_t *q_full = empty + R::kStages, *q_empty = q_full + 2, *s_full = q_empty + 2, *s_read = s_full + 2;
    uint64_t *p_full = s_read + 2, *pv_done = p_full + 4, *drained = pv_done + 2, *live_full = drained + 2;  // p_full: [half][64 keys]
    uint32_t *slot = reinterpret_cast<uint32_t *>(live_full + kLive);
    __shared__ Start start;
    __shared__ TcCursor kept[8];        // the softmax warps' places: in registers they would push scores out
    __shared__ volatile int begun[2];  // units whose weights a half has begun with
    const int warp = threadIdx.x >> 5, lane = threadIdx.x & 31;

    if (threadIdx.x == 0) {
        for (int i = 0; i < R::kStages; ++i) {
            mbar_init(full + i, 128);
            mbar_init(empty + i, 2);
        }
        for (int i = 0; i < 2; ++i) {
            mbar_init(s_full + i, 1);
            mbar_init(s_read + i, 4);
            mbar_init(p_full + 2 * i, 4);
            mbar_init(p_full + 2 * i + 1, 4);
            mbar_init(pv_done + i, 1);
            mbar_init(q_full + i, 128);
            mbar_init(q_empty + i, 1);
            mbar_init(drained + i, 1);
        }
        begun[0] = begun[1] = 0;
        for (int i = 0; i < kLive; ++i) mbar_init(live_full + i, 4);
        fence_mbar_init();
    }
    if (warp == 12) {
        tmem_alloc(slot, 512);
        tmem_relinquish();
        tc_fence_before();
    }
    pdl_begin();
    find_start(a, bins, &start);
    tc_fence_after();
    const uint32_t tmem = *slot;
    if (threadIdx.x == 0 && a.tc_part) {
        TcRecord &r = tc_parts<D>(a.tc_part, gridDim.x).records[blockIdx.x];
        r.x0 = start.x0;
        r.u0 = start.u0;
        r.u1 = start.u1;
        r.total = start.total;
        r.s = start.s;
        r.h = start.h;
        r.rt = start.rt;
    }
    int64_t left = start.x1 - start.x0;
    TcCursor at;
    at.s = start.s;
    at.rt = start.rt;
    at.h = start.h;
    at.pos = start.pos;
    if (left > 0) {
        at.open(a);
        at.w = tile_keys(a, at.q, at.rt);
    }
    const int steps = (a.d + 15) / 16, width = steps * 16;  // 16-element steps of a head
    bool ok = true;

    if (warp < 8) {
        // ------------------------------------------------ softmax and output: thread a row
        asm volatile("setmaxnreg.inc.sync.aligned.u32 184;");
        const int half = warp >> 2;
        const uint32_t lanes = static_cast<uint32_t>((warp & 3) * 32) << 16;
        const uint32_t s_at = tmem + lanes + half * 128, p_at = tmem + lanes + R::kPAt + half * R::kPStep;
        const uint32_t o_at_ = tmem + lanes + R::kOAt + half * D;
        uint32_t s_phase = 0, pv_phase = 0;  // parities of the next waits
        int unit = 0;                        // of the block, for the ring of masks
        bool passed = false;                 // the half has passed units by, which the other one takes its time for
        if (lane == 0) kept[warp] = at;
        __syncwarp();
        auto go_on = [&](TcCursor &place) {
            place.next_tile(a);
            __syncwarp();
            if (lane == 0) kept[warp] = place;
            __syncwarp();
        };
        while (left > 0 && ok) {
            Segment seg;
            int first_key, lo = 0, hi = 0, lo_most, hi_least;
            {
                TcCursor here = kept[warp];
                const int rows = here.rows(a);
                seg = take(here, left);
                if (rows <= half * 128 || seg.count == 0) {  // nothing in this half
                    unit += seg.count;
                    passed = true;
                    if (!R::kApart && half == 1 && (warp & 3) == 0 && lane == 0) begun[1] = unit;
                    go_on(here);
                    continue;
                }
                first_key = (here.w.first + seg.begin) * kTcUnit;
                const int r = half * 128 + (warp & 3) * 32 + lane;
                const uint32_t r0 = here.rt * static_cast<uint32_t>(kTcRows), group = a.group;
                if (r < rows) keys_of(a, here.q, static_cast<int>((r0 + r) / group), lo, hi);
                // keys that every row of the half sees: from the last query's first to the first query's last
                int x;
                keys_of(a, here.q, static_cast<int>((r0 + half * 128) / group), x, hi_least);
                keys_of(a, here.q, static_cast<int>((r0 + min(rows, half * 128 + 128) - 1) / group), lo_most, x);
            }
            float m = -INFINITY, l = 0.f;
            for (int i = 0; i < seg.count; ++i, ++unit) {
                const int key0 = first_key + i * kTcUnit;
                // The scores first: the mask of a unit whose scores are there is in its place, and is not replaced before P V has used
                // the weights.  (A half that has passed tiles by would take an earlier turn of the mask's barrier for its own.)
                if ((passed ? !mbar_wait_warp(s_full + half, s_phase, status, kPassedLimit) : !wait_bar(s_full + half, s_phase, status)) ||
                    !wait_bar(live_full + unit % kLive, (unit / kLive) & 1, status)) {
                    ok = false;
                    break;
                }
                passed = false;
                s_phase ^= 1;
                tc_fence_after();
                const uint4 there = *reinterpret_cast<const uint4 *>(live + (unit % kLive) * 4);
                if (!(key0 >= lo_most && key0 + kTcUnit <= hi_least && (there.x & there.y & there.z & there.w) == 0xffffffffu)) {
                    // few units: their scores are masked where they lie
#pragma unroll 1
                    for (int c = 0; c < 4; ++c) {
                        // bits [lo, hi) of the 32 keys
                        const int b0 = min(max(lo - key0 - 32 * c, 0), 32), b1 = min(max(hi - key0 - 32 * c, 0), 32);
                        const uint32_t below = b1 == 32 ? 0xffffffffu : (1u << b1) - 1, under = b0 == 32 ? 0xffffffffu : (1u << b0) - 1;
                        const uint32_t seen = live[(unit % kLive) * 4 + c] & below & ~under;
                        float v[32];
                        tmem_ld32(s_at + 32 * c, v);
                        tmem_wait_ld();
#pragma unroll
                        for (int e = 0; e < 32; ++e)
                            if (!(seen >> e & 1)) v[e] = -INFINITY;
                        tmem_st32(s_at + 32 * c, v);
                    }
                    tmem_wait_st();
                }
                float z[128];
#pragma unroll
                for (int c = 0; c < 4; ++c) tmem_ld32(s_at + 32 * c, z + 32 * c);
                tmem_wait_ld();
                if constexpr (R::kApart) {
                    tc_fence_before();
                    __syncwarp();
                    if (lane == 0) mbar_arrive(s_read + half);
                    __syncwarp();
                }
                float top[4] = {-INFINITY, -INFINITY, -INFINITY, -INFINITY};
#pragma unroll
                for (int e = 0; e < 128; e += 8)
#pragma unroll
                    for (int c = 0; c < 4; ++c) top[c] = fmaxf(top[c], fmaxf(z[e + 2 * c], z[e + 2 * c + 1]));
                const float most = fmaxf(fmaxf(top[0], top[1]), fmaxf(top[2], top[3])) * a.scale;
                if constexpr (R::kApart) {  // the last P V of the tile has read its weights, and O is at rest
                    if (i > 0) {
                        if (!wait_bar(pv_done + half, pv_phase ^ 1, status)) {
                            ok = false;
                            break;
                        }
                        tc_fence_after();
                    }
                }
                if (i == 0) {
                    m = most;
                } else if (__any_sync(0xffffffffu, most > m + kRaise)) {
                    // where P replaces S, S was computed after the last P V ended
                    const float raised = fmaxf(m, most), factor = raised == -INFINITY ? 1.f : exp2_fast(m - raised);
                    m = raised;
                    l *= factor;
#pragma unroll 1
                    for (int c = 0; c < width; c += 16) {
                        uint32_t o[16];
                        tmem_ld16(o_at_ + c, o);
                        tmem_wait_ld();
#pragma unroll
                        for (int e = 0; e < 16; ++e) o[e] = __float_as_uint(__uint_as_float(o[e]) * factor);
                        tmem_st16(o_at_ + c, o);
                    }
                }
                if (!R::kApart && (warp & 3) == 0 && lane == 0) begun[half] = unit + 1;
                const float ref = m == -INFINITY ? 0.f : -m;
                const float2 ref2 = make_float2(ref, ref), scale2 = make_float2(a.scale, a.scale);
                float2 sum0 = make_float2(0.f, 0.f), sum1 = sum0;
#pragma unroll
                for (int c = 0; c < 2; ++c) {
                    float p[32];  // pairs of weights
#pragma unroll
                    for (int e = 0; e < 32; e += 2) {
                        float2 v0 = fma2(make_float2(z[64 * c + 2 * e], z[64 * c + 2 * e + 1]), scale2, ref2);
                        float2 v1 = fma2(make_float2(z[64 * c + 2 * e + 2], z[64 * c + 2 * e + 3]), scale2, ref2);
                        v0 = make_float2(exp2_fast(v0.x), exp2_fast(v0.y));
                        v1 = make_float2(exp2_fast(v1.x), exp2_fast(v1.y));
                        sum0 = add2(sum0, v0);
                        sum1 = add2(sum1, v1);
                        p[e] = __uint_as_float(pack2<T>(v0.x, v0.y));
                        p[e + 1] = __uint_as_float(pack2<T>(v1.x, v1.y));
                    }
                    tmem_st32(p_at + 32 * c, p);
                    tmem_wait_st();
                    tc_fence_before();
                    __syncwarp();
                    if (lane == 0) mbar_arrive(p_full + 2 * half + c);
                    __syncwarp();
                }
                l += (sum0.x + sum0.y) + (sum1.x + sum1.y);
                pv_phase ^= 1;
            }
            if (!ok) break;
            // the last P V of the share
            if (!wait_bar(pv_done + half, pv_phase ^ 1, status)) {
                ok = false;
                break;
            }
            tc_fence_after();
            const bool complete = seg.whole && seg.last;
            const int64_t part_slot = 2 * blockIdx.x + (seg.whole ? 1 : 0);
            const float inv = l == 0.f ? 0.f : 1.f / l;
            TcCursor here = kept[warp];
            const int rows = here.rows(a), r = half * 128 + (warp & 3) * 32 + lane;
            const uint32_t row = here.rt * static_cast<uint32_t>(kTcRows) + r, group = a.group;
            const int qi = static_cast<int>(row / group), head = here.h * a.group + static_cast<int>(row - qi * group);
            const int64_t place = r < rows ? o_at(a, here.q, qi, head) : -1;
            const TcParts parts = tc_parts<D>(a.tc_part, gridDim.x);
            // Through shared memory where there is room (chunk c of row r at c ^ (r & 7)), so that stores take whole lines: a
            // thread's own row touches a line for every 32 bytes, and holds up all else that goes to memory.
            uint8_t *out = smem + R::kOut + half * R::kHalf + (warp & 3) * 32 * 128;
            float *sums = parts.sums + (part_slot * D) * kTcRows + r;
#pragma unroll 1
            for (int c0 = 0; c0 < a.d; c0 += 64) {
#pragma unroll 1
                for (int c = c0; c < c0 + 64 && c < a.d; c += 16) {  // short code: each tile comes here once
                    uint32_t raw[16];
                    __syncwarp();
                    tmem_ld16(o_at_ + c, raw);
                    tmem_wait_ld();
                    if (!complete) {
#pragma unroll
                        for (int e = 0; e < 16; ++e) sums[static_cast<int64_t>(c + e) * kTcRows] = __uint_as_float(raw[e]);
                    } else {
                        uint32_t w[8];
#pragma unroll
                        for (int e = 0; e < 8; ++e) w[e] = pack2<T>(__uint_as_float(raw[2 * e]) * inv, __uint_as_float(raw[2 * e + 1]) * inv);
                        if constexpr (!R::kStaged) {
                            T *y = static_cast<T *>(a.out) + place + c;
                            if (place < 0) continue;
                            if (a.out_vec8 && c + 16 <= a.d && (reinterpret_cast<uintptr_t>(y) & 31) == 0) {  // a whole sector
                                asm volatile("st.global.v8.b32 [%0], {%1,%2,%3,%4,%5,%6,%7,%8};" ::"l"(y), "r"(w[0]), "r"(w[1]), "r"(w[2]),
                                             "r"(w[3]), "r"(w[4]), "r"(w[5]), "r"(w[6]), "r"(w[7])
                                             : "memory");
                            } else if (a.out_vec8) {
                                *reinterpret_cast<uint4 *>(y) = make_uint4(w[0], w[1], w[2], w[3]);
                                if (c + 8 < a.d) *reinterpret_cast<uint4 *>(y + 8) = make_uint4(w[4], w[5], w[6], w[7]);
                            } else {
                                uint16_t *h = reinterpret_cast<uint16_t *>(y);
#pragma unroll
                                for (int j = 0; j < 16; ++j)
                                    if (c + j < a.d) h[j] = static_cast<uint16_t>(w[j >> 1] >> (16 * (j & 1)));
                            }
                            continue;
                        }
                        const int k = (c - c0) / 8;
                        *reinterpret_cast<uint4 *>(out + lane * 128 + ((k ^ (lane & 7)) * 16)) = make_uint4(w[0], w[1], w[2], w[3]);
                        *reinterpret_cast<uint4 *>(out + lane * 128 + (((k + 1) ^ (lane & 7)) * 16)) = make_uint4(w[4], w[5], w[6], w[7]);
                    }
                }
                __syncwarp();
                if (!complete || !R::kStaged) continue;
                const int k = lane & 7, col = c0 + 8 * k;
#pragma unroll 1
                for (int i = 0; i < 32; i += 4) {
                    const int rr = i + (lane >> 3);
                    const int64_t to = __shfl_sync(0xffffffffu, place, rr);
                    if (to < 0 || col >= a.d) continue;
                    const uint4 v = *reinterpret_cast<const uint4 *>(out + rr * 128 + ((k ^ (rr & 7)) * 16));
                    T *y = static_cast<T *>(a.out) + to + col;
                    if (a.out_vec8) {
                        *reinterpret_cast<uint4 *>(y) = v;
                    } else {
                        const uint32_t w[4] = {v.x, v.y, v.z, v.w};
                        uint16_t *h = reinterpret_cast<uint16_t *>(y);
#pragma unroll
                        for (int j = 0; j < 8; ++j) h[j] = static_cast<uint16_t>(w[j >> 1] >> (16 * (j & 1)));
                    }
                }
                __syncwarp();
            }
            if (r < rows) {
                if (!complete) {
                    const int64_t base = part_slot * (2 * kTcRows);
                    parts.stats[base + r] = m;
                    parts.stats[base + kTcRows + r] = l;
                } else if (a.lse) {
                    a.lse[lse_at(a, here.q, qi, head)] = l == 0.f ? -INFINITY : kLn2 * m + logf(l);
                }
            }
            tc_fence_before();  // O is read before the next tile's first P, after which it is written again
            go_on(here);
        }
    } else {
        asm volatile("setmaxnreg.dec.sync.aligned.u32 72;");
        if (warp < 12) {
            // ------------------------------------------------ loads: each warp 32 keys of a unit
            const int quarter = warp - 8, chunks = width / 8;
            constexpr int kChunks = D / 8, kPass = 32 / kChunks;  // 16-byte chunks of a row, rows a pass
            const int chunk = lane % kChunks, sub = lane / kChunks;
            const uint32_t base = smem_addr(smem);
            const uint32_t at_chunk = (chunk >> 3) * R::kHalf;
            int st = 0, unit = 0, uses = 0;
            uint32_t phase = 0, q_phase[2] = {0, 0};
            int page = -1, row = 0;
            auto find = [&](int u) {
                const int key = (at.w.first + u) * kTcUnit + quarter * 32 + lane;
                page = -1;
                if (key >= at.w.lo && key < at.w.hi) {
                    const int column = key / a.page_size;
                    row = key - column * a.page_size;
                    page = page_of(a, at.s, column);
                }
            };
            auto claim = [&]() {  // the next stage is free
                if (!wait_bar(empty + st, phase ^ 1, status)) ok = false;
            };
            // The warp's keys to the next stage: rows that lie in pages by tiled copies where all 32 are there, else by
            // cp.async, with zeros for those that are not.
            auto fill = [&](const void *from, const CUtensorMap &map, bool whole, int pg, int rw, int64_t place) {
                const uint32_t to = base + R::kRing + st * R::kTile;
                if (whole) {
                    const int boxes = 32 / a.box, box = lane % boxes, part = lane / boxes;
                    const int p = __shfl_sync(0xffffffffu, pg, box * a.box), r = __shfl_sync(0xffffffffu, rw, box * a.box);
                    if (lane == 0) expect_bytes(full + st, 32 * 128 * (D / 64));
                    __syncwarp();
                    if (part < D / 64)
                        tma_box(to + part * R::kHalf + (quarter * 32 + box * a.box) * 128, &map, part * 64, r, at.h, p, full + st);
                    if (lane == 0) arrive_warp(full + st);
                    __syncwarp();
                } else {
                    const T *p = static_cast<const T *>(from);
#pragma unroll 4
                    for (int i = 0; i < 32 / kPass; ++i) {
                        const int rr = i * kPass + sub;
                        const int64_t off = __shfl_sync(0xffffffffu, place, rr);
                        const bool there = off >= 0 && chunk * 8 < a.d;
                        const int key = quarter * 32 + rr;
                        if (chunk < chunks)
                            copy16(to + at_chunk + key * 128 + (((chunk & 7) ^ (key & 7)) * 16), there ? p + off + chunk * 8 : p, there ? 16 : 0);
                    }
                    copy_arrive(full + st);
                }
                ++uses;
                if (++st == R::kStages) {
                    st = 0;
                    phase ^= 1;
                }
            };
            while (left > 0 && ok) {
                const int rows = at.rows(a);
                const Segment seg = take(at, left);
                if (seg.count > 0) find(seg.begin);
                for (int i = 0; i < seg.count && ok; ++i, ++unit) {
                    const int64_t pk = page < 0 ? -1 : page * a.k_page + at.h * a.k_head + row * a.k_row;
                    const int64_t pv = page < 0 ? -1 : page * a.v_page + at.h * a.v_head + row * a.v_row;
                    const uint32_t live_keys = __ballot_sync(0xffffffffu, page >= 0);
                    const bool whole = a.box && live_keys == 0xffffffffu;
                    const int pg = page, rw = row;
                    if (i + 1 < seg.count) find(seg.begin + i + 1);
                    claim();
                    if (!ok) break;
                    // the ring's stages free the mask's place long before: see kLive
                    if (lane == 0) {
                        live[(unit % kLive) * 4 + quarter] = live_keys;
                        mbar_arrive(live_full + unit % kLive);
                    }
                    __syncwarp();
                    fill(a.k, k_map, whole, pg, rw, pk);
                    for (int half = 0; i == 0 && half * 128 < rows; ++half) {  // the tile's rows of q
                        if (!wait_bar(q_empty + half, q_phase[half] ^ 1, status)) {
                            ok = false;
                            break;
                        }
                        q_phase[half] ^= 1;
                        const uint32_t mine = at.rt * static_cast<uint32_t>(kTcRows) + half * 128 + quarter * 32 + (a.q_box ? 0 : lane);
                        const uint32_t group = a.group, qi = mine / group;
                        const int head = at.h * a.group + static_cast<int>(mine - qi * group);
                        if (a.q_box) {
                            if (lane == 0) expect_bytes(q_full + half, 32 * 128 * (D / 64));
                            __syncwarp();
                            if (lane < D / 64)
                                tma_box(base + half * R::kTile + lane * R::kHalf + quarter * 32 * 128, &q_map, lane * 64, head,
                                        static_cast<int>(a.offsets ? at.q.first + qi : qi), a.offsets ? 0 : static_cast<int>(at.q.first),
                                        q_full + half);
                            if (lane == 0) arrive_warp(q_full + half);
                        } else {
                            // a lane finds a row, as it does for keys
                            const T *q = static_cast<const T *>(a.q);
                            const int64_t place = half * 128 + quarter * 32 + lane < rows ? q_at(a, at.q, static_cast<int>(qi), head) : -1;
                            const uint32_t to = half * R::kTile + at_chunk;
#pragma unroll 4
                            for (int j = 0; j < 32 / kPass; ++j) {
                                const int rr = j * kPass + sub, r = quarter * 32 + rr;
                                const int64_t off = __shfl_sync(0xffffffffu, place, rr);
                                const bool there = off >= 0 && chunk * 8 < a.d;
                                const uint32_t dst = to + r * 128 + (((chunk & 7) ^ (r & 7)) * 16);
                                if (chunk >= chunks) continue;
                                if (a.q_vec) {
                                    copy16(base + dst, there ? q + off + chunk * 8 : q, there ? 16 : 0);
                                } else {  // zeros are stored as well: the arrival below does not wait for cp.async
                                    uint32_t w[4] = {0, 0, 0, 0};
                                    if (there) {
                                        const uint16_t *e = reinterpret_cast<const uint16_t *>(q + off + chunk * 8);
#pragma unroll
                                        for (int k = 0; k < 4; ++k) w[k] = e[2 * k] | static_cast<uint32_t>(e[2 * k + 1]) << 16;
                                    }
                                    *reinterpret_cast<uint4 *>(smem + dst) = make_uint4(w[0], w[1], w[2], w[3]);
                                }
                            }
                            __syncwarp();
                            if (a.q_vec) copy_arrive(q_full + half);
                            else mbar_arrive(q_full + half);
                        }
                        __syncwarp();
                    }
                    if (!ok) break;
                    claim();
                    if (!ok) break;
                    fill(a.v, v_map, whole, pg, rw, pv);
                }
                at.next_tile(a);
            }
            copy_commit();
            copy_wait<0>();
            if (!ok) {  // tiled copies still in flight land before the block may end
                for (int i = 0; i < min(uses, R::kStages); ++i) {
                    if (--st < 0) {
                        st = R::kStages - 1;
                        phase ^= 1;
                    }
                    wait_bar(full + st, phase, status);
                }
                if (uses > 0) wait_bar(q_full, q_phase[0] ^ 1, status);
                if (uses > 0) wait_bar(q_full + 1, q_phase[1] ^ 1, status);
            }
        } else if (warp < 14) {
            // ------------------------------------------------ MMAs: a warp a half, so that neither waits for the other's softmax
            constexpr uint32_t kFmt = std::is_same<T, __nv_bfloat16>::value ? 1u : 0u;
            const int half = warp - 12;
            const uint32_t types = (1u << 4) | (kFmt << 7) | (kFmt << 10) | (8u << 24);
            const uint32_t qk = types | (static_cast<uint32_t>(kTcUnit >> 3) << 17);
            const uint32_t pv = types | (1u << 16) | (static_cast<uint32_t>(width >> 3) << 17);  // values: MN-major
            const uint32_t base = smem_addr(smem), q_base = base + half * R::kTile;
            const uint32_t s_to = tmem + half * 128, p_from = tmem + R::kPAt + half * R::kPStep, o_to = tmem + R::kOAt + half * D;
            int st = 0, unit = 0;
            uint32_t phase = 0, q_phase = 0, unit_phase = 0;  // unit_phase: of this half's next weights
            bool first = true, both = false;  // no product of this half yet; the tile has rows in both
            auto wait_on = [&](uint64_t *bar, uint32_t parity) {
                if (!wait_bar(bar, parity, status)) ok = false;
                tc_fence_after();
                return ok;
            };
            auto wait_copy = [&](uint64_t *bar, uint32_t parity) {
                const bool there = wait_on(bar, parity);
                fence_proxy_async_smem();  // cp.async writes through the generic proxy
                return there;
            };
            auto advance = [&]() {
                if (++st == R::kStages) {
                    st = 0;
                    phase ^= 1;
                }
            };
            // S = Q K^T, once what lies in its place has been used: the weights, or within a tile the scores before (a tile's last
            // weights have been there when the next begins).
            auto scores = [&](bool within, bool there) {
                if (!there && !wait_copy(full + st, phase)) return false;
                if (R::kApart) {
                    if (within && !wait_on(s_read + half, unit_phase)) return false;
                } else {
                    if (!first && !wait_on(pv_done + half, unit_phase ^ 1)) return false;
                }
                if (!R::kApart && both) {
                    // Half a turn apart: while the one half's products run, the other's softmax does.  Nothing but time depends
                    // on it.
                    const long long t0 = clock64();
                    while (begun[half ^ 1] < unit + half && clock64() - t0 < 20000) __nanosleep(20);
                    __syncwarp();
                }
                ++unit;
                const uint32_t k = base + R::kRing + st * R::kTile;
                for (int i = 0; i < steps; ++i) {
                    const uint32_t off = (i >> 2) * R::kHalf + (i & 3) * 32;
                    mma_f16_ss_warp(s_to, swizzled(q_base + off, 16), swizzled(k + off, 16), qk, i > 0);
                }
                mma_commit_warp(s_full + half);
                mma_commit_warp(empty + st);
                advance();
                return true;
            };
            while (left > 0 && ok) {
                const bool mine = at.rows(a) > half * 128;
                both = at.rows(a) > 128;
                const Segment seg = take(at, left);
                if (seg.count > 0 && !mine) {  // no rows: the stages pass by
                    unit += seg.count;
                    for (int i = 0; i < 2 * seg.count && wait_copy(full + st, phase); ++i, advance()) {
                        if (lane == 0) mbar_arrive(empty + st);
                        __syncwarp();
                    }
                } else if (seg.count > 0) {
                    if (!wait_copy(q_full + half, q_phase)) break;
                    q_phase ^= 1;
                    if (!scores(false, false)) break;
                    first = false;
                    for (int i = 0; i < seg.count; ++i) {
                        const bool more = i + 1 < seg.count;
                        if (!more) mma_commit_warp(q_empty + half);
                        const int v_stage = st;
                        const uint32_t v_phase = phase, v = base + R::kRing + v_stage * R::kTile;
                        advance();
                        if (R::kApart && more && !scores(true, false)) break;
                        // the copies are there long before the weights; waiting for them after these would cost the fences' time
                        if (!wait_copy(full + v_stage, v_phase)) break;
                        if (!R::kApart && more && !wait_copy(full + st, phase)) break;
#pragma unroll
                        for (int c = 0; c < 2; ++c) {
                            if (!wait_on(p_full + 2 * half + c, unit_phase)) break;
#pragma unroll
                            for (int j = 4 * c; j < 4 * c + 4; ++j)
                                mma_f16_ts_warp(o_to, p_from + j * 8, swizzled(v + j * 2048, R::kHalf), pv, (i | j) > 0);
                        }
                        if (!ok) break;
                        mma_commit_warp(pv_done + half);
                        mma_commit_warp(empty + v_stage);
                        unit_phase ^= 1;
                        if (!R::kApart && more && !scores(true, true)) break;
                    }
                }
                at.next_tile(a);
            }
            // whatever was issued has ended before the tensor memory is given back
            mma_commit_warp(drained + half);
            wait_bar(drained + half, 0, status);
        }
    }
    __syncwarp();
    tc_fence_before();
    __syncthreads();
    if (warp == 12) {
        tc_fence_after();
        tmem_dealloc(tmem, 512);
    }
}

// Joins a tile that several blocks share, as the streaming kernel's parts are: block (b, 32 rows) does where b is the first
// block whose share begins inside the tile.  A lane a row, a warp an eighth of the columns.  (Short code: the launch runs it
// once, and fetching instructions takes most of the time.)
template <typename T, int D>
__global__ void __launch_bounds__(256) join_tc_kernel(const AttnArgs a, const int blocks)
{
    constexpr int kCols = D / 8;
    const int b = blockIdx.x + 1, lane = threadIdx.x & 31, col = (threadIdx.x >> 5) * kCols;
    pdl_begin();
    const TcParts space = tc_parts<D>(a.tc_part, blocks);
    const TcRecord rec = space.records[b];
    const int64_t before = space.records[b - 1].x0;
    if (rec.total == 0 || rec.x0 <= rec.u0 || rec.x0 >= rec.u1 || before > rec.u0) return;
    const Sequence q = sequence(a, rec.s);
    const int left = q.n * a.group - rec.rt * kTcRows, rows = left < kTcRows ? left : kTcRows, r = blockIdx.y * 32 + lane;
    if (r >= rows || col >= a.d) return;
    // parts of blocks c0 .. end - 1; with fewer units than blocks, those between that have a share
    const int c0 = b - 1, end = static_cast<int>((rec.u1 * blocks + rec.total - 1) / rec.total);
    const bool sparse = rec.total < blocks;
    float most = -INFINITY, sum = 0.f, o[kCols];
#pragma unroll
    for (int j = 0; j < kCols; ++j) o[j] = 0.f;
    auto add = [&](int c) {
        const int64_t slot = 2 * c + (c == c0 ? 1 : 0);
        const float *stat = space.stats + slot * (2 * kTcRows) + r, *p = space.sums + (slot * D + col) * kTcRows + r;
        float v[kCols];
#pragma unroll
        for (int j = 0; j < kCols; ++j) v[j] = p[j * kTcRows];
        const float m = stat[0], l = stat[kTcRows];
        const float raised = fmaxf(most, m), ref = raised == -INFINITY ? 0.f : raised;
        const float f = exp2_fast(most - ref), w = exp2_fast(m - ref);
        most = raised;
        sum = sum * f + l * w;
#pragma unroll
        for (int j = 0; j < kCols; ++j) o[j] = o[j] * f + v[j] * w;
    };
    if (sparse) {
#pragma unroll 1
        for (int c = c0; c < end; ++c)
            if (rec.total * (c + 1) / blocks > rec.total * c / blocks) add(c);
    } else {
        int c = c0;
#pragma unroll 1
        for (; c + 4 <= end; c += 4) {  // four at a time: the loads do not wait for one another
#pragma unroll
            for (int i = 0; i < 4; ++i) add(c + i);
        }
#pragma unroll 1
        for (; c < end; ++c) add(c);
    }
    const uint32_t row = rec.rt * static_cast<uint32_t>(kTcRows) + r, group = a.group;
    const int qi = static_cast<int>(row / group), head = rec.h * a.group + static_cast<int>(row - qi * group);
    const float inv = sum == 0.f ? 0.f : 1.f / sum;
    T *y = static_cast<T *>(a.out) + o_at(a, q, qi, head) + col;
#pragma unroll
    for (int j = 0; j < kCols; j += 8) {
        if (col + j >= a.d) break;
        if (a.out_vec8) {
            *reinterpret_cast<uint4 *>(y + j) = make_uint4(pack2<T>(o[j] * inv, o[j + 1] * inv), pack2<T>(o[j + 2] * inv, o[j + 3] * inv),
                                                           pack2<T>(o[j + 4] * inv, o[j + 5] * inv), pack2<T>(o[j + 6] * inv, o[j + 7] * inv));
        } else {
#pragma unroll
            for (int i = 0; i < 8; ++i) y[j + i] = from_f32<T>(o[j + i] * inv);
        }
    }
    if (a.lse && col == 0) a.lse[lse_at(a, q, qi, head)] = sum == 0.f ? -INFINITY : kLn2 * most + logf(sum);
}

int padded(int d) { return d <= 64 ? 64 : 128; }

// A map of (elements, y, z, w), boxes of 64 x rows x tall elements; false where none can be made.
template <typename T>
bool map_of(CUtensorMap *map, const void *p, const int64_t (&size)[4], const int64_t (&step)[3], int rows, int tall)
{
    const EncodeTiled encode = encode_tiled();
    if (!encode || !p || reinterpret_cast<uintptr_t>(p) % 16) return false;
    cuuint64_t dims[4], strides[3];
    for (int i = 0; i < 4; ++i) {
        if (size[i] <= 0) return false;
        dims[i] = static_cast<cuuint64_t>(size[i]);
    }
    for (int i = 0; i < 3; ++i) {
        const int64_t bytes = size[i + 1] == 1 ? 16 : step[i] * 2;
        if (bytes <= 0 || bytes % 16 || bytes >= INT64_C(1) << 40) return false;
        strides[i] = static_cast<cuuint64_t>(bytes);
    }
    const cuuint32_t box[4] = {64, static_cast<cuuint32_t>(rows), static_cast<cuuint32_t>(tall), 1}, unit[4] = {1, 1, 1, 1};
    return encode(map, std::is_same<T, __half>::value ? CU_TENSOR_MAP_DATA_TYPE_FLOAT16 : CU_TENSOR_MAP_DATA_TYPE_BFLOAT16, 4,
                  const_cast<void *>(p), dims, strides, box, unit, CU_TENSOR_MAP_INTERLEAVE_NONE, CU_TENSOR_MAP_SWIZZLE_128B,
                  CU_TENSOR_MAP_L2_PROMOTION_L2_256B, CU_TENSOR_MAP_FLOAT_OOB_FILL_NONE) == CUDA_SUCCESS;
}

template <typename T, int D>
cudaError_t launch(AttnArgs a, cudaStream_t st)
{
    using R = TcRing<D>;
    int *status = device_status_ptr();
    if (!status) return cudaErrorNotSupported;
    cudaError_t e = raise_smem<attention_tc_kernel<T, D>>(R::kSmem);
    if (e != cudaSuccess) return e;
    // Tiled copies take 32 rows of a page, or 16, where pages hold a multiple of that (or a sequence has one page); smaller
    // ones would take as long to issue as cp.async.
    CUtensorMap q_map = {}, k_map = {}, v_map = {};
    a.box = !a.table || a.page_size % 32 == 0 ? 32 : (a.page_size % 16 == 0 ? 16 : 0);
    const int64_t size[4] = {a.d, a.page_size, a.kv_heads, a.pages};
    if (a.box && (!map_of<T>(&k_map, a.k, size, {a.k_row, a.k_head, a.k_page}, a.box, 1) ||
                  !map_of<T>(&v_map, a.v, size, {a.v_row, a.v_head, a.v_page}, a.box, 1)))
        a.box = 0;
    // 32 rows of q are whole tokens' heads, or a part of one's
    a.q_box = 32 % a.group == 0 || a.group % 32 == 0 ? 32 : 0;
    const int64_t q_size[4] = {a.d, a.heads, a.offsets ? a.t : a.each, a.offsets ? 1 : a.seqs};
    if (a.q_box && !map_of<T>(&q_map, a.q, q_size, {a.hq, a.ldq, a.q_seq}, a.group < 32 ? a.group : 32, a.group < 32 ? 32 / a.group : 1))
        a.q_box = 0;
    const int blocks = device_sm_count();
    e = launch_pdl(attention_tc_kernel<T, D>, dim3(blocks), kTcThreads, R::kSmem, st, 1, q_map, k_map, v_map, a, status);
    // nothing is shared where every tile is one unit
    if (e != cudaSuccess || blocks < 2 || static_cast<int64_t>(a.width) * a.page_size <= kTcUnit) return e;
    const int64_t rows = (a.offsets ? a.t : a.each) * static_cast<int64_t>(a.group);
    return launch_pdl(join_tc_kernel<T, D>, dim3(blocks - 1, static_cast<unsigned>(rows < kTcRows ? (rows + 31) / 32 : kTcRows / 32)), 256, 0, st,
                      1, a, blocks);
}

}  // namespace

size_t attention_tc_workspace(int d)
{
    const size_t blocks = device_sm_count();
    return 2 * blocks * kTcRows * (padded(d) + 2) * sizeof(float) + blocks * sizeof(TcRecord);
}

cudaError_t launch_attention_tc(const AttnArgs &a, int dtype, cudaStream_t st)
{
    if (a.t == 0 || a.seqs == 0) return cudaSuccess;
    if (a.d <= 64) return dtype == QNN_F16 ? launch<__half, 64>(a, st) : launch<__nv_bfloat16, 64>(a, st);
    return dtype == QNN_F16 ? launch<__half, 128>(a, st) : launch<__nv_bfloat16, 128>(a, st);
}

}  // namespace qnn
