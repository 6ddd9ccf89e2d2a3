// Attention of few rows over a cache: keys and values are streamed once, whatever page they lie in.
//
// The work is the sequences' keys in units of 64 (128 for heads of 64 and less), for every key head (and every 16 rows, where
// a sequence has more), one after another; every block takes an even share of all units, so short and long sequences mix
// without idle SMs and one long sequence occupies them all.  Units of one (sequence, key head) that fall to several blocks leave a part each (the
// sum of 2^(z - m) v, m and the sum of 2^(z - m)) in the workspace, and a second launch joins them in order, so the result
// does not depend on which block was first.
//
// A block is four warps.  Each warp takes a quarter of a unit's keys: S = Q K^T on the m16n8k16 MMA with the rows on the M side,
// the running maximum of all four warps through shared memory; then each warp takes a quarter of the head's columns over
// all keys, so a block holds one accumulator and not four that had to be added.  Keys and values come by cp.async, 16
// bytes a lane, several units ahead and across the borders of sequences; keys that the cache does not have (past the
// length, in no page) are filled with zeros, whatever lies there, and masked.  Rows of 128 bytes and more are stored with
// 16-byte chunk c of row r at c ^ (r & 7): no bank conflicts for ldmatrix.
// P is rounded to the element type for the second MMA (off by half a step at most, 2^-8 of it for bf16, as the values are);
// the sum of P, the maximum and the accumulator are 32-bit.
// Bound by HBM over long caches: 64 users with up to 24575 keys each, 8 key heads of 128, pages of 16: 545 us, 5.7 TB/s (0.84
// of a copy's).  Short sequences with a key head for each query head are bound by a pair's own work, some 8 us a block: 200
// windows of 256 keys, 16 heads of 64, 83 us (2.2 TB/s).  One user over 8191 keys 13 us, and the join 7.
// Heads above 128 elements come here with any number of rows.  Every 16 rows go over the keys that any query of their sequence
// sees, so neither a prompt's causal half nor a window shorter than it saves work there: 4096 tokens, 16 on 4 heads of 256, take
// 2.66 ms with and without a window of 1024 (products alone 31 and 71 us); 64 * 1 tokens over 8192 keys 365 us (0.87 of a
// copy's rate).
#include "attention.cuh"

namespace qnn {
namespace {

constexpr int kRowsThreads = 128;
// Keys of a unit: 32 KB of keys and values up to heads of 128, so that a unit's barriers weigh alike.  (Heads of 64, units of
// 128 keys, two blocks an SM: 57 us for 32 * 20 heads over 1500 keys, one query each; units of 64 and six stages 68, three
// blocks with four stages 85.)
constexpr int rows_unit(int d) { return d <= 64 ? 128 : 64; }
constexpr int rows_per_sm(int d) { return d <= 128 ? 2 : 1; }  // blocks: as registers and shared memory allow

template <int D>
struct RowsRing {
    static constexpr int kUnit = rows_unit(D), kStages = 3, kPerSm = rows_per_sm(D);
    static constexpr uint32_t kRow = D * 2, kTile = kUnit * kRow, kQ = 16 * kRow, kStage = 2 * kTile + kQ;
    static constexpr uint32_t kP = kStages * kStage, kPRow = kUnit * 2, kSmem = kP + 16 * kPRow;
};

// Of a block: where its first unit lies.  total 0: nothing was queued.
struct PartRecord {
    int64_t x0, u0, u1, total;  // first unit; units of the pair that holds the block's first unit; all units
    int s, h, rt, pad;
};

struct PartSpace {
    float *sums, *stats;    // [2 * blocks][16][D], [2 * blocks][32]: m, then l
    PartRecord *records;    // [blocks]
};

template <int D>
__host__ __device__ inline PartSpace part_space(float *p, int blocks)
{
    PartSpace s;
    s.sums = p;
    s.stats = p + static_cast<int64_t>(2 * blocks) * 16 * D;
    s.records = reinterpret_cast<PartRecord *>(s.stats + 2 * blocks * 32);
    return s;
}

// The units of a sequence: 64-key units of a pair (at least one, so that empty rows are written), row tiles.
struct SeqUnits {
    int units, tiles, first;  // first: unit number of the oldest key that any query sees
    int lo, hi;
};

template <int kUnit>
__device__ __forceinline__ SeqUnits seq_units(const AttnArgs &a, const Sequence &q)
{
    SeqUnits u = {0, 0, 0, 0, 0};
    const int64_t rows = static_cast<int64_t>(q.n) * a.group;
    if (q.n <= 0 || rows > a.few) return u;
    int lo, hi, l2, h2;
    keys_of(a, q, 0, lo, hi);
    keys_of(a, q, q.n - 1, l2, h2);
    u.lo = lo;
    u.hi = h2 > hi ? h2 : hi;
    u.first = lo / kUnit;
    u.units = (u.hi + kUnit - 1) / kUnit - u.first;
    if (u.units < 1) u.units = 1;
    u.tiles = static_cast<int>((rows + 15) / 16);
    return u;
}

// A place in the order of units.
template <int kUnit>
struct Cursor {
    Sequence q;
    SeqUnits w;
    int s, rt, h, u;

    __device__ __forceinline__ void open(const AttnArgs &a)
    {
        q = sequence(a, s);
        w = seq_units<kUnit>(a, q);
    }
    __device__ __forceinline__ void next(const AttnArgs &a)
    {
        if (++u < w.units) return;
        u = 0;
        if (++h < a.kv_heads) return;
        h = 0;
        if (++rt < w.tiles) return;
        rt = 0;
        do {
            if (++s >= a.seqs) return;
            open(a);
        } while (w.tiles == 0);
    }
};

template <typename T, int D>
__global__ void __launch_bounds__(kRowsThreads, RowsRing<D>::kPerSm) attention_rows_kernel(const AttnArgs a)
{
    using R = RowsRing<D>;
    constexpr int kUnit = R::kUnit, kKeys = kUnit / 4;  // of a unit, of a warp
    constexpr int kChunks = D / 8, kSteps = D / 16, kCols = D / 4, kBlocks = kCols / 8;
    extern __shared__ __align__(1024) uint8_t smem[];
    __shared__ int64_t scratch[kRowsThreads / 32];
    __shared__ int64_t start_first;
    __shared__ int start_seq;
    __shared__ float wmax[4][16], wsum[4][16];
    __shared__ uint32_t vmask[R::kStages][4];
    const int tid = threadIdx.x, lane = tid & 31, warp = tid >> 5, g = lane >> 2, t4 = lane & 3;
    const int blocks = gridDim.x;
    const uint32_t base = smem_addr(smem);
    pdl_begin();

    // all units, and where this block's share begins
    int64_t mine = 0, total = 0;
    for (int s = tid; s < a.seqs; s += kRowsThreads) {
        const SeqUnits w = seq_units<kUnit>(a, sequence(a, s));
        mine += static_cast<int64_t>(w.units) * w.tiles * a.kv_heads;
    }
    block_scan<kRowsThreads>(mine, scratch, total);
    const int64_t x0 = total * blockIdx.x / blocks, x1 = total * (blockIdx.x + 1) / blocks;
    const PartSpace space = part_space<D>(a.part, blocks);
    if (total == 0) {
        if (tid == 0 && a.part) space.records[blockIdx.x].total = 0;
        return;
    }
    if (tid == 0) start_seq = 0;
    int64_t carry = 0;
    for (int s0 = 0; s0 < a.seqs; s0 += kRowsThreads) {
        const int s = s0 + tid;
        int64_t n = 0, all;
        if (s < a.seqs) {
            const SeqUnits w = seq_units<kUnit>(a, sequence(a, s));
            n = static_cast<int64_t>(w.units) * w.tiles * a.kv_heads;
        }
        const int64_t before = carry + block_scan<kRowsThreads>(n, scratch, all);
        if (n > 0 && before <= x0 && x0 < before + n) {
            start_seq = s;
            start_first = before;
        }
        carry += all;
        if (carry > x0) break;
    }
    __syncthreads();

    Cursor<kUnit> load;
    load.s = start_seq;
    load.open(a);
    {
        const int64_t in = x0 - start_first;
        const int pair = static_cast<int>(in / load.w.units);
        load.u = static_cast<int>(in - static_cast<int64_t>(pair) * load.w.units);
        load.rt = pair / a.kv_heads;
        load.h = pair - load.rt * a.kv_heads;
        if (tid == 0 && a.part) {
            PartRecord &r = space.records[blockIdx.x];
            r.x0 = x0;
            r.u0 = x0 - load.u;
            r.u1 = r.u0 + load.w.units;
            r.total = total;
            r.s = load.s;
            r.h = load.h;
            r.rt = load.rt;
        }
    }
    Cursor<kUnit> at = load;
    int64_t left = x1 - x0, to_load = left;

    // Where the warp's keys and values lie: a lane knows kKeys / 16 of the 32 or 64 offsets (keys, then values); -1 for none.
    constexpr int kPlaces = kKeys / 16;
    int64_t place[kPlaces];
    auto find = [&]() {  // of the load cursor's unit
#pragma unroll
        for (int i = 0; i < kPlaces; ++i) {
            const bool of_k = kPlaces == 1 ? lane < 16 : i == 0;
            const int key = (load.w.first + load.u) * kUnit + warp * kKeys + (kPlaces == 1 ? lane & 15 : lane);
            place[i] = -1;
            if (key >= load.w.lo && key < load.w.hi) {
                const int column = key / a.page_size, row = key - column * a.page_size;
                const int page = page_of(a, load.s, column);
                if (page >= 0)
                    place[i] = of_k ? page * a.k_page + load.h * a.k_head + row * a.k_row : page * a.v_page + load.h * a.v_head + row * a.v_row;
            }
        }
    };
    bool opened = true;  // the unit to load is the block's first of its pair
    auto fetch = [&](int stage) {
        const uint32_t to = base + stage * R::kStage;
        const uint32_t live = __ballot_sync(0xffffffffu, place[0] >= 0);
        if (lane == 0) vmask[stage][warp] = kKeys == 16 ? live & 0xffff : live;
        constexpr int kPass = 32 / (kChunks < 32 ? kChunks : 32);  // rows a pass
        const int chunk = lane % kChunks, sub = lane / kChunks;
#pragma unroll
        for (int kv = 0; kv < 2; ++kv)
#pragma unroll
            for (int i = 0; i < kKeys / kPass; ++i) {
                const int r = i * kPass + sub;
                const int64_t off = __shfl_sync(0xffffffffu, place[kPlaces == 1 ? 0 : kv], kPlaces == 1 ? kv * 16 + r : r);
                const T *p = static_cast<const T *>(kv ? a.v : a.k);
                const bool ok = off >= 0 && chunk * 8 < a.d;
                const int row = warp * kKeys + r;
                copy16(to + kv * R::kTile + row * R::kRow + ((chunk ^ (row & 7)) * 16), ok ? p + off + chunk * 8 : p, ok ? 16 : 0);
            }
        if (opened) {  // the pair's rows of q, beside its first keys
            const int rows = min(16, load.q.n * a.group - load.rt * 16);
            for (int i = tid; i < 16 * kChunks; i += kRowsThreads) {
                const int r = i / kChunks, c = i % kChunks, row = load.rt * 16 + r, qi = row / a.group;
                const bool ok = r < rows && c * 8 < a.d;
                const T *p = static_cast<const T *>(a.q);
                if (ok) p += q_at(a, load.q, qi, load.h * a.group + row - qi * a.group) + c * 8;
                const uint32_t dst = to + 2 * R::kTile + r * R::kRow + ((c ^ (r & 7)) * 16);
                if (a.q_vec || !ok) {
                    copy16(dst, p, ok ? 16 : 0);
                } else {
                    const uint16_t *e = reinterpret_cast<const uint16_t *>(p);
                    uint4 v;
                    v.x = e[0] | static_cast<uint32_t>(e[1]) << 16;
                    v.y = e[2] | static_cast<uint32_t>(e[3]) << 16;
                    v.z = e[4] | static_cast<uint32_t>(e[5]) << 16;
                    v.w = e[6] | static_cast<uint32_t>(e[7]) << 16;
                    *reinterpret_cast<uint4 *>(smem + (dst - base)) = v;
                }
            }
        }
    };
    auto fetch_next = [&](int stage) {
        if (to_load > 0) {
            fetch(stage);
            if (--to_load > 0) {
                load.next(a);
                opened = load.u == 0;
                find();
            }
        }
        copy_commit();
    };
    if (left > 0) find();
#pragma unroll
    for (int i = 0; i < R::kStages - 1; ++i) fetch_next(i);

    uint32_t aq[kSteps][4];
    float o[kBlocks][4], m[2], l[2];
    int lo[2], hi[2], lo_most = 0, hi_least = 0;
    bool first = true;      // the unit is the block's first of its pair
    bool whole = at.u == 0; // ... and the pair's first
    int stage = 0;
    for (; left > 0; --left) {
        copy_wait<R::kStages - 2>();
        __syncthreads();
        fetch_next(stage == 0 ? R::kStages - 1 : stage - 1);
        const uint32_t from = base + stage * R::kStage;
        if (first) {
#pragma unroll
            for (int k = 0; k < kSteps; ++k) {
                const int r = (lane & 7) + ((lane >> 3) & 1) * 8, c = 2 * k + (lane >> 4);
                ldsm4(aq[k], from + 2 * R::kTile + r * R::kRow + ((c ^ (r & 7)) * 16));
            }
#pragma unroll
            for (int n = 0; n < kBlocks; ++n)
#pragma unroll
                for (int i = 0; i < 4; ++i) o[n][i] = 0.f;
#pragma unroll
            for (int i = 0; i < 2; ++i) {
                m[i] = -INFINITY;
                l[i] = 0.f;
                const int row = at.rt * 16 + g + 8 * i, qi = row / a.group;
                lo[i] = hi[i] = 0;
                if (qi < at.q.n) keys_of(a, at.q, qi, lo[i], hi[i]);
            }
            // keys that every row sees: from the last query's first to the first query's last
            const int q0 = at.rt * 16 / a.group, q1 = min(at.q.n - 1, (at.rt * 16 + 15) / a.group);
            int x, y;
            keys_of(a, at.q, q0, x, hi_least);
            keys_of(a, at.q, q1, lo_most, y);
        }
        // scores of this warp's keys
        constexpr int kZ = kKeys / 8;
        const int key0 = (at.w.first + at.u) * kUnit + warp * kKeys;
        float z[kZ][4];
#pragma unroll
        for (int n = 0; n < kZ; ++n)
#pragma unroll
            for (int i = 0; i < 4; ++i) z[n][i] = 0.f;
#pragma unroll
        for (int k = 0; k < kSteps; ++k)
#pragma unroll
            for (int n = 0; n < kZ; n += 2) {
                uint32_t b[4];
                const int r = warp * kKeys + n * 8 + (lane & 7) + ((lane >> 4) << 3), c = 2 * k + ((lane >> 3) & 1);
                ldsm4(b, from + r * R::kRow + ((c ^ (r & 7)) * 16));
                mma16816<T>(z[n], aq[k], b[0], b[1]);
                mma16816<T>(z[n + 1], aq[k], b[2], b[3]);
            }
        const uint32_t live = vmask[stage][warp];
        const bool clear = live == (kKeys == 16 ? 0xffffu : 0xffffffffu) && key0 >= lo_most && key0 + kKeys <= hi_least;
        float top[2] = {-INFINITY, -INFINITY};
#pragma unroll
        for (int n = 0; n < kZ; ++n)
#pragma unroll
            for (int i = 0; i < 4; ++i) {
                const int col = n * 8 + t4 * 2 + (i & 1), key = key0 + col;
                const bool ok = clear || (key >= lo[i >> 1] && key < hi[i >> 1] && (live >> col & 1));
                z[n][i] = ok ? z[n][i] * a.scale : -INFINITY;
                top[i >> 1] = fmaxf(top[i >> 1], z[n][i]);
            }
#pragma unroll
        for (int i = 0; i < 2; ++i) {
            top[i] = fmaxf(top[i], __shfl_xor_sync(0xffffffffu, top[i], 1));
            top[i] = fmaxf(top[i], __shfl_xor_sync(0xffffffffu, top[i], 2));
            if (t4 == 0) wmax[warp][g + 8 * i] = top[i];
        }
        __syncthreads();
        bool moved = false;
        float factor[2], at_m[2];
#pragma unroll
        for (int i = 0; i < 2; ++i) {
            const int r = g + 8 * i;
            const float most = fmaxf(fmaxf(fmaxf(wmax[0][r], wmax[1][r]), fmaxf(wmax[2][r], wmax[3][r])), m[i]);
            at_m[i] = most == -INFINITY ? 0.f : most;
            factor[i] = exp2_fast(m[i] - at_m[i]);
            moved = moved || most != m[i];
            m[i] = most;
            l[i] *= factor[i];
        }
        if (__any_sync(0xffffffffu, moved)) {
#pragma unroll
            for (int n = 0; n < kBlocks; ++n)
#pragma unroll
                for (int i = 0; i < 4; ++i) o[n][i] *= factor[i >> 1];
        }
        const uint32_t sp = base + R::kP;
#pragma unroll
        for (int n = 0; n < kZ; ++n)
#pragma unroll
            for (int i = 0; i < 2; ++i) {
                const float p0 = exp2_fast(z[n][2 * i] - at_m[i]), p1 = exp2_fast(z[n][2 * i + 1] - at_m[i]);
                l[i] += p0 + p1;
                const int r = g + 8 * i;
                *reinterpret_cast<uint32_t *>(smem + R::kP + r * R::kPRow + (((warp * kZ + n) ^ (r & 7)) * 16) + t4 * 4) = pack2<T>(p0, p1);
            }
        __syncthreads();
        // this warp's columns over all keys
#pragma unroll
        for (int k = 0; k < kUnit / 16; ++k) {
            uint32_t ap[4];
            const int pr = (lane & 7) + ((lane >> 3) & 1) * 8, pc = 2 * k + (lane >> 4);
            ldsm4(ap, sp + pr * R::kPRow + ((pc ^ (pr & 7)) * 16));
            const int r = k * 16 + (lane & 7) + ((lane >> 3) & 1) * 8;
#pragma unroll
            for (int n = 0; n < kBlocks; n += 2) {
                uint32_t b[4];
                const int c = warp * kBlocks + n + (lane >> 4);
                ldsm4_trans(b, from + R::kTile + r * R::kRow + ((c ^ (r & 7)) * 16));
                mma16816<T>(o[n], ap, b[0], b[1]);
                mma16816<T>(o[n + 1], ap, b[2], b[3]);
            }
        }
        first = false;
        const bool last = at.u + 1 == at.w.units;
        if (last || left == 1) {
            // sums of all warps
#pragma unroll
            for (int i = 0; i < 2; ++i) {
                l[i] += __shfl_xor_sync(0xffffffffu, l[i], 1);
                l[i] += __shfl_xor_sync(0xffffffffu, l[i], 2);
                if (t4 == 0) wsum[warp][g + 8 * i] = l[i];
            }
            __syncthreads();
            const bool complete = whole && last;
            // first slot: the pair began before this block's share; second: it goes on after it
            const int slot = 2 * blockIdx.x + (whole ? 1 : 0);
#pragma unroll
            for (int i = 0; i < 2; ++i) {
                const int r = g + 8 * i, row = at.rt * 16 + r, qi = row / a.group;
                if (qi >= at.q.n) continue;
                const int head = at.h * a.group + row - qi * a.group;
                const float sum = wsum[0][r] + wsum[1][r] + wsum[2][r] + wsum[3][r];
                if (complete) {
                    const float inv = sum == 0.f ? 0.f : 1.f / sum;
                    T *y = static_cast<T *>(a.out) + o_at(a, at.q, qi, head);
#pragma unroll
                    for (int n = 0; n < kBlocks; ++n) {
                        const int col = warp * kCols + n * 8 + t4 * 2;
                        if (col < a.d) {
                            const float v0 = o[n][2 * i] * inv, v1 = o[n][2 * i + 1] * inv;
                            if (a.out_vec) {
                                *reinterpret_cast<uint32_t *>(y + col) = pack2<T>(v0, v1);
                            } else {
                                y[col] = from_f32<T>(v0);
                                y[col + 1] = from_f32<T>(v1);
                            }
                        }
                    }
                    if (a.lse && warp == 0 && t4 == 0)
                        a.lse[lse_at(a, at.q, qi, head)] = sum == 0.f ? -INFINITY : kLn2 * m[i] + logf(sum);
                } else {
                    float *y = space.sums + (static_cast<int64_t>(slot) * 16 + r) * D;
#pragma unroll
                    for (int n = 0; n < kBlocks; ++n)
                        *reinterpret_cast<float2 *>(y + warp * kCols + n * 8 + t4 * 2) = make_float2(o[n][2 * i], o[n][2 * i + 1]);
                    if (warp == 0 && t4 == 0) {
                        space.stats[slot * 32 + r] = m[i];
                        space.stats[slot * 32 + 16 + r] = sum;
                    }
                }
            }
            first = true;
            whole = true;
        }
        at.next(a);
        if (++stage == R::kStages) stage = 0;
    }
}

// Joins a pair that several blocks share: block (b, row) does where b is the first block whose share begins inside the pair.
// The block before it, where the pair begins, left its part in its second slot, the others in their first.
constexpr int kJoinWarps = 8;
template <typename T, int D>
__global__ void __launch_bounds__(32 * kJoinWarps) join_rows_kernel(const AttnArgs a, const int blocks)
{
    constexpr int kVec = D / 32;
    __shared__ float part_max[kJoinWarps], part_sum[kJoinWarps], part_o[kJoinWarps][D];
    const int b = blockIdx.x + 1, r = blockIdx.y, lane = threadIdx.x & 31, warp = threadIdx.x >> 5;
    pdl_begin();
    const PartSpace space = part_space<D>(a.part, blocks);
    const PartRecord rec = space.records[b];
    const int64_t before = space.records[b - 1].x0;
    if (rec.total == 0 || rec.x0 <= rec.u0 || rec.x0 >= rec.u1 || before > rec.u0) return;
    const Sequence q = sequence(a, rec.s);
    const int row = rec.rt * 16 + r, qi = row / a.group;
    if (qi >= q.n) return;
    const int head = rec.h * a.group + row - qi * a.group;
    // parts of blocks c0 .. end - 1; with fewer units than blocks, those between that have a share
    const int c0 = b - 1, end = static_cast<int>((rec.u1 * blocks + rec.total - 1) / rec.total);
    const bool sparse = rec.total < blocks;
    auto none = [&](int c) { return sparse && rec.total * (c + 1) / blocks <= rec.total * c / blocks; };
    auto slot_of = [&](int c) { return 2 * c + (c == c0 ? 1 : 0); };
    float most = -INFINITY;
    for (int c = c0 + threadIdx.x; c < end; c += 32 * kJoinWarps)
        if (!none(c)) most = fmaxf(most, space.stats[slot_of(c) * 32 + r]);
#pragma unroll
    for (int d = 16; d; d >>= 1) most = fmaxf(most, __shfl_xor_sync(0xffffffffu, most, d));
    if (lane == 0) part_max[warp] = most;
    __syncthreads();
#pragma unroll
    for (int w = 0; w < kJoinWarps; ++w) most = fmaxf(most, part_max[w]);
    const float ref = most == -INFINITY ? 0.f : most;
    float sum = 0.f, o[kVec];
#pragma unroll
    for (int i = 0; i < kVec; ++i) o[i] = 0.f;
#pragma unroll 4
    for (int c = c0 + warp; c < end; c += kJoinWarps) {
        if (none(c)) continue;
        const int slot = slot_of(c);
        const float w = exp2_fast(space.stats[slot * 32 + r] - ref);
        sum += w * space.stats[slot * 32 + 16 + r];
        const float *p = space.sums + (static_cast<int64_t>(slot) * 16 + r) * D + lane;
#pragma unroll
        for (int i = 0; i < kVec; ++i) o[i] += w * p[32 * i];
    }
#pragma unroll
    for (int i = 0; i < kVec; ++i) part_o[warp][lane + 32 * i] = o[i];
    if (lane == 0) part_sum[warp] = sum;
    __syncthreads();
    sum = 0.f;
#pragma unroll
    for (int w = 0; w < kJoinWarps; ++w) sum += part_sum[w];
    const float inv = sum == 0.f ? 0.f : 1.f / sum;
    T *y = static_cast<T *>(a.out) + o_at(a, q, qi, head);
    for (int c = threadIdx.x; c < a.d; c += 32 * kJoinWarps) {
        float v = 0.f;
#pragma unroll
        for (int w = 0; w < kJoinWarps; ++w) v += part_o[w][c];
        y[c] = from_f32<T>(v * inv);
    }
    if (a.lse && threadIdx.x == 0) a.lse[lse_at(a, q, qi, head)] = sum == 0.f ? -INFINITY : kLn2 * most + logf(sum);
}

int padded(int d) { return d <= 64 ? 64 : (d <= 128 ? 128 : 256); }

template <typename T, int D>
cudaError_t launch(const AttnArgs &a, cudaStream_t st)
{
    using R = RowsRing<D>;
    cudaError_t e = raise_smem<attention_rows_kernel<T, D>>(R::kSmem);
    if (e != cudaSuccess) return e;
    const int blocks = attention_rows_blocks(a.d);
    e = launch_pdl(attention_rows_kernel<T, D>, dim3(blocks), kRowsThreads, R::kSmem, st, 1, a);
    if (e != cudaSuccess || blocks < 2) return e;
    // nothing is shared where every pair is one unit
    const int64_t rows = (a.offsets ? a.t : a.each) * static_cast<int64_t>(a.group);
    if (static_cast<int64_t>(a.width) * a.page_size <= R::kUnit) return cudaSuccess;
    return launch_pdl(join_rows_kernel<T, D>, dim3(blocks - 1, static_cast<unsigned>(rows < 16 ? rows : 16)), 32 * kJoinWarps, 0, st, 1, a, blocks);
}

template <typename T>
cudaError_t launch_d(const AttnArgs &a, cudaStream_t st)
{
    switch (padded(a.d)) {
        case 64: return launch<T, 64>(a, st);
        case 128: return launch<T, 128>(a, st);
        default: return launch<T, 256>(a, st);
    }
}

}  // namespace

int attention_rows_blocks(int d) { return device_sm_count() * rows_per_sm(d); }

size_t attention_rows_workspace(int d)
{
    const size_t blocks = attention_rows_blocks(d);
    return 2 * blocks * (16 * padded(d) + 32) * sizeof(float) + blocks * sizeof(PartRecord);
}

cudaError_t launch_attention_rows(const AttnArgs &a, int dtype, cudaStream_t st)
{
    if (a.t == 0 || a.seqs == 0) return cudaSuccess;
    return dtype == QNN_F16 ? launch_d<__half>(a, st) : launch_d<__nv_bfloat16>(a, st);
}

}  // namespace qnn
