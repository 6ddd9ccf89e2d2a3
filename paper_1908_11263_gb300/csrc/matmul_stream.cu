// Matrix product for few rows of x: the weights are streamed once, straight into the fragments of mma.sync.
//
// A unit of work is 32 image rows against a tile of NT rows of x (8, 16 or 32).  Resident blocks share the units evenly,
// each a contiguous run of them (rows first, then tiles, experts one after another; the number of live tiles is known
// only on the device).  The warps of a block split K, and their partial sums are added in shared memory in a fixed order;
// where K is short, sets of four or two warps take units of their own, so that a warp has several blocks of a unit between
// its ends.
// Every warp copies its own blocks of the image (cp.async, whole lines) into a ring of its own, several blocks ahead and
// across the ends of units: no registers hold loads in flight and no barrier of the block stands between a copy and its
// use.  A lane's vector of packed codes is its A fragment; 32 bytes of a row of x are its B fragment.  The product is
// bound by the weight bytes or, for the narrow codes, by the instructions that expand them, not by the tensor cores:
// 1 x 8192 x 8192 takes 23 us with 16-bit weights (5.8 TB/s), 18 INT-8, 13 INT-4 and INT-2.
// Where units fill less than half of the blocks, a cluster of blocks takes one unit and splits its K further: the others
// write their sums into the first one's shared memory, which adds them in the order of the ranks.
#include <algorithm>

#include "matmul.cuh"

namespace qnn {
namespace {

constexpr int kStreamWarps = 8;

template <typename T>
__device__ __forceinline__ void mma16816(float (&c)[4], const uint32_t (&a)[4], uint32_t b0, uint32_t b1);
template <>
__device__ __forceinline__ void mma16816<__half>(float (&c)[4], const uint32_t (&a)[4], uint32_t b0, uint32_t b1)
{
    asm("mma.sync.aligned.m16n8k16.row.col.f32.f16.f16.f32 {%0,%1,%2,%3}, {%4,%5,%6,%7}, {%8,%9}, {%0,%1,%2,%3};"
                 : "+f"(c[0]), "+f"(c[1]), "+f"(c[2]), "+f"(c[3])
                 : "r"(a[0]), "r"(a[1]), "r"(a[2]), "r"(a[3]), "r"(b0), "r"(b1));
}
template <>
__device__ __forceinline__ void mma16816<__nv_bfloat16>(float (&c)[4], const uint32_t (&a)[4], uint32_t b0, uint32_t b1)
{
    asm("mma.sync.aligned.m16n8k16.row.col.f32.bf16.bf16.f32 {%0,%1,%2,%3}, {%4,%5,%6,%7}, {%8,%9}, {%0,%1,%2,%3};"
                 : "+f"(c[0]), "+f"(c[1]), "+f"(c[2]), "+f"(c[3])
                 : "r"(a[0]), "r"(a[1]), "r"(a[2]), "r"(a[3]), "r"(b0), "r"(b1));
}

__device__ __forceinline__ void cp_async16(uint32_t dst, const void *src)
{
    asm volatile("cp.async.cg.shared.global [%0], [%1], 16;" ::"r"(dst), "l"(src) : "memory");
}

// The first `bytes` of the 16, zeros after them.
__device__ __forceinline__ void cp_async16_part(uint32_t dst, const void *src, uint32_t bytes)
{
    asm volatile("cp.async.cg.shared.global [%0], [%1], 16, %2;" ::"r"(dst), "l"(src), "r"(bytes) : "memory");
}

__device__ __forceinline__ uint4 lds16(uint32_t at)
{
    uint4 v;
    asm volatile("ld.shared.v4.b32 {%0,%1,%2,%3}, [%4];" : "=r"(v.x), "=r"(v.y), "=r"(v.z), "=r"(v.w) : "r"(at) : "memory");
    return v;
}

// A slot of a warp's ring holds kSub 32 x 64 blocks of weights, neighbours in K, as the image has them, and the same
// columns of NT rows of x: 128 bytes a row and block, 16-byte chunk c of row r at chunk c ^ (r & 7) (no bank conflicts
// when a lane takes two neighbouring chunks of its row).  Narrow codes and few rows take more blocks a slot, which halves
// the instructions around the copies.  Two blocks of eight warps share an SM where that leaves a warp two slots or more
// (one warp a scheduler issues an instruction every eight cycles or so here, so warps count); otherwise one block has it
// alone.
template <int BITS, int NT>
struct Ring {
    static constexpr int kSub = NT > 8 || BITS > 4 ? 1 : 2;
    static constexpr int kWBytes = 32 * 64 * BITS / 8, kXBytes = NT * 128;  // of one block
    static constexpr int kSlotBytes = kSub * (kWBytes + kXBytes);
    static constexpr int kPartBytes = 2 * kStreamWarps * 32 * (NT + 1) * 4;  // two units deep: one barrier a unit
    static constexpr int kTabBytes = 4 * 1025 + 12;
    static constexpr int slots(int per_sm)
    {
        const int n = (227 * 1024 / per_sm - 1024 - kPartBytes - kTabBytes) / kStreamWarps / kSlotBytes;
        return n > 8 ? 8 : n;
    }
    static constexpr int kPerSm = slots(2) >= 2 ? 2 : 1;
    static constexpr int kSlots = slots(kPerSm);
    static constexpr int kWarpBytes = kSlots * kSlotBytes;
    static constexpr int kSmem = kStreamWarps * kWarpBytes + kPartBytes + kTabBytes;
    static_assert(kSlots >= 2, "a ring has two slots at least");
};

__device__ __forceinline__ void cluster_arrive() { asm volatile("barrier.cluster.arrive.release.aligned;" ::: "memory"); }
__device__ __forceinline__ void cluster_wait() { asm volatile("barrier.cluster.wait.acquire.aligned;" ::: "memory"); }

// Stores a float at this shared-memory address of the cluster's first block.
__device__ __forceinline__ void st_first(uint32_t at, float v)
{
    asm volatile("{\n\t.reg .b32 q;\n\tmapa.shared::cluster.u32 q, %0, 0;\n\tst.shared::cluster.f32 [q], %1;\n\t}" ::"r"(at), "f"(v)
                 : "memory");
}

// Value pairs of half-row h (rows 8 h + g), columns 16 t .. 16 t + 15, from a lane's words of a block.
template <typename T, int BITS>
__device__ __forceinline__ void expand_row(const uint32_t *w, int h, uint32_t (&v)[8])
{
    if constexpr (BITS == 16) {
#pragma unroll
        for (int i = 0; i < 8; ++i) v[i] = w[h * 8 + i];
    } else {
        expand16<T, BITS>(w + h * (BITS / 2), v);
    }
}

// Where a unit's tile lies: expert, first place or row, rows.
struct StreamTile {
    int expert, count;
    int64_t first;
};

template <typename T, int BITS, int NT>
__global__ void __launch_bounds__(kStreamWarps * 32, Ring<BITS, NT>::kPerSm) matmul_stream_kernel(const MatmulArgs a, const int ranks, const int wpu)
{
    using R = Ring<BITS, NT>;
    constexpr int kN = NT / 8;
    constexpr int kChains = kN == 1 ? 2 : 1;  // accumulator sets: a single narrow tile has too few independent MMAs
    constexpr uint32_t kBlock = R::kWBytes;
    extern __shared__ __align__(16) uint8_t smem[];
    using Part = float[kStreamWarps * 32][NT + 1];
    Part *parts = reinterpret_cast<Part *>(smem + kStreamWarps * R::kWarpBytes);
    int *tab = reinterpret_cast<int *>(smem + kStreamWarps * R::kWarpBytes + R::kPartBytes);  // tiles before each expert
    const int lane = threadIdx.x & 31, warp = threadIdx.x >> 5, g = lane >> 2, t = lane & 3;
    // sets of `wpu` warps (all eight where a cluster splits K)
    const int sets = kStreamWarps / wpu, set = warp / wpu, in_set = warp - set * wpu, set_threads = wpu * 32;
    const int tid = threadIdx.x - set * set_threads;
    const int rank = blockIdx.x % ranks, share = blockIdx.x / ranks * sets + set, shares = gridDim.x / ranks * sets;
    auto set_barrier = [&]() { asm volatile("bar.sync %0, %1;" ::"r"(set + 1), "r"(set_threads) : "memory"); };

    if (ranks > 1) cluster_arrive();  // (this block has started)
    pdl_begin();
    int tiles = static_cast<int>((a.rows + NT - 1) / NT);
    if (a.offsets) {
        if (warp == 0) expert_tiles(a.offsets, a.experts, NT, tab);
        __syncthreads();
        tiles = tab[a.experts];
        if (a.zero_tail)  // rows that no expert fills
            for (int64_t r = a.offsets[a.experts] + blockIdx.x; r < a.rows; r += gridDim.x)
                for (int c = threadIdx.x; c < a.m; c += blockDim.x) static_cast<T *>(a.y)[r * a.ldy + c] = from_f32<T>(0.f);
    }
    const int units = tiles * a.mb;
    const int u0 = static_cast<int>(static_cast<int64_t>(units) * share / shares);
    const int u1 = static_cast<int>(static_cast<int64_t>(units) * (share + 1) / shares);

    auto tile_of = [&](int tile) {
        StreamTile r;
        r.expert = 0;
        if (a.offsets) {
            r.expert = find_expert(tab, a.experts, tile);
            r.first = a.offsets[r.expert] + static_cast<int64_t>(tile - tab[r.expert]) * NT;
            r.count = static_cast<int>(min(static_cast<int64_t>(NT), a.offsets[r.expert + 1] - r.first));
        } else {
            r.first = static_cast<int64_t>(tile) * NT;
            r.count = static_cast<int>(min(static_cast<int64_t>(NT), a.rows - r.first));
        }
        return r;
    };

    // this warp's share of K, in slots: columns (kb0 + i * step) * 64 ..., i < per
    const int kb0 = (rank * wpu + in_set) * R::kSub, step = ranks * wpu * R::kSub;
    const int per = kb0 < a.kb ? (a.kb - kb0 + step - 1) / step : 0;
    const uint32_t wstep = step * kBlock;
    const uint32_t ring = smem_addr(smem) + warp * R::kWarpBytes;

    // ---- copies, ahead of the sums: instruction i of a block of x takes rows 4 i .. 4 i + 3, eight lanes a row
    int cu = u0;                              // next unit to copy from
    int ck = a.kb, ctile = -1, ccount = 0;    // next column block of the unit before it, its tile, the tile's rows
    const uint8_t *wtile = nullptr, *wsrc = nullptr;
    const T *xrow[2 * kN];
    // this lane's place among a block's rows of x: row lane / 8 (and every fourth after it), swizzled chunk lane % 8
    const uint32_t xlane = (lane >> 3) * 128 + ((lane & 7) ^ (lane >> 3)) * 16;
    auto copy_next = [&](uint32_t slot) {
        if (ck >= a.kb) {
            const int tile = cu / a.mb, mb = cu - tile * a.mb;
            ++cu;
            if (tile != ctile) {
                ctile = tile;
                const StreamTile p = tile_of(tile);
                ccount = p.count;
                wtile = a.image + static_cast<size_t>(p.expert) * a.mb * a.kb * kBlock + lane * 16;
#pragma unroll
                for (int i = 0; i < 2 * kN; ++i) {
                    // rows past the count repeat the last one; nothing is stored of them
                    int64_t row = p.first + min(i * 4 + (lane >> 3), p.count - 1);
                    if (a.gather) row = a.order[row] / a.top;
                    xrow[i] = static_cast<const T *>(a.x) + row * a.ldx + (lane & 7) * 8;
                }
            }
            ck = kb0;
            wsrc = wtile + (static_cast<size_t>(mb) * a.kb + kb0) * kBlock;
        }
        // slot: the blocks' weights one after another, then their x
        const uint32_t wdst = slot + lane * 16, xdst = slot + R::kSub * R::kWBytes + xlane;
        if ((ck + R::kSub) * 64 <= a.k && a.x_vec) {  // whole blocks: the common case, few instructions
#pragma unroll
            for (int i = 0; i < R::kSub * R::kWBytes / 512; ++i) cp_async16(wdst + i * 512, wsrc + i * 512);
#pragma unroll
            for (int i = 0; i < 2 * kN; ++i) {
                if (i * 4 >= ccount) break;
                const T *p = xrow[i] + ck * 64;
                // rows four apart differ in bit 2 of the swizzle
                const uint32_t to = (i & 1 ? xdst ^ 64 : xdst) + i * 512;
#pragma unroll
                for (int s = 0; s < R::kSub; ++s) cp_async16(to + s * R::kXBytes, p + s * 64);
            }
        } else {
#pragma unroll
            for (int s = 0; s < R::kSub; ++s) {
                if (ck + s >= a.kb) break;
#pragma unroll
                for (int i = 0; i < R::kWBytes / 512; ++i) cp_async16(wdst + s * kBlock + i * 512, wsrc + s * kBlock + i * 512);
                const int k0 = (ck + s) * 64;
                const int left = 2 * (a.k - k0 - (lane & 7) * 8);  // bytes of the row from this lane's chunk on
#pragma unroll
                for (int i = 0; i < 2 * kN; ++i) {
                    if (i * 4 >= ccount) break;
                    const T *p = xrow[i] + k0;
                    const uint32_t to = (i & 1 ? xdst ^ 64 : xdst) + i * 512 + s * R::kXBytes;
                    if (a.x_vec) {
                        cp_async16_part(to, left > 0 ? p : static_cast<const T *>(a.x), max(0, min(16, left)));
                    } else {  // rows that are not 16-byte aligned, two bytes at a time
                        const uint16_t *q = reinterpret_cast<const uint16_t *>(p);
#pragma unroll
                        for (int e = 0; e < 8; ++e) {
                            const uint16_t v = 2 * e < left ? q[e] : 0;
                            asm volatile("st.shared.u16 [%0], %1;" ::"r"(to + e * 2), "h"(v) : "memory");
                        }
                    }
                }
            }
        }
        ck += step;
        wsrc += wstep;
    };

    // ---- sums
    float acc[kChains][2][kN][4] = {};
    StreamTile cur = {0, 0, 0};
    int cur_tile = -1;
    const int chans = a.gated ? 16 : 32, shift = a.gated ? 4 : 5;
    const int my_c = tid & (chans - 1), my_r = a.gated ? (my_c >> 3) * 16 + (my_c & 7) : my_c;
    float2 q0, q1;  // scale and bias of this thread's channel (gate and up), loaded while the unit's blocks arrive
    int cur_mb = 0;
    auto begin_unit = [&](int unit) {
        const int tile = unit / a.mb;
        cur_mb = unit - tile * a.mb;
        if (tile != cur_tile) {
            cur_tile = tile;
            cur = tile_of(tile);
        }
        const float2 *params = a.params + (static_cast<int64_t>(cur.expert) * a.mb + cur_mb) * 32;
        q0 = params[my_r];
        if (a.gated) q1 = params[my_r + 8];
    };
    auto finish_unit = [&](int unit) {
        Part &part = parts[(unit - u0) & 1];
#pragma unroll
        for (int j = 0; j < 2; ++j)
#pragma unroll
            for (int n = 0; n < kN; ++n)
#pragma unroll
                for (int i = 0; i < 4; ++i) {
                    float s = acc[0][j][n][i];
                    if (kChains == 2) s += acc[kChains - 1][j][n][i];
                    part[warp * 32 + j * 16 + g + (i >> 1) * 8][n * 8 + 2 * t + (i & 1)] = s;
                    acc[0][j][n][i] = acc[kChains - 1][j][n][i] = 0.f;
                }
        set_barrier();
        // row r of the image, row n of x, added over the set's warps (or over the blocks of a cluster)
        auto sum = [&](const Part &part, int r, int n) {
            const float *p = &part[set * wpu * 32 + r][n];
            constexpr int kStep = 32 * (NT + 1);
            float s = p[0] + p[kStep];
            if (wpu > 2) s += p[2 * kStep] + p[3 * kStep];
            if (wpu > 4) s += (p[4 * kStep] + p[5 * kStep]) + (p[6 * kStep] + p[7 * kStep]);
            return s;
        };
        const Part *from = &part;
        if (ranks > 1) {  // one unit a cluster: the second buffer takes the blocks' sums, zeros where there is no block
            cluster_wait();
            for (int i = threadIdx.x; i < 32 * NT; i += kStreamWarps * 32) {
                const int r = i / NT, n = i % NT;
                st_first(smem_addr(&parts[1][rank * 32 + r][n]), sum(part, r, n));
                if (rank + ranks < kStreamWarps) st_first(smem_addr(&parts[1][(rank + ranks) * 32 + r][n]), 0.f);
                if (ranks == 2 && rank + 4 < kStreamWarps) {
                    st_first(smem_addr(&parts[1][(rank + 4) * 32 + r][n]), 0.f);
                    st_first(smem_addr(&parts[1][(rank + 6) * 32 + r][n]), 0.f);
                }
            }
            cluster_arrive();
            cluster_wait();
            if (rank > 0) return;
            from = &parts[1];
        }
        const int64_t col = static_cast<int64_t>(cur_mb) * chans + my_c;
        if (col < a.m)
            for (int n = tid >> shift; n < cur.count; n += set_threads >> shift) {
                float s = activate(fmaf(sum(*from, my_r, n), q0.x, q0.y), a.act);
                if (a.gated) s *= fmaf(sum(*from, my_r + 8, n), q1.x, q1.y);
                finish<T>(a, cur.first + n, col, s);
            }
    };

    const int total = per * (u1 - u0);
    int copied = 0;
#pragma unroll
    for (int i = 0; i < R::kSlots; ++i) {
        if (copied < total) {
            copy_next(ring + i * R::kSlotBytes);
            ++copied;
        }
        asm volatile("cp.async.commit_group;" ::: "memory");
    }
    int unit = u0, in_unit = 0, slot = 0;
    if (u0 < u1) begin_unit(u0);
    for (int done = 0; done < total; ++done) {
        asm volatile("cp.async.wait_group %0;" ::"n"(R::kSlots - 1) : "memory");
        __syncwarp();
        const uint32_t base = ring + slot * R::kSlotBytes;
#pragma unroll
        for (int s = 0; s < R::kSub; ++s) {
            if (kb0 + in_unit * step + s >= a.kb) break;
            const uint32_t at = base + s * R::kWBytes, xat = base + R::kSub * R::kWBytes + s * R::kXBytes;
            uint32_t w[BITS * 2], x[kN][8];
#pragma unroll
            for (int i = 0; i < BITS / 2; ++i) {
                // packed codes lie as the lanes take them; of 16-bit rows, chunks 2 t and 2 t + 1 of half-row i / 2, row g
                const uint4 q = lds16(BITS == 16 ? at + (i >> 1) * 1024 + g * 128 + ((2 * t + (i & 1)) ^ g) * 16 : at + i * 512 + lane * 16);
                w[4 * i] = q.x; w[4 * i + 1] = q.y; w[4 * i + 2] = q.z; w[4 * i + 3] = q.w;
            }
#pragma unroll
            for (int n = 0; n < kN; ++n)
#pragma unroll
                for (int i = 0; i < 2; ++i) {
                    const uint4 q = lds16(xat + (n * 8 + g) * 128 + ((2 * t + i) ^ g) * 16);
                    x[n][4 * i] = q.x; x[n][4 * i + 1] = q.y; x[n][4 * i + 2] = q.z; x[n][4 * i + 3] = q.w;
                }
#pragma unroll
            for (int j = 0; j < 2; ++j) {
                uint32_t lo[8], hi[8];
                expand_row<T, BITS>(w, 2 * j, lo);
                expand_row<T, BITS>(w, 2 * j + 1, hi);
#pragma unroll
                for (int k = 0; k < 4; ++k) {
                    const uint32_t f[4] = {lo[2 * k], hi[2 * k], lo[2 * k + 1], hi[2 * k + 1]};
#pragma unroll
                    for (int n = 0; n < kN; ++n) mma16816<T>(acc[k & (kChains - 1)][j][n], f, x[n][2 * k], x[n][2 * k + 1]);
                }
            }
        }
        __syncwarp();  // every lane has its words: the slot is free
        if (copied < total) {
            copy_next(base);
            ++copied;
        }
        asm volatile("cp.async.commit_group;" ::: "memory");
        slot = slot + 1 == R::kSlots ? 0 : slot + 1;
        if (++in_unit == per) {
            in_unit = 0;
            finish_unit(unit);
            if (++unit < u1) begin_unit(unit);
        }
    }
    // warps without columns of their own take part in every sum
    while (unit < u1) {
        finish_unit(unit);
        if (++unit < u1) begin_unit(unit);
    }
}

template <typename T, int BITS, int NT>
cudaError_t launch_one(const MatmulArgs &a, int64_t tiles, cudaStream_t st)
{
    using R = Ring<BITS, NT>;
    const cudaError_t e = raise_smem<matmul_stream_kernel<T, BITS, NT>>(R::kSmem);
    if (e != cudaSuccess) return e;
    // A block for every slot of the GPU, or for every unit; K split over clusters while those fill half of the slots at most
    // and every warp keeps a slot of K.
    const int64_t slots = R::kPerSm * device_sm_count(), units = tiles * a.mb;
    int ranks = 1;
    while (!a.offsets && ranks < 8 && 2 * ranks * units <= slots && a.kb >= 2 * ranks * kStreamWarps * R::kSub) ranks *= 2;
    // Warps to a unit: fewer while a warp has less than eight blocks of it.  (30 experts of 2 * 1024 rows
    // and 2048 columns, INT-4: 27.7 us with four warps a unit, 28.7 with eight.)
    int wpu = kStreamWarps;
    while (ranks == 1 && wpu > 2 && a.kb < 8 * wpu && 2 * units > slots * (kStreamWarps / wpu)) wpu /= 2;
    const int64_t sets = kStreamWarps / wpu;
    const int64_t shares = ranks > 1 ? units : std::min(slots, (units + sets - 1) / sets);
    return launch_pdl(matmul_stream_kernel<T, BITS, NT>, dim3(static_cast<unsigned>(shares * ranks)), kStreamWarps * 32, R::kSmem, st,
                      ranks, a, ranks, wpu);
}

template <typename T, int BITS>
cudaError_t launch_nt(const MatmulArgs &a, int nt, int64_t tiles, cudaStream_t st)
{
    if (nt == 8) return launch_one<T, BITS, 8>(a, tiles, st);
    if (nt == 16) return launch_one<T, BITS, 16>(a, tiles, st);
    return launch_one<T, BITS, 32>(a, tiles, st);
}

template <typename T>
cudaError_t launch_bits(const MatmulArgs &a, int bits, int nt, int64_t tiles, cudaStream_t st)
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
    return dtype == QNN_F16 ? launch_bits<__half>(a, bits, nt, tiles, st)
                            : launch_bits<__nv_bfloat16>(a, bits, nt, tiles, st);
}

}  // namespace qnn
