// Shared by the attention kernels: the sequences of a call, the keys that a row may see, and small helpers.
//
// The rows of a sequence and key head are its queries times the query heads that share the key head ("group"), the heads of
// a query one after another: row r is query r / group, head r % group.  They meet the same keys, so one tile of keys
// serves all of them.  Query i of n stands at position length - n + i.
#pragma once

#include <type_traits>

#include "attention.h"
#include "block_common.cuh"

namespace qnn {

constexpr float kLn2 = 0.6931471805599453f;

struct Sequence {
    int64_t first;  // row of q of its first query, or its place among the sequences without offsets
    int n;          // queries
    int keys;       // in the cache: the length, as far as the table reaches
    int at;         // position of the first query
};

__device__ __forceinline__ Sequence sequence(const AttnArgs &a, int s)
{
    Sequence q;
    if (a.offsets) {
        const int64_t b = a.offsets[s], e = a.offsets[s + 1];
        q.first = b < 0 ? 0 : (b > a.t ? a.t : b);
        const int64_t end = e < q.first ? q.first : (e > a.t ? a.t : e);
        q.n = static_cast<int>(end - q.first);
    } else {
        q.first = s;
        q.n = a.each;
    }
    const int room = a.width * a.page_size, length = a.lengths ? a.lengths[s] : room;
    q.keys = length < 0 ? 0 : (length < room ? length : room);
    const int64_t at = static_cast<int64_t>(length) - q.n;
    q.at = static_cast<int>(at < -0x7fffffffll ? -0x7fffffffll : at);
    return q;
}

// Keys [lo, hi) that query i sees.
__device__ __forceinline__ void keys_of(const AttnArgs &a, const Sequence &q, int i, int &lo, int &hi)
{
    const int64_t p = static_cast<int64_t>(q.at) + i;
    hi = a.causal && p + 1 < q.keys ? (p < 0 ? 0 : static_cast<int>(p + 1)) : q.keys;
    const int64_t first = p - a.window + 1;
    lo = a.window && first > 0 ? (first < hi ? static_cast<int>(first) : hi) : 0;
}

// Elements from the start of q (out) to head h of query i.
__device__ __forceinline__ int64_t q_at(const AttnArgs &a, const Sequence &q, int i, int h)
{
    return (a.offsets ? (q.first + i) * a.ldq : q.first * a.q_seq + i * a.ldq) + h * a.hq;
}
__device__ __forceinline__ int64_t o_at(const AttnArgs &a, const Sequence &q, int i, int h)
{
    return (a.offsets ? (q.first + i) * a.ldo : q.first * a.o_seq + i * a.ldo) + h * a.ho;
}
__device__ __forceinline__ int64_t lse_at(const AttnArgs &a, const Sequence &q, int i, int h)
{
    return (a.offsets ? q.first + i : q.first * a.each + i) * a.heads + h;
}

// The page that holds key j of sequence s, -1 where there is none.
__device__ __forceinline__ int page_of(const AttnArgs &a, int s, int column)
{
    const int page = a.table ? a.table[s * a.ldt + column] : s;
    return page >= 0 && page < a.pages ? page : -1;
}

// Sum of a value over the block's threads before this one, and over all of them.  `scratch` holds THREADS / 32 sums; all
// threads call it.
template <int THREADS>
__device__ __forceinline__ int64_t block_scan(int64_t v, int64_t *scratch, int64_t &total)
{
    const int lane = threadIdx.x & 31, warp = threadIdx.x >> 5;
    int64_t in = v;
#pragma unroll
    for (int d = 1; d < 32; d *= 2) {
        const int64_t o = __shfl_up_sync(0xffffffffu, in, d);
        if (lane >= d) in += o;
    }
    __syncthreads();
    if (lane == 31) scratch[warp] = in;
    __syncthreads();
    int64_t before = 0;
    total = 0;
#pragma unroll
    for (int w = 0; w < THREADS / 32; ++w) {
        if (w < warp) before += scratch[w];
        total += scratch[w];
    }
    return before + in - v;
}

// The first `bytes` of 16 from global to shared memory, zeros after them.
__device__ __forceinline__ void copy16(uint32_t dst, const void *src, uint32_t bytes)
{
    asm volatile("cp.async.cg.shared.global [%0], [%1], 16, %2;" ::"r"(dst), "l"(src), "r"(bytes) : "memory");
}
__device__ __forceinline__ void copy_commit() { asm volatile("cp.async.commit_group;" ::: "memory"); }
template <int N>
__device__ __forceinline__ void copy_wait()
{
    asm volatile("cp.async.wait_group %0;" ::"n"(N) : "memory");
}

// 2^x; -inf gives 0.
__device__ __forceinline__ float exp2_fast(float x)
{
    float y;
    asm("ex2.approx.ftz.f32 %0, %1;" : "=f"(y) : "f"(x));
    return y;
}

template <typename T>
__device__ __forceinline__ void mma16816(float (&c)[4], const uint32_t (&a)[4], uint32_t b0, uint32_t b1)
{
    if constexpr (sizeof(T) == 2 && std::is_same<T, __half>::value)
        asm("mma.sync.aligned.m16n8k16.row.col.f32.f16.f16.f32 {%0,%1,%2,%3}, {%4,%5,%6,%7}, {%8,%9}, {%0,%1,%2,%3};"
            : "+f"(c[0]), "+f"(c[1]), "+f"(c[2]), "+f"(c[3])
            : "r"(a[0]), "r"(a[1]), "r"(a[2]), "r"(a[3]), "r"(b0), "r"(b1));
    else
        asm("mma.sync.aligned.m16n8k16.row.col.f32.bf16.bf16.f32 {%0,%1,%2,%3}, {%4,%5,%6,%7}, {%8,%9}, {%0,%1,%2,%3};"
            : "+f"(c[0]), "+f"(c[1]), "+f"(c[2]), "+f"(c[3])
            : "r"(a[0]), "r"(a[1]), "r"(a[2]), "r"(a[3]), "r"(b0), "r"(b1));
}

__device__ __forceinline__ void ldsm4(uint32_t (&v)[4], uint32_t at)
{
    asm volatile("ldmatrix.sync.aligned.m8n8.x4.shared.b16 {%0,%1,%2,%3}, [%4];"
                 : "=r"(v[0]), "=r"(v[1]), "=r"(v[2]), "=r"(v[3])
                 : "r"(at)
                 : "memory");
}
__device__ __forceinline__ void ldsm4_trans(uint32_t (&v)[4], uint32_t at)
{
    asm volatile("ldmatrix.sync.aligned.m8n8.x4.trans.shared.b16 {%0,%1,%2,%3}, [%4];"
                 : "=r"(v[0]), "=r"(v[1]), "=r"(v[2]), "=r"(v[3])
                 : "r"(at)
                 : "memory");
}

}  // namespace qnn
