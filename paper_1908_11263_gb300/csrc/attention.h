// Host-side interfaces between the C ABI (capi_attention.cu) and the attention kernels: what a launch is given.
#pragma once

#include <cstddef>
#include <cstdint>
#include <cuda_runtime.h>

#include "internal.h"
#include "qnn.h"

namespace qnn {

// ---- rotary positions, alone or on the way into the cache -- rope.cu
struct RotateArgs {
    int64_t t;                  // tokens
    int d, half, interleaved;   // head dimension, rotated pairs
    int wide;                   // positions are int64
    float amplitude;
    const uint64_t *turns;      // [half]
    const void *positions;      // [t], or null: the tokens' places in their sequences
    // rotated to another place: x -> y
    int heads;
    const void *x;
    void *y;
    int64_t ldx, hx, ldy, hy;
    // rotated (k) and copied (v) into the cache; seqs < 0: no cache
    int kv_heads;
    const void *k, *v;
    void *k_pages, *v_pages;
    int64_t ldk, hk, ldv, hv;
    int64_t k_page, k_head, k_row, v_page, v_head, v_row;
    int64_t pages, ldt;
    int seqs, width, page_size;
    int64_t each;               // tokens of every sequence without offsets
    const int32_t *table, *lengths, *offsets;
};
cudaError_t launch_rotate(const RotateArgs &a, int dtype, cudaStream_t st);

// ---- attention -- attention_rows.cu, attention_tc.cu
struct AttnArgs {
    const void *q, *k, *v;
    void *out;
    float *lse;                 // [t][heads] or null
    const int32_t *table, *lengths, *offsets;
    int64_t q_seq, ldq, hq, o_seq, ldo, ho;  // elements; the sequences' strides without offsets
    int64_t k_page, k_head, k_row, v_page, v_head, v_row;
    int64_t pages, ldt, t;
    int seqs, width, page_size, each;  // each: queries of every sequence without offsets
    int heads, kv_heads, group, d;
    int causal, window;         // window 0: none
    int q_vec, out_vec, out_vec8;  // rows of q are 16-byte aligned; rows of out hold aligned pairs; are 16-byte aligned
    int box, q_box;             // attention_tc: rows that a tiled copy takes of a page, and of q (0: none)
    int few;                    // rows (queries * group) of a sequence up to which it is the streaming kernel's; the rest is attention_tc's
    float scale;                // of q k, times log2(e)
    float *part, *tc_part;      // workspaces of attention_rows and attention_tc, or null
};
// Blocks of the streaming kernel, and the bytes that the parts of shared rows take.
int attention_rows_blocks(int d);
size_t attention_rows_workspace(int d);
cudaError_t launch_attention_rows(const AttnArgs &a, int dtype, cudaStream_t st);
size_t attention_tc_workspace(int d);
cudaError_t launch_attention_tc(const AttnArgs &a, int dtype, cudaStream_t st);  // heads of 128 elements at most

}  // namespace qnn
