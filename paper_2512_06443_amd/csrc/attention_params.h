// What the host side of the attention (attention.hip) and its kernels (attention_kernel.hip.h, compiled once for each type of the cache) share.
#pragma once

#include <hip/hip_runtime.h>

#include <cstddef>
#include <cstdint>

#include "vlut.h"

namespace vlut_attention {

struct AttendParams {
    const void *q, *k, *v;
    int64_t q_sequence, q_token, q_head;                               // strides in elements
    int64_t k_page, k_head, k_token, v_page, v_head, v_token;
    const int32_t *prefix_pages, *page_table, *own_lens, *query_lens;
    int64_t table_stride;
    void* out;
    int64_t out_sequence, out_token, out_head;
    float* lse;
    float *part_o, *part_ml;           // [Hk][B n G][slot][D], [Hk][B n G][slot][2]; slots: the prefix' splits, then the own parts'
    float scale_log2;                  // scale * log2(e): exponentials are powers of two
    int out_type;                      // VLUT_TYPE_*
    int B, n, Hk, G, D, page_log, pages;
    int P, max_own;
    int prefix_splits, prefix_chunk;   // keys per split
    int own_heads_together;            // Hk where a token's heads are worked on by one XCD, else 1
    int own_splits, own_share, own_step;   // waves to a range; its keys are a multiple of own_step but for the end
    int prefix_tiles, own_tiles;       // tiles of rows
    int prefix_per_xcd, own_per_xcd;   // workgroups
    int rows;                          // B n G
    int direct;                        // a single part: workgroups store the result
};

inline int log2_of(int64_t v) {
    int k = 0;
    while (((int64_t)1 << k) < v) ++k;
    return k;
}
inline int64_t ceil_div(int64_t a, int64_t b) { return (a + b - 1) / b; }

constexpr int kFewKeys = 32;           // keys of a wave's step where rows are few
__host__ __device__ constexpr int few_pitch(int DP) { return DP * 2 + 32; }
__host__ __device__ constexpr int few_lds(int DP) { return 4 * kFewKeys * few_pitch(DP); }
__host__ __device__ constexpr int few_waves(int DP, int MT) { return DP > 128 ? 1 : (MT > 1 ? 2 : (DP > 64 ? 2 : 4)); }   // of a SIMD
__host__ __device__ constexpr int many_keys(int DP) { return DP > 128 ? 32 : 64; }
__host__ __device__ constexpr int many_k_pitch(int DP) { return DP * 2 + 16; }
__host__ __device__ constexpr int many_v_pitch(int DP) { return DP * 2 + 64; }
__host__ __device__ constexpr int many_buffer(int DP) { return many_keys(DP) * (many_k_pitch(DP) + many_v_pitch(DP)); }

struct AttendPlan {
    int MT, waves, own_mt, DP;         // tile of the prefix: 16 * MT rows; MT = 0: 32 for each of the waves, by a kernel of its own
    int own_share, own_step, own_heads_together, grouped;
    int prefix_tiles, prefix_splits, prefix_chunk, prefix_per_xcd, own_tiles, own_splits, own_per_xcd, direct;
    int combine_lanes_log, combine_blocks;
    int64_t rows;
    size_t o_bytes, ml_bytes;
};

__attribute__((visibility("hidden"))) int launch_bf16(const AttendPlan& a, const AttendParams& p, hipStream_t stream);
__attribute__((visibility("hidden"))) int launch_f16(const AttendPlan& a, const AttendParams& p, hipStream_t stream);

}  // namespace vlut_attention
