// What the host side of the attention of chunks (chunk.hip) and its kernels (chunk_kernel.hip.h, compiled once for each type of the cache) share.
#pragma once

#include <hip/hip_runtime.h>

#include <cstddef>
#include <cstdint>

#include "vlut.h"

namespace vlut_chunk {

struct ChunkParams {
    const void *q, *k, *v;
    int64_t q_token, q_head;                                           // strides in elements
    int64_t k_page, k_head, k_token, v_page, v_head, v_token;
    const int32_t *page_table, *starts, *lens;
    int64_t table_stride;
    void* out;
    int64_t out_token, out_head;
    float* lse;
    float *few_o, *few_ml;             // parts of sequences with few rows: [split][B][Hk][few_rows][D], [..][2]
    float *many_o, *many_ml;           // of the others: [split][N][heads][D], [..][2]
    float scale_log2;                  // scale * log2(e): exponentials are powers of two
    int out_type;                      // VLUT_TYPE_*
    int N, B, Hk, G, D, page_log, pages, max_len;
    int window;                        // keys that a query sees at most
    int few_rows;                      // a sequence of up to so many rows per key head is a few-row one (0: none is)
    int few_splits, few_chunk, few_per_xcd;                            // parts at most, keys of a part, workgroups of an XCD
    int many_splits, many_chunk, many_tiles, many_per_xcd, many_rows;  // many_tiles: at most; many_rows: of a tile
};

constexpr int kFewRows = 32;

// Of a workgroup with RW x KW waves: RW groups of 32 rows, the keys of a step shared by KW.
// Where memory is loaded straight to LDS (FAST) rows of keys lie one behind the other in several stages, a wave's own ones where waves share the keys; else
// they go through registers, to rows that are padded.
__host__ __device__ constexpr int few_waves(int DP, bool FAST) { return FAST && DP > 128 ? 2 : 4; }          // KW where rows are few
__host__ __device__ constexpr int wave_keys(int DP, int KW) { return KW > 1 || DP > 128 ? 32 : 64; }
__host__ __device__ constexpr int step_keys(int DP, int KW) { return wave_keys(DP, KW) * KW; }
__host__ __device__ constexpr int k_pitch(int DP) { return DP * 2 + 16; }
__host__ __device__ constexpr int v_pitch(int DP) { return DP * 2 + 64; }
__host__ __device__ constexpr int buffer_bytes_of(int DP, int KW) { return step_keys(DP, KW) * (k_pitch(DP) + v_pitch(DP)); }
__host__ __device__ constexpr int buffers(int KW) { return KW > 1 ? 1 : 2; }
__host__ __device__ constexpr int stages(int DP, int RW, int KW) { return KW > 1 ? 2 : (RW > 4 || DP > 128 ? 3 : 2); }
__host__ __device__ constexpr int stage_bytes(int DP, int KW) { return step_keys(DP, KW) * DP * 4; }
__host__ __device__ constexpr int turn_features(int DP) { return DP > 64 ? 64 : 32; }       // that leave through LDS together
__host__ __device__ constexpr int most_of(int a, int b) { return a > b ? a : b; }
// Keys and values, or what results leave through: rows of a wave, or the parts of KW waves.
__host__ __device__ constexpr int tile_bytes(int DP, int RW, int KW, bool FAST) {
    return most_of(FAST ? stages(DP, RW, KW) * stage_bytes(DP, KW) : buffers(KW) * buffer_bytes_of(DP, KW),
                   KW > 1 ? KW * 32 * (DP + 4) * 4 : RW * 32 * (turn_features(DP) + 4) * 4);
}
constexpr int kStretch = 16384;        // keys whose pages' numbers are in LDS (FAST, 8 keys a page at least)
constexpr int kStretchPages = kStretch / 8 + 2;
__host__ __device__ constexpr int lds_bytes(int DP, int RW, int KW, bool FAST) {
    return tile_bytes(DP, RW, KW, FAST) + RW * KW * 32 * 8 + RW * 32 * 12 + 16 + (FAST ? kStretchPages * 4 : 0);
}

struct ChunkPlan {
    int DP, many_waves;                // waves of a workgroup where rows are many
    int few, many;                     // whether there is such a launch
    int few_splits, few_chunk, few_row_places, many_splits, many_chunk, many_tiles, many_rows;
    int few_per_xcd, many_per_xcd;
    int fast;                          // heads of a multiple of 8 features in rows of 16 bytes' alignment, 8 keys share their page, strides of 31 bits
    size_t few_o_bytes, few_ml_bytes, many_o_bytes, many_ml_bytes;
    size_t bytes() const { return few_o_bytes + few_ml_bytes + many_o_bytes + many_ml_bytes; }
};

__attribute__((visibility("hidden"))) int launch_bf16(const ChunkPlan& a, const ChunkParams& p, hipStream_t stream);
__attribute__((visibility("hidden"))) int launch_f16(const ChunkPlan& a, const ChunkParams& p, hipStream_t stream);

}  // namespace vlut_chunk
