// What the host side of the attention of chunks (chunk.hip) and its kernels (chunk_kernel.hip.h, compiled once for each type of the cache and of the outputs) share.
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
    float inverse_g;                   // 1 / G
    int N, B, Hk, G, D, page_log, pages, max_len;
    int window;                        // keys that a query sees at most
    int few_rows;                      // a sequence of up to so many rows per key head is a few-row one (0: none is)
    int few_splits, few_chunk, few_per_xcd;                            // parts at most, keys of a part, workgroups of an XCD
    int many_splits, many_chunk, many_tiles, many_per_xcd;     // many_tiles: at most
};

constexpr int kFewRows = 32, kManyRows = 128;        // of a tile

// How keys and values come to LDS: through registers; straight, a dword or 16 bytes a lane; of rows that are as long as LDS has them; rows of 4, 12, 20, ... features that
// lie one behind the other in memory, 8 of them (16 D bytes) at a time and one behind the other in LDS too.
constexpr int kThroughRegisters = 0, kDwords = 1, kVectors = 2, kWholeVectors = 3, kRuns = 4;

// A workgroup's waves: RW groups of 32 rows, the keys of a step shared by KW.  Where rows are few 1 x 4 (features past 128: 1 x 2); where they are many 4 x 1 or 4 x 2
// (features past 128: 4 x 1).  Of the workgroups of four waves a unit has room for two, of 4 x 1 with features past 128 for one.
__host__ __device__ constexpr int few_waves(int DP) { return DP > 128 ? 2 : 4; }
__host__ __device__ constexpr bool own_keys(int RW, int LOAD) { return RW == 1 && LOAD != kThroughRegisters; }      // waves have their keys for themselves
__host__ __device__ constexpr int wave_keys(int DP, int RW) { return RW == 1 || DP > 128 ? 32 : 64; }
__host__ __device__ constexpr int step_keys(int DP, int RW, int KW) { return wave_keys(DP, RW) * KW; }
__host__ __device__ constexpr int k_pitch(int DP, int LOAD) { return DP * 2 + (LOAD == kThroughRegisters ? 16 : 0); }
__host__ __device__ constexpr int v_pitch(int DP, int LOAD) { return DP * 2 + (LOAD == kThroughRegisters ? 64 : 0); }
// Through registers: a stage is a step's keys and values.  Straight: the KW groups of waves have rings of stages of their keys and values each, AHEAD of which are on
// their way.
__host__ __device__ constexpr int stage_bytes(int DP, int RW, int KW, int LOAD) { return step_keys(DP, RW, KW) * (k_pitch(DP, LOAD) + v_pitch(DP, LOAD)); }
__host__ __device__ constexpr int stages(int RW) { return RW == 1 ? 1 : 2; }
__host__ __device__ constexpr int ahead(int DP) { return DP > 128 ? 2 : 1; }
__host__ __device__ constexpr int ring(int DP, int RW) { return RW == 1 ? 1 : ahead(DP) + 1; }
__host__ __device__ constexpr int ring_bytes(int DP, int RW) { return ring(DP, RW) * wave_keys(DP, RW) * DP * 4; }
__host__ __device__ constexpr int buffers_bytes(int DP, int RW, int KW, int LOAD) {
    return LOAD == kThroughRegisters ? stages(RW) * stage_bytes(DP, RW, KW, LOAD) : KW * ring_bytes(DP, RW);
}
__host__ __device__ constexpr int turn_features(int DP) { return DP > 64 ? 64 : 32; }       // that leave through LDS together
__host__ __device__ constexpr int most_of(int a, int b) { return a > b ? a : b; }
// Keys and values, or what results leave through: for each wave 32 rows, of the features that leave together, or of half of them all.
__host__ __device__ constexpr int leave_pitch(int DP, int KW) { return (KW == 1 ? turn_features(DP) : DP / 2) + 4; }
__host__ __device__ constexpr int tile_bytes(int DP, int RW, int KW, int LOAD) { return most_of(buffers_bytes(DP, RW, KW, LOAD), RW * KW * 32 * leave_pitch(DP, KW) * 4); }
__host__ __device__ constexpr int stretch(int RW, int KW) { return RW == 1 ? 4096 : (RW * KW == 4 ? 8192 : 16384); }        // keys whose pages' numbers are in LDS (8 keys a page at least)
__host__ __device__ constexpr int lds_bytes(int DP, int RW, int KW, int LOAD) {
    return tile_bytes(DP, RW, KW, LOAD) + RW * KW * 32 * 20 + 16 + (LOAD == kThroughRegisters ? 0 : (stretch(RW, KW) / 8 + 2) * 4);
}

struct ChunkPlan {
    int DP, key_waves, load;           // KW where rows are many; how keys come to LDS
    int few, many;                     // whether there are such workgroups
    int few_splits, few_chunk, few_row_places, many_splits, many_chunk, many_tiles;
    int few_per_xcd, many_per_xcd;
    size_t few_o_bytes, few_ml_bytes, many_o_bytes, many_ml_bytes;
    size_t bytes() const { return few_o_bytes + few_ml_bytes + many_o_bytes + many_ml_bytes; }
};

// For outputs of the cache's type, and of fp32.
__attribute__((visibility("hidden"))) int launch_bf16(const ChunkPlan& a, const ChunkParams& p, hipStream_t stream);
__attribute__((visibility("hidden"))) int launch_bf16_f32(const ChunkPlan& a, const ChunkParams& p, hipStream_t stream);
__attribute__((visibility("hidden"))) int launch_f16(const ChunkPlan& a, const ChunkParams& p, hipStream_t stream);
__attribute__((visibility("hidden"))) int launch_f16_f32(const ChunkPlan& a, const ChunkParams& p, hipStream_t stream);

}  // namespace vlut_chunk
