// Attention of chunks of new tokens over a paged cache, for MI355X (gfx950): its host side and part of the C ABI; the kernels are in four more units, one
// for each type of the cache and of the outputs.
#include <hip/hip_runtime.h>

#include <algorithm>
#include <cmath>
#include <cstdint>

#include "vlut.h"

#include "chunk_params.h"
#include "host_checks.h"

namespace {

using namespace vlut_chunk;

constexpr int kUnits = 256;            // compute units that a launch is to fill
constexpr int64_t kMost = (int64_t)1 << 30, kMostBlocks = (int64_t)1 << 22;

int64_t ceil_div(int64_t a, int64_t b) { return (a + b - 1) / b; }
size_t whole_lines(size_t bytes) { return (bytes + 255) & ~(size_t)255; }
int log2_of(int64_t v) {
    int k = 0;
    while (((int64_t)1 << k) < v) ++k;
    return k;
}

int plan_chunks(int64_t N, int64_t B, int64_t Hq, int64_t Hk, int64_t D, int64_t max_queries, int64_t max_len, int64_t window, ChunkPlan* out) {
    if (N < 1 || N >= ((int64_t)1 << 24) || B < 1 || B >= ((int64_t)1 << 24) || Hk < 1 || Hq < 1 || Hq >= (1 << 16) || Hq % Hk) return VLUT_ERR_SHAPE;
    if (max_len < 0 || max_len >= kMost || max_queries < 0 || window < 0 || window >= kMost || D < 1 || N * Hq >= kMost) return VLUT_ERR_SHAPE;
    if (D < 8 || D > VLUT_MAX_HEAD_FEATURES || D % 4) return VLUT_ERR_UNSUPPORTED;
    ChunkPlan a{};
    const int64_t G = Hq / Hk, most_rows = std::min(max_queries, N) * G;
    // Keys that a tile of `tokens` neighbouring tokens sees, at most (those of a window begin at a multiple of 32, up to 31 keys earlier).
    const auto seen = [&](int64_t tokens) { return std::max<int64_t>(1, window ? std::min(max_len, window + tokens) + 31 : max_len); };
    a.DP = D <= 64 ? 64 : (D <= 128 ? 128 : 256);
    a.many = most_rows > kFewRows;
    // With one sequence that may have many rows there is nothing for a launch for few.
    a.few = !a.many || (B > 1 && G <= kFewRows);
    if (a.few) {
        a.few_row_places = (int)std::min<int64_t>(kFewRows, std::max<int64_t>(1, most_rows / G) * G);
        // Parts only so that 640 waves are at work, each of four steps at least where there are many: a wave's way to its first keys and its results' way out take as long
        // as seven steps, and those that join parts 4 us.  32 steps at most, so that one long sequence among short ones does not keep the others' units waiting, or more
        // where those would be more than 8192 workgroups.  us of the kernels with parts of 1, 2, 4, 8, 16 / 32 steps, joining included, 32 query and 8 key heads of 128 in bf16
        // (20 and 5 where it says so): a sequence of 1000 keys 15.0, 15.9, 18.0, 18.9; of 2000 (20, 5) 15.5, 15.5, 18.2, 23.0, 28.8; of 8000 31, 24, 21, 24, 33 / 54; 4 of 8000
        // 55, 40, 33, 31, 34 / 55; 8 of 4000 50, 37, 32, 31, 36 / 52; 16 of up to 4000 87, 63, 52, 49, 49 / 57; 32 of 8 queries behind up to 3000 (20, 5) 91, 68, 56, 51,
        // 64 / 49; 48 of up to 4095 154, 119, 101, 98, 98 / 94; 64 of 2048 to 4095 252, 187, 161, 147, 147 / 147; 13 of up to 1990 in windows of 1024, 32 heads of 100 that
        // are not shared, 79, 59, 51, 57, 37 / 37.  8 query and 2 key heads of 256 features, parts of 1, 4, 8, 16, 32 steps of two waves: a sequence of 8000 keys 42, 25, 30, 44,
        // 74; 16 of up to 4000 63, 33, 32, 45, 75; 64 of 2048 to 4095 163, 99, 87, 80, 84.  What this takes is within 6 % of the best of each, of the last 11.
        const int64_t step = step_keys(a.DP, 1, few_waves(a.DP)), keys = seen(kFewRows), steps = ceil_div(keys, step);
        const int64_t wanted = ceil_div(640, few_waves(a.DP) * B * Hk);
        const int64_t least = std::min<int64_t>(4, ceil_div(steps, 6)), most = std::max<int64_t>(32, ceil_div(B * Hk * steps, 8192));
        const int64_t per = std::min(most, std::max(least, ceil_div(steps, wanted)));
        a.few_chunk = (int)(step * per);
        a.few_splits = (int)ceil_div(keys, a.few_chunk);
        const int64_t blocks = ceil_div(B * Hk * a.few_splits, 8);
        if (8 * blocks >= kMostBlocks) return VLUT_ERR_SHAPE;
        a.few_per_xcd = (int)blocks;
        if (a.few_splits > 1) {
            const size_t parts = (size_t)a.few_splits * (size_t)B * (size_t)Hk * (size_t)a.few_row_places;
            a.few_o_bytes = whole_lines(parts * (size_t)D * 4);
            a.few_ml_bytes = whole_lines(parts * 8);
        }
    }
    if (a.many) {
        const int64_t rows = N * G, keys = seen(kManyRows / G + 1);
        a.many_tiles = (int)std::min(rows / kManyRows + B, (rows + B * (kManyRows - 1)) / kManyRows);
        // As many as there are if all sequences with many rows have as many as they may have.
        const int64_t tiles = std::min<int64_t>(a.many_tiles, ceil_div(rows, most_rows) * ceil_div(most_rows, kManyRows)) * Hk;
        // Two workgroups of four waves on a unit, one's waits beside the other's work, where there are tiles for that; else one whose eight waves share the keys, unless
        // those are so many that parts of them are as good.  us, 4 x 1 / 4 x 2, parts joined included, 20 query and 5 key heads of 128 in bf16: 4096 tokens 148 / 159, in
        // windows of 16 24 / 39, of 1024 94 / 109, 2500 tokens 80 / 68; 32 and 8 heads: 16384 tokens 2890 / 3100, 4096 198 / 230, of 64 features 133 / 161, 2048 72 / 69, 1024
        // 42 / 32, behind 4096 132 / 123, 8192 222 / 218, 16384 442 / 460; 256 behind 16384 111 / 112; 32 heads of 100 that are not shared, 909 tokens in windows of 1024, 61 / 58.
        // (A cache that goes through registers is 4 x 1 in any case, which is not known here: half of the places stay empty where these are 2.)
        a.key_waves = a.DP <= 128 && tiles < 2 * kUnits && keys < 12288 ? 2 : 1;
        const int64_t slots = (a.DP <= 128 && a.key_waves == 1 ? 2 : 1) * kUnits, step = step_keys(a.DP, 4, a.key_waves);
        // Parts of 512 keys at least.  us with 256 / 512 / 1024 / 2048: 128 behind 4096 35, 35, 37, 43, behind 1024 25, 24, 26, 30; 256 behind 4096 46, 46, 46, 51; of 256
        // features, 8 and 2 heads, 512 behind 4096 57, 57, 71, 99.
        const int64_t splits = std::min(std::max<int64_t>(1, slots / tiles), ceil_div(keys, 512));
        a.many_chunk = (int)(ceil_div(ceil_div(keys, splits), step) * step);
        a.many_splits = (int)ceil_div(keys, a.many_chunk);
        const int64_t blocks = ceil_div(a.many_tiles * Hk * a.many_splits, 8);
        if (8 * blocks >= kMostBlocks) return VLUT_ERR_SHAPE;
        a.many_per_xcd = (int)blocks;
        if (a.many_splits > 1) {
            const size_t parts = (size_t)a.many_splits * (size_t)N * (size_t)Hq;
            a.many_o_bytes = whole_lines(parts * (size_t)D * 4);
            a.many_ml_bytes = whole_lines(parts * 8);
        }
    }
    // (workgroups that join the parts, of 1024 / DP rows each)
    if (a.bytes() && ceil_div(N * Hq, 1024 / a.DP) >= 4 * kMostBlocks) return VLUT_ERR_SHAPE;
    *out = a;
    return VLUT_OK;
}

// Eight keys share their page, rows start at a multiple of `unit` elements, and strides and the offsets inside a page fit 31 bits, in bytes.
bool grouped_by_eight(const vlut_cache& c, int unit) {
    bool ok = c.page_size >= 8 && (uintptr_t)c.k % (2 * unit) == 0 && (uintptr_t)c.v % (2 * unit) == 0;
    for (int64_t s : {c.k_page_stride, c.v_page_stride}) ok = ok && s >= 0 && s < ((int64_t)1 << 30) && s % unit == 0;
    for (int64_t s : {c.k_head_stride, c.v_head_stride}) ok = ok && s % unit == 0;
    for (int64_t s : {c.k_token_stride, c.v_token_stride}) ok = ok && s >= 0 && s < ((int64_t)1 << 30) / std::max<int64_t>(c.page_size, 8) && s % unit == 0;
    return ok;
}

// Rows of D features, an odd number of fours, one behind the other: 8 of them begin and end at whole 16 bytes.
bool in_runs(const vlut_cache& c, int64_t D) {
    bool ok = c.k_token_stride == D && c.v_token_stride == D && (uintptr_t)c.k % 16 == 0 && (uintptr_t)c.v % 16 == 0;
    for (int64_t s : {c.k_page_stride, c.v_page_stride, c.k_head_stride, c.v_head_stride}) ok = ok && s % 8 == 0;
    return ok;
}

}  // namespace

extern "C" {

size_t vlut_chunk_attention_bytes(int64_t N, int64_t B, int64_t q_heads, int64_t k_heads, int64_t D, int64_t max_queries, int64_t max_len, int64_t window) {
    ChunkPlan a;
    return plan_chunks(N, B, q_heads, k_heads, D, max_queries, max_len, window, &a) == VLUT_OK ? a.bytes() : 0;
}

int vlut_query_chunk_attention(int64_t N, int64_t B, int64_t q_heads, int64_t k_heads, int64_t D, int64_t max_queries, int64_t max_len, int64_t window, int* out6) {
    if (!out6) return VLUT_ERR_NULL;
    ChunkPlan a;
    const int rc = plan_chunks(N, B, q_heads, k_heads, D, max_queries, max_len, window, &a);
    if (rc != VLUT_OK) return rc;
    out6[0] = a.few ? a.few_row_places : 0;
    out6[1] = a.few_splits;
    out6[2] = a.few_chunk;
    out6[3] = a.many ? kManyRows : 0;
    out6[4] = a.many_splits;
    out6[5] = a.many_chunk;
    return VLUT_OK;
}

int vlut_chunk_attention(const vlut_heads* q, const vlut_cache* cache, const int32_t* page_table, int64_t table_stride, const int32_t* query_starts, const int32_t* lens,
                         int64_t N, int64_t B, int64_t D, int64_t max_queries, int64_t max_len, int64_t window, float scale, const vlut_heads* out, float* lse_or_null,
                         void* workspace, size_t workspace_bytes, void* stream) {
    if (!q || !out) return VLUT_ERR_NULL;
    int rc = check_cache(cache);
    if (rc != VLUT_OK) return rc;
    ChunkPlan a;
    rc = plan_chunks(N, B, q->heads, cache->heads, D, max_queries, max_len, window, &a);
    if (rc != VLUT_OK) return rc;
    if (!q->data || !out->data || !query_starts || !lens || (max_len > 0 && !page_table)) return VLUT_ERR_NULL;
    if (out->heads != q->heads || q->type != cache->type || (out->type != cache->type && out->type != VLUT_TYPE_F32)) return VLUT_ERR_SHAPE;
    if (cache->pages >= ((int64_t)1 << 31)) return VLUT_ERR_SHAPE;
    if (!(scale > 0.0f) || !std::isfinite(scale)) return VLUT_ERR_UNSUPPORTED;
    if (!at_dwords(q->data, 0, q->token_stride, q->head_stride, 2) ||
        !at_dwords(cache->k, cache->k_page_stride, cache->k_head_stride, cache->k_token_stride, 2) ||
        !at_dwords(cache->v, cache->v_page_stride, cache->v_head_stride, cache->v_token_stride, 2) ||
        !at_dwords(out->data, 0, out->token_stride, out->head_stride, type_bytes(out->type)))
        return VLUT_ERR_UNSUPPORTED;
    if (a.bytes()) {
        if (!workspace) return VLUT_ERR_NULL;
        if (workspace_bytes < a.bytes()) return VLUT_ERR_SMALL_BUFFER;
        if ((uintptr_t)workspace % 16) return VLUT_ERR_UNSUPPORTED;
    }
    if (!grouped_by_eight(*cache, 2)) a.load = kThroughRegisters;
    else if (D % 8) a.load = a.DP <= 128 && in_runs(*cache, D) ? kRuns : kDwords;
    else if (!grouped_by_eight(*cache, 8)) a.load = kDwords;
    else a.load = D < a.DP ? kVectors : kWholeVectors;
    ChunkParams p{};
    p.q = q->data;
    p.k = cache->k;
    p.v = cache->v;
    p.q_token = q->token_stride;
    p.q_head = q->head_stride;
    p.k_page = cache->k_page_stride;
    p.k_head = cache->k_head_stride;
    p.k_token = cache->k_token_stride;
    p.v_page = cache->v_page_stride;
    p.v_head = cache->v_head_stride;
    p.v_token = cache->v_token_stride;
    p.page_table = page_table;
    p.starts = query_starts;
    p.lens = lens;
    p.table_stride = table_stride;
    p.out = (void*)out->data;
    p.out_token = out->token_stride;
    p.out_head = out->head_stride;
    p.lse = lse_or_null;
    unsigned char* at = (unsigned char*)workspace;
    p.few_o = (float*)at;
    p.few_ml = (float*)(at += a.few_o_bytes);
    p.many_o = (float*)(at += a.few_ml_bytes);
    p.many_ml = (float*)(at += a.many_o_bytes);
    p.scale_log2 = (float)((double)scale * 1.4426950408889634);
    p.inverse_g = 1.0f / (float)(q->heads / cache->heads);
    p.N = (int)N;
    p.B = (int)B;
    p.Hk = cache->heads;
    p.G = q->heads / cache->heads;
    p.D = (int)D;
    p.page_log = log2_of(cache->page_size);
    p.pages = (int)cache->pages;
    p.max_len = (int)max_len;
    p.window = (int)(window ? window : kMost);
    p.few_rows = a.few ? a.few_row_places : 0;
    p.few_splits = a.few_splits;
    p.few_chunk = a.few_chunk;
    p.few_per_xcd = a.few_per_xcd;
    p.many_splits = a.many_splits;
    p.many_chunk = a.many_chunk;
    p.many_tiles = a.many_tiles;
    p.many_per_xcd = a.many_per_xcd;
    if (out->type == VLUT_TYPE_F32) return cache->type == VLUT_TYPE_BF16 ? launch_bf16_f32(a, p, (hipStream_t)stream) : launch_f16_f32(a, p, (hipStream_t)stream);
    return cache->type == VLUT_TYPE_BF16 ? launch_bf16(a, p, (hipStream_t)stream) : launch_f16(a, p, (hipStream_t)stream);
}

}  // extern "C"
