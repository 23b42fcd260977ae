// Between the projections of a decoder layer, for MI355X (gfx950): norms and rotation of heads, the paged cache, attention over a shared prefix.
// The heads' kernels, the host side of the attention, and their part of the C ABI; a translation unit beside vlut.hip, as those of the attention's kernels.
#include <hip/hip_runtime.h>

#include <algorithm>
#include <cmath>
#include <cstdint>

#include "vlut.h"

#include "attention_params.h"
#include "common.hip.h"
#include "host_checks.h"
#include "launch.hip.h"
#include "heads_kernel.hip.h"

namespace {

using namespace vlut_attention;

constexpr int kUnits = 256;            // compute units that a launch is to fill
constexpr int64_t kMostBlocks = 1 << 24;       // of 256 threads

// ---------------------------------------------------------------------------------------------
// Heads
// ---------------------------------------------------------------------------------------------
// The checks that norm_rope and append_kv share; fills in p but for where rows go.
int heads_params(HeadsParams& p, const vlut_heads* const (&in)[3], float eps, const vlut_rotation* rot, int64_t N, int64_t D, Alignment& a) {
    if (N < 1 || N >= kMaxDim || D < 2 || D > VLUT_MAX_HEAD_FEATURES || D % 2) return VLUT_ERR_SHAPE;
    if (!(eps >= 0.0f)) return VLUT_ERR_SHAPE;
    int64_t heads = 0;
    a.stride(D / 2);
    int type = -1;
    for (int i = 0; i < 3; ++i) {
        p.kind[i] = HeadRows{};
        if (!in[i]) continue;
        if (!in[i]->data) return VLUT_ERR_NULL;
        if (in[i]->heads < 1 || in[i]->heads >= (1 << 16) || !type_ok(in[i]->type) || (type >= 0 && in[i]->type != type)) return VLUT_ERR_SHAPE;
        type = in[i]->type;
        heads += in[i]->heads;
        HeadRows& k = p.kind[i];
        k.in = in[i]->data;
        k.in_token = in[i]->token_stride;
        k.in_head = in[i]->head_stride;
        k.heads = in[i]->heads;
        a.pointer(k.in, type_bytes(type));
        a.stride(k.in_token);
        a.stride(k.in_head);
        if (i < 2) {
            k.weight = in[i]->weight;
            k.weight_head = in[i]->weight_stride;
            if (k.weight) {
                a.pointer(k.weight, 4);
                a.stride(k.weight_head);
            }
        }
    }
    p.R = 0;
    p.cos = p.sin = nullptr;
    p.positions = nullptr;
    p.table_rows = 0;
    p.interleaved = 0;
    if (rot) {
        if (!rot->cos || !rot->sin || !rot->positions) return VLUT_ERR_NULL;
        if (rot->features < 2 || rot->features > D || rot->features % 2 || rot->rows < 1) return VLUT_ERR_SHAPE;
        p.R = rot->features;
        p.cos = rot->cos;
        p.sin = rot->sin;
        p.positions = rot->positions;
        p.table_rows = rot->rows;
        p.interleaved = rot->interleaved != 0;
        a.pointer(p.cos, 4);
        a.pointer(p.sin, 4);
        a.stride(p.R / 2);
    }
    p.eps = eps;
    p.D = (int)D;
    p.heads = (unsigned)heads;
    p.slots = nullptr;
    p.slot_end = 0;
    p.page_log = 0;
    if (N * heads >= ((int64_t)1 << 31)) return VLUT_ERR_SHAPE;
    p.tokens = (unsigned)N;
    return VLUT_OK;
}

template <class TI, class TO>
int launch_heads_t(const HeadsParams& p, int vec, int together, dim3 grid, hipStream_t stream) {
    if (vec == 4) return together > 1 ? launch(heads_kernel<TI, TO, 4, 2>, grid, 256, 0, stream, p) : launch(heads_kernel<TI, TO, 4, 1>, grid, 256, 0, stream, p);
    if (vec == 2) return together > 1 ? launch(heads_kernel<TI, TO, 2, 4>, grid, 256, 0, stream, p) : launch(heads_kernel<TI, TO, 2, 1>, grid, 256, 0, stream, p);
    return launch(heads_kernel<TI, TO, 1, 1>, grid, 256, 0, stream, p);
}
template <class TI>
int launch_heads_out(const HeadsParams& p, int out, int vec, int together, dim3 grid, hipStream_t stream) {
    if (out == VLUT_TYPE_F32) return launch_heads_t<TI, float>(p, vec, together, grid, stream);
    if (out == VLUT_TYPE_BF16) return launch_heads_t<TI, __bf16>(p, vec, together, grid, stream);
    return launch_heads_t<TI, _Float16>(p, vec, together, grid, stream);
}
int launch_heads(HeadsParams& p, int in, int out, int vec, hipStream_t stream) {
    // lanes of a row: enough for its units (at most 64; a lane has two where pairs are single)
    p.lanes_log = std::min(6, log2_of((p.D + 2 * vec - 1) / (2 * vec)));
    const unsigned per = 256u >> p.lanes_log;
    // Heads together where rows are enough for two workgroups of such groups on every unit.  us for one / two / four together, 4096 tokens: 40 heads of
    // 128 from fp32 28.2 / 27.5 / 27.8, 16 heads to a cache 12.0 / 11.5 / 12.3, 64 heads of 100 (vectors of two) 57.5 / 48.5 / 45.0.
    const int most = vec == 4 ? 2 : (vec == 2 ? 4 : 1), together = (uint64_t)p.tokens * p.heads >= 8ull * kUnits * per ? most : 1;
    unsigned blocks = 0;
    for (HeadRows& k : p.kind) {
        k.groups_of_token = (unsigned)((k.heads + together - 1) / together);
        k.groups = p.tokens * k.groups_of_token;
        blocks += (k.groups + per - 1) / per;
        k.end_block = blocks;
    }
    // A launch's threads are numbered in 32 bits: more are several launches.
    constexpr unsigned most_blocks = 1u << 23;
    int rc = VLUT_OK;
    for (p.first_block = 0; rc == VLUT_OK && p.first_block < blocks; p.first_block += most_blocks) {
        const dim3 grid(std::min(blocks - p.first_block, most_blocks));
        if (in == VLUT_TYPE_F32) rc = launch_heads_out<float>(p, out, vec, together, grid, stream);
        else if (in == VLUT_TYPE_BF16) rc = launch_heads_out<__bf16>(p, out, vec, together, grid, stream);
        else rc = launch_heads_out<_Float16>(p, out, vec, together, grid, stream);
    }
    return rc;
}

// Rows that go to a tensor of their own.
int rows_out(HeadRows& k, const vlut_heads* out, int type, Alignment& a) {
    if (!out || !out->data) return VLUT_ERR_NULL;
    if (out->heads != k.heads || out->type != type) return VLUT_ERR_SHAPE;
    k.out = (void*)out->data;
    k.out_token = out->token_stride;
    k.out_head = out->head_stride;
    a.pointer(k.out, type_bytes(type));
    a.stride(k.out_token);
    a.stride(k.out_head);
    return VLUT_OK;
}

// ---------------------------------------------------------------------------------------------
// Attention
// ---------------------------------------------------------------------------------------------

// grouped: 16 keys share their page, as the kernel for many rows wants it.  neighbours: a token's heads are neighbours in memory.
int plan_attention(int64_t B, int64_t n, int64_t Hq, int64_t Hk, int64_t D, int64_t P, int64_t max_own, bool grouped, bool neighbours, AttendPlan* out) {
    if (B < 1 || n < 1 || Hk < 1 || Hq < 1 || Hq >= (1 << 16) || Hq % Hk || B >= kMaxDim || n >= kMaxDim) return VLUT_ERR_SHAPE;
    if (P < 0 || max_own < 0 || P >= ((int64_t)1 << 30) || max_own >= ((int64_t)1 << 30) || D < 1) return VLUT_ERR_SHAPE;
    if (D < 8 || D > VLUT_MAX_HEAD_FEATURES || D % 4) return VLUT_ERR_UNSUPPORTED;
    const int64_t G = Hq / Hk, own_rows = n * G, rows = own_rows < ((int64_t)1 << 30) ? B * own_rows : own_rows;       // (below 2^54)
    if (rows >= ((int64_t)1 << 30) || rows * Hk >= ((int64_t)1 << 30)) return VLUT_ERR_SHAPE;
    AttendPlan a{};
    a.grouped = grouped;
    a.own_heads_together = neighbours ? (int)Hk : 1;
    a.rows = rows;
    a.DP = D <= 64 ? 64 : (D <= 128 ? 128 : 256);
    a.own_mt = own_rows <= 16 || a.DP > 128 ? 1 : 2;        // (of 256 features two tiles' O and queries do not fit the registers)
    // Tiles of 16 or 32 rows whose waves share the keys, or, where the prefix' products are many, a launch of its own with 32 rows a wave.  us, by tiles /
    // that launch, 8 key heads, for bf16 outputs (fp32): 128 features, 256 rows a head, 2048 keys 22 / 30 (23 / 33), 4096 28 / 34 (29 / 36), 6000 32 / 33
    // (33 / 36), 8192 39 / 37 (40 / 40), 12000 50 / 42 (51 / 47); 512 rows, 2048 keys 24 / 34, 4096 34 / 37 (37 / 41), 6000 44 / 42 (48 / 47); 64 features, 256
    // rows, 8192 keys 26 / 30 (29 / 32), 12000 33 / 31 (37 / 34), 16384 41 / 34 (48 / 38); 256 features, 256 rows, 1024 keys 28 / 39, 2048 45 / 41, 4096
    // 65 / 44 (66 / 46); 128 rows, 3900 keys 34 / 39; one key head, 800 rows, 4096 keys 28 / 41, 6000 37 / 44, 8192 46 / 45.
    // (The two meet at half as many products again as said here, where up to a tenth of the time lies between them, now that the launch's weights have a
    // term more than when the limit was set.)
    const int64_t few_products = a.DP > 128 ? 3500000 : 1280000000 / a.DP;
    const bool many = P > 0 && rows > 64 && grouped && rows * P * Hk > few_products;
    // Tiles of 16 where 32 would read less but a step per workgroup is about all there is: us, 32 / 16, 8 key heads of 128: 64 rows a head, 2048 keys, own 512
    // 16.5 / 15.2; 256 rows, 500 keys, own 100 17.7 / 15.9; 5 key heads, 64 rows, 2048 keys, own 256 13.9 / 12.9.  (64 rows, 8192 keys 22.8 / 23.4; 128
    // rows, 8192 keys 23.4 / 28.5.)  Of 256 features 32 rows would not fit the registers: 64 rows, 4096 keys 35.6 / 30.3.
    const bool few_steps = own_rows <= 16 && Hk * ceil_div(rows, 16) * ceil_div(P, 128) + B * Hk * ceil_div(max_own, 128) <= 4 * kUnits;
    a.MT = many ? 0 : (P == 0 ? a.own_mt : (rows <= 16 || few_steps || a.DP > 128 ? 1 : 2));
    a.waves = a.MT == 0 && a.DP <= 128 && rows > 128 ? 8 : 4;
    a.own_tiles = (int)ceil_div(own_rows, 16 * a.own_mt);
    const int64_t own_units = B * Hk * a.own_tiles;
    const int64_t slots = kUnits * few_waves(a.DP, a.MT == 0 ? a.own_mt : a.MT);            // workgroups of four waves that run at once
    // Waves to a range of own tokens: as many as have a step in it and as leave the workgroups of all ranges room at once.  (24 sequences of 150
    // to 300 tokens, 32 heads of 100, a range a head: 4 waves 31.7 us, in two rounds; 2 waves, in one, 25.8 us.)
    a.own_share = 4;
    while (a.own_share > 1 && (kFewKeys * a.own_share / 2 >= max_own || own_units * a.own_share > 4 * slots)) a.own_share /= 2;
    a.own_step = a.own_share * kFewKeys;
    const int64_t own_steps = ceil_div(max_own, a.own_step);
    const auto own_blocks = [&](int64_t splits) { return ceil_div(ceil_div(B * splits * Hk / a.own_heads_together, 8) * a.own_heads_together * a.own_tiles, 4 / a.own_share) * 8; };
    int64_t per_own;
    if (a.MT > 0) {                            // steps per range: the fewest with which all workgroups run at once
        a.prefix_tiles = (int)ceil_div(rows, 16 * a.MT);
        const int64_t steps = ceil_div(P, 128), most = std::max(steps, own_steps);
        const auto blocks = [&](int64_t per) { return ceil_div(Hk * a.prefix_tiles * ceil_div(steps, per), 8) * 8 + own_blocks(ceil_div(own_steps, per)); };
        int64_t per = std::max<int64_t>(1, ceil_div(Hk * a.prefix_tiles * steps + ceil_div(own_units * own_steps, 4 / a.own_share), slots));
        for (int more = 0; more < 8 && per < most && blocks(per) > slots; ++more) ++per;
        a.prefix_chunk = (int)(128 * std::min(per, std::max<int64_t>(1, steps)));       // (`per` may be any number where rows are many)
        per_own = own_blocks(1) >= slots ? std::max<int64_t>(1, own_steps) : per;
    } else {
        a.prefix_tiles = (int)ceil_div(rows, 32 * a.waves);
        const int64_t keys = many_keys(a.DP), splits = std::min(std::max<int64_t>(1, 8 / a.waves * kUnits / (Hk * a.prefix_tiles)), ceil_div(P, 256));
        a.prefix_chunk = (int)(ceil_div(ceil_div(P, splits), keys) * keys);
        per_own = std::max<int64_t>(1, ceil_div(own_steps, std::max<int64_t>(1, slots / own_blocks(1))));
    }
    a.prefix_splits = P > 0 ? (int)ceil_div(P, a.prefix_chunk) : 0;
    a.own_splits = (int)ceil_div(own_steps, per_own);
    if (a.prefix_splits + a.own_splits == 0) a.own_splits = 1;      // nothing is seen: a workgroup stores that
    const int64_t prefix_blocks = ceil_div(Hk * a.prefix_tiles * a.prefix_splits, 8) * 8, own_all = own_blocks(a.own_splits);
    const int parts_log = log2_of(ceil_div(a.prefix_splits + a.own_splits, 4)), groups_log = log2_of(1024 / a.DP);      // (combine_kernel's)
    a.combine_lanes_log = std::min(groups_log, parts_log);
    const int64_t combine_blocks = ceil_div(rows * Hk, 1 << (groups_log - a.combine_lanes_log));
    // A launch's threads are numbered in 32 bits.
    if (a.MT > 0 ? prefix_blocks + own_all >= kMostBlocks : (own_all >= kMostBlocks || prefix_blocks * a.waves / 4 >= kMostBlocks)) return VLUT_ERR_SHAPE;
    a.prefix_per_xcd = (int)(prefix_blocks / 8);
    a.own_per_xcd = (int)(own_all / 8);
    a.direct = a.MT > 0 && a.prefix_splits + a.own_splits == 1;
    if (!a.direct) {
        if (combine_blocks >= kMostBlocks) return VLUT_ERR_SHAPE;
        a.combine_blocks = (int)combine_blocks;
        const size_t parts = (size_t)(a.prefix_splits + a.own_splits) * (size_t)Hk * (size_t)rows;
        a.o_bytes = (parts * (size_t)D * 4 + 255) & ~(size_t)255;
        a.ml_bytes = parts * 8;
    }
    *out = a;
    return VLUT_OK;
}

// Sixteen keys share their page, and strides and the offsets inside a page fit 31 bits, in bytes.
bool grouped_keys(const vlut_cache& c) {
    bool ok = c.page_size >= 16;
    for (int64_t s : {c.k_page_stride, c.v_page_stride}) ok = ok && s >= 0 && s < ((int64_t)1 << 30);
    for (int64_t s : {c.k_token_stride, c.v_token_stride}) ok = ok && s >= 0 && s < ((int64_t)1 << 30) / std::max<int64_t>(c.page_size, 16);
    return ok;
}

}  // namespace

extern "C" {

int vlut_norm_rope(const vlut_heads* q, const vlut_heads* k_or_null, float eps, const vlut_rotation* rotation_or_null, int64_t N, int64_t D,
                   const vlut_heads* q_out, const vlut_heads* k_out_or_null, void* stream) {
    if (!q || !q_out || !k_or_null != !k_out_or_null) return VLUT_ERR_NULL;
    HeadsParams p;
    Alignment a;
    const vlut_heads* const in[3] = {q, k_or_null, nullptr};
    int rc = heads_params(p, in, eps, rotation_or_null, N, D, a);
    if (rc != VLUT_OK) return rc;
    if (!type_ok(q_out->type)) return VLUT_ERR_SHAPE;
    if ((rc = rows_out(p.kind[0], q_out, q_out->type, a)) != VLUT_OK) return rc;
    if (k_or_null && (rc = rows_out(p.kind[1], k_out_or_null, q_out->type, a)) != VLUT_OK) return rc;
    return launch_heads(p, q->type, q_out->type, a.vec, (hipStream_t)stream);
}

int vlut_append_kv(const vlut_heads* k, const vlut_heads* v, const vlut_heads* q_or_null, float eps, const vlut_rotation* rotation_or_null,
                   const int64_t* slots, int64_t N, int64_t D, const vlut_cache* cache, const vlut_heads* q_out_or_null, void* stream) {
    if (!k || !v || !slots || !q_or_null != !q_out_or_null) return VLUT_ERR_NULL;
    int rc = check_cache(cache);
    if (rc != VLUT_OK) return rc;
    HeadsParams p;
    Alignment a;
    const vlut_heads* const in[3] = {q_or_null, k, v};
    rc = heads_params(p, in, eps, rotation_or_null, N, D, a);
    if (rc != VLUT_OK) return rc;
    if (k->heads != cache->heads || v->heads != cache->heads) return VLUT_ERR_SHAPE;
    if (q_or_null && (rc = rows_out(p.kind[0], q_out_or_null, cache->type, a)) != VLUT_OK) return rc;
    for (int i = 1; i < 3; ++i) {
        HeadRows& r = p.kind[i];
        r.by_slot = 1;
        r.out = i == 1 ? cache->k : cache->v;
        r.out_token = i == 1 ? cache->k_page_stride : cache->v_page_stride;
        r.out_head = i == 1 ? cache->k_head_stride : cache->v_head_stride;
        r.out_row = i == 1 ? cache->k_token_stride : cache->v_token_stride;
        a.pointer(r.out, 2);
        a.stride(r.out_token);
        a.stride(r.out_head);
        a.stride(r.out_row);
    }
    p.slots = slots;
    p.slot_end = cache->pages * cache->page_size;
    p.page_log = log2_of(cache->page_size);
    return launch_heads(p, k->type, cache->type, a.vec, (hipStream_t)stream);
}

size_t vlut_shared_prefix_attention_bytes(int64_t B, int64_t n, int64_t Hq, int64_t Hk, int64_t D, int64_t prefix_len, int64_t max_own_len) {
    size_t most = 0;                   // (of any cache)
    for (int kind = 0; kind < 4; ++kind) {
        AttendPlan a;
        if (plan_attention(B, n, Hq, Hk, D, prefix_len, max_own_len, kind & 1, kind & 2, &a) != VLUT_OK) return 0;
        most = std::max(most, a.o_bytes + a.ml_bytes);
    }
    return most;
}

int vlut_query_shared_prefix_attention(int64_t B, int64_t n, int64_t Hq, int64_t Hk, int64_t D, int64_t prefix_len, int64_t max_own_len, int* out4) {
    if (!out4) return VLUT_ERR_NULL;
    AttendPlan a;
    const int rc = plan_attention(B, n, Hq, Hk, D, prefix_len, max_own_len, true, false, &a);
    if (rc != VLUT_OK) return rc;
    out4[0] = a.MT > 0 ? 16 * a.MT : 32 * a.waves;
    out4[1] = a.prefix_splits;
    out4[2] = a.own_splits;
    out4[3] = 8 * (a.prefix_per_xcd + a.own_per_xcd);
    return VLUT_OK;
}

int vlut_shared_prefix_attention(const vlut_heads* q, int64_t q_sequence_stride, const vlut_cache* cache, const int32_t* prefix_pages, int64_t prefix_len,
                                 const int32_t* page_table, int64_t table_stride, const int32_t* own_lens, int64_t max_own_len,
                                 const int32_t* query_lens_or_null, int64_t B, int64_t n, int64_t D, float scale, const vlut_heads* out,
                                 int64_t out_sequence_stride, float* lse_or_null, void* workspace, size_t workspace_bytes, void* stream) {
    if (!q || !out) return VLUT_ERR_NULL;
    int rc = check_cache(cache);
    if (rc != VLUT_OK) return rc;
    AttendPlan a;
    rc = plan_attention(B, n, q->heads, cache->heads, D, prefix_len, max_own_len, grouped_keys(*cache), cache->k_head_stride < cache->k_token_stride, &a);
    if (rc != VLUT_OK) return rc;
    if (!q->data || !out->data || !own_lens || (prefix_len > 0 && !prefix_pages) || (max_own_len > 0 && !page_table)) return VLUT_ERR_NULL;
    if (out->heads != q->heads || q->type != cache->type || (out->type != cache->type && out->type != VLUT_TYPE_F32)) return VLUT_ERR_SHAPE;
    if (cache->pages >= ((int64_t)1 << 31)) return VLUT_ERR_SHAPE;
    if (!(scale > 0.0f) || !std::isfinite(scale)) return VLUT_ERR_UNSUPPORTED;
    if (!at_dwords(q->data, q_sequence_stride, q->token_stride, q->head_stride, 2) ||
        !at_dwords(cache->k, cache->k_page_stride, cache->k_head_stride, cache->k_token_stride, 2) ||
        !at_dwords(cache->v, cache->v_page_stride, cache->v_head_stride, cache->v_token_stride, 2) ||
        !at_dwords(out->data, out_sequence_stride, out->token_stride, out->head_stride, type_bytes(out->type)))
        return VLUT_ERR_UNSUPPORTED;
    if (a.o_bytes) {
        if (!workspace) return VLUT_ERR_NULL;
        if (workspace_bytes < a.o_bytes + a.ml_bytes) return VLUT_ERR_SMALL_BUFFER;
        if ((uintptr_t)workspace % 16) return VLUT_ERR_UNSUPPORTED;
    }
    AttendParams p{};
    p.q = q->data;
    p.k = cache->k;
    p.v = cache->v;
    p.q_sequence = q_sequence_stride;
    p.q_token = q->token_stride;
    p.q_head = q->head_stride;
    p.k_page = cache->k_page_stride;
    p.k_head = cache->k_head_stride;
    p.k_token = cache->k_token_stride;
    p.v_page = cache->v_page_stride;
    p.v_head = cache->v_head_stride;
    p.v_token = cache->v_token_stride;
    p.prefix_pages = prefix_pages;
    p.page_table = page_table;
    p.own_lens = own_lens;
    p.query_lens = query_lens_or_null;
    p.table_stride = table_stride;
    p.out = (void*)out->data;
    p.out_sequence = out_sequence_stride;
    p.out_token = out->token_stride;
    p.out_head = out->head_stride;
    p.lse = lse_or_null;
    p.part_o = (float*)workspace;
    p.part_ml = (float*)((unsigned char*)workspace + a.o_bytes);
    p.scale_log2 = (float)((double)scale * 1.4426950408889634);
    p.out_type = out->type;
    p.B = (int)B;
    p.n = (int)n;
    p.Hk = cache->heads;
    p.G = q->heads / cache->heads;
    p.D = (int)D;
    p.page_log = log2_of(cache->page_size);
    p.pages = (int)cache->pages;
    p.P = (int)prefix_len;
    p.max_own = (int)max_own_len;
    p.prefix_splits = a.prefix_splits;
    p.prefix_chunk = a.prefix_chunk;
    p.own_splits = a.own_splits;
    p.own_share = a.own_share;
    p.own_heads_together = a.own_heads_together;
    p.own_step = a.own_step;
    p.prefix_tiles = a.prefix_tiles;
    p.own_tiles = a.own_tiles;
    p.prefix_per_xcd = a.prefix_per_xcd;
    p.own_per_xcd = a.own_per_xcd;
    p.rows = (int)a.rows;
    p.direct = a.direct;
    return cache->type == VLUT_TYPE_BF16 ? launch_bf16(a, p, (hipStream_t)stream) : launch_f16(a, p, (hipStream_t)stream);
}

}  // extern "C"
