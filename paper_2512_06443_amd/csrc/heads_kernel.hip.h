// Norms of query and key heads, the rotation by position, and the way of keys and values into a paged cache: one pass over the heads.
// Part of the translation unit attention.hip (included there, in this order).
#pragma once

#include "vectors.hip.h"

namespace {

// ---------------------------------------------------------------------------------------------
// A row is one head of one token, D features:
//   y = x / sqrt(mean(x^2) + eps) * w          (without a weight: y = x)
//   (a, b) -> (a cos - b sin, b cos + a sin)   for the R / 2 pairs of the first R features, (i, i + R/2) or (2i, 2i + 1)
// all in fp32, rounded once where it is stored.  The rows of a token are its query heads, then its key heads, then its value heads (which
// are only converted); each goes to a tensor or, by the token's slot, into a page.  A workgroup has rows of one kind.
// A unit is two vectors of VEC features that rotate with each other (or, past R, two neighbouring ones), and a lane has one unit (two
// of VEC = 1): a pair never leaves its lane, and the only exchange is the sum of squares over the row's 2^lanes_log lanes.
// Bound by memory: every row is read once and written once, the tables once per token and kind.  4096 tokens, 40 heads of 128 features, fp32 to bf16,
// 128 MB: 25.9 us, 4.9 TB/s (a large copy: 5.3); 16 heads to a cache, 50 MB: 10.4 us, 4.8 TB/s; one token: 2.5 us, a launch.
// ---------------------------------------------------------------------------------------------
struct HeadRows {              // what the rows of one kind (queries, keys, values) are read from and written to; strides in elements
    const void* in;
    const float* weight;       // null: no norm
    void* out;
    int64_t in_token, in_head, weight_head;
    int64_t out_token, out_head;       // out_token: of a page where the rows go by slots
    int64_t out_row;                   // of a token inside its page
    int heads, by_slot;
    unsigned groups, groups_of_token, end_block;       // groups of HEADS heads: all, of a token; the first workgroup behind the kind's
};

struct HeadsParams {
    HeadRows kind[3];
    const float *cos, *sin;
    const int64_t *positions, *slots;
    int64_t table_rows, slot_end;
    float eps;
    unsigned tokens, heads;    // heads of all kinds per token
    unsigned first_block;      // of this launch
    int D, R, interleaved, lanes_log, page_log;
};

// HEADS neighbouring heads of a token per group of lanes, whose loads are on their way together and whose rotation is loaded once.
template <class TI, class TO, int VEC, int HEADS>
__global__ void __launch_bounds__(256) heads_kernel(const HeadsParams p) {
    constexpr int UNITS = VEC == 1 ? 2 : 1;         // of a lane: D <= 256 has at most 128 units of one pair
    const int lane = (int)threadIdx.x & ((1 << p.lanes_log) - 1);
    const unsigned at_block = p.first_block + blockIdx.x;
    const int which = at_block < p.kind[0].end_block ? 0 : (at_block < p.kind[1].end_block ? 1 : 2);
    const HeadRows& k = p.kind[which];
    const unsigned block = at_block - (which == 0 ? 0u : p.kind[which - 1].end_block), group = block * (256u >> p.lanes_log) + (threadIdx.x >> p.lanes_log);
    const bool alive = group < k.groups;
    const unsigned r = alive ? group : k.groups - 1;        // (the exchange below wants every lane)
    const unsigned token = r / k.groups_of_token;
    const int first = (int)(r - token * k.groups_of_token) * HEADS;
    const int half = p.R / 2, rotating = half / VEC, units = p.D / (2 * VEC);
    int at[UNITS][2];
#pragma unroll
    for (int s = 0; s < UNITS; ++s) {
        const int u = lane + (s << p.lanes_log);
        const bool halves = u < rotating && !p.interleaved;
        at[s][0] = halves ? u * VEC : u * 2 * VEC;
        at[s][1] = halves ? half + u * VEC : at[s][0] + VEC;
    }
    float x[HEADS][UNITS][2][VEC];
    const TI* const in = (const TI*)k.in + (int64_t)token * k.in_token;
#pragma unroll
    for (int i = 0; i < HEADS; ++i) {
        const TI* const row = in + min(first + i, k.heads - 1) * k.in_head;
#pragma unroll
        for (int s = 0; s < UNITS; ++s)
            if (lane + (s << p.lanes_log) < units) {
#pragma unroll
                for (int h = 0; h < 2; ++h) load_floats<TI, VEC>(x[i][s][h], row + at[s][h]);
            }
    }
    bool placed = true;                             // inside the rotation's tables
    float c[UNITS][VEC], n[UNITS][VEC];
    const bool rotated = which < 2 && p.R > 0;
    if (rotated) {
        int64_t position = p.positions[token];
        placed = position >= 0 && position < p.table_rows;
        position = placed ? position : 0;
#pragma unroll
        for (int s = 0; s < UNITS; ++s) {
            const int u = lane + (s << p.lanes_log);
            if (u >= rotating) continue;
            load_floats<float, VEC>(c[s], p.cos + position * half + u * VEC);
            load_floats<float, VEC>(n[s], p.sin + position * half + u * VEC);
            if (!placed) {
#pragma unroll
                for (int i = 0; i < VEC; ++i) c[s][i] = n[s][i] = __builtin_nanf("");
            }
        }
    }
    bool kept = alive;
    int64_t to = (int64_t)token * k.out_token;
    if (k.by_slot) {
        const int64_t slot = p.slots[token];
        kept = alive && slot >= 0 && slot < p.slot_end;
        to = (slot >> p.page_log) * k.out_token + (slot & ((1 << p.page_log) - 1)) * k.out_row;
    }
#pragma unroll
    for (int i = 0; i < HEADS; ++i) {
        float squares = 0.0f;
#pragma unroll
        for (int s = 0; s < UNITS; ++s)
            if (lane + (s << p.lanes_log) < units) {
#pragma unroll
                for (int h = 0; h < 2; ++h)
#pragma unroll
                    for (int e = 0; e < VEC; ++e) squares += x[i][s][h][e] * x[i][s][h][e];
            }
        for (int m = 1 << p.lanes_log >> 1; m; m >>= 1) squares += __shfl_xor(squares, m);
        const float inverse = 1.0f / sqrtf(squares / (float)p.D + p.eps);
        if (!kept || first + i >= k.heads) continue;
        TO* const out = (TO*)k.out + to + (first + i) * k.out_head;
#pragma unroll
        for (int s = 0; s < UNITS; ++s) {
            const int u = lane + (s << p.lanes_log);
            if (u >= units) continue;
            float (&y)[2][VEC] = x[i][s];
            if (k.weight) {
#pragma unroll
                for (int h = 0; h < 2; ++h) {
                    float w[VEC];
                    load_floats<float, VEC>(w, k.weight + (first + i) * k.weight_head + at[s][h]);
#pragma unroll
                    for (int e = 0; e < VEC; ++e) y[h][e] = y[h][e] * inverse * w[e];
                }
            }
            if (rotated && u < rotating) {
                if (p.interleaved && VEC > 1) {
                    float* const flat = &y[0][0];   // pairs of neighbours through both vectors
#pragma unroll
                    for (int e = 0; e < VEC; ++e) {
                        const float a = flat[2 * e], b = flat[2 * e + 1];
                        flat[2 * e] = a * c[s][e] - b * n[s][e];
                        flat[2 * e + 1] = b * c[s][e] + a * n[s][e];
                    }
                } else {
#pragma unroll
                    for (int e = 0; e < VEC; ++e) {
                        const float a = y[0][e], b = y[1][e];
                        y[0][e] = a * c[s][e] - b * n[s][e];
                        y[1][e] = b * c[s][e] + a * n[s][e];
                    }
                }
            }
#pragma unroll
            for (int h = 0; h < 2; ++h) store_floats<TO, VEC>(out + at[s][h], y[h]);
        }
    }
}

}  // namespace
