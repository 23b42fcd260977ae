// Attention of chunks of new tokens, packed one sequence behind the other, over a paged cache.
// Part of the translation units chunk_bf16.hip and chunk_f16.hip (included there, in this order).
#pragma once

#include "matrix_parts.hip.h"

namespace {

using namespace vlut_chunk;

// ---------------------------------------------------------------------------------------------
// Query j of a sequence with n new tokens and len tokens in all has position pos = len - n + j and sees the keys max(0, pos - window + 1) .. pos:
//   s = scale * q . k,  m a number near max s,  l = sum exp(s - m),  O = sum exp(s - m) v,  output O / l;   nothing seen: 0
// A row is a query token and one of the G query heads that read a key head, token by token, so that the rows of a tile are neighbours in position and see
// nearly the same keys.  A workgroup has a tile of rows of one sequence and key head and a part of the keys that any of them sees.
//   Many rows: RW waves of 32 rows, whose keys and values go through LDS for all of them, 64 keys a step.
//   Few rows (up to 32: single tokens, drafts): one tile of 32 rows and KW waves that share a step's keys, 32 each; they meet in LDS at the end.
// A sequence's tile of more keys than a part holds is several workgroups; combine_chunks joins the parts: with M = max m_i the sums of exp(m_i - M) l_i and
// exp(m_i - M) O_i are those of the whole.
//
// Both products run transposed on the matrix cores, S^T = K Q^T and O^T = V^T P^T: a query is a column, its m and l are one number per lane, and P^T goes from
// one product to the next in its registers, the keys of both in the order in which S^T comes out.  V^T is read out of the row-major V in LDS by
// transposing reads.
// m is not the running maximum: it is the largest score of the first step in which the row sees anything, and stays, so that nothing but sums is in the loop
// and O is never multiplied.  Weights are powers of two of the scores above m and may be as large as their type's range; where that does not do (bf16: l
// shows 2^40 or O leaves fp32; fp16: O is no number) the part is begun again with the largest of all its scores, which a sweep over K finds.
// P goes to the second product in the cache's type.  For 16-bit outputs that is one rounding more of the size of the output's own, of terms whose errors
// are independent (bf16 2.3e-3 of the result instead of 1.7e-3); for fp32 it is carried in further terms, each what the rounding of those before it left: 24 bits, three of bf16
// or two of fp16.
// ---------------------------------------------------------------------------------------------

struct Chunk {                         // of a sequence: its first token's row and position; bad: a length that cannot be
    int start, queries, len, base, bad;
};
__device__ __forceinline__ Chunk chunk_of(const ChunkParams& p, int b) {
    Chunk c;
    c.start = p.starts[b];
    const int next = p.starts[b + 1];
    c.queries = c.start >= 0 && next >= c.start && next <= p.N ? next - c.start : 0;
    c.len = p.lens[b];
    c.bad = c.len < 0 || c.len > p.max_len;
    if (c.bad) c.len = 0;
    c.base = c.len - c.queries;
    return c;
}
// The keys that any of the queries j0 .. j1 sees, from a multiple of 32 on, and the parts that they are.
struct Range {
    int first, end, parts;
};
__device__ __forceinline__ Range range_of(const ChunkParams& p, const Chunk& c, int j0, int j1, int keys_of_part) {
    Range r;
    r.end = min(c.len, max(0, c.base + j1 + 1));
    r.first = min(max(0, c.base + j0 - p.window + 1), r.end) & ~31;
    r.parts = max(1, (int)(((unsigned)(r.end - r.first) + (unsigned)keys_of_part - 1) / (unsigned)keys_of_part));
    return r;
}

__device__ __forceinline__ void store_four(const ChunkParams& p, int64_t at, const f32x4& o) {
    if (p.out_type == VLUT_TYPE_F32) *(dword_aligned_f32x4*)((float*)p.out + at) = o;
    else if (p.out_type == VLUT_TYPE_BF16) {
        typedef __bf16 x4 __attribute__((ext_vector_type(4), aligned(4)));
        *(x4*)((__bf16*)p.out + at) = x4{(__bf16)o.x, (__bf16)o.y, (__bf16)o.z, (__bf16)o.w};
    } else {
        typedef _Float16 x4 __attribute__((ext_vector_type(4), aligned(4)));
        *(x4*)((_Float16*)p.out + at) = x4{(_Float16)o.x, (_Float16)o.y, (_Float16)o.z, (_Float16)o.w};
    }
}

// What a workgroup works on.
struct Tile {
    Chunk seq;
    int b, h, row0, row_end;           // rows of the sequence and key head: query * G + head
    int first, end;                    // keys
    int split, direct;
};
// Where row `row` of a tile's part is among the parts.
template <bool FEW>
__device__ __forceinline__ int64_t part_at(const ChunkParams& p, const Chunk& c, int b, int h, int row, int split, int places) {
    if constexpr (FEW) return (((int64_t)split * p.B + b) * p.Hk + h) * places + row;
    const int j = row / p.G;
    return ((int64_t)split * p.N + c.start + j) * (p.Hk * p.G) + h * p.G + row - j * p.G;
}

// Values that are no numbers.  Zeros stand for them in the products' steps of which some row does not see every key (0 times them would reach every row); they, and
// infinities that rows see, which weights of 0 or in several terms make NaN of, are settled here, once the results are stored, by a look at the part's values: a row's
// feature with such values among the keys that it sees is their sum, with weights of 1, or 0 for a score of -inf.  NaN with infinities of both signs.
// Rows: those of `rows` (bits, from row0 on).  Not part of the loops: a flag and a look at the results; where there is something to settle, a read of V per wave.
template <class T, int DP, bool FEW>
__device__ __forceinline__ void settle_chunk(const ChunkParams& p, const Tile& t, int row0, unsigned rows) {
    constexpr int F = DP / 64;
    const int lane = (int)threadIdx.x & 63, d = F * lane, mask = (1 << p.page_log) - 1;
    const bool has = d < p.D;
    const int32_t* const pages = p.page_table + t.b * p.table_stride;
    auto token = [&](const void* of, int key, int64_t page_stride, int64_t head_stride, int64_t token_stride) {
        const int id = pages[key >> p.page_log];
        return (const T*)of + ((unsigned)id < (unsigned)p.pages ? id : 0) * page_stride + t.h * head_stride + (key & mask) * token_stride + d;
    };
    unsigned touched[F] = {};                  // rows whose feature has been set
    for (int key = t.first; key < t.end; ++key) {
        const T* const v = token(p.v, key, p.v_page, p.v_head, p.v_token);
        bool odd = false;
        float x[F] = {};
        for (int f = 0; f < F && has; ++f) {
            x[f] = d + f < p.D ? (float)v[f] : 0.0f;
            odd |= is_odd(x[f]);
        }
        if (!__any(odd)) continue;
        const T* const k = token(p.k, key, p.k_page, p.k_head, p.k_token);
        for (unsigned left = rows; left; left &= left - 1) {
            const int r = __builtin_ctz(left), row = row0 + r, j = row / p.G, g = row - j * p.G, pos = t.seq.base + j;
            if (key > pos || key <= pos - p.window) continue;
            const T* const q = (const T*)p.q + (t.seq.start + j) * p.q_token + (int64_t)(t.h * p.G + g) * p.q_head + d;
            float s = 0.0f;
            for (int f = 0; f < F && has; ++f)
                if (d + f < p.D) s += (float)q[f] * (float)k[f];
            for (int m = 1; m < 64; m *= 2) s += __shfl_xor(s, m);
            const float weight = s > -__builtin_inff() ? 1.0f : 0.0f;
            const int64_t out = (t.seq.start + j) * p.out_token + (int64_t)(t.h * p.G + g) * p.out_head + d;
            const int64_t part = part_at<FEW>(p, t.seq, t.b, t.h, row, t.split, p.few_rows) * p.D + d;
            for (int f = 0; f < F && has; ++f)
                if (is_odd(x[f])) {
                    float was = 0.0f;
                    float* const o = (FEW ? p.few_o : p.many_o) + part + f;
                    if (touched[f] >> r & 1) was = !t.direct ? *o : (p.out_type == VLUT_TYPE_F32 ? ((const float*)p.out)[out + f] : (float)((const T*)p.out)[out + f]);
                    touched[f] |= 1u << r;
                    was += weight * x[f];
                    if (!t.direct) *o = was;
                    else if (p.out_type == VLUT_TYPE_F32) ((float*)p.out)[out + f] = was;
                    else ((T*)p.out)[out + f] = (T)was;
                }
        }
    }
}

// A tile's part.  FAST: heads of DP features, and 8 neighbouring keys share their page, so that addresses are worked out once per wave.
template <class T, int DP, int RW, int KW, int TERMS, bool FAST>
__device__ __forceinline__ void attend_chunk(const ChunkParams& p, const Tile& t, unsigned char* lds) {
    typedef typename Number<T>::x8 x8;
    constexpr bool FEW = KW > 1, WIDE = Number<T>::kWide;
    constexpr int NW = RW * KW, WK = wave_keys(DP, KW), KT = WK / 32, KEYS = step_keys(DP, KW), KS = DP / 16, CH = DP / 8, PER = 64 * NW / CH, LI = KEYS / PER, GK = 64 / CH;
    constexpr int KP = k_pitch(DP), VP = v_pitch(DP), BYTES = buffer_bytes_of(DP, KW), DT = DP / 32;
    constexpr float LIFT = 0.5f * Number<T>::kLift;            // (scores after the first step may be larger)
    static_assert(PER * LI == KEYS, "whole loads");
    const int tid = (int)threadIdx.x, lane = tid & 63, wave = __builtin_amdgcn_readfirstlane(tid >> 6), rw = wave % RW, kw = wave / RW;
    const int l32 = lane & 31, half = lane >> 5, l16 = lane & 15;
    const int wave_row0 = t.row0 + 32 * rw, row = wave_row0 + l32;
    const int first_key = t.first, end_key = t.end;

    float* const row_m = (float*)(lds + tile_bytes(DP, RW, KW));       // [KW][32 RW], then l
    float* const row_l = row_m + 32 * NW;
    int* const again = (int*)(row_l + 32 * NW);                        // then: whether there is something to settle
    if (tid == 0) again[0] = again[1] = 0;
    wg_barrier_lds();                                                  // (they are set ahead of the first step's barrier)

    // rows past the tile's end do as its last one
    const int real = min(row, t.row_end - 1), j = real / p.G, pos = t.seq.base + j;
    x8 q[KS];
    {
        const T* const src = (const T*)p.q + (t.seq.start + j) * p.q_token + (int64_t)(t.h * p.G + real - j * p.G) * p.q_head;
#pragma unroll
        for (int ks = 0; ks < KS; ++ks) {
            const int chunk = 2 * ks + half;
            q[ks] = __builtin_bit_cast(x8, chunk_moved<FAST>(*(const dword_aligned_i32x4*)(src + chunk_at<FAST>(chunk, p.D)), chunk, p.D));
        }
    }
    const int sees_from = max(0, pos - p.window + 1), sees_to = min(end_key, pos + 1);
    const bool blind = sees_to <= max(sees_from, first_key);           // nothing of this part
    // of the wave's rows, and of the workgroup's: from where to where all of them see, and any
    auto position = [&](int of) { return t.seq.base + min(of, t.row_end - 1) / p.G; };
    const int low = position(min(wave_row0, t.row_end - 1)), high = position(wave_row0 + 31);
    const int all_from = max(0, high - p.window + 1), all_to = low + 1, any_from = max(0, low - p.window + 1), any_to = wave_row0 < t.row_end ? high + 1 : 0;
    const int tile_low = position(t.row0), tile_high = position(t.row_end - 1), tile_from = max(0, tile_high - p.window + 1), tile_to = tile_low + 1;

    const int32_t* const pages = p.page_table + t.b * p.table_stride;
    const T* const kh = (const T*)p.k + t.h * p.k_head;
    const T* const vh = (const T*)p.v + t.h * p.v_head;
    const int mask = (1 << p.page_log) - 1, last = end_key - 1, last_group = last & ~(GK - 1);
    const int chunk = lane % CH, to_key = GK * wave + lane / CH;
    const unsigned at = 2u * (unsigned)chunk_at<FAST>(chunk, p.D), k_lane = (unsigned)(lane / CH) * 2u * (unsigned)p.k_token + at, v_lane = (unsigned)(lane / CH) * 2u * (unsigned)p.v_token + at;
    const unsigned to_k = (unsigned)(to_key * KP + 16 * chunk), to_v = (unsigned)(KEYS * KP + to_key * VP + 16 * chunk);
    i32x4 kr[LI], vr[LI];
    int ids[LI];
    unsigned bad = 0;                          // ids: the next keys' pages; bad: a bit for each loaded key (group) that is in none
    // (keys past the part read its last one, or another of that one's group: scores are masked, V is zeroed)
    auto key_of_load = [&](int kt, int i) { return FAST ? min(kt + PER * i + GK * wave, last_group) : min(kt + PER * i + to_key, last); };
    auto look_up = [&](int kt) {
#pragma unroll
        for (int i = 0; i < LI; ++i) ids[i] = pages[key_of_load(kt, i) >> p.page_log];
    };
    auto load = [&](int kt) {
        bad = 0;
#pragma unroll
        for (int i = 0; i < LI; ++i) {
            const int in_page = key_of_load(kt, i) & mask;
            const unsigned named = FAST ? (unsigned)__builtin_amdgcn_readfirstlane(ids[i]) : (unsigned)ids[i];
            const bool page = named < (unsigned)p.pages;
            bad |= page ? 0u : 1u << i;
            const uint64_t id = page ? named : 0u;
            if constexpr (FAST) {              // (strides are below 2^31 bytes here, and so are offsets inside a page)
                kr[i] = *(const dword_aligned_i32x4*)((const unsigned char*)kh + (id * (unsigned)p.k_page * 2u + (unsigned)in_page * 2u * (unsigned)p.k_token) + k_lane);
                vr[i] = *(const dword_aligned_i32x4*)((const unsigned char*)vh + (id * (unsigned)p.v_page * 2u + (unsigned)in_page * 2u * (unsigned)p.v_token) + v_lane);
            } else {
                kr[i] = *(const dword_aligned_i32x4*)(kh + (int64_t)id * p.k_page + in_page * p.k_token + chunk_at<FAST>(chunk, p.D));
                vr[i] = *(const dword_aligned_i32x4*)(vh + (int64_t)id * p.v_page + in_page * p.v_token + chunk_at<FAST>(chunk, p.D));
            }
        }
    };
    auto store = [&](int kt, unsigned char* to) {
        if (bad) {                             // a number that is no page: whoever sees its keys gets NaN
#pragma unroll
            for (int i = 0; i < LI; ++i)
                if (bad >> i & 1) {
                    constexpr int N = (int)Number<T>::kNan;
                    kr[i] = i32x4{N, N, N, N};
                }
        }
        if (kt + KEYS > min(end_key, tile_to) || kt < tile_from) {     // not every row sees every key
            unsigned odd = 0;
#pragma unroll
            for (int i = 0; i < LI; ++i) {
                if (kt + PER * i + to_key >= end_key) vr[i] = i32x4{0, 0, 0, 0};
#pragma unroll
                for (int w = 0; w < 4; ++w) {
                    const unsigned x = (unsigned)vr[i][w];
                    constexpr unsigned high_bits = Number<T>::kExponents & 0xffff0000u, low_bits = Number<T>::kExponents & 0xffffu;
                    const unsigned drop = ((x & high_bits) == high_bits ? 0xffff0000u : 0u) | ((x & low_bits) == low_bits ? 0xffffu : 0u);
                    vr[i][w] = (int)(x & ~drop);
                    odd |= drop;
                }
            }
            if (odd) again[1] = 1;
        }
#pragma unroll
        for (int i = 0; i < LI; ++i) {
            *(i32x4*)(to + to_k + PER * i * KP) = chunk_moved<FAST>(kr[i], chunk, p.D);
            *(i32x4*)(to + to_v + PER * i * VP) = chunk_moved<FAST>(vr[i], chunk, p.D);
        }
    };

    // All keys of the part, in steps: use(kt, K and V in LDS) between two barriers each.
    auto sweep = [&](auto use) {
        if (first_key >= end_key) return;
        look_up(first_key);
        load(first_key);
        look_up(first_key + KEYS);
#pragma unroll
        for (int ks = 0; ks < KS; ++ks) arrived(q[ks]);
        store(first_key, lds);
        int turn = 0;
        for (int kt = first_key; kt < end_key; kt += KEYS, turn ^= 1) {
            wg_barrier_lds();
            load(kt + KEYS);                   // (behind the last step too, from the last keys)
            look_up(kt + 2 * KEYS);
            if constexpr (buffers(KW) == 2) {
                use(kt, lds + turn * BYTES);
                if (kt + KEYS < end_key) store(kt + KEYS, lds + (turn ^ 1) * BYTES);
            } else {
                use(kt, lds);
                if (kt + KEYS < end_key) {
                    wg_barrier_lds();
                    store(kt + KEYS, lds);
                }
            }
        }
    };
    f32x16 s[KT], o[DT];
    float m = 0.0f, l;
    auto score = [&](int k0, const unsigned char* buf) {
#pragma unroll
        for (int i = 0; i < KT; ++i)
#pragma unroll
            for (int e = 0; e < 16; ++e) s[i][e] = 0.0f;
#pragma unroll
        for (int ks = 0; ks < KS; ++ks)
#pragma unroll
            for (int i = 0; i < KT; ++i) s[i] = mfma32(__builtin_bit_cast(x8, *(const i32x4*)(buf + (32 * i + l32) * KP + 32 * ks + 16 * half)), q[ks], s[i]);
        in_turn<KS * KT, 1, 1, 6, 0, 0>();
        if (k0 + WK > min(all_to, end_key) || k0 < all_from) {
            const int to = sees_to - k0 - 4 * half, from = sees_from - k0 - 4 * half;
#pragma unroll
            for (int i = 0; i < KT; ++i)
#pragma unroll
                for (int e = 0; e < 16; ++e) {
                    const int key = 32 * i + (e & 3) + 8 * (e >> 2);
                    if (key >= to || key < from) s[i][e] = -__builtin_inff();
                }
        }
    };
    // the largest score of a step, times scale_log2
    auto largest = [&]() {
        float top = s[0][0];
#pragma unroll
        for (int i = 0; i < KT; ++i)
#pragma unroll
            for (int e = 0; e < 16; ++e) top = fmaxf(top, s[i][e]);
        return fmaxf(top, __shfl_xor(top, 32)) * p.scale_log2;
    };
    auto finite = [&]() {
        float zero = 0.0f;                     // (or NaN)
#pragma unroll
        for (int dt = 0; dt < DT; ++dt)
#pragma unroll
            for (int e = 0; e < 16; ++e) zero = __builtin_fmaf(o[dt][e], 0.0f, zero);
        return zero == 0.0f;
    };
    const float none = -__builtin_inff();
    for (bool known = false;;) {
        l = 0.0f;
        if (!known) m = blind ? 0.0f : none;
#pragma unroll
        for (int dt = 0; dt < DT; ++dt)
#pragma unroll
            for (int e = 0; e < 16; ++e) o[dt][e] = 0.0f;
        sweep([&](int kt, const unsigned char* buf) {
            const int k0 = kt + WK * kw;
            if (k0 >= min(any_to, end_key) || k0 + WK <= any_from) return;             // (the wave's rows see nothing of it)
            const unsigned char* const kb = buf + WK * kw * KP;
            const unsigned v_at = lds_base_of((void*)(buf + KEYS * KP + WK * kw * VP)) + (4 * half + (l16 >> 2)) * VP + 32 * ((lane >> 4) & 1) + 8 * (l16 & 3);
            score(k0, kb);
            if (!known && __any(m == none)) {
                const float top = largest() - LIFT;
                m = m == none ? top : m;
            }
            const float shift = m == none ? 0.0f : m;
            // Sixteen keys at a time; the weights and V of the next are made and read while the matrix cores are on these.
            x8 vf[DT], pf[TERMS], next[TERMS];
            auto weigh = [&](int st, x8 (&w)[TERMS]) {
#pragma unroll
                for (int i = 0; i < 8; ++i) {
                    float left = exp2_fast(__builtin_fmaf(s[st >> 1][8 * (st & 1) + i], p.scale_log2, -shift));
                    l += left;
#pragma unroll
                    for (int k = 0; k < TERMS; ++k) {
                        w[k][i] = (T)left;
                        if (k + 1 < TERMS) left -= (float)(T)left;
                    }
                }
            };
            auto read_v = [&](int st, int dt) {
                const s16x4 v0 = lds_read_transposed(v_at + 16 * st * VP + 64 * dt), v1 = lds_read_transposed(v_at + (16 * st + 8) * VP + 64 * dt);
                return __builtin_bit_cast(x8, __builtin_shufflevector(v0, v1, 0, 1, 2, 3, 4, 5, 6, 7));
            };
#pragma unroll
            for (int dt = 0; dt < DT; ++dt) vf[dt] = read_v(0, dt);
            weigh(0, pf);
            __builtin_amdgcn_sched_barrier(0);
#pragma unroll
            for (int st = 0; st < 2 * KT; ++st) {
                if (st + 1 < 2 * KT) weigh(st + 1, next);
#pragma unroll
                for (int dt = 0; dt < DT; ++dt) {
#pragma unroll
                    for (int k = 0; k < TERMS; ++k) o[dt] = mfma32(vf[dt], pf[k], o[dt]);
                    if (st + 1 < 2 * KT) vf[dt] = read_v(st + 1, dt);
                }
#pragma unroll
                for (int k = 0; k < TERMS; ++k) pf[k] = next[k];
                in_turn<DT, TERMS, 2, 0, 20 * TERMS / DT, 8 / DT>();
                __builtin_amdgcn_sched_barrier(0);
            }
        });
        // (a lane's O is of the keys of both halves)
        const float both = l + __shfl_xor(l, 32);
        if (!finite() || (WIDE && !(both < 0x1p40f))) again[0] = 1;
        __syncthreads();
        if (!again[0] || known) break;
        known = true;
        m = none;
        sweep([&](int kt, const unsigned char* buf) {
            const int k0 = kt + WK * kw;
            if (k0 >= min(any_to, end_key) || k0 + WK <= any_from) return;
            score(k0, buf + WK * kw * KP);
            m = fmaxf(m, largest() - LIFT);
        });
        __syncthreads();
    }
    l += __shfl_xor(l, 32);
    if (t.seq.bad) l = __builtin_nanf("");
    if (l == 0.0f) m = none;                   // (nothing is of any weight: m may be anything)

    // The results leave through LDS (nobody reads the buffers any more), so that a store has whole lines.
    auto put = [&](int r, int d, const f32x4& x, float total) {        // row r of the tile, its O from feature d on and its l
        if (t.row0 + r >= t.row_end || d >= p.D) return;
        bool odd = false;
#pragma unroll
        for (int i = 0; i < 4; ++i) odd |= is_odd(x[i]);
        if (odd && total == total) again[1] = 1;
        const int at_row = t.row0 + r;
        if (t.direct) {
            const int its = at_row / p.G;
            store_four(p, (t.seq.start + its) * p.out_token + (int64_t)(t.h * p.G + at_row - its * p.G) * p.out_head + d,
                       total == 0.0f ? f32x4{0, 0, 0, 0} : x * (1.0f / total));
        } else *(f32x4*)((FEW ? p.few_o : p.many_o) + part_at<FEW>(p, t.seq, t.b, t.h, at_row, t.split, p.few_rows) * p.D + d) = x;
    };
    auto put_sums = [&](int r, float top, float total) {
        const int at_row = t.row0 + r;
        if (at_row >= t.row_end) return;
        if (!t.direct) *(f32x2*)((FEW ? p.few_ml : p.many_ml) + part_at<FEW>(p, t.seq, t.b, t.h, at_row, t.split, p.few_rows) * 2) = f32x2{top, total};
        else if (p.lse) {
            const int its = at_row / p.G;
            p.lse[(int64_t)(t.seq.start + its) * (p.Hk * p.G) + t.h * p.G + at_row - its * p.G] = lse_of(top, total);
        }
    };
    if constexpr (!FEW) {
        constexpr int TF = turn_features(DP), TP = TF + 4;             // floats from row to row
        float* const turned = (float*)lds + wave * 32 * TP;
        if (half == 0) row_l[32 * wave + l32] = l;
        __builtin_amdgcn_wave_barrier();
#pragma unroll
        for (int d0 = 0; d0 < DP; d0 += TF) {
#pragma unroll
            for (int i = 0; i < TF / 8; ++i) {
                const int dt = d0 / 32 + i / 4, e = 4 * (i & 3);
                *(f32x4*)(turned + l32 * TP + 8 * i + 4 * half) = f32x4{o[dt][e], o[dt][e + 1], o[dt][e + 2], o[dt][e + 3]};
            }
            __builtin_amdgcn_wave_barrier();
            constexpr int LANES = TF / 4;      // of a row
#pragma unroll
            for (int i = 0; i < 32 * LANES / 64; ++i) {
                const int r = i * (64 / LANES) + lane / LANES, d = 4 * (lane % LANES);
                put(32 * wave + r, d0 + d, *(const f32x4*)(turned + r * TP + d), row_l[32 * wave + r]);
            }
            __builtin_amdgcn_wave_barrier();
        }
        if (half == 0) put_sums(32 * wave + l32, m, l);
    } else {
        constexpr int TP = DP + 4;
        float* const turned = (float*)lds + wave * 32 * TP;
        if (half == 0) {
            row_m[32 * wave + l32] = m;
            row_l[32 * wave + l32] = l;
        }
        __syncthreads();
        float top = none;
#pragma unroll
        for (int w = 0; w < KW; ++w) top = fmaxf(top, row_m[32 * w + l32]);
        const float factor = m == none ? 0.0f : exp2_fast(m - top);
        // (a part without weight says nothing, whatever 0 times its values is)
        const bool counts = l != 0.0f;
#pragma unroll
        for (int i = 0; i < DP / 8; ++i) {
            const int dt = i / 4, e = 4 * (i & 3);
            f32x4 x = f32x4{o[dt][e], o[dt][e + 1], o[dt][e + 2], o[dt][e + 3]} * factor;
            *(f32x4*)(turned + l32 * TP + 8 * i + 4 * half) = counts ? x : f32x4{0, 0, 0, 0};
        }
        __syncthreads();
        if (half == 0) row_l[32 * wave + l32] = counts ? l * factor : 0.0f;
        __syncthreads();
        constexpr int LANES = DP / 4, ROWS = 64 * NW / LANES;
        const int d = 4 * (tid % LANES);
#pragma unroll
        for (int i = 0; i < 32 / ROWS; ++i) {
            const int r = i * ROWS + tid / LANES;
            f32x4 x = f32x4{0, 0, 0, 0};
            float total = 0.0f;
#pragma unroll
            for (int w = 0; w < KW; ++w) {
                x += *(const f32x4*)((const float*)lds + (32 * w + r) * TP + d);
                total += row_l[32 * w + r];
            }
            put(r, d, x, total);
        }
        if (wave == 0 && half == 0) {
            float total = 0.0f;
#pragma unroll
            for (int w = 0; w < KW; ++w) total += row_l[32 * w + l32];
            put_sums(l32, total == 0.0f ? none : top, total);
        }
    }
    __syncthreads();
    if (__builtin_expect(again[1] != 0, 0)) {
        // every wave settles its own rows, or its share of them
        __threadfence();
        unsigned rows = 0;
        for (int r = 0; r < 32; ++r) {
            float total = 0.0f;
            if constexpr (FEW) {
                if (r % KW != kw) continue;
                for (int w = 0; w < KW; ++w) total += row_l[32 * w + r];
            } else total = row_l[32 * wave + r];
            if (wave_row0 + r < t.row_end && total == total) rows |= 1u << r;
        }
        settle_chunk<T, DP, FEW>(p, t, wave_row0, rows);
    }
}

// Few rows: workgroups are numbered sequence by sequence, key head by key head, part by part.
template <class T, int DP, int TERMS, bool FAST>
__global__ void __launch_bounds__(256, DP > 128 ? 1 : 2) few_rows_kernel(const ChunkParams p) {
    extern __shared__ __align__(16) unsigned char lds[];
    const int i = ((int)blockIdx.x & 7) * p.few_per_xcd + ((int)blockIdx.x >> 3);
    Tile t;
    t.split = i % p.few_splits;
    t.h = i / p.few_splits % p.Hk;
    t.b = i / p.few_splits / p.Hk;
    if (t.b >= p.B) return;
    t.seq = chunk_of(p, t.b);
    t.row0 = 0;
    t.row_end = t.seq.queries * p.G;
    if (t.row_end == 0) return;
    if (t.row_end > p.few_rows) {
        // another launch's; where there is none, more queries than the caller said that there are: NaN
        if (p.many_per_xcd == 0 && t.split == 0)
            for (int64_t x = threadIdx.x; x < (int64_t)t.row_end * (p.D / 4); x += 256) {
                const int row = (int)(x / (p.D / 4)), j = row / p.G, d = 4 * (int)(x % (p.D / 4));
                const float nan = __builtin_nanf("");
                store_four(p, (t.seq.start + j) * p.out_token + (int64_t)(t.h * p.G + row - j * p.G) * p.out_head + d, f32x4{nan, nan, nan, nan});
                if (p.lse && d == 0) p.lse[(int64_t)(t.seq.start + j) * (p.Hk * p.G) + t.h * p.G + row - j * p.G] = nan;
            }
        return;
    }
    const Range r = range_of(p, t.seq, 0, t.seq.queries - 1, p.few_chunk);
    if (t.split >= r.parts) return;
    t.direct = r.parts == 1;
    t.first = r.first + t.split * p.few_chunk;
    t.end = t.first + min(r.end - t.first, p.few_chunk);
    attend_chunk<T, DP, 1, 4, TERMS, FAST>(p, t, lds);
}

// Many rows: tile `at` of the sequences' tiles, one sequence behind the other and the last tile of each, which sees the most, first.
template <class T, int DP, int RW, int TERMS, bool FAST>
__global__ void __launch_bounds__(64 * RW, DP > 128 ? 1 : 2) many_rows_kernel(const ChunkParams p) {
    extern __shared__ __align__(16) unsigned char lds[];
    constexpr int ROWS = 32 * RW;
    const int i = ((int)blockIdx.x & 7) * p.many_per_xcd + ((int)blockIdx.x >> 3), lane = (int)threadIdx.x & 63;
    int at = i % p.many_tiles;
    Tile t;
    t.split = i / p.many_tiles % p.many_splits;
    t.h = i / p.many_tiles / p.many_splits;
    if (t.h >= p.Hk) return;
    t.b = -1;
    for (int b0 = 0; b0 < p.B; b0 += 64) {
        const int b = b0 + lane;
        int rows = 0;
        if (b < p.B) {
            const int start = p.starts[b], next = p.starts[b + 1];
            rows = start >= 0 && next >= start && next <= p.N ? (next - start) * p.G : 0;
        }
        const int tiles = rows > p.few_rows ? (rows + ROWS - 1) / ROWS : 0;
        int sum = tiles;
#pragma unroll
        for (int m = 1; m < 64; m *= 2) {
            const int other = __shfl_up(sum, m);
            if (lane >= m) sum += other;
        }
        const uint64_t past = __ballot(sum > at);
        if (past) {
            const int f = __builtin_ctzll(past);
            t.b = b0 + f;
            at = __shfl(sum, f) - 1 - at;
            break;
        }
        at -= __shfl(sum, 63);
    }
    t.b = __builtin_amdgcn_readfirstlane(t.b);
    at = __builtin_amdgcn_readfirstlane(at);
    if (t.b < 0) return;
    t.seq = chunk_of(p, t.b);
    t.row0 = at * ROWS;
    t.row_end = min(t.row0 + ROWS, t.seq.queries * p.G);
    const Range r = range_of(p, t.seq, t.row0 / p.G, (t.row_end - 1) / p.G, p.many_chunk);
    if (t.split >= r.parts) return;
    t.direct = r.parts == 1;
    t.first = r.first + t.split * p.many_chunk;
    t.end = t.first + min(r.end - t.first, p.many_chunk);
    attend_chunk<T, DP, RW, 1, TERMS, FAST>(p, t, lds);
}

// The parts of every row joined, where there are several: DP / 4 threads have four features each.
template <class T, int DP>
__global__ void __launch_bounds__(256) combine_chunks(const ChunkParams p) {
    constexpr int PER = DP / 4, ROWS = 256 / PER;
    const int Hq = p.Hk * p.G, d = (int)(threadIdx.x % PER) * 4, lane = (int)threadIdx.x & 63;
    const int64_t row = (int64_t)blockIdx.x * ROWS + threadIdx.x / PER;
    // the sequence of the workgroup's first row, by the whole wave, and on from there
    const int first_token = (int)((int64_t)blockIdx.x * ROWS / Hq), token = (int)min(row / Hq, (int64_t)p.N - 1), head = (int)(row % Hq);
    int b = p.B;
    for (int b0 = 0; b0 < p.B; b0 += 64) {
        const uint64_t past = __ballot(b0 + lane < p.B && p.starts[min(b0 + lane, p.B - 1) + 1] > first_token);
        if (past) {
            b = b0 + __builtin_ctzll(past);
            break;
        }
    }
    while (b < p.B && p.starts[b + 1] <= token) ++b;
    if (row >= (int64_t)p.N * Hq || d >= p.D || b >= p.B) return;
    const Chunk c = chunk_of(p, b);
    const int j = token - c.start;
    if (j < 0 || j >= c.queries) return;
    const int h = head / p.G, in_head = j * p.G + head - h * p.G;
    const bool few = c.queries * p.G <= p.few_rows;
    if (!few && p.many_per_xcd == 0) return;   // (more queries than the caller said: NaN already, and there are no such parts)
    const int row0 = few ? 0 : in_head / p.many_rows * p.many_rows, row_end = few ? c.queries * p.G : min(row0 + p.many_rows, c.queries * p.G);
    const Range r = range_of(p, c, row0 / p.G, (row_end - 1) / p.G, few ? p.few_chunk : p.many_chunk);
    if (r.parts == 1) return;
    float top = -__builtin_inff(), total = 0.0f;
    f32x4 x = f32x4{0, 0, 0, 0};
    for (int s0 = 0; s0 < r.parts; s0 += 4) {
        float m[4], l[4];
        f32x4 o[4];
#pragma unroll
        for (int i = 0; i < 4; ++i) {
            const int s = min(s0 + i, r.parts - 1);
            const int64_t at = few ? part_at<true>(p, c, b, h, in_head, s, p.few_rows) : part_at<false>(p, c, b, h, in_head, s, 0);
            const f32x2 ml = *(const f32x2*)((few ? p.few_ml : p.many_ml) + at * 2);
            m[i] = ml.x;
            l[i] = ml.y;
            o[i] = *(const f32x4*)((few ? p.few_o : p.many_o) + at * p.D + d);
            if (s0 + i >= r.parts || l[i] == 0.0f) {
                m[i] = -__builtin_inff();
                l[i] = 0.0f;
                o[i] = f32x4{0, 0, 0, 0};
            }
        }
        const float now = fmaxf(fmaxf(fmaxf(m[0], m[1]), fmaxf(m[2], m[3])), top), shift = now == -__builtin_inff() ? 0.0f : now;
        const float factor = exp2_fast(top - shift);
        x *= factor;
        total *= factor;
#pragma unroll
        for (int i = 0; i < 4; ++i) {
            const float f = exp2_fast(m[i] - shift);
            total += f * l[i];
            x += o[i] * f;
        }
        top = now;
    }
    store_four(p, token * p.out_token + head * p.out_head + d, total == 0.0f ? f32x4{0, 0, 0, 0} : x * (1.0f / total));
    if (p.lse && d == 0) p.lse[row] = lse_of(top, total);
}

}  // namespace
