// Attention for a batch of sequences that share a prefix, over a paged cache.
// Part of the translation units attention_bf16.hip and attention_f16.hip (included there, in this order).
#pragma once

#include "matrix_parts.hip.h"

namespace {

using namespace vlut_attention;

// ---------------------------------------------------------------------------------------------
// For every query row q (a query token and one of its heads) over the keys it sees, s = scale * q . k:
//   m = max s,  l = sum exp(s - m),  O = sum exp(s - m) v,  output O / l;   nothing seen: 0
// Parts of the keys are worked out apart and joined: with M = max m_i the sums of exp(m_i - M) l_i and exp(m_i - M) O_i are those of the whole.
// The parts: the shared prefix, once for the rows of all sequences that read the same key head (B * n * G of them, G query heads to a key
// head), cut into prefix_splits ranges; and each sequence's own tokens for its n * G rows, cut into own_splits.  A workgroup has one
// range and one tile of rows.  One launch works out all of them (attend_few_kernel); where the rows and the prefix are many, the prefix has a
// launch of its own (attend_many_kernel), behind that of the own tokens.  combine_kernel joins the parts; a single part is stored as the result.
//
// Both products run transposed on the matrix cores, S^T = K Q^T and O^T = V^T P^T: a query is a column, so that its m, l and the factor
// of its O are one number per lane.  The columns of S^T come out with four neighbouring keys in a lane; P^T is taken in with the keys in exactly that
// order (the order of a sum's terms is free as long as V^T has the same), so that P goes from one product to the next without leaving its
// registers.  V^T is read out of the row-major V in LDS by transposing reads (ds_read_b64_tr_b16: the 16 lanes of a group give the addresses of 4
// rows x 16 features, and get four rows of one feature each).
// Scores, m, l and O are fp32, and l sums P before any rounding.  The matrix cores take no fp32, so that P is carried to the second product in terms of
// the cache's type, each what the rounding of those before it left.  For outputs of 16 bits: two (16 bits of bf16, 22 of fp16), so that the output's own
// rounding is what is left.  For fp32: what carries 24 bits of bf16, three, or two of fp16.  A caller gets the same bits from either kernel.  A term more is
// half as many matrix instructions again where rows are many: 256 rows a head, 32768 keys, 8 heads 46 us with one, 60 with two (one would leave bf16 outputs 40 %
// further off); 1024 rows a head, 8192 keys 58 with two, 73 with three (two would leave fp32 outputs 2.4e-6 of the result off instead of 4e-7).  Where rows are
// few, bound by memory or latency: 64 sequences of 8 key heads behind 4096 31.7 us with two, 34.2 with three.
// fp16: P is lifted by a power of two (Number::kLift), since weights below 2^-14 would lose bits and those below 2^-25 everything.
// ---------------------------------------------------------------------------------------------
// What a query row sees.  base: own position of the sequence's query 0; bad: lengths that cannot be.
struct Sequence {
    int len, queries, base, bad;
};
__device__ __forceinline__ Sequence sequence_of(const AttendParams& p, int b) {
    Sequence s;
    s.len = p.own_lens[b];
    s.queries = p.query_lens ? p.query_lens[b] : p.n;
    s.bad = s.len < 0 || s.len > p.max_own || s.queries < 0 || s.queries > p.n;
    if (s.bad) s.len = 0;
    s.base = s.len - s.queries;
    return s;
}

// The result of a row from its O / l (dl: 1 / l; 0 where nothing is seen).
__device__ __forceinline__ void store_result(const AttendParams& p, int64_t at, const f32x4& o) {
    if (p.out_type == VLUT_TYPE_F32) *(dword_aligned_f32x4*)((float*)p.out + at) = o;
    else if (p.out_type == VLUT_TYPE_BF16) {
        typedef __bf16 x4 __attribute__((ext_vector_type(4), aligned(4)));
        *(x4*)((__bf16*)p.out + at) = x4{(__bf16)o.x, (__bf16)o.y, (__bf16)o.z, (__bf16)o.w};
    } else {
        typedef _Float16 x4 __attribute__((ext_vector_type(4), aligned(4)));
        *(x4*)((_Float16*)p.out + at) = x4{(_Float16)o.x, (_Float16)o.y, (_Float16)o.z, (_Float16)o.w};
    }
}

// Whether a number out of a list of pages is one of the cache's.  Asked where the page is used: asked where it is loaded, it would wait for the keys
// and values that have been asked for before it.
__device__ __forceinline__ bool is_page(const AttendParams& p, int id) { return (unsigned)id < (unsigned)p.pages; }

// The kernel's parameters, its first argument, read again: as the reference that the loops have they would wait in registers throughout.  For a kernel
// itself alone: a function that is not part of one has no such argument.
__device__ __forceinline__ const AttendParams& parameters() {
#if defined(__HIP_DEVICE_COMPILE__)
    auto at = __builtin_amdgcn_kernarg_segment_ptr();
    asm volatile("" : "+s"(at));
    return *(const AttendParams*)at;
#else
    static AttendParams none;
    return none;
#endif
}
// Infinite values that a row sees.  P's further terms are zero or negative, so that their products with an infinity are NaN or the other infinity, and the
// sum is NaN where the formula has that infinity.  A part (or result) that came out as no number although its weights are numbers is therefore settled by the
// wave that stored it: its rows (bits of `rows`, from row0 on) get, in the features concerned, the sum of the infinities and NaN among the values of the range's
// keys that they see, with weights of 1, or 0 for a score of -inf.  (Where there are none, finite values passed 32 bits: NaN.)
// It reads V once more, and keys and queries where it finds such values, straight from memory and after everything else, so that it takes nothing from the
// loops: a look at their results, 0.2 us of 12.3 for 16 sequences of 256 behind 2048, 0.7 of 73 for 8 of 16384.  Where there is something to settle: 64
// sequences behind 32768, 92 us, one infinite value of the prefix 480 us, one in every range and key head 600.
template <class T, int DP>
__device__ __forceinline__ void settle_odd(const int32_t* pages, int h, int first_key, int end_key, int row0, unsigned rows, bool own, const Sequence& seq, int slot) {
    constexpr int F = DP / 64, AHEAD = 8;                          // features of a lane; keys at a time
    const AttendParams& p = parameters();
    // (or what is worked out from these waits in registers too)
    h = there(h), first_key = there(first_key), end_key = there(end_key), row0 = there(row0), slot = there(slot);
    const int lane = (int)threadIdx.x & 63, d = F * lane, nG = p.n * p.G, mask = (1 << p.page_log) - 1;
    const bool has = d < p.D;
    __threadfence();                                               // (other lanes have stored the results)
    struct Row {
        int b, j, head;
    };
    auto row_at = [&](int row) {
        const int b = row / nG, in_seq = row - b * nG, j = in_seq / p.G;
        return Row{b, j, h * p.G + in_seq - j * p.G};
    };
    auto result = [&](int row) -> int64_t {
        if (!p.direct) return (((int64_t)h * p.rows + row) * (p.prefix_splits + p.own_splits) + slot) * p.D + d;
        const Row r = row_at(row);
        return r.b * p.out_sequence + r.j * p.out_token + r.head * p.out_head + d;
    };
    auto get = [&](int64_t at) -> float {
        if (!p.direct) return p.part_o[at];
        if (p.out_type == VLUT_TYPE_F32) return ((const float*)p.out)[at];
        return (float)((const T*)p.out)[at];                       // (outputs of 16 bits are of the cache's type)
    };
    auto set = [&](int64_t at, float x) {
        if (!p.direct) p.part_o[at] = x;
        else if (p.out_type == VLUT_TYPE_F32) ((float*)p.out)[at] = x;
        else ((T*)p.out)[at] = (T)x;
    };
    auto token = [&](const void* of, int key, int64_t page_stride, int64_t head_stride, int64_t token_stride) {
        const int id = pages[key >> p.page_log];
        return (const T*)of + (is_page(p, id) ? id : 0) * page_stride + h * head_stride + (key & mask) * token_stride + d;
    };
    unsigned lost[F] = {};                                         // a bit for each row
#pragma unroll 1
    for (unsigned left = rows; left; left &= left - 1) {
        const int r = __builtin_ctz(left);
        const int64_t at = result(row0 + r);
        if (p.direct && !own && sequence_of(p, row_at(row0 + r).b).bad) continue;      // (NaN for that)
        for (int f = 0; f < F && has; ++f)
            if (is_odd(get(at + f))) {
                lost[f] |= 1u << r;
                set(at + f, 0.0f);
            }
    }
#pragma unroll 1
    for (int key0 = first_key; key0 < end_key; key0 += AHEAD) {
        unsigned x[AHEAD][F > 1 ? F / 2 : 1];                      // (rows start at a dword)
#pragma unroll
        for (int i = 0; i < AHEAD; ++i) {
            const T* const v = token(p.v, min(key0 + i, end_key - 1), p.v_page, p.v_head, p.v_token);
            if constexpr (F == 1) x[i][0] = has ? *(const unsigned short*)v : 0u;
            else {
#pragma unroll
                for (int w = 0; w < F / 2; ++w) x[i][w] = has ? ((const unsigned*)v)[w] : 0u;
            }
        }
        unsigned found = 0;
#pragma unroll
        for (int i = 0; i < AHEAD; ++i) {
            bool odd = false;
#pragma unroll
            for (unsigned w : x[i]) odd |= has_odd<T>(w);
            found |= key0 + i < end_key && __any(odd) ? 1u << i : 0u;
        }
#pragma unroll 1
        for (; found; found &= found - 1) {
            const int key = key0 + __builtin_ctz(found);
            const T* const v = token(p.v, key, p.v_page, p.v_head, p.v_token);
            const T* const k = token(p.k, key, p.k_page, p.k_head, p.k_token);
#pragma unroll 1
            for (unsigned left = rows; left; left &= left - 1) {
                const int r = __builtin_ctz(left);
                const Row its = row_at(row0 + r);
                if (own && key > seq.base + its.j) continue;
                const T* const q = (const T*)p.q + its.b * p.q_sequence + its.j * p.q_token + its.head * p.q_head + d;
                float s = 0.0f;
                for (int f = 0; f < F && has; ++f) s += (float)q[f] * (float)k[f];
                for (int m = 1; m < 64; m *= 2) s += __shfl_xor(s, m);
                const float weight = s > -__builtin_inff() ? 1.0f : 0.0f;
                const int64_t at = result(row0 + r);
                for (int f = 0; f < F && has; ++f)
                    if ((lost[f] >> r & 1) && is_odd((float)v[f])) set(at + f, get(at + f) + weight * (float)v[f]);
            }
        }
    }
#pragma unroll 1
    for (unsigned left = rows; left; left &= left - 1) {
        const int r = __builtin_ctz(left);
        const int64_t at = result(row0 + r);
        for (int f = 0; f < F && has; ++f)
            if ((lost[f] >> r & 1) && get(at + f) == 0.0f) set(at + f, __builtin_nanf(""));
    }
}

// One range of keys for up to 16 * MT query rows, few enough that memory is what bounds it.  A wave takes 32 keys a step (K straight to registers, V
// through a piece of LDS of its own, no barrier); the next 32 are on their way while the present ones are worked on.  `share` waves
// have the range in turn: 4 or 2, which join at the end through LDS, or 1 where ranges are short and many.  keep: the range is one
// (the waves of a workgroup meet in the join).
// 16 rows a tile, since a wave's K in registers serves one matrix instruction of 16 x 16 x 32 each way; two tiles share K, V and their LDS reads
// where there are more rows (more tiles: O does not fit the registers).  Two workgroups of four waves on a unit have 100 KB of loads on their way.
// Measured, 8 key heads of 128 features in bf16: 8 sequences of up to 16384 own tokens behind 1000, 338 MB: 70 us, 4.8 TB/s (a large copy: 5.3); 64 of up
// to 512, 102 MB: 24.6 us, 4.2 TB/s, of which the first loads' latency and unequal lengths take a fifth.  Short ranges are bound by latency, a chain
// of page number, keys, scores, join and parts: one sequence of 40 tokens behind 512, 6.2 us; 16 of 256 behind 2048, 9.4 us.
// 24 sequences, 32 heads of 100 features that are not shared, 5 queries each over 300 own tokens and 1500 shared ones, 88 MB: 37 us, 2.4 TB/s, bound by what
// a wave issues and waits for per step (12 steps of the prefix, 5 of own tokens).
// Returns the rows that the wave has to settle (settle_odd).
template <class T, int DP, int MT, int TERMS, bool WHOLE, bool GROUPED>
__device__ unsigned attend_few(const AttendParams& p, const int32_t* pages, int h, int first_key, int end_key, int row0, int row_end, bool own, const Sequence& seq, int slot,
                           int share, bool keep, unsigned char* lds) {
    typedef typename Number<T>::x8 x8;
    constexpr int KS = DP / 32, CH = DP / 8, PER = 64 / CH, VI = kFewKeys / PER, PITCH = few_pitch(DP);
    const int lane = (int)threadIdx.x & 63, wave = __builtin_amdgcn_readfirstlane((int)threadIdx.x >> 6);
    const int l16 = lane & 15, grp = lane >> 4;
    unsigned char* const mine = lds + wave * kFewKeys * PITCH;
    const unsigned mine_at = lds_base_of(mine);
    const int nG = p.n * p.G, stride = share * kFewKeys;

    x8 q[MT][KS];
    int limit[MT];
#pragma unroll
    for (int mt = 0; mt < MT; ++mt) {
        const int row = min(row0 + 16 * mt + l16, row_end - 1);
        const int b = row / nG, in_seq = row - b * nG, j = in_seq / p.G, g = in_seq - j * p.G;
        const T* src = (const T*)p.q + b * p.q_sequence + j * p.q_token + (int64_t)(h * p.G + g) * p.q_head;
        limit[mt] = own ? min(end_key, seq.base + j + 1) : end_key;
#pragma unroll
        for (int ks = 0; ks < KS; ++ks) {
            const int chunk = 4 * ks + grp;
            q[mt][ks] = __builtin_bit_cast(x8, chunk_moved<WHOLE>(*(const dword_aligned_i32x4*)(src + chunk_at<WHOLE>(chunk, p.D)), chunk, p.D));
        }
    }
    // keys below `all_see` are seen by every row of the tile
    const int all_see = own ? min(end_key, seq.base + (row0 % nG) / p.G + 1) : end_key;

    float m[MT], l[MT];
    f32x4 o[MT][DP / 16];
#pragma unroll
    for (int mt = 0; mt < MT; ++mt) {
        m[mt] = -__builtin_inff();
        l[mt] = 0.0f;
#pragma unroll
        for (int dt = 0; dt < DP / 16; ++dt) o[mt][dt] = f32x4{0, 0, 0, 0};
    }

    const T* const kh = (const T*)p.k + h * p.k_head;
    const T* const vh = (const T*)p.v + h * p.v_head;
    const int mask = (1 << p.page_log) - 1, last = end_key - 1;
    const int v_chunk = lane % CH, v_key = lane / CH;
    i32x4 kr[2][KS], vr[VI];
    // Pages of 32 keys, and their rows.  GROUPED: every 16 keys share a page, whose number a wave has two of (Pages), and addresses are worked out
    // once per wave; else a lane looks up one key's.  Keys past the range read its last one or another row of that one's page: scores are
    // masked, V is zeroed.
    struct Pages {
        int id[GROUPED ? 2 : 1];
    };
    const unsigned k_lane = GROUPED ? 2u * (unsigned)l16 * (unsigned)p.k_token : 0u;
    const unsigned v_lane = GROUPED ? 2u * ((unsigned)v_key * (unsigned)p.v_token + (unsigned)chunk_at<WHOLE>(v_chunk, p.D)) : 0u;
    auto look_up = [&](int kt) {
        Pages g;
        if constexpr (GROUPED) {
#pragma unroll
            for (int t = 0; t < 2; ++t) g.id[t] = pages[min(kt + 16 * t, last & ~15) >> p.page_log];
        } else g.id[0] = pages[min(kt + (lane & 31), last) >> p.page_log];
        return g;
    };
    // the first row of 16 keys that share a page
    auto rows_of = [&](const T* of, int64_t page_stride, int64_t token_stride, int kt, int t, const Pages& g) {
        const unsigned named = (unsigned)__builtin_amdgcn_readfirstlane(g.id[GROUPED ? t : 0]), id = is_page(p, (int)named) ? named : 0u;
        return (const unsigned char*)of + ((uint64_t)id * 2u * (unsigned)page_stride + (unsigned)(min(kt + 16 * t, last & ~15) & mask) * 2u * (unsigned)token_stride);
    };
    auto load_k = [&](int kt, const Pages& g) {
#pragma unroll
        for (int t = 0; t < 2; ++t) {
            if constexpr (GROUPED) {
                const unsigned char* const src = rows_of(kh, p.k_page, p.k_token, kt, t, g);
#pragma unroll
                for (int ks = 0; ks < KS; ++ks) kr[t][ks] = *(const dword_aligned_i32x4*)(src + (k_lane + 2u * (unsigned)chunk_at<WHOLE>(4 * ks + grp, p.D)));
            } else {
                const int key = min(kt + 16 * t + l16, last), id = __shfl(g.id[0], 16 * t + l16);
                const T* src = kh + (is_page(p, id) ? id : 0) * p.k_page + (key & mask) * p.k_token;
#pragma unroll
                for (int ks = 0; ks < KS; ++ks) kr[t][ks] = *(const dword_aligned_i32x4*)(src + chunk_at<WHOLE>(4 * ks + grp, p.D));
            }
        }
    };
    auto load_v = [&](int kt, const Pages& g) {
#pragma unroll
        for (int i = 0; i < VI; ++i) {
            if constexpr (GROUPED)
                vr[i] = *(const dword_aligned_i32x4*)(rows_of(vh, p.v_page, p.v_token, kt, PER * i / 16, g) + (unsigned)(PER * i % 16) * 2u * (unsigned)p.v_token + v_lane);
            else {
                const int k_in = PER * i + v_key, key = min(kt + k_in, last), id = __shfl(g.id[0], k_in);
                const T* src = vh + (is_page(p, id) ? id : 0) * p.v_page + (key & mask) * p.v_token;
                vr[i] = *(const dword_aligned_i32x4*)(src + chunk_at<WHOLE>(v_chunk, p.D));
            }
        }
    };

    int kt = first_key + kFewKeys * (wave & (share - 1));
    Pages page, next_page;
    if (kt < end_key) {
        page = look_up(kt);
        next_page = look_up(kt + stride);
        load_v(kt, page);
        load_k(kt, page);
#pragma unroll
        for (int mt = 0; mt < MT; ++mt)
#pragma unroll
            for (int ks = 0; ks < KS; ++ks) arrived(q[mt][ks]);
    }
    auto step = [&](auto more) {
        const bool some_masked = kt + kFewKeys > all_see;
        // V to LDS, zeros for keys past the range
        unsigned odd = 0;
#pragma unroll
        for (int i = 0; i < VI; ++i) vr[i] = chunk_moved<WHOLE>(vr[i], v_chunk, p.D);
        if (some_masked) {
#pragma unroll
            for (int i = 0; i < VI; ++i) {
                if (kt + PER * i + v_key >= end_key) vr[i] = i32x4{0, 0, 0, 0};
#pragma unroll
                for (int w = 0; w < 4; ++w) odd |= has_odd<T>((unsigned)vr[i][w]);
            }
        }
#pragma unroll
        for (int i = 0; i < VI; ++i) *(i32x4*)(mine + (PER * i + v_key) * PITCH + 16 * v_chunk) = vr[i];
        // What comes next, in the order in which it is waited for: the page after the next, V, K.  Also behind the last step, from its last key: in a
        // branch, registers that are loaded on one way alone would be copied, and waited for, where the ways meet.
        Pages page_after;
        if constexpr (more.value) {
            page_after = look_up(kt + 2 * stride);
            load_v(kt + stride, next_page);
        }
        x8 kf[2][KS];
#pragma unroll
        for (int t = 0; t < 2; ++t)
#pragma unroll
            for (int ks = 0; ks < KS; ++ks) kf[t][ks] = __builtin_bit_cast(x8, chunk_moved<WHOLE>(kr[t][ks], 4 * ks + grp, p.D));
        f32x4 s[MT][2];
#pragma unroll
        for (int mt = 0; mt < MT; ++mt)
#pragma unroll
            for (int t = 0; t < 2; ++t) {
                s[mt][t] = f32x4{0, 0, 0, 0};
#pragma unroll
                for (int ks = 0; ks < KS; ++ks) s[mt][t] = mfma16(kf[t][ks], q[mt][ks], s[mt][t]);
            }
        // A number that is no page: not read, and whoever sees its keys gets NaN
        bool no_page = !is_page(p, page.id[0]);
        if constexpr (GROUPED) no_page = no_page || !is_page(p, page.id[1]);
        if (__any(no_page)) {
#pragma unroll
            for (int t = 0; t < 2; ++t)
#pragma unroll
                for (int i = 0; i < 4; ++i)
                    if (!is_page(p, GROUPED ? page.id[GROUPED ? t : 0] : __shfl(page.id[0], 16 * t + 4 * grp + i))) {
#pragma unroll
                        for (int mt = 0; mt < MT; ++mt) s[mt][t][i] = __builtin_nanf("");
                    }
        }
        if constexpr (more.value) load_k(kt + stride, next_page);
        x8 pf[MT][TERMS];
#pragma unroll
        for (int mt = 0; mt < MT; ++mt) {
            if (some_masked) {
                const int seen = limit[mt] - kt - 4 * grp;
#pragma unroll
                for (int t = 0; t < 2; ++t)
#pragma unroll
                    for (int i = 0; i < 4; ++i)
                        if (16 * t + i >= seen) s[mt][t][i] = -__builtin_inff();
            }
            float top = fmaxf(fmaxf(fmaxf(s[mt][0].x, s[mt][0].y), fmaxf(s[mt][0].z, s[mt][0].w)), fmaxf(fmaxf(s[mt][1].x, s[mt][1].y), fmaxf(s[mt][1].z, s[mt][1].w)));
            top = fmaxf(top, __shfl_xor(top, 16));
            top = fmaxf(top, __shfl_xor(top, 32));
            const float now = fmaxf(m[mt], __builtin_fmaf(top, p.scale_log2, -Number<T>::kLift)), shift = now == -__builtin_inff() ? 0.0f : now;
            const float factor = exp2_fast(m[mt] - shift);
            m[mt] = now;
            l[mt] *= factor;
#pragma unroll
            for (int t = 0; t < 2; ++t)
#pragma unroll
                for (int i = 0; i < 4; ++i) {
                    const float e = exp2_fast(__builtin_fmaf(s[mt][t][i], p.scale_log2, -shift));
                    l[mt] += e;
                    float left = e;
#pragma unroll
                    for (int k = 0; k < TERMS; ++k) {
                        pf[mt][k][4 * t + i] = (T)left;
                        left -= (float)(T)left;
                    }
                }
#pragma unroll
            for (int dt = 0; dt < DP / 16; ++dt) o[mt][dt] *= factor;
        }
        if (some_masked && __any(odd)) {
            // An infinity or NaN among the values, and rows that do not see all of them: 0 * inf would reach those too.  Such values are added
            // to the rows that see them one by one and taken out of V.  P goes to the ends of V's rows for that, which are free.
#pragma unroll
            for (int mt = 0; mt < MT; ++mt) {
#pragma unroll
                for (int e = 0; e < 8; ++e) *(T*)(mine + (16 * (e >> 2) + 4 * grp + (e & 3)) * PITCH + 2 * DP + 2 * l16) = pf[mt][0][e];
                __builtin_amdgcn_wave_barrier();
                for (int key = 0; key < kFewKeys && kt + key < end_key; ++key) {
                    const bool seen = kt + key < limit[mt];
                    const float weight = (float)*(const T*)(mine + key * PITCH + 2 * DP + 2 * l16);
#pragma unroll
                    for (int dt = 0; dt < DP / 16; ++dt)
#pragma unroll
                        for (int i = 0; i < 4; ++i) {
                            const float x = (float)*(const T*)(mine + key * PITCH + 32 * dt + 8 * grp + 2 * i);
                            if (seen && is_odd(x)) o[mt][dt][i] += weight * x;
                        }
                }
                __builtin_amdgcn_wave_barrier();
            }
#pragma unroll 1
            for (int i = 0; i < VI; ++i)
#pragma unroll 1
                for (int e = 0; e < 8; ++e) {
                    T* const x = (T*)(mine + (PER * i + v_key) * PITCH + 16 * v_chunk) + e;
                    if (is_odd((float)*x)) *x = (T)0.0f;
                }
            __builtin_amdgcn_wave_barrier();
        }
        __builtin_amdgcn_sched_barrier(0);
#pragma unroll
        for (int dt = 0; dt < DP / 16; ++dt) {
            const unsigned at = mine_at + (4 * grp + (l16 >> 2)) * PITCH + 32 * dt + 8 * (l16 & 3);
            const s16x4 v0 = lds_read_transposed(at), v1 = lds_read_transposed(at + 16 * PITCH);
            const x8 vf = __builtin_bit_cast(x8, __builtin_shufflevector(v0, v1, 0, 1, 2, 3, 4, 5, 6, 7));
#pragma unroll
            for (int mt = 0; mt < MT; ++mt)
#pragma unroll
                for (int k = 0; k < TERMS; ++k) o[mt][dt] = mfma16(vf, pf[mt][k], o[mt][dt]);
        }
        in_turn<DP / 16, TERMS * MT, 2, 4, 0, 0>();
        if constexpr (more.value) {
            page = next_page;
            next_page = page_after;
        }
    };
    for (; kt + stride < end_key; kt += stride) step(std::true_type{});
    if (kt < end_key) step(std::false_type{});

    // A row's result from threads that have some of its features each: the part as it is, or O / l.
    struct Row {
        int64_t at;
        float factor;
        bool real;
    };
    auto begin_row = [&](int row, float top, float total, bool first) {
        Row r;
        if (!p.direct) {
            const int64_t part = ((int64_t)h * p.rows + row) * (p.prefix_splits + p.own_splits) + slot;
            r.at = part * p.D;
            if (first) *(f32x2*)(p.part_ml + part * 2) = own && seq.bad ? f32x2{__builtin_nanf(""), __builtin_nanf("")} : f32x2{top, total};
            return r;
        }
        const int b = row / nG, in_seq = row - b * nG, j = in_seq / p.G, g = in_seq - j * p.G;
        const Sequence its = own ? seq : sequence_of(p, b);
        if (its.bad) total = __builtin_nanf("");
        r.real = (its.bad || j < its.queries) && total != 0.0f;
        r.factor = 1.0f / total;
        r.at = b * p.out_sequence + j * p.out_token + (int64_t)(h * p.G + g) * p.out_head;
        if (first && p.lse) p.lse[((int64_t)b * p.n + j) * p.Hk * p.G + h * p.G + g] = r.real ? lse_of(top, total) : -__builtin_inff();
        return r;
    };
    auto put = [&](const Row& r, int d, f32x4 x) {
        if (d >= p.D) return;
        if (!p.direct) *(f32x4*)(p.part_o + r.at + d) = x;
        else store_result(p, r.at + d, r.real ? x * r.factor : f32x4{0, 0, 0, 0});
    };
#pragma unroll
    for (int mt = 0; mt < MT; ++mt) {
        l[mt] += __shfl_xor(l[mt], 16);
        l[mt] += __shfl_xor(l[mt], 32);
    }
    unsigned odd_rows = 0;                     // whose result is none although their weights are numbers
    if (share == 1) {
#pragma unroll
        for (int mt = 0; mt < MT; ++mt) {
            const int row = row0 + 16 * mt + l16;
            const bool real = row < row_end && keep;
            float zero = 0.0f;
#pragma unroll
            for (int dt = 0; dt < DP / 16; ++dt)
#pragma unroll
                for (int i = 0; i < 4; ++i) zero = __builtin_fmaf(o[mt][dt][i], 0.0f, zero);
            const uint64_t odd = __ballot(real && zero != 0.0f && l[mt] == l[mt]);
            odd_rows |= (unsigned)((odd | odd >> 16 | odd >> 32 | odd >> 48) & 0xffff) << (16 * mt);
            if (!real) continue;
            const Row r = begin_row(row, m[mt], l[mt], grp == 0);
#pragma unroll
            for (int dt = 0; dt < DP / 16; ++dt) put(r, 16 * dt + 4 * grp, o[mt][dt]);
        }
        return odd_rows;
    }
    // The waves' parts: 16 rows at a time through LDS, 16 threads for a row.
    constexpr int OP = DP + 4, F4 = DP / 64;                       // floats per row; vectors of four per thread
    float* const all_o = (float*)lds;                              // [wave][16][OP]
    float* const all_ml = all_o + 4 * 16 * OP;                     // [wave][16][2]
    const int first_wave = wave & ~(share - 1);                    // of those that share the range
#pragma unroll
    for (int mt = 0; mt < MT; ++mt) {
        __syncthreads();
#pragma unroll
        for (int dt = 0; dt < DP / 16; ++dt) *(f32x4*)(all_o + (wave * 16 + l16) * OP + 16 * dt + 4 * grp) = o[mt][dt];
        if (grp == 0) {
            all_ml[(wave * 16 + l16) * 2] = m[mt];
            all_ml[(wave * 16 + l16) * 2 + 1] = l[mt];
        }
        __syncthreads();
        for (int r = ((wave - first_wave) * 64 + lane) >> 4; r < 16; r += 4 * share) {
            const int part = lane & 15, row = row0 + 16 * mt + r;
            bool odd = false;
            if (row < row_end && keep) {
                float top = -__builtin_inff(), total = 0.0f;
                for (int w = first_wave; w < first_wave + share; ++w) top = fmaxf(top, all_ml[(w * 16 + r) * 2]);
                const float shift = top == -__builtin_inff() ? 0.0f : top;
                f32x4 x[F4] = {};
                for (int w = first_wave; w < first_wave + share; ++w) {
                    const float f = exp2_fast(all_ml[(w * 16 + r) * 2] - shift);
                    total += f * all_ml[(w * 16 + r) * 2 + 1];
#pragma unroll
                    for (int v = 0; v < F4; ++v) x[v] += *(f32x4*)(all_o + (w * 16 + r) * OP + (part + 16 * v) * 4) * f;
                }
                const Row to = begin_row(row, top, total, part == 0);
                float zero = 0.0f;
#pragma unroll
                for (int v = 0; v < F4; ++v) {
                    put(to, (part + 16 * v) * 4, x[v]);
#pragma unroll
                    for (int i = 0; i < 4; ++i) zero = __builtin_fmaf(x[v][i], 0.0f, zero);
                }
                odd = zero != 0.0f && total == total;
            }
            const uint64_t odds = __ballot(odd);
            if (odds) {
#pragma unroll
                for (int g = 0; g < 4; ++g) odd_rows |= odds >> (16 * g) & 0xffff ? 1u << (16 * mt + r - grp + g) : 0u;
            }
        }
    }
    return __builtin_amdgcn_readfirstlane(odd_rows);
}

// One range of the prefix for 32 * NW query rows, many enough that memory is not what bounds it: K and V of 64 keys (32 where D is
// over 128) in LDS for all NW waves, which have 32 rows each.  Two buffers: the next keys travel to registers while the present ones are
// worked on, and are stored behind them; one barrier per step.
// 32 rows a wave, the matrix instruction's 32 x 32 x 16; 64 would halve the LDS reads, but their O has to live in the accumulation registers, and the
// copies cost more.  Two waves on a SIMD, so that one's exponentials go beside the other's matrix instructions.
// Measured, 8 heads of 128 features, bf16: 256 rows a head, 32768 keys, P in two terms, 52 GFLOP: 60 us, 850 TFLOP/s, 62 % of the rate of a large product;
// 1024 rows, 8192 keys, P in three terms, 69 GFLOP: 73 us, 940 TFLOP/s.  Counted there, of a SIMD's cycles (1.75 GHz): matrix cores busy 46 % and 51 %, vector units
// 43 % and 48 %, LDS 21 % and 18 % with hardly a conflict; of a wave's, a third it issues, a third it waits for its turn or for a unit, a third (27 %) for data
// and barriers.  So no unit is full: matrix and vector work of a SIMD's two waves, which the barrier holds in one phase, follow each other for the most
// part instead of lying beside each other.
// What the vector units have to do beside the matrix instructions is kept short:
//   - a wave's load covers GK neighbouring keys, which share their page (the host sees to it): addresses are worked out once per wave;
//   - O is not multiplied with every new maximum, and maxima are not looked for: m is the largest score of the first step, and weights are powers of
//     two of the scores above it.  Where that does not do (bf16: the sum of weights shows one of 2^40 or so; fp16, whose weights have to stay
//     below 2^15: a maximum per step shows one; a first step whose scores are all -inf, which says nothing of the others; an O past fp32 by weights above 1)
//     the range is begun again with the largest of all its scores, which a sweep over K finds.  (64 sequences behind 32768, such scores in every range: 92 -> 162
//     us, fp16 96 -> 169.)
//     (Multiplying where it is needed, in a branch, costs as much as always: O's registers are copied where the ways meet.)
// Returns the rows that the wave has to settle.
template <class T, int DP, int TERMS, int NW, bool WHOLE>
__device__ unsigned attend_many(const AttendParams& p, const int32_t* pages, int h, int first_key, int end_key, int row0, int row_end, int slot, unsigned char* lds) {
    typedef typename Number<T>::x8 x8;
    constexpr int KEYS = many_keys(DP), KT = KEYS / 32, KS = DP / 16, CH = DP / 8, PER = 64 * NW / CH, LI = KEYS / PER, GK = 64 / CH;
    constexpr int KP = many_k_pitch(DP), VP = many_v_pitch(DP);
    constexpr bool WIDE = Number<T>::kWide;
    constexpr float LIFT = 0.5f * Number<T>::kLift;            // (scores after the first step may be larger)
    const int tid = (int)threadIdx.x, lane = tid & 63, wave = __builtin_amdgcn_readfirstlane(tid >> 6);
    const int l32 = lane & 31, half = lane >> 5, l16 = lane & 15;
    const int nG = p.n * p.G, row = row0 + 32 * wave + l32;

    x8 q[KS];
    {
        const int real = min(row, row_end - 1), b = real / nG, in_seq = real - b * nG, j = in_seq / p.G, g = in_seq - j * p.G;
        const T* src = (const T*)p.q + b * p.q_sequence + j * p.q_token + (int64_t)(h * p.G + g) * p.q_head;
#pragma unroll
        for (int ks = 0; ks < KS; ++ks) {
            const int chunk = 2 * ks + half;
            q[ks] = __builtin_bit_cast(x8, chunk_moved<WHOLE>(*(const dword_aligned_i32x4*)(src + chunk_at<WHOLE>(chunk, p.D)), chunk, p.D));
        }
    }

    const T* const kh = (const T*)p.k + h * p.k_head;
    const T* const vh = (const T*)p.v + h * p.v_head;
    const int mask = (1 << p.page_log) - 1, last_group = (end_key - 1) & ~(GK - 1);
    const int chunk = lane % CH, to_key = GK * wave + lane / CH;
    const unsigned at = 2u * (unsigned)chunk_at<WHOLE>(chunk, p.D), k_lane = (unsigned)(lane / CH) * 2u * (unsigned)p.k_token + at, v_lane = (unsigned)(lane / CH) * 2u * (unsigned)p.v_token + at;
    const unsigned to_k = (unsigned)(to_key * KP + 16 * chunk), to_v = (unsigned)(KEYS * KP + to_key * VP + 16 * chunk);
    i32x4 kr[LI], vr[LI];
    int ids[LI], bad = 0;                      // the next keys' pages; a bit for each loaded group that is in none
    // (groups past the range read the last one: scores are masked, V is zeroed)
    auto group = [&](int kt, int i) { return min(kt + PER * i + GK * wave, last_group); };
    auto look_up = [&](int kt) {
#pragma unroll
        for (int i = 0; i < LI; ++i) ids[i] = pages[group(kt, i) >> p.page_log];
    };
    auto load = [&](int kt) {
        bad = 0;
#pragma unroll
        for (int i = 0; i < LI; ++i) {
            const unsigned in_page = (unsigned)(group(kt, i) & mask), named = (unsigned)__builtin_amdgcn_readfirstlane(ids[i]);
            const bool page = named < (unsigned)p.pages;
            bad |= page ? 0 : 1 << i;
            // (strides are below 2^31 bytes here, and so are offsets inside a page)
            const uint64_t id = page ? named : 0u;
            kr[i] = *(const dword_aligned_i32x4*)((const unsigned char*)kh + (id * (unsigned)p.k_page * 2u + in_page * 2u * (unsigned)p.k_token) + k_lane);
            vr[i] = *(const dword_aligned_i32x4*)((const unsigned char*)vh + (id * (unsigned)p.v_page * 2u + in_page * 2u * (unsigned)p.v_token) + v_lane);
        }
    };
    auto store = [&](int kt, unsigned char* to) {
        if (bad) {
#pragma unroll
            for (int i = 0; i < LI; ++i)
                if (bad >> i & 1) {
                    constexpr int N = (int)Number<T>::kNan;
                    kr[i] = i32x4{N, N, N, N};
                }
        }
        if (kt + KEYS > end_key) {
#pragma unroll
            for (int i = 0; i < LI; ++i)
                if (kt + PER * i + to_key >= end_key) vr[i] = i32x4{0, 0, 0, 0};
        }
#pragma unroll
        for (int i = 0; i < LI; ++i) {
            *(i32x4*)(to + to_k + PER * i * KP) = chunk_moved<WHOLE>(kr[i], chunk, p.D);
            *(i32x4*)(to + to_v + PER * i * VP) = chunk_moved<WHOLE>(vr[i], chunk, p.D);
        }
    };

    // All keys of the range, in steps: use(kt, K and V in LDS) between two barriers each.
    auto sweep = [&](auto use) {
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
            use(kt, lds + turn * many_buffer(DP));
            if (kt + KEYS < end_key) store(kt + KEYS, lds + (turn ^ 1) * many_buffer(DP));
        }
    };
    f32x16 s[KT], o[DP / 32];
    float m = 0.0f, l;
    auto score = [&](int kt, const unsigned char* buf) {
#pragma unroll
        for (int t = 0; t < KT; ++t)
#pragma unroll
            for (int i = 0; i < 16; ++i) s[t][i] = 0.0f;
#pragma unroll
        for (int ks = 0; ks < KS; ++ks)
#pragma unroll
            for (int t = 0; t < KT; ++t) s[t] = mfma32(__builtin_bit_cast(x8, *(const i32x4*)(buf + (32 * t + l32) * KP + 32 * ks + 16 * half)), q[ks], s[t]);
        in_turn<KS * KT, 1, 1, 6, 0, 0>();
        if (kt + KEYS > end_key) {
            int left = end_key - kt;
            arrived_scalar(left);              // (or its comparisons are made in every step, ahead of the branch)
            const int seen = left - 4 * half;
#pragma unroll
            for (int t = 0; t < KT; ++t)
#pragma unroll
                for (int i = 0; i < 16; ++i)
                    if (32 * t + (i & 3) + 8 * (i >> 2) >= seen) s[t][i] = -__builtin_inff();
        }
    };
    // the largest score of a step, times scale_log2
    auto largest = [&]() {
        float top = s[0][0];
#pragma unroll
        for (int t = 0; t < KT; ++t)
#pragma unroll
            for (int i = 0; i < 16; ++i) top = fmaxf(top, s[t][i]);
        return fmaxf(top, __shfl_xor(top, 32)) * p.scale_log2;
    };
    auto finite = [&]() {
        float zero = 0.0f;                     // (or NaN)
#pragma unroll
        for (int dt = 0; dt < DP / 32; ++dt)
#pragma unroll
            for (int i = 0; i < 16; ++i) zero = __builtin_fmaf(o[dt][i], 0.0f, zero);
        return zero == 0.0f;
    };
    int* const again = (int*)(lds + 2 * many_buffer(DP));
    if (tid == 0) *again = 0;                  // (the sweep's first barrier is between this and what follows)
    for (bool known = false;;) {
        bool over = false;
        l = 0.0f;
#pragma unroll
        for (int dt = 0; dt < DP / 32; ++dt)
#pragma unroll
            for (int i = 0; i < 16; ++i) o[dt][i] = 0.0f;
        sweep([&](int kt, const unsigned char* buf) {
            const unsigned v_at = lds_base_of((void*)(buf + KEYS * KP)) + (4 * half + (l16 >> 2)) * VP + 32 * ((lane >> 4) & 1) + 8 * (l16 & 3);
            score(kt, buf);
            if (kt == first_key && !known) m = largest() - LIFT;
            if constexpr (!WIDE) over |= largest() > m + 15.0f;              // (no branch here)
            const float shift = m == -__builtin_inff() ? 0.0f : m;
            // Sixteen keys at a time; the weights and V of the next are made and read while the matrix cores are on these.
            x8 vf[DP / 32], pf[TERMS], next[TERMS];
            auto weigh = [&](int st, x8 (&w)[TERMS]) {
#pragma unroll
                for (int i = 0; i < 8; ++i) {
                    float left = exp2_fast(__builtin_fmaf(s[st >> 1][8 * (st & 1) + i], p.scale_log2, -shift));
                    l += left;
#pragma unroll
                    for (int k = 0; k < TERMS; ++k) {
                        w[k][i] = (T)left;
                        left -= (float)(T)left;
                    }
                }
            };
            auto read_v = [&](int st, int dt) {
                const s16x4 v0 = lds_read_transposed(v_at + 16 * st * VP + 64 * dt), v1 = lds_read_transposed(v_at + (16 * st + 8) * VP + 64 * dt);
                return __builtin_bit_cast(x8, __builtin_shufflevector(v0, v1, 0, 1, 2, 3, 4, 5, 6, 7));
            };
#pragma unroll
            for (int dt = 0; dt < DP / 32; ++dt) vf[dt] = read_v(0, dt);
            weigh(0, pf);
            __builtin_amdgcn_sched_barrier(0);
#pragma unroll
            for (int st = 0; st < 2 * KT; ++st) {
                if (st + 1 < 2 * KT) weigh(st + 1, next);
#pragma unroll
                for (int dt = 0; dt < DP / 32; ++dt) {
#pragma unroll
                    for (int k = 0; k < TERMS; ++k) o[dt] = mfma32(vf[dt], pf[k], o[dt]);
                    if (st + 1 < 2 * KT) vf[dt] = read_v(st + 1, dt);
                }
#pragma unroll
                for (int k = 0; k < TERMS; ++k) pf[k] = next[k];
                if constexpr (TERMS == 2) in_turn<(DP / 32) * 2, 1, 1, 0, 20 / (DP / 32), 4 / (DP / 32)>();
                else in_turn<DP / 32, TERMS, 2, 0, 20 * TERMS / (DP / 32), 8 / (DP / 32)>();
                __builtin_amdgcn_sched_barrier(0);
            }
        });
        // (both halves' weights: a lane's O is of the keys of both)
        if constexpr (WIDE) over = !(l + __shfl_xor(l, 32) < (finite() ? 0x1p40f : (float)(end_key - first_key + 1))) || m == -__builtin_inff();
        if (over) *again = 1;
        __syncthreads();
        if (!*again || known) break;
        known = true;
        m = -__builtin_inff();
        sweep([&](int kt, const unsigned char* buf) {
            score(kt, buf);
            m = fmaxf(m, largest() - LIFT);
        });
        __syncthreads();
        if (tid == 0) *again = 0;
    }
    l += __shfl_xor(l, 32);
    const uint64_t odd = __ballot(row < row_end && !finite() && l == l);
    // O turned through the wave's piece of LDS (nobody reads the buffers any more), 32 features at a time, so that a store has whole lines.
    constexpr int TP = 36;                     // floats from row to row
    float* const turned = (float*)lds + wave * 32 * TP;
    const int64_t stride = p.prefix_splits + p.own_splits, part0 = ((int64_t)h * p.rows + row0 + 32 * wave) * stride + slot;
    const int rows_here = row_end - row0 - 32 * wave;
#pragma unroll
    for (int dt = 0; dt < DP / 32; ++dt) {
#pragma unroll
        for (int i = 0; i < 4; ++i) *(f32x4*)(turned + l32 * TP + 8 * i + 4 * half) = f32x4{o[dt][4 * i], o[dt][4 * i + 1], o[dt][4 * i + 2], o[dt][4 * i + 3]};
        __builtin_amdgcn_wave_barrier();
#pragma unroll
        for (int i = 0; i < 4; ++i) {
            const int r = 8 * i + (lane >> 3), d = 32 * dt + 4 * (lane & 7);
            const f32x4 x = *(const f32x4*)(turned + r * TP + 4 * (lane & 7));
            if (r < rows_here && d < p.D) *(f32x4*)(p.part_o + (part0 + r * stride) * p.D + d) = x;
        }
        __builtin_amdgcn_wave_barrier();
    }
    if (half == 0 && row < row_end) *(f32x2*)(p.part_ml + (part0 + l32 * stride) * 2) = f32x2{m, l};
    return (unsigned)(odd | odd >> 32);
}

// Few rows: ranges of the prefix for 16 * MT rows, and of the sequences' own tokens for 16 * OWN.  WHOLE: D is DP.  GROUPED: 16 keys share a page.
// Workgroups go to the 8 XCDs in turn; those of one range, which differ in their rows alone, are given to one XCD (one L2).
template <class T, int DP, int MT, int OWN, int TERMS, bool WHOLE, bool GROUPED>
__global__ void __launch_bounds__(256, few_waves(DP, MT)) attend_few_kernel(const AttendParams p) {
    extern __shared__ __align__(16) unsigned char lds[];
    const int xcd = (int)blockIdx.x & 7, place = (int)blockIdx.x >> 3;
    if (place < p.prefix_per_xcd) {
        const int i = xcd * p.prefix_per_xcd + place;
        const int tile = i % p.prefix_tiles, rest = i / p.prefix_tiles, split = rest % p.prefix_splits, h = rest / p.prefix_splits;
        if (h >= p.Hk) return;
        const int first = split * p.prefix_chunk, end = min(p.P, first + p.prefix_chunk);
        const unsigned odd = attend_few<T, DP, MT, TERMS, WHOLE, GROUPED>(p, p.prefix_pages, h, first, end, tile * 16 * MT, p.rows, false, Sequence{}, split, 4, true, lds);
        if (__builtin_expect(odd != 0, 0)) settle_odd<T, DP>(p.prefix_pages, h, first, end, tile * 16 * MT, odd, false, Sequence{}, split);
        return;
    }
    // Sequences differ in length, so that their ranges go round the XCDs; the tiles of a range stay together, and the heads of a token where they are
    // neighbours in memory, with lines that two heads share.
    const int at_once = 4 / p.own_share, own_place = (place - p.prefix_per_xcd) * at_once + __builtin_amdgcn_readfirstlane((int)threadIdx.x >> 6) / p.own_share;
    const int tile = own_place % p.own_tiles, j = own_place / p.own_tiles, together = p.own_heads_together;
    const int rest = j / together * 8 + xcd, inner = j % together, heads = p.Hk / together;       // together: Hk or 1
    const int h = together > 1 ? inner : rest / p.own_splits % heads, bs = together > 1 ? rest : rest / p.own_splits / heads * p.own_splits + rest % p.own_splits;
    const int split = bs % p.own_splits, b = min(bs / p.own_splits, p.B - 1);
    const bool keep = bs / p.own_splits < p.B;
    const Sequence seq = sequence_of(p, b);
    const int steps = (seq.len + p.own_step - 1) / p.own_step, per = (steps + p.own_splits - 1) / p.own_splits, nG = p.n * p.G;
    const int seen = seq.base + (min((tile + 1) * 16 * OWN, nG) - 1) / p.G + 1;          // by the tile's last query
    const int first = min(split * per * p.own_step, seq.len), end = keep ? min(min(first + per * p.own_step, seq.len), max(first, seen)) : first;
    const unsigned odd = attend_few<T, DP, OWN, TERMS, WHOLE, GROUPED>(p, p.page_table + b * p.table_stride, h, first, end, b * nG + tile * 16 * OWN, (b + 1) * nG, true, seq,
                                                                p.prefix_splits + split, p.own_share, keep, lds);
    if (__builtin_expect(odd != 0, 0))
        settle_odd<T, DP>(p.page_table + b * p.table_stride, h, first, end, b * nG + tile * 16 * OWN, odd, true, seq, p.prefix_splits + split);
}

// Many rows: ranges of the prefix for 32 rows of each of NW waves, with P in TERMS terms.  XCDs as above.
template <class T, int DP, int NW, int TERMS, bool WHOLE>
__global__ void __launch_bounds__(64 * NW, DP > 128 ? NW / 4 : 2) attend_many_kernel(const AttendParams p) {
    extern __shared__ __align__(16) unsigned char lds[];
    const int i = ((int)blockIdx.x & 7) * p.prefix_per_xcd + ((int)blockIdx.x >> 3);
    const int tile = i % p.prefix_tiles, rest = i / p.prefix_tiles, split = rest % p.prefix_splits, h = rest / p.prefix_splits;
    if (h >= p.Hk) return;
    const int first = split * p.prefix_chunk, end = min(p.P, first + p.prefix_chunk);
    const unsigned odd = attend_many<T, DP, TERMS, NW, WHOLE>(p, p.prefix_pages, h, first, end, tile * 32 * NW, p.rows, split, lds);
    if (__builtin_expect(odd != 0, 0))
        settle_odd<T, DP>(p.prefix_pages, h, first, end, tile * 32 * NW + 32 * ((int)threadIdx.x >> 6), odd, false, Sequence{}, split);
}

// The parts of every row joined.  DP / 4 threads have four features each of a row's part, 2^lanes_log such groups share a row's parts, and
// the rest of the workgroup has other rows.  A group takes four parts at a time, loads ahead of sums, and the groups meet in LDS.
// One pass over the parts, bound by memory: 2048 rows of 33 parts of 128 features, 35 MB, 8.4 us, 4.1 TB/s; with few parts by its launch, 2.4 us.
template <int DP>
__global__ void __launch_bounds__(256) combine_kernel(const AttendParams p, const int lanes_log) {
    constexpr int PER = DP / 4, GROUPS = 256 / PER;
    __shared__ f32x4 parts[GROUPS][PER];
    __shared__ float tops[GROUPS], totals[GROUPS];
    const int group = (int)threadIdx.x / PER, d = (int)(threadIdx.x % PER) * 4, lanes = 1 << lanes_log;
    const int all = p.Hk * p.rows;
    const int row = (int)blockIdx.x * (GROUPS >> lanes_log) + (group >> lanes_log), at_row = min(row, all - 1), at_d = min(d, p.D - 4);
    const int slots = p.prefix_splits + p.own_splits;
    float top = -__builtin_inff(), total = 0.0f;
    f32x4 x = f32x4{0, 0, 0, 0};
    for (int s0 = group & (lanes - 1); s0 < slots; s0 += 4 * lanes) {
        float m[4], l[4];
        f32x4 o[4];
#pragma unroll
        for (int i = 0; i < 4; ++i) {
            const int s = s0 + i * lanes;
            const int64_t at = (int64_t)at_row * slots + min(s, slots - 1);
            m[i] = p.part_ml[at * 2];
            l[i] = p.part_ml[at * 2 + 1];
            o[i] = *(const f32x4*)(p.part_o + at * p.D + at_d);
            if (s >= slots) {
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
    if (lanes > 1) {
        parts[group][d / 4] = x;
        if (d == 0) {
            tops[group] = top;
            totals[group] = total;
        }
        __syncthreads();
        if (group & (lanes - 1)) return;
        float now = top;
        for (int g = 1; g < lanes; ++g) now = fmaxf(now, tops[group + g]);
        const float shift = now == -__builtin_inff() ? 0.0f : now;
        const float factor = exp2_fast(top - shift);
        x *= factor;
        total *= factor;
        for (int g = 1; g < lanes; ++g) {
            const float f = exp2_fast(tops[group + g] - shift);
            total += f * totals[group + g];
            x += parts[group + g][d / 4] * f;
        }
        top = now;
    }
    if (row >= all || d >= p.D) return;
    const int h = row / p.rows, in_head = row - h * p.rows, nG = p.n * p.G;
    const int b = in_head / nG, in_seq = in_head - b * nG, j = in_seq / p.G, g = in_seq - j * p.G;
    const Sequence seq = sequence_of(p, b);
    const bool real = seq.bad || j < seq.queries;
    if (seq.bad) total = __builtin_nanf("");
    x = !real || total == 0.0f ? f32x4{0, 0, 0, 0} : x * (1.0f / total);
    store_result(p, b * p.out_sequence + j * p.out_token + (int64_t)(h * p.G + g) * p.out_head + d, x);
    if (p.lse && d == 0) p.lse[((int64_t)b * p.n + j) * p.Hk * p.G + h * p.G + g] = real ? lse_of(top, total) : -__builtin_inff();
}

}  // namespace
