// Attention of chunks of new tokens, packed one sequence behind the other, over a paged cache.
// Part of the translation units of the chunks' kernels, one for each type of the cache and of the outputs (included there, in this order).
#pragma once

#include "matrix_parts.hip.h"

namespace {

using namespace vlut_chunk;

// ---------------------------------------------------------------------------------------------
// Query j of a sequence with n new tokens and len tokens in all has position pos = len - n + j and sees the keys max(0, pos - window + 1) .. pos:
//   s = scale * q . k,  m a number near max s,  l = sum exp(s - m),  O = sum exp(s - m) v,  output O / l;   nothing seen: 0
// A row is a query token and one of the G query heads that read a key head, token by token, so that the rows of a tile are neighbours in position and see
// nearly the same keys.  A workgroup has a tile of rows of one sequence and key head and a part of the keys that any of them sees.
//   Many rows: tiles of 128, RW = 4 waves of 32, whose keys and values go through LDS for all of them, 64 keys a step; two workgroups on a unit, or where tiles are few
//   KW = 2 such groups of waves with every other 64 keys each, which meet in LDS at the end.
//   Few rows (up to 32: single tokens, drafts): one tile of 32 rows and KW = 4 waves (of more than 128 features 2) with 32 of a step's keys each, two workgroups on a unit.
// A sequence's tile of more keys than a part holds is several workgroups; combine_chunks joins the parts: with M = max m_i the sums of exp(m_i - M) l_i and
// exp(m_i - M) O_i are those of the whole.
//
// Both products run transposed on the matrix cores, S^T = K Q^T and O^T = V^T P^T: a query is a column, its m and l are one number per lane, and P^T goes from
// one product to the next in its registers, the keys of both in the order in which S^T comes out.  V^T is read out of the row-major V in LDS by
// transposing reads.
// m is not the running maximum: it is the largest score of the first step in which the row sees anything, and stays, so that nothing but sums is in the loop
// and O is never multiplied.  Weights are powers of two of the scores above m and may be as large as their type's range; where that does not do (bf16: l
// shows 2^40 or O 2^64; fp16: O is no number) the part is begun again with the largest of all its scores, which a sweep over K finds, and
// (bf16) where O passes 2^64 all the same, once more with weights that add up to 1 at most.
// P goes to the second product in terms of the cache's type, each what the rounding of those before it left: two for 16-bit outputs (one would be a second rounding of the
// size of the output's own: bf16 2.3e-3 of the result, not 1.7e-3), for fp32 those that carry 24 bits, three of bf16 or two of fp16.
// What bounds it.  Few rows: the bytes of keys and values; 64 sequences of 3100 keys, 8 key heads of 128, 145 us or 5.3 TB/s, what a large copy reaches; 13 sequences and
// 32 key heads of 100 (windows of 1024) 38 us.  A single sequence: the way through memory, 10 us, of which a step is 1.  Many rows: a step of a wave is 1536 cycles of the
// matrix cores, some 1200 of its 32 exponentials and roundings a lane and 256 of LDS, which four waves share, so that two waves of a SIMD cover each other in part; 16384 tokens,
// 32 and 8 heads of 128, 2850 us: 0.77 PFLOP/s of the formula's operations, 1.16 with the weights' second term, 0.86 of what a large product reaches; 4096 tokens of 20
// and 5 heads 150 us (0.57 and 0.86), of which a quarter is units that wait for the last tiles.  fp32 outputs, three products with V instead of two, a third longer.
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

// Terms of the cache's type that carry the weights of one row to outputs of type O: 24 bits for fp32, two for 16 bits.
template <class T, class O>
__host__ __device__ constexpr int terms() { return sizeof(O) == 4 ? Number<T>::kTerms : 2; }
template <class O>
__device__ __forceinline__ void store_four(void* out, int64_t at, const f32x4& o) {
    if constexpr (sizeof(O) == 4) *(dword_aligned_f32x4*)((float*)out + at) = o;
    else {
        typedef O x4 __attribute__((ext_vector_type(4), aligned(4)));
        *(x4*)((O*)out + at) = x4{(O)o.x, (O)o.y, (O)o.z, (O)o.w};
    }
}

// What a workgroup works on.
struct Tile {
    Chunk seq;
    int b, h, row0, row_end;           // rows of the sequence and key head: query * G + head
    int j0, g0;                        // row0's
    int first, end;                    // keys
    int split, direct;
};
// The query of row row0 + r, r < 256: exact, as (x + 1/2) / G is 1 / (2 G) away from a whole number at least, and x far below 2^21.
__device__ __forceinline__ int query_of(const ChunkParams& p, const Tile& t, int r) { return t.j0 + (int)(((float)(t.g0 + r) + 0.5f) * p.inverse_g); }
// Where a row of a tile's part is among the parts: `row` where rows are few, else the query and its head.
template <bool FEW>
__device__ __forceinline__ int64_t part_at(const ChunkParams& p, const Chunk& c, int b, int h, int row, int j, int head, int split) {
    if constexpr (FEW) return (((int64_t)split * p.B + b) * p.Hk + h) * p.few_rows + row;
    return ((int64_t)split * p.N + c.start + j) * (p.Hk * p.G) + head;
}

// Values that are no numbers.  Zeros stand for them in the products' steps of which some row does not see every key (0 times them would reach every row); they, and
// infinities that rows see, which weights of 0 or in several terms make NaN of, are settled here, once the results are stored, by a look at the part's values: a row's
// feature with such values among the keys that it sees is their sum, with weights of 1, or 0 for a score of -inf.  NaN with infinities of both signs.
// Rows: those of `rows` (bits, from row0 on).  Not part of the loops: a flag and a look at the results; where there is something to settle, a read of V per wave.
template <class T, class O, int DP, bool FEW>
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
            const int r = __builtin_ctz(left), row = row0 + r, j = query_of(p, t, row - t.row0), head = t.h * p.G + row - j * p.G, pos = t.seq.base + j;
            if (key > pos || key <= pos - p.window) continue;
            const T* const q = (const T*)p.q + (t.seq.start + j) * p.q_token + head * p.q_head + d;
            float s = 0.0f;
            for (int f = 0; f < F && has; ++f)
                if (d + f < p.D) s += (float)q[f] * (float)k[f];
            for (int m = 1; m < 64; m *= 2) s += __shfl_xor(s, m);
            const float weight = s > -__builtin_inff() ? 1.0f : 0.0f;
            O* const out = (O*)p.out + (t.seq.start + j) * p.out_token + head * p.out_head + d;
            float* const part = (FEW ? p.few_o : p.many_o) + part_at<FEW>(p, t.seq, t.b, t.h, row, j, head, t.split) * p.D + d;
            for (int f = 0; f < F && has; ++f)
                if (is_odd(x[f])) {
                    float sum = weight * x[f];
                    if (touched[f] >> r & 1) sum += t.direct ? (float)out[f] : part[f];
                    touched[f] |= 1u << r;
                    if (t.direct) out[f] = (O)sum;
                    else part[f] = sum;
                }
        }
    }
}

// The kernel's parameters, its first argument, read again: what is wanted behind the loops only would wait in registers throughout.
__device__ __forceinline__ const ChunkParams& parameters() {
#if defined(__HIP_DEVICE_COMPILE__)
    auto at = __builtin_amdgcn_kernarg_segment_ptr();
    asm volatile("" : "+s"(at));
    return *(const ChunkParams*)at;
#else
    static ChunkParams none;
    return none;
#endif
}
// The compiler knows nothing of x from here on.
__device__ __forceinline__ void stay(int& x) {
#if defined(__HIP_DEVICE_COMPILE__)
    asm volatile("" : "+v"(x));
#endif
}

__device__ __forceinline__ void stay_scalar(unsigned& x) {
#if defined(__HIP_DEVICE_COMPILE__)
    asm volatile("" : "+s"(x));
#endif
}
__device__ __forceinline__ void pinned(float& x) {
#if defined(__HIP_DEVICE_COMPILE__)
    asm volatile("" : "+v"(x));
#endif
}

// 16 bytes (or a dword) per lane from `base` + `at` on to LDS, lane after lane from `to` on.  Written out: the compiler, when it issues such a load itself, waits for all of them
// ahead of every LDS read that follows.  No result register; the LDS address is in M0.
#if defined(__HIP_DEVICE_COMPILE__)
__device__ __forceinline__ void load_to_lds(const unsigned char* base, unsigned at, unsigned to) {
    asm volatile("s_mov_b32 m0, %0\n\ts_nop 0\n\tglobal_load_lds_dwordx4 %1, %2" ::"s"(to), "v"(at), "s"(base) : "memory", "m0");
}
// A dword of the lanes whose `at` is below `end`; all lanes of the wave have to be active.
__device__ __forceinline__ void load_dword_to_lds(const unsigned char* base, unsigned at, unsigned from, unsigned end, unsigned to) {
    asm volatile("s_mov_b32 m0, %0\n\tv_cmpx_gt_u32_e32 vcc, %3, %2\n\tglobal_load_lds_dword %1, %4\n\ts_mov_b64 exec, -1" ::"s"(to), "v"(from), "v"(at), "s"(end), "s"(base) : "memory", "m0", "vcc");
}
template <int N>
__device__ __forceinline__ void wait_loads() { asm volatile("s_waitcnt vmcnt(%0)" ::"n"(N < 63 ? N : 63) : "memory"); }
__device__ __forceinline__ void wait_lds() { asm volatile("s_waitcnt lgkmcnt(0)" ::: "memory"); }
#else
inline __device__ void load_to_lds(const unsigned char*, unsigned, unsigned) {}
inline __device__ void load_dword_to_lds(const unsigned char*, unsigned, unsigned, unsigned, unsigned) {}
template <int N>
inline __device__ void wait_loads() {}
inline __device__ void wait_lds() {}
#endif
template <class V>
__device__ __forceinline__ V& at_lds(unsigned at) {
#if defined(__HIP_DEVICE_COMPILE__)
    return *(V*)(__attribute__((address_space(3))) V*)at;
#else
    static V none;
    return none;
#endif
}

// Without what is no number: zeros for it, and whether there was any.
template <class T>
__device__ __forceinline__ i32x4 without_odd(i32x4 v, unsigned& odd) {
    constexpr unsigned high = Number<T>::kExponents & 0xffff0000u, low = Number<T>::kExponents & 0xffffu;
#pragma unroll
    for (int w = 0; w < 4; ++w) {
        const unsigned x = (unsigned)v[w];
        const unsigned drop = ((x & high) == high ? 0xffff0000u : 0u) | ((x & low) == low ? 0xffffu : 0u);
        v[w] = (int)(x & ~drop);
        odd |= drop;
    }
    return v;
}

struct Yes { static constexpr bool value = true; };
struct No { static constexpr bool value = false; };
template <int N>
struct Count { static constexpr int value = N; };

// A tile's part.  Where keys and values are loaded straight to LDS they are asked for AHEAD steps ahead, addresses worked out once per wave and 8 keys.  Each stage is
// exactly LOADS loads per wave, also past the end of the part, where its last keys are loaded again, so that vmcnt((AHEAD - 1) * LOADS) stands for "the
// stage that was asked for first is there"; what else a wave loads meanwhile only makes that wait longer.
// (Through registers instead, 4096 tokens took 188 us, not 150, and 64 sequences 218, not 180, when all else was alike.)
// Rows of LDS are DP features one behind the other, 16-byte chunks c at c ^ f(row): of keys, so that 16 rows' chunks lie in 64 banks; of values, so that the four
// rows of a transposing read do.  Chunks behind D are not loaded: zeros from before the first stage.  Rows of an odd number of fours (kRuns) are one behind the other as they
// are in memory, in which place they are in different banks by themselves; what is read behind a row is the next one's beginning, and not used.  (A dword a lane instead,
// whatever the rows' places: 13 sequences of 32 heads of 100 56 us, not 44.)
// Where rows are few each wave has its keys for itself, and none waits for another; a step's keys are asked for as soon as the first product is done with
// the ones before, its values behind the second.
template <class T, class O, int DP, int RW, int KW, int LOAD>
__device__ __forceinline__ void attend_chunk(const ChunkParams& p, const Tile& t, unsigned char* lds) {
    typedef typename Number<T>::x8 x8;
    constexpr int TERMS = terms<T, O>();
    constexpr bool FEW = RW == 1, WIDE = Number<T>::kWide, DIRECT = LOAD != kThroughRegisters, RUNS = LOAD == kRuns, OWN_KEYS = own_keys(RW, LOAD);
    constexpr int NW = RW * KW, WK = wave_keys(DP, RW), KT = WK / 32, KEYS = step_keys(DP, RW, KW), KS = DP / 16, CH = DP / 8, GK = 64 / CH, DT = DP / 32;
    // Of a SIMD's two waves the one with matrix instructions alone goes first, then the one whose products with V have weights between them, so that they take turns: 1024 behind
    // 16384 468 -> 429 us, behind 8192 229 -> 217, 4096 tokens 151 -> 148.  Little either way for 64 features, whose products are half as long beside as many weights (133 -> 132),
    // and for 256, of which a SIMD has one wave (132 -> 132): not there.
    constexpr bool TURNS = !FEW && DP == 128;
    // What a row's reference weighs.  fp16: weights below 2^-25 are lost, n 2^-25 for n keys, which beside 2^4 is what sums of n keys in 32 bits may be off, n / 32 half steps; more
    // where that leaves room enough for scores after the first step's, and all that there is where the largest of all is known.
    constexpr float LIFT = 0.5f * Number<T>::kLift, FIRST_LIFT = 4.0f / 14.0f * Number<T>::kLift;
    // The last time that a part is worked on: with the largest of all scores; bf16, where sums of values near the type's largest are no numbers, with weights that add up to 1.
    constexpr int LAST = WIDE ? 2 : 1;
    const int tid = (int)threadIdx.x, lane = tid & 63, wave = __builtin_amdgcn_readfirstlane(tid >> 6), rw = wave % RW, kw = wave / RW;
    const int l32 = lane & 31, half = lane >> 5, l16 = lane & 15;
    const int wave_row0 = t.row0 + 32 * rw, row = wave_row0 + l32;
    const int first_key = t.first, end_key = t.end;

    // behind the buffers: the waves' m and l where they share rows, where the rows' results go and their factors, flags (the part is to be begun again,
    // for the first and the second time, [0] and [2]; there is something to settle, [1]), pages' numbers
    float* const row_m = (float*)(lds + tile_bytes(DP, RW, KW, LOAD));
    float* const row_l = row_m + 32 * NW;
    int64_t* const row_to = (int64_t*)(row_l + 32 * NW);
    float* const row_factor = (float*)(row_to + 32 * NW);
    int* const again = (int*)(row_factor + 32 * NW);
    int* const page_ids = again + 4;
    if (tid == 0) again[0] = again[1] = again[2] = 0;
    if constexpr (LOAD == kDwords || LOAD == kVectors) {
        for (int x = 16 * tid; x < tile_bytes(DP, RW, KW, LOAD); x += 16 * 64 * NW) *(i32x4*)(lds + x) = i32x4{0, 0, 0, 0};
    }
    wg_barrier_lds();                                                  // (they are set ahead of the first step's barrier)

    // rows past the tile's end do as its last one
    const int real = min(row, t.row_end - 1), j = query_of(p, t, real - t.row0), pos = t.seq.base + j;
    x8 q[KS];
    {
        const T* const src = (const T*)p.q + (t.seq.start + j) * p.q_token + (int64_t)(t.h * p.G + real - j * p.G) * p.q_head;
#pragma unroll
        for (int ks = 0; ks < KS; ++ks) {
            const int chunk = 2 * ks + half;
            q[ks] = __builtin_bit_cast(x8, chunk_moved<LOAD == kWholeVectors>(*(const dword_aligned_i32x4*)(src + chunk_at<LOAD == kWholeVectors>(chunk, p.D)), chunk, p.D));
        }
    }
    const int sees_from = max(0, pos - p.window + 1), sees_to = min(end_key, pos + 1);
    const bool blind = sees_to <= max(sees_from, first_key);           // nothing of this part
    // of the wave's rows, and of the workgroup's: from where to where all of them see
    auto position = [&](int of) { return t.seq.base + __builtin_amdgcn_readfirstlane(query_of(p, t, min(of, t.row_end - 1) - t.row0)); };
    const int low = position(wave_row0), high = position(wave_row0 + 31);
    const int all_from = max(0, high - p.window + 1), all_to = min(end_key, low + 1);
    const int tile_from = max(0, position(t.row_end - 1) - p.window + 1), tile_to = min(end_key, position(t.row0) + 1);

    // Where the row's result and its sums go, worked out while the first keys are on their way; the waves that share a row have it both.
    int64_t row_sums;
    {
        const int its = query_of(p, t, row - t.row0), head = t.h * p.G + row - its * p.G;
        const int64_t part = part_at<FEW>(p, t.seq, t.b, t.h, row, its, head, t.split);
        row_sums = t.direct ? (int64_t)(t.seq.start + its) * (p.Hk * p.G) + head : part;
        if (half == 0) row_to[FEW ? l32 : 32 * wave + l32] = t.direct ? (t.seq.start + its) * p.out_token + head * p.out_head : part * p.D;
    }

    const int32_t* const pages = p.page_table + t.b * p.table_stride;
    const T* const kh = (const T*)p.k + t.h * p.k_head;
    const T* const vh = (const T*)p.v + t.h * p.v_head;
    const int page_log = p.page_log, mask = (1 << page_log) - 1, last = end_key - 1;
    const float scale_log2 = p.scale_log2;

    // Where a lane reads: of keys, 8 features of row l32 (and 32 rows further); of values, a corner of a transposing read.
    constexpr bool TURNED = DIRECT && !RUNS;
    // (bytes of a row)
    const int row_k = RUNS ? 2 * p.D : k_pitch(DP, LOAD), row_v = RUNS ? 2 * p.D : v_pitch(DP, LOAD);
    auto turn_k = [](int r) { return DP == 64 ? (r >> 1) & 7 : r & 15; };
    auto turn_v = [](int r) { return DP == 64 ? 4 * ((r >> 1) & 1) : 4 * (r & 3); };
    const unsigned k_lane = (unsigned)(l32 * row_k + 16 * (TURNED ? half ^ turn_k(l32) : half));
    const int v_row = 4 * half + (l16 >> 2), v_chunk = 2 * ((lane >> 4) & 1) + ((l16 & 3) >> 1);
    const unsigned v_lane = (unsigned)(v_row * row_v + 16 * (TURNED ? v_chunk ^ turn_v(v_row) : v_chunk) + 8 * (l16 & 1));
    auto k_at = [&](unsigned base, int ks) { return TURNED ? (base + k_lane) ^ (unsigned)(32 * ks) : base + k_lane + (unsigned)(32 * ks); };
    auto v_at = [&](unsigned base, int dt) { return TURNED ? (base + v_lane) ^ (unsigned)(64 * dt) : base + v_lane + (unsigned)(64 * dt); };
    const unsigned lds0 = lds_base_of(lds);

    // All keys of the part, in steps: multiply(first key of the step, where the wave's keys are), weigh_up(first key, where its values are).
    auto sweep = [&](auto multiply, auto weigh_up) {
        if (first_key >= end_key) return;
        if constexpr (DIRECT) {
            // Of a load: its bytes, rows or the parts of one, loads of a wave and step.  OWN: keys that a wave loads.
            constexpr int UNIT = LOAD == kDwords ? 4 : 16, BYTES = 64 * UNIT, ROW = 2 * DP, RPI = BYTES > ROW ? BYTES / ROW : 1, SPLIT = ROW > BYTES ? ROW / BYTES : 1;
            // (runs: 8 keys are D vectors)
            constexpr int RUN_LOADS = DP / 64;
            constexpr int OWN = OWN_KEYS ? WK : WK / RW, LOADS = RUNS ? OWN / 8 * RUN_LOADS : OWN / RPI * SPLIT, PERIOD = UNIT == 16 ? 16 / RPI : 1;
            constexpr int AHEAD = OWN_KEYS ? 1 : ahead(DP), PART = WK * 2 * DP;           // bytes of a stage's keys, or values
            static_assert(OWN % 8 == 0 && 8 % RPI == 0, "whole groups of 8 keys");
            // the rings of the wave's group (or of the wave alone), the wave's keys in a step and where they are in a stage
            const unsigned k_ring = lds0 + kw * ring_bytes(DP, RW), v_ring = k_ring + ring(DP, RW) * PART, v_ring_end = v_ring + ring(DP, RW) * PART;
            const int in_stage = OWN_KEYS ? 0 : OWN * rw, own0 = WK * kw + in_stage;
            const unsigned char *const kb = (const unsigned char*)kh, *const vb = (const unsigned char*)vh;
            const unsigned k_page = 2u * (unsigned)p.k_page, v_page = 2u * (unsigned)p.v_page, k_token = 2u * (unsigned)p.k_token, v_token = 2u * (unsigned)p.v_token;
            const int row_in = lane * UNIT / ROW;
            const unsigned row_bytes = 2u * (unsigned)p.D, run_bytes = 8 * row_bytes;
            // vectors: a lane's offsets, which repeat every 16 rows, and whether there is such a chunk
            unsigned k_from[PERIOD], v_from[PERIOD];
            bool has_k[PERIOD], has_v[PERIOD];
            if constexpr (UNIT == 16 && !RUNS) {
#pragma unroll
                for (int x = 0; x < PERIOD; ++x) {
                    const int r = in_stage + RPI * x + row_in, ck = (lane % CH) ^ turn_k(r), cv = (lane % CH) ^ turn_v(r);
                    k_from[x] = (unsigned)row_in * k_token + 16u * (unsigned)ck;
                    v_from[x] = (unsigned)row_in * v_token + 16u * (unsigned)cv;
                    has_k[x] = LOAD == kWholeVectors || 16u * (unsigned)ck < row_bytes;
                    has_v[x] = LOAD == kWholeVectors || 16u * (unsigned)cv < row_bytes;
                }
            }
            // dwords: a lane's place in its row
            const unsigned in_row = (unsigned)(lane * UNIT % ROW), k_in = (unsigned)row_in * k_token, v_in = (unsigned)row_in * v_token;
            for (int s0 = first_key; s0 < end_key; s0 += stretch(RW, KW)) {
                const int s1 = s0 + min(end_key - s0, stretch(RW, KW)), id0 = s0 >> page_log, ids = ((s1 - 1) >> page_log) - id0 + 1;
                if (s0 > first_key) {
                    wait_loads<0>();
                    __syncthreads();           // (nobody reads the stretch before any more)
                }
                for (int x = tid; x < ids; x += 64 * NW) {
                    const int id = pages[id0 + x];
                    page_ids[x] = (unsigned)id < (unsigned)p.pages ? id : -1;
                }
                __syncthreads();
#pragma unroll
                for (int ks = 0; ks < KS; ++ks) arrived(q[ks]);
                const int last_group = (s1 - 1) & ~7;
                unsigned bad = 0;              // a bit for every 8 keys of the wave in every stage, the newest lowest, that are in no page
                // a stage's keys (Yes, No), values (No, Yes) or both
                auto issue = [&](int kt, unsigned k_stage, unsigned v_stage, auto keys, auto values) {
                    // (or multiples of these wait in registers, more than there are)
                    unsigned k_step = k_token, v_step = v_token;
                    stay_scalar(k_step);
                    stay_scalar(v_step);
#pragma unroll
                    for (int g = 0; g < OWN / 8; ++g) {
                        const int key = min(kt + own0 + 8 * g, last_group);
                        const int named = __builtin_amdgcn_readfirstlane(page_ids[(key >> page_log) - id0]);
                        if constexpr (keys.value) bad = bad << 1 | (unsigned)(named < 0);
                        const unsigned id = (unsigned)max(named, 0), in_page = (unsigned)(key & mask);
                        const unsigned char* const k = kb + ((uint64_t)id * k_page + in_page * k_token);
                        const unsigned char* const v = vb + ((uint64_t)id * v_page + in_page * v_token);
                        if constexpr (RUNS) {
#pragma unroll
                            for (int part = 0; part < RUN_LOADS; ++part) {
                                const unsigned of = (unsigned)(16 * lane + BYTES * part), to = (unsigned)((in_stage + 8 * g) * row_k + BYTES * part);
                                if (of >= run_bytes) continue;
                                if constexpr (keys.value) load_to_lds(k, of, k_stage + to);
                                if constexpr (values.value) load_to_lds(v, of, v_stage + to);
                            }
                        } else
#pragma unroll
                        for (int i = 0; i < 8 / RPI; ++i) {
                            const int r = 8 * g + RPI * i;
                            const unsigned to_k = k_stage + (unsigned)((in_stage + r) * ROW), to_v = v_stage + (unsigned)((in_stage + r) * ROW);
                            if constexpr (UNIT == 16) {
                                const int x = r / RPI % PERIOD;
                                if constexpr (keys.value)
                                    if (has_k[x]) load_to_lds(k + (unsigned)(RPI * i) * k_step, k_from[x], to_k);
                                if constexpr (values.value)
                                    if (has_v[x]) load_to_lds(v + (unsigned)(RPI * i) * v_step, v_from[x], to_v);
                            } else {
                                const unsigned fk = 16u * (unsigned)turn_k(in_stage + r), fv = 16u * (unsigned)turn_v(in_stage + r);
#pragma unroll
                                for (int part = 0; part < SPLIT; ++part) {
                                    const unsigned ck = (in_row + (unsigned)(part * BYTES)) ^ fk, cv = (in_row + (unsigned)(part * BYTES)) ^ fv;
                                    if constexpr (keys.value)
                                        load_dword_to_lds(k + (unsigned)(RPI * i) * k_step, ck, RPI > 1 ? k_in + ck : ck, row_bytes, to_k + part * BYTES);
                                    if constexpr (values.value)
                                        load_dword_to_lds(v + (unsigned)(RPI * i) * v_step, cv, RPI > 1 ? v_in + cv : cv, row_bytes, to_v + part * BYTES);
                                }
                            }
                        }
                    }
                };
                // What the wave has loaded of the step kt, once it is there: a number that is no page (whoever sees its keys gets NaN), values of keys that not
                // every row sees.  newer: stages asked for since.
                auto mend_keys = [&](unsigned stage, int newer) {
                    const unsigned its = bad >> (newer * (OWN / 8)) & ((1u << (OWN / 8)) - 1);
                    constexpr int N = (int)Number<T>::kNan;
                    if (RUNS) {
                        if (its != 0)
                            for (int g = 0; g < OWN / 8; ++g)
                                for (unsigned of = 16u * (unsigned)lane; of < run_bytes && (its >> (OWN / 8 - 1 - g) & 1); of += BYTES)
                                    at_lds<i32x4>(stage + (unsigned)((in_stage + 8 * g) * row_k) + of) = i32x4{N, N, N, N};
                    } else if (its != 0) {
                        // (only what is loaded again: chunks behind D are zeros for every step)
#pragma unroll
                        for (int x = 0; x < OWN / GK; ++x) {
                            const int r = in_stage + GK * x + lane / CH, left = LOAD == kWholeVectors ? 8 : p.D - 8 * ((lane % CH) ^ turn_k(r));
                            if ((its >> (OWN / 8 - 1 - GK * x / 8) & 1) && left > 0)
                                at_lds<i32x4>(stage + (unsigned)((in_stage + GK * x) * ROW + 16 * lane)) = i32x4{N, N, left > 4 ? N : 0, left > 4 ? N : 0};
                        }
                    }
                };
                auto mend_values = [&](int kt, unsigned stage) {
                    if (kt + KEYS > tile_to || kt < tile_from) {
                        unsigned odd = 0;
                        if (RUNS) {
#pragma unroll
                            for (int g = 0; g < OWN / 8; ++g) {
                                // bytes of the keys that there are
                                const int there = min(max(end_key - (kt + own0 + 8 * g), 0), 8) * row_v;
#pragma unroll
                                for (int part = 0; part < RUN_LOADS; ++part) {
                                    const unsigned of = (unsigned)(16 * lane + BYTES * part), at = stage + (unsigned)((in_stage + 8 * g) * row_v) + of;
                                    if (of >= run_bytes) continue;
                                    i32x4 v = without_odd<T>(at_lds<i32x4>(at), odd);
                                    if ((int)of >= there) v.x = v.y = 0;
                                    if ((int)of + 8 >= there) v.z = v.w = 0;
                                    at_lds<i32x4>(at) = v;
                                }
                            }
                        } else
#pragma unroll
                        for (int x = 0; x < OWN / GK; ++x) {
                            const unsigned at = stage + (unsigned)((in_stage + GK * x) * ROW + 16 * lane);
                            i32x4 v = without_odd<T>(at_lds<i32x4>(at), odd);
                            if (kt + own0 + GK * x + lane / CH >= end_key) v = i32x4{0, 0, 0, 0};
                            at_lds<i32x4>(at) = v;
                        }
                        if (odd) again[1] = 1;
                    }
                };
                if constexpr (OWN_KEYS) {
                    issue(s0, k_ring, v_ring, Yes{}, No{});
                    issue(s0, k_ring, v_ring, No{}, Yes{});
                    for (int kt = s0; kt < s1; kt += KEYS) {
                        wait_loads<LOADS>();
                        mend_keys(k_ring, 0);
                        multiply(kt, k_ring);
                        wait_lds();            // (the reads are done: LDS may be written)
                        issue(kt + KEYS, k_ring, v_ring, Yes{}, No{});         // (behind the last step too, from the last keys)
                        wait_loads<LOADS>();
                        mend_values(kt, v_ring);
                        weigh_up(kt, v_ring);
                        wait_lds();
                        issue(kt + KEYS, k_ring, v_ring, No{}, Yes{});
                    }
                } else {
                    // stages: the one that is worked on, and the one that is asked for
                    unsigned now = 0, next = 0;
                    auto on = [&](unsigned& stage) { stage = v_ring + stage + PART == v_ring_end ? 0 : stage + PART; };
                    auto next_stage = [&](int kt) {
                        issue(kt, k_ring + next, v_ring + next, Yes{}, Yes{});
                        on(next);
                    };
#pragma unroll
                    for (int x = 0; x < AHEAD; ++x) next_stage(s0 + x * KEYS);
                    for (int kt = s0; kt < s1; kt += KEYS) {
                        wait_loads<2 * (AHEAD - 1) * LOADS>();
                        mend_keys(k_ring + now, AHEAD - 1);
                        mend_values(kt, v_ring + now);
                        wg_barrier_lds();      // the stage of step kt is there, for all waves, and nobody reads the one before any more
                        next_stage(kt + AHEAD * KEYS);                 // (behind the last step too, from the last keys)
                        multiply(kt, k_ring + now);
                        weigh_up(kt, v_ring + now);
                        on(now);
                    }
                }
            }
            wait_loads<0>();
        } else {
            constexpr int PER = 64 * NW / CH, LI = KEYS / PER, BYTES = stage_bytes(DP, RW, KW, LOAD);
            static_assert(PER * LI == KEYS, "whole loads");
            const int chunk = lane % CH, to_key = GK * wave + lane / CH;
            const unsigned to_k = (unsigned)(to_key * row_k + 16 * chunk), to_v = (unsigned)(KEYS * row_k + to_key * row_v + 16 * chunk);
            i32x4 kr[LI], vr[LI];
            int ids[LI];
            unsigned bad = 0;                  // ids: the next keys' pages; bad: a bit for each loaded key that is in none
            // (keys past the part read its last one: scores are masked, V is zeroed)
            auto look_up = [&](int kt) {
#pragma unroll
                for (int i = 0; i < LI; ++i) ids[i] = pages[min(kt + PER * i + to_key, last) >> page_log];
            };
            auto load = [&](int kt) {
                bad = 0;
#pragma unroll
                for (int i = 0; i < LI; ++i) {
                    const int in_page = min(kt + PER * i + to_key, last) & mask;
                    const bool page = (unsigned)ids[i] < (unsigned)p.pages;
                    bad |= page ? 0u : 1u << i;
                    const int64_t id = page ? ids[i] : 0;
                    kr[i] = *(const dword_aligned_i32x4*)(kh + id * p.k_page + in_page * p.k_token + chunk_at<false>(chunk, p.D));
                    vr[i] = *(const dword_aligned_i32x4*)(vh + id * p.v_page + in_page * p.v_token + chunk_at<false>(chunk, p.D));
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
                if (kt + KEYS > tile_to || kt < tile_from) {
                    unsigned odd = 0;
#pragma unroll
                    for (int i = 0; i < LI; ++i) {
                        if (kt + PER * i + to_key >= end_key) vr[i] = i32x4{0, 0, 0, 0};
                        vr[i] = without_odd<T>(vr[i], odd);
                    }
                    if (odd) again[1] = 1;
                }
#pragma unroll
                for (int i = 0; i < LI; ++i) {
                    *(i32x4*)(to + to_k + PER * i * row_k) = chunk_moved<false>(kr[i], chunk, p.D);
                    *(i32x4*)(to + to_v + PER * i * row_v) = chunk_moved<false>(vr[i], chunk, p.D);
                }
            };
            const unsigned own_k = (unsigned)(WK * kw * row_k), own_v = (unsigned)(KEYS * row_k + WK * kw * row_v);
            look_up(first_key);
            load(first_key);
            look_up(first_key + KEYS);
#pragma unroll
            for (int ks = 0; ks < KS; ++ks) arrived(q[ks]);
            store(first_key, lds);
            int turn = 0;
            for (int kt = first_key; kt < end_key; kt += KEYS, turn ^= 1) {
                wg_barrier_lds();
                load(kt + KEYS);               // (behind the last step too, from the last keys)
                look_up(kt + 2 * KEYS);
                if constexpr (stages(RW) == 2) {
                    multiply(kt, lds0 + turn * BYTES + own_k);
                    weigh_up(kt, lds0 + turn * BYTES + own_v);
                    if (kt + KEYS < end_key) store(kt + KEYS, lds + (turn ^ 1) * BYTES);
                } else {
                    multiply(kt, lds0 + own_k);
                    weigh_up(kt, lds0 + own_v);
                    if (kt + KEYS < end_key) {
                        wg_barrier_lds();
                        store(kt + KEYS, lds);
                    }
                }
            }
        }
    };
    f32x16 s[KT], o[DT];
    float m = 0.0f, l;
    auto multiply = [&](int, unsigned base) {
        if constexpr (TURNS) __builtin_amdgcn_s_setprio(2);
#pragma unroll
        for (int i = 0; i < KT; ++i)
#pragma unroll
            for (int e = 0; e < 16; ++e) s[i][e] = 0.0f;
#pragma unroll
        for (int ks = 0; ks < KS; ++ks) {
            const unsigned at = k_at(base, ks);
#pragma unroll
            for (int i = 0; i < KT; ++i) {
                i32x4 k;
                if constexpr (RUNS) {
                    // (behind a row is the next one, whatever it holds)
                    const int left = p.D - 8 * half - 16 * ks;
                    const i32x2 a = at_lds<i32x2>(at + 32 * i * row_k), b = at_lds<i32x2>(at + 32 * i * row_k + 8);
                    if (DP == 64 || 2 * ks >= KS) k = i32x4{left > 0 ? a.x : 0, left > 0 ? a.y : 0, left > 4 ? b.x : 0, left > 4 ? b.y : 0};
                    else k = i32x4{a.x, a.y, b.x, b.y};
                } else k = at_lds<i32x4>(at + 32 * i * row_k);
                s[i] = mfma32(__builtin_bit_cast(x8, k), q[ks], s[i]);
            }
        }
        in_turn<KS * KT, 1, 1, 6, 0, 0>();
        if constexpr (TURNS) __builtin_amdgcn_s_setprio(0);
    };
    auto hide = [&](int k0) {
        if (k0 + WK > all_to || k0 < all_from) {
            int to = sees_to - k0 - 4 * half, from = sees_from - k0 - 4 * half;
            stay(to);                          // (or the comparisons are made in every step, ahead of the branch)
            stay(from);
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
        return fmaxf(top, __shfl_xor(top, 32)) * scale_log2;
    };
    // Every result is a number, and none above 2^64, so that those of all waves and parts together are numbers too.
    auto finite = [&]() {
        float squares[4] = {};                 // (or infinite, or NaN)
#pragma unroll
        for (int dt = 0; dt < DT; ++dt)
#pragma unroll
            for (int e = 0; e < 16; ++e) {
                if (RUNS && 32 * dt + 8 * (e >> 2) + 4 * half >= p.D) continue;
                squares[e & 3] = __builtin_fmaf(o[dt][e], o[dt][e], squares[e & 3]);
            }
        return squares[0] + squares[1] + squares[2] + squares[3] < __builtin_inff();
    };
    const float none = -__builtin_inff();
    for (int turn = 0;; ++turn) {
        l = 0.0f;
        if (turn == 0) m = blind ? 0.0f : none;
#pragma unroll
        for (int dt = 0; dt < DT; ++dt)
#pragma unroll
            for (int e = 0; e < 16; ++e) o[dt][e] = 0.0f;
        auto weigh_up = [&](int kt, unsigned v_base) {
            hide(kt + WK * kw);
            if (turn == 0 && __any(m == none)) {
                // fp16: the largest of a few keys says little of later ones, which may be up to 2^12 above it; of 16 and more 2^9
                const int k0 = kt + WK * kw, seen = min(sees_to, k0 + WK) - max(sees_from, k0);
                const float top = largest() - (seen < 16 ? FIRST_LIFT : LIFT);
                m = m == none ? top : m;
            }
            const float shift = m == none ? 0.0f : m;
            float sum = 0.0f;                  // of this step: l has an addition a step, not one a key, as it may be large beside a key
            // Sixteen keys at a time; the weights and V of the next are made and read while the matrix cores are on these.
            x8 vf[DT], pf[TERMS], next[TERMS];
            unsigned v_from[DT];
#pragma unroll
            for (int dt = 0; dt < DT; ++dt) v_from[dt] = v_at(v_base, dt);
            auto weigh = [&](int st, x8 (&w)[TERMS]) {
#pragma unroll
                for (int i = 0; i < 8; ++i) {
                    float left = exp2_fast(__builtin_fmaf(s[st >> 1][8 * (st & 1) + i], scale_log2, -shift));
                    sum += left;
#pragma unroll
                    for (int k = 0; k < TERMS; ++k) {
                        w[k][i] = (T)left;
                        if (k + 1 < TERMS) left -= (float)(T)left;
                    }
                }
            };
            auto read_v = [&](int st, int dt) {
                const s16x4 v0 = lds_read_transposed(v_from[dt] + 16 * st * row_v), v1 = lds_read_transposed(v_from[dt] + (16 * st + 8) * row_v);
                return __builtin_bit_cast(x8, __builtin_shufflevector(v0, v1, 0, 1, 2, 3, 4, 5, 6, 7));
            };
#pragma unroll
            for (int dt = 0; dt < DT; ++dt) vf[dt] = read_v(0, dt);
            weigh(0, pf);
            __builtin_amdgcn_sched_barrier(0);
            if constexpr (TURNS) __builtin_amdgcn_s_setprio(1);
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
            if constexpr (TURNS) __builtin_amdgcn_s_setprio(0);
            l += sum;
            pinned(l);                         // (or the sums are made behind the loop, from registers that wait for that)
        };
        sweep(multiply, weigh_up);
        // (a lane's O is of the keys of both halves)
        const float both = l + __shfl_xor(l, 32);
        // (rows whose scores are no numbers are what they are)
        if ((both == both && !finite()) || (WIDE && both >= 0x1p40f)) again[turn < LAST ? 2 * turn : 1] = 1;   // the last time: something to settle
        __syncthreads();
        if (turn == LAST || !again[2 * turn]) break;
        if (turn == 0) {
            m = none;
            sweep(multiply, [&](int kt, unsigned) {
                hide(kt + WK * kw);
                m = fmaxf(m, largest() - Number<T>::kLift);
            });
            __syncthreads();
        } else m += (float)(32 - __builtin_clz(t.seq.len));
    }
    l += __shfl_xor(l, 32);
    if (t.seq.bad) l = __builtin_nanf("");
    if (l == 0.0f) m = none;                   // (nothing is of any weight: m may be anything)

    // The results leave through LDS (nobody reads the buffers any more), so that a store has whole lines.
    const ChunkParams& z = parameters();
    float* const parts = FEW ? z.few_o : z.many_o;
    // Row r of the tile: what its result is multiplied with (to `slot`), 1 / l, or 1 where it is a part; its sums, by one of those who place it.
    auto place = [&](int r, int slot, float top, float total, bool sums) {
        row_factor[slot] = total != total ? total : (total == 0.0f ? 0.0f : (t.direct ? 1.0f / total : 1.0f));
        if (!sums || t.row0 + r >= t.row_end) return;
        if (!t.direct) *(f32x2*)((FEW ? z.few_ml : z.many_ml) + row_sums * 2) = f32x2{top, total};
        else if (z.lse) z.lse[row_sums] = lse_of(top, total);
    };
    // COUNT rows at once: r0, r0 + step, ..., each the lane's four features from d on, read at from + i * pitch
    auto put = [&](auto count, int r0, int step, int slot0, int d, auto read) {
        constexpr int COUNT = decltype(count)::value;
        f32x4 x[COUNT];
        float factor[COUNT];
        int64_t to[COUNT];
#pragma unroll
        for (int i = 0; i < COUNT; ++i) {
            x[i] = read(i);
            factor[i] = row_factor[slot0 + i * step];
            to[i] = row_to[slot0 + i * step] + d;
        }
#pragma unroll
        for (int i = 0; i < COUNT; ++i) {
            const f32x4 y = factor[i] == 0.0f ? f32x4{0, 0, 0, 0} : x[i] * factor[i];
            if (t.row0 + r0 + i * step < t.row_end && d < z.D) {
                if (t.direct) store_four<O>(z.out, to[i], y);
                else *(f32x4*)(parts + to[i]) = y;
            }
        }
    };
    constexpr int LP = leave_pitch(DP, KW);
    float* const own = (float*)lds + wave * 32 * LP;
    if constexpr (FEW) {
        constexpr int HALF = DP / 2, LANES = HALF / 4, ROWS = 64 * NW / LANES < 32 ? 64 * NW / LANES : 32;
        if (half == 0) {
            row_m[32 * wave + l32] = m;
            row_l[32 * wave + l32] = l;
        }
        __syncthreads();
        float top = none;
#pragma unroll
        for (int w = 0; w < KW; ++w) top = fmaxf(top, row_m[32 * w + l32]);
        const float factor = m == none ? 0.0f : exp2_fast(m - top);
        const bool counts = l != 0.0f;         // (a part without weight says nothing, whatever 0 times its values is)
        if (wave == 0 && half == 0) {
            float total = 0.0f;
#pragma unroll
            for (int w = 0; w < KW; ++w) {
                const float part = row_l[32 * w + l32], its = row_m[32 * w + l32];
                total += part == 0.0f ? 0.0f : part * (its == none ? 0.0f : exp2_fast(its - top));
            }
            place(l32, l32, total == 0.0f ? none : top, total, true);
        }
#pragma unroll
        for (int d0 = 0; d0 < DP; d0 += HALF) {
#pragma unroll
            for (int i = 0; i < HALF / 8; ++i) {
                const int dt = (d0 + 8 * i) / 32, e = 4 * (i & 3);
                const f32x4 x = f32x4{o[dt][e], o[dt][e + 1], o[dt][e + 2], o[dt][e + 3]} * factor;
                *(f32x4*)(own + l32 * LP + 8 * i + 4 * half) = counts ? x : f32x4{0, 0, 0, 0};
            }
            __syncthreads();
            const int r0 = tid / LANES, d = 4 * (tid % LANES);
            if (r0 < ROWS)
                put(Count<32 / ROWS>{}, r0, ROWS, r0, d0 + d, [&](int i) {
                    f32x4 x = f32x4{0, 0, 0, 0};
#pragma unroll
                    for (int w = 0; w < KW; ++w) x += *(const f32x4*)((const float*)lds + (32 * w + r0 + i * ROWS) * LP + d);
                    return x;
                });
            if (d0 == 0) __syncthreads();
        }
    } else {
        constexpr int TF = turn_features(DP), LANES = TF / 4, ROWS = 64 / LANES;       // features that leave together, lanes of a row, rows of a store
        float* turned = own;
        int d_first = 0;
        if constexpr (KW > 1) {                // the two waves of a row have half of the features each from here on: each hands the other's over
            const int other = wave ^ RW;
            auto four = [&](int i) { return f32x4{o[i / 4][4 * (i & 3)], o[i / 4][4 * (i & 3) + 1], o[i / 4][4 * (i & 3) + 2], o[i / 4][4 * (i & 3) + 3]}; };
#pragma unroll
            for (int i = 0; i < DP / 16; ++i) *(f32x4*)(own + l32 * LP + 8 * i + 4 * half) = kw == 0 ? four(i + DP / 16) : four(i);
            if (half == 0) {
                row_m[32 * wave + l32] = m;
                row_l[32 * wave + l32] = l;
            }
            __syncthreads();
            const float om = row_m[32 * other + l32], ol = row_l[32 * other + l32], top = fmaxf(m, om);
            const float f = m == none ? 0.0f : exp2_fast(m - top), of = om == none ? 0.0f : exp2_fast(om - top);
            const bool counts = l != 0.0f, other_counts = ol != 0.0f;
            turned = (float*)lds + other * 32 * LP;    // (which nobody else reads)
            f32x4 y[DP / 16];
#pragma unroll
            for (int i = 0; i < DP / 16; ++i) y[i] = *(const f32x4*)(turned + l32 * LP + 8 * i + 4 * half);
#pragma unroll
            for (int i = 0; i < DP / 16; ++i) {
                const f32x4 x = kw == 0 ? four(i) : four(i + DP / 16);
#pragma unroll
                for (int e = 0; e < 4; ++e) o[i / 4][4 * (i & 3) + e] = (counts ? x[e] * f : 0.0f) + (other_counts ? y[i][e] * of : 0.0f);
            }
            l = (counts ? l * f : 0.0f) + (other_counts ? ol * of : 0.0f);
            m = l == 0.0f ? none : top;
            d_first = kw * (DP / 2);
        }
        if (half == 0) place(32 * rw + l32, 32 * wave + l32, m, l, kw == 0);
        __builtin_amdgcn_wave_barrier();
#pragma unroll
        for (int d0 = 0; d0 < (KW > 1 ? DP / 2 : DP); d0 += TF) {
#pragma unroll
            for (int i = 0; i < TF / 8; ++i) {
                const int dt = d0 / 32 + i / 4, e = 4 * (i & 3);
                *(f32x4*)(turned + l32 * LP + 8 * i + 4 * half) = f32x4{o[dt][e], o[dt][e + 1], o[dt][e + 2], o[dt][e + 3]};
            }
            __builtin_amdgcn_wave_barrier();
            const int r = lane / LANES, d = 4 * (lane % LANES);
            put(Count<32 / ROWS>{}, 32 * rw + r, ROWS, 32 * wave + r, d_first + d0 + d, [&](int i) { return *(const f32x4*)(turned + (r + i * ROWS) * LP + d); });
            __builtin_amdgcn_wave_barrier();
        }
    }
    wg_barrier_lds();                          // (no wait for the stores)
    if (__builtin_expect(again[1] != 0, 0)) {
        // every wave settles its own rows, or its share of them
        __threadfence();
        __syncthreads();
        unsigned rows = 0;
        for (int r = kw; r < 32; r += KW) {
            const float factor = row_factor[FEW ? r : 32 * wave + r];
            // (a row that nothing is of any weight for is 0; its part says what it has seen, as others may weigh something)
            if (wave_row0 + r < t.row_end && factor == factor && !(t.direct && factor == 0.0f)) rows |= 1u << r;
        }
        settle_chunk<T, O, DP, FEW>(z, t, wave_row0, rows);
    }
}

// Workgroup `i` of those for few rows, sequence by sequence, key head by key head, part by part.
template <class T, class O, int DP, int LOAD>
__device__ __forceinline__ void few_rows(const ChunkParams& p, int i, unsigned char* lds) {
    Tile t;
    t.split = i % p.few_splits;
    t.h = i / p.few_splits % p.Hk;
    t.b = i / p.few_splits / p.Hk;
    if (t.b >= p.B) return;
    t.seq = chunk_of(p, t.b);
    t.row0 = t.j0 = t.g0 = 0;
    t.row_end = t.seq.queries * p.G;
    if (t.row_end == 0) return;
    if (t.row_end > p.few_rows) {
        // worked on as many rows; where nobody does, more queries than the caller said that there are: NaN
        if (p.many_per_xcd == 0 && t.split == 0)
            for (int64_t x = threadIdx.x; x < (int64_t)t.row_end * (p.D / 4); x += 64 * few_waves(DP)) {
                const int row = (int)(x / (p.D / 4)), j = row / p.G, d = 4 * (int)(x % (p.D / 4));
                const float nan = __builtin_nanf("");
                store_four<O>(p.out, (t.seq.start + j) * p.out_token + (int64_t)(t.h * p.G + row - j * p.G) * p.out_head + d, f32x4{nan, nan, nan, nan});
                if (p.lse && d == 0) p.lse[(int64_t)(t.seq.start + j) * (p.Hk * p.G) + t.h * p.G + row - j * p.G] = nan;
            }
        return;
    }
    const Range r = range_of(p, t.seq, 0, t.seq.queries - 1, p.few_chunk);
    if (t.split >= r.parts) return;
    t.direct = r.parts == 1;
    t.first = r.first + t.split * p.few_chunk;
    t.end = t.first + min(r.end - t.first, p.few_chunk);
    attend_chunk<T, O, DP, 1, few_waves(DP), LOAD>(p, t, lds);
}

// Workgroup `i` of those for many rows: tile `at` of the sequences' tiles, one sequence behind the other, of each the one that sees most first; their parts and key heads
// side by side.
template <class T, class O, int DP, int KW, int LOAD>
__device__ __forceinline__ void many_rows(const ChunkParams& p, int i, unsigned char* lds) {
    constexpr int RW = 4, ROWS = kManyRows;
    static_assert(ROWS == 32 * RW, "32 rows a wave");
    const int lane = (int)threadIdx.x & 63;
    Tile t;
    t.h = i % p.Hk;
    t.split = i / p.Hk % p.many_splits;
    int at = i / p.Hk / p.many_splits;
    if (at >= p.many_tiles) return;
    t.b = -1;
    if (p.B == 1) {
        t.seq = chunk_of(p, 0);
        const int rows = t.seq.queries * p.G, tiles = rows > p.few_rows ? (rows + ROWS - 1) / ROWS : 0;
        if (at < tiles) {
            t.b = 0;
            at = tiles - 1 - at;
        }
    } else for (int b0 = 0; b0 < p.B; b0 += 64) {
        const Chunk c = b0 + lane < p.B ? chunk_of(p, b0 + lane) : Chunk{};
        const int rows = c.queries * p.G, tiles = rows > p.few_rows ? (rows + ROWS - 1) / ROWS : 0;
        int sum = tiles;
#pragma unroll
        for (int m = 1; m < 64; m *= 2) {
            const int other = __shfl_up(sum, m);
            if (lane >= m) sum += other;
        }
        const uint64_t past = __ballot(sum > at);
        if (past) {
            const int f = __builtin_ctzll(past), t_end = __shfl(sum, f);
            t.b = b0 + f;
            at = t_end - 1 - at;
            auto its_own = [&](int x) { return __builtin_amdgcn_readlane(x, __builtin_amdgcn_readfirstlane(f)); };
            t.seq = Chunk{its_own(c.start), its_own(c.queries), its_own(c.len), its_own(c.base), its_own(c.bad)};
            break;
        }
        at -= __shfl(sum, 63);
    }
    t.b = __builtin_amdgcn_readfirstlane(t.b);
    at = __builtin_amdgcn_readfirstlane(at);
    if (t.b < 0) return;
    t.row0 = at * ROWS;
    t.row_end = min(t.row0 + ROWS, t.seq.queries * p.G);
    t.j0 = t.row0 / p.G;
    t.g0 = t.row0 - t.j0 * p.G;
    const Range r = range_of(p, t.seq, t.j0, __builtin_amdgcn_readfirstlane(query_of(p, t, t.row_end - 1 - t.row0)), p.many_chunk);
    if (t.split >= r.parts) return;
    t.direct = r.parts == 1;
    t.first = r.first + t.split * p.many_chunk;
    t.end = t.first + min(r.end - t.first, p.many_chunk);
    attend_chunk<T, O, DP, RW, KW, LOAD>(p, t, lds);
}

// Workgroups go to the 8 XCDs in turn, so that an XCD has every eighth of them: those of one key head, or of few, which read the same keys, where 8 and the number of key
// heads have a divisor, and tiles that see much and little alike.  Where its 32 units have room for two workgroups each, the second ones go the other way, so that who has
// the most has the least beside it.
template <class T, class O, int DP, int KW, int LOAD>
__global__ void __launch_bounds__(256 * KW, DP > 128 ? 1 : 2) many_rows_kernel(const ChunkParams p) {
    extern __shared__ __align__(16) unsigned char lds[];
    const int both = min(p.many_per_xcd, 64);
    int place = (int)blockIdx.x >> 3;
    if (KW == 1 && DP <= 128 && place >= 32 && place < both) place = both - 1 - (place - 32);
    many_rows<T, O, DP, KW, LOAD>(p, 8 * place + ((int)blockIdx.x & 7), lds);
}
template <class T, class O, int DP, int LOAD>
__global__ void __launch_bounds__(64 * few_waves(DP), DP > 128 ? 1 : 2) few_rows_kernel(const ChunkParams p) {
    extern __shared__ __align__(16) unsigned char lds[];
    few_rows<T, O, DP, LOAD>(p, ((int)blockIdx.x & 7) * p.few_per_xcd + ((int)blockIdx.x >> 3), lds);
}

// The parts of every row joined, where there are several: DP / 4 threads have four features each.
template <class O, int DP>
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
    const int row0 = few ? 0 : in_head / kManyRows * kManyRows, row_end = few ? c.queries * p.G : min(row0 + kManyRows, c.queries * p.G);
    const Range r = range_of(p, c, row0 / p.G, (row_end - 1) / p.G, few ? p.few_chunk : p.many_chunk);
    if (r.parts == 1) return;
    float top = -__builtin_inff(), total = 0.0f;
    f32x4 x = f32x4{0, 0, 0, 0}, odd = f32x4{0, 0, 0, 0};      // odd: infinities and NaN, as they are whatever their parts weigh
    for (int s0 = 0; s0 < r.parts; s0 += 4) {
        float m[4], l[4];
        f32x4 o[4];
#pragma unroll
        for (int i = 0; i < 4; ++i) {
            const int s = min(s0 + i, r.parts - 1);
            const int64_t at = few ? part_at<true>(p, c, b, h, in_head, j, head, s) : part_at<false>(p, c, b, h, in_head, j, head, s);
            const f32x2 ml = *(const f32x2*)((few ? p.few_ml : p.many_ml) + at * 2);
            m[i] = ml.x;
            l[i] = ml.y;
            o[i] = *(const f32x4*)((few ? p.few_o : p.many_o) + at * p.D + d);
        }
        // (behind all of the loads, which are on their way together)
#pragma unroll
        for (int i = 0; i < 4; ++i) {
            const bool none = s0 + i >= r.parts, nothing = none || l[i] == 0.0f;
            m[i] = nothing ? -__builtin_inff() : m[i];
            l[i] = nothing ? 0.0f : l[i];
#pragma unroll
            for (int e = 0; e < 4; ++e) {
                const bool no_number = is_odd(o[i][e]);
                odd[e] += no_number && !none ? o[i][e] : 0.0f;
                o[i][e] = no_number || none ? 0.0f : o[i][e];
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
    x = total == 0.0f ? f32x4{0, 0, 0, 0} : x * (1.0f / total) + odd;
    store_four<O>(p.out, token * p.out_token + head * p.out_head + d, x);
    if (p.lse && d == 0) p.lse[row] = lse_of(top, total);
}

}  // namespace
