// Log probabilities, entropy and the most probable tokens of rows of logits, in one pass over them.
// Part of the translation unit layer.hip (included there, in this order).
#pragma once

#include "vectors.hip.h"

namespace {

// ---------------------------------------------------------------------------------------------
// For a row x of V logits, z = x / temperature:
//   m = max z,  l = sum exp(z - m),  d = sum exp(z - m) (m - z)
//   log p(i) = z_i - m - log l,   entropy = -sum p log p = log l + d / l
// (only terms of one sign are added in l and d).  Exponentials are powers of two of c times a difference of logits, c = log2(e) / temperature;
// m stays a logit, since times c a row of the type's lowest values would leave 32 bits.
// A logit of -inf is a token that is not allowed: it adds nothing.  A row of nothing else has log probabilities of -inf and an entropy of 0.
// A thread keeps its own m, l and d over its logits; they meet at the end of the part, and those of a row's parts in logits_join_kernel:
//   m = max m_i,  l = sum exp(m_i - m) l_i,  d = sum exp(m_i - m) (d_i + (m - m_i) l_i).
// The largest: a key of 64 bits, the logit's bits in the order of its value ahead of ~index, orders tokens as they are to come out, ties by the lowest
// index, and no two are alike.  Of a chunk of 256 threads' logits: the k-th largest of a wave's threads' own largest ones is a bound that k of the chunk's logits
// reach, and few more do (found bit by bit, by how many lanes reach it; its upper half will do); later chunks have the k-th largest so far, which only larger ones
// pass.  What passes goes to a list in LDS, in any order, and every key's rank is the number of larger ones.
// Bound by the bytes where rows are many: 2048 rows of 32000 in fp32, the largest one too, 262 MB in 57 us or 4.6 TB/s.  Few rows are in parts, to fill the card: one of
// 128000 with its 20 largest 7.3 us, and 6.0 to join 63 parts, both the way of one part through memory, sums and ranks.  (The bound by the k-th largest of a wave, found
// through LDS instead of bit by bit: 101 us and 20.)
// ---------------------------------------------------------------------------------------------
constexpr int kTopKeys = 1024;                 // of the list in LDS
constexpr int kLogitThreads = 256;

struct LogitsParams {
    const void* logits;
    const int64_t* tokens;                     // null: no token is asked for
    float *logprob, *entropy, *top_logprobs;   // null where not wanted
    int64_t* top_ids;
    int64_t row_stride, first_row;
    float* part_sums;                          // [rows][parts][4]: m, l, d
    uint64_t* part_keys;                       // [rows][parts][top]
    int V, top, parts, part;                   // logits of a part, a multiple of the chunk
    float c, inverse_temperature;              // c: log2(e) / temperature
};

__device__ __forceinline__ unsigned ordered_bits(float x) {
    const unsigned u = __builtin_bit_cast(unsigned, x + 0.0f);         // (-0 is 0)
    return u & 0x80000000u ? ~u : u | 0x80000000u;
}
__device__ __forceinline__ float from_ordered(unsigned u) { return __builtin_bit_cast(float, u & 0x80000000u ? u & 0x7fffffffu : ~u); }
__device__ __forceinline__ uint64_t key_of(float x, int index) { return (uint64_t)ordered_bits(x) << 32 | (unsigned)~index; }

// The larger one, NaN where x is.
__device__ __forceinline__ float at_least(float x, float least) {
#if defined(__HIP_DEVICE_COMPILE__)
    return __builtin_elementwise_maximum(x, least);
#else
    return x;
#endif
}

// m, l, d of logits that are added one after the other.
struct LogSum {                                // (m: a logit; d in powers of two)
    float m = -__builtin_inff(), l = 0.0f, d = 0.0f;
    // everything in terms of the maximum `now` >= m
    __device__ __forceinline__ void raise(float now, float c) {
        if (now == m || now == -__builtin_inff()) return;
        const float rise = (now - m) * c, f = __builtin_amdgcn_exp2f(-rise);           // (0 for the first)
        d = l == 0.0f || f == 0.0f ? 0.0f : f * (d + rise * l);
        l *= f;
        m = now;
    }
    __device__ __forceinline__ void join(float om, float ol, float od, float c) {
        LogSum o;
        o.m = om, o.l = ol, o.d = od;
        const float now = fmaxf(m, om);
        raise(now, c);
        o.raise(now, c);
        l += o.l;
        d += o.d;
    }
};

struct TopList {                               // of a workgroup, in LDS
    uint64_t keys[kTopKeys];
    uint64_t best[64];                         // the largest so far, in order
    uint64_t maxima[kLogitThreads];
    uint64_t found;
    int count;
    unsigned bounds[kLogitThreads / 64];
};

// keys[0 .. count) of the list, ranked: the `top` largest go to best[], behind them the rest is 0 (no key).  All threads call it, behind a barrier; it ends with one.
__device__ __forceinline__ void rank_keys(TopList& s, int count, int top) {
    const int tid = (int)threadIdx.x;
    uint64_t mine[kTopKeys / kLogitThreads];
    int rank[kTopKeys / kLogitThreads];
#pragma unroll
    for (int i = 0; i < kTopKeys / kLogitThreads; ++i) {
        const int at = tid + i * kLogitThreads;
        mine[i] = at < count ? s.keys[at] : 0;
        rank[i] = 0;
    }
    if (count <= kLogitThreads) {
#pragma unroll 8
        for (int j = 0; j < count; ++j) rank[0] += s.keys[j] > mine[0];
    } else
        for (int j = 0; j < count; ++j) {
            const uint64_t other = s.keys[j];
#pragma unroll
            for (int i = 0; i < kTopKeys / kLogitThreads; ++i) rank[i] += other > mine[i];
        }
#pragma unroll
    for (int i = 0; i < kTopKeys / kLogitThreads; ++i)
        if (tid + i * kLogitThreads < count && rank[i] < top) s.best[rank[i]] = mine[i];
    if (tid >= count && tid < top) s.best[tid] = 0;
    __syncthreads();
}

// The largest `top` of what the threads hold and of best[] (count `had`), where more pass the bound than the list holds: one after the other, each the largest
// below the one before.  Equal logits by the thousand, say.
template <int E, class Key>
__device__ __forceinline__ int extract_keys(TopList& s, Key key, int had, int top) {
    const int tid = (int)threadIdx.x;
    const uint64_t old = tid < had ? s.best[tid] : 0;
    uint64_t below = ~(uint64_t)0;
    int n = 0;
    for (; n < top; ++n) {
        uint64_t most = old < below ? old : 0;
#pragma unroll
        for (int e = 0; e < E; ++e) {
            const uint64_t k = key(e);
            if (k < below && k > most) most = k;
        }
        s.maxima[tid] = most;
        __syncthreads();
        if (tid < 64) {
            for (int i = 1; i < kLogitThreads / 64; ++i) most = max(most, s.maxima[tid + 64 * i]);
#pragma unroll
            for (int m = 32; m; m >>= 1) {
                const uint64_t other = (uint64_t)__shfl_xor((unsigned)(most >> 32), m) << 32 | (unsigned)__shfl_xor((unsigned)most, m);
                most = max(most, other);
            }
            if (tid == 0) s.found = most;
        }
        __syncthreads();
        below = s.found;
        if (below == 0) break;
        if (tid == 0) s.best[n] = below;
        __syncthreads();                       // (the next turn writes maxima and found)
    }
    __syncthreads();
    if (tid >= n && tid < top) s.best[tid] = 0;
    __syncthreads();
    return n;
}

// A bound that at least `top` of the wave's lanes' numbers reach, by their upper 16 bits; 0 where there are not as many that are not 0.
__device__ __forceinline__ unsigned bound_of_wave(unsigned mine, int top) {
    unsigned bound = 0;
#pragma unroll
    for (int bit = 31; bit >= 16; --bit) {
        const unsigned tried = bound | 1u << bit;
        if (__popcll(__ballot(mine >= tried)) >= top) bound = tried;
    }
    return bound;
}

// A chunk's keys into best[], which has `had` keys (0 where empty).  value(e): the bits of the thread's e-th one in order, 0 for none; key(e): its key; most: the largest
// value.  Returns the new count.
template <int E, class Value, class Key>
__device__ __forceinline__ int take_keys(TopList& s, unsigned most, Value value, Key key, int had, int top) {
    const int tid = (int)threadIdx.x;
    unsigned bound = 1;                        // values from here on are wanted
    if (had < top) {
        const unsigned of_wave = bound_of_wave(most, top);
        if ((tid & 63) == 0) s.bounds[tid >> 6] = of_wave;
        __syncthreads();
#pragma unroll
        for (int w = 0; w < kLogitThreads / 64; ++w) bound = max(bound, s.bounds[w]);
    } else bound = (unsigned)(s.best[top - 1] >> 32) + 1;      // (equal ones behind it come later)
    const bool any = most >= bound;
    if (!__syncthreads_or(any)) return had;
    if (tid == 0) s.count = had;
    if (tid < had) s.keys[tid] = s.best[tid];
    __syncthreads();
    if (any) {
        unsigned wanted = 0;
#pragma unroll
        for (int e = 0; e < E; ++e) wanted |= value(e) >= bound ? 1u << e : 0u;
        int at = atomicAdd(&s.count, __popc(wanted));
#pragma unroll
        for (int e = 0; e < E; ++e)
            if (wanted >> e & 1) {
                if (at < kTopKeys) s.keys[at] = key(e);
                ++at;
            }
    }
    __syncthreads();
    const int count = s.count;
    if (count > kTopKeys) return extract_keys<E>(s, key, had, top);
    rank_keys(s, count, top);
    return min(count, top);
}

// The sum over the 64 lanes of a wave, in every lane and in an order that does not change.
__device__ __forceinline__ float wave_sum_f32(float v) {
    auto add = [&](int other) { v += __builtin_bit_cast(float, other); };
    add(lane_xor16<1>(__builtin_bit_cast(int, v)));
    add(lane_xor16<2>(__builtin_bit_cast(int, v)));
    add(lane_xor7(__builtin_bit_cast(int, v)));                        // (quads are uniform by now)
    add(lane_xor16<8>(__builtin_bit_cast(int, v)));
    float r[4];
#pragma unroll
    for (int i = 0; i < 4; ++i) r[i] = __builtin_bit_cast(float, __builtin_amdgcn_readlane(__builtin_bit_cast(int, v), 16 * i));
    return (r[0] + r[1]) + (r[2] + r[3]);
}
// The sums of all threads, in every thread.
__device__ __forceinline__ LogSum workgroup_log_sum(LogSum s, float (&of)[kLogitThreads / 64][3], float c) {
    s.raise(wave_max_f32(s.m), c);             // (no m is NaN)
    s.l = wave_sum_f32(s.l);
    s.d = wave_sum_f32(s.d);
    if (((int)threadIdx.x & 63) == 0) {
        float* const at = of[threadIdx.x >> 6];
        at[0] = s.m, at[1] = s.l, at[2] = s.d;
    }
    __syncthreads();
    s.m = of[0][0], s.l = of[0][1], s.d = of[0][2];
#pragma unroll
    for (int w = 1; w < kLogitThreads / 64; ++w) s.join(of[w][0], of[w][1], of[w][2], c);
    return s;
}

// The logit of the token that is asked for, or NaN.  Asked for first of all: two trips to memory, one behind the other.
template <class T>
__device__ __forceinline__ float asked(const LogitsParams& p, int64_t row) {
    if (!p.logprob || threadIdx.x != 0) return 0.0f;
    const int64_t token = p.tokens[row];
    return token >= 0 && token < p.V ? (float)((const T*)p.logits)[row * p.row_stride + token] : __builtin_nanf("");
}

// What a row comes out as, from its sums and its largest keys (count of them; the row's other logits are -inf or no numbers).
template <class T>
__device__ __forceinline__ void store_row(const LogitsParams& p, int64_t row, const LogSum& sum, float its, const TopList& s, int count) {
    const int tid = (int)threadIdx.x;
    const T* const x = (const T*)p.logits + row * p.row_stride;
    const float nan = __builtin_nanf(""), ln2 = 0.69314718055994531f;
    const bool none = sum.l == 0.0f;                                   // no token is allowed
    const float log_l = logf(sum.l);
    auto logprob = [&](float of) { return none ? (of != of ? nan : -__builtin_inff()) : (of - sum.m) * p.inverse_temperature - log_l; };
    if (tid == 0) {
        if (p.logprob) p.logprob[row] = its != its ? nan : logprob(its);
        if (p.entropy) p.entropy[row] = none ? 0.0f : log_l + sum.d / sum.l * ln2;
    }
    if (tid >= 64 || p.top == 0) return;
    int64_t* const ids = p.top_ids + row * p.top;
    float* const probs = p.top_logprobs + row * p.top;
    if (tid < count) {
        const uint64_t key = s.best[tid];
        ids[tid] = (int64_t)~(unsigned)key;
        probs[tid] = logprob(from_ordered((unsigned)(key >> 32)));
    }
    if (count < p.top) {                       // then the first of the others: among the row's first `top`, as `count` are all that are not such
        const float first = (float)x[min(tid, p.V - 1)];
        const bool other = tid < p.top && !(first > -__builtin_inff());
        const uint64_t mask = __ballot(other);
        const int at = count + __popcll(mask & (((uint64_t)1 << tid) - 1));
        if (other && at < p.top) {
            ids[at] = tid;
            probs[at] = sum.l != sum.l ? nan : logprob(first);
        }
    }
}

// A part of a row, E logits of a thread at a time; the row where it has one part.
template <class T, int VEC, int E>
__global__ void __launch_bounds__(kLogitThreads) logits_kernel(const LogitsParams p) {
    __shared__ TopList s;
    __shared__ float sums[kLogitThreads / 64][3];
    constexpr int CHUNK = kLogitThreads * E;
    const int tid = (int)threadIdx.x;
    const int64_t in_call = blockIdx.x / (unsigned)p.parts, row = p.first_row + in_call;
    const int part = (int)(blockIdx.x % (unsigned)p.parts);
    const int first = part * p.part, end = min(p.V, first + p.part);
    const T* const x = (const T*)p.logits + row * p.row_stride;
    LogSum sum;
    int count = 0;
    const float its = p.parts == 1 ? asked<T>(p, row) : 0.0f;
    auto index = [&](int at, int e) { return at + ((e / VEC) * kLogitThreads + tid) * VEC + e % VEC; };
    RawVec<T, VEC> raw[E / VEC];
    auto load = [&](int at) {                  // (VEC divides V; past the part others' logits, or the last ones)
#pragma unroll
        for (int i = 0; i < E / VEC; ++i) raw[i].load(x, min(index(at, i * VEC), p.V - VEC));
    };
    load(first);
    for (int at = first; at < end; at += CHUNK) {
        float v[E];
        float top = -__builtin_inff();
#pragma unroll
        for (int i = 0; i < E / VEC; ++i) {
            float f[VEC];
            raw[i].floats(f);
            const bool in = index(at, i * VEC) < end;
#pragma unroll
            for (int e = 0; e < VEC; ++e) {
                v[i * VEC + e] = in ? f[e] : -__builtin_inff();
                top = fmaxf(top, v[i * VEC + e]);
            }
        }
        if (at + CHUNK < end) load(at + CHUNK);                        // (on their way meanwhile)
        sum.raise(fmaxf(sum.m, top), p.c);
        const float m = sum.m == -__builtin_inff() ? 0.0f : sum.m;     // (-inf where all are, or are no numbers)
        float l[2] = {}, d[2] = {};
#pragma unroll
        for (int e = 0; e < E; ++e) {
            const float u = at_least((v[e] - m) * p.c, -200.0f), w = __builtin_amdgcn_exp2f(u);        // (2^-200 is 0 in 32 bits, and so is 0 times 200)
            l[e & 1] += w;
            d[e & 1] = __builtin_fmaf(w, u, d[e & 1]);
        }
        sum.l += l[0] + l[1];
        sum.d -= d[0] + d[1];
        if (p.top > 0)
            count = take_keys<E>(s, top > -__builtin_inff() ? ordered_bits(top) : 0u, [&](int e) { return v[e] > -__builtin_inff() ? ordered_bits(v[e]) : 0u; },
                                 [&](int e) { return v[e] > -__builtin_inff() ? key_of(v[e], index(at, e)) : 0; }, count, p.top);
    }
    sum = workgroup_log_sum(sum, sums, p.c);
    if (p.parts == 1) {
        store_row<T>(p, row, sum, its, s, count);
        return;
    }
    const int64_t at = in_call * p.parts + part;
    if (tid == 0) *(float4*)(p.part_sums + at * 4) = make_float4(sum.m, sum.l, sum.d, 0.0f);
    if (tid < p.top) p.part_keys[at * p.top + tid] = tid < count ? s.best[tid] : 0;
}

// The parts of a row joined; at most E keys a thread.
constexpr int kMostParts = 64, kJoinKeys = kMostParts * 64 / kLogitThreads;
template <class T>
__global__ void __launch_bounds__(kLogitThreads) logits_join_kernel(const LogitsParams p) {
    __shared__ TopList s;
    __shared__ float sums[kLogitThreads / 64][3];
    const int tid = (int)threadIdx.x;
    const int64_t in_call = blockIdx.x, row = p.first_row + in_call;
    const float its = asked<T>(p, row);
    const int all = p.parts * p.top;
    uint64_t keys[kJoinKeys];
#pragma unroll
    for (int e = 0; e < kJoinKeys; ++e) {
        const int at = tid + e * kLogitThreads;
        keys[e] = at < all ? p.part_keys[in_call * all + at] : 0;
    }
    LogSum sum;
    if (tid < p.parts) {
        const float4 part = *(const float4*)(p.part_sums + (in_call * p.parts + tid) * 4);
        sum.m = part.x, sum.l = part.y, sum.d = part.z;
    }
    sum = workgroup_log_sum(sum, sums, p.c);
    int count = 0;
    if (p.top > 0) {
        unsigned most = 0;
#pragma unroll
        for (int e = 0; e < kJoinKeys; ++e) most = max(most, (unsigned)(keys[e] >> 32));
        count = take_keys<kJoinKeys>(s, most, [&](int e) { return (unsigned)(keys[e] >> 32); }, [&](int e) { return keys[e]; }, 0, p.top);
    }
    store_row<T>(p, row, sum, its, s, count);
}

}  // namespace
