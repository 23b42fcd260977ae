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
// A thread keeps its own m, l and d over its logits; they meet at the end of the part, and those of a row's parts in join_kernel:
//   m = max m_i,  l = sum exp(m_i - m) l_i,  d = sum exp(m_i - m) (d_i + (m - m_i) l_i).
// The largest: a key of 64 bits, the logit's bits in the order of its value ahead of ~index, orders tokens as they are to come out, ties by the lowest
// index, and no two are alike.  Of a chunk of 256 threads' logits: the k-th largest of the threads' own largest ones is a bound that k of the chunk's logits
// reach, and few more do; later chunks have the k-th largest so far.  What passes the bound goes to a list in LDS, in any order, and every key's rank is
// the number of larger ones.
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
    int count;
    uint64_t found;
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

// A chunk's keys into best[], which has `had` keys (0 where empty).  key(e): the thread's e-th key, 0 for none.  Returns the new count.
template <int E, class Key>
__device__ __forceinline__ int take_keys(TopList& s, Key key, int had, int top) {
    const int tid = (int)threadIdx.x;
    uint64_t bound;                            // keys from here on are wanted
    if (had < top) {
        uint64_t most = 0;
#pragma unroll
        for (int e = 0; e < E; ++e) most = max(most, key(e));
        s.maxima[tid] = most;
        if (tid == 0) s.found = 0;
        __syncthreads();
        int rank = 0;
        for (int j = 0; j < kLogitThreads; ++j) rank += s.maxima[j] > most;
        // (maxima of 0 are alike: none of them has a rank below top where top other ones are there)
        if (rank == top - 1 && most != 0) s.found = most;
        __syncthreads();
        bound = max(s.found, (uint64_t)1);
    } else bound = s.best[top - 1] + 1;
    unsigned wanted = 0;
#pragma unroll
    for (int e = 0; e < E; ++e) wanted |= key(e) >= bound ? 1u << e : 0u;
    if (!__syncthreads_or(wanted != 0)) return had;
    if (tid == 0) s.count = had;
    if (tid < had) s.keys[tid] = s.best[tid];
    __syncthreads();
    if (wanted) {
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

// The sums of all threads, in every thread (an order that does not change).
__device__ __forceinline__ LogSum workgroup_log_sum(LogSum s, float (&of)[kLogitThreads / 64][3], float c) {
#pragma unroll
    for (int m = 32; m; m >>= 1) {
        const float om = __shfl_xor(s.m, m), ol = __shfl_xor(s.l, m), od = __shfl_xor(s.d, m);
        // (either lane of a pair has to get the same bits)
        LogSum a = s, b;
        b.m = om, b.l = ol, b.d = od;
        if ((int)threadIdx.x & m) {
            const LogSum t = a;
            a = b;
            b = t;
        }
        a.join(b.m, b.l, b.d, c);
        s = a;
    }
    if (((int)threadIdx.x & 63) == 0) {
        float* const at = of[threadIdx.x >> 6];
        at[0] = s.m, at[1] = s.l, at[2] = s.d;
    }
    __syncthreads();
    s.m = of[0][0], s.l = of[0][1], s.d = of[0][2];
    for (int w = 1; w < kLogitThreads / 64; ++w) s.join(of[w][0], of[w][1], of[w][2], c);
    return s;
}

// What a row comes out as, from its sums and its largest keys (count of them; the row's other logits are -inf or no numbers).
template <class T>
__device__ __forceinline__ void store_row(const LogitsParams& p, int64_t row, const LogSum& sum, const TopList& s, int count) {
    const int tid = (int)threadIdx.x;
    const T* const x = (const T*)p.logits + row * p.row_stride;
    const float nan = __builtin_nanf(""), ln2 = 0.69314718055994531f;
    const bool none = sum.l == 0.0f;                                   // no token is allowed
    const float log_l = logf(sum.l);
    auto logprob = [&](float of) { return none ? (of != of ? nan : -__builtin_inff()) : (of - sum.m) * p.inverse_temperature - log_l; };
    if (tid == 0) {
        if (p.logprob) {
            const int64_t token = p.tokens[row];
            p.logprob[row] = token >= 0 && token < p.V ? logprob((float)x[token]) : nan;
        }
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
    for (int at = first; at < end; at += CHUNK) {
        RawVec<T, VEC> raw[E / VEC];
        auto index = [&](int e) { return at + ((e / VEC) * kLogitThreads + tid) * VEC + e % VEC; };
#pragma unroll
        for (int i = 0; i < E / VEC; ++i) raw[i].load(x, min(index(i * VEC), p.V - VEC));        // (VEC divides V)
        float v[E];
        float top = -__builtin_inff();
#pragma unroll
        for (int i = 0; i < E / VEC; ++i) {
            float f[VEC];
            raw[i].floats(f);
            const bool in = index(i * VEC) < end;
#pragma unroll
            for (int e = 0; e < VEC; ++e) {
                v[i * VEC + e] = in ? f[e] : -__builtin_inff();
                top = fmaxf(top, v[i * VEC + e]);
            }
        }
        sum.raise(fmaxf(sum.m, top), p.c);
        const float m = sum.m == -__builtin_inff() ? 0.0f : sum.m;     // (-inf where all are, or are no numbers, which make l none)
#pragma unroll
        for (int e = 0; e < E; ++e) {
            const float u = (v[e] - m) * p.c, w = __builtin_amdgcn_exp2f(u);
            sum.l += w;
            sum.d = __builtin_fmaf(w, w > 0.0f ? -u : 0.0f, sum.d);
        }
        if (p.top > 0)
            count = take_keys<E>(s, [&](int e) { return v[e] > -__builtin_inff() ? key_of(v[e], index(e)) : 0; }, count, p.top);
    }
    sum = workgroup_log_sum(sum, sums, p.c);
    if (p.parts == 1) {
        store_row<T>(p, row, sum, s, count);
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
    LogSum sum;
    if (tid < p.parts) {
        const float4 part = *(const float4*)(p.part_sums + (in_call * p.parts + tid) * 4);
        sum.m = part.x, sum.l = part.y, sum.d = part.z;
    }
    sum = workgroup_log_sum(sum, sums, p.c);
    int count = 0;
    if (p.top > 0) {
        const int all = p.parts * p.top;
        uint64_t keys[kJoinKeys];
#pragma unroll
        for (int e = 0; e < kJoinKeys; ++e) {
            const int at = tid + e * kLogitThreads;
            keys[e] = at < all ? p.part_keys[in_call * all + at] : 0;
        }
        count = take_keys<kJoinKeys>(s, [&](int e) { return keys[e]; }, 0, p.top);
    }
    store_row<T>(p, row, sum, s, count);
}

}  // namespace
