// Rows of tokens between the products of a layer: activation, gate, norm, the sum with the residual, and the next norm, in one pass.
// Part of the translation unit layer.hip (included there, in this order).
#pragma once

#include "vectors.hip.h"

namespace {

// ---------------------------------------------------------------------------------------------
// A row is one token of K features.  Behind a block (RESIDUAL):
//   t = y / sqrt(mean(y^2) + eps) * weight    (t = y without a weight)
//   h = residual + scale * act(gate) * t      (scale * t without a gate)
//   x = h / sqrt(mean(h^2) + eps) * next_weight
// inside one:
//   t = act(gate) * y                         (act(y) without a gate),  h = t / sqrt(mean(t^2) + eps) * weight   (h = t without a weight)
// all in fp32, rounded once where it is stored; x is of the h that was not rounded.
// A workgroup has a row, and a thread keeps its NV vectors of VEC features of everything in registers from the loads, which are on their way together, to
// the stores: the only exchanges are the two sums of squares.
// Bound by its bytes: 4096 rows of 4096 features in 16 bits, both norms and a gate, 134 MB in 25 us where some of them are in the cache, in calls one behind the other 30 us or
// 4.5 TB/s (a large copy: 5.3); 1024 rows of 6912 in fp32 with their gate 85 MB in 15 us (the cache holds some of them).  One row: 2.2 us, a launch and two trips to memory.
// Features that a thread has: launch_rows.  32 are more than its registers hold and go through scratch memory in part; only rows of more than 16384 features have them.
// ---------------------------------------------------------------------------------------------
struct RowsParams {
    const void *y, *gate, *residual;           // gate: null for none; residual: of RESIDUAL
    const float *weight, *next_weight;         // null: no such norm
    void *h, *x;                               // x: null where next_weight is
    int64_t y_row, gate_row, residual_row, h_row, x_row;       // strides in elements; gate_row 0: one gate for all rows
    int64_t first_row;                         // of this launch
    int K, activation, gate_f32, h_type, x_type;
    float eps, scale;
};

template <int VEC>
__device__ __forceinline__ void store_as(void* base, int type, int64_t at, const float (&v)[VEC]) {
    if (type == VLUT_TYPE_F32) store_floats<float, VEC>((float*)base + at, v);
    else if (type == VLUT_TYPE_BF16) store_floats<__bf16, VEC>((__bf16*)base + at, v);
    else store_floats<_Float16, VEC>((_Float16*)base + at, v);
}

__device__ __forceinline__ float sigmoid_of(float x) { return 1.0f / (1.0f + expf(-x)); }
template <int N>
__device__ __forceinline__ void activate(float (&v)[N], int activation) {
#pragma unroll
    for (int i = 0; i < N; ++i) {
        const float x = v[i];
        if (activation == VLUT_ACTIVATION_SIGMOID) v[i] = sigmoid_of(x);
        else if (activation == VLUT_ACTIVATION_SILU) v[i] = x * sigmoid_of(x);
        else if (activation == VLUT_ACTIVATION_RELU2) v[i] = x > 0.0f ? x * x : x != x ? x : 0.0f;
        else if (activation == VLUT_ACTIVATION_GELU) v[i] = 0.5f * x * erfcf(x * -0.70710678118654752f);      // (0.5 (1 + erf) would cancel for x < 0)
    }
}

// The sum over the workgroup, in every thread and in an order that does not change.  A barrier is between two uses of `parts`: the two sums have one each.
__device__ __forceinline__ float workgroup_sum(float v, float* parts) {
#pragma unroll
    for (int m = 32; m; m >>= 1) v += __shfl_xor(v, m);
    const int waves = ((int)blockDim.x + 63) >> 6;
    if (waves == 1) return v;
    if (((int)threadIdx.x & 63) == 0) parts[threadIdx.x >> 6] = v;
    __syncthreads();
    v = 0.0f;
    for (int w = 0; w < waves; ++w) v += parts[w];
    return v;
}

template <class TY, class TR, int VEC, int NV, bool RESIDUAL>
__global__ void __launch_bounds__(1024) rows_kernel(const RowsParams p) {
    __shared__ float parts[2][16];
    const int64_t row = p.first_row + blockIdx.x;
    const int vectors = p.K / VEC, threads = (int)blockDim.x, tid = (int)threadIdx.x;
    RawVec<TY, VEC> y[NV];
    RawVec<TR, VEC> residual[NV];
    int at[NV];
#pragma unroll
    for (int i = 0; i < NV; ++i) at[i] = VEC * min(tid + i * threads, vectors - 1);      // (past the row: its last vector, not counted and not stored)
#pragma unroll
    for (int i = 0; i < NV; ++i) y[i].load(p.y, row * p.y_row + at[i]);
    if constexpr (RESIDUAL) {
#pragma unroll
        for (int i = 0; i < NV; ++i) residual[i].load(p.residual, row * p.residual_row + at[i]);
    }
    float t[NV][VEC], g[NV][VEC];
    if (p.gate) {
        if (p.gate_f32) {
#pragma unroll
            for (int i = 0; i < NV; ++i) load_floats<float, VEC>(g[i], (const float*)p.gate + row * p.gate_row + at[i]);
        } else {
#pragma unroll
            for (int i = 0; i < NV; ++i) load_floats<TY, VEC>(g[i], (const TY*)p.gate + row * p.gate_row + at[i]);
        }
    } else {
#pragma unroll
        for (int i = 0; i < NV; ++i)
#pragma unroll
            for (int e = 0; e < VEC; ++e) g[i][e] = 1.0f;
    }
#pragma unroll
    for (int i = 0; i < NV; ++i) y[i].floats(t[i]);
    if (p.activation != VLUT_ACTIVATION_NONE) {
#pragma unroll
        for (int i = 0; i < NV; ++i) {
            if (!RESIDUAL && !p.gate) activate(t[i], p.activation);
            else activate(g[i], p.activation);
        }
    }
    if constexpr (!RESIDUAL) {
#pragma unroll
        for (int i = 0; i < NV; ++i)
#pragma unroll
            for (int e = 0; e < VEC; ++e) t[i][e] *= g[i][e];
    }
    auto norm = [&](const float* weight, float* of) {
        float squares = 0.0f;
#pragma unroll
        for (int i = 0; i < NV; ++i)
            if (tid + i * threads < vectors) {
#pragma unroll
                for (int e = 0; e < VEC; ++e) squares += t[i][e] * t[i][e];
            }
        const float inverse = 1.0f / sqrtf(workgroup_sum(squares, of) / (float)p.K + p.eps);
#pragma unroll
        for (int i = 0; i < NV; ++i) {
            float w[VEC];
            load_floats<float, VEC>(w, weight + at[i]);
#pragma unroll
            for (int e = 0; e < VEC; ++e) t[i][e] = t[i][e] * inverse * w[e];
        }
    };
    if (p.weight) norm(p.weight, parts[0]);
    if constexpr (RESIDUAL) {
#pragma unroll
        for (int i = 0; i < NV; ++i) {
            float r[VEC];
            residual[i].floats(r);
#pragma unroll
            for (int e = 0; e < VEC; ++e) t[i][e] = r[e] + p.scale * t[i][e] * g[i][e];
        }
    }
#pragma unroll
    for (int i = 0; i < NV; ++i)
        if (tid + i * threads < vectors) {
            if constexpr (RESIDUAL) store_floats<TR, VEC>((TR*)p.h + row * p.h_row + at[i], t[i]);
            else store_as<VEC>(p.h, p.h_type, row * p.h_row + at[i], t[i]);
        }
    if constexpr (RESIDUAL) {
        if (!p.next_weight) return;
        norm(p.next_weight, parts[1]);
#pragma unroll
        for (int i = 0; i < NV; ++i)
            if (tid + i * threads < vectors) store_as<VEC>(p.x, p.x_type, row * p.x_row + at[i], t[i]);
    }
}

}  // namespace
