// Around the products of a decoder layer, for MI355X (gfx950): the norms before and after a block with its gate and residual, and log probabilities.
// Their kernels, host side and part of the C ABI; a translation unit beside vlut.hip.
#include <hip/hip_runtime.h>

#include <algorithm>
#include <cmath>
#include <cstdint>

#include "vlut.h"

#include "common.hip.h"
#include "host_checks.h"
#include "launch.hip.h"
#include "rows_kernel.hip.h"
#include "logits_kernel.hip.h"

namespace {

constexpr int64_t kMostRows = 1 << 24;
constexpr int kUnits = 256;            // compute units that a launch is to fill

// ---------------------------------------------------------------------------------------------
// Rows
// ---------------------------------------------------------------------------------------------
int check_rows(const vlut_rows* r, Alignment& a) {
    if (!r->data) return VLUT_ERR_NULL;
    if (!type_ok(r->type)) return VLUT_ERR_SHAPE;
    a.pointer(r->data, type_bytes(r->type));
    a.stride(r->row_stride);
    return VLUT_OK;
}

template <class TY, class TR, int VEC, bool RESIDUAL>
int launch_rows_e(const RowsParams& p, int per, unsigned rows, int threads, hipStream_t stream) {
    if (per == 4) return launch(rows_kernel<TY, TR, VEC, 4 / VEC, RESIDUAL>, dim3(rows), threads, 0, stream, p);
    if (per == 8) return launch(rows_kernel<TY, TR, VEC, 8 / VEC, RESIDUAL>, dim3(rows), threads, 0, stream, p);
    if (per == 16) return launch(rows_kernel<TY, TR, VEC, 16 / VEC, RESIDUAL>, dim3(rows), threads, 0, stream, p);
    return launch(rows_kernel<TY, TR, VEC, 32 / VEC, RESIDUAL>, dim3(rows), threads, 0, stream, p);
}
template <class TY, class TR, bool RESIDUAL>
int launch_rows_v(const RowsParams& p, int vec, int per, unsigned rows, int threads, hipStream_t stream) {
    return vec == 4 ? launch_rows_e<TY, TR, 4, RESIDUAL>(p, per, rows, threads, stream) : launch_rows_e<TY, TR, 1, RESIDUAL>(p, per, rows, threads, stream);
}
template <class TY>
int launch_rows_r(const RowsParams& p, bool residual, int residual_type, int vec, int per, unsigned rows, int threads, hipStream_t stream) {
    if (!residual) return launch_rows_v<TY, float, false>(p, vec, per, rows, threads, stream);
    if (residual_type == VLUT_TYPE_F32) return launch_rows_v<TY, float, true>(p, vec, per, rows, threads, stream);
    if (residual_type == VLUT_TYPE_BF16) return launch_rows_v<TY, __bf16, true>(p, vec, per, rows, threads, stream);
    return launch_rows_v<TY, _Float16, true>(p, vec, per, rows, threads, stream);
}
int launch_rows(RowsParams& p, int type, bool residual, int residual_type, int vec, int64_t N, hipStream_t stream) {
    if (vec == 2) vec = 1;
    // Features of a thread: 16 where rows are many; the fewest, so that a row's chain of loads and sums is the shortest, where they are few.  us with 4 / 16: one row of 2560
    // 2.2 / 3.0, of 4096 3.5 / 4.2, 64 of those 4.4 / 5.1, 400 6.6 / 6.4, 512 7.0 / 6.8, 4096 33 / 25; 2048 of 2560 15 / 10 (8 lie between, or 1 us below).
    int per = N >= 2 * kUnits ? 16 : 4;
    while (per < 32 && (p.K + per - 1) / per > 1024) per *= 2;
    const int threads = std::max(1, (int)(((p.K + per - 1) / per + 63) / 64)) * 64;
    // A launch's threads are numbered in 32 bits: more are several launches.
    const int64_t most = ((int64_t)1 << 31) / threads;
    int rc = VLUT_OK;
    for (p.first_row = 0; rc == VLUT_OK && p.first_row < N; p.first_row += most) {
        const unsigned rows = (unsigned)std::min(N - p.first_row, most);
        if (type == VLUT_TYPE_F32) rc = launch_rows_r<float>(p, residual, residual_type, vec, per, rows, threads, stream);
        else if (type == VLUT_TYPE_BF16) rc = launch_rows_r<__bf16>(p, residual, residual_type, vec, per, rows, threads, stream);
        else rc = launch_rows_r<_Float16>(p, residual, residual_type, vec, per, rows, threads, stream);
    }
    return rc;
}

// What both calls share: the block's output or input, its gate and norm.
int rows_params(RowsParams& p, const vlut_rows* y, const float* weight, const vlut_rows* gate, int activation, float eps, int64_t N, int64_t K, Alignment& a) {
    if (N < 1 || N >= kMostRows || K < 1) return VLUT_ERR_SHAPE;
    if (K > VLUT_MAX_ROW_FEATURES) return VLUT_ERR_UNSUPPORTED;
    if (!(eps >= 0.0f) || activation < VLUT_ACTIVATION_NONE || activation > VLUT_ACTIVATION_GELU) return VLUT_ERR_SHAPE;
    p = RowsParams{};
    a.stride(K);
    int rc = check_rows(y, a);
    if (rc != VLUT_OK) return rc;
    p.y = y->data;
    p.y_row = y->row_stride;
    if (gate) {
        if ((rc = check_rows(gate, a)) != VLUT_OK) return rc;
        if (gate->type != y->type && gate->type != VLUT_TYPE_F32) return VLUT_ERR_SHAPE;
        p.gate = gate->data;
        p.gate_row = gate->row_stride;
        p.gate_f32 = gate->type == VLUT_TYPE_F32;
    }
    p.weight = weight;
    if (weight) a.pointer(weight, 4);
    p.activation = activation;
    p.eps = eps;
    p.K = (int)K;
    return VLUT_OK;
}

// ---------------------------------------------------------------------------------------------
// Logits
// ---------------------------------------------------------------------------------------------
struct LogitsPlan {
    int per, part, parts;              // logits of a thread and chunk, of a part; parts of a row
    size_t sums_bytes, keys_bytes;
};
int plan_logits(int64_t N, int64_t V, int top, LogitsPlan* out) {
    if (N < 1 || N >= kMostRows || V < 1 || V >= ((int64_t)1 << 30) || top < 0 || top > V) return VLUT_ERR_SHAPE;
    if (top > VLUT_MAX_TOP) return VLUT_ERR_UNSUPPORTED;
    LogitsPlan a{};
    // Parts so that there are four workgroups for each unit, of 2048 logits at least: 8 a thread, which are on their way at once, or of longer parts 16.  us with 2048 / 4096 /
    // 8192: one row of 32000 12.7, 15.5, 16.3, of 128000 13.0, 17.6, 20.9, 33 of 50001 12.0, 14.6, 16.9, 64 of 32000 10.6, 11.9, 12.3.  With two workgroups a unit the
    // last two 13.3 and 11.8.  8 / 16 logits a thread: one row of 128000 13.0, 13.6, of 2^20 29.0, 23.3, 33 of 50001 12.0, 12.2; 256 of 128000 33.8, 37.0, 2048 of 32000
    // 55.6, 55.1.
    const int64_t wanted = std::min<int64_t>({kMostParts, (4 * kUnits + N - 1) / N, (V + 2047) / 2048});
    const int64_t part = (V + wanted - 1) / wanted;
    a.per = part <= 4096 ? 8 : 16;
    const int64_t chunk = kLogitThreads * a.per;
    a.part = (int)((part + chunk - 1) / chunk * chunk);
    a.parts = (int)((V + a.part - 1) / a.part);
    if (a.parts > 1) {
        a.sums_bytes = (size_t)N * a.parts * 16;
        a.keys_bytes = (size_t)N * a.parts * top * 8;
    }
    *out = a;
    return VLUT_OK;
}
template <class T, int VEC>
int launch_logits_v(const LogitsParams& p, int per, unsigned blocks, hipStream_t stream) {
    return per == 8 ? launch(logits_kernel<T, VEC, 8>, dim3(blocks), kLogitThreads, 0, stream, p) : launch(logits_kernel<T, VEC, 16>, dim3(blocks), kLogitThreads, 0, stream, p);
}
template <class T>
int launch_logits(LogitsParams& p, const LogitsPlan& a, int vec, int64_t N, hipStream_t stream) {
    constexpr int64_t most = (int64_t)1 << 23;     // workgroups of a launch (parts are several only where rows are few)
    int rc = VLUT_OK;
    for (p.first_row = 0; rc == VLUT_OK && p.first_row < N; p.first_row += most) {
        const unsigned blocks = (unsigned)(std::min(N - p.first_row, most) * a.parts);
        if (vec == 4) rc = launch_logits_v<T, 4>(p, a.per, blocks, stream);
        else rc = launch_logits_v<T, 1>(p, a.per, blocks, stream);
    }
    p.first_row = 0;
    if (rc == VLUT_OK && a.parts > 1) rc = launch(logits_join_kernel<T>, dim3((unsigned)N), kLogitThreads, 0, stream, p);
    return rc;
}

}  // namespace

extern "C" {

int vlut_residual_norm(const vlut_rows* y, const float* weight_or_null, const vlut_rows* gate_or_null, int activation, float scale, const vlut_rows* residual,
                       const float* next_weight_or_null, float eps, int64_t N, int64_t K, const vlut_rows* h, const vlut_rows* x_or_null, void* stream) {
    if (!y || !residual || !h || !next_weight_or_null != !x_or_null) return VLUT_ERR_NULL;
    RowsParams p;
    Alignment a;
    int rc = rows_params(p, y, weight_or_null, gate_or_null, activation, eps, N, K, a);
    if (rc != VLUT_OK) return rc;
    if ((!gate_or_null && activation != VLUT_ACTIVATION_NONE) || !std::isfinite(scale)) return VLUT_ERR_SHAPE;
    for (const vlut_rows* r : {residual, h, x_or_null})
        if (r && (rc = check_rows(r, a)) != VLUT_OK) return rc;
    if (h->type != residual->type) return VLUT_ERR_SHAPE;
    p.residual = residual->data;
    p.residual_row = residual->row_stride;
    p.h = (void*)h->data;
    p.h_row = h->row_stride;
    p.h_type = h->type;
    p.scale = scale;
    p.next_weight = next_weight_or_null;
    if (x_or_null) {
        a.pointer(next_weight_or_null, 4);
        p.x = (void*)x_or_null->data;
        p.x_row = x_or_null->row_stride;
        p.x_type = x_or_null->type;
    }
    return launch_rows(p, y->type, true, residual->type, a.vec, N, (hipStream_t)stream);
}

int vlut_gated_norm(const vlut_rows* x, const vlut_rows* gate_or_null, int activation, const float* weight_or_null, float eps, int64_t N, int64_t K,
                    const vlut_rows* out, void* stream) {
    if (!x || !out) return VLUT_ERR_NULL;
    RowsParams p;
    Alignment a;
    int rc = rows_params(p, x, weight_or_null, gate_or_null, activation, eps, N, K, a);
    if (rc != VLUT_OK || (rc = check_rows(out, a)) != VLUT_OK) return rc;
    p.h = (void*)out->data;
    p.h_row = out->row_stride;
    p.h_type = out->type;
    return launch_rows(p, x->type, false, 0, a.vec, N, (hipStream_t)stream);
}

size_t vlut_token_logprobs_bytes(int64_t N, int64_t V, int top) {
    LogitsPlan a;
    return plan_logits(N, V, top, &a) == VLUT_OK ? a.sums_bytes + a.keys_bytes : 0;
}

int vlut_token_logprobs(const vlut_rows* logits, const int64_t* tokens_or_null, float temperature, int top, int64_t N, int64_t V, float* logprob_or_null,
                        float* entropy_or_null, int64_t* top_ids_or_null, float* top_logprobs_or_null, void* workspace, size_t workspace_bytes, void* stream) {
    if (!logits) return VLUT_ERR_NULL;
    LogitsPlan a;
    const int rc = plan_logits(N, V, top, &a);
    if (rc != VLUT_OK) return rc;
    if (!logits->data || !tokens_or_null != !logprob_or_null || (top > 0) != (top_ids_or_null != nullptr) || !top_ids_or_null != !top_logprobs_or_null) return VLUT_ERR_NULL;
    if (!logprob_or_null && !entropy_or_null && top == 0) return VLUT_ERR_NULL;
    if (!type_ok(logits->type) || !(temperature > 0.0f) || !std::isfinite(temperature) ||
        !std::isfinite((float)(1.4426950408889634 / (double)temperature)))
        return VLUT_ERR_SHAPE;
    if (a.parts > 1) {
        if (!workspace) return VLUT_ERR_NULL;
        if (workspace_bytes < a.sums_bytes + a.keys_bytes) return VLUT_ERR_SMALL_BUFFER;
        if ((uintptr_t)workspace % 16) return VLUT_ERR_UNSUPPORTED;
    }
    Alignment v;
    v.pointer(logits->data, type_bytes(logits->type));
    v.stride(logits->row_stride);
    v.stride(V);
    LogitsParams p{};
    p.logits = logits->data;
    p.row_stride = logits->row_stride;
    p.tokens = tokens_or_null;
    p.logprob = logprob_or_null;
    p.entropy = entropy_or_null;
    p.top_ids = top_ids_or_null;
    p.top_logprobs = top_logprobs_or_null;
    p.part_sums = (float*)workspace;
    p.part_keys = (uint64_t*)((unsigned char*)workspace + a.sums_bytes);
    p.V = (int)V;
    p.top = top;
    p.parts = a.parts;
    p.part = a.part;
    p.c = (float)(1.4426950408889634 / (double)temperature);
    p.inverse_temperature = (float)(1.0 / (double)temperature);
    if (logits->type == VLUT_TYPE_F32) return launch_logits<float>(p, a, v.vec, N, (hipStream_t)stream);
    if (logits->type == VLUT_TYPE_BF16) return launch_logits<__bf16>(p, a, v.vec, N, (hipStream_t)stream);
    return launch_logits<_Float16>(p, a, v.vec, N, (hipStream_t)stream);
}

}  // extern "C"
