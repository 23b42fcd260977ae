// The native form of chunk_attention, residual_norm, gated_norm and token_logprobs.  Part of torch_calls.cpp (included there, behind attention_calls.h); what is said there holds.
#pragma once

namespace {

struct LayerApi {                              // in the order of binding._NATIVE_LAYER_ORDER
    decltype(&vlut_chunk_attention) chunk_attention;
    decltype(&vlut_chunk_attention_bytes) chunk_attention_bytes;
    decltype(&vlut_residual_norm) residual_norm;
    decltype(&vlut_gated_norm) gated_norm;
    decltype(&vlut_token_logprobs) token_logprobs;
    decltype(&vlut_token_logprobs_bytes) token_logprobs_bytes;
};
constexpr int kLayerApiCount = (int)(sizeof(LayerApi) / sizeof(void*));
LayerApi g_layer;
bool g_layer_bound = false;

bool layer_call(Py_ssize_t n, Py_ssize_t want) { return g_layer_bound && n == want && !at::impl::torch_function_mode_enabled(); }

// Every tensor is on the current device (whose current stream the call gets).
template <class... T>
bool here(const T*... t) {
    const c10::DeviceIndex current = c10::hip::current_device();
    return (... && (!t || t->device().index() == current));
}

// chunk_attention(q, k_cache, v_cache, page_table, query_starts, lens, max_queries, max_len, window, scale, dtype, out, want_lse, workspace)
PyObject* py_chunk_attention(PyObject*, PyObject* const* o, Py_ssize_t n) {
    return guarded([&]() -> PyObject* {
        const at::Tensor *q, *gout, *gws;
        vlut_cache cache;
        int64_t max_queries, max_len, window;
        float scale;
        if (!layer_call(n, 14) || !features(q = plain(o[0]), 3)) Py_RETURN_NONE;
        const int64_t N = q->size(0), Hq = q->size(1), D = q->size(2);
        const at::Tensor *kc = plain(o[1]), *vc = plain(o[2]), *table = plain(o[3]), *starts = plain(o[4]), *lens = plain(o[5]);
        if (D < 1 || !cache_of(kc, vc, D, cache) || cache.page_size < 1 || !table || table->scalar_type() != at::kInt || table->dim() != 2 ||
            (table->size(1) > 1 && table->stride(1) != 1))
            Py_RETURN_NONE;
        const int64_t B = table->size(0), room = table->size(1) * cache.page_size;
        if (!starts || starts->scalar_type() != at::kInt || starts->dim() != 1 || starts->size(0) != B + 1 || !starts->is_contiguous() || !indices(lens, at::kInt, B)) Py_RETURN_NONE;
        if (o[6] == Py_None) max_queries = N;
        else if (!whole(o[6], max_queries)) Py_RETURN_NONE;
        if (o[7] == Py_None) max_len = room;
        else if (!whole(o[7], max_len)) Py_RETURN_NONE;
        if (max_len > room || !whole(o[8], window)) Py_RETURN_NONE;
        if (o[9] == Py_None) scale = (float)std::pow((double)D, -0.5);
        else if (!real(o[9], scale)) Py_RETURN_NONE;
        c10::ScalarType type = q->scalar_type();
        const int want_lse = PyObject_IsTrue(o[12]);
        if (want_lse < 0) { PyErr_Clear(); Py_RETURN_NONE; }
        if (!type_of(o[10], type) || !optional_features(o[11], gout, 3) || (gout && !same_sizes(*gout, *q)) || !workspace(o[13], gws) ||
            !here(q, kc, vc, table, starts, lens, gout, gws))
            Py_RETURN_NONE;
        at::Tensor out, lse, ws;
        if (gout) out = *gout;
        if (gws) ws = *gws;
        int rc;
        without_gil([&] {
            if (!gout) out = make(q->sizes(), type, q->device());
            if (want_lse) lse = make({N, Hq}, at::kFloat, q->device());
            if (!gws) {
                const size_t need = g_layer.chunk_attention_bytes(N, B, Hq, cache.heads, D, max_queries, max_len, window);
                if (need) ws = make({(int64_t)need}, at::kByte, q->device());
            }
            const vlut_heads qi = heads_of(*q), oi = heads_of(out);
            rc = g_layer.chunk_attention(&qi, &cache, (const int32_t*)table->data_ptr(), table->stride(0), (const int32_t*)starts->data_ptr(), (const int32_t*)lens->data_ptr(),
                                         N, B, D, max_queries, max_len, window, scale, &oi, ptr<float>(lse), ptr<void>(ws), ws.defined() ? bytes_of(ws) : 0, stream());
        });
        return result(rc, out, lse);
    });
}

bool rows_like(const at::Tensor* t, int64_t N, int64_t K) { return features(t, 2) && t->size(0) == N && t->size(1) == K; }
bool row_weight(const at::Tensor* w, int64_t K) { return !w || (w->scalar_type() == at::kFloat && w->dim() == 1 && w->size(0) == K && w->is_contiguous()); }
vlut_rows rows_of(const at::Tensor& t) { return {t.data_ptr(), t.stride(0), number_type(t.scalar_type())}; }
// [N][K], or [K] for all tokens
bool gate_of(const at::Tensor* gate, int64_t N, int64_t K, vlut_rows& r) {
    if (!gate) return true;
    if (rows_like(gate, N, K)) {
        r = rows_of(*gate);
        return true;
    }
    if (!features(gate, 1) || gate->size(0) != K) return false;
    r = {gate->data_ptr(), 0, number_type(gate->scalar_type())};
    return true;
}
bool activation_of(PyObject* o, int& code) {
    if (o == Py_None) {
        code = VLUT_ACTIVATION_NONE;
        return true;
    }
    if (!PyUnicode_CheckExact(o)) return false;
    static const char* const names[] = {"none", "sigmoid", "silu", "relu2", "gelu"};
    for (code = 0; code < 5; ++code)
        if (PyUnicode_CompareWithASCIIString(o, names[code]) == 0) return true;
    return false;
}

// residual_norm(y, residual, weight, gate, activation, scale, next_weight, eps, dtype, out, next_out)
PyObject* py_residual_norm(PyObject*, PyObject* const* o, Py_ssize_t n) {
    return guarded([&]() -> PyObject* {
        const at::Tensor *y, *residual, *w, *gate, *nw, *gout, *gnext;
        int activation;
        float scale, eps;
        vlut_rows g;
        if (!layer_call(n, 11) || !features(y = plain(o[0]), 2)) Py_RETURN_NONE;
        const int64_t N = y->size(0), K = y->size(1);
        if (!rows_like(residual = plain(o[1]), N, K) || !optional(o[2], w) || !optional(o[3], gate) || !activation_of(o[4], activation) || !real(o[5], scale) ||
            !optional(o[6], nw) || !real(o[7], eps) || !optional(o[9], gout) || !optional(o[10], gnext) || !row_weight(w, K) || !row_weight(nw, K) ||
            !gate_of(gate, N, K, g) || (gout && !rows_like(gout, N, K)) || (gnext && (!nw || !rows_like(gnext, N, K))) || !here(y, residual, w, gate, nw, gout, gnext))
            Py_RETURN_NONE;
        c10::ScalarType type = y->scalar_type();
        if (!type_of(o[8], type)) Py_RETURN_NONE;
        at::Tensor out, next;
        if (gout) out = *gout;
        if (gnext) next = *gnext;
        int rc;
        without_gil([&] {
            if (!gout) out = make({N, K}, residual->scalar_type(), y->device());
            if (nw && !gnext) next = make({N, K}, type, y->device());
            const vlut_rows yi = rows_of(*y), ri = rows_of(*residual), ho = rows_of(out);
            vlut_rows xo;
            if (nw) xo = rows_of(next);
            rc = g_layer.residual_norm(&yi, w ? (const float*)w->data_ptr() : nullptr, gate ? &g : nullptr, activation, scale, &ri,
                                       nw ? (const float*)nw->data_ptr() : nullptr, eps, N, K, &ho, nw ? &xo : nullptr, stream());
        });
        return result(rc, out, next);
    });
}

// gated_norm(x, gate, activation, weight, eps, dtype, out): a tuple of out
PyObject* py_gated_norm(PyObject*, PyObject* const* o, Py_ssize_t n) {
    return guarded([&]() -> PyObject* {
        const at::Tensor *x, *gate, *w, *gout;
        int activation;
        float eps;
        vlut_rows g;
        if (!layer_call(n, 7) || !features(x = plain(o[0]), 2)) Py_RETURN_NONE;
        const int64_t N = x->size(0), K = x->size(1);
        c10::ScalarType type = x->scalar_type();
        if (!optional(o[1], gate) || !activation_of(o[2], activation) || !optional(o[3], w) || !real(o[4], eps) || !type_of(o[5], type) || !optional(o[6], gout) ||
            !row_weight(w, K) || !gate_of(gate, N, K, g) || (gout && !rows_like(gout, N, K)) || !here(x, gate, w, gout))
            Py_RETURN_NONE;
        at::Tensor out;
        if (gout) out = *gout;
        int rc;
        without_gil([&] {
            if (!gout) out = make({N, K}, type, x->device());
            const vlut_rows xi = rows_of(*x), oo = rows_of(out);
            rc = g_layer.gated_norm(&xi, gate ? &g : nullptr, activation, w ? (const float*)w->data_ptr() : nullptr, eps, N, K, &oo, stream());
        });
        return result(rc, out);
    });
}

// token_logprobs(logits, tokens, top, temperature, want_entropy, workspace)
PyObject* py_token_logprobs(PyObject*, PyObject* const* o, Py_ssize_t n) {
    return guarded([&]() -> PyObject* {
        const at::Tensor *logits, *tokens, *gws;
        int64_t top;
        float temperature;
        if (!layer_call(n, 6) || !features(logits = plain(o[0]), 2) || !optional(o[1], tokens) || !whole(o[2], top) || !real(o[3], temperature) || !workspace(o[5], gws)) Py_RETURN_NONE;
        const int64_t N = logits->size(0), V = logits->size(1);
        const int want_entropy = PyObject_IsTrue(o[4]);
        if (want_entropy < 0) { PyErr_Clear(); Py_RETURN_NONE; }
        if ((tokens && !indices(tokens, at::kLong, N)) || top < 0 || top > VLUT_MAX_TOP || !here(logits, tokens, gws)) Py_RETURN_NONE;
        at::Tensor logprob, entropy, ids, logprobs, ws;
        if (gws) ws = *gws;
        int rc;
        without_gil([&] {
            const c10::Device dev = logits->device();
            if (tokens) logprob = make({N}, at::kFloat, dev);
            if (want_entropy) entropy = make({N}, at::kFloat, dev);
            if (top > 0) {
                ids = make({N, top}, at::kLong, dev);
                logprobs = make({N, top}, at::kFloat, dev);
            }
            if (!gws) {
                const size_t need = g_layer.token_logprobs_bytes(N, V, (int)top);
                if (need) ws = make({(int64_t)need}, at::kByte, dev);
            }
            const vlut_rows li = rows_of(*logits);
            rc = g_layer.token_logprobs(&li, tokens ? (const int64_t*)tokens->data_ptr() : nullptr, temperature, (int)top, N, V, ptr<float>(logprob), ptr<float>(entropy),
                                        ptr<int64_t>(ids), ptr<float>(logprobs), ptr<void>(ws), ws.defined() ? bytes_of(ws) : 0, stream());
        });
        return result(rc, logprob, entropy, ids, logprobs);
    });
}

// bind_layer(addresses): as bind_attention
PyObject* py_bind_layer(PyObject*, PyObject* const* o, Py_ssize_t n) {
    void* address[kLayerApiCount];
    if (!addresses(o, n, address, kLayerApiCount)) return nullptr;
    std::memcpy((void*)&g_layer, address, sizeof(g_layer));
    g_layer_bound = true;
    Py_RETURN_NONE;
}

}  // namespace
