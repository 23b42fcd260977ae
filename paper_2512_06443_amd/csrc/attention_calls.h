// The native form of norm_rope, append_kv and shared_prefix_attention.  Part of torch_calls.cpp (included there, behind its helpers); what is said
// there holds: None for every argument that is not known to be ordinary or fails a check, before anything is launched, and the Python
// form raises the error.
// Host time of a call, Python / native form, us (what ctypes' structures, torch.empty and attribute reads take): norm_rope of one token 20 / 6, append_kv with
// queries 21 / 5, shared_prefix_attention, two launches, 21 / 9.
#pragma once

#include <torch/csrc/Dtype.h>

#include <cmath>

namespace {

struct AttentionApi {                          // in the order of binding._NATIVE_ATTENTION_ORDER
    decltype(&vlut_norm_rope) norm_rope;
    decltype(&vlut_append_kv) append_kv;
    decltype(&vlut_shared_prefix_attention) attention;
    decltype(&vlut_shared_prefix_attention_bytes) attention_bytes;
};
constexpr int kAttentionApiCount = (int)(sizeof(AttentionApi) / sizeof(void*));
AttentionApi g_attention;
bool g_attention_bound = false;

bool attention_call(Py_ssize_t n, Py_ssize_t want) { return g_attention_bound && n == want && !at::impl::torch_function_mode_enabled(); }

int number_type(c10::ScalarType t) { return t == at::kFloat ? VLUT_TYPE_F32 : (t == at::kBFloat16 ? VLUT_TYPE_BF16 : (t == at::kHalf ? VLUT_TYPE_F16 : -1)); }
// features (the last dimension) contiguous, a type of heads
bool features(const at::Tensor* t, int64_t dim) {
    return t && t->dim() == dim && number_type(t->scalar_type()) >= 0 && (t->size(dim - 1) <= 1 || t->stride(dim - 1) == 1);
}
bool indices(const at::Tensor* t, c10::ScalarType type, int64_t size) {
    return t && t->scalar_type() == type && t->dim() == 1 && t->is_contiguous() && t->numel() >= size;
}
// None, or tensor
bool optional_features(PyObject* o, const at::Tensor*& t, int64_t dim) { return optional(o, t) && (!t || features(t, dim)); }
bool same_sizes(const at::Tensor& a, const at::Tensor& b) { return a.sizes() == b.sizes(); }
bool norm_weight(const at::Tensor* w, const at::Tensor* of) {
    if (!w) return true;
    if (!of || w->scalar_type() != at::kFloat) return false;
    const int64_t H = of->size(1), D = of->size(2);
    if (!((w->dim() == 1 && w->size(0) == D) || (w->dim() == 2 && w->size(0) == H && w->size(1) == D))) return false;
    return D == 1 || w->stride(w->dim() - 1) == 1;
}
vlut_heads heads_of(const at::Tensor& t, const at::Tensor* w = nullptr) {
    return {t.data_ptr(), w ? (const float*)w->data_ptr() : nullptr, t.stride(0), t.stride(1), w && w->dim() == 2 ? w->stride(0) : 0, (int32_t)t.size(1),
            number_type(t.scalar_type())};
}
bool rotation_of(PyObject* positions, PyObject* cos, PyObject* sin, PyObject* interleaved, int64_t N, vlut_rotation& r, bool& any) {
    const at::Tensor *p, *c, *s;
    if (!optional(positions, p) || !optional(cos, c) || !optional(sin, s) || !PyBool_Check(interleaved)) return false;
    any = p != nullptr;
    if ((c != nullptr) != any || (s != nullptr) != any) return false;
    if (!any) return true;
    for (const at::Tensor* t : {c, s})
        if (t->scalar_type() != at::kFloat || t->dim() != 2 || !t->is_contiguous() || !same_sizes(*t, *c)) return false;
    if (!indices(p, at::kLong, N)) return false;
    r = {(const float*)c->data_ptr(), (const float*)s->data_ptr(), (const int64_t*)p->data_ptr(), c->size(0), (int32_t)(2 * c->size(1)), interleaved == Py_True};
    return true;
}
bool cache_of(const at::Tensor* k, const at::Tensor* v, int64_t D, vlut_cache& c) {
    if (!features(k, 4) || !features(v, 4) || !same_sizes(*k, *v) || k->scalar_type() != v->scalar_type() || k->size(3) != D) return false;
    c = {k->data_ptr(), v->data_ptr(), k->size(0), k->size(2), k->stride(0), k->stride(1), k->stride(2), v->stride(0), v->stride(1), v->stride(2),
         (int32_t)k->size(1), number_type(k->scalar_type())};
    return true;
}
// None (then `type` stays), or a dtype
bool type_of(PyObject* o, c10::ScalarType& type) {
    if (o == Py_None) return true;
    if (!THPDtype_Check(o)) return false;
    type = reinterpret_cast<THPDtype*>(o)->scalar_type;
    return number_type(type) >= 0;
}

// norm_rope(q, k, positions, cos, sin, q_weight, k_weight, eps, interleaved, dtype, q_out, k_out)
PyObject* py_norm_rope(PyObject*, PyObject* const* o, Py_ssize_t n) {
    return guarded([&]() -> PyObject* {
        const at::Tensor *q, *k, *qw, *kw, *gq, *gk;
        float eps;
        vlut_rotation rot;
        bool rotated;
        if (!attention_call(n, 12) || !features(q = plain(o[0]), 3) || !optional_features(o[1], k, 3) || !optional(o[5], qw) || !optional(o[6], kw) || !real(o[7], eps) ||
            !optional_features(o[10], gq, 3) || !optional_features(o[11], gk, 3))
            Py_RETURN_NONE;
        const int64_t N = q->size(0), D = q->size(2);
        if ((k && (k->size(0) != N || k->size(2) != D)) || !norm_weight(qw, q) || (k && !norm_weight(kw, k)) || !rotation_of(o[2], o[3], o[4], o[8], N, rot, rotated)) Py_RETURN_NONE;
        c10::ScalarType type = gq ? gq->scalar_type() : q->scalar_type();
        if (!type_of(o[9], type) || (gq && !same_sizes(*gq, *q)) || (gk && (!k || !same_sizes(*gk, *k)))) Py_RETURN_NONE;
        at::Tensor q_out, k_out;
        if (gq) q_out = *gq;
        if (gk) k_out = *gk;
        int rc;
        without_gil([&] {
            if (!gq) q_out = make(q->sizes(), type, q->device());
            if (k && !gk) k_out = make(k->sizes(), type, q->device());
            const vlut_heads qi = heads_of(*q, qw), qo = heads_of(q_out);
            vlut_heads ki, ko;
            if (k) {
                ki = heads_of(*k, kw);
                ko = heads_of(k_out);
            }
            rc = g_attention.norm_rope(&qi, k ? &ki : nullptr, eps, rotated ? &rot : nullptr, N, D, &qo, k ? &ko : nullptr, stream());
        });
        return result(rc, q_out, k_out);
    });
}

// append_kv(k, v, slots, k_cache, v_cache, positions, cos, sin, k_weight, eps, interleaved, q, q_weight, q_out): a tuple of q_out or None
PyObject* py_append_kv(PyObject*, PyObject* const* o, Py_ssize_t n) {
    return guarded([&]() -> PyObject* {
        const at::Tensor *k, *v, *q, *kw, *qw, *gq, *slots;
        float eps;
        vlut_rotation rot;
        vlut_cache cache;
        bool rotated;
        if (!attention_call(n, 14) || !features(k = plain(o[0]), 3) || !features(v = plain(o[1]), 3) || !same_sizes(*k, *v)) Py_RETURN_NONE;
        const int64_t N = k->size(0), D = k->size(2);
        const at::Tensor *kc = plain(o[3]), *vc = plain(o[4]);
        if (!indices(slots = plain(o[2]), at::kLong, N) || !cache_of(kc, vc, D, cache) || !optional(o[8], kw) || !real(o[9], eps) || !optional_features(o[11], q, 3) ||
            !optional(o[12], qw) || !optional_features(o[13], gq, 3) || !norm_weight(kw, k) || (q && !norm_weight(qw, q)) ||
            !rotation_of(o[5], o[6], o[7], o[10], N, rot, rotated))
            Py_RETURN_NONE;
        if ((q && (q->size(0) != N || q->size(2) != D)) || (gq && (!q || !same_sizes(*gq, *q)))) Py_RETURN_NONE;
        at::Tensor q_out;
        if (gq) q_out = *gq;
        int rc;
        without_gil([&] {
            if (q && !gq) q_out = make(q->sizes(), kc->scalar_type(), q->device());
            const vlut_heads ki = heads_of(*k, kw), vi = heads_of(*v);
            vlut_heads qi, qo;
            if (q) {
                qi = heads_of(*q, qw);
                qo = heads_of(q_out);
            }
            rc = g_attention.append_kv(&ki, &vi, q ? &qi : nullptr, eps, rotated ? &rot : nullptr, (const int64_t*)slots->data_ptr(), N, D, &cache, q ? &qo : nullptr, stream());
        });
        return result(rc, q_out);
    });
}

// shared_prefix_attention(q, k_cache, v_cache, prefix_pages, prefix_len, page_table, own_lens, query_lens, max_own_len, scale, dtype, out, want_lse, workspace)
PyObject* py_shared_prefix_attention(PyObject*, PyObject* const* o, Py_ssize_t n) {
    return guarded([&]() -> PyObject* {
        const at::Tensor *q, *prefix, *table, *lens, *queries, *gout, *gws;
        vlut_cache cache;
        int64_t prefix_len, max_own = 0;
        float scale;
        if (!attention_call(n, 14) || !features(q = plain(o[0]), 4)) Py_RETURN_NONE;
        const int64_t B = q->size(0), nq = q->size(1), Hq = q->size(2), D = q->size(3);
        const at::Tensor *kc = plain(o[1]), *vc = plain(o[2]);
        if (!cache_of(kc, vc, D, cache) || !optional(o[3], prefix) || !whole(o[4], prefix_len) || !optional(o[5], table) || !indices(lens = plain(o[6]), at::kInt, B) ||
            !optional(o[7], queries) || !optional_features(o[11], gout, 4) || !workspace(o[13], gws) || D < 1 || cache.page_size < 1)
            Py_RETURN_NONE;
        if (table && (table->scalar_type() != at::kInt || table->dim() != 2 || table->size(0) != B || (table->size(1) > 1 && table->stride(1) != 1))) Py_RETURN_NONE;
        const int64_t room = table ? table->size(1) * cache.page_size : 0;
        if (o[8] == Py_None) max_own = room;
        else if (!whole(o[8], max_own)) Py_RETURN_NONE;
        if (max_own > room || (queries && !indices(queries, at::kInt, B))) Py_RETURN_NONE;
        if (prefix_len > 0 && !indices(prefix, at::kInt, (prefix_len - 1) / cache.page_size + 1)) Py_RETURN_NONE;
        if (o[9] == Py_None) scale = (float)std::pow((double)D, -0.5);
        else if (!real(o[9], scale)) Py_RETURN_NONE;
        c10::ScalarType type = q->scalar_type();
        const int want_lse = PyObject_IsTrue(o[12]);
        if (want_lse < 0) { PyErr_Clear(); Py_RETURN_NONE; }
        if (!type_of(o[10], type) || (gout && !same_sizes(*gout, *q))) Py_RETURN_NONE;
        at::Tensor out, lse, ws;
        if (gout) out = *gout;
        if (gws) ws = *gws;
        int rc;
        without_gil([&] {
            if (!gout) out = make(q->sizes(), type, q->device());
            if (want_lse) lse = make({B, nq, Hq}, at::kFloat, q->device());
            if (!gws) {
                const size_t need = g_attention.attention_bytes(B, nq, Hq, cache.heads, D, prefix_len, max_own);
                if (need) ws = make({(int64_t)need}, at::kByte, q->device());
            }
            auto rows = [&](const at::Tensor& t) { return vlut_heads{t.data_ptr(), nullptr, t.stride(1), t.stride(2), 0, (int32_t)Hq, number_type(t.scalar_type())}; };
            const vlut_heads qi = rows(*q), oi = rows(out);
            rc = g_attention.attention(&qi, q->stride(0), &cache, prefix ? (const int32_t*)prefix->data_ptr() : nullptr, prefix_len,
                                       table ? (const int32_t*)table->data_ptr() : nullptr, table ? table->stride(0) : 0, (const int32_t*)lens->data_ptr(), max_own,
                                       queries ? (const int32_t*)queries->data_ptr() : nullptr, B, nq, D, scale, &oi, out.stride(0), ptr<float>(lse), ptr<void>(ws),
                                       ws.defined() ? bytes_of(ws) : 0, stream());
        });
        return result(rc, out, lse);
    });
}

// bind_attention(addresses): the functions of the loaded library, as whole numbers in the order of AttentionApi
PyObject* py_bind_attention(PyObject*, PyObject* const* o, Py_ssize_t n) {
    void* address[kAttentionApiCount];
    if (!addresses(o, n, address, kAttentionApiCount)) return nullptr;
    std::memcpy((void*)&g_attention, address, sizeof(g_attention));
    g_attention_bound = true;
    Py_RETURN_NONE;
}

}  // namespace
