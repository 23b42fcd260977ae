// Which instance of the kernels for chunks a call runs, and its launch.
// Part of the translation units chunk_bf16.hip and chunk_f16.hip (included there, in this order).
#pragma once

namespace {

template <class T, int DP, int TERMS, bool FAST>
int launch_few_rows(const ChunkPlan& a, const ChunkParams& p, hipStream_t stream) {
    static std::atomic<unsigned> done{0};
    constexpr int waves = few_waves(DP, FAST), lds = lds_bytes(DP, 1, waves, FAST);
    auto kfn = few_rows_kernel<T, DP, TERMS, FAST>;
    if (lds > 64 * 1024 && !allow_lds((const void*)kfn, lds, done)) return VLUT_ERR_DEVICE;
    return launch(kfn, dim3(8u * (unsigned)a.few_per_xcd), 64 * waves, lds, stream, p);
}
template <class T, int DP, int RW, int TERMS, bool FAST>
int launch_many_rows(const ChunkPlan& a, const ChunkParams& p, hipStream_t stream) {
    static std::atomic<unsigned> done{0};
    constexpr int lds = lds_bytes(DP, RW, 1, FAST);
    auto kfn = many_rows_kernel<T, DP, RW, TERMS, FAST>;
    if (lds > 64 * 1024 && !allow_lds((const void*)kfn, lds, done)) return VLUT_ERR_DEVICE;
    return launch(kfn, dim3(8u * (unsigned)a.many_per_xcd), 64 * RW, lds, stream, p);
}
template <class T, int DP, int TERMS, bool FAST>
int launch_parts(const ChunkPlan& a, const ChunkParams& p, hipStream_t stream) {
    int rc = VLUT_OK;
    if (a.many) {
        if constexpr (DP <= 128) rc = a.many_waves == 8 ? launch_many_rows<T, DP, 8, TERMS, FAST>(a, p, stream) : launch_many_rows<T, DP, 4, TERMS, FAST>(a, p, stream);
        else rc = launch_many_rows<T, DP, 4, TERMS, FAST>(a, p, stream);
    }
    if (rc == VLUT_OK && a.few) rc = launch_few_rows<T, DP, TERMS, FAST>(a, p, stream);
    if (rc != VLUT_OK || a.bytes() == 0) return rc;
    constexpr int rows = 256 / (DP / 4);
    return launch(combine_chunks<T, DP>, dim3((unsigned)(((int64_t)p.N * p.Hk * p.G + rows - 1) / rows)), 256, 0, stream, p);
}
template <class T, int DP, int TERMS>
int launch_terms(const ChunkPlan& a, const ChunkParams& p, hipStream_t stream) {
    return a.fast ? launch_parts<T, DP, TERMS, true>(a, p, stream) : launch_parts<T, DP, TERMS, false>(a, p, stream);
}
template <class T, int DP>
int launch_d(const ChunkPlan& a, const ChunkParams& p, hipStream_t stream) {
    return p.out_type == VLUT_TYPE_F32 ? launch_terms<T, DP, Number<T>::kTerms>(a, p, stream) : launch_terms<T, DP, 1>(a, p, stream);
}
template <class T>
int launch_chunks(const ChunkPlan& a, const ChunkParams& p, hipStream_t stream) {
    if (a.DP == 64) return launch_d<T, 64>(a, p, stream);
    if (a.DP == 128) return launch_d<T, 128>(a, p, stream);
    return launch_d<T, 256>(a, p, stream);
}

}  // namespace
