// Which instance of the kernels for chunks a call runs, and its launch.
// Part of the translation units of the chunks' kernels (included there, in this order).
#pragma once

namespace {

template <class T, int DP, int TERMS, int LOAD>
int launch_few(const ChunkPlan& a, const ChunkParams& p, hipStream_t stream) {
    static std::atomic<unsigned> done{0};
    constexpr int lds = lds_bytes(DP, 1, few_waves(DP), LOAD);
    static_assert(lds <= 80 * 1024, "two workgroups a unit");
    auto kfn = few_rows_kernel<T, DP, TERMS, LOAD>;
    if (lds > 64 * 1024 && !allow_lds((const void*)kfn, lds, done)) return VLUT_ERR_DEVICE;
    return launch(kfn, dim3(8u * (unsigned)a.few_per_xcd), 64 * few_waves(DP), lds, stream, p);
}
template <class T, int DP, int KW, int TERMS, int LOAD>
int launch_many(const ChunkPlan& a, const ChunkParams& p, hipStream_t stream) {
    static std::atomic<unsigned> done{0};
    constexpr int lds = lds_bytes(DP, 4, KW, LOAD);
    static_assert(lds <= (KW == 1 && DP <= 128 ? 80 : 160) * 1024, "one or two workgroups a unit");
    auto kfn = many_rows_kernel<T, DP, KW, TERMS, LOAD>;
    if (lds > 64 * 1024 && !allow_lds((const void*)kfn, lds, done)) return VLUT_ERR_DEVICE;
    return launch(kfn, dim3(8u * (unsigned)a.many_per_xcd), 256 * KW, lds, stream, p);
}
template <class T, int DP, int TERMS, int LOAD>
int launch_parts(const ChunkPlan& a, const ChunkParams& p, hipStream_t stream) {
    int rc = VLUT_OK;
    if (a.many) {
        if constexpr (DP <= 128 && LOAD != kThroughRegisters) rc = a.key_waves == 2 ? launch_many<T, DP, 2, TERMS, LOAD>(a, p, stream) : launch_many<T, DP, 1, TERMS, LOAD>(a, p, stream);
        else rc = launch_many<T, DP, 1, TERMS, LOAD>(a, p, stream);
    }
    if (rc == VLUT_OK && a.few) rc = launch_few<T, DP, TERMS, LOAD>(a, p, stream);
    if (rc != VLUT_OK || a.bytes() == 0) return rc;
    constexpr int rows = 256 / (DP / 4);
    return launch(combine_chunks<typename Output<T, TERMS>::type, DP>, dim3((unsigned)(((int64_t)p.N * p.Hk * p.G + rows - 1) / rows)), 256, 0, stream, p);
}
template <class T, int DP, int TERMS>
int launch_loads(const ChunkPlan& a, const ChunkParams& p, hipStream_t stream) {
    if (a.load == kWholeVectors) return launch_parts<T, DP, TERMS, kWholeVectors>(a, p, stream);
    if (a.load == kVectors) return launch_parts<T, DP, TERMS, kVectors>(a, p, stream);
    if constexpr (DP <= 128)
        if (a.load == kRuns) return launch_parts<T, DP, TERMS, kRuns>(a, p, stream);
    if (a.load == kDwords) return launch_parts<T, DP, TERMS, kDwords>(a, p, stream);
    return launch_parts<T, DP, TERMS, kThroughRegisters>(a, p, stream);
}
template <class T, int TERMS>
int launch_chunks(const ChunkPlan& a, const ChunkParams& p, hipStream_t stream) {
    if (a.DP == 64) return launch_loads<T, 64, TERMS>(a, p, stream);
    if (a.DP == 128) return launch_loads<T, 128, TERMS>(a, p, stream);
    return launch_loads<T, 256, TERMS>(a, p, stream);
}

}  // namespace
