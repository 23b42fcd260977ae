// Which instance of the kernels for chunks a call runs, and its launch.
// Part of the translation units of the chunks' kernels (included there, in this order).
#pragma once

namespace {

template <class T, class O, int DP, int LOAD>
int launch_few(const ChunkPlan& a, const ChunkParams& p, hipStream_t stream) {
    static std::atomic<unsigned> done{0};
    constexpr int lds = lds_bytes(DP, 1, few_waves(DP), LOAD);
    static_assert(lds <= 80 * 1024, "two workgroups a unit");
    auto kfn = few_rows_kernel<T, O, DP, LOAD>;
    if (lds > 64 * 1024 && !allow_lds((const void*)kfn, lds, done)) return VLUT_ERR_DEVICE;
    return launch(kfn, dim3(8u * (unsigned)a.few_per_xcd), 64 * few_waves(DP), lds, stream, p);
}
template <class T, class O, int DP, int KW, int LOAD>
int launch_many(const ChunkPlan& a, const ChunkParams& p, hipStream_t stream) {
    static std::atomic<unsigned> done{0};
    constexpr int lds = lds_bytes(DP, 4, KW, LOAD);
    static_assert(lds <= (KW == 1 && DP <= 128 ? 80 : 160) * 1024, "one or two workgroups a unit");
    auto kfn = many_rows_kernel<T, O, DP, KW, LOAD>;
    if (lds > 64 * 1024 && !allow_lds((const void*)kfn, lds, done)) return VLUT_ERR_DEVICE;
    return launch(kfn, dim3(8u * (unsigned)a.many_per_xcd), 256 * KW, lds, stream, p);
}
template <class T, class O, int DP, int LOAD>
int launch_parts(const ChunkPlan& a, const ChunkParams& p, hipStream_t stream) {
    int rc = VLUT_OK;
    if (a.many) {
        if constexpr (DP <= 128 && LOAD != kThroughRegisters) rc = a.key_waves == 2 ? launch_many<T, O, DP, 2, LOAD>(a, p, stream) : launch_many<T, O, DP, 1, LOAD>(a, p, stream);
        else rc = launch_many<T, O, DP, 1, LOAD>(a, p, stream);
    }
    if (rc == VLUT_OK && a.few) rc = launch_few<T, O, DP, LOAD>(a, p, stream);
    if (rc != VLUT_OK || a.bytes() == 0) return rc;
    constexpr int rows = 256 / (DP / 4);
    return launch(combine_chunks<O, DP>, dim3((unsigned)(((int64_t)p.N * p.Hk * p.G + rows - 1) / rows)), 256, 0, stream, p);
}
template <class T, class O, int DP>
int launch_loads(const ChunkPlan& a, const ChunkParams& p, hipStream_t stream) {
    if (a.load == kWholeVectors) return launch_parts<T, O, DP, kWholeVectors>(a, p, stream);
    if (a.load == kVectors) return launch_parts<T, O, DP, kVectors>(a, p, stream);
    if constexpr (DP <= 128)
        if (a.load == kRuns) return launch_parts<T, O, DP, kRuns>(a, p, stream);
    if (a.load == kDwords) return launch_parts<T, O, DP, kDwords>(a, p, stream);
    return launch_parts<T, O, DP, kThroughRegisters>(a, p, stream);
}
template <class T, class O>
int launch_chunks(const ChunkPlan& a, const ChunkParams& p, hipStream_t stream) {
    if (a.DP == 64) return launch_loads<T, O, 64>(a, p, stream);
    if (a.DP == 128) return launch_loads<T, O, 128>(a, p, stream);
    return launch_loads<T, O, 256>(a, p, stream);
}

}  // namespace
