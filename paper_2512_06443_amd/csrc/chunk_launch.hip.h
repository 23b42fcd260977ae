// Which instance of the kernels for chunks a call runs, and its launch.
// Part of the translation units of the chunks' kernels (included there, in this order).
#pragma once

namespace {

template <class T, int DP, int RW, int TERMS, int LOAD>
int launch_chunk(const ChunkPlan& a, const ChunkParams& p, hipStream_t stream) {
    static std::atomic<unsigned> done{0};
    constexpr int lds = most_of(lds_bytes(DP, RW, LOAD), lds_bytes(DP, 1, LOAD));
    static_assert(lds <= 160 * 1024, "what a unit has");
    auto kfn = chunk_kernel<T, DP, RW, TERMS, LOAD>;
    if (lds > 64 * 1024 && !allow_lds((const void*)kfn, lds, done)) return VLUT_ERR_DEVICE;
    int rc = launch(kfn, dim3(8u * (unsigned)(a.many_per_xcd + a.few_per_xcd)), 64 * waves_of(DP), lds, stream, p);
    if (rc != VLUT_OK || a.bytes() == 0) return rc;
    constexpr int rows = 256 / (DP / 4);
    return launch(combine_chunks<typename Output<T, TERMS>::type, DP>, dim3((unsigned)(((int64_t)p.N * p.Hk * p.G + rows - 1) / rows)), 256, 0, stream, p);
}
template <class T, int DP, int TERMS, int LOAD>
int launch_waves(const ChunkPlan& a, const ChunkParams& p, hipStream_t stream) {
    if constexpr (DP <= 128)
        if (a.row_waves == 8) return launch_chunk<T, DP, 8, TERMS, LOAD>(a, p, stream);
    return launch_chunk<T, DP, 4, TERMS, LOAD>(a, p, stream);
}
template <class T, int DP, int TERMS>
int launch_loads(const ChunkPlan& a, const ChunkParams& p, hipStream_t stream) {
    if (a.load == kWholeVectors) return launch_waves<T, DP, TERMS, kWholeVectors>(a, p, stream);
    if (a.load == kVectors) return launch_waves<T, DP, TERMS, kVectors>(a, p, stream);
    if (a.load == kDwords) return launch_waves<T, DP, TERMS, kDwords>(a, p, stream);
    return launch_chunk<T, DP, 4, TERMS, kThroughRegisters>(a, p, stream);
}
template <class T, int TERMS>
int launch_chunks(const ChunkPlan& a, const ChunkParams& p, hipStream_t stream) {
    if (a.DP == 64) return launch_loads<T, 64, TERMS>(a, p, stream);
    if (a.DP == 128) return launch_loads<T, 128, TERMS>(a, p, stream);
    return launch_loads<T, 256, TERMS>(a, p, stream);
}

}  // namespace
