// Which instance of the attention's kernels a call runs, and its launch.
// Part of the translation units attention_bf16.hip and attention_f16.hip (included there, in this order).
#pragma once

namespace {

int log2_of(int64_t v) {
    int k = 0;
    while (((int64_t)1 << k) < v) ++k;
    return k;
}
int64_t ceil_div(int64_t a, int64_t b) { return (a + b - 1) / b; }

bool allow_lds(const void* kfn, int bytes, std::atomic<unsigned>& done_mask) {
    int dev = 0;
    if (hipGetDevice(&dev) != hipSuccess) return false;
    const unsigned bit = (dev >= 0 && dev < 32) ? (1u << dev) : 0u;
    if (bit && (done_mask.load(std::memory_order_relaxed) & bit)) return true;
    if (hipFuncSetAttribute(kfn, hipFuncAttributeMaxDynamicSharedMemorySize, bytes) != hipSuccess) {
        (void)hipGetLastError();
        return false;
    }
    done_mask.fetch_or(bit, std::memory_order_relaxed);
    return true;
}

template <class T, int DP, int MT, int NW, int TERMS, int OWN, bool WHOLE>
int launch_attend_t(const AttendPlan& a, const AttendParams& p, hipStream_t stream) {
    static std::atomic<unsigned> done{0};
    constexpr int lds = MT == 0 ? std::max(2 * many_buffer(DP) + 16, few_lds(DP, NW)) : few_lds(DP, NW);
    auto kfn = attend_kernel<T, DP, MT, NW, TERMS, OWN, WHOLE>;
    if (lds > 64 * 1024 && !allow_lds((const void*)kfn, lds, done)) return VLUT_ERR_DEVICE;
    return launch(kfn, dim3((unsigned)(a.prefix_blocks + a.own_blocks)), 64 * NW, lds, stream, p);
}
template <class T, int DP, int NW, bool WHOLE>
int launch_attend_many(const AttendPlan& a, const AttendParams& p, hipStream_t stream) {
    if (p.out_type == VLUT_TYPE_F32) return a.own_mt == 1 ? launch_attend_t<T, DP, 0, NW, 2, 1, WHOLE>(a, p, stream) : launch_attend_t<T, DP, 0, NW, 2, 2, WHOLE>(a, p, stream);
    return a.own_mt == 1 ? launch_attend_t<T, DP, 0, NW, 1, 1, WHOLE>(a, p, stream) : launch_attend_t<T, DP, 0, NW, 1, 2, WHOLE>(a, p, stream);
}
template <class T, int DP, bool WHOLE>
int launch_attend_w(const AttendPlan& a, const AttendParams& p, hipStream_t stream) {
    if (a.MT == 1) return launch_attend_t<T, DP, 1, 4, 0, 1, WHOLE>(a, p, stream);
    if (a.MT == 2) return a.own_mt == 1 ? launch_attend_t<T, DP, 2, 4, 0, 1, WHOLE>(a, p, stream) : launch_attend_t<T, DP, 2, 4, 0, 2, WHOLE>(a, p, stream);
    if constexpr (DP <= 128)
        if (a.waves == 8) return launch_attend_many<T, DP, 8, WHOLE>(a, p, stream);
    return launch_attend_many<T, DP, 4, WHOLE>(a, p, stream);
}
template <class T, int DP>
int launch_attend_d(const AttendPlan& a, const AttendParams& p, hipStream_t stream) {
    const int rc = p.D == DP ? launch_attend_w<T, DP, true>(a, p, stream) : launch_attend_w<T, DP, false>(a, p, stream);
    if (rc != VLUT_OK || a.direct) return rc;
    constexpr int groups = 256 / (DP / 4);
    const int lanes_log = std::min(log2_of(groups), log2_of(ceil_div(a.prefix_splits + a.own_splits, 4)));
    return launch(combine_kernel<DP>, dim3((unsigned)ceil_div(a.rows * p.Hk, groups >> lanes_log)), 256, 0, stream, p, lanes_log);
}
template <class T>
int launch_attend(const AttendPlan& a, const AttendParams& p, hipStream_t stream) {
    if (a.DP == 64) return launch_attend_d<T, 64>(a, p, stream);
    if (a.DP == 128) return launch_attend_d<T, 128>(a, p, stream);
    return launch_attend_d<T, 256>(a, p, stream);
}

}  // namespace
