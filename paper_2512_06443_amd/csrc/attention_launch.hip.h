// Which instance of the attention's kernels a call runs, and its launch.
// Part of the translation units attention_bf16.hip and attention_f16.hip (included there, in this order).
#pragma once

namespace {

template <class T, int DP, int MT, int OWN, int TERMS, bool WHOLE, bool GROUPED>
int launch_few_t(const AttendParams& p, hipStream_t stream) {
    static std::atomic<unsigned> done{0};
    constexpr int lds = few_lds(DP);
    auto kfn = attend_few_kernel<T, DP, MT, OWN, TERMS, WHOLE, GROUPED>;
    if (lds > 64 * 1024 && !allow_lds((const void*)kfn, lds, done)) return VLUT_ERR_DEVICE;
    return launch(kfn, dim3(8u * (unsigned)(p.prefix_per_xcd + p.own_per_xcd)), 256, lds, stream, p);
}
template <class T, int DP, int MT, int OWN, int TERMS, bool WHOLE>
int launch_few_terms(const AttendPlan& a, const AttendParams& p, hipStream_t stream) {
    return a.grouped ? launch_few_t<T, DP, MT, OWN, TERMS, WHOLE, true>(p, stream) : launch_few_t<T, DP, MT, OWN, TERMS, false, false>(p, stream);
}
template <class T, int DP, int MT, int OWN, bool WHOLE>
int launch_few(const AttendPlan& a, const AttendParams& p, hipStream_t stream) {
    if (p.out_type == VLUT_TYPE_F32) return launch_few_terms<T, DP, MT, OWN, Number<T>::kTerms, WHOLE>(a, p, stream);
    return launch_few_terms<T, DP, MT, OWN, 2, WHOLE>(a, p, stream);
}
template <class T, int DP, int NW, int TERMS, bool WHOLE>
int launch_many(const AttendPlan& a, const AttendParams& p, hipStream_t stream) {
    static std::atomic<unsigned> done{0};
    constexpr int lds = 2 * many_buffer(DP) + 16;
    auto kfn = attend_many_kernel<T, DP, NW, TERMS, WHOLE>;
    if (lds > 64 * 1024 && !allow_lds((const void*)kfn, lds, done)) return VLUT_ERR_DEVICE;
    return launch(kfn, dim3(8u * (unsigned)a.prefix_per_xcd), 64 * NW, lds, stream, p);
}
template <class T, int DP, int NW, bool WHOLE>
int launch_many_terms(const AttendPlan& a, const AttendParams& p, hipStream_t stream) {
    if (p.out_type == VLUT_TYPE_F32) return launch_many<T, DP, NW, Number<T>::kTerms, WHOLE>(a, p, stream);
    return launch_many<T, DP, NW, 2, WHOLE>(a, p, stream);
}
template <class T, int DP, bool WHOLE>
int launch_attend_w(const AttendPlan& a, const AttendParams& p, hipStream_t stream) {
    if (a.MT == 1) return launch_few<T, DP, 1, 1, WHOLE>(a, p, stream);
    if constexpr (DP <= 128)
        if (a.MT == 2) return a.own_mt == 1 ? launch_few<T, DP, 2, 1, WHOLE>(a, p, stream) : launch_few<T, DP, 2, 2, WHOLE>(a, p, stream);
    if (a.own_per_xcd > 0) {                   // the sequences' own tokens alone
        AttendParams own = p;
        own.prefix_per_xcd = 0;
        int rc;
        if constexpr (DP > 128) rc = launch_few<T, DP, 1, 1, WHOLE>(a, own, stream);
        else rc = a.own_mt == 1 ? launch_few<T, DP, 1, 1, WHOLE>(a, own, stream) : launch_few<T, DP, 2, 2, WHOLE>(a, own, stream);
        if (rc != VLUT_OK) return rc;
    }
    if constexpr (DP <= 128)
        if (a.waves == 8) return launch_many_terms<T, DP, 8, WHOLE>(a, p, stream);
    return launch_many_terms<T, DP, 4, WHOLE>(a, p, stream);
}
template <class T, int DP>
int launch_attend_d(const AttendPlan& a, const AttendParams& p, hipStream_t stream) {
    const int rc = p.D == DP ? launch_attend_w<T, DP, true>(a, p, stream) : launch_attend_w<T, DP, false>(a, p, stream);
    if (rc != VLUT_OK || a.direct) return rc;
    return launch(combine_kernel<DP>, dim3((unsigned)a.combine_blocks), 256, 0, stream, p, a.combine_lanes_log);
}
template <class T>
int launch_attend(const AttendPlan& a, const AttendParams& p, hipStream_t stream) {
    if (a.DP == 64) return launch_attend_d<T, 64>(a, p, stream);
    if (a.DP == 128) return launch_attend_d<T, 128>(a, p, stream);
    return launch_attend_d<T, 256>(a, p, stream);
}

}  // namespace
