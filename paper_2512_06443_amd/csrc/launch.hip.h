// How the host side of both translation units launches a kernel.
#pragma once

namespace {

// A launch by the runtime's call itself: <<< >>> (hipLaunchKernelGGL) hands the same arguments over through a thread's stack of
// configurations first, 2.35 us of the host against 2.15.
template <class T>
struct AsIs { using type = T; };
template <class... Args>
int launch(void (*kfn)(Args...), dim3 grid, int threads, int lds, hipStream_t stream, typename AsIs<Args>::type... args) {
    void* list[] = {(void*)&args...};
    if (hipLaunchKernel((const void*)kfn, grid, dim3((unsigned)threads), list, (size_t)lds, stream) == hipSuccess) return VLUT_OK;
    (void)hipGetLastError();                     // (reported here: not once more to whoever asks next)
    return VLUT_ERR_DEVICE;
}

}  // namespace
