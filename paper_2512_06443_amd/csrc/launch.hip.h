// How the host sides of the translation units launch a kernel.
#pragma once

#include <atomic>

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

// More LDS than a kernel has by itself, asked for once per kernel and device.
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

}  // namespace
