// What the attention's kernels share: the matrix instructions on either type of a cache, rows of features, and the compiler's order of things.
// Part of the translation units attention_bf16.hip, attention_f16.hip, chunk_bf16.hip, chunk_bf16_f32.hip, chunk_f16.hip and chunk_f16_f32.hip.
#pragma once

namespace {

typedef float f32x2 __attribute__((ext_vector_type(2)));
typedef float f32x4 __attribute__((ext_vector_type(4)));
typedef float f32x16 __attribute__((ext_vector_type(16)));
typedef short s16x4 __attribute__((ext_vector_type(4)));
typedef i32x4 dword_aligned_i32x4 __attribute__((aligned(4)));     // rows may start at any dword
typedef float dword_aligned_f32x4 __attribute__((ext_vector_type(4), aligned(4)));
typedef __attribute__((address_space(3))) s16x4 lds_s16x4;

template <class T>
struct Number;
template <>
struct Number<__bf16> {
    typedef __bf16 x8 __attribute__((ext_vector_type(8)));
    static constexpr unsigned kExponents = 0x7f807f80u, kNan = 0x7fc07fc0u;
    static constexpr bool kWide = true;               // weights may be as large as fp32's
    static constexpr float kLift = 0.0f;
    static constexpr int kTerms = 3;                  // that carry 24 bits
};
template <>
struct Number<_Float16> {
    typedef _Float16 x8 __attribute__((ext_vector_type(8)));
    static constexpr unsigned kExponents = 0x7c007c00u, kNan = 0x7e007e00u;
    static constexpr bool kWide = false;
    static constexpr float kLift = 14.0f;             // weights are up to 2^14, so that those of 2^-38 of the largest are no zeros yet (less where the largest is not known)
    static constexpr int kTerms = 2;
};
#if defined(__HIP_DEVICE_COMPILE__)
__device__ __forceinline__ f32x4 mfma16(Number<__bf16>::x8 a, Number<__bf16>::x8 b, f32x4 c) { return __builtin_amdgcn_mfma_f32_16x16x32_bf16(a, b, c, 0, 0, 0); }
__device__ __forceinline__ f32x4 mfma16(Number<_Float16>::x8 a, Number<_Float16>::x8 b, f32x4 c) { return __builtin_amdgcn_mfma_f32_16x16x32_f16(a, b, c, 0, 0, 0); }
__device__ __forceinline__ f32x16 mfma32(Number<__bf16>::x8 a, Number<__bf16>::x8 b, f32x16 c) { return __builtin_amdgcn_mfma_f32_32x32x16_bf16(a, b, c, 0, 0, 0); }
__device__ __forceinline__ f32x16 mfma32(Number<_Float16>::x8 a, Number<_Float16>::x8 b, f32x16 c) { return __builtin_amdgcn_mfma_f32_32x32x16_f16(a, b, c, 0, 0, 0); }
__device__ __forceinline__ s16x4 lds_read_transposed(unsigned at) { return __builtin_amdgcn_ds_read_tr16_b64_v4i16((lds_s16x4*)at); }
__device__ __forceinline__ float exp2_fast(float x) { return __builtin_amdgcn_exp2f(x); }
#else
template <class A> inline __device__ f32x4 mfma16(A, A, f32x4 c) { return c; }
template <class A> inline __device__ f32x16 mfma32(A, A, f32x16 c) { return c; }
inline __device__ s16x4 lds_read_transposed(unsigned) { return s16x4{}; }
inline __device__ float exp2_fast(float x) { return x; }
#endif

// Eight features of a row from feature 8 * chunk on, zeros past D (D >= 8 and a multiple of four).  Nothing past the row is read: a chunk
// that D ends in is read four features earlier and moved.
template <bool WHOLE>
__device__ __forceinline__ int chunk_at(int chunk, int D) { return WHOLE ? 8 * chunk : (8 * chunk >= D ? 0 : min(8 * chunk, D - 8)); }
template <bool WHOLE>
__device__ __forceinline__ i32x4 chunk_moved(i32x4 x, int chunk, int D) {
    if constexpr (WHOLE) return x;
    const int left = D - 8 * chunk;
    if (left >= 8) return x;
    return left <= 0 ? i32x4{0, 0, 0, 0} : i32x4{x.z, x.w, 0, 0};
}

__device__ __forceinline__ float lse_of(float m, float l) { return l == 0.0f ? -__builtin_inff() : (m + __builtin_amdgcn_logf(l)) * 0.69314718055994531f; }

// The compiler waits for what it loaded ahead of a loop again in every turn of it, and so for the loads of that turn: `x` is there from here on.
template <class V>
__device__ __forceinline__ void arrived(V& x) {
#if defined(__HIP_DEVICE_COMPILE__)
    i32x4 y = __builtin_bit_cast(i32x4, x);
    asm volatile("" : "+v"(y));
    x = __builtin_bit_cast(V, y);
#endif
}

__device__ __forceinline__ void arrived_scalar(int& x) {
#if defined(__HIP_DEVICE_COMPILE__)
    asm volatile("" : "+s"(x));
#endif
}
__device__ __forceinline__ int there(int x) {                      // (a number that all lanes have)
    x = __builtin_amdgcn_readfirstlane(x);
    arrived_scalar(x);
    return x;
}

// The order of a stretch of code that ends here: AHEAD reads of LDS in front, then, GROUPS times, MFMAS matrix instructions, READS reads, VALU vector
// instructions and EXPS exponentials.  Left to itself the compiler reads what an instruction needs right before it and waits, or all that is needed
// far ahead, in registers that others want.
template <int GROUPS, int MFMAS, int READS, int AHEAD, int VALU, int EXPS>
__device__ __forceinline__ void in_turn() {
#if defined(__HIP_DEVICE_COMPILE__)
    if constexpr (AHEAD > 0) __builtin_amdgcn_sched_group_barrier(0x100, AHEAD, 0);
#pragma unroll
    for (int i = 0; i < GROUPS; ++i) {
        __builtin_amdgcn_sched_group_barrier(0x8, MFMAS, 0);
        __builtin_amdgcn_sched_group_barrier(0x100, READS, 0);
        if constexpr (VALU > 0) __builtin_amdgcn_sched_group_barrier(0x2, VALU, 0);
        if constexpr (EXPS > 0) __builtin_amdgcn_sched_group_barrier(0x400, EXPS, 0);
    }
#endif
}

// An infinity or NaN: a number, either of two.
template <class T>
__device__ __forceinline__ bool has_odd(unsigned x) {
    constexpr unsigned high = Number<T>::kExponents & 0xffff0000u, low = Number<T>::kExponents & 0xffffu;
    return ((x & high) == high) | ((x & low) == low);
}
__device__ __forceinline__ bool is_odd(float x) { return !(fabsf(x) < __builtin_inff()); }

}  // namespace
