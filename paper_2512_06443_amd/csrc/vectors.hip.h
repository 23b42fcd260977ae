// Vectors of N numbers of a type, read and written as fp32.
#pragma once

namespace {

template <class T, int N>
using Vec = T __attribute__((ext_vector_type(N)));
template <class T, int N>
struct LoadVec {
    typedef Vec<T, N> type;
};
template <class T>
struct LoadVec<T, 1> {
    typedef T type;
};

template <class T, int N>
__device__ __forceinline__ void load_floats(float (&v)[N], const T* p) {
    typedef typename LoadVec<T, N>::type L;
    const L x = *(const L*)p;
    if constexpr (N == 1) v[0] = (float)x;
    else {
#pragma unroll
        for (int i = 0; i < N; ++i) v[i] = (float)x[i];
    }
}
template <class T, int N>
__device__ __forceinline__ void store_floats(T* p, const float (&v)[N]) {
    typedef typename LoadVec<T, N>::type L;
    L x;
    if constexpr (N == 1) x = (T)v[0];
    else {
#pragma unroll
        for (int i = 0; i < N; ++i) x[i] = (T)v[i];
    }
    *(L*)p = x;
}

// A vector as it is in memory, for loads that are on their way together.
template <class T, int VEC>
struct RawVec {
    typename LoadVec<T, VEC>::type v;
    __device__ __forceinline__ void load(const void* base, int64_t at) { v = *(const typename LoadVec<T, VEC>::type*)((const T*)base + at); }
    __device__ __forceinline__ void floats(float (&f)[VEC]) const {
        if constexpr (VEC == 1) f[0] = (float)v;
        else {
#pragma unroll
            for (int i = 0; i < VEC; ++i) f[i] = (float)v[i];
        }
    }
};

}  // namespace
