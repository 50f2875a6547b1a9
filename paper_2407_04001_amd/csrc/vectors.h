// Device helpers of the layer operators: 16-byte vectors of elements that need
// no more than an element's alignment, conversions, and sums and maxima over a
// wave or a workgroup.
#pragma once

#include <hip/hip_runtime.h>

#include <cstdint>

namespace pase {

template <typename T> constexpr int kVec = 16 / sizeof(T);   // elements of one 16-byte vector

typedef uint32_t u32x4 __attribute__((ext_vector_type(4)));

// 16 bytes at any element's address: one global_load/store_dwordx4 (the
// architecture takes unaligned global addresses).
template <typename T> struct __attribute__((packed, aligned(sizeof(T)))) Unaligned16 {
    u32x4 v;
};

template <typename T> union Pack {
    u32x4 v;
    T e[kVec<T>];
};

// Elements at p .. p + n - 1 (n may be below 1 or above a vector), the rest `fill`.
template <typename T> __device__ __forceinline__ Pack<T> load_pack(const T *p, int64_t n, T fill) {
    Pack<T> r;
    if (n >= kVec<T>) {
        r.v = reinterpret_cast<const Unaligned16<T> *>(p)->v;
    } else {
#pragma unroll
        for (int j = 0; j < kVec<T>; j++) r.e[j] = j < n ? p[j] : fill;
    }
    return r;
}

template <typename T> __device__ __forceinline__ void store_pack(T *p, int64_t n, const Pack<T> &r) {
    if (n >= kVec<T>) {
        reinterpret_cast<Unaligned16<T> *>(p)->v = r.v;
    } else {
#pragma unroll
        for (int j = 0; j < kVec<T>; j++)
            if (j < n) p[j] = r.e[j];
    }
}


template <int N> __device__ __forceinline__ void wave_sum(float (&v)[N]) {
#pragma unroll
    for (int d = 32; d; d >>= 1)
#pragma unroll
        for (int i = 0; i < N; i++) v[i] += __shfl_xor(v[i], d, 64);
}

__device__ __forceinline__ float wave_max(float v) {
#pragma unroll
    for (int d = 32; d; d >>= 1) v = fmaxf(v, __shfl_xor(v, d, 64));
    return v;
}

// Sums over the WAVES waves of a workgroup, the same in every thread; `lds` holds
// N * WAVES floats and may be used again after the next barrier.
template <int WAVES, int N> __device__ __forceinline__ void group_sum(float (&v)[N], float *lds) {
    wave_sum(v);
    if (WAVES == 1) return;
    const int wave = threadIdx.x >> 6;
    if ((threadIdx.x & 63) == 0)
#pragma unroll
        for (int i = 0; i < N; i++) lds[i * WAVES + wave] = v[i];
    __syncthreads();
#pragma unroll
    for (int i = 0; i < N; i++) {
        float s = 0;
#pragma unroll
        for (int w = 0; w < WAVES; w++) s += lds[i * WAVES + w];
        v[i] = s;
    }
}

template <int WAVES> __device__ __forceinline__ float group_max(float v, float *lds) {
    v = wave_max(v);
    if (WAVES == 1) return v;
    if ((threadIdx.x & 63) == 0) lds[threadIdx.x >> 6] = v;
    __syncthreads();
    v = lds[0];
#pragma unroll
    for (int w = 1; w < WAVES; w++) v = fmaxf(v, lds[w]);
    return v;
}

// A launch holds fewer than 2^32 threads; operators with more cut their rows or tiles into several.
inline int64_t most_blocks(int threads) { return ((1ll << 32) - 1) / threads; }

template <typename F, typename... Args>
inline int launch(F *kernel, int64_t blocks, int threads, void *stream, Args... args) {
    void *ptrs[] = {(void *)&args...};
    if (blocks > most_blocks(threads)) return (int)hipErrorInvalidConfiguration;
    return (int)hipLaunchKernel(reinterpret_cast<const void *>(kernel), dim3((unsigned)blocks), dim3(threads), ptrs, 0,
                                static_cast<hipStream_t>(stream));
}

}  // namespace pase
