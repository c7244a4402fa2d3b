// What the kernels on logits and on packed weights share: element types, reductions over a workgroup.
#pragma once
#include <hip/hip_runtime.h>

#include <cstdint>

#include "../../../include/qsdp.h"

namespace qsdp_lm {

// Elements of the three formats as the kernels read and write them; arithmetic is binary32 throughout.
struct F32 {
    typedef float raw;
    static __device__ __forceinline__ float get(raw v) { return v; }
    static __device__ __forceinline__ raw put(float v) { return v; }
};
struct BF16 {
    typedef uint16_t raw;
    static __device__ __forceinline__ float get(raw v) { return __uint_as_float((uint32_t)v << 16); }
    static __device__ __forceinline__ raw put(float v) {  // to nearest even; a NaN keeps a set mantissa bit
        const uint32_t u = __float_as_uint(v);
        return (uint16_t)(v != v ? (u >> 16) | 0x40u : (u + 0x7FFFu + ((u >> 16) & 1u)) >> 16);
    }
};
struct F16 {
    typedef _Float16 raw;
    static __device__ __forceinline__ float get(raw v) { return (float)v; }
    static __device__ __forceinline__ raw put(float v) { return (_Float16)v; }
};

constexpr float kNegInf = -__builtin_inff();

// Reductions over a workgroup of THREADS threads: every thread gets the result. The sums are in a fixed order, so a call
// gives the same bits every time.
template <int THREADS, class T, class Op>
__device__ __forceinline__ T reduce_block(T v, Op op, T* scratch) {
    for (int d = 32; d; d >>= 1) v = op(v, __shfl_xor(v, d));
    if constexpr (THREADS > 64) {
        const int wave = threadIdx.x / 64;
        __syncthreads();  // the scratch of the reduction before this one has been read
        if (threadIdx.x % 64 == 0) scratch[wave] = v;
        __syncthreads();
        v = scratch[0];
        for (int w = 1; w < THREADS / 64; ++w) v = op(v, scratch[w]);
    }
    return v;
}
struct Add {
    template <class T>
    __device__ __forceinline__ T operator()(T a, T b) const { return a + b; }
};
struct Max {
    __device__ __forceinline__ float operator()(float a, float b) const { return fmaxf(a, b); }
    template <class T>
    __device__ __forceinline__ T operator()(T a, T b) const { return a > b ? a : b; }
};

}  // namespace qsdp_lm
