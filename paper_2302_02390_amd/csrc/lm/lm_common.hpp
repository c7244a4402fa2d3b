// What the kernels on logits and on packed weights share: element types, 16-byte pieces of rows, reductions.
#pragma once
#include <hip/hip_runtime.h>

#include <cstdint>

#include "../../../include/qsdp.h"

namespace qsdp_lm {

typedef uint32_t u32x4 __attribute__((ext_vector_type(4)));
// Rows start wherever their stride puts them: 16 bytes at the alignment of an element are one access on gfx950 all the same.
typedef uint32_t u32x4_anywhere __attribute__((ext_vector_type(4), aligned(2)));
typedef float f32x2 __attribute__((ext_vector_type(2)));

constexpr float kNegInf = -__builtin_inff();

// Elements of the three formats as the kernels read and write them; arithmetic is binary32 throughout. PER elements share
// 16 bytes; word(v, k) and pair() take and give the two (or one) that share word k of them.
struct F32 {
    typedef float raw;
    static constexpr int PER = 4;
    static constexpr uint32_t NONE = 0xff800000u;  // a word of -inf
    static __device__ __forceinline__ float get(raw v) { return v; }
    static __device__ __forceinline__ raw put(float v) { return v; }
    static __device__ __forceinline__ float at(u32x4 v, int e) { return __uint_as_float(v[e]); }
    static __device__ __forceinline__ u32x4 pack(const float* d) {
        return u32x4{__float_as_uint(d[0]), __float_as_uint(d[1]), __float_as_uint(d[2]), __float_as_uint(d[3])};
    }
};
struct BF16 {
    typedef uint16_t raw;
    typedef __bf16 pair __attribute__((ext_vector_type(2)));
    static constexpr int PER = 8;
    static constexpr uint32_t NONE = 0xff80ff80u;
    static __device__ __forceinline__ float get(raw v) { return __uint_as_float((uint32_t)v << 16); }
    static __device__ __forceinline__ uint32_t two(float a, float b) {  // to nearest even
        return __builtin_bit_cast(uint32_t, __builtin_convertvector((f32x2{a, b}), pair));
    }
    static __device__ __forceinline__ raw put(float v) { return (raw)two(v, v); }
    static __device__ __forceinline__ float at(u32x4 v, int e) {
        return __uint_as_float(e % 2 ? v[e / 2] & 0xffff0000u : v[e / 2] << 16);
    }
    static __device__ __forceinline__ u32x4 pack(const float* d) {
        return u32x4{two(d[0], d[1]), two(d[2], d[3]), two(d[4], d[5]), two(d[6], d[7])};
    }
};
struct F16 {
    typedef _Float16 raw;
    typedef _Float16 pair __attribute__((ext_vector_type(2)));
    static constexpr int PER = 8;
    static constexpr uint32_t NONE = 0xfc00fc00u;
    static __device__ __forceinline__ float get(raw v) { return (float)v; }
    static __device__ __forceinline__ raw put(float v) { return (_Float16)v; }
    static __device__ __forceinline__ uint32_t two(float a, float b) {
        return __builtin_bit_cast(uint32_t, __builtin_convertvector((f32x2{a, b}), pair));
    }
    static __device__ __forceinline__ float at(u32x4 v, int e) {
        const uint32_t word = v[e / 2];
        return (float)__builtin_bit_cast(pair, word)[e % 2];
    }
    static __device__ __forceinline__ u32x4 pack(const float* d) {
        return u32x4{two(d[0], d[1]), two(d[2], d[3]), two(d[4], d[5]), two(d[6], d[7])};
    }
};

template <class T>
__device__ __forceinline__ u32x4 load16(const typename T::raw* p) {
    return __builtin_nontemporal_load(reinterpret_cast<const u32x4_anywhere*>(p));
}
template <class T>
__device__ __forceinline__ void store16(typename T::raw* p, u32x4 v) {
    __builtin_nontemporal_store(v, reinterpret_cast<u32x4_anywhere*>(p));
}
// Elements [from, to) of 16 bytes, the others -inf; and back.
template <class T>
__device__ __forceinline__ u32x4 load_part(const typename T::raw* p, int from, int to) {
    typename T::raw e[T::PER];
    u32x4 v = {T::NONE, T::NONE, T::NONE, T::NONE};
    __builtin_memcpy(e, &v, 16);
#pragma unroll
    for (int k = 0; k < T::PER; ++k)
        if (k >= from && k < to) e[k] = p[k];
    __builtin_memcpy(&v, e, 16);
    return v;
}
template <class T>
__device__ __forceinline__ void store_part(typename T::raw* p, u32x4 v, int from, int to) {
    typename T::raw e[T::PER];
    __builtin_memcpy(e, &v, 16);
#pragma unroll
    for (int k = 0; k < T::PER; ++k)
        if (k >= from && k < to) p[k] = e[k];
}

// ---- reductions -------------------------------------------------------------------------------------------------------
struct Add {
    template <class T>
    __device__ __forceinline__ T operator()(T a, T b) const { return a + b; }
};
struct Max {
    __device__ __forceinline__ float operator()(float a, float b) const { return fmaxf(a, b); }
    __device__ __forceinline__ uint32_t operator()(uint32_t a, uint32_t b) const { return a > b ? a : b; }
    __device__ __forceinline__ int operator()(int a, int b) const { return a > b ? a : b; }
};

template <int CTRL, class T>
__device__ __forceinline__ T dpp(T v) {
    return __builtin_bit_cast(T, __builtin_amdgcn_update_dpp(0, __builtin_bit_cast(int, v), CTRL, 0xf, 0xf, false));
}
// Over each quad, each row of 16 lanes, the wave: every lane gets the result. Additions pair up in a fixed order.
template <class T, class Op>
__device__ __forceinline__ T reduce4(T v, Op op) {
    v = op(v, dpp<0xB1>(v));  // lanes 1 0 3 2
    return op(v, dpp<0x4E>(v));  // lanes 2 3 0 1
}
template <class T, class Op>
__device__ __forceinline__ T reduce16(T v, Op op) {
    v = reduce4(v, op);
    v = op(v, dpp<0x141>(v));  // mirrored within eight
    return op(v, dpp<0x140>(v));  // mirrored within sixteen
}
template <class T, class Op>
__device__ __forceinline__ T reduce64(T v, Op op) {
    v = reduce16(v, op);
    const uint32_t u = __builtin_bit_cast(uint32_t, v);
    const auto rows = __builtin_amdgcn_permlane16_swap(u, u, false, false);
    v = op(__builtin_bit_cast(T, (uint32_t)rows[0]), __builtin_bit_cast(T, (uint32_t)rows[1]));
    const uint32_t w = __builtin_bit_cast(uint32_t, v);
    const auto halves = __builtin_amdgcn_permlane32_swap(w, w, false, false);
    return op(__builtin_bit_cast(T, (uint32_t)halves[0]), __builtin_bit_cast(T, (uint32_t)halves[1]));
}

// Over a workgroup: every thread gets the result. scratch: a word for each wave.
template <int THREADS, class T, class Op>
__device__ __forceinline__ T reduce_block(T v, Op op, T* scratch) {
    v = reduce64(v, op);
    if constexpr (THREADS > 64) {
        __syncthreads();  // the scratch of the reduction before this one has been read
        if (threadIdx.x % 64 == 0) scratch[threadIdx.x / 64] = v;
        __syncthreads();
        v = scratch[0];
#pragma unroll
        for (int w = 1; w < THREADS / 64; ++w) v = op(v, scratch[w]);
    }
    return v;
}

// The thread's wave as a number that is the same for all its lanes, so that what depends on it is scalar.
__device__ __forceinline__ int wave_index() { return __builtin_amdgcn_readfirstlane((int)threadIdx.x / 64); }

}  // namespace qsdp_lm
