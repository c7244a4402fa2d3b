// What the kernels of a training step share: eight elements of a row in a lane.
#pragma once
#include <type_traits>

#include "../lm/lm_common.hpp"

namespace qsdp_train {

using namespace qsdp_lm;

typedef float f32x4 __attribute__((ext_vector_type(4)));

constexpr uint64_t kMaxGrid = 1u << 20;

// Eight consecutive elements as they lie in memory: 16 bytes, or 32 of binary32.
template <class T>
struct Raw8 {
    static constexpr int WORDS = 8 / T::PER;
    u32x4 word[WORDS];

    // the `left` elements that the row has from p on, up to eight, and zeros behind them
    __device__ __forceinline__ void load(const typename T::raw* p, int left) {
        if (left >= 8) {
#pragma unroll
            for (int i = 0; i < WORDS; ++i) word[i] = load16<T>(p + i * T::PER);
        } else {
            typename T::raw e[8];
#pragma unroll
            for (int i = 0; i < 8; ++i) e[i] = i < left ? p[i] : typename T::raw(0);
            __builtin_memcpy(word, e, sizeof(e));
            again();  // packed, or all would be held one by one for the sake of these
        }
    }
    __device__ __forceinline__ void none() {
#pragma unroll
        for (int i = 0; i < WORDS; ++i) word[i] = u32x4{0, 0, 0, 0};
    }
    // Makes the compiler take what follows from the elements as new.
    __device__ __forceinline__ void again() {
#pragma unroll
        for (int i = 0; i < WORDS; ++i) asm volatile("" : "+v"(word[i]));
    }
    __device__ __forceinline__ float at(int e) const { return T::at(word[e / T::PER], e % T::PER); }
};

// Eight results rounded to the format, those past the row's end left out.
template <class T>
__device__ __forceinline__ void store8(typename T::raw* p, int left, const float* v) {
    if (left >= 8) {
#pragma unroll
        for (int i = 0; i < Raw8<T>::WORDS; ++i) store16<T>(p + i * T::PER, T::pack(v + i * T::PER));
    } else {
#pragma unroll
        for (int i = 0; i < 8; ++i)
            if (i < left) p[i] = T::put(v[i]);
    }
}

typedef uint32_t u32x2 __attribute__((ext_vector_type(2)));

// Eight codes of 8-bit floating point, to nearest even.
__device__ __forceinline__ u32x2 codes8(const float* v) {
    u32x2 c;
#pragma unroll
    for (int i = 0; i < 2; ++i) {
        int word = __builtin_amdgcn_cvt_pk_fp8_f32(v[4 * i], v[4 * i + 1], 0, false);
        word = __builtin_amdgcn_cvt_pk_fp8_f32(v[4 * i + 2], v[4 * i + 3], word, true);
        c[i] = (uint32_t)word;
    }
    return c;
}

// Over the lanes that are 16 and 32 apart.
__device__ __forceinline__ float largest_of_rows(float v) {
    uint32_t u = __builtin_bit_cast(uint32_t, v);
    const auto a = __builtin_amdgcn_permlane16_swap(u, u, false, false);
    v = fmaxf(__builtin_bit_cast(float, (uint32_t)a[0]), __builtin_bit_cast(float, (uint32_t)a[1]));
    u = __builtin_bit_cast(uint32_t, v);
    const auto b = __builtin_amdgcn_permlane32_swap(u, u, false, false);
    return fmaxf(__builtin_bit_cast(float, (uint32_t)b[0]), __builtin_bit_cast(float, (uint32_t)b[1]));
}

// Eight parameters in a format that the call names, zeros past the row's end. Asked for first and turned into numbers later, so that
// several groups are on their way together.
struct Parameters8 {
    u32x4 word[2];

    __device__ __forceinline__ void load(const void* p, qsdp_dtype dtype, int k, int left) {
        word[0] = word[1] = u32x4{0, 0, 0, 0};
        if (!p || left <= 0) return;
        if (dtype == QSDP_F32) {
            Raw8<F32> raw;
            raw.load(static_cast<const float*>(p) + k, left);
            word[0] = raw.word[0];
            word[1] = raw.word[1];
        } else {
            Raw8<BF16> raw;
            raw.load(static_cast<const uint16_t*>(p) + k, left);
            word[0] = raw.word[0];
        }
    }
    // `none` where there are none
    __device__ __forceinline__ void get(const void* p, qsdp_dtype dtype, float none, float* v) const {
#pragma unroll
        for (int e = 0; e < 8; ++e) {
            const float of_f32 = F32::at(word[e / 4], e % 4), of_bf16 = BF16::at(word[0], e), of_f16 = F16::at(word[0], e);
            v[e] = !p ? none : dtype == QSDP_F32 ? of_f32 : dtype == QSDP_BF16 ? of_bf16 : of_f16;
        }
    }
};

}  // namespace qsdp_train
