// What the kernels of a training step share: eight elements of a row in a lane.
#pragma once
#include "../lm/lm_common.hpp"

namespace qsdp_train {

using namespace qsdp_lm;

constexpr uint64_t kMaxGrid = 1u << 20;

// Eight consecutive elements as they lie in memory: 16 bytes, or 32 of binary32.
template <class T>
struct Raw8 {
    static constexpr int WORDS = 8 / T::PER;
    u32x4 word[WORDS];

    // elements k ... k + 7 of a row of n, zeros past its end
    __device__ __forceinline__ void load(const typename T::raw* row, uint64_t k, uint64_t n) {
        if (k + 8 <= n) {
#pragma unroll
            for (int i = 0; i < WORDS; ++i) word[i] = load16<T>(row + k + i * T::PER);
        } else {
            typename T::raw e[8];
#pragma unroll
            for (int i = 0; i < 8; ++i) e[i] = k + i < n ? row[k + i] : typename T::raw(0);
            __builtin_memcpy(word, e, sizeof(e));
        }
    }
    __device__ __forceinline__ void none() {
#pragma unroll
        for (int i = 0; i < WORDS; ++i) word[i] = u32x4{0, 0, 0, 0};
    }
    __device__ __forceinline__ float at(int e) const { return T::at(word[e / T::PER], e % T::PER); }
};

// Eight results rounded to the format, those past the row's end left out.
template <class T>
__device__ __forceinline__ void store8(typename T::raw* row, uint64_t k, uint64_t n, const float* v) {
    if (k + 8 <= n) {
#pragma unroll
        for (int i = 0; i < Raw8<T>::WORDS; ++i) store16<T>(row + k + i * T::PER, T::pack(v + i * T::PER));
    } else {
#pragma unroll
        for (int i = 0; i < 8; ++i)
            if (k + i < n) row[k + i] = T::put(v[i]);
    }
}

// Eight parameters (binary32, bf16 or binary16 by the call), `none` where there are none.
__device__ __forceinline__ void parameters8(const void* p, qsdp_dtype dtype, uint64_t k, uint64_t n, float none, float* v) {
    if (!p) {
#pragma unroll
        for (int e = 0; e < 8; ++e) v[e] = none;
        return;
    }
    if (dtype == QSDP_F32) {
        const float* w = static_cast<const float*>(p) + k;
#pragma unroll
        for (int e = 0; e < 8; ++e) v[e] = k + e < n ? w[e] : 0.0f;
    } else {
        const uint16_t* w = static_cast<const uint16_t*>(p) + k;
#pragma unroll
        for (int e = 0; e < 8; ++e) {
            const uint16_t raw = k + e < n ? w[e] : 0;
            v[e] = dtype == QSDP_BF16 ? BF16::get(raw) : F16::get(__builtin_bit_cast(_Float16, raw));
        }
    }
}

}  // namespace qsdp_train
