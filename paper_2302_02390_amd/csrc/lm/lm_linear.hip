// Tokens rounded to 8 bits with a scale each, and their product with weights held as packed 8-bit codes.
//
//   x_rk ~ s_r q_rk,  w_nk = base_nb + scale_nb c_nk  (b: the bucket of k in channel n)
//   y_rn = s_r sum_b [scale_nb D_rnb + (base_nb + 128 scale_nb) Q_rb] + bias_n
//   D_rnb = sum_{k in b} q_rk (c_nk - 128),  Q_rb = sum_{k in b} q_rk
// D and Q are whole numbers and exact: |D| <= 127 * 128 * 8192 < 2^31 by the largest bucket. c - 128 as a signed byte is c
// with its top bit flipped, so the packed codes go into the matrix instructions as they are but for one xor.
#include "lm_common.hpp"
#include "lm_linear.hpp"

namespace qsdp_lm {
namespace {

typedef int v4i __attribute__((ext_vector_type(4)));

constexpr int kTokenThreads = 256;

// s = max |x| times the rounded 1/127, q = rint(x / s) with an IEEE division in binary32; slots past k are zero.
template <class T>
__global__ __launch_bounds__(kTokenThreads) void tokens_kernel(TokenParams p) {
    __shared__ float scratch[kTokenThreads / 64];
    __shared__ int counts[kTokenThreads / 64];
    for (uint64_t row = blockIdx.x; row < p.rows; row += gridDim.x) {
        const auto* x = static_cast<const typename T::raw*>(p.x) + row * p.stride;
        int8_t* codes = p.codes + row * p.pitch;
        float most = 0.0f;
        int odd = 0;  // a NaN or an infinity
        for (uint64_t k = threadIdx.x; k < p.k; k += kTokenThreads) {
            const float a = fabsf(T::get(x[k]));
            odd |= !(a < __builtin_inff());
            most = fmaxf(most, a);
        }
        most = reduce_block<kTokenThreads>(most, Max(), scratch);
        odd = reduce_block<kTokenThreads>(odd, Max(), counts);
        const float scale = odd ? __builtin_nanf("") : most * (1.0f / 127.0f);
        for (uint32_t b = 0; b < p.buckets; ++b) {
            const uint64_t lo = (uint64_t)b * p.bucket, hi = b + 1 == p.buckets ? p.pitch : lo + p.bucket;
            int sum = 0;
            for (uint64_t k = lo + threadIdx.x; k < hi; k += kTokenThreads) {
                int q = 0;
                if (k < p.k && scale > 0.0f) q = (int)fminf(fmaxf(rintf(T::get(x[k]) / scale), -127.0f), 127.0f);
                codes[k] = (int8_t)q;
                sum += q;
            }
            sum = reduce_block<kTokenThreads>(sum, Add(), counts);
            if (threadIdx.x == 0) p.sums[row * p.buckets + b] = (float)sum;  // below 2^24: exact
        }
        if (threadIdx.x == 0) p.scale[row] = scale;
    }
}

// A wave computes 16 channels x 16 tokens: the codes of a channel and of a token come in pieces of 64, 16 bytes to a lane.
template <class O>
__global__ __launch_bounds__(64) void matmul_kernel(MatmulParams p) {
    const int lane = threadIdx.x, i = lane % 16, part = lane / 16;
    const uint64_t tiles = (p.n + 15) / 16;
    const uint64_t n0 = blockIdx.x % tiles * 16, m0 = blockIdx.x / tiles * 16;
    const uint64_t wn = n0 + i < p.n ? n0 + i : p.n - 1, xm = m0 + i < p.m ? m0 + i : p.m - 1;
    const uint8_t* w = p.w + wn * p.w_pitch;
    const int8_t* x = p.x + xm * p.x_pitch;
    float acc[4] = {0.0f, 0.0f, 0.0f, 0.0f};
    for (uint32_t b = 0; b < p.buckets; ++b) {
        // 16 bytes at a time as far as there are tokens' codes: those past k are zero, whatever the weights hold there
        const uint64_t lo = (uint64_t)b * p.bucket, end = (p.k + 15) / 16 * 16, hi = lo + p.bucket < end ? lo + p.bucket : end;
        v4i d = {0, 0, 0, 0};
        for (uint64_t k = lo; k < hi; k += 64) {
            v4i wv = {0, 0, 0, 0}, xv = {0, 0, 0, 0};
            if (k + part * 16 < hi) {
                wv = *reinterpret_cast<const v4i*>(w + k + part * 16);
                wv = wv ^ (int)0x80808080;
                xv = *reinterpret_cast<const v4i*>(x + k + part * 16);
            }
            d = __builtin_amdgcn_mfma_i32_16x16x64_i8(wv, xv, d, 0, 0, 0);
        }
        const float q = p.x_sums[xm * p.buckets + b];
        for (int c = 0; c < 4; ++c) {
            const uint64_t n = n0 + part * 4 + c;
            if (n < p.n) {
                const float base = p.meta[2 * (n * p.buckets + b)], scale = p.meta[2 * (n * p.buckets + b) + 1];
                acc[c] += fmaf(scale, (float)d[c], fmaf(128.0f, scale, base) * q);
            }
        }
    }
    if (m0 + i >= p.m) return;
    const float s = p.x_scale[m0 + i];
    auto* y = static_cast<typename O::raw*>(p.y) + (m0 + i) * p.y_stride;
    for (int c = 0; c < 4; ++c) {
        const uint64_t n = n0 + part * 4 + c;
        if (n < p.n) y[n] = O::put(p.bias ? fmaf(s, acc[c], p.bias[n]) : s * acc[c]);
    }
}

}  // namespace

hipError_t launch_tokens(qsdp_dtype dtype, const TokenParams& p, hipStream_t s) {
    const dim3 grid((unsigned)(p.rows < (1u << 20) ? p.rows : (1u << 20)));
    auto kernel = dtype == QSDP_F32 ? tokens_kernel<F32> : dtype == QSDP_BF16 ? tokens_kernel<BF16> : tokens_kernel<F16>;
    hipLaunchKernelGGL(kernel, grid, dim3(kTokenThreads), 0, s, p);
    return hipGetLastError();
}

hipError_t launch_matmul(qsdp_dtype out, const MatmulParams& p, hipStream_t s) {
    const dim3 grid((unsigned)((p.n + 15) / 16 * ((p.m + 15) / 16)));
    auto kernel = out == QSDP_F32 ? matmul_kernel<F32> : out == QSDP_BF16 ? matmul_kernel<BF16> : matmul_kernel<F16>;
    hipLaunchKernelGGL(kernel, grid, dim3(64), 0, s, p);
    return hipGetLastError();
}

}  // namespace qsdp_lm
