// Kernels on rows of logits: log probabilities with entropy and top alternatives, their gradient, and distillation from a
// teacher's top logits. One workgroup per row.
#include "lm_common.hpp"
#include "lm_rows.hpp"

namespace qsdp_lm {
namespace {

constexpr int kThreads = 256;
constexpr float kLog2e = 1.44269504088896341f;
constexpr float kLn2 = 0.69314718055994531f;
// Where exp2 has long been 0: keeps 0 * (-inf) out of the sums.
constexpr float kLeast = -400.0f;

// A row's maximum m (0 where nothing is finite, so that differences stay -inf), and its sums of 2^a and a 2^a,
// a = (z - m) log2(e) / temperature.
struct RowSums {
    float m, total, mean;
    bool empty;
};

template <class T, bool MEAN>
__device__ RowSums row_sums(const typename T::raw* z, uint64_t n, float scale2, float* scratch) {
    RowSums r;
    float m = kNegInf;
    for (uint64_t j = threadIdx.x; j < n; j += kThreads) m = fmaxf(m, T::get(z[j]));
    m = reduce_block<kThreads>(m, Max(), scratch);
    const float at = m == kNegInf ? 0.0f : m;
    float total = 0.0f, mean = 0.0f;
    for (uint64_t j = threadIdx.x; j < n; j += kThreads) {
        const float a = (T::get(z[j]) - at) * scale2;
        const float e = exp2f(a);
        total += e;
        if (MEAN) mean += e * fmaxf(a, kLeast);
    }
    r.total = reduce_block<kThreads>(total, Add(), scratch);
    r.mean = MEAN ? reduce_block<kThreads>(mean, Add(), scratch) : 0.0f;
    r.m = m;
    r.empty = r.total == 0.0f;
    return r;
}

// Order of the alternatives: value downwards (a NaN above all), then index upwards; larger keys first.
__device__ __forceinline__ uint64_t order_key(float z, uint32_t index) {
    const uint32_t u = __float_as_uint(z + 0.0f);
    const uint32_t key = z != z ? 0xFFFFFFFFu : (u >> 31) ? ~u : u | 0x80000000u;
    return (uint64_t)key << 32 | (0xFFFFFFFFu - index);
}
__device__ __forceinline__ uint32_t key_index(uint64_t key) { return 0xFFFFFFFFu - (uint32_t)key; }

template <class T>
__device__ void score_row(const ScoreParams& p, uint64_t row) {
    __shared__ float scratch[kThreads / 64];
    __shared__ uint64_t keys[128];
    __shared__ int counts[kThreads / 64];
    __shared__ int found;
    const uint64_t n = p.in.vocab;
    const auto* z = static_cast<const typename T::raw*>(p.in.logits) + row * p.in.stride;
    const float scale2 = p.in.inv_temperature * kLog2e;
    const RowSums r = row_sums<T, true>(z, n, scale2, scratch);
    const float log2_total = log2f(r.total);
    if (threadIdx.x == 0) {
        if (p.logprob) {
            const int64_t t = p.tokens[row];
            float v = 0.0f;
            if (t >= 0) v = r.empty ? kNegInf : __builtin_nanf("");
            if (t >= 0 && (uint64_t)t < n && !r.empty) v = (T::get(z[t]) - r.m) * p.in.inv_temperature - log2_total * kLn2;
            p.logprob[row] = v;
        }
        if (p.entropy) p.entropy[row] = r.empty ? 0.0f : (log2_total - r.mean / r.total) * kLn2;
        if (p.stats) {
            p.stats[2 * row] = r.m;
            p.stats[2 * row + 1] = log2_total * kLn2;
        }
    }
    if (p.top == 0) return;
    // the key of the last alternative, bit by bit: the largest that at least `top` keys reach
    uint64_t least = 0;
    for (int bit = 63; bit >= 0; --bit) {
        const uint64_t trial = least | 1ull << bit;
        int count = 0;
        for (uint64_t j = threadIdx.x; j < n; j += kThreads) count += order_key(T::get(z[j]), (uint32_t)j) >= trial;
        if (reduce_block<kThreads>(count, Add(), counts) >= p.top) least = trial;
    }
    if (threadIdx.x == 0) found = 0;
    __syncthreads();
    for (uint64_t j = threadIdx.x; j < n; j += kThreads) {
        const uint64_t key = order_key(T::get(z[j]), (uint32_t)j);
        if (key >= least) keys[atomicAdd(&found, 1)] = key;
    }
    __syncthreads();
    for (int i = threadIdx.x; i < p.top; i += kThreads) {
        int rank = 0;
        for (int o = 0; o < p.top; ++o) rank += keys[o] > keys[i];
        const uint32_t j = key_index(keys[i]);
        p.top_index[row * p.top + rank] = (int32_t)j;
        p.top_logprob[row * p.top + rank] = 
            r.empty ? kNegInf : (T::get(z[j]) - r.m) * p.in.inv_temperature - log2_total * kLn2;
    }
}

// d z_j = (g ([j = i] - p_j) - h p_j (log p_j + entropy)) / temperature
template <class T>
__device__ void score_backward_row(const ScoreBackwardParams& p, uint64_t row) {
    const uint64_t n = p.in.vocab;
    const auto* z = static_cast<const typename T::raw*>(p.in.logits) + row * p.in.stride;
    auto* dz = static_cast<typename T::raw*>(p.d_logits) + row * p.d_stride;
    const float m = p.stats[2 * row], log_total = p.stats[2 * row + 1];
    const bool empty = log_total == kNegInf;
    const float scale2 = p.in.inv_temperature * kLog2e, log2_total = log_total * kLog2e;
    int64_t token = p.tokens ? p.tokens[row] : -1;
    if ((uint64_t)token >= n) token = -1;
    const float g = p.d_logprob && token >= 0 ? p.d_logprob[row] * p.in.inv_temperature : 0.0f;
    const float h = p.d_entropy ? p.d_entropy[row] * p.in.inv_temperature : 0.0f;
    const float entropy = p.d_entropy ? p.entropy[row] : 0.0f;
    for (uint64_t j = threadIdx.x; j < n; j += kThreads) {
        const float a = (T::get(z[j]) - m) * scale2 - log2_total;
        const float prob = exp2f(a);
        const float d = -prob * (g + h * (fmaxf(a, kLeast) * kLn2 + entropy)) + ((int64_t)j == token ? g : 0.0f);
        dz[j] = T::put(empty ? 0.0f : d);
    }
}

// The teacher's list of a row: its softmax, the places that count, and the student's logits there.
struct List {
    float p[128], z[128];
    int32_t index[128];
};

template <class T>
__device__ void distill_row(const DistillParams& p, uint64_t row) {
    __shared__ float scratch[kThreads / 64];
    __shared__ List list;
    const uint64_t n = p.in.vocab;
    const auto* z = static_cast<const typename T::raw*>(p.in.logits) + row * p.in.stride;
    const float scale2 = p.in.inv_temperature * kLog2e;
    // teacher: softmax over the slots that are there
    const int k = (int)threadIdx.x;
    int32_t index = -1;
    float u = kNegInf;
    if (k < p.top) {
        index = p.teacher_index[row * p.top + k];
        if (index < 0 || (uint64_t)index >= n) index = -1;
        if (index >= 0) u = p.teacher_logit[row * p.top + k];
    }
    const float um = reduce_block<kThreads>(u, Max(), scratch);
    const float ua = (u - (um == kNegInf ? 0.0f : um)) * scale2;
    const float e = index >= 0 ? exp2f(ua) : 0.0f;
    const float mass = reduce_block<kThreads>(e, Add(), scratch);
    const bool taught = mass != 0.0f;  // a NaN counts as taught
    const float prob = taught ? e / mass : 0.0f;
    const float log2_p = ua - log2f(mass);
    if (k < p.top) {
        list.p[k] = prob;
        list.index[k] = index;
        list.z[k] = index >= 0 ? T::get(z[index]) : 0.0f;
    }
    int64_t label = p.labels && p.alpha < 1.0f ? p.labels[row] : -1;
    const bool bad_label = label >= 0 && (uint64_t)label >= n;
    if (bad_label) label = -1;
    // student
    float m, soft2, hard2;  // maximum, log2 of the sums at the temperature and at 1
    if (p.loss) {
        const RowSums s = row_sums<T, false>(z, n, scale2, scratch);
        const RowSums o = row_sums<T, false>(z, n, kLog2e, scratch);
        m = s.m, soft2 = log2f(s.total), hard2 = log2f(o.total);
        if (p.stats && k == 0) {
            p.stats[3 * row] = m;
            p.stats[3 * row + 1] = soft2 * kLn2;
            p.stats[3 * row + 2] = hard2 * kLn2;
        }
        const bool empty = soft2 == kNegInf;
        float kl = 0.0f;
        if (prob > 0.0f || prob != prob) {
            const float log2_q = empty ? kNegInf : (list.z[k] - m) * scale2 - soft2;
            kl = prob * (log2_p - log2_q);
        }
        kl = reduce_block<kThreads>(kl, Add(), scratch) * kLn2;
        if (k == 0) {
            float loss = p.alpha > 0.0f ? p.alpha * p.temperature * p.temperature * kl : 0.0f;
            if (label >= 0)
                loss -= (1.0f - p.alpha) * (empty ? kNegInf : ((T::get(z[label]) - m) * kLog2e - hard2) * kLn2);
            p.loss[row] = bad_label ? __builtin_nanf("") : loss;
        }
    } else {
        m = p.stats[3 * row], soft2 = p.stats[3 * row + 1] * kLog2e, hard2 = p.stats[3 * row + 2] * kLog2e;
    }
    if (!p.d_logits) return;
    const float* scales = p.loss ? p.row_scale : p.d_loss;
    const float g = scales ? scales[row] : 1.0f;
    const float soft = taught ? g * p.alpha * p.temperature : 0.0f, hard = label >= 0 ? g * (1.0f - p.alpha) : 0.0f;
    const bool empty = soft2 == kNegInf;
    auto* dz = static_cast<typename T::raw*>(p.d_logits) + row * p.d_stride;
    const float z_label = label >= 0 ? T::get(z[label]) : 0.0f;
    __syncthreads();  // everything outside the own elements has been read: the gradient may overwrite the logits
    auto grad = [&](float v) {
        float d = 0.0f;
        if (soft != 0.0f) d += soft * exp2f((v - m) * scale2 - soft2);
        if (hard != 0.0f) d += hard * exp2f((v - m) * kLog2e - hard2);
        return d;
    };
    for (uint64_t j = threadIdx.x; j < n; j += kThreads) dz[j] = T::put(empty ? 0.0f : grad(T::get(z[j])));
    if (empty) return;
    __syncthreads();
    // the places of the list, once more with their targets; slots of the same index write the same value
    auto target = [&](int32_t j) {
        float sum = 0.0f;
        for (int o = 0; o < p.top; ++o) sum += list.index[o] == j ? list.p[o] : 0.0f;
        return soft * sum + ((int64_t)j == label ? hard : 0.0f);
    };
    if (k < p.top && index >= 0) dz[index] = T::put(grad(list.z[k]) - target(index));
    if (k == 0 && label >= 0) dz[label] = T::put(grad(z_label) - target((int32_t)label));
}

// A workgroup takes every gridDim-th row.
template <class P, void (*ROW)(const P&, uint64_t)>
__global__ __launch_bounds__(kThreads) void rows_kernel(P p) {
    for (uint64_t row = blockIdx.x; row < p.in.rows; row += gridDim.x) {
        ROW(p, row);
        __syncthreads();  // the next row uses the same shared memory
    }
}

template <class P>
using Kernel = void (*)(P);

constexpr uint64_t kMaxGrid = 1u << 20;

template <class P>
hipError_t go(Kernel<P> f32, Kernel<P> bf16, Kernel<P> f16, qsdp_dtype dtype, const P& p, hipStream_t s) {
    const Kernel<P> kernel = dtype == QSDP_F32 ? f32 : dtype == QSDP_BF16 ? bf16 : f16;
    hipLaunchKernelGGL(kernel, dim3((unsigned)(p.in.rows < kMaxGrid ? p.in.rows : kMaxGrid)), dim3(kThreads), 0, s, p);
    return hipGetLastError();
}

}  // namespace

#define QSDP_LM_ROWS(P, ROW, dtype, p, s) \
    go<P>(rows_kernel<P, ROW<F32>>, rows_kernel<P, ROW<BF16>>, rows_kernel<P, ROW<F16>>, dtype, p, s)
hipError_t launch_score(qsdp_dtype dtype, const ScoreParams& p, hipStream_t s) {
    return QSDP_LM_ROWS(ScoreParams, score_row, dtype, p, s);
}
hipError_t launch_score_backward(qsdp_dtype dtype, const ScoreBackwardParams& p, hipStream_t s) {
    return QSDP_LM_ROWS(ScoreBackwardParams, score_backward_row, dtype, p, s);
}
hipError_t launch_distill(qsdp_dtype dtype, const DistillParams& p, hipStream_t s) {
    return QSDP_LM_ROWS(DistillParams, distill_row, dtype, p, s);
}
#undef QSDP_LM_ROWS

}  // namespace qsdp_lm
