// An AdamW step over many tensors at once, moments in 32 bits or in 8.
//
//   m' = beta1 m + (1 - beta1) g, v' = beta2 v + (1 - beta2) g^2, x' = x - lr (m' / bias1 / (sqrt(v' / bias2) + eps) + decay x)
// In 8 bits a block of 256 elements shares its largest |m| and largest sqrt v, M and R:
//   m = M c |c| / 127^2, sqrt v = R c^2 / 255^2
// The squares give small values small steps: 2 / c of the value, 1.6 % (m) and 0.8 % (sqrt v) at the top, and reach down to 2^-14 and
// 2^-16 of the largest. A moment moves by less than half a step at a time, so rounding to the nearest code would hold it where it
// is: it goes to one of its two neighbours, upwards with the probability that makes the mean right. The draw is shared: one
// Philox block per 256 elements gives a word for m and one for v, element i adds i times the golden ratio, so the thresholds
// of a block are spread evenly and each is uniform. They are odd multiples of 2^-13, never 0 or 1: what lies within rounding of
// a code goes to that code, whichever of its neighbours the approximate square root names first. A positive v never gets code
// 0: its quotient with an m that has not vanished would be eps's.
#include "../qsdp_device.hpp"
#include "train_adamw.hpp"
#include "train_common.hpp"

namespace qsdp_train {
namespace {

constexpr float kMostM = 127.0f * 127.0f, kMostV = 255.0f * 255.0f;
constexpr float kLeast = 0x1p-96f;  // a block whose largest value is below is kept as zeros

struct Step {
    float lr, beta1, beta2, rest1, rest2, eps, inverse1, inverse2, decay;

    // the new m and v, in the order of operations of qsdp_fused_adamw_step
    __device__ __forceinline__ void moments(float g, float& m, float& v) const {
        m = fmaf(beta1, m, rest1 * g);
        v = fmaf(beta2, v, (rest2 * g) * g);
    }
    __device__ __forceinline__ float weight(float x, float m, float root) const {
        const float u = (m * inverse1) / fmaf(root, inverse2, eps);
        return fmaf(-lr, fmaf(decay, x, u), x);
    }
};

typedef uint32_t u32x2 __attribute__((ext_vector_type(2)));

// Over the 32 lanes that share a block: all get the largest.
__device__ __forceinline__ float largest32(float v) {
    v = reduce16(v, Max());
    const uint32_t u = __builtin_bit_cast(uint32_t, v);
    const auto rows = __builtin_amdgcn_permlane16_swap(u, u, false, false);
    return fmaxf(__builtin_bit_cast(float, (uint32_t)rows[0]), __builtin_bit_cast(float, (uint32_t)rows[1]));
}

// The code of a value that is not negative, `scaled` in units of the code's square; word: the upper 12 bits are the threshold.
__device__ __forceinline__ float code_of(float scaled, uint32_t word, float most) {
    const float c = floorf(__builtin_amdgcn_sqrtf(scaled));
    const float t = fmaf((float)(word >> 20), 0x1p-12f, 0x1p-13f);
    const float up = scaled - c * c > fmaf(2.0f, c, 1.0f) * t ? c + 1.0f : c;
    return fminf(up, most);
}

__device__ __forceinline__ void gradients(const qsdp_adamw_tensor& t, uint64_t at, uint64_t n, float* g) {
    if (t.g_dtype == QSDP_F32) {
        Raw8<F32> raw;
        raw.load(static_cast<const float*>(t.g), at, n);
#pragma unroll
        for (int e = 0; e < 8; ++e) g[e] = raw.at(e);
    } else if (t.g_dtype == QSDP_BF16) {
        Raw8<BF16> raw;
        raw.load(static_cast<const uint16_t*>(t.g), at, n);
#pragma unroll
        for (int e = 0; e < 8; ++e) g[e] = raw.at(e);
    } else {
        Raw8<F16> raw;
        raw.load(static_cast<const _Float16*>(t.g), at, n);
#pragma unroll
        for (int e = 0; e < 8; ++e) g[e] = raw.at(e);
    }
}

__device__ __forceinline__ void floats(const void* p, uint64_t at, uint64_t n, float* v) {
    Raw8<F32> raw;
    raw.load(static_cast<const float*>(p), at, n);
#pragma unroll
    for (int e = 0; e < 8; ++e) v[e] = raw.at(e);
}

__device__ __forceinline__ void put_weights(const qsdp_adamw_tensor& t, uint64_t at, const float* x) {
    store8<F32>(t.x, at, t.n, x);
    if (t.x16) {
        if (t.x16_dtype == QSDP_BF16) store8<BF16>(static_cast<uint16_t*>(t.x16), at, t.n, x);
        else store8<F16>(static_cast<_Float16*>(t.x16), at, t.n, x);
    }
}

// Eight codes, those past the tensor's end zero and left as they are.
__device__ __forceinline__ u32x2 load_codes(const uint8_t* p, uint64_t at, uint64_t n) {
    if (at + 8 <= n) return __builtin_nontemporal_load(reinterpret_cast<const u32x2*>(p + at));
    u32x2 v = {0, 0};
#pragma unroll
    for (int e = 0; e < 8; ++e)
        if (at + e < n) v[e / 4] |= (uint32_t)p[at + e] << (e % 4 * 8);
    return v;
}
__device__ __forceinline__ void store_codes(uint8_t* p, uint64_t at, uint64_t n, u32x2 v) {
    if (at + 8 <= n) {
        __builtin_nontemporal_store(v, reinterpret_cast<u32x2*>(p + at));
    } else {
#pragma unroll
        for (int e = 0; e < 8; ++e)
            if (at + e < n) p[at + e] = (uint8_t)(v[e / 4] >> (e % 4 * 8));
    }
}

__global__ __launch_bounds__(256) void adamw_kernel(AdamWParams p) {
    const uint64_t piece = p.first + blockIdx.x;
    const int lane = threadIdx.x % 64;
    // The tensor of this piece: the last whose first piece is not behind it. 64 tensors are looked at together.
    uint32_t low = 0, high = p.count;
    while (high - low > 1) {
        const uint32_t step = (high - low + 63) / 64, at = low + lane * step;
        const bool before = at < high && p.table[at].first <= piece;
        const uint32_t passed = (uint32_t)__popcll(__ballot(before));  // the first one is always before it
        low += (passed - 1) * step;
        high = low + step < high ? low + step : high;
    }
    const qsdp_adamw_tensor t = p.table[__builtin_amdgcn_readfirstlane(low)];
    Step s;
    float bias1 = p.bias1, bias2 = p.bias2, scale = 1.0f;
    s.lr = p.lr;
    if (p.schedule) {
        s.lr = p.schedule[0];
        bias1 = p.schedule[1];
        bias2 = p.schedule[2];
    }
    if (p.grad_scale) {
        scale = *p.grad_scale;
        if (!(fabsf(scale) < __builtin_inff())) return;
    }
    s.lr *= t.lr_scale;
    s.beta1 = p.beta1;
    s.beta2 = p.beta2;
    s.rest1 = 1.0f - p.beta1;
    s.rest2 = 1.0f - p.beta2;
    s.eps = p.eps;
    s.inverse1 = 1.0f / bias1;
    s.inverse2 = 1.0f / sqrtf(bias2);
    s.decay = t.weight_decay;
    const uint64_t local = piece - t.first, at = local * kPiece + threadIdx.x * 8;
    const bool some = at < t.n;
    float x[8], g[8];
    if (t.state_bits == 32) {
        if (!some) return;
        float m[8], v[8];
        floats(t.x, at, t.n, x);
        gradients(t, at, t.n, g);
        floats(t.m, at, t.n, m);
        floats(t.v, at, t.n, v);
#pragma unroll
        for (int e = 0; e < 8; ++e) {
            if (p.grad_scale) g[e] *= scale;
            s.moments(g[e], m[e], v[e]);
            x[e] = s.weight(x[e], m[e], sqrtf(v[e]));
        }
        put_weights(t, at, x);
        store8<F32>(static_cast<float*>(t.m), at, t.n, m);
        store8<F32>(static_cast<float*>(t.v), at, t.n, v);
        return;
    }
    // a wave has two blocks, whose draws are scalar
    const uint64_t pair = local * (kPiece / kBlock) + wave_index() * 2;
    const uint64_t seed = p.seed + (p.seed_increment ? *p.seed_increment : 0);
    uint32_t word[2][4];
#pragma unroll
    for (int b = 0; b < 2; ++b) {
        const uint64_t block = t.first * (kPiece / kBlock) + pair + b;
        qsdp::philox4x32_10((uint32_t)block, (uint32_t)(block >> 32), 3u, 0u, (uint32_t)seed, (uint32_t)(seed >> 32), word[b]);
    }
    if (pair * kBlock >= t.n) return;  // whole waves, as lanes that share a block meet below
    const uint64_t block = pair + (lane >= 32);
    u32x2 mc = {0, 0}, vc = {0, 0};
    float2 top = make_float2(0.0f, 0.0f);
    float2* scales = reinterpret_cast<float2*>(t.scale) + block;
    if (some) {
        floats(t.x, at, t.n, x);
        gradients(t, at, t.n, g);
        mc = load_codes(static_cast<const uint8_t*>(t.m), at, t.n);
        vc = load_codes(static_cast<const uint8_t*>(t.v), at, t.n);
        top = *scales;
    } else {
#pragma unroll
        for (int e = 0; e < 8; ++e) x[e] = g[e] = 0.0f;
    }
    const float m_unit = top.x * (1.0f / kMostM), v_unit = top.y * (1.0f / kMostV);
    float m[8], root[8], m_top = 0.0f, v_top = 0.0f;
#pragma unroll
    for (int e = 0; e < 8; ++e) {
        const float c = (float)(int8_t)(mc[e / 4] >> (e % 4 * 8)), d = (float)(uint8_t)(vc[e / 4] >> (e % 4 * 8));
        const float r = v_unit * (d * d);
        float v = r * r;
        m[e] = m_unit * (c * fabsf(c));
        if (p.grad_scale) g[e] *= scale;
        s.moments(g[e], m[e], v);
        root[e] = sqrtf(v);
        x[e] = s.weight(x[e], m[e], root[e]);
        m_top = fmaxf(m_top, fabsf(m[e]));
        v_top = fmaxf(v_top, root[e]);
    }
    m_top = largest32(m_top);
    v_top = largest32(v_top);
    if (!some) return;
    put_weights(t, at, x);
    m_top = m_top >= kLeast ? m_top : 0.0f;
    v_top = v_top >= kLeast ? v_top : 0.0f;
    const float m_per = m_top > 0.0f ? kMostM / m_top : 0.0f, v_per = v_top > 0.0f ? kMostV / v_top : 0.0f;
    const uint32_t in = (lane % 32) * 8;
    const uint32_t m_word = (lane < 32 ? word[0][0] : word[1][0]) + in * 0x9E3779B9u;
    const uint32_t v_word = (lane < 32 ? word[0][1] : word[1][1]) + in * 0x9E3779B9u;
    mc = vc = u32x2{0, 0};
#pragma unroll
    for (int e = 0; e < 8; ++e) {
        const float c = code_of(fabsf(m[e]) * m_per, m_word + e * 0x9E3779B9u, 127.0f);
        float d = code_of(root[e] * v_per, v_word + e * 0x9E3779B9u, 255.0f);
        if (root[e] > 0.0f && v_top > 0.0f) d = fmaxf(d, 1.0f);
        mc[e / 4] |= ((uint32_t)(int)copysignf(c, m[e]) & 0xffu) << (e % 4 * 8);
        vc[e / 4] |= (uint32_t)d << (e % 4 * 8);
    }
    store_codes(static_cast<uint8_t*>(t.m), at, t.n, mc);
    store_codes(static_cast<uint8_t*>(t.v), at, t.n, vc);
    if (lane % 32 == 0) *scales = make_float2(m_top, v_top);
}

}  // namespace

hipError_t launch_adamw(AdamWParams p, uint64_t pieces, hipStream_t s) {
    for (p.first = 0; p.first < pieces; p.first += kMaxGrid) {
        const uint64_t left = pieces - p.first;
        hipLaunchKernelGGL(adamw_kernel, dim3((unsigned)(left < kMaxGrid ? left : kMaxGrid)), dim3(256), 0, s, p);
        const hipError_t e = hipGetLastError();
        if (e != hipSuccess) return e;
    }
    return hipSuccess;
}

}  // namespace qsdp_train
