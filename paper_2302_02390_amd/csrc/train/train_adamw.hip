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
// An infinite second moment, of a finite gradient whose square overflows, is held with this R: its code 255 stands for 2^64, whose square is
// infinite again, codes up to 254 for finite squares. (With R = inf all other elements of the block would be infinite or NaN in the next step.)
constexpr float kMostRoot = 0x1p64f;

struct Step {
    float lr, beta1, beta2, rest1, rest2, eps, inverse1, inverse2, decay;

    // the new m and v, in the order of operations of qsdp_fused_adamw_step
    __device__ __forceinline__ void moments(float g, float& m, float& v) const {
        m = fmaf(beta1, m, rest1 * g);
        v = fmaf(beta2, v, (rest2 * g) * g);
    }
    // the quotient to two units in the last place, of an update that is itself small beside x
    __device__ __forceinline__ float weight(float x, float m, float root) const {
        const float u = (m * inverse1) * __builtin_amdgcn_rcpf(fmaf(root, inverse2, eps));
        return fmaf(-lr, fmaf(decay, x, u), x);
    }
};

// Four consecutive elements, zeros past the tensor's end; and back.
template <class T>
__device__ __forceinline__ void load4(const void* p, uint64_t at, uint64_t n, float* v) {
    typedef typename T::raw raw;
    typedef raw anywhere __attribute__((ext_vector_type(4), aligned(sizeof(raw))));
    const raw* from = static_cast<const raw*>(p) + at;
    if (at + 4 <= n) {
        const anywhere four = __builtin_nontemporal_load(reinterpret_cast<const anywhere*>(from));
#pragma unroll
        for (int e = 0; e < 4; ++e) v[e] = T::get(four[e]);
    } else {
#pragma unroll
        for (int e = 0; e < 4; ++e) v[e] = at + e < n ? T::get(from[e]) : 0.0f;
    }
}
template <class T>
__device__ __forceinline__ void store4(void* p, uint64_t at, uint64_t n, const float* v) {
    typedef typename T::raw raw;
    typedef raw anywhere __attribute__((ext_vector_type(4), aligned(sizeof(raw))));
    raw* to = static_cast<raw*>(p) + at;
    if (at + 4 <= n) {
        if constexpr (sizeof(raw) == 4) {
            __builtin_nontemporal_store(anywhere{v[0], v[1], v[2], v[3]}, reinterpret_cast<anywhere*>(to));
        } else {
            typedef uint32_t two __attribute__((ext_vector_type(2), aligned(2)));
            __builtin_nontemporal_store(two{T::two(v[0], v[1]), T::two(v[2], v[3])}, reinterpret_cast<two*>(to));
        }
    } else {
#pragma unroll
        for (int e = 0; e < 4; ++e)
            if (at + e < n) to[e] = T::put(v[e]);
    }
}

// The root to nearest of finite numbers from 2^-96 on, in a third of the instructions that all numbers take: Newton's step for both the
// root and half its reciprocal, and the rest of the square (Markstein).
__device__ __forceinline__ float root_of(float v) {
    const float y = __builtin_amdgcn_rsqf(v), s = v * y, h = 0.5f * y, e = fmaf(-h, s, 0.5f);
    const float s1 = fmaf(s, e, s);
    return fmaf(fmaf(-s1, s1, v), fmaf(h, e, h), s1);
}

// The code of a value that is not negative, `scaled` in units of the code's square; word: the upper 12 bits are the threshold.
__device__ __forceinline__ float code_of(float scaled, uint32_t word) {
    const float c = floorf(__builtin_amdgcn_sqrtf(scaled));
    const float t = fmaf((float)(word >> 20), 0x1p-12f, 0x1p-13f);
    return fmaf(fmaf(2.0f, c, 1.0f), -t, scaled - c * c) > 0.0f ? c + 1.0f : c;  // all exact but the last rounding, which keeps the sign
}

// The largest over the wave of four values: in the lanes of row q (of 16), that of value q. Halves and rows change places between two
// registers at a time, so that both are reduced by the same instructions.
__device__ __forceinline__ float largest_of_four(float a, float b, float c, float d) {
    auto halves = [](float u, float v) __attribute__((always_inline)) {
        const auto s = __builtin_amdgcn_permlane32_swap(__float_as_uint(u), __float_as_uint(v), false, false);
        return fmaxf(__uint_as_float(s[0]), __uint_as_float(s[1]));
    };
    const auto s = __builtin_amdgcn_permlane16_swap(__float_as_uint(halves(a, c)), __float_as_uint(halves(b, d)), false, false);
    return reduce16(fmaxf(__uint_as_float(s[0]), __uint_as_float(s[1])), Max());
}

__device__ __forceinline__ void gradients(const qsdp_adamw_tensor& t, uint64_t at, float* g) {
    if (t.g_dtype == QSDP_F32) load4<F32>(t.g, at, t.n, g);
    else if (t.g_dtype == QSDP_BF16) load4<BF16>(t.g, at, t.n, g);
    else load4<F16>(t.g, at, t.n, g);
}

__device__ __forceinline__ void put_weights(const qsdp_adamw_tensor& t, uint64_t at, const float* x) {
    store4<F32>(t.x, at, t.n, x);
    if (t.x16) {
        if (t.x16_dtype == QSDP_BF16) store4<BF16>(t.x16, at, t.n, x);
        else store4<F16>(t.x16, at, t.n, x);
    }
}

// Four codes, zeros past the tensor's end; and back, what lies behind left as it is.
__device__ __forceinline__ uint32_t load_codes(const void* p, uint64_t at, uint64_t n) {
    const uint8_t* from = static_cast<const uint8_t*>(p) + at;
    if (at + 4 <= n) return __builtin_nontemporal_load(reinterpret_cast<const uint32_t*>(from));
    uint32_t v = 0;
#pragma unroll
    for (int e = 0; e < 4; ++e)
        if (at + e < n) v |= (uint32_t)from[e] << (e * 8);
    return v;
}
__device__ __forceinline__ void store_codes(void* p, uint64_t at, uint64_t n, uint32_t v) {
    uint8_t* to = static_cast<uint8_t*>(p) + at;
    if (at + 4 <= n) {
        __builtin_nontemporal_store(v, reinterpret_cast<uint32_t*>(to));
    } else {
#pragma unroll
        for (int e = 0; e < 4; ++e)
            if (at + e < n) to[e] = (uint8_t)(v >> (e * 8));
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
    float scale = 1.0f;
    s.lr = p.lr;
    s.inverse1 = p.inverse1;
    s.inverse2 = p.inverse2;
    if (p.schedule) {
        s.lr = p.schedule[0];
        s.inverse1 = 1.0f / p.schedule[1];
        s.inverse2 = 1.0f / sqrtf(p.schedule[2]);
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
    s.decay = t.weight_decay;
    // A wave has two blocks of 256 elements, a lane four neighbours of each, so that every access of the wave is one run.
    const uint64_t block = (piece - t.first) * (kPiece / kBlock) + wave_index() * 2;
    if (block * kBlock >= t.n) return;
    const uint64_t at[2] = {block * kBlock + lane * 4, (block + 1) * kBlock + lane * 4};
    float x[2][4], g[2][4], m[2][4];
#pragma unroll
    for (int j = 0; j < 2; ++j) {
        load4<F32>(t.x, at[j], t.n, x[j]);
        gradients(t, at[j], g[j]);
        if (p.grad_scale)
#pragma unroll
            for (int e = 0; e < 4; ++e) g[j][e] *= scale;
    }
    if (t.state_bits == 32) {
        float v[2][4];
#pragma unroll
        for (int j = 0; j < 2; ++j) {
            load4<F32>(t.m, at[j], t.n, m[j]);
            load4<F32>(t.v, at[j], t.n, v[j]);
        }
#pragma unroll
        for (int j = 0; j < 2; ++j) {
#pragma unroll
            for (int e = 0; e < 4; ++e) {
                s.moments(g[j][e], m[j][e], v[j][e]);
                x[j][e] = s.weight(x[j][e], m[j][e], sqrtf(v[j][e]));
            }
            put_weights(t, at[j], x[j]);
            store4<F32>(t.m, at[j], t.n, m[j]);
            store4<F32>(t.v, at[j], t.n, v[j]);
        }
        return;
    }
    uint32_t mc[2], vc[2];
    float2 top[2];
    float2* scales = reinterpret_cast<float2*>(t.scale) + block;
#pragma unroll
    for (int j = 0; j < 2; ++j) {
        mc[j] = load_codes(t.m, at[j], t.n);
        vc[j] = load_codes(t.v, at[j], t.n);
        top[j] = (block + j) * kBlock < t.n ? scales[j] : make_float2(0.0f, 0.0f);
    }
    // the draws are scalar, a block for each
    const uint64_t seed = p.seed + (p.seed_increment ? *p.seed_increment : 0);
    float root[2][4], m_top[2], v_top[2];
#pragma unroll
    for (int j = 0; j < 2; ++j) {
        const float m_unit = top[j].x * (1.0f / kMostM), v_unit = top[j].y * (1.0f / kMostV);
        const uint32_t biased = mc[j] ^ 0x80808080u;  // as unsigned bytes about 128
        bool special = false;
#pragma unroll
        for (int e = 0; e < 4; ++e) {
            const float c = (float)(uint8_t)(biased >> (e * 8)) - 128.0f, d = (float)(uint8_t)(vc[j] >> (e * 8));
            const float r = v_unit * (d * d);
            root[j][e] = r * r;
            m[j][e] = m_unit * (c * fabsf(c));
            s.moments(g[j][e], m[j][e], root[j][e]);
            special |= !(root[j][e] >= kLeast && root[j][e] < __builtin_inff());
        }
        if (__any(special)) {
#pragma unroll
            for (int e = 0; e < 4; ++e) {
                const float exact = sqrtf(root[j][e]);
                x[j][e] = s.weight(x[j][e], m[j][e], exact);
                root[j][e] = fminf(exact, kMostRoot);
            }
        } else {
#pragma unroll
            for (int e = 0; e < 4; ++e) {
                root[j][e] = root_of(root[j][e]);
                x[j][e] = s.weight(x[j][e], m[j][e], root[j][e]);
            }
        }
        m_top[j] = fmaxf(fmaxf(fabsf(m[j][0]), fabsf(m[j][1])), fmaxf(fabsf(m[j][2]), fabsf(m[j][3])));
        v_top[j] = fmaxf(fmaxf(root[j][0], root[j][1]), fmaxf(root[j][2], root[j][3]));
        put_weights(t, at[j], x[j]);
    }
    // rows of 16 lanes: M of the first block, its R, M of the second, its R; and what their quotients with the codes' squares are
    float tops = largest_of_four(m_top[0], v_top[0], m_top[1], v_top[1]);
    tops = tops >= kLeast ? tops : 0.0f;  // (R is 0 or from 2^-75 on)
    const float per = tops > 0.0f ? (lane & 16 ? kMostV : kMostM) / tops : 0.0f;
    auto of_row = [&](float v, int row) __attribute__((always_inline)) {
        return __uint_as_float((uint32_t)__builtin_amdgcn_readlane((int)__float_as_uint(v), row * 16));
    };
#pragma unroll
    for (int j = 0; j < 2; ++j) {
        const float m_per = of_row(per, 2 * j), v_per = of_row(per, 2 * j + 1);
        const uint64_t number = t.first * (kPiece / kBlock) + block + j;
        uint32_t word[4];
        qsdp::philox4x32_10((uint32_t)number, (uint32_t)(number >> 32), 3u, 0u, (uint32_t)seed, (uint32_t)(seed >> 32), word);
        mc[j] = vc[j] = 0;
#pragma unroll
        for (int e = 0; e < 4; ++e) {
            const uint32_t golden = (lane * 4 + e) * 0x9E3779B9u;
            const float c = fminf(code_of(fabsf(m[j][e]) * m_per, word[0] + golden), 127.0f);
            // at least 1 for a root that is not 0, which is from 2^-75 on; past 255 the conversion stops
            const float d = fmaxf(code_of(root[j][e] * v_per, word[1] + golden), fminf(root[j][e] * 0x1p76f, 1.0f));
            mc[j] = __builtin_amdgcn_cvt_pk_u8_f32(copysignf(c, m[j][e]) + 128.0f, e, mc[j]);
            vc[j] = __builtin_amdgcn_cvt_pk_u8_f32(d, e, vc[j]);
        }
        store_codes(t.m, at[j], t.n, mc[j] ^ 0x80808080u);
        store_codes(t.v, at[j], t.n, vc[j]);
        if (lane == 0 && (block + j) * kBlock < t.n) scales[j] = make_float2(of_row(tops, 2 * j), of_row(tops, 2 * j + 1));
    }
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
