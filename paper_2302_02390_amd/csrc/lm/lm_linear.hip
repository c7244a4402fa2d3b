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

constexpr uint64_t kMaxGrid = 1u << 20;

typedef int v4i __attribute__((ext_vector_type(4)));

// ---- tokens --------------------------------------------------------------------------------------------------------------
// s = max |x| times the rounded 1/127, q = rint(x / s) with an IEEE division in binary32; slots past k are zero. A workgroup
// per token, which keeps the token in registers between its maximum and its codes: eight elements to a thread at a time, of
// which the NV-th part is the last that is held; a longer token is read twice.
template <class T>
struct Eight {
    float v[8];
    // elements k ... k + 7 of n, zeros past the end
    __device__ __forceinline__ void load(const typename T::raw* x, uint64_t k, uint64_t n) {
        if (k + 8 <= n) {
            if constexpr (T::PER == 8) {
                const u32x4 p = load16<T>(x + k);
#pragma unroll
                for (int e = 0; e < 8; ++e) v[e] = T::at(p, e);
            } else {
                const u32x4 p = load16<T>(x + k), q = load16<T>(x + k + 4);
#pragma unroll
                for (int e = 0; e < 4; ++e) v[e] = T::at(p, e), v[4 + e] = T::at(q, e);
            }
        } else {
#pragma unroll
            for (int e = 0; e < 8; ++e) v[e] = k + e < n ? T::get(x[k + e]) : 0.0f;
        }
    }
};

template <class T, int THREADS, int NV>
__global__ __launch_bounds__(THREADS) void tokens_kernel(TokenParams p) {
    __shared__ float scratch[THREADS / 64];
    __shared__ int counts[THREADS / 64];
    const uint64_t row = p.first + blockIdx.x;
    const auto* x = static_cast<const typename T::raw*>(p.x) + row * p.stride;
    uint64_t* codes = reinterpret_cast<uint64_t*>(p.codes + row * p.pitch);
    const uint32_t pieces = (uint32_t)(p.pitch / 8);
    Eight<T> held[NV];
    float most = 0.0f;
    bool odd = false;  // a NaN or an infinity
    for (uint32_t first = 0; first < pieces; first += THREADS * NV) {
#pragma unroll
        for (int i = 0; i < NV; ++i) {
            const uint32_t at = first + i * THREADS + threadIdx.x;
            if (at < pieces) held[i].load(x, (uint64_t)at * 8, p.k);
            else
#pragma unroll
                for (int e = 0; e < 8; ++e) held[i].v[e] = 0.0f;
        }
#pragma unroll
        for (int i = 0; i < NV; ++i)
#pragma unroll
            for (int e = 0; e < 8; ++e) {
                const float a = fabsf(held[i].v[e]);
                odd |= !(a < __builtin_inff());
                most = fmaxf(most, a);
            }
    }
    if (__ballot(odd)) most = __builtin_inff();
    most = reduce_block<THREADS>(most, Max(), scratch);
    const float scale = most < __builtin_inff() ? most * (1.0f / 127.0f) : __builtin_nanf("");
    if (threadIdx.x == 0) p.scale[row] = scale;
    const bool some = scale > 0.0f;
    for (uint32_t b = 0; b < p.buckets; ++b) {
        const uint32_t lo = b * (p.bucket / 8), hi = b + 1 == p.buckets ? pieces : lo + p.bucket / 8;
        int sum = 0;
        for (uint32_t first = lo / (THREADS * NV) * (THREADS * NV); first < hi; first += THREADS * NV) {
#pragma unroll
            for (int i = 0; i < NV; ++i) {
                const uint32_t at = first + i * THREADS + threadIdx.x;
                if (at < lo || at >= hi) continue;
                if (pieces > THREADS * NV) held[i].load(x, (uint64_t)at * 8, p.k);
                uint32_t word[2] = {0, 0};
#pragma unroll
                for (int e = 0; e < 8; ++e) {
                    const float q = fminf(fmaxf(rintf(held[i].v[e] / scale), -127.0f), 127.0f);
                    const int c = some ? (int)q : 0;
                    sum += c;
                    word[e / 4] |= (uint32_t)(c & 0xff) << (e % 4 * 8);
                }
                codes[at] = (uint64_t)word[1] << 32 | word[0];
            }
        }
        sum = reduce_block<THREADS>(sum, Add(), counts);
        if (threadIdx.x == 0) p.sums[row * p.buckets + b] = (float)sum;  // below 2^24: exact
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

// Four consecutive elements, or the first `count` of them, wherever they start.
template <class O>
__device__ __forceinline__ void put4(typename O::raw* y, const float* v, int count) {
    if (count == 4) {
        if constexpr (sizeof(typename O::raw) == 4) {
            typedef float anywhere __attribute__((ext_vector_type(4), aligned(4)));
            *reinterpret_cast<anywhere*>(y) = anywhere{v[0], v[1], v[2], v[3]};
        } else {
            typedef uint32_t anywhere __attribute__((ext_vector_type(2), aligned(2)));
            *reinterpret_cast<anywhere*>(y) = anywhere{O::two(v[0], v[1]), O::two(v[2], v[3])};
        }
    } else {
#pragma unroll
        for (int c = 0; c < 3; ++c)
            if (c < count) y[c] = O::put(v[c]);
    }
}

// ---- tiles ----------------------------------------------------------------------------------------------------------------
// A workgroup computes TN channels x TM tokens in steps of 128 codes. Both operands' codes go straight from memory into LDS,
// two steps deep: while one is multiplied the next is on its way, and one barrier a step separates them. LDS holds rows of
// 128 bytes whose eight pieces of 16 are permuted by the row (piece c of row r in place c ^ (r % 8)), so that sixteen rows
// read the same piece from all banks; the permutation is in the addresses that the lanes read from memory. A wave multiplies
// WN channels (first operand, so that four consecutive channels of a token end up in a lane) by WM tokens.
constexpr int kStep = 128;

typedef __attribute__((address_space(1))) const void* global_ptr;
typedef __attribute__((address_space(3))) void* lds_ptr;

template <int TN, int TM, int WN, int WM>
struct Tile {
    static constexpr int WAVES = TN / WN * (TM / WM), THREADS = WAVES * 64;
    static constexpr int ROWS = TN + TM, BYTES = ROWS * kStep;      // of a step in LDS
    static constexpr int W_LOADS = TN / 8 / WAVES, X_LOADS = TM / 8 / WAVES;  // of 8 rows, for each wave
    static_assert(TN % (8 * WAVES) == 0 && TM % (8 * WAVES) == 0, "whole loads");
};

// Which tile: workgroups go to the eight dies in turn, so each die takes a contiguous run of the tiles, which walk through
// `kBand` token tiles for every channel tile and share their operands in the die's L2.
constexpr uint32_t kDies = 8, kBand = 4;

__device__ __forceinline__ void place(uint32_t id, uint32_t n_tiles, uint32_t m_tiles, uint32_t& n, uint32_t& m) {
    const uint32_t all = n_tiles * m_tiles, each = all / kDies, more = all % kDies, die = id % kDies;
    const uint32_t at = die * each + (die < more ? die : more) + id / kDies;
    const uint32_t band = at / (kBand * n_tiles), left = m_tiles - band * kBand, high = left < kBand ? left : kBand;
    const uint32_t in = at - band * kBand * n_tiles;
    n = in / high;
    m = band * kBand + in % high;
}

template <int TN, int TM, int WN, int WM, bool BUCKETS, class O>
__global__ __launch_bounds__((TN / WN) * (TM / WM) * 64, 2) void tiles_kernel(MatmulParams p, uint32_t n_tiles,
                                                                                 uint32_t m_tiles) {
    typedef Tile<TN, TM, WN, WM> S;
    __shared__ __attribute__((aligned(1024))) uint8_t lds[2][S::BYTES];
    constexpr int A = WN / 16, B = WM / 16;
    uint32_t n_tile, m_tile;
    place(blockIdx.x, n_tiles, m_tiles, n_tile, m_tile);
    const int lane = threadIdx.x % 64, wave = __builtin_amdgcn_readfirstlane((int)threadIdx.x / 64);
    const uint64_t n0 = (uint64_t)n_tile * TN, m0 = (uint64_t)m_tile * TM;
    // what the lane loads: a piece of 16 bytes of a row of eight; rows past the matrix are its last one
    const uint32_t piece = (uint32_t)((lane % 8) ^ (lane / 8)) * 16;
    uint32_t w_at[S::W_LOADS], x_at[S::X_LOADS];
#pragma unroll
    for (int i = 0; i < S::W_LOADS; ++i) {
        uint64_t row = (uint64_t)(wave * S::W_LOADS + i) * 8 + lane / 8;
        if (n0 + row >= p.n) row = p.n - 1 - n0;
        w_at[i] = (uint32_t)(row * p.w_pitch) + piece;
    }
#pragma unroll
    for (int i = 0; i < S::X_LOADS; ++i) {
        uint64_t row = (uint64_t)(wave * S::X_LOADS + i) * 8 + lane / 8;
        if (m0 + row >= p.m) row = p.m - 1 - m0;
        x_at[i] = (uint32_t)(row * p.x_pitch) + piece;
    }
    const uint8_t* w = p.w + n0 * p.w_pitch;
    const int8_t* x = p.x + m0 * p.x_pitch;
    auto fetch = [&](uint8_t* to, uint32_t k0) __attribute__((always_inline)) {
        const uint8_t* wk = w + k0;
        const int8_t* xk = x + k0;
        // a channel's codes end at a multiple of 32: pieces past that are read from its start, the tokens' codes there are zero
        const bool past = k0 + piece >= p.w_pitch;
#pragma unroll
        for (int i = 0; i < S::W_LOADS; ++i)
            __builtin_amdgcn_global_load_lds((global_ptr)(wk + (past ? w_at[i] - piece : w_at[i])),
                                             (lds_ptr)(to + (wave * S::W_LOADS + i) * 1024), 16, 0, 0);
#pragma unroll
        for (int i = 0; i < S::X_LOADS; ++i)
            __builtin_amdgcn_global_load_lds((global_ptr)(xk + x_at[i]),
                                             (lds_ptr)(to + TN * kStep + (wave * S::X_LOADS + i) * 1024), 16, 0, 0);
    };
    const int wn = wave % (TN / WN) * WN, wm = wave / (TN / WN) * WM;
    const int r = lane % 16, part = lane / 16;
    v4i d[A][B];
#pragma unroll
    for (int a = 0; a < A; ++a)
#pragma unroll
        for (int b = 0; b < B; ++b) d[a][b] = v4i{0, 0, 0, 0};
    auto multiply = [&](const uint8_t* from) __attribute__((always_inline)) {
#pragma unroll
        for (int k = 0; k < 2; ++k) {
            const int at = r * kStep + ((k * 4 + part) ^ (r % 8)) * 16;
            v4i wv[A], xv[B];
#pragma unroll
            for (int a = 0; a < A; ++a)
                wv[a] = *reinterpret_cast<const v4i*>(from + (wn + a * 16) * kStep + at) ^ (int)0x80808080;
#pragma unroll
            for (int b = 0; b < B; ++b) xv[b] = *reinterpret_cast<const v4i*>(from + (TN + wm + b * 16) * kStep + at);
#pragma unroll
            for (int a = 0; a < A; ++a)
#pragma unroll
                for (int b = 0; b < B; ++b) d[a][b] = __builtin_amdgcn_mfma_i32_16x16x64_i8(wv[a], xv[b], d[a][b], 0, 0, 0);
        }
    };
    const uint32_t steps = (uint32_t)((p.k + kStep - 1) / kStep);
    fetch(lds[0], 0);
    for (uint32_t s = 0; s < steps; ++s) {
        asm volatile("s_waitcnt vmcnt(0)" ::: "memory");
        __syncthreads();  // this step's codes are there, and the step before has been multiplied
        if (s + 1 < steps) fetch(lds[(s + 1) & 1], (s + 1) * kStep);
        multiply(lds[s & 1]);
    }
    // d[a][b][c]: channel wn + a * 16 + part * 4 + c of token wm + b * 16 + r
    const float* meta = p.meta + 2 * (n0 + wn + part * 4);
    const float* bias = p.bias ? p.bias + n0 + wn + part * 4 : nullptr;
    const int64_t left = (int64_t)(p.n - n0) - wn - part * 4;  // channels from the lane's first one on
#pragma unroll
    for (int a = 0; a < A; ++a) {
        if (left <= a * 16) continue;
        const int count = left - a * 16 < 4 ? (int)(left - a * 16) : 4;
        float step[4], centre[4], add[4];
#pragma unroll
        for (int c = 0; c < 4; ++c) {
            const int n = a * 16 + (c < count ? c : 0);
            step[c] = meta[2 * n + 1];
            centre[c] = fmaf(128.0f, step[c], meta[2 * n]);
            add[c] = bias ? bias[n] : 0.0f;
        }
#pragma unroll
        for (int b = 0; b < B; ++b) {
            const uint64_t m = m0 + wm + b * 16 + r;
            if (m >= p.m) continue;
            const float scale = p.x_scale[m], sum = p.x_sums[m];
            float v[4];
#pragma unroll
            for (int c = 0; c < 4; ++c) v[c] = fmaf(scale, fmaf(step[c], (float)d[a][b][c], centre[c] * sum), add[c]);
            put4<O>(static_cast<typename O::raw*>(p.y) + m * p.y_stride + n0 + wn + part * 4 + a * 16, v, count);
        }
    }
}

}  // namespace

template <class T>
static hipError_t launch_tokens_of(TokenParams p, hipStream_t s) {
    for (p.first = 0; p.first < p.rows; p.first += kMaxGrid) {
        const dim3 grid((unsigned)(p.rows - p.first < kMaxGrid ? p.rows - p.first : kMaxGrid));
        if (p.pitch <= 8 * 64) hipLaunchKernelGGL((tokens_kernel<T, 64, 1>), grid, dim3(64), 0, s, p);
        else if (p.pitch <= 8 * 256) hipLaunchKernelGGL((tokens_kernel<T, 256, 1>), grid, dim3(256), 0, s, p);
        else hipLaunchKernelGGL((tokens_kernel<T, 256, 4>), grid, dim3(256), 0, s, p);
        const hipError_t e = hipGetLastError();
        if (e != hipSuccess) return e;
    }
    return hipSuccess;
}

hipError_t launch_tokens(qsdp_dtype dtype, const TokenParams& p, hipStream_t s) {
    return dtype == QSDP_F32 ? launch_tokens_of<F32>(p, s) : dtype == QSDP_BF16 ? launch_tokens_of<BF16>(p, s) : launch_tokens_of<F16>(p, s);
}

template <int TN, int TM, int WN, int WM, class O>
static hipError_t launch_tiles(const MatmulParams& p, hipStream_t s) {
    const uint32_t n_tiles = (uint32_t)((p.n + TN - 1) / TN), m_tiles = (uint32_t)((p.m + TM - 1) / TM);
    hipLaunchKernelGGL((tiles_kernel<TN, TM, WN, WM, false, O>), dim3(n_tiles * m_tiles), dim3(Tile<TN, TM, WN, WM>::THREADS), 0,
                       s, p, n_tiles, m_tiles);
    return hipGetLastError();
}

hipError_t launch_matmul(qsdp_dtype out, const MatmulParams& p, hipStream_t s) {
    if (p.m > 64 && p.buckets == 1)
        return out == QSDP_F32    ? launch_tiles<256, 256, 64, 128, F32>(p, s)
               : out == QSDP_BF16 ? launch_tiles<256, 256, 64, 128, BF16>(p, s)
                                  : launch_tiles<256, 256, 64, 128, F16>(p, s);
    const dim3 grid((unsigned)((p.n + 15) / 16 * ((p.m + 15) / 16)));
    auto kernel = out == QSDP_F32 ? matmul_kernel<F32> : out == QSDP_BF16 ? matmul_kernel<BF16> : matmul_kernel<F16>;
    hipLaunchKernelGGL(kernel, grid, dim3(64), 0, s, p);
    return hipGetLastError();
}

}  // namespace qsdp_lm
