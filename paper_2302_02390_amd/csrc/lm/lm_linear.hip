// Tokens rounded to 8 bits with a scale each, and their product with weights held as packed 8-bit codes.
//
//   x_rk ~ s_r q_rk,  w_nk = base_nb + scale_nb c_nk  (b: the bucket of k in channel n)
//   y_rn = s_r sum_b [scale_nb D_rnb + (base_nb + 128 scale_nb) Q_rb] + bias_n
//   D_rnb = sum_{k in b} q_rk (c_nk - 128),  Q_rb = sum_{k in b} q_rk
// D and Q are whole numbers and exact: |D| <= 127 * 128 * 8192 < 2^31 by the largest bucket. c - 128 as a signed byte is c
// with its top bit flipped, so the packed codes go into the matrix instructions as they are but for one xor.
#include <type_traits>

#include "lm_common.hpp"
#include "lm_linear.hpp"
#include "lm_plan.hpp"

namespace qsdp_lm {
namespace {

constexpr uint64_t kMaxGrid = 1u << 20;

typedef int v4i __attribute__((ext_vector_type(4)));

// ---- tokens --------------------------------------------------------------------------------------------------------------
// s = max |x| times the rounded 1/127, q = rint(x / s) with an IEEE division in binary32; slots past k are zero. A workgroup
// per token, which keeps the token in registers between its maximum and its codes: eight elements to a thread at a time, of
// which the NV-th part is the last that is held; a longer token is read twice. HBM bounds it for many tokens: 8192 of 8192 bf16
// elements 45 us, 4.5 TB/s both ways. Buckets are added up one after the other, so many short ones cost (8192 in eight: 68 us).
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
    const float inv = 1.0f / scale;
    const bool some = scale > 0.0f, plain = inv < 0x1p100f && inv > 0x1p-100f;  // the product is as good as the quotient
    for (uint32_t b = 0; b < p.buckets; ++b) {
        const uint32_t lo = b * (p.bucket / 8), hi = b + 1 == p.buckets ? pieces : lo + p.bucket / 8;
        int sum = 0;
        for (uint32_t first = lo / (THREADS * NV) * (THREADS * NV); first < hi; first += THREADS * NV) {
#pragma unroll
            for (int i = 0; i < NV; ++i) {
                const uint32_t at = first + i * THREADS + threadIdx.x;
                if (at < lo || at >= hi) continue;
                if (pieces > THREADS * NV) held[i].load(x, (uint64_t)at * 8, p.k);
                // x times 1 / s is within 2^-15 of x / s: unless it is that near to a tie, both round to the same code
                float q[8], near = 1.0f;
#pragma unroll
                for (int e = 0; e < 8; ++e) {
                    const float about = held[i].v[e] * inv;
                    q[e] = rintf(about);
                    near = fminf(near, fabsf(fabsf(about - q[e]) - 0.5f));
                }
                if (!(near > 0x1p-14f) || !plain)
#pragma unroll
                    for (int e = 0; e < 8; ++e) q[e] = rintf(held[i].v[e] / scale);
                uint32_t word[2] = {0, 0};
#pragma unroll
                for (int e = 0; e < 8; ++e)  // as unsigned bytes about 128, turned into signed ones below
                    word[e / 4] = __builtin_amdgcn_cvt_pk_u8_f32(fminf(fmaxf(q[e], -127.0f), 127.0f) + 128.0f, e % 4, word[e / 4]);
                word[0] = some ? word[0] ^ 0x80808080u : 0u;
                word[1] = some ? word[1] ^ 0x80808080u : 0u;
                sum = __builtin_amdgcn_sdot4((int)word[0], 0x01010101, sum, false);
                sum = __builtin_amdgcn_sdot4((int)word[1], 0x01010101, sum, false);
                codes[at] = (uint64_t)word[1] << 32 | word[0];
            }
        }
        sum = reduce_block<THREADS>(sum, Add(), counts);
        if (threadIdx.x == 0) p.sums[row * p.buckets + b] = (float)sum;  // below 2^24: exact
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
// STAGES steps deep: while one is multiplied the next ones are on their way, and one barrier a step separates them. LDS holds rows of
// 128 bytes whose eight pieces of 16 are permuted by the row (piece c of row r in place c ^ (r % 8)), so that sixteen rows
// read the same piece from all banks; the permutation is in the addresses that the lanes read from memory. A wave multiplies
// WN channels (first operand, so that four consecutive channels of a token end up in a lane) by WM tokens. Large products: 8192^3
// 495 us, 2223 TOP/s (the library's int8 product 2202), 8192 x 2048 x 8192 117-122 us. What bounds them there is the turn of the
// steps: the matrix units are busy in 51 % of the cycles, a third of the waves' time goes to waits for loads
// and reads of LDS and to the barrier that ends each step, which two waves to a SIMD do not fill; the LDS takes their reads without
// delay (2 %) and without conflicts. The 256-wide tile spills 4 (fp32 outputs) to
// 16 registers, the 128-wide one of several buckets 2, all outside the loop over the steps. With several buckets, in 128-wide
// tiles that add their sums up at each end, 8192 x 2048 x 8192 takes 193 us in eight.
typedef __attribute__((address_space(1))) const void* global_ptr;
typedef __attribute__((address_space(3))) void* lds_ptr;

// Until at most N of the wave's loads are on their way: those into LDS are not the compiler's to wait for.
template <int N>
__device__ __forceinline__ void wait_loads() {
    static_assert(N < 64, "six bits");
    asm volatile("s_waitcnt vmcnt(%0)" ::"n"(N) : "memory");
}

// Until the wave's reads of LDS (and scalar loads) are done, in a form that the compiler counts and does not repeat.
__device__ __forceinline__ void wait_reads() {
    __builtin_amdgcn_sched_barrier(0);
    __builtin_amdgcn_s_waitcnt(0xc07f);  // lgkmcnt(0)
    __builtin_amdgcn_sched_barrier(0);
}

// The workgroup's waves meet; unlike __syncthreads, without waiting for the loads that are on their way. What a wave has
// read from LDS before is in its registers, as it has been multiplied.
__device__ __forceinline__ void meet_here() { asm volatile("s_barrier" ::: "memory"); }

// Reads of LDS (and loads from memory) go between the matrix instructions of the same stretch of code: a wave whose reads wait
// for the LDS issues nothing else, and all waves are at the same place.
template <int READS, int PRODUCTS, int LOADS, int I = 0>
__device__ __forceinline__ void interleave() {
    if constexpr (I < READS) {
        __builtin_amdgcn_sched_group_barrier(0x100, 1, 0);
        if constexpr (I < LOADS) __builtin_amdgcn_sched_group_barrier(0x010, 1, 0);
        __builtin_amdgcn_sched_group_barrier(0x008, (I + 1) * PRODUCTS / READS - I * PRODUCTS / READS, 0);
        interleave<READS, PRODUCTS, LOADS, I + 1>();
    } else {
        __builtin_amdgcn_sched_barrier(0);
    }
}

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

// GROUPS of such teams share a tile of several buckets where there are fewer tiles than compute units: each takes a run of the steps,
// and their sums meet in LDS in the order of the groups. All make the same number of steps; those past a group's run multiply by zero.
template <int TN, int TM, int WN, int WM, int STAGES, bool BUCKETS, int GROUPS, class O>
__global__ __launch_bounds__((TN / WN) * (TM / WM) * GROUPS * 64, 2) void tiles_kernel(MatmulParams p, uint32_t n_tiles,
                                                                                 uint32_t m_tiles) {
    typedef Tile<TN, TM, WN, WM> S;
    __shared__ __attribute__((aligned(1024))) uint8_t all[GROUPS][STAGES][S::BYTES];
    constexpr int A = WN / 16, B = WM / 16;
    uint32_t n_tile, m_tile;
    place(blockIdx.x, n_tiles, m_tiles, n_tile, m_tile);
    const int lane = threadIdx.x % 64, team = __builtin_amdgcn_readfirstlane((int)threadIdx.x / 64);
    const int wave = GROUPS == 1 ? team : team % S::WAVES, group = GROUPS == 1 ? 0 : team / S::WAVES;
    uint8_t(*lds)[S::BYTES] = all[group];
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
    const uint32_t total = (uint32_t)((p.k + kStep - 1) / kStep), steps = (total + GROUPS - 1) / GROUPS;
    const uint32_t begin = group * steps, mine = begin >= total ? 0 : total - begin < steps ? total - begin : steps;
    auto fetch = [&](uint8_t* to, uint32_t at) __attribute__((always_inline)) {
        const uint32_t k0 = (GROUPS == 1 || begin + at < total ? begin + at : total - 1) * kStep;
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
    // a half of a step's codes (64) for the wave's channels and tokens, and their product
    v4i wv[2][A], xv[2][B];
    auto read = [&](auto set, const uint8_t* from) __attribute__((always_inline)) {
        const int at = r * kStep + ((set * 4 + part) ^ (r % 8)) * 16;
#pragma unroll
        for (int a = 0; a < A; ++a) wv[set][a] = *reinterpret_cast<const v4i*>(from + (wn + a * 16) * kStep + at);
#pragma unroll
        for (int b = 0; b < B; ++b) xv[set][b] = *reinterpret_cast<const v4i*>(from + (TN + wm + b * 16) * kStep + at);
    };
    auto multiply = [&](auto set, uint32_t s) __attribute__((always_inline)) {
        if constexpr (GROUPS > 1) {
            const int keep = s < mine ? -1 : 0;
#pragma unroll
            for (int b = 0; b < B; ++b) xv[set][b] &= keep;
        }
#pragma unroll
        for (int a = 0; a < A; ++a) {
            const v4i signed_w = wv[set][a] ^ (int)0x80808080;
#pragma unroll
            for (int b = 0; b < B; ++b) d[a][b] = __builtin_amdgcn_mfma_i32_16x16x64_i8(signed_w, xv[set][b], d[a][b], 0, 0, 0);
        }
    };
    const std::integral_constant<int, 0> one;
    const std::integral_constant<int, 1> other;
    // d[a][b][c]: channel wn + a * 16 + part * 4 + c of token wm + b * 16 + r
    const int64_t left = (int64_t)(p.n - n0) - wn - part * 4;  // channels from the lane's first one on
    const float* meta = p.meta + 2 * p.buckets * (n0 + wn + part * 4);
    // of channels in several buckets: the sum over the buckets so far, added to at the end of each
    float sum_of[BUCKETS ? A : 1][BUCKETS ? B : 1][4];
    if constexpr (BUCKETS) {
#pragma unroll
        for (int a = 0; a < A; ++a)
#pragma unroll
            for (int b = 0; b < B; ++b)
#pragma unroll
                for (int c = 0; c < 4; ++c) sum_of[a][b][c] = 0.0f;
    }
    const uint32_t per = p.bucket / kStep;  // where there are several buckets
    uint32_t bucket = BUCKETS ? begin / per : 0, next = (bucket + 1) * per;
#pragma unroll
    for (int s = 0; s < STAGES - 1; ++s)
        if ((uint32_t)s < steps) fetch(lds[s], s);
    // Step `at` is there for all waves: its loads are done (those behind it may be on their way), and so is the reading of the
    // step before, whose place the step STAGES - 1 further takes. While a half is multiplied the next one comes out of LDS,
    // over the barrier as well: reading and multiplying would otherwise take turns, as the barrier has all waves do the same.
    constexpr int LOADS = S::W_LOADS + S::X_LOADS;
    // the bucket that ends with step s, or the part of it that ends with the group's run; the last step adds the tokens' sum
    auto fold = [&](uint32_t s) __attribute__((always_inline)) {
        if constexpr (BUCKETS) {
            const bool ends = begin + s + 1 == next || begin + s + 1 == total;
            if (GROUPS == 1 ? !ends : s >= mine || (!ends && s + 1 != mine)) return;
            float sums[B];
#pragma unroll
            for (int b = 0; b < B; ++b) {
                const uint64_t m = m0 + wm + b * 16 + r;
                sums[b] = ends ? p.x_sums[(m < p.m ? m : p.m - 1) * p.buckets + bucket] : 0.0f;
            }
#pragma unroll
            for (int a = 0; a < A; ++a)
#pragma unroll
                for (int c = 0; c < 4; ++c) {
                    const int64_t n = a * 16 + c < left ? a * 16 + c : left - 1;  // within the matrix, from the lane's first on
                    const float2 of = left > 0 ? *reinterpret_cast<const float2*>(meta + 2 * (n * p.buckets + bucket))
                                               : make_float2(0.0f, 0.0f);
                    const float centre = fmaf(128.0f, of.y, of.x);
#pragma unroll
                    for (int b = 0; b < B; ++b) {
                        sum_of[a][b][c] += fmaf(of.y, (float)d[a][b][c], centre * sums[b]);
                        d[a][b][c] = 0;
                    }
                }
            ++bucket;
            next += per;
        }
    };
    auto first_half = [&](uint32_t s) __attribute__((always_inline)) {
        wait_reads();  // ahead of the next ones: more than fifteen cannot be counted
        read(other, lds[s % STAGES]);
        multiply(one, s);
        interleave<A + B, A * B, 0>();
        wait_reads();  // the step is in registers
    };
    wait_loads<0>();
    meet_here();
    if (STAGES - 1 < steps) fetch(lds[STAGES - 1], STAGES - 1);
    wait_reads();
    read(one, lds[0]);
    uint32_t s = 0;
    for (; s + STAGES < steps; ++s) {
        first_half(s);
        wait_loads<(STAGES - 2) * LOADS>();
        meet_here();
        fetch(lds[s % STAGES], s + STAGES);
        read(one, lds[(s + 1) % STAGES]);
        multiply(other, s);
        interleave<A + B, A * B, LOADS>();
        fold(s);
    }
    for (; s + 1 < steps; ++s) {
        first_half(s);
        wait_loads<0>();
        meet_here();
        read(one, lds[(s + 1) % STAGES]);
        multiply(other, s);
        interleave<A + B, A * B, 0>();
        fold(s);
    }
    first_half(s);
    multiply(other, s);
    fold(s);
    if constexpr (GROUPS > 1) {
        static_assert(BUCKETS, "sums of whole numbers are not shared");
        static_assert((GROUPS - 1) * TN * TM * 4 <= GROUPS * STAGES * S::BYTES, "the sums of the other groups");
        v4i* meet = reinterpret_cast<v4i*>(&all[0][0][0]);
        auto place_of = [&](int g, int a, int b) { return ((g - 1) * A * B + a * B + b) * S::THREADS + wave * 64 + lane; };
        __syncthreads();
        if (group) {
#pragma unroll
            for (int a = 0; a < A; ++a)
#pragma unroll
                for (int b = 0; b < B; ++b) {
#pragma unroll
                    for (int c = 0; c < 4; ++c) d[a][b][c] = __float_as_int(sum_of[a][b][c]);
                    meet[place_of(group, a, b)] = d[a][b];
                }
        }
        __syncthreads();
        if (group) return;
#pragma unroll
        for (int g = 1; g < GROUPS; ++g)
#pragma unroll
            for (int a = 0; a < A; ++a)
#pragma unroll
                for (int b = 0; b < B; ++b) {
                    const v4i more = meet[place_of(g, a, b)];
#pragma unroll
                    for (int c = 0; c < 4; ++c) {
                        const int word = more[c];
                        sum_of[a][b][c] += __int_as_float(word);
                    }
                }
    }
    // every scale is read before the first output is written: the compiler cannot know them apart
    const float* bias = p.bias ? p.bias + n0 + wn + part * 4 : nullptr;
    float scale[B], sums[B];
#pragma unroll
    for (int b = 0; b < B; ++b) {
        const uint64_t m = m0 + wm + b * 16 + r < p.m ? m0 + wm + b * 16 + r : p.m - 1;
        scale[b] = p.x_scale[m];
        sums[b] = BUCKETS ? 0.0f : p.x_sums[m];
    }
    float step[A][4], centre[A][4], add[A][4];
#pragma unroll
    for (int a = 0; a < A; ++a)
#pragma unroll
        for (int c = 0; c < 4; ++c) {
            const int64_t n = a * 16 + c < left ? a * 16 + c : left - 1;  // as in fold
            const float2 of = BUCKETS || left <= 0 ? make_float2(0.0f, 0.0f) : *reinterpret_cast<const float2*>(meta + 2 * n);
            step[a][c] = of.y;
            centre[a][c] = fmaf(128.0f, of.y, of.x);
            add[a][c] = bias && left > 0 ? bias[n] : 0.0f;
        }
#pragma unroll
    for (int b = 0; b < B; ++b) {
        const uint64_t m = m0 + wm + b * 16 + r;
        if (m >= p.m) continue;
        auto* y = static_cast<typename O::raw*>(p.y) + m * p.y_stride + n0 + wn + part * 4;
#pragma unroll
        for (int a = 0; a < A; ++a) {
            if (left <= a * 16) continue;
            float v[4];
#pragma unroll
            for (int c = 0; c < 4; ++c) {
                if constexpr (BUCKETS) v[c] = fmaf(scale[b], sum_of[a][b][c], add[a][c]);
                else v[c] = fmaf(scale[b], fmaf(step[a][c], (float)d[a][b][c], centre[a][c] * sums[b]), add[a][c]);
            }
            put4<O>(y + a * 16, v, left - a * 16 < 4 ? (int)(left - a * 16) : 4);
        }
    }
}

// ---- few tokens ----------------------------------------------------------------------------------------------------------
// The weights are read once and bound the time. A workgroup takes 16 channels and all tokens (16 * MT); its waves share the
// codes of a channel: by buckets, or a bucket's codes among several waves, so that enough loads are on their way. Each wave
// moves its codes through LDS of its own, as the tiles do, and waits for nobody. Whole numbers meet in LDS before they are
// scaled; waves that take whole buckets scale their own, and their sums meet in the order of the waves. One token times 8192 x 2048
// 6.3 us (2.7 TB/s: the latency of the loads, and as many bytes of tokens through LDS as of weights).
template <int MT, int WAVES, int STAGES, class O>
__global__ __launch_bounds__(WAVES * 64) void few_kernel(MatmulParams p) {
    constexpr int ROWS = 16 + 16 * MT, LOADS = 2 + 2 * MT;
    __shared__ __attribute__((aligned(1024))) uint8_t lds[WAVES][STAGES][ROWS * kStep];
    __shared__ int meet[WAVES][MT][4][64];
    const int lane = threadIdx.x % 64, wave = __builtin_amdgcn_readfirstlane((int)threadIdx.x / 64);
    const int i = lane % 16, part = lane / 16;
    const uint64_t n0 = (uint64_t)blockIdx.x * 16;
    const uint32_t piece = (uint32_t)((lane % 8) ^ (lane / 8)) * 16;
    const uint8_t* w = p.w + n0 * p.w_pitch;
    uint32_t w_at[2], x_at[2 * MT];
#pragma unroll
    for (int l = 0; l < 2; ++l) {
        uint64_t row = l * 8 + lane / 8;
        if (n0 + row >= p.n) row = p.n - 1 - n0;
        w_at[l] = (uint32_t)(row * p.w_pitch) + piece;
    }
#pragma unroll
    for (int l = 0; l < 2 * MT; ++l) {
        const uint32_t row = l * 8 + lane / 8;
        x_at[l] = (uint32_t)((row < p.m ? row : (uint32_t)p.m - 1) * p.x_pitch) + piece;
    }
    auto fetch = [&](uint8_t* to, uint32_t k0) __attribute__((always_inline)) {
        const bool past = k0 + piece >= p.w_pitch;  // as in the tiles
#pragma unroll
        for (int l = 0; l < 2; ++l)
            __builtin_amdgcn_global_load_lds((global_ptr)(w + k0 + (past ? w_at[l] - piece : w_at[l])), (lds_ptr)(to + l * 1024), 16, 0, 0);
#pragma unroll
        for (int l = 0; l < 2 * MT; ++l)
            __builtin_amdgcn_global_load_lds((global_ptr)(p.x + k0 + x_at[l]), (lds_ptr)(to + (2 + l) * 1024), 16, 0, 0);
    };
    // steps [from, to) of 128 codes
    auto multiply = [&](uint32_t from, uint32_t to, v4i (&d)[MT]) __attribute__((always_inline)) {
#pragma unroll
        for (int s = 0; s < STAGES - 1; ++s)
            if (from + s < to) fetch(lds[wave][s], (from + s) * kStep);
        uint32_t slot = 0;
        for (uint32_t s = from; s < to; ++s) {
            if (s + STAGES - 1 < to) {
                fetch(lds[wave][slot == 0 ? STAGES - 1 : slot - 1], (s + STAGES - 1) * kStep);
                wait_loads<(STAGES - 1) * LOADS>();
            } else {
                wait_loads<0>();
            }
            const uint8_t* at = lds[wave][slot] + i * kStep;
#pragma unroll
            for (int k = 0; k < 2; ++k) {
                const int in = ((k * 4 + part) ^ (i % 8)) * 16;
                const v4i wv = *reinterpret_cast<const v4i*>(at + in) ^ (int)0x80808080;
#pragma unroll
                for (int t = 0; t < MT; ++t) {
                    const v4i xv = *reinterpret_cast<const v4i*>(at + (16 + t * 16) * kStep + in);
                    d[t] = __builtin_amdgcn_mfma_i32_16x16x64_i8(wv, xv, d[t], 0, 0, 0);
                }
            }
            slot = slot + 1 == STAGES ? 0 : slot + 1;
            wait_reads();  // the slot has been read before it is filled again
        }
    };
    const bool shared = p.buckets < WAVES;  // several waves to a bucket
    const uint32_t parts = shared ? WAVES / p.buckets : 1;
    const uint32_t steps = (uint32_t)((p.k + kStep - 1) / kStep), each_bucket = (p.bucket + kStep - 1) / kStep;
    const uint64_t first = n0 + part * 4;
    auto scaled = [&](const int* d, uint32_t bucket, int t, float* v) __attribute__((always_inline)) {
        const uint64_t m = t * 16 + i < (int)p.m ? t * 16 + i : p.m - 1;
        const float sum = p.x_sums[m * p.buckets + bucket];
#pragma unroll
        for (int c = 0; c < 4; ++c) {
            const uint64_t n = first + c < p.n ? first + c : p.n - 1;
            const float2 of = *reinterpret_cast<const float2*>(p.meta + 2 * (n * p.buckets + bucket));
            v[c] += fmaf(of.y, (float)d[c], fmaf(128.0f, of.y, of.x) * sum);
        }
    };
    if (shared) {
        v4i d[MT];
#pragma unroll
        for (int t = 0; t < MT; ++t) d[t] = v4i{0, 0, 0, 0};
        const uint32_t bucket = wave / parts, at = wave % parts;
        if (bucket < p.buckets) {
            const uint32_t lo = bucket * each_bucket, stop = lo + each_bucket < steps ? lo + each_bucket : steps;
            const uint32_t each = (stop - lo + parts - 1) / parts, from = lo + at * each;
            if (from < stop) multiply(from, from + each < stop ? from + each : stop, d);
        }
#pragma unroll
        for (int t = 0; t < MT; ++t)
#pragma unroll
            for (int c = 0; c < 4; ++c) meet[wave][t][c][lane] = d[t][c];
    } else {
        float v[MT][4];
#pragma unroll
        for (int t = 0; t < MT; ++t)
#pragma unroll
            for (int c = 0; c < 4; ++c) v[t][c] = 0.0f;
        for (uint32_t b = wave; b < p.buckets; b += WAVES) {
            v4i d[MT];
#pragma unroll
            for (int t = 0; t < MT; ++t) d[t] = v4i{0, 0, 0, 0};
            const uint32_t lo = b * each_bucket;
            multiply(lo, lo + each_bucket < steps ? lo + each_bucket : steps, d);
#pragma unroll
            for (int t = 0; t < MT; ++t) {
                const int whole[4] = {d[t][0], d[t][1], d[t][2], d[t][3]};
                scaled(whole, b, t, v[t]);
            }
        }
#pragma unroll
        for (int t = 0; t < MT; ++t)
#pragma unroll
            for (int c = 0; c < 4; ++c) meet[wave][t][c][lane] = __float_as_int(v[t][c]);
    }
    __syncthreads();
    for (int t = wave; t < MT; t += WAVES) {
        float v[4] = {0.0f, 0.0f, 0.0f, 0.0f};
        if (shared) {
            for (uint32_t b = 0; b < p.buckets; ++b) {
                int d[4] = {0, 0, 0, 0};
                for (uint32_t a = 0; a < parts; ++a)
#pragma unroll
                    for (int c = 0; c < 4; ++c) d[c] += meet[b * parts + a][t][c][lane];
                scaled(d, b, t, v);
            }
        } else {
            for (int a = 0; a < WAVES; ++a)
#pragma unroll
                for (int c = 0; c < 4; ++c) v[c] += __int_as_float(meet[a][t][c][lane]);
        }
        const uint64_t m = t * 16 + i;
        if (m >= p.m || first >= p.n) continue;
        const float s = p.x_scale[m];
        const int count = p.n - first < 4 ? (int)(p.n - first) : 4;
#pragma unroll
        for (int c = 0; c < 4; ++c) v[c] = p.bias ? fmaf(s, v[c], p.bias[c < count ? first + c : first]) : s * v[c];
        put4<O>(static_cast<typename O::raw*>(p.y) + m * p.y_stride + first, v, count);
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

template <int TN, int TM, int WN, int WM, int STAGES, bool BUCKETS, int GROUPS, class O>
static hipError_t launch_tiles_of(const MatmulParams& p, hipStream_t s) {
    const uint32_t n_tiles = (uint32_t)((p.n + TN - 1) / TN), m_tiles = (uint32_t)((p.m + TM - 1) / TM);
    // in several launches where the tiles are more than a grid holds
    const uint32_t most = kMaxGrid / n_tiles ? kMaxGrid / n_tiles : 1;
    for (uint32_t done = 0; done < m_tiles; done += most) {
        const uint32_t now = m_tiles - done < most ? m_tiles - done : most;
        const uint64_t first = (uint64_t)done * TM;
        MatmulParams q = p;
        q.x += first * p.x_pitch;
        q.x_scale += first;
        q.x_sums += first * p.buckets;
        q.m = p.m - first < (uint64_t)now * TM ? p.m - first : (uint64_t)now * TM;
        q.y = static_cast<typename O::raw*>(p.y) + first * p.y_stride;
        hipLaunchKernelGGL((tiles_kernel<TN, TM, WN, WM, STAGES, BUCKETS, GROUPS, O>), dim3(n_tiles * now),
                           dim3(Tile<TN, TM, WN, WM>::THREADS * GROUPS), 0, s, q, n_tiles, now);
        const hipError_t e = hipGetLastError();
        if (e != hipSuccess) return e;
    }
    return hipSuccess;
}

template <int MT, int WAVES, int STAGES, class O>
static hipError_t launch_few(const MatmulParams& p, hipStream_t s) {
    hipLaunchKernelGGL((few_kernel<MT, WAVES, STAGES, O>), dim3((unsigned)((p.n + 15) / 16)), dim3(WAVES * 64), 0, s, p);
    return hipGetLastError();
}

// The tile with one bucket to a channel, or with several.
template <int TN, int TM, int WN, int WM, int STAGES, class O>
static hipError_t launch_tiles(const MatmulParams& p, hipStream_t s) {
    return p.buckets > 1 ? launch_tiles_of<TN, TM, WN, WM, STAGES, true, 1, O>(p, s)
                         : launch_tiles_of<TN, TM, WN, WM, STAGES, false, 1, O>(p, s);
}

template <class O>
static hipError_t launch_matmul_to(const MatmulParams& p, hipStream_t s) {
    switch (choose_product(p.m, p.n, p.k, p.buckets)) {
        case Product::FEW_16_8: return launch_few<1, 8, 2, O>(p, s);
        case Product::FEW_16_4: return launch_few<1, 4, 3, O>(p, s);
        case Product::FEW_32_8: return launch_few<2, 8, 2, O>(p, s);
        case Product::FEW_32_4: return launch_few<2, 4, 2, O>(p, s);
        case Product::TILE_64_TEAMS: return launch_tiles_of<64, 64, 32, 32, 2, true, 4, O>(p, s);
        case Product::TILE_64_DEEP: return launch_tiles<64, 64, 32, 32, 4, O>(p, s);
        case Product::TILE_64: return launch_tiles<64, 64, 32, 32, 2, O>(p, s);
        case Product::TILE_128: return launch_tiles<128, 128, 64, 64, 2, O>(p, s);
        case Product::TILE_256: return launch_tiles_of<256, 256, 64, 128, 2, false, 1, O>(p, s);
    }
    return hipErrorInvalidValue;
}

hipError_t launch_matmul(qsdp_dtype out, const MatmulParams& p, hipStream_t s) {
    return out == QSDP_F32 ? launch_matmul_to<F32>(p, s) : out == QSDP_BF16 ? launch_matmul_to<BF16>(p, s) : launch_matmul_to<F16>(p, s);
}

}  // namespace qsdp_lm
