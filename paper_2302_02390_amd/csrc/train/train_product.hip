// Products of rows in 8-bit floating point with a scale for each 128 elements:
//
//   y_mn = sum over blocks of a_scale[block, m] b_scale[block, n] sum over the block of a_mk b_nk  (+ bias_n) (+ y_mn)
// The sum over a block is one matrix instruction (16 x 16 x 128, binary32 out), which the scales' product multiplies into the
// result: four multiplications and additions of a wave for each instruction, which run beside the next one.
// That instruction aligns the products of eight neighbours of k to the largest of them and cuts off what lies some 15 bits below:
// random operands' sums come out 1.3e-5 of their norm off (16 x 16 x 128 and 32 x 32 x 64 alike; codes within a factor of 2^9 are
// exact). That is lost in 16-bit results, whose rounding is 2^-9 or 2^-12. Results in binary32 go by bf16 instructions
// (EXACT): every code is a bf16 number, the products are exact, and the matrix units take twice the time.
#include "train_blocks.hpp"
#include "train_common.hpp"
#include "train_plan.hpp"

namespace qsdp_train {
namespace {

typedef int v4i __attribute__((ext_vector_type(4)));
typedef int v8i __attribute__((ext_vector_type(8)));
typedef float v4f __attribute__((ext_vector_type(4)));
typedef __bf16 v2bf __attribute__((ext_vector_type(2)));
typedef __bf16 v8bf __attribute__((ext_vector_type(8)));
typedef __attribute__((address_space(1))) const void* global_ptr;
typedef __attribute__((address_space(3))) void* lds_ptr;

// Until at most N of the wave's loads are on their way: those into LDS are not the compiler's to wait for.
template <int N>
__device__ __forceinline__ void wait_loads() {
    static_assert(N < 64, "six bits");
    asm volatile("s_waitcnt vmcnt(%0)" ::"n"(N) : "memory");
}

// Until the wave's reads of LDS are done, in a form that the compiler counts and does not repeat.
__device__ __forceinline__ void wait_reads() {
    __builtin_amdgcn_sched_barrier(0);
    __builtin_amdgcn_s_waitcnt(0xc07f);  // lgkmcnt(0)
    __builtin_amdgcn_sched_barrier(0);
}

// The workgroup's waves meet; unlike __syncthreads, without waiting for the loads that are on their way.
__device__ __forceinline__ void meet_here() { asm volatile("s_barrier" ::: "memory"); }

// 32 codes as the matrix instructions take them: as they are, or as bf16 numbers.
template <bool EXACT>
struct Operand {
    v8i codes;
    __device__ __forceinline__ explicit Operand(v8i c) : codes(c) {}
};
template <>
struct Operand<true> {
    v8bf part[4];
    __device__ __forceinline__ explicit Operand(v8i c) {
#pragma unroll
        for (int g = 0; g < 4; ++g) {
            v2bf two[4];
#pragma unroll
            for (int i = 0; i < 2; ++i) {
                two[2 * i] = __builtin_amdgcn_cvt_scalef32_pk_bf16_fp8(c[2 * g + i], 1.0f, false);
                two[2 * i + 1] = __builtin_amdgcn_cvt_scalef32_pk_bf16_fp8(c[2 * g + i], 1.0f, true);
            }
            __builtin_memcpy(&part[g], two, 16);
        }
    }
};

__device__ __forceinline__ v4f product(const Operand<false>& a, const Operand<false>& b) {
    return __builtin_amdgcn_mfma_scale_f32_16x16x128_f8f6f4(a.codes, b.codes, v4f{0.0f, 0.0f, 0.0f, 0.0f}, 0, 0, 0, 0, 0, 0);
}
__device__ __forceinline__ v4f product(const Operand<true>& a, const Operand<true>& b) {
    v4f sum = {0.0f, 0.0f, 0.0f, 0.0f};
#pragma unroll
    for (int g = 0; g < 4; ++g) sum = __builtin_amdgcn_mfma_f32_16x16x32_bf16(a.part[g], b.part[g], sum, 0, 0, 0);
    return sum;
}

// The lane's 32 codes of a row in LDS: two of its eight pieces, which the row has permuted. Both operands take the same ones, so it
// does not matter which of the block's elements the instruction takes them for.
__device__ __forceinline__ v8i fragment(const uint8_t* row, int first, int second) {
    const v4i p = *reinterpret_cast<const v4i*>(row + first), q = *reinterpret_cast<const v4i*>(row + second);
    return __builtin_shufflevector(p, q, 0, 1, 2, 3, 4, 5, 6, 7);
}

// ---- results ---------------------------------------------------------------------------------------------------------------
// Four consecutive results of a row, or the first `count` of them.
template <class O>
__device__ __forceinline__ void put_to(typename O::raw* y, float* v, int count, bool accumulate) {
    if (count == 4) {
        if constexpr (sizeof(typename O::raw) == 4) {
            typedef float anywhere __attribute__((ext_vector_type(4), aligned(4)));
            anywhere* to = reinterpret_cast<anywhere*>(y);
            anywhere r = {v[0], v[1], v[2], v[3]};
            if (accumulate) {
                const anywhere old = *to;
#pragma unroll
                for (int c = 0; c < 4; ++c) r[c] += old[c];
            }
            *to = r;
        } else {
            typedef uint32_t anywhere __attribute__((ext_vector_type(2), aligned(2)));
            anywhere* to = reinterpret_cast<anywhere*>(y);
            if (accumulate) {
                const anywhere old = *to;
                const u32x4 both = {old[0], old[1], 0, 0};
#pragma unroll
                for (int c = 0; c < 4; ++c) v[c] += O::at(both, c);
            }
            *to = anywhere{O::two(v[0], v[1]), O::two(v[2], v[3])};
        }
    } else {
#pragma unroll
        for (int c = 0; c < 3; ++c)
            if (c < count) y[c] = O::put(accumulate ? v[c] + O::get(y[c]) : v[c]);
    }
}

__device__ __forceinline__ void put4(const ProductParams& p, uint64_t m, uint64_t n, float* v) {
    const int count = p.n - n < 4 ? (int)(p.n - n) : 4;
    if (p.bias)
#pragma unroll
        for (int c = 0; c < 4; ++c) v[c] += p.bias[c < count ? n + c : n];
    const uint64_t at = m * p.y_stride + n;
    if (p.out == QSDP_F32) put_to<F32>(static_cast<float*>(p.y) + at, v, count, p.accumulate);
    else if (p.out == QSDP_BF16) put_to<BF16>(static_cast<uint16_t*>(p.y) + at, v, count, p.accumulate);
    else put_to<F16>(static_cast<_Float16*>(p.y) + at, v, count, p.accumulate);
}

// ---- tiles -----------------------------------------------------------------------------------------------------------------
template <int TN, int TM, int WN, int WM, bool SQUARE>
struct Tile {
    static constexpr int WAVES = TN / WN * (TM / WM), THREADS = WAVES * 64;
    static constexpr int CODES = (TN + TM) * (int)kWide;           // bytes of a step's codes in LDS,
    static constexpr int SCALES = TM + (SQUARE ? 0 : TN);          // and its scales
    static constexpr int BYTES = CODES + SCALES * 4;
    static constexpr int B_LOADS = TN / 8 / WAVES, A_LOADS = TM / 8 / WAVES;  // of 8 rows, for each wave
    static constexpr int LOADS = B_LOADS + A_LOADS + 1 + (SQUARE ? 0 : 1);
    static_assert(TN % (8 * WAVES) == 0 && TM % (8 * WAVES) == 0 && TN % 64 == 0 && TM % 64 == 0, "whole loads");
};

// Which tile: workgroups go to the eight dies in turn, so each die takes a contiguous run of the tiles, which walk through
// `kBand` tiles of rows for every tile of columns and share their operands in the die's L2.
constexpr uint32_t kDies = 8, kBand = 4;

__device__ __forceinline__ void place(uint32_t id, uint32_t n_tiles, uint32_t m_tiles, uint32_t& n, uint32_t& m) {
    const uint32_t all = n_tiles * m_tiles, each = all / kDies, more = all % kDies, die = id % kDies;
    const uint32_t at = die * each + (die < more ? die : more) + id / kDies;
    const uint32_t band = at / (kBand * n_tiles), left = m_tiles - band * kBand, high = left < kBand ? left : kBand;
    const uint32_t in = at - band * kBand * n_tiles;
    n = in / high;
    m = band * kBand + in % high;
}

// A workgroup computes TN columns x TM rows of y in steps of a block of 128. Both operands' codes go straight from memory into
// LDS, two steps deep, and one barrier a step separates them. LDS holds rows of 128 bytes whose eight pieces of 16 are permuted by the
// row (piece c of row r in place c ^ (r % 8)), so that sixteen rows read the same piece from all banks; the permutation is in the
// addresses that the lanes read from memory. A wave multiplies WN columns (first operand, so that four consecutive columns of a row
// of y end up in a lane) by WM rows: it keeps a step's columns in registers and walks over the rows.
template <int TN, int TM, int WN, int WM, int STAGES, bool SQUARE, bool EXACT>
__global__ __launch_bounds__((TN / WN) * (TM / WM) * 64, 2) void tiles_kernel(ProductParams p, uint32_t n_tiles, uint32_t m_tiles) {
    typedef Tile<TN, TM, WN, WM, SQUARE> S;
    __shared__ __attribute__((aligned(1024))) uint8_t lds[STAGES][S::BYTES];
    constexpr int A = WN / 16, B = WM / 16;
    uint32_t n_tile, m_tile;
    place(blockIdx.x, n_tiles, m_tiles, n_tile, m_tile);
    const int lane = threadIdx.x % 64, wave = wave_index();
    const uint64_t n0 = (uint64_t)n_tile * TN, m0 = (uint64_t)m_tile * TM;
    // what the lane loads: a piece of 16 bytes of a row of eight; rows past the matrix are its last one
    const uint32_t piece = (uint32_t)((lane % 8) ^ (lane / 8)) * 16;
    uint32_t b_at[S::B_LOADS], a_at[S::A_LOADS];
#pragma unroll
    for (int i = 0; i < S::B_LOADS; ++i) {
        uint64_t row = (uint64_t)(wave * S::B_LOADS + i) * 8 + lane / 8;
        if (n0 + row >= p.n) row = p.n - 1 - n0;
        b_at[i] = (uint32_t)(row * p.pitch) + piece;
    }
#pragma unroll
    for (int i = 0; i < S::A_LOADS; ++i) {
        uint64_t row = (uint64_t)(wave * S::A_LOADS + i) * 8 + lane / 8;
        if (m0 + row >= p.m) row = p.m - 1 - m0;
        a_at[i] = (uint32_t)(row * p.pitch) + piece;
    }
    const uint8_t* b = p.b + n0 * p.pitch;
    const uint8_t* a = p.a + m0 * p.pitch;
    // scales: 64 to a load; waves that have none of their own load another's again
    const int a_part = wave % (TM / 64) * 64, b_part = wave % (TN / 64) * 64;
    const float* a_scale = p.a_scale + (m0 + a_part + lane < p.m ? m0 + a_part + lane : p.m - 1);
    const float* b_scale = SQUARE ? p.b_scale : p.b_scale + (n0 + b_part + lane < p.n ? n0 + b_part + lane : p.n - 1);
    auto fetch = [&](uint8_t* to, uint32_t s) __attribute__((always_inline)) {
        const uint32_t k0 = s * kWide;
#pragma unroll
        for (int i = 0; i < S::B_LOADS; ++i)
            __builtin_amdgcn_global_load_lds((global_ptr)(b + k0 + b_at[i]), (lds_ptr)(to + (wave * S::B_LOADS + i) * 1024), 16, 0, 0);
#pragma unroll
        for (int i = 0; i < S::A_LOADS; ++i)
            __builtin_amdgcn_global_load_lds((global_ptr)(a + k0 + a_at[i]),
                                             (lds_ptr)(to + TN * kWide + (wave * S::A_LOADS + i) * 1024), 16, 0, 0);
        __builtin_amdgcn_global_load_lds((global_ptr)(a_scale + s * p.a_rows), (lds_ptr)(to + S::CODES + a_part * 4), 4, 0, 0);
        if constexpr (!SQUARE)
            __builtin_amdgcn_global_load_lds((global_ptr)(b_scale + s * p.n), (lds_ptr)(to + S::CODES + (TM + b_part) * 4), 4, 0, 0);
    };
    const int wn = wave % (TN / WN) * WN, wm = wave / (TN / WN) * WM;
    const int r = lane % 16, part = lane / 16;
    const int first = (part ^ (r % 8)) * 16, second = ((4 + part) ^ (r % 8)) * 16;
    const uint64_t n_blocks = blocks_of(p.n);
    const float* square = p.b_scale + ((n0 + wn) / kWide < n_blocks ? (n0 + wn) / kWide : n_blocks - 1);
    const uint32_t steps = (uint32_t)(p.pitch / kWide);
    v4f sum[A][B];
#pragma unroll
    for (int i = 0; i < A; ++i)
#pragma unroll
        for (int j = 0; j < B; ++j) sum[i][j] = v4f{0.0f, 0.0f, 0.0f, 0.0f};
#pragma unroll
    for (int s = 0; s < STAGES - 1; ++s)
        if ((uint32_t)s < steps) fetch(lds[s], s);
    for (uint32_t s = 0; s < steps; ++s) {
        wait_loads<0>();
        meet_here();
        if (s + STAGES - 1 < steps) fetch(lds[(s + STAGES - 1) % STAGES], s + STAGES - 1);
        const uint8_t* from = lds[s % STAGES];
        const float* scales = reinterpret_cast<const float*>(from + S::CODES);
        const float of_b = SQUARE ? square[s * n_blocks] : 1.0f;
        v8i bv[A];
#pragma unroll
        for (int i = 0; i < A; ++i) bv[i] = fragment(from + (wn + i * 16 + r) * kWide, first, second);
#pragma unroll
        for (int j = 0; j < B; ++j) {
            const Operand<EXACT> av(fragment(from + (TN + wm + j * 16 + r) * kWide, first, second));
            const float of = scales[wm + j * 16 + r] * of_b;
#pragma unroll
            for (int i = 0; i < A; ++i) {
                const v4f part_sum = product(Operand<EXACT>(bv[i]), av);
                v4f by = {of, of, of, of};
                if constexpr (!SQUARE) by = *reinterpret_cast<const v4f*>(scales + TM + wn + i * 16 + part * 4) * of;
#pragma unroll
                for (int c = 0; c < 4; ++c) sum[i][j][c] = fmaf(part_sum[c], by[c], sum[i][j][c]);
            }
        }
        wait_reads();
        meet_here();
    }
    // sum[i][j][c]: column wn + i * 16 + part * 4 + c of row wm + j * 16 + r
#pragma unroll
    for (int j = 0; j < B; ++j) {
        const uint64_t m = m0 + wm + j * 16 + r;
        if (m >= p.m) continue;
#pragma unroll
        for (int i = 0; i < A; ++i) {
            const uint64_t n = n0 + wn + i * 16 + part * 4;
            if (n >= p.n) continue;
            float v[4] = {sum[i][j][0], sum[i][j][1], sum[i][j][2], sum[i][j][3]};
            put4(p, m, n, v);
        }
    }
}

}  // namespace

template <int TN, int TM, int WN, int WM, int STAGES, bool SQUARE, bool EXACT>
static hipError_t launch_tiles(const ProductParams& p, hipStream_t s) {
    const uint32_t n_tiles = (uint32_t)((p.n + TN - 1) / TN);
    const uint64_t m_tiles = (p.m + TM - 1) / TM;
    // in several launches where the tiles are more than a grid holds
    const uint64_t most = kMaxGrid / n_tiles ? kMaxGrid / n_tiles : 1;
    for (uint64_t done = 0; done < m_tiles; done += most) {
        const uint64_t now = m_tiles - done < most ? m_tiles - done : most, first = done * TM;
        ProductParams q = p;
        q.a += first * p.pitch;
        q.a_scale += first;
        q.m = p.m - first < now * TM ? p.m - first : now * TM;
        q.y = static_cast<uint8_t*>(p.y) + first * p.y_stride * (p.out == QSDP_F32 ? 4 : 2);
        hipLaunchKernelGGL((tiles_kernel<TN, TM, WN, WM, STAGES, SQUARE, EXACT>), dim3(n_tiles * (unsigned)now),
                           dim3(Tile<TN, TM, WN, WM, SQUARE>::THREADS), 0, s, q, n_tiles, (uint32_t)now);
        const hipError_t e = hipGetLastError();
        if (e != hipSuccess) return e;
    }
    return hipSuccess;
}

template <bool SQUARE, bool EXACT>
static hipError_t launch_product_of(const ProductParams& p, hipStream_t s) {
    return launch_tiles<64, 64, 32, 32, 2, SQUARE, EXACT>(p, s);
}

hipError_t launch_product(bool b_square, const ProductParams& p, hipStream_t s) {
    if (p.out == QSDP_F32) return b_square ? launch_product_of<true, true>(p, s) : launch_product_of<false, true>(p, s);
    return b_square ? launch_product_of<true, false>(p, s) : launch_product_of<false, false>(p, s);
}

}  // namespace qsdp_train
