// Kernels on rows of logits: log probabilities with entropy and top alternatives, their gradient, and distillation from a
// teacher's top logits. A workgroup per row; its threads hold the row in registers in the logits' format, 16 bytes to a
// piece, and in LDS what is left, so that the logits are read once whatever follows: maximum, sums of exponentials, alternatives,
// gradient. Rows of more than 51968 (binary32) or 103935 (16 bits) logits do not fit and are read once per use, chunk by chunk
// (2048 rows of 65536 fp32 logits with 20 alternatives 162 us, of 131072 329, in bf16 185; without alternatives 178 and 93).
#include <type_traits>

#include "lm_common.hpp"
#include "lm_plan.hpp"
#include "lm_rows.hpp"

// A lambda is part of the function that calls it: what it refers to has to stay in registers.
#define QSDP_INLINE __attribute__((always_inline))

namespace qsdp_lm {
namespace {

constexpr float kLog2e = 1.44269504088896341f;
constexpr float kLn2 = 0.69314718055994531f;
// Where exp2 has long been 0: keeps 0 * (-inf) out of the sums.
constexpr float kLeast = -400.0f;

// The same number, unknown to the compiler: what follows from it is computed where it is used, and not once ahead of all
// passes over a row, which would take more registers than the row.
__device__ __forceinline__ uint32_t fresh(uint32_t scalar) {
    asm volatile("" : "+s"(scalar));
    return scalar;
}
__device__ __forceinline__ uint32_t fresh_thread() {
    uint32_t thread = threadIdx.x;
    asm volatile("" : "+v"(thread));
    return thread;
}

// f(0) ... f(N - 1), each number a constant: registers cannot be indexed.
template <int N, class F>
__device__ __forceinline__ void times(F f) {
    if constexpr (N > 0) {
        times<N - 1>(f);
        f(std::integral_constant<int, N - 1>());
    }
}

// Nothing is moved past every fourth element: side by side, a piece's elements take more registers than the row leaves.
__device__ __forceinline__ void keep_order(int e) {
    if (e % 4 == 3) __builtin_amdgcn_sched_barrier(0);
}

__device__ __forceinline__ float exp2_fast(float a) { return __builtin_amdgcn_exp2f(a); }  // 1 ulp, 0 below 2^-126

// A value that is the same for all threads, in a scalar register.
__device__ __forceinline__ float same(float v) {
    return __builtin_bit_cast(float, __builtin_amdgcn_readfirstlane(__builtin_bit_cast(int, v)));
}

// ---- a row in pieces -----------------------------------------------------------------------------------------------
// Piece i of a thread holds elements (first + i * THREADS + thread) * PER - lead ... of the row; what is not of the row is
// -inf. Pieces start at multiples of four bytes: a row of 16-bit elements that does not has a lead of one (loads of 16 bytes at
// odd elements reach three quarters of the rate: 4096 rows of 50257 logits 87 us, 69 with it).
// The first NV are in registers, up to HELD more in LDS, in places that only their thread uses. STREAM: the row has more
// pieces than the workgroup holds and passes through chunk by chunk.
enum class Rest { NONE, HELD, STREAM };

template <class T, int THREADS, int NV, Rest REST>
struct Row {
    static constexpr uint32_t CHUNK = THREADS * NV;  // pieces in registers
    static constexpr bool STREAM = REST == Rest::STREAM;
    static constexpr uint32_t ROOM = REST == Rest::HELD ? held_pieces(THREADS) : 0;
    static constexpr int HELD = (int)((ROOM + THREADS - 1) / THREADS);
    const typename T::raw* z;
    u32x4* held;
    uint32_t n, lead, pieces, first;  // n and pieces with the lead
    u32x4 v[NV];

    __device__ __forceinline__ Row(const typename T::raw* z_, uint64_t n_, u32x4* held_) : z(z_), held(held_) {
        lead = sizeof(typename T::raw) == 2 ? (uint32_t)(reinterpret_cast<uintptr_t>(z_) / 2 % 2) : 0u;
        n = (uint32_t)n_ + lead;
        pieces = (n + T::PER - 1) / T::PER;
        load(0);
    }
    // Of the pieces that are not whole: the first one of a row with a lead, and the one that the row ends in.
    __device__ __forceinline__ u32x4 load_edge(uint32_t at) const {
        return load_part<T>(z - lead + (uint64_t)at * T::PER, at == 0 ? (int)lead : 0, at == n / T::PER ? (int)(n % T::PER) : T::PER);
    }
    __device__ __forceinline__ uint32_t chunks() const { return STREAM ? (pieces + CHUNK - 1) / CHUNK : 1u; }
    __device__ __forceinline__ void load(uint32_t chunk) {
        first = STREAM ? chunk * CHUNK : 0u;
        const uint32_t whole = fresh(n) / T::PER, thread = fresh_thread();
        const typename T::raw* from = z - lead;
        times<NV>([&](auto i) QSDP_INLINE {
            const uint32_t at = first + i * THREADS;  // a scalar: the thread's part of the address is the same for all i
            v[i] = u32x4{T::NONE, T::NONE, T::NONE, T::NONE};
            if (at + thread < whole && (i > 0 || at + thread >= lead)) v[i] = load16<T>(from + (uint64_t)at * T::PER + thread * T::PER);
        });
        const uint32_t slot = whole - first;  // of the piece that the row ends in, if it is no whole one
        if constexpr (HELD > 0) {
            u32x4 more[HELD];
            times<HELD>([&](auto i) QSDP_INLINE {
                const uint32_t at = CHUNK + i * THREADS;
                more[i] = u32x4{T::NONE, T::NONE, T::NONE, T::NONE};
                if (at + thread < whole) more[i] = load16<T>(from + (uint64_t)at * T::PER + thread * T::PER);
            });
            times<HELD>([&](auto i) QSDP_INLINE {
                if (i * THREADS + thread < ROOM) held[i * THREADS + thread] = more[i];
            });
            if (n % T::PER != 0 && slot >= CHUNK && slot % THREADS == thread) held[slot - CHUNK] = load_edge(whole);
        }
        if (lead > 0 && first == 0 && thread == 0) v[0] = load_edge(0);
        if (n % T::PER != 0 && slot < CHUNK && slot % THREADS == thread && (lead == 0 || whole > 0)) {
            const u32x4 last = load_edge(whole);
            times<NV>([&](auto i) QSDP_INLINE {
                if (slot / THREADS == (uint32_t)i) v[i] = last;
            });
        }
    }
    // f(piece, i, index of its first element) for the pieces that the thread's wave has any of. Those in registers are made
    // opaque: otherwise the compiler keeps their elements unpacked from one pass to the next, in twice the registers and more.
    template <class F>
    __device__ __forceinline__ void in_registers(F f) {
        times<NV>([&](auto i) QSDP_INLINE { asm volatile("" : "+v"(v[i])); });
        const uint32_t end = fresh(pieces), wave = (uint32_t)wave_index() * 64, lane = threadIdx.x % 64;
        times<NV>([&](auto i) QSDP_INLINE {
            const uint32_t at = first + i * THREADS + wave;
            if (at < end) f(v[i], i, (at + lane) * T::PER - lead);
        });
    }
    template <class F>
    __device__ __forceinline__ void in_lds(F f) {
        if constexpr (HELD > 0) {
            const uint32_t end = fresh(pieces), wave = (uint32_t)wave_index() * 64, thread = fresh_thread();
            times<HELD>([&](auto i) QSDP_INLINE {
                const uint32_t at = CHUNK + i * THREADS + wave;
                if (at < end) f(held[i * THREADS + thread], i, (at + thread % 64) * T::PER - lead);
            });
        }
    }
    template <class F>
    __device__ __forceinline__ void pieces_of_wave(F f) {
        in_registers(f);
        in_lds(f);
    }
    // all chunks in turn; a row of one chunk stays where it is
    template <class F>
    __device__ __forceinline__ void each_chunk(F f) {
        if constexpr (STREAM) {
            for (uint32_t c = 0;;) {
                f();
                if (++c >= chunks()) break;
                load(c);
            }
        } else {
            f();
        }
    }
    __device__ __forceinline__ void again() {
        if (STREAM) load(0);
    }
    // to[..] = f(element) for all of them; pieces that are not whole go by themselves, once for all i
    template <class F>
    __device__ __forceinline__ void write(typename T::raw* to, F f) {
        const uint32_t whole = fresh(n) / T::PER;
        pieces_of_wave([&](const u32x4& piece, auto, uint32_t index) QSDP_INLINE {
            float d[T::PER];
            const u32x4 here = piece;
            times<T::PER>([&](auto e) QSDP_INLINE {
                d[e] = f(T::at(here, e));
                keep_order(e);
            });
            if (index + lead < whole * T::PER && (int32_t)index >= 0) store16<T>(to + index, T::pack(d));
        });
        const uint32_t slot = whole - first, thread = threadIdx.x;
        auto edge = [&](const u32x4& piece, uint32_t at) QSDP_INLINE {
            float d[T::PER];
            times<T::PER>([&](auto e) QSDP_INLINE { d[e] = f(T::at(piece, e)); });
            store_part<T>(to - lead + (uint64_t)at * T::PER, T::pack(d), at == 0 ? (int)lead : 0,
                          at == whole ? (int)(n % T::PER) : T::PER);
        };
        if (lead > 0 && first == 0 && thread == 0) edge(v[0], 0);
        if (n % T::PER != 0 && slot < CHUNK + ROOM && slot % THREADS == thread && (lead == 0 || whole > 0)) {
            u32x4 last = v[0];
            times<NV>([&](auto i) QSDP_INLINE {
                if (slot / THREADS == (uint32_t)i) last = v[i];
            });
            if (HELD > 0 && slot >= CHUNK) last = held[slot - CHUNK];
            edge(last, whole);
        }
    }
    // A bit for every element of the thread in registers, or in LDS, for which hit(value) holds: bit i * PER + e. -inf past the
    // row counts like any.
    template <bool LDS, class H>
    __device__ __forceinline__ uint64_t mask(H hit) {
        static_assert((NV > HELD ? NV : HELD) * T::PER <= 64, "a bit for every element");
        uint32_t low = 0, high = 0;
        auto look = [&](const u32x4& piece, auto i, uint32_t) QSDP_INLINE {
            const u32x4 here = piece;
            times<T::PER>([&](auto e) QSDP_INLINE {
                constexpr int bit = decltype(i)::value * T::PER + decltype(e)::value;
                if (bit < 32) low |= hit(T::at(here, e)) ? 1u << (bit % 32) : 0u;
                else high |= hit(T::at(here, e)) ? 1u << (bit % 32) : 0u;
            });
        };
        if constexpr (LDS) in_lds(look);
        else in_registers(look);
        return (uint64_t)high << 32 | low;
    }
    template <class H>
    __device__ __forceinline__ uint32_t count(H hit) {
        return (uint32_t)__popcll(mask<false>(hit)) + (HELD > 0 ? (uint32_t)__popcll(mask<true>(hit)) : 0u);
    }
    // element of a bit of the mask
    template <bool LDS>
    __device__ __forceinline__ uint32_t index_of(int bit) const {
        return ((LDS ? CHUNK : first) + (uint32_t)bit / T::PER * THREADS + threadIdx.x) * T::PER + (uint32_t)bit % T::PER - lead;
    }
};

// ---- exponents -------------------------------------------------------------------------------------------------------------
// (z - m) slope for many z, m the largest of them, by one multiply-add: z slope - back, with back = m slope rounded. `rest` is
// what that rounding leaves, the same for all z: the true exponent is the multiply-add's plus rest, of a magnitude of 2^-24 of
// back's. Where that is large (rows of the format's lowest value or highest) two different z are so far apart that only m's own
// exponential is not zero: any power of two for slope keeps it so, and with it back is exact.
struct Line {
    float slope, back, rest;
    __device__ __forceinline__ Line(float m, float slope_) : slope(slope_) {
        m = m == kNegInf ? 0.0f : m;
        back = m * slope;
        rest = -fmaf(m, slope, -back);
        if (!(fabsf(back) < 536870912.0f)) {
            slope = ldexpf(1.0f, 59 - __builtin_amdgcn_frexp_expf(m));
            back = m * slope;
            rest = 0.0f;
        }
        slope = same(slope), back = same(back), rest = same(rest);
    }
    __device__ __forceinline__ float at(float z) const { return fmaf(z, slope, -back); }
};

// ---- sums of exponentials --------------------------------------------------------------------------------------------
// The maximum m and, with a = (z - m) * scale2, the sums s of 2^a and u of 2^a a, over part of a row. Where nothing is
// above -inf all three stay at their start; a NaN or +inf makes the sums NaN.
struct Sums {
    float m, s, u;
};
__device__ __forceinline__ float shift_of(float m, float top, float scale2) { return fmaxf((m - top) * scale2, kLeast); }
__device__ __forceinline__ void rescale(Sums& a, float top, float scale2) {
    if (a.m == top) return;
    const float d = shift_of(a.m, top, scale2), f = exp2_fast(d);
    a.u = f * fmaf(d, a.s, a.u);
    a.s = f * a.s;
    a.m = top;
}

// The lane's maximum over the pieces of a chunk. A NaN may win or lose: the sums of its wave are NaN either way.
template <class R>
__device__ __forceinline__ float lane_max(R& row, F32) {
    float most = kNegInf;
    row.pieces_of_wave([&](const u32x4& piece, auto, uint32_t) QSDP_INLINE {
        const u32x4 here = piece;
        times<4>([&](auto e) QSDP_INLINE { most = fmaxf(most, F32::at(here, e)); });
    });
    return most;
}
template <class R>
__device__ __forceinline__ float lane_max(R& row, F16) {  // two at a time
    F16::pair most = {(_Float16)kNegInf, (_Float16)kNegInf};
    row.pieces_of_wave([&](const u32x4& piece, auto, uint32_t) QSDP_INLINE {
        const u32x4 here = piece;
        times<4>([&](auto k) QSDP_INLINE {
            const uint32_t word = here[(int)k];
            most = __builtin_elementwise_max(most, __builtin_bit_cast(F16::pair, word));
        });
    });
    return fmaxf((float)most[0], (float)most[1]);
}
template <class R>
__device__ __forceinline__ float lane_max(R& row, BF16) {
    // Two at a time as 16-bit integers: the largest signed one is the maximum unless it is negative; then all are, and the
    // smallest unsigned one is.
    typedef short two __attribute__((ext_vector_type(2)));
    typedef unsigned short two_u __attribute__((ext_vector_type(2)));
    two top = {-32768, -32768};
    two_u low = {0xffff, 0xffff};
    row.pieces_of_wave([&](const u32x4& piece, auto, uint32_t) QSDP_INLINE {
        const u32x4 here = piece;
        times<4>([&](auto k) QSDP_INLINE {
            const uint32_t word = here[(int)k];
            top = __builtin_elementwise_max(top, __builtin_bit_cast(two, word));
            low = __builtin_elementwise_min(low, __builtin_bit_cast(two_u, word));
        });
    });
    const int larger = top[0] > top[1] ? top[0] : top[1];
    const uint32_t smaller = low[0] < low[1] ? low[0] : low[1];
    const float most = __uint_as_float((larger >= 0 ? (uint32_t)larger : smaller) << 16);
    return most == most ? most : kNegInf;  // of a lane with nothing, or a NaN
}

// Adds a chunk to a wave's sums, lane by lane; the maximum is the wave's own, so that no workgroup has to meet for it, and
// `most` the lane's. MORE: the sum of another power of the same differences as well, of 2^(a * ratio).
enum class Second { NONE, SQUARE, OTHER };

template <bool MEAN, Second MORE, class R, class T>
__device__ __forceinline__ void add_chunk(R& row, float scale2, float other2, Sums& a, float& second, float& most, T tag) {
    most = fmaxf(most, lane_max(row, tag));
    const float m = same(reduce64(most, Max()));
    if (a.m != m) {
        if (MORE == Second::SQUARE) second *= exp2_fast(2.0f * shift_of(a.m, m, scale2));
        if (MORE == Second::OTHER) second *= exp2_fast(shift_of(a.m, m, other2));
        rescale(a, m, scale2);
    }
    const Line line(m, scale2), other(m, MORE == Second::OTHER ? other2 : 0.0f);
    float s = 0.0f, u = 0.0f, o = 0.0f;
    row.pieces_of_wave([&](const u32x4& piece, auto, uint32_t) QSDP_INLINE {
        const u32x4 here = piece;
        times<T::PER>([&](auto e) QSDP_INLINE {
            const float z = T::at(here, e), d = line.at(z), p = exp2_fast(d);
            s += p;
            if (MEAN) u = fmaf(p, fmaxf(d, kLeast), u);
            if (MORE == Second::SQUARE) o = fmaf(p, p, o);
            if (MORE == Second::OTHER) o += exp2_fast(other.at(z));
            keep_order(e);
        });
    });
    const float f = exp2_fast(line.rest);
    a.s = fmaf(f, s, a.s);
    if (MEAN) a.u = fmaf(f, fmaf(line.rest, s, u), a.u);
    if (MORE == Second::SQUARE) second = fmaf(f * f, o, second);
    if (MORE == Second::OTHER) second = fmaf(exp2_fast(other.rest), o, second);
}

// The workgroup's sums from its waves'; every thread gets them. room: 4 floats for each wave.
template <int THREADS, bool MEAN, Second MORE>
__device__ __forceinline__ Sums join(Sums a, float scale2, float other2, float& second, float (*room)[4]) {
    constexpr int WAVES = THREADS / 64;
    a.s = reduce64(a.s, Add());
    if (MEAN) a.u = reduce64(a.u, Add());
    if (MORE != Second::NONE) second = reduce64(second, Add());
    if (threadIdx.x % 64 == 0) {
        float* w = room[threadIdx.x / 64];
        w[0] = a.m, w[1] = a.s, w[2] = a.u, w[3] = second;
    }
    __syncthreads();
    const int w = threadIdx.x % 16;
    Sums b = {kNegInf, 0.0f, 0.0f};
    float c = 0.0f;
    if (w < WAVES) b = {room[w][0], room[w][1], room[w][2]}, c = room[w][3];
    const float m = reduce16(b.m, Max());
    if (MORE == Second::SQUARE) c *= exp2_fast(b.m == m ? 0.0f : 2.0f * shift_of(b.m, m, scale2));
    if (MORE == Second::OTHER) c *= exp2_fast(b.m == m ? 0.0f : shift_of(b.m, m, other2));
    rescale(b, m, scale2);
    if (MORE != Second::NONE) second = reduce16(c, Add());
    return {m, reduce16(b.s, Add()), MEAN ? reduce16(b.u, Add()) : 0.0f};
}

// ---- top alternatives ------------------------------------------------------------------------------------------------
// Order: value downwards (a NaN above all, the two zeros equal), then index upwards; larger keys first.
// The search has no vector register to spare at 64: it spills two at most, of values that are the same for a wave's elements.
__device__ __forceinline__ uint32_t value_key(float z) {
    const uint32_t u = __float_as_uint(z + 0.0f);
    return z != z ? 0xffffffffu : (int32_t)u < 0 ? ~u : u | 0x80000000u;
}
__device__ __forceinline__ float key_value(uint32_t key) {
    return __uint_as_float(key == 0xffffffffu ? 0x7fc00000u : (int32_t)key < 0 ? key ^ 0x80000000u : ~key);
}
// Low bits of a value's key that its format leaves all zero or all one.
template <class T>
constexpr int key_low_bits() { return sizeof(typename T::raw) == 4 ? 0 : T::NONE == BF16::NONE ? 16 : 13; }

constexpr uint32_t kKeyNan = 0xffffffffu, kKeyNegInf = 0x007fffffu;
constexpr int kMostTop = 128;
constexpr uint32_t kRoom = 512;  // candidates that are ranked

template <int THREADS>
struct TopRoom {
    static constexpr int GROUPS = THREADS < 256 ? THREADS : 256;
    union {
        uint32_t group[GROUPS];  // until the threshold is known
        uint64_t list[kRoom];
    };
    uint32_t words[THREADS / 64];
    uint32_t count, least, exact;
};

// Appends the row's elements for which hit(value) holds to the list, as far as it has room, and counts all of them. They are
// few and read from memory once more: which of its registers a thread needs is not known when the code is compiled.
template <class T, int THREADS, class R, class H>
__device__ __forceinline__ void collect(R& row, TopRoom<THREADS>& room, H hit) {
    auto append = [&](uint64_t mine, auto lds) QSDP_INLINE {
        if (mine == 0) return;
        uint32_t to = atomicAdd(&room.count, (uint32_t)__popcll(mine));
        for (; mine != 0 && to < kRoom; mine &= mine - 1, ++to) {
            const uint32_t index = row.template index_of<decltype(lds)::value>(__ffsll((unsigned long long)mine) - 1);
            room.list[to] = (uint64_t)value_key(T::get(row.z[index])) << 32 | ~index;
        }
    };
    row.again();
    row.each_chunk([&]() QSDP_INLINE { append(row.template mask<false>(hit), std::false_type()); });
    if (R::HELD > 0) append(row.template mask<true>(hit), std::true_type());
}

// The `top` first elements, as keys in room.list[0 .. return value), in no order and with some more. Threshold: the top-th
// largest of up to 256 groups' maxima, which at least `top` elements reach and on ordinary data not many more (about
// -g log(1 - top / g) of g groups: 74 for 64). Where too many reach it (ties, masks, large values in few groups) or a NaN takes
// part, the top-th value itself is found bit by bit, and of its equals the first by index are taken: 32 passes over the row,
// which is slow (48 rows of 50257 bf16 logits with 20 alternatives 11 us, 73 where a mask leaves 30 neighbours; 16 rows of 1000
// fp32 ones 5.5 us with 20 alternatives, 104 with 128).
template <class T, int THREADS, class R>
__device__ __forceinline__ uint32_t top_list(R& row, uint32_t top, bool plain, float most, TopRoom<THREADS>& room) {
    constexpr int GROUPS = TopRoom<THREADS>::GROUPS, SHARE = THREADS / GROUPS, LOW = key_low_bits<T>();
    const int lane = threadIdx.x % 64, wave = wave_index();
    if (threadIdx.x == 0) room.count = 0;
    float m = most;  // the thread's
    if (SHARE >= 2) m = fmaxf(m, dpp<0xB1>(m));
    if (SHARE >= 4) m = fmaxf(m, dpp<0x4E>(m));
    if (threadIdx.x % SHARE == 0) room.group[threadIdx.x / SHARE] = value_key(m);
    __syncthreads();
    if (wave == 0) {
        uint32_t key[GROUPS / 64];
#pragma unroll
        for (int g = 0; g < GROUPS / 64; ++g) key[g] = room.group[g * 64 + lane] >> LOW;
        uint32_t high = 0;
        for (int bit = 31 - LOW; bit >= 0; --bit) {
            const uint32_t trial = high | 1u << bit;
            uint32_t reach = 0;
#pragma unroll
            for (int g = 0; g < GROUPS / 64; ++g) reach += __popcll(__ballot(key[g] >= trial));
            if (reach >= top) high = trial;
            if (reach == top) break;  // the bits below need not be known
        }
        high <<= LOW;
        if ((int32_t)high >= 0) high |= (1u << LOW) - 1;  // a negative value's low bits
        high = high > kKeyNegInf ? high : kKeyNegInf;
        uint32_t reach = 0;  // a group's maximum, not only a bound
#pragma unroll
        for (int g = 0; g < GROUPS / 64; ++g) reach |= __ballot(key[g] == high >> LOW) != 0;
        if (lane == 0) room.least = high, room.exact = reach;
    }
    __syncthreads();
    uint32_t least = room.least;
    bool known = plain && room.exact;
    float bound = key_value(least);
    if (plain && bound != kNegInf) {
        collect<T>(row, room, [&](float z) QSDP_INLINE { return z >= bound; });
        __syncthreads();
        if (room.count <= kRoom) return room.count;
    }
    // the value bit by bit, unless the threshold is it already: fewer than `top` are above it
    uint32_t above;
    for (;;) {
        if (!known) {
            uint32_t nans = 0;
            row.again();
            row.each_chunk([&]() QSDP_INLINE { nans += row.count([](float z) QSDP_INLINE { return z != z; }); });
            nans = reduce_block<THREADS>(nans, Add(), room.words);
            least = 0;
            for (int bit = 31; bit >= 0; --bit) {
                const float trial = key_value(least | 1u << bit);  // nothing reaches a NaN but NaNs
                uint32_t reach = 0;
                row.again();
                row.each_chunk([&]() QSDP_INLINE { reach += row.count([&](float z) QSDP_INLINE { return z >= trial; }); });
                if (reduce_block<THREADS>(reach, Add(), room.words) + nans >= top) least |= 1u << bit;
            }
            least = least < kKeyNegInf ? kKeyNegInf : least;
        }
        bound = key_value(least);
        __syncthreads();
        if (threadIdx.x == 0) room.count = 0;
        __syncthreads();
        if (least != kKeyNan) collect<T>(row, room, [&](float z) QSDP_INLINE { return !(z <= bound); });
        __syncthreads();
        above = room.count;
        if (above < top) break;
        known = false;
    }
    // of the equal ones the first by index: a piece of every thread at a time, which is the order of the row
    uint32_t found = above;
    const uint64_t below = (1ull << lane) - 1;
    auto equal = [&](float z) QSDP_INLINE { return z == bound || (z != z && bound != bound); };
    auto take = [&](uint64_t mine, auto lds, uint32_t rounds) QSDP_INLINE {
        for (uint32_t i = 0; i < rounds && found < top; ++i, mine >>= T::PER) {
            const uint32_t index = row.template index_of<decltype(lds)::value>((int)i * T::PER);
            uint32_t bits = (uint32_t)mine & ((1u << T::PER) - 1);
            const uint32_t end = row.n - row.lead;
            if ((int32_t)index < 0) bits &= ~1u;  // a lead's place
            else if (index + T::PER > end) bits &= index < end ? (1u << (end - index)) - 1 : 0u;
            if ((int32_t)index < 0 && end < T::PER) bits &= (2u << end) - 1;
            const uint32_t many = __popc(bits);
            uint32_t before = 0, total = 0;  // the lanes' counts, bit by bit
#pragma unroll
            for (int b = 0; b < 4; ++b) {
                const uint64_t lanes = __ballot(many >> b & 1);
                before += __popcll(lanes & below) << b;
                total += __popcll(lanes) << b;
            }
            __syncthreads();
            if (lane == 0) room.words[wave] = total;
            __syncthreads();
            uint32_t to = found + before;
            for (int w = 0; w < THREADS / 64; ++w) {
                to += w < wave ? room.words[w] : 0u;
                found += room.words[w];
            }
            for (; bits != 0 && to < top; bits &= bits - 1, ++to)
                room.list[to] = (uint64_t)least << 32 | ~(index + (uint32_t)(__ffs((int)bits) - 1));
        }
    };
    row.again();
    for (uint32_t c = 0; c < row.chunks() && found < top; ++c) {
        if (c > 0) row.load(c);
        take(row.template mask<false>(equal), std::false_type(), R::CHUNK / THREADS);
    }
    if (R::HELD > 0 && found < top) take(row.template mask<true>(equal), std::true_type(), R::HELD);
    __syncthreads();
    return top;
}

// The logit of a row's token, NaN where it has none.
template <class T>
__device__ __forceinline__ float logit_of(const typename T::raw* z, int64_t token, uint64_t vocab) {
    const bool exists = (uint64_t)token < vocab;
    const float v = T::get(z[exists ? token : 0]);  // asked for in any case, so that nothing waits here
    return exists ? v : __builtin_nanf("");
}

// A row's results from its sums; one thread's work.
__device__ __forceinline__ void put_score(const ScoreParams& p, uint64_t r, const Sums& a, float log_total, int64_t token,
                                          float z_token) {
    const bool empty = a.s == 0.0f;
    if (p.logprob) {
        float v = (z_token - a.m) * p.in.inv_temperature - log_total;
        if (empty && z_token == z_token) v = kNegInf;
        p.logprob[r] = token < 0 ? 0.0f : v;
    }
    if (p.entropy) p.entropy[r] = empty ? 0.0f : log_total - a.u / a.s * kLn2;
    if (p.stats) {
        p.stats[2 * r] = a.s == a.s ? a.m : a.s;  // of a NaN or +inf: no maximum either
        p.stats[2 * r + 1] = log_total;
    }
}
__device__ __forceinline__ void put_top(const ScoreParams& p, uint64_t r, uint32_t rank, uint64_t key, const Sums& a, float log_total) {
    p.top_index[r * p.top + rank] = (int32_t)~(uint32_t)key;
    p.top_logprob[r * p.top + rank] =
        a.s == 0.0f ? kNegInf : (key_value((uint32_t)(key >> 32)) - a.m) * p.in.inv_temperature - log_total;
}

// m, S = sum 2^a and U = sum 2^a a with a = (z - m) scale2 give the log probability of any logit, and the entropy log S - U ln2 / S.
// Alternatives: the `top`-th largest of the threads' group maxima is a threshold that at least `top` logits reach; the few that
// do are collected and each is ranked by how many come before it.
// HBM bounds calls of many rows: 4096 rows of 50257 bf16 logits 73 us (5.6 TB/s of reads), of fp32 ones with 64 alternatives
// 158 us (5.2 TB/s). A call of one row is bound by its workgroup's chain of reductions: 50257 logits 10 us.
// PART: one of kParts parts of a row, to be joined.
template <class T, int THREADS, int NV, Rest REST, bool TOP, bool PART>
__global__ __launch_bounds__(THREADS, REST == Rest::STREAM ? 4 : 8) void score_kernel(ScoreParams p) {
    __shared__ float waves[THREADS / 64][4];
    __shared__ u32x4 held[REST == Rest::HELD ? held_pieces(THREADS) : 1];
    const uint64_t item = p.in.first + blockIdx.x, r = PART ? item / kParts : item;
    const uint64_t lo = PART ? item % kParts * p.per : 0, left = p.in.vocab - lo;
    const auto* z = static_cast<const typename T::raw*>(p.in.logits) + r * p.in.stride + lo;
    const float scale2 = p.in.inv_temperature * kLog2e;
    // the token is asked for ahead of the row, its logit right behind it
    const int64_t token = !PART && p.logprob ? p.tokens[r] : -1;
    Row<T, THREADS, NV, REST> row(z, PART && left > p.per ? p.per : left, held);
    const float z_token = PART ? 0.0f : logit_of<T>(z, token, p.in.vocab);
    Sums a = {kNegInf, 0.0f, 0.0f};
    float most = kNegInf, none = 0.0f;
    row.each_chunk([&]() QSDP_INLINE { add_chunk<true, Second::NONE>(row, scale2, 0.0f, a, none, most, T()); });
    a = join<THREADS, true, Second::NONE>(a, scale2, 0.0f, none, waves);
    float log_total = logf(a.s);
    if constexpr (TOP) {  // scalars: the search leaves no vector register to spare (fp32, 64 alternatives 192 us without, 158 with)
        a = {same(a.m), same(a.s), same(a.u)};
        log_total = same(log_total);
    }
    if (threadIdx.x == 0) {
        if (PART) p.heads[item] = make_float4(a.m, a.s, a.u, 0.0f);
        else put_score(p, r, a, log_total, token, z_token);
    }
    if constexpr (TOP) {
        __shared__ TopRoom<THREADS> room;
        const uint32_t top = (uint32_t)p.top;
        const uint32_t count = top_list<T>(row, top, a.s == a.s, most, room);
        // eight lanes count for a candidate how many are before it
        for (uint32_t i = threadIdx.x / 8; i < count; i += THREADS / 8) {
            const uint64_t key = room.list[i];
            uint32_t rank = 0;
            for (uint32_t o = threadIdx.x % 8; o < count; o += 8) rank += room.list[o] > key;
            rank = reduce4(rank, Add());
            rank += dpp<0x141>(rank);
            if (rank < top && threadIdx.x % 8 == 0) {
                if (PART) p.keys[item * top + rank] = key - lo;  // its low word is the complement of the index
                else put_top(p, r, rank, key, a, log_total);
            }
        }
    }
}

// The parts of a row: their sums by one maximum; their alternatives, each list in order, by how many of the other lists are
// before each.
template <class T>
__global__ __launch_bounds__(256) void score_join_kernel(ScoreParams p) {
    __shared__ uint64_t keys[kParts * kMostTop];
    const uint64_t r = p.in.first + blockIdx.x;
    const uint32_t top = (uint32_t)p.top, all = top * (uint32_t)kParts;
    const auto* z = static_cast<const typename T::raw*>(p.in.logits) + r * p.in.stride;
    const int64_t token = p.logprob ? p.tokens[r] : -1;
    for (uint32_t i = threadIdx.x; i < all; i += 256) keys[i] = p.keys[r * all + i];
    const uint32_t part = threadIdx.x % 16;
    Sums a = {kNegInf, 0.0f, 0.0f};
    if (part < kParts) {
        const float4 head = p.heads[r * kParts + part];
        a = {head.x, head.y, head.z};
    }
    const float z_token = logit_of<T>(z, token, p.in.vocab);
    const float m = reduce16(a.m, Max());
    rescale(a, m, p.in.inv_temperature * kLog2e);
    a = {m, reduce16(a.s, Add()), reduce16(a.u, Add())};
    const float log_total = logf(a.s);
    if (threadIdx.x == 0) put_score(p, r, a, log_total, token, z_token);
    __syncthreads();
    for (uint32_t i = threadIdx.x; i < all; i += 256) {
        const uint64_t key = keys[i];
        uint32_t rank = i % top;
        for (uint32_t q = 0; q < kParts; ++q) {
            if (q == i / top) continue;
            uint32_t from = 0, to = top;
            while (from < to) {
                const uint32_t mid = (from + to) / 2;
                if (keys[q * top + mid] > key) from = mid + 1;
                else to = mid;
            }
            rank += from;
        }
        if (rank < top) put_top(p, r, rank, key, a, log_total);
    }
}

// ---- gradient of log probability and entropy --------------------------------------------------------------------------
// Element by element once a row's sums are known: rows are cut into segments of 256 threads x 4 x 16 bytes.
constexpr int kSegment = 4;

template <class T>
struct Segment {
    static constexpr uint32_t PIECES = 256 * kSegment;
    uint64_t row;
    uint32_t n, first;
    static uint64_t of(uint64_t n) { return ((n + T::PER - 1) / T::PER + PIECES - 1) / PIECES; }
    __device__ __forceinline__ Segment(uint64_t item, uint32_t n_) : n(n_) {
        const uint32_t each = ((n + T::PER - 1) / T::PER + PIECES - 1) / PIECES;
        row = item / each;
        first = (uint32_t)(item % each) * PIECES;
    }
    __device__ __forceinline__ uint32_t lo() const { return first * T::PER; }
    __device__ __forceinline__ uint32_t hi() const { return n - lo() < PIECES * T::PER ? n : lo() + PIECES * T::PER; }
    __device__ __forceinline__ void load(const typename T::raw* z, u32x4* v) const {
        times<kSegment>([&](auto i) QSDP_INLINE {
            const uint32_t at = first + i * 256 + threadIdx.x;
            v[i] = u32x4{0, 0, 0, 0};
            if (at < n / T::PER) v[i] = load16<T>(z + (uint64_t)at * T::PER);
            else if (at == n / T::PER) v[i] = load_part<T>(z + (uint64_t)at * T::PER, 0, (int)(n % T::PER));
        });
    }
    // dz[j] = f(z[j], j), and `more` on top at one place (~0: nowhere)
    template <class F>
    __device__ __forceinline__ void write(const u32x4* v, typename T::raw* dz, F f, uint32_t place, float more) const {
        times<kSegment>([&](auto i) QSDP_INLINE {
            const uint32_t at = first + i * 256 + threadIdx.x;
            float d[T::PER];
            times<T::PER>([&](auto e) QSDP_INLINE { d[e] = f(T::at(v[i], e), at * T::PER + e); });
            if (place / T::PER == at) times<T::PER>([&](auto e) QSDP_INLINE { d[e] += place % T::PER == e ? more : 0.0f; });
            if (at < n / T::PER) store16<T>(dz + (uint64_t)at * T::PER, T::pack(d));
            else if (at == n / T::PER) store_part<T>(dz + (uint64_t)at * T::PER, T::pack(d), 0, (int)(n % T::PER));
        });
    }
};

// d z_j = (g ([j = i] - p_j) - h p_j (log p_j + entropy)) / temperature. HBM bounds it: 4096 rows of 50257 bf16 logits 142 us,
// 5.8 TB/s both ways; a plain copy reaches 5.95.
template <class T, bool ENTROPY>
__global__ __launch_bounds__(256) void score_backward_kernel(ScoreBackwardParams p) {
    const uint32_t n = (uint32_t)p.in.vocab;
    const float scale2 = p.in.inv_temperature * kLog2e;
    const Segment<T> part(p.in.first + blockIdx.x, n);
    const uint64_t r = part.row;
    u32x4 v[kSegment];
    part.load(static_cast<const typename T::raw*>(p.in.logits) + r * p.in.stride, v);
    const float m = same(p.stats[2 * r]), log_total = same(p.stats[2 * r + 1]), log2_total = log_total * kLog2e;
    auto* dz = static_cast<typename T::raw*>(p.d_logits) + r * p.d_stride;
    if (log_total == kNegInf) {
        part.write(v, dz, [](float, uint32_t) QSDP_INLINE { return 0.0f; }, ~0u, 0.0f);
        return;
    }
    const int64_t asked = p.d_logprob && p.tokens ? p.tokens[r] : -1;
    const uint32_t token = (uint64_t)asked < (uint64_t)n ? (uint32_t)asked : ~0u;  // ~0: none
    const float g = token != ~0u ? p.d_logprob[r] * p.in.inv_temperature : 0.0f;
    const float h = ENTROPY ? p.d_entropy[r] * p.in.inv_temperature * kLn2 : 0.0f;  // entropies in bits below
    // p = f e, log2 p = a + rest - log2_total, e = 2^a
    const Line line(m, scale2);
    const float f = exp2f(line.rest - log2_total);
    const float off = -f * (ENTROPY ? fmaf(h, fmaf(p.entropy[r], kLog2e, line.rest - log2_total), g) : g), times_a = -f * h;
    part.write(v, dz, [&](float z, uint32_t) QSDP_INLINE {
        const float a = line.at(z);
        return exp2_fast(a) * (ENTROPY ? fmaf(times_a, fmaxf(a, kLeast), off) : off);
    }, token, g);
}

// ---- distillation ------------------------------------------------------------------------------------------------------
// The teacher's list of a row: probabilities, their logs to base 2, places, and the student's logits there.
struct List {
    float p[kMostTop], log2_p[kMostTop], z[kMostTop];
    int32_t index[kMostTop];
};

__device__ __forceinline__ uint32_t label_of(int64_t asked, uint32_t n) {  // ~0: none
    return __builtin_amdgcn_readfirstlane((uint64_t)asked < (uint64_t)n ? (uint32_t)asked : ~0u);
}

// One exponential: at 1 where the list has no part, else at the temperature.
template <Second MORE>
__device__ __forceinline__ float one_scale2(const DistillParams& p) {
    return MORE == Second::NONE && p.alpha == 0.0f ? kLog2e : p.in.inv_temperature * kLog2e;
}

template <class T, int THREADS>
__device__ __forceinline__ bool fill_list(const DistillParams& p, const typename T::raw* z, uint64_t r, List& list,
                                          float* scratch) {
    const float teacher2 = p.in.inv_temperature * kLog2e;
    const int k = (int)threadIdx.x;
    int32_t index = -1;
    float u = kNegInf;
    if (k < p.top) {
        index = p.teacher_index[r * p.top + k];
        if (index < 0 || (uint64_t)index >= p.in.vocab) index = -1;
        list.index[k] = index;
        list.z[k] = 0.0f;
        if (index >= 0) {
            u = p.teacher_logit[r * p.top + k];
            list.z[k] = T::get(z[index]);
        }
    }
    const float um = reduce_block<THREADS>(u, Max(), scratch);
    const float ua = (u - (um == kNegInf ? 0.0f : um)) * teacher2;
    const float e = index >= 0 ? exp2f(ua) : 0.0f;
    const float mass = reduce_block<THREADS>(e, Add(), scratch);
    if (k < p.top) {
        list.p[k] = mass != 0.0f ? e / mass : 0.0f;
        list.log2_p[k] = ua - log2f(mass);
    }
    return mass != 0.0f;  // a NaN counts as taught
}

// What the gradient of a row's loss is made of: d z_v = soft 2^(...) + hard 2^(...), less the targets at the list's places and
// at the label. MORE: the exponentials at 1 are others than the
// temperature's (scale2), or their squares at temperature 2; otherwise one serves.
template <Second MORE>
struct Slope {
    Line line, other;  // exponents at the temperature (or the only ones), and at 1
    float soft, hard;  // of the targets
    float p1, p2;      // d z_v = p1 e + p2 f, f = e^2 at temperature 2: the sums and the lines' rests are in them
    uint32_t label;    // ~0: none
    bool none;
    __device__ __forceinline__ Slope(const DistillParams& p, float scale2, float m, float soft_log, float hard_log, bool taught,
                                     uint32_t label_, float g)
        : line(m, scale2), other(m, MORE == Second::OTHER ? kLog2e : 0.0f), label(label_) {
        soft = same(taught ? g * p.alpha * p.temperature : 0.0f);
        hard = same(label != ~0u ? g * (1.0f - p.alpha) : 0.0f);
        none = soft_log == kNegInf || (soft == 0.0f && hard == 0.0f);
        p1 = same((MORE == Second::NONE ? soft + hard : soft) * exp2f(line.rest - soft_log));
        p2 = MORE == Second::NONE ? 0.0f : same(hard * exp2f((MORE == Second::SQUARE ? 2.0f * line.rest : other.rest) - hard_log));
    }
    __device__ __forceinline__ float operator()(float z) const {
        const float e = exp2_fast(line.at(z));
        if (MORE == Second::NONE) return p1 * e;
        if (MORE == Second::SQUARE) return e * fmaf(p2, e, p1);
        return fmaf(p2, exp2_fast(other.at(z)), p1 * e);
    }
    __device__ __forceinline__ float target(const List& list, int top, uint32_t j) const {
        float sum = 0.0f;
#pragma unroll 1
        for (int o = 0; o < top; ++o) sum += (uint32_t)list.index[o] == j ? list.p[o] : 0.0f;
        return soft * sum + (j == label ? hard : 0.0f);
    }
    // The places of the list and the label, among elements [lo, hi), once more with their targets; slots of the same index
    // write the same value. After a barrier behind the writes of all elements.
    template <class T>
    __device__ __forceinline__ void aim(const List& list, int top, float z_label, typename T::raw* dz, uint32_t lo,
                                        uint32_t hi) const {
        const int k = (int)threadIdx.x;
        if (k < top) {
            const uint32_t j = (uint32_t)list.index[k];
            if (j >= lo && j < hi) dz[j] = T::put((*this)(list.z[k]) - target(list, top, j));
        }
        if (k == 0 && label >= lo && label < hi) dz[label] = T::put((*this)(z_label) - target(list, top, label));
    }
};

// Loss, and in the same pass the gradient if it is asked for: the row is still in registers and LDS when its sums are known. Two
// sums at once (at the temperature and at 1), where both terms are asked for, by one exponential if the temperature is 2: the
// square of e^(t/2) is e^t. HBM bounds it: 8192 rows of 50257 bf16 logits with 32 in the list 333 us, 4.9 TB/s both ways (at
// temperature 3, by two exponentials, a hundredth more; 2048 rows with 64 101 us, at temperature 3 110). The loss alone 150 us, 5.5
// TB/s of reads.
template <class T, int THREADS, int NV, Rest REST, Second MORE>
__global__ __launch_bounds__(THREADS, REST == Rest::STREAM ? 4 : 8) void distill_kernel(DistillParams p) {
    __shared__ float waves[THREADS / 64][4], scratch[THREADS / 64];
    __shared__ u32x4 held[REST == Rest::HELD ? held_pieces(THREADS) : 1];
    __shared__ List list;
    const uint64_t r = p.in.first + blockIdx.x;
    const uint32_t n = (uint32_t)p.in.vocab;
    const auto* z = static_cast<const typename T::raw*>(p.in.logits) + r * p.in.stride;
    const float scale2 = one_scale2<MORE>(p);
    Row<T, THREADS, NV, REST> row(z, n, held);
    const bool taught = fill_list<T, THREADS>(p, z, r, list, scratch);
    const int64_t asked = p.labels && p.alpha < 1.0f ? p.labels[r] : -1;
    const uint32_t label = label_of(asked, n);
    const float z_label = same(label != ~0u ? T::get(z[label]) : 0.0f);
    Sums a = {kNegInf, 0.0f, 0.0f};
    float most = kNegInf, second = 0.0f;
    row.each_chunk([&]() QSDP_INLINE { add_chunk<false, MORE>(row, scale2, kLog2e, a, second, most, T()); });
    a = join<THREADS, false, MORE>(a, scale2, kLog2e, second, waves);
    // maximum, log2 of the sums at the temperature and at 1
    const float m = same(a.m), soft_log = same(log2f(a.s)), hard_log = MORE == Second::NONE ? soft_log : same(log2f(second));
    const bool empty = soft_log == kNegInf;
    const int k = (int)threadIdx.x;
    float kl = 0.0f;  // the temperature times the sum, in natural units: the lowest logit divided by it may be past the format
    if (k < p.top) {
        const float prob = list.p[k];
        if (prob > 0.0f || prob != prob) {
            const float scaled_q = empty ? kNegInf : (list.z[k] - m) - p.temperature * (soft_log * kLn2);
            kl = prob * (p.temperature * (list.log2_p[k] * kLn2) - scaled_q);
        }
    }
    kl = reduce_block<THREADS>(kl, Add(), scratch);
    if (k == 0) {
        float loss = p.alpha > 0.0f ? p.alpha * p.temperature * kl : 0.0f;
        if (label != ~0u) loss -= (1.0f - p.alpha) * (empty ? kNegInf : (z_label - m) - hard_log * kLn2);
        p.loss[r] = asked >= (int64_t)n ? __builtin_nanf("") : loss;
        if (p.stats) {
            p.stats[3 * r] = m;
            p.stats[3 * r + 1] = soft_log * kLn2;
            p.stats[3 * r + 2] = hard_log * kLn2;
        }
    }
    if (!p.d_logits) return;
    auto* dz = static_cast<typename T::raw*>(p.d_logits) + r * p.d_stride;
    const Slope<MORE> slope(p, scale2, m, soft_log, hard_log, taught, label, same(p.row_scale ? p.row_scale[r] : 1.0f));
    row.again();
    __syncthreads();  // the list is there, and what is read outside the own pieces has been read
    if (slope.none) {
        for (uint32_t j = threadIdx.x; j < n; j += THREADS) dz[j] = T::put(0.0f);
        return;
    }
    row.each_chunk([&]() QSDP_INLINE { row.write(dz, slope); });
    __syncthreads();
    slope.template aim<T>(list, p.top, z_label, dz, 0, n);
}

// The gradient alone, from the row's statistics: rows are cut into segments as for the gradient of log probabilities, each of which
// computes the list's probabilities. 8192 rows of 50257 bf16 logits with 32 in the list 289 us (5.7 TB/s both ways), 2048 rows with
// 64 90 us (4.6).
template <class T, Second MORE>
__global__ __launch_bounds__(256) void distill_backward_kernel(DistillParams p) {
    __shared__ float scratch[4];
    __shared__ List list;
    const uint32_t n = (uint32_t)p.in.vocab;
    const Segment<T> part(p.in.first + blockIdx.x, n);
    const uint64_t r = part.row;
    const auto* z = static_cast<const typename T::raw*>(p.in.logits) + r * p.in.stride;
    auto* dz = static_cast<typename T::raw*>(p.d_logits) + r * p.d_stride;
    u32x4 v[kSegment];
    part.load(z, v);
    const bool taught = fill_list<T, 256>(p, z, r, list, scratch);
    const uint32_t label = label_of(p.labels && p.alpha < 1.0f ? p.labels[r] : -1, n);
    const float z_label = same(label != ~0u ? T::get(z[label]) : 0.0f);
    const Slope<MORE> slope(p, one_scale2<MORE>(p), same(p.stats[3 * r]), same(p.stats[3 * r + 1] * kLog2e),
                            same(p.stats[3 * r + 2] * kLog2e), taught, label, same(p.d_loss[r]));
    const bool nothing = slope.none;
    __syncthreads();  // the list is there
    part.write(v, dz, [&](float v, uint32_t) QSDP_INLINE { return nothing ? 0.0f : slope(v); }, ~0u, 0.0f);
    if (nothing) return;
    __syncthreads();
    slope.template aim<T>(list, p.top, z_label, dz, part.lo(), part.hi());
}

// ---- which kernel ------------------------------------------------------------------------------------------------------
// A workgroup for each of `work` items (rows or parts of them), in several launches where they are more than a grid holds:
// a loop over rows inside a kernel costs it 20 registers.
constexpr uint64_t kMaxGrid = 1u << 20;

template <class P>
hipError_t go(void (*kernel)(P), int threads, uint64_t work, P p, hipStream_t s) {
    for (p.in.first = 0; p.in.first < work; p.in.first += kMaxGrid) {
        const uint64_t left = work - p.in.first;
        hipLaunchKernelGGL(kernel, dim3((unsigned)(left < kMaxGrid ? left : kMaxGrid)), dim3(threads), 0, s, p);
        const hipError_t e = hipGetLastError();
        if (e != hipSuccess) return e;
    }
    return hipSuccess;
}

// f with the threads, pieces per thread and Rest of the team for rows of n elements (see choose_row). SHORT: there are rows for
// the smallest team (parts of rows are longer).
template <class T, bool FOUR, bool SHORT, class F>
hipError_t by_length(uint64_t n, F f) {
    const std::integral_constant<int, 8> eight;
    const std::integral_constant<int, 512> half;
    const std::integral_constant<int, 1024> most;
    const std::integral_constant<Rest, Rest::NONE> none;
    const std::integral_constant<Rest, Rest::HELD> held;
    switch (choose_row(row_pieces(n, T::PER), FOUR)) {
        case RowTeam::T128:
            if constexpr (SHORT) return f(std::integral_constant<int, 128>(), std::integral_constant<int, 2>(), none);
            break;
        case RowTeam::T256: return f(std::integral_constant<int, 256>(), eight, none);
        case RowTeam::T512: return f(half, eight, none);
        case RowTeam::T512_LDS:
            if constexpr (FOUR) return f(half, eight, held);
            break;
        case RowTeam::T1024: return f(most, eight, none);
        case RowTeam::T1024_LDS: return f(most, eight, held);
        case RowTeam::STREAM: return f(most, eight, std::integral_constant<Rest, Rest::STREAM>());
    }
    return hipErrorInvalidValue;
}

}  // namespace

template <class T>
hipError_t launch_score(const ScoreParams& p, hipStream_t s) {
    auto rows = [&](auto top) {
        if (p.heads)
            return by_length<T, false, false>(p.per, [&](auto threads, auto nv, auto rest) {
                return go(score_kernel<T, threads, nv, rest, top, true>, threads, p.in.rows * kParts, p, s);
            });
        if constexpr (top)
            if (score_by_four(p.in.rows, p.top))
                return by_length<T, true, true>(p.in.vocab, [&](auto threads, auto nv, auto rest) {
                    return go(score_kernel<T, threads, nv, rest, top, false>, threads, p.in.rows, p, s);
                });
        return by_length<T, false, true>(p.in.vocab, [&](auto threads, auto nv, auto rest) {
            return go(score_kernel<T, threads, nv, rest, top, false>, threads, p.in.rows, p, s);
        });
    };
    const hipError_t e = p.top ? rows(std::true_type()) : rows(std::false_type());
    if (e != hipSuccess || !p.heads) return e;
    return go(score_join_kernel<T>, 256, p.in.rows, p, s);
}

template <class T>
hipError_t launch_score_backward(const ScoreBackwardParams& p, hipStream_t s) {
    const uint64_t work = p.in.rows * Segment<T>::of(p.in.vocab);
    return p.d_entropy ? go(score_backward_kernel<T, true>, 256, work, p, s)
                       : go(score_backward_kernel<T, false>, 256, work, p, s);
}

template <class T>
hipError_t launch_distill(const DistillParams& p, hipStream_t s) {
    const bool both = p.alpha > 0.0f && p.alpha < 1.0f && p.temperature != 1.0f;
    auto launch = [&](auto more) {
        if (!p.loss) return go(distill_backward_kernel<T, more>, 256, p.in.rows * Segment<T>::of(p.in.vocab), p, s);
        return by_length<T, true, true>(p.in.vocab, [&](auto threads, auto nv, auto rest) {
            return go(distill_kernel<T, threads, nv, rest, more>, threads, p.in.rows, p, s);
        });
    };
    if (!both) return launch(std::integral_constant<Second, Second::NONE>());
    if (p.temperature == 2.0f) return launch(std::integral_constant<Second, Second::SQUARE>());
    return launch(std::integral_constant<Second, Second::OTHER>());
}

// an object for each format
template hipError_t launch_score<QSDP_LM_FORMAT>(const ScoreParams&, hipStream_t);
template hipError_t launch_score_backward<QSDP_LM_FORMAT>(const ScoreBackwardParams&, hipStream_t);
template hipError_t launch_distill<QSDP_LM_FORMAT>(const DistillParams&, hipStream_t);

}  // namespace qsdp_lm
