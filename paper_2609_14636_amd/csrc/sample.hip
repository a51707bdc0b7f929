// sample.hip -- the next token of each row of logits, from given random numbers.
//
// With s = (z - max z) / T the token is the kept v with the largest s_v - log noise_v: of independent
// exponentials with rates exp(s_v) the first to ring, which is v with probability exp(s_v) / sum.  top-k,
// top-p and min-p each keep a leading part of the entries in order of z (lowest index first among equal ones), so
// the kept set is one prefix of that order, and sorting a row is not needed to find its end.
//
// One workgroup of sixteen waves per row; of few rows, up to sixteen workgroups look through a part each first.
//   Greedy and unfiltered rows are one pass: the largest z, or the largest key, with its index.
//   Filtered rows: a first pass takes each thread's maximum.  The k-th largest of those 1,024 values is at
//   most the row's k-th largest entry, so the entries from there on (somewhat more than k) hold the first k; a second
//   pass, which finds the row in the caches, gathers them into LDS.  Up to 256 of them: a thread each, which counts the
//   larger ones and sums their masses; more are sorted.  min-p bounds the entries below by itself.  top-p alone has no such bound: the cut is put
//   where some tens of entries lie above, and lower if their mass does not reach top_p of the row's.
//   Rows that do not fit this (a nucleus or a k of thousands, rows of equal logits) take the exact way by the
//   digits of the logits' bits: histograms of counts and masses, 11 bits at a time, lead to the last kept value.
// What bounds it, and what it takes (bf16 rows of 151,936): 256 unfiltered rows 39 us, 6.0 TB/s of logits and numbers, so
// memory; one row with top-k and top-p 13 us in two launches, 64 rows 16: chains of dependent loads and barriers, so every
// wave does what is short for itself.  64 rows with top-p alone take 18 us where their nuclei have some tens of
// entries, and 340 where they have thousands (one row 250): the atomics of the histograms, which meet in some tens of bins.
// Sums of masses are integers of 2^-40 of the largest entry's, or run in a fixed order, so a row's
// result does not depend on timing.
#include <cstddef>

#include "common.hpp"

namespace stride {
namespace {

typedef uint32_t u32x4 __attribute__((ext_vector_type(4)));

constexpr int kThreads = 1024;
constexpr int kWaves = kThreads / kWave;
constexpr int kList = 2048;       // gathered entries that a row can have
constexpr int kBins = 2048;       // 11 bits
constexpr int kCutBins = 256;
constexpr int kCount = 256;       // entries up to which ranks are counted
// threads whose maximum lies above the cut for top-p alone, at first and where their mass falls short
constexpr int kGuess[2] = {64, 700};
constexpr int kMaxParts = 16;     // workgroups of a row in the first kernel for few rows
constexpr int kPartThreads = 256;
constexpr int kPartList = 128;    // entries that a part hands on
constexpr int kPartGuess = 24;    // as kGuess, in a part
constexpr float kLog2e = 1.4426950408889634f;
constexpr float kMassUnit = 1099511627776.0f;  // 2^40

template <int DT>
struct Elem {
    static constexpr int n = DT == STRIDE_BF16 ? 8 : 4;
    static constexpr int low_bits = DT == STRIDE_BF16 ? 10 : 0;  // of the ordered key that all values share
    static constexpr int digits = DT == STRIDE_BF16 ? 2 : 3;     // of 11 bits (the last of float: 10)
};

// What a part of a row leaves for the row's workgroup: its largest value and the mass relative to it (for top-p alone),
// the value from which on its entries are in the list, their number, whether it has NaN or +inf; of a greedy row its
// first entry, of an unfiltered one the winner's index (-1: none) and the point its keys were relative to.
struct alignas(16) Part {
    float top, sum, cut, ref;
    uint32_t n, bad;
    int32_t at;
    uint32_t spare;
    uint64_t first, spare64;
    uint64_t list[kPartList];
};

struct SampleArgs {
    const void *logits;
    const float *noise, *temperature, *top_p, *min_p;
    const int32_t *top_k;
    int32_t *ids;
    uint32_t *flags;
    Part *parts;  // [n_rows, n_parts], or NULL
    int64_t n_rows, ld, noise_ld;
    int32_t vocab, n_parts;
};

// What a workgroup shares.
struct Shared {
    uint64_t mass[kBins];   // or the gathered entries, kList of them
    uint32_t count[kBins];
    alignas(16) uint64_t pair[kCount + 8][2];  // an entry and its mass
    uint64_t wave64[kWaves];
    double waved[kWaves];
    float2 wavef[kWaves];
    uint32_t bad, n_list, found;
    uint64_t above_mass, found_u64;
    uint32_t above_count;
};

__device__ __forceinline__ float ex2(float x) { return __builtin_amdgcn_exp2f(x); }
__device__ __forceinline__ float lg2(float x) { return __builtin_amdgcn_logf(x); }  // takes subnormal x for 0
__device__ __forceinline__ float lg2_all(float x) { return x < 0x1p-126f ? lg2(x * 0x1p32f) - 32.0f : lg2(x); }

// Bits of x in the order of its values; -0 and 0 are one value.
__device__ __forceinline__ uint32_t ordered(float x) {
    const uint32_t b = __float_as_uint(x + 0.0f);
    return b ^ ((uint32_t)((int32_t)b >> 31) | 0x80000000u);
}
// Larger for a larger key, then for a lower index.
__device__ __forceinline__ uint64_t entry(float x, int32_t i) {
    return (uint64_t)ordered(x) << 32 | (uint32_t)~i;
}
__device__ __forceinline__ float value_of(uint32_t o) {
    return __uint_as_float(o ^ ((o >> 31) ? 0x80000000u : 0xFFFFFFFFu));
}

// x of another lane, by a move within the vector unit: within rows of 16 lanes, then row to row (lanes that get
// nothing keep `old`).  After the six moves of STRIDE_WAVE_STEPS lane 63 has the result over the wave.
template <int Ctrl, int Rows>
__device__ __forceinline__ uint32_t moved(uint32_t old, uint32_t x) {
    return __builtin_amdgcn_update_dpp(old, x, Ctrl, Rows, 0xF, false);
}
#define STRIDE_WAVE_STEPS(S) S(0x111, 0xF) S(0x112, 0xF) S(0x114, 0xF) S(0x118, 0xF) S(0x142, 0xA) S(0x143, 0xC)

__device__ __forceinline__ uint64_t wave_max(uint64_t x) {
#define S(C, R)                                                                                                     \
    {                                                                                                               \
        const uint64_t y = (uint64_t)moved<C, R>(0, (uint32_t)(x >> 32)) << 32 | moved<C, R>(0, (uint32_t)x);       \
        x = x > y ? x : y;                                                                                          \
    }
    STRIDE_WAVE_STEPS(S)
#undef S
    return (uint64_t)(uint32_t)__builtin_amdgcn_readlane((int)(x >> 32), kWave - 1) << 32 |
           (uint32_t)__builtin_amdgcn_readlane((int)x, kWave - 1);
}
__device__ __forceinline__ float wave_max(float x) {
    const uint32_t low = 0xFF800000u;
#define S(C, R) x = fmaxf(x, __uint_as_float(moved<C, R>(low, __float_as_uint(x))));
    STRIDE_WAVE_STEPS(S)
#undef S
    return __uint_as_float((uint32_t)__builtin_amdgcn_readlane((int)__float_as_uint(x), kWave - 1));
}
// Inclusive sum over the lanes.
__device__ __forceinline__ uint32_t wave_upto(uint32_t x) {
#define S(C, R) x += moved<C, R>(0, x);
    STRIDE_WAVE_STEPS(S)
#undef S
    return x;
}

// Over the workgroup; every thread has the result.  A barrier on both sides.
__device__ __forceinline__ uint64_t block_max(uint64_t x, Shared &sh) {
    x = wave_max(x);
    __syncthreads();
    if ((threadIdx.x & (kWave - 1)) == 0) sh.wave64[threadIdx.x / kWave] = x;
    __syncthreads();
    x = sh.wave64[0];
#pragma unroll
    for (int i = 1; i < kWaves; ++i) x = sh.wave64[i] > x ? sh.wave64[i] : x;
    return x;
}
// The largest of two values at once.
__device__ __forceinline__ float2 block_max2(float x, float y, Shared &sh) {
    float2 r = make_float2(wave_max(x), wave_max(y));
    __syncthreads();
    if ((threadIdx.x & (kWave - 1)) == 0) sh.wavef[threadIdx.x / kWave] = r;
    __syncthreads();
#pragma unroll
    for (int i = 0; i < kWaves; ++i) {
        r.x = fmaxf(r.x, sh.wavef[i].x);
        r.y = fmaxf(r.y, sh.wavef[i].y);
    }
    return r;
}
__device__ __forceinline__ double block_sum(double x, Shared &sh) {
#pragma unroll
    for (int o = kWave / 2; o > 0; o >>= 1) x += __shfl_xor(x, o, kWave);
    __syncthreads();
    if ((threadIdx.x & (kWave - 1)) == 0) sh.waved[threadIdx.x / kWave] = x;
    __syncthreads();
    x = sh.waved[0];
#pragma unroll
    for (int i = 1; i < kWaves; ++i) x += sh.waved[i];
    return x;
}
// Sum of the lower threads' x; `all` is everyone's.
__device__ __forceinline__ uint64_t block_before(uint64_t x, uint64_t &all, Shared &sh) {
    const int lane = threadIdx.x & (kWave - 1), wave = threadIdx.x / kWave;
    uint64_t upto = x;
#pragma unroll
    for (int o = 1; o < kWave; o <<= 1) {
        const uint64_t y = __shfl_up((unsigned long long)upto, o, kWave);
        if (lane >= o) upto += y;
    }
    __syncthreads();
    if (lane == kWave - 1) sh.wave64[wave] = upto;
    __syncthreads();
    uint64_t before = upto - x;
    all = 0;
#pragma unroll
    for (int i = 0; i < kWaves; ++i) {
        if (i < wave) before += sh.wave64[i];
        all += sh.wave64[i];
    }
    return before;
}

template <int DT>
__device__ __forceinline__ void widen(const u32x4 &w, float *x) {
#pragma unroll
    for (int i = 0; i < 4; ++i) {
        if (DT == STRIDE_BF16) {
            x[2 * i] = __uint_as_float(w[i] << 16);
            x[2 * i + 1] = __uint_as_float(w[i] & 0xFFFF0000u);
        } else {
            x[i] = __uint_as_float(w[i]);
        }
    }
}

// A row's words of 16 bytes: every thread takes each kThreads-th, Flight of them on their way at once.
constexpr int kFlight = 8;
template <int DT>
struct Row {
    static constexpr int E = Elem<DT>::n;
    const u32x4 *p;
    int32_t vocab;
    __device__ __forceinline__ u32x4 load(int i) const {  // -inf past the row, and in the last word's padding
        const uint32_t none = DT == STRIDE_BF16 ? 0xFF80FF80u : 0xFF800000u;
        u32x4 x = {none, none, none, none};
        if (i * E < vocab) x = p[i];
        return x;
    }
    __device__ __forceinline__ u32x4 masked(u32x4 x, int i) const {
        const int n = vocab - i * E;
        if (n < E) {
#pragma unroll
            for (int e = 0; e < 4; ++e) {
                if (DT == STRIDE_BF16) {
                    if (2 * e >= n) x[e] = 0xFF80FF80u;
                    else if (2 * e + 1 >= n) x[e] = (x[e] & 0xFFFFu) | 0xFF800000u;
                } else if (e >= n) {
                    x[e] = 0xFF800000u;
                }
            }
        }
        return x;
    }
    // f(word, index of its first entry) for this thread's words in ascending order, and for words past the row, all
    // of them -inf, so that every thread has the same number.
    template <int U, class F>
    __device__ __forceinline__ void each(F f) const {
        const int nw = (vocab + E - 1) / E;
        for (int i0 = threadIdx.x; i0 - (int)threadIdx.x < nw; i0 += kThreads * U) {
            u32x4 x[U];
#pragma unroll
            for (int u = 0; u < U; ++u) x[u] = load(i0 + u * kThreads);
#pragma unroll
            for (int u = 0; u < U; ++u) f(masked(x[u], i0 + u * kThreads), (i0 + u * kThreads) * E);
        }
    }
};

typedef short i16x2 __attribute__((ext_vector_type(2)));
typedef unsigned short u16x2 __attribute__((ext_vector_type(2)));

// The largest value seen and whether any was NaN or +inf.  bf16 takes two entries per step by their bits: as signed
// numbers those of values from 0 on are in order (and NaN and +inf are the largest), as unsigned ones those below are
// in reverse order, the least of all where no value from 0 on is there, and negative NaN are the largest.
template <int DT>
struct Largest;
template <>
struct Largest<STRIDE_BF16> {
    i16x2 top = {-32768, -32768};
    u16x2 least = {0xFFFF, 0xFFFF}, most = {0, 0};
    __device__ __forceinline__ void add(const u32x4 &w) {
#pragma unroll
        for (int i = 0; i < 4; ++i) {
            const uint32_t x = w[i];  // a bit cast of the element itself takes the vector's first
            top = __builtin_elementwise_max(top, __builtin_bit_cast(i16x2, x));
            least = __builtin_elementwise_min(least, __builtin_bit_cast(u16x2, x));
            most = __builtin_elementwise_max(most, __builtin_bit_cast(u16x2, x));
        }
    }
    __device__ __forceinline__ bool bad() const {
        const short t = top[0] > top[1] ? top[0] : top[1];
        const unsigned short m = most[0] > most[1] ? most[0] : most[1];
        return t >= 0x7F80 || m > 0xFF80;
    }
    __device__ __forceinline__ float value() const {
        const short t = top[0] > top[1] ? top[0] : top[1];
        const unsigned short l = least[0] < least[1] ? least[0] : least[1];
        return __uint_as_float((uint32_t)(t >= 0 ? (unsigned short)t : l) << 16);
    }
};
template <>
struct Largest<STRIDE_F32> {
    float top = -INFINITY;
    bool odd = false;
    __device__ __forceinline__ void add(const u32x4 &w) {
#pragma unroll
        for (int i = 0; i < 4; ++i) {
            const float x = __uint_as_float(w[i]);
            odd |= !(x < INFINITY);
            top = fmaxf(top, x);
        }
    }
    __device__ __forceinline__ bool bad() const { return odd; }
    __device__ __forceinline__ float value() const { return top; }
};

// A row's largest key so far with its index (0: none), and whether it has NaN or +inf (in first_entry) or what was
// asked for could be told (in choose).
struct Found {
    uint64_t best;
    bool yes;
};

// The row's first entry in the order, and whether the row has NaN or +inf.
template <int DT>
__device__ __attribute__((noinline)) Found first_entry(const Row<DT> row, Shared &sh) {
    bool bad = false;
    float top = -INFINITY;
    int at = -1;
    row.template each<4>([&](const u32x4 &w, int i) __attribute__((always_inline)) {
        float x[Elem<DT>::n];
        widen<DT>(w, x);
#pragma unroll
        for (int e = 0; e < Elem<DT>::n; ++e) {
            bad |= !(x[e] < INFINITY);
            if (x[e] > top) {
                top = x[e];
                at = i + e;
            }
        }
    });
    return {block_max(at < 0 ? (uint64_t)0 : entry(top, at), sh), bad};
}

// s - log noise of one entry, in units of log 2 (s2 = s log2 e).
__device__ __forceinline__ float race(float s2, float noise) { return s2 - lg2_all(noise); }

// The winner among entries as they come, unfiltered.  Keys are relative to `ref`, one of the thread's own entries, which
// moves up when a later one passes it by more than kFar (in units of log 2): a key's rounding is that of a number of that
// size, 4e-6 at most, whatever is masked by large values before or after and at any temperature.
constexpr float kFar = 32.0f;
template <int DT>
struct Race {
    static constexpr int E = Elem<DT>::n;
    float ref = -INFINITY, top = -INFINITY;
    int at = -1;
    __device__ __forceinline__ void add(const float *x, const u32x4 *noise, int i, float c) {
        float m = x[0];
#pragma unroll
        for (int e = 1; e < E; ++e) m = fmaxf(m, x[e]);
        if ((m - ref) * c > kFar) {
            if (top < INFINITY) top += (ref - m) * c;
            ref = m;
        }
#pragma unroll
        for (int e = 0; e < E; ++e) {
            // no key above -inf for an entry of -inf, whatever its noise
            const float key = __builtin_fmaf(x[e] - ref, c, -lg2(__uint_as_float(noise[e / 4][e % 4])));
            if (key > top) {
                top = key;
                at = i + e;
            }
        }
    }
    // Over the wave: every lane has the winner (0: none) and what it is relative to.
    __device__ __forceinline__ uint64_t of_wave(float c, float &wave_ref) const {
        wave_ref = wave_max(at < 0 ? -INFINITY : ref);
        return wave_max(moved_to(at < 0 ? (uint64_t)0 : entry(top, at), ref, wave_ref, c));
    }
    // A winner relative to `from` as one relative to `to`.
    static __device__ __forceinline__ uint64_t moved_to(uint64_t x, float from, float to, float c) {
        const float key = value_of((uint32_t)(x >> 32));
        return x == 0 || key == INFINITY ? x : (uint64_t)ordered(key + (from - to) * c) << 32 | (uint32_t)x;
    }
};
// An infinite key: the winner's noise is 0 or below the normal range, and the row is passed again with its logarithm.
__device__ __forceinline__ bool infinite(uint64_t best) { return (uint32_t)(best >> 32) == ordered(INFINITY); }

// The largest key, relative to `ref`, of this thread's words among [begin, end), with its index (0: none).
template <int DT, int Threads>
__device__ __attribute__((noinline)) uint64_t race_again(const Row<DT> row, const float *noise, float c, float ref, int begin, int end) {
    constexpr int E = Elem<DT>::n;
    float top = -INFINITY;
    int at = -1;
    for (int i = begin + (int)threadIdx.x; i < end; i += Threads) {
        float x[E];
        widen<DT>(row.masked(row.load(i), i), x);
#pragma unroll
        for (int e = 0; e < E; ++e) {
            if (!(x[e] > -INFINITY)) continue;
            const float key = __builtin_fmaf(x[e] - ref, c, -lg2_all(noise[i * E + e]));
            if (key > top) {
                top = key;
                at = i * E + e;
            }
        }
    }
    return at < 0 ? (uint64_t)0 : entry(top, at);
}

struct Filter {
    float c, min_s2;     // log2 e / T; the least s that min-p keeps, in units of log 2
    float top, top_p;    // top: the row's largest z
    int k;               // 0: all
    bool p;
};
// s in units of log 2: 0 for the largest z, whatever its size and the temperature.
__device__ __forceinline__ float s2_of(const Filter &f, float x) { return (x - f.top) * f.c; }
// Mass of an entry in units of 2^-40 of the largest one's.
__device__ __forceinline__ uint64_t mass_of(const Filter &f, float x) { return (uint64_t)(ex2(s2_of(f, x)) * kMassUnit); }

// Filtered row, exact for any row: the last kept value and how many entries of that value are kept, by 11-bit
// digits of the ordered key from the top, then the race among the kept ones.
template <int DT>
__device__ __attribute__((noinline)) uint64_t by_digits(const Row<DT> row, const float *noise, const Filter f, Shared &sh) {
    constexpr int E = Elem<DT>::n, kLow = Elem<DT>::low_bits, kDigits = Elem<DT>::digits;
    uint32_t last = 0;          // key of the last kept value, without its low bits
    uint64_t keep_equal = ~0ull;  // how many of that value
    uint64_t equal = 0;
    double whole = -1.0;        // the mass top-p refers to
    for (int goal = 0; goal < 2; ++goal) {  // 0: top-k, 1: top-p
        if (goal == 0 ? f.k == 0 : !f.p) continue;
        uint32_t prefix = 0;
        uint64_t above_n = 0, above_m = 0, bin_n = 0, bin_m = 0;
        double target = 0.0;
        int shift = 32 - kLow;
        for (int d = 0; d < kDigits; ++d) {
            const int bits = shift < 11 ? shift : 11;
            shift -= bits;
            __syncthreads();
            for (int i = threadIdx.x; i < kBins; i += kThreads) {
                sh.count[i] = 0;
                sh.mass[i] = 0;
            }
            __syncthreads();
            row.template each<2>([&](const u32x4 &w, int) __attribute__((always_inline)) {
                float x[E];
                widen<DT>(w, x);
#pragma unroll
                for (int e = 0; e < E; ++e) {
                    const uint32_t o = ordered(x[e]) >> kLow;
                    // -inf entries (and those past the row) are never kept
                    if (x[e] > -INFINITY && (d == 0 || (o >> (shift + bits)) == prefix)) {
                        const uint32_t b = (o >> shift) & ((1u << bits) - 1);
                        atomicAdd(&sh.count[b], 1u);
                        const uint64_t m = mass_of(f, x[e]);
                        if (m) atomicAdd(reinterpret_cast<unsigned long long *>(&sh.mass[b]), (unsigned long long)m);
                    }
                }
            });
            __syncthreads();
            // two bins per thread, the largest values first
            const int b0 = kBins - 1 - 2 * (int)threadIdx.x, b1 = b0 - 1;
            const uint64_t n0 = sh.count[b0], n1 = sh.count[b1], m0 = sh.mass[b0], m1 = sh.mass[b1];
            uint64_t all_n, all_m;
            uint64_t bn = block_before(n0 + n1, all_n, sh) + above_n;
            uint64_t bm = block_before(m0 + m1, all_m, sh) + above_m;
            if (d == 0) {
                if (goal == 1) {
                    if (whole < 0.0) whole = (double)all_m;
                    target = (double)f.top_p * whole;
                    if (!(target > 0.0)) target = 0.5;  // the first entry alone
                }
                if (threadIdx.x == 0) sh.found = ~0u;
                __syncthreads();
            }
#pragma unroll
            for (int j = 0; j < 2; ++j) {
                const uint64_t n = j ? n1 : n0, m = j ? m1 : m0;
                const bool here = goal == 0 ? bn < (uint64_t)f.k && bn + n >= (uint64_t)f.k
                                            : (double)bm < target && (double)(bm + m) >= target;
                if (here) {
                    sh.found = (uint32_t)(j ? b1 : b0);
                    sh.above_count = (uint32_t)bn;
                    sh.above_mass = bm;
                    sh.found_u64 = m;
                    sh.n_list = (uint32_t)n;
                }
                bn += n;
                bm += m;
            }
            __syncthreads();
            if (sh.found == ~0u) break;  // fewer finite entries than k: all of them
            prefix = prefix << bits | sh.found;
            above_n = sh.above_count;
            above_m = sh.above_mass;
            bin_n = sh.n_list;
            bin_m = sh.found_u64;
        }
        if (sh.found == ~0u) {
            __syncthreads();
            continue;
        }
        const uint64_t each = bin_n ? bin_m / bin_n : 0;  // all of the last bin's entries are one value
        uint64_t r;
        if (goal == 0) {
            r = (uint64_t)f.k - above_n;
            whole = (double)(above_m + r * each);
        } else {
            r = (uint64_t)ceil((target - (double)above_m) / (double)each);
            r = r < 1 ? 1 : r;
        }
        // top-p's end lies in top-k's part, or at the same value with no more entries
        if (prefix == last && keep_equal < r) r = keep_equal;
        last = prefix;
        keep_equal = r;
        equal = bin_n;
        __syncthreads();
    }
    const bool some_equal = keep_equal < equal;  // the lowest indices of the last value
    uint64_t best = 0, run = 0;
    row.template each<1>([&](const u32x4 &w, int i) __attribute__((always_inline)) {
        float x[E];
        widen<DT>(w, x);
        uint64_t mine = 0, before = 0;
        if (some_equal) {  // the same for the whole workgroup
#pragma unroll
            for (int e = 0; e < E; ++e) mine += x[e] > -INFINITY && (ordered(x[e]) >> kLow) == last;
            uint64_t all;
            before = run + block_before(mine, all, sh);
            run += all;
        }
#pragma unroll
        for (int e = 0; e < E; ++e) {
            const uint32_t o = ordered(x[e]) >> kLow;
            bool keep = x[e] > -INFINITY && o >= last;
            if (some_equal && keep && o == last) keep = before++ < keep_equal;
            const float s2 = s2_of(f, x[e]);
            if (keep && s2 >= f.min_s2) {
                const float key = race(s2, noise[i + e]);
                if (key > -INFINITY) {
                    const uint64_t y = entry(key, i + e);
                    best = y > best ? y : best;
                }
            }
        }
    });
    return block_max(best, sh);
}

// The row's token from its n gathered entries, all of those from some value on: the largest key of the kept ones.
// None if top-p's mass goes beyond them, which only a list that is not `whole_list` can say; `whole` is the mass
// that top-p refers to, but for rows with top-k, whose own it is.
__device__ __attribute__((noinline)) Found choose(uint32_t n, bool whole_list, double whole, const float *noise, const Filter f,
                                                  Shared &sh) {
    const int tid = threadIdx.x;
    const bool row_mass = f.p && !f.k;
    uint64_t *list = sh.mass;
    // ---- of each entry: its rank, the mass before it and its own ----
    const int per = n <= kCount ? 1 : 2;
    uint64_t x[2] = {0, 0}, m[2] = {0, 0}, before[2] = {0, 0}, all = 0;
    uint32_t rank[2] = {0, 0};
    if (per == 1) {
        constexpr uint32_t kStep = 8;  // entries asked for at once
        if (tid < (int)n) {
            x[0] = list[tid];
            m[0] = mass_of(f, value_of((uint32_t)(x[0] >> 32)));
        }
        if (tid < (int)(n + kStep - 1)) {
            sh.pair[tid][0] = x[0];
            sh.pair[tid][1] = m[0];
        }
        __syncthreads();
        if ((tid & ~(kWave - 1)) < (int)n) {  // the waves that have entries
            for (uint32_t i = 0; i < n; i += kStep) {
                ulonglong2 y[kStep];
#pragma unroll
                for (uint32_t j = 0; j < kStep; ++j) y[j] = *reinterpret_cast<const ulonglong2 *>(sh.pair[i + j]);
#pragma unroll
                for (uint32_t j = 0; j < kStep; ++j) {
                    const bool more = y[j].x > x[0];
                    rank[0] += more;
                    before[0] += more ? y[j].y : 0;
                }
            }
            const uint32_t last = (f.k && (uint32_t)f.k < n ? (uint32_t)f.k : n) - 1;
            if (tid < (int)n && rank[0] == last) sh.above_mass = before[0] + m[0];
        }
        __syncthreads();
        all = sh.above_mass;
    } else {  // sorted, largest first (a bitonic network)
        uint32_t size = 2;
        while (size < n) size *= 2;
        for (uint32_t i = n + tid; i < size; i += kThreads) list[i] = 0;
        for (uint32_t span = 2; span <= size; span *= 2)
            for (uint32_t step = span / 2; step > 0; step /= 2) {
                __syncthreads();
                for (uint32_t t = tid; t < size / 2; t += kThreads) {
                    const uint32_t i = 2 * t - (t & (step - 1)), j = i + step;
                    const uint64_t u = list[i], v = list[j];
                    if ((u < v) == ((i & span) == 0)) {
                        list[i] = v;
                        list[j] = u;
                    }
                }
            }
        __syncthreads();
#pragma unroll
        for (int j = 0; j < 2; ++j) {
            rank[j] = 2 * tid + j;
            x[j] = rank[j] < n ? list[rank[j]] : 0;
            if (rank[j] < n && (f.k == 0 || rank[j] < (uint32_t)f.k))
                m[j] = mass_of(f, value_of((uint32_t)(x[j] >> 32)));
        }
        before[0] = block_before(m[0] + m[1], all, sh);
        before[1] = before[0] + m[0];
    }
    if (!row_mass) whole = (double)all;
    const double target = (double)f.top_p * whole;
    if (!whole_list && row_mass && (double)all < target) return {0, false};
    // ---- the race among the kept ones ----
    uint64_t best = 0;
#pragma unroll
    for (int j = 0; j < 2; ++j) {
        if (j >= per || x[j] == 0) continue;
        const float s2 = s2_of(f, value_of((uint32_t)(x[j] >> 32)));
        if (rank[j] == 0 || ((f.k == 0 || rank[j] < (uint32_t)f.k) && (!f.p || (double)before[j] < target) && s2 >= f.min_s2)) {
            const int32_t id = (int32_t)~(uint32_t)x[j];
            const float key = race(s2, noise[id]);
            if (key > -INFINITY) {
                const uint64_t y = entry(key, id);
                best = y > best ? y : best;
            }
        }
    }
    return {block_max(best, sh), true};
}

// The value at or below which `want` of the threads' maxima lie at least: the lower border of the bin of a histogram
// over [low, top] that holds the want-th largest; -inf where there is none.  Every wave finds it for itself.
__device__ __forceinline__ float cut_of(const uint32_t *count, int want, float top, float scale) {
    const int lane = threadIdx.x & (kWave - 1);
    const uint4 n = *reinterpret_cast<const uint4 *>(&count[4 * lane]);
    const uint32_t mine = n.x + n.y + n.z + n.w, upto = wave_upto(mine);
    const uint64_t have = __ballot(upto >= (uint32_t)want);
    if (!have) return -INFINITY;
    const int at = __builtin_ctzll(have);
    uint32_t u = upto - mine;
    int bin = 4 * lane;
    u += n.x;
    if (u < (uint32_t)want) u += n.y, ++bin;
    if (u < (uint32_t)want) u += n.z, ++bin;
    if (u < (uint32_t)want) ++bin;
    // and what the roundings of a bin's number may be off
    return top - ((float)__builtin_amdgcn_readlane(bin, at) + 1.01f) / scale;
}

// A row's parameters; false if they are out of range.
__device__ __forceinline__ bool parameters(const SampleArgs &a, int64_t r, float &temp, float &min_p, bool &plain, Filter &f) {
    temp = a.temperature ? a.temperature[r] : 0.0f;
    min_p = a.min_p ? a.min_p[r] : 0.0f;
    const float top_p = a.top_p ? a.top_p[r] : 1.0f;
    const int32_t top_k = a.top_k ? a.top_k[r] : 0;
    // below 2^-100 the quotients of distinct logits are infinite either way
    f.c = kLog2e / fmaxf(temp, 0x1p-100f);
    f.k = top_k > 0 && top_k < a.vocab ? top_k : 0;
    f.p = top_p < 1.0f;
    f.top_p = top_p;
    f.min_s2 = min_p > 0.0f ? lg2_all(min_p) : -INFINITY;
    plain = f.k == 0 && !f.p && min_p == 0.0f;
    return temp >= 0.0f && temp < INFINITY && top_p == top_p && min_p >= 0.0f;
}

// The least value that min-p keeps beside `top`, or somewhat less.
__device__ __forceinline__ float min_p_cut(const Filter &f, float top) {
    return top + fminf(f.min_s2, 0.0f) / f.c * 1.0001f - 1e-6f * fabsf(top);
}

// ---- few rows ----
// First kernel where a row for each CU would leave most of them idle: n_parts workgroups of a row look through a
// sixteenth of it or more each, as the row's workgroup would (thread maxima, a cut, the entries above it; the first
// entry, or the largest key), and hand on what they found.  One filtered row of 151,936 bf16 logits takes 19 us in one
// workgroup, 13 in sixteen parts.
template <int DT>
__global__ __launch_bounds__(kPartThreads) void sample_parts_kernel(SampleArgs a) {
    constexpr int E = Elem<DT>::n, U = 2, kPartWaves = kPartThreads / kWave;
    __shared__ __attribute__((aligned(16))) uint32_t s_count[kCutBins];
    __shared__ uint64_t s_best[kPartWaves], s_list[kPartList];
    __shared__ float2 s_ends[kPartWaves];
    __shared__ float s_sum[kPartWaves];
    __shared__ uint32_t s_n, s_bad;
    const int64_t b = block_index<kPartThreads>();
    if (b >= a.n_rows * a.n_parts) return;
    const int64_t r = b / a.n_parts;
    const int part = (int)(b - r * a.n_parts), tid = threadIdx.x, lane = tid & (kWave - 1), wave = tid / kWave;
    float temp, min_p;
    bool plain;
    Filter f;
    const bool good = parameters(a, r, temp, min_p, plain, f);
    const Row<DT> row = {reinterpret_cast<const u32x4 *>(static_cast<const char *>(a.logits) + r * a.ld * (DT == STRIDE_BF16 ? 2 : 4)),
                         a.vocab};
    const float *noise = a.noise + r * a.noise_ld;
    Part &out = a.parts[b];
    const int words = (a.vocab + E - 1) / E, per = (words + a.n_parts - 1) / a.n_parts;
    const int begin = part * per, end = begin + per < words ? begin + per : words;
    // the thread's first words, all of them where parts are not larger, stay in registers for the second pass
    constexpr int kHeld = 5;
    u32x4 held[kHeld];
#pragma unroll
    for (int u = 0; u < kHeld; ++u) {
        const int i = begin + tid + u * kPartThreads;
        held[u] = row.masked(row.load(i < end ? i : words), i);
    }
    auto each = [&](auto f) __attribute__((always_inline)) {  // f(word, its first entry's index) in ascending order
#pragma unroll
        for (int u = 0; u < kHeld; ++u) f(held[u], (begin + tid + u * kPartThreads) * E);
        for (int i0 = begin + tid + kHeld * kPartThreads; i0 < end; i0 += kPartThreads * U) {
            u32x4 x[U];
#pragma unroll
            for (int u = 0; u < U; ++u) x[u] = row.load(i0 + u * kPartThreads < end ? i0 + u * kPartThreads : words);
#pragma unroll
            for (int u = 0; u < U; ++u) f(row.masked(x[u], i0 + u * kPartThreads), (i0 + u * kPartThreads) * E);
        }
    };
    if (!good) return;  // the row's workgroup says so
    s_count[tid] = 0;
    if (tid == 0) {
        s_n = 0;
        s_bad = 0;
    }
    __syncthreads();
    Largest<DT> largest;
    if (temp == 0.0f || plain) {
        Race<DT> race;
        const u32x4 *nw = reinterpret_cast<const u32x4 *>(noise);
        each([&](const u32x4 &w, int i) __attribute__((always_inline)) {
            float x[E];
            widen<DT>(w, x);
            largest.add(w);
            if (temp > 0.0f) {
                u32x4 q[E / 4];
#pragma unroll
                for (int j = 0; j < E / 4; ++j) {
                    q[j] = u32x4{};
                    if (i + 4 * j < a.vocab) q[j] = __builtin_nontemporal_load(nw + i / 4 + j);
                }
                race.add(x, q, i, f.c);
            } else {
#pragma unroll
                for (int e = 0; e < E; ++e)
                    if (x[e] > race.top) {
                        race.top = x[e];
                        race.at = i + e;
                    }
            }
        });
        float ref = 0.0f;
        uint64_t m;
        if (temp > 0.0f) m = race.of_wave(f.c, ref);
        else m = wave_max(race.at < 0 ? (uint64_t)0 : entry(race.top, race.at));
        if (lane == 0) {
            s_best[wave] = m;
            s_ends[wave].x = ref;
        }
        if (largest.bad()) s_bad = 1;
        __syncthreads();
        uint64_t best = 0;
        ref = s_ends[0].x;
#pragma unroll
        for (int i = 1; i < kPartWaves; ++i) ref = fmaxf(ref, s_ends[i].x);
#pragma unroll
        for (int i = 0; i < kPartWaves; ++i) {
            const uint64_t y = temp > 0.0f ? Race<DT>::moved_to(s_best[i], s_ends[i].x, ref, f.c) : s_best[i];
            best = y > best ? y : best;
        }
        if (temp > 0.0f && infinite(best)) {  // the same for the whole workgroup
            const uint64_t again = wave_max(race_again<DT, kPartThreads>(row, noise, f.c, ref, begin, end));
            __syncthreads();
            if (lane == 0) s_best[wave] = again;
            __syncthreads();
            best = s_best[0];
#pragma unroll
            for (int i = 1; i < kPartWaves; ++i) best = s_best[i] > best ? s_best[i] : best;
        }
        if (tid == 0) {
            out.first = best;
            out.at = best ? (int32_t)~(uint32_t)best : -1;
            out.ref = ref;
            out.bad = s_bad;
        }
        return;
    }
    each([&](const u32x4 &w, int) __attribute__((always_inline)) { largest.add(w); });
    const float mine = largest.value();
    const float wm = wave_max(mine), wl = wave_max(mine > -INFINITY ? -mine : -INFINITY);
    if (lane == 0) s_ends[wave] = make_float2(wm, wl);
    if (largest.bad()) s_bad = 1;
    __syncthreads();
    float top = -INFINITY, low = -INFINITY;
#pragma unroll
    for (int i = 0; i < kPartWaves; ++i) {
        top = fmaxf(top, s_ends[i].x);
        low = fmaxf(low, s_ends[i].y);
    }
    low = -low;
    f.top = top;
    const bool row_mass = f.p && !f.k;
    const float scale = low < top ? (float)(kCutBins - 1) / (top - low) : 0.0f;
    const bool sharp = scale > 0.0f && scale < INFINITY;
    if (sharp && mine > -INFINITY) atomicAdd(&s_count[min((int)((top - mine) * scale), kCutBins - 1)], 1u);
    __syncthreads();
    float cut = -INFINITY;
    // of the row's first k a part has a share: the cut leaves it twice that and some, and the row's workgroup goes by the
    // highest of the parts' cuts, or falls back where that does not reach k
    const int want = f.k ? min(f.k, 2 * f.k / a.n_parts + 16) : f.p ? kPartGuess : 0;
    if (want > 0 && want <= kPartThreads && sharp) cut = cut_of(s_count, want, top, scale);
    if (min_p > 0.0f && !f.k) cut = min_p_cut(f, top);
    float sum = 0.0f;
    if (top > -INFINITY) {
        each([&](const u32x4 &w, int i) __attribute__((always_inline)) {
            float x[E];
            widen<DT>(w, x);
            float m = x[0];
#pragma unroll
            for (int e = 1; e < E; ++e) m = fmaxf(m, x[e]);
            if (m >= cut && m > -INFINITY) {
                const float least = fmaxf(cut, -3.4028235e38f);
#pragma unroll
                for (int e = 0; e < E; ++e)
                    if (x[e] >= least) {
                        const uint32_t at = atomicAdd(&s_n, 1u);
                        if (at < kPartList) s_list[at] = entry(x[e], i + e);
                    }
            }
            if (row_mass) {
                float y = 0.0f;
#pragma unroll
                for (int e = 0; e < E; ++e) y += ex2(s2_of(f, x[e]));
                sum += y;
            }
        });
    }
    if (row_mass) {
#pragma unroll
        for (int o = kWave / 2; o > 0; o >>= 1) sum += __shfl_xor(sum, o, kWave);
        if (lane == 0) s_sum[wave] = sum;
    }
    __syncthreads();
    const uint32_t n = s_n;
    for (uint32_t i = tid; i < n && i < kPartList; i += kPartThreads) out.list[i] = s_list[i];
    if (tid == 0) {
        out.top = top;
        out.cut = cut;
        out.n = n;
        out.bad = s_bad;
        out.sum = 0.0f;
        if (row_mass) {
#pragma unroll
            for (int i = 0; i < kPartWaves; ++i) out.sum += s_sum[i];
        }
    }
}

// The row's token from what its parts left.  None where the lists do not hold all that may be kept (a part with more
// entries than its list, a nucleus beyond them); of a row with NaN or +inf, or only -inf, the entry is 0.
template <int DT>
__device__ __forceinline__ Found from_parts(const SampleArgs &a, int64_t r, const Row<DT> &row, float temp, float min_p,
                                            bool plain, Filter f, Shared &sh) {
    const Part *parts = a.parts + r * a.n_parts;
    const float *noise = a.noise + r * a.noise_ld;
    const int tid = threadIdx.x, lane = tid & (kWave - 1);
    // Everything that may be needed is asked for at once (entries past a list's end are not used): every wave has
    // the parts' heads, a lane one of them, and a thread two entries of the lists.
    Part head = {};
    const bool mine = lane < a.n_parts;
    if (mine) __builtin_memcpy(&head, &parts[lane], offsetof(Part, list));
    uint64_t e[2];
#pragma unroll
    for (int j = 0; j < 2; ++j) {
        const int i = tid + j * kThreads;
        e[j] = i < a.n_parts * kPartList ? parts[i / kPartList].list[i % kPartList] : 0;
    }
    if (__any(mine && head.bad)) return {0, true};
    if (temp == 0.0f) return {wave_max(mine ? head.first : (uint64_t)0), true};
    if (plain) {  // the parts' winners, relative to one point
        const int at = mine ? head.at : -1;
        const float ref = wave_max(at >= 0 ? head.ref : -INFINITY);
        uint64_t x = 0;
        if (at >= 0) {
            const float z = DT == STRIDE_BF16 ? __uint_as_float((uint32_t)reinterpret_cast<const uint16_t *>(row.p)[at] << 16)
                                              : reinterpret_cast<const float *>(row.p)[at];
            const float key = __builtin_fmaf(z - ref, f.c, -lg2_all(noise[at]));
            if (key > -INFINITY) x = entry(key, at);
        }
        const uint64_t best = wave_max(x);
        return {best, best != 0};  // no noise that can win: the first entry, which the parts do not have
    }
    f.top = wave_max(mine ? head.top : -INFINITY);
    if (!(f.top > -INFINITY)) return {0, true};
    if (__any(mine && head.n > kPartList)) return {0, false};
    const float cut = wave_max(mine ? head.cut : -INFINITY);  // all entries from here on are in the lists
    double whole = 0.0;
    if (f.p && !f.k) {
        double x = mine && head.top > -INFINITY ? (double)head.sum * (double)ex2((head.top - f.top) * f.c) : 0.0;
#pragma unroll
        for (int o = kMaxParts / 2; o > 0; o >>= 1) x += __shfl_xor(x, o, kWave);
        whole = __shfl(x, 0, kWave) * (double)kMassUnit;
    }
    // all entries from `cut` on are in the lists: this thread's two of them, and a histogram over them for a cut nearer
    // to the k-th largest (the parts together hand on many times k)
    const float scale = cut > -INFINITY && cut < f.top ? (float)(kCutBins - 1) / (f.top - cut) : 0.0f;
    const int want = f.k ? f.k : f.p && min_p == 0.0f ? kGuess[0] : 0;
    const bool sharp = want > 0 && scale > 0.0f && scale < INFINITY;
    float z[2];
#pragma unroll
    for (int j = 0; j < 2; ++j) {
        const int i = tid + j * kThreads, p = i / kPartList;  // the same part for 128 threads
        const uint32_t n = __shfl(head.n, p < kMaxParts ? p : 0, kWave);
        const bool there = p < a.n_parts && (uint32_t)(i % kPartList) < n;
        z[j] = there ? value_of((uint32_t)(e[j] >> 32)) : -INFINITY;
        if (z[j] < cut) z[j] = -INFINITY;
        if (sharp && z[j] > -INFINITY) atomicAdd(&sh.count[min((int)((f.top - z[j]) * scale), kCutBins - 1)], 1u);
    }
    __syncthreads();
    const float near = sharp ? cut_of(sh.count, want, f.top, scale) : -INFINITY;
#pragma unroll 1
    for (int tries = near > cut ? 0 : 1; tries < 2; ++tries) {  // then all of them
        const float from = tries == 0 ? near : cut;
#pragma unroll
        for (int j = 0; j < 2; ++j)
            if (z[j] > -INFINITY && z[j] >= from) sh.mass[atomicAdd(&sh.n_list, 1u)] = e[j];
        __syncthreads();
        const bool whole_list = from == -INFINITY || (min_p > 0.0f && !f.k);
        if (f.k && !whole_list && sh.n_list < (uint32_t)f.k) return {0, false};
        const Found x = choose(sh.n_list, whole_list, whole, noise, f, sh);
        if (x.yes) return {x.best, x.best != 0};
        __syncthreads();
        if (tid == 0) sh.n_list = 0;
        __syncthreads();
    }
    return {0, false};
}

template <int DT, bool Parts>
__global__ __launch_bounds__(kThreads) void sample_kernel(SampleArgs a) {
    constexpr int E = Elem<DT>::n;
    __shared__ __attribute__((aligned(16))) Shared sh;
    const int64_t r = block_index<kThreads>();
    if (r >= a.n_rows) return;
    const int tid = threadIdx.x;
    const void *base = static_cast<const char *>(a.logits) + r * a.ld * (DT == STRIDE_BF16 ? 2 : 4);
    const Row<DT> row = {static_cast<const u32x4 *>(base), a.vocab};
    float temp, min_p;
    bool plain;
    Filter f;
    if (!parameters(a, r, temp, min_p, plain, f)) {
        if (tid == 0) {
            raise_flag(a.flags, STRIDE_FLAG_BAD_SAMPLING);
            a.ids[r] = -1;
        }
        return;
    }
    const float *noise = a.noise + r * a.noise_ld;

    bool bad = false;
    uint64_t best = 0;
    if (tid == 0) {
        sh.bad = 0;
        sh.n_list = 0;
    }
    if (tid < kCutBins) sh.count[tid] = 0;
    if (Parts) {
        __syncthreads();
        const Found x = from_parts<DT>(a, r, row, temp, min_p, plain, f, sh);
        if (x.yes) {
            if (tid == 0) {
                if (x.best == 0) raise_flag(a.flags, STRIDE_FLAG_NONFINITE);
                a.ids[r] = x.best ? (int32_t)~(uint32_t)x.best : -1;
            }
            return;
        }
        __syncthreads();
        if (tid == 0) sh.n_list = 0;
        if (tid < kCutBins) sh.count[tid] = 0;  // the parts' entries are in it
    }
    if (temp == 0.0f) {
        const Found x = first_entry<DT>(row, sh);
        best = x.best;
        bad = x.yes;
    } else if (plain) {
        Race<DT> race;
        const u32x4 *nw = reinterpret_cast<const u32x4 *>(noise);
        const int words = (a.vocab + E - 1) / E;
        Largest<DT> seen;
        constexpr int U = 2;  // words on their way with their random numbers: six loads of bf16 rows (twelve were no faster)
        for (int i0 = tid; i0 < words; i0 += kThreads * U) {
            u32x4 w[U], q[U][E / 4];
#pragma unroll
            for (int u = 0; u < U; ++u) {
                const int i = i0 + u * kThreads;
                w[u] = row.load(i);
#pragma unroll
                for (int j = 0; j < E / 4; ++j) {
                    q[u][j] = u32x4{};
                    if (i * E + 4 * j < a.vocab) q[u][j] = __builtin_nontemporal_load(nw + i * (E / 4) + j);
                }
            }
#pragma unroll
            for (int u = 0; u < U; ++u) {
                const int i = i0 + u * kThreads;
                float x[E];
                const u32x4 z = row.masked(w[u], i);
                seen.add(z);
                widen<DT>(z, x);
                race.add(x, q[u], i * E, f.c);
            }
        }
        bad |= seen.bad();
        float ref;
        best = race.of_wave(f.c, ref);
        if ((tid & (kWave - 1)) == 0) {
            sh.wave64[tid / kWave] = best;
            sh.wavef[tid / kWave].x = ref;
        }
        __syncthreads();
        ref = sh.wavef[0].x;
#pragma unroll
        for (int i = 1; i < kWaves; ++i) ref = fmaxf(ref, sh.wavef[i].x);
        best = 0;
#pragma unroll
        for (int i = 0; i < kWaves; ++i) {
            const uint64_t y = Race<DT>::moved_to(sh.wave64[i], sh.wavef[i].x, ref, f.c);
            best = y > best ? y : best;
        }
        if (infinite(best)) best = block_max(race_again<DT, kThreads>(row, noise, f.c, ref, 0, words), sh);
    } else {
        // ---- first pass: every thread's maximum ----
        Largest<DT> largest;
        row.template each<kFlight>([&](const u32x4 &w, int) __attribute__((always_inline)) { largest.add(w); });
        const float mine = largest.value();
        bad = largest.bad();
        if (bad) sh.bad = 1;
        const float2 ends = block_max2(mine, mine > -INFINITY ? -mine : -INFINITY, sh);
        f.top = ends.x;
        const float low = -ends.y;
        if (!sh.bad && f.top > -INFINITY) {
            // ---- the cut, the entries above it, and the row's mass for top-p alone ----
            const float scale = low < f.top ? (float)(kCutBins - 1) / (f.top - low) : 0.0f;
            const bool row_mass = f.p && !f.k, sharp = scale > 0.0f && scale < INFINITY;
            if (sharp && mine > -INFINITY) atomicAdd(&sh.count[min((int)((f.top - mine) * scale), kCutBins - 1)], 1u);
            __syncthreads();
            uint64_t *list = sh.mass;
            double whole = 0.0;
            bool fits = false;
#pragma unroll 1
            for (int tries = 0; tries < (row_mass && min_p == 0.0f ? 2 : 1) && !fits; ++tries) {
                float cut = -INFINITY;
                const int want = f.k ? f.k : f.p ? kGuess[tries] : 0;
                if (want > 0 && want <= kThreads && sharp) cut = cut_of(sh.count, want, f.top, scale);
                // min-p's own bound, where top-p does not ask for the mass of a top-k beyond it
                bool whole_list = cut == -INFINITY;
                if (min_p > 0.0f && !(f.k && f.p)) {
                    const float least = min_p_cut(f, f.top);
                    if (least >= cut || (row_mass && least > -INFINITY)) {
                        cut = least;
                        whole_list = true;
                    }
                }
                float sum = 0.0f;
                row.template each<kFlight>([&](const u32x4 &w, int i) __attribute__((always_inline)) {
                    float x[E];
                    widen<DT>(w, x);
                    float m = x[0];
#pragma unroll
                    for (int e = 1; e < E; ++e) m = fmaxf(m, x[e]);
                    if (m >= cut && m > -INFINITY) {
                        const float least = fmaxf(cut, -3.4028235e38f);
#pragma unroll
                        for (int e = 0; e < E; ++e)
                            if (x[e] >= least) {
                                const uint32_t at = atomicAdd(&sh.n_list, 1u);
                                if (at < kList) list[at] = entry(x[e], i + e);
                            }
                    }
                    if (row_mass && tries == 0) {
                        float y = 0.0f;
#pragma unroll
                        for (int e = 0; e < E; ++e) y += ex2(s2_of(f, x[e]));
                        sum += y;
                    }
                });
                if (row_mass && tries == 0) whole = block_sum((double)sum, sh) * (double)kMassUnit;
                __syncthreads();
                const uint32_t n = sh.n_list;
                fits = n <= kList && (whole_list || !f.k || n >= (uint32_t)f.k);
                if (!fits) break;
                const Found x = choose(n, whole_list, whole, noise, f, sh);
                best = x.best;
                fits = x.yes;
                if (!fits) {  // top-p alone, and the guess fell short
                    __syncthreads();
                    if (tid == 0) sh.n_list = 0;
                    __syncthreads();
                }
            }
            if (!fits) best = by_digits<DT>(row, noise, f, sh);
        }
    }
    __syncthreads();
    if (bad) sh.bad = 1;
    __syncthreads();
    bad = sh.bad != 0;
    if (best == 0 && !bad && temp > 0.0f) best = first_entry<DT>(row, sh).best;  // no noise that can win: the first entry
    if (tid == 0) {
        if (bad || best == 0) {
            raise_flag(a.flags, STRIDE_FLAG_NONFINITE);
            a.ids[r] = -1;
        } else {
            a.ids[r] = (int32_t)~(uint32_t)best;
        }
    }
}

}  // namespace

namespace {

// Workgroups per row of the first kernel: up to 1,024 over all rows, where the vocabulary has work for them; 1: there is
// none.  64 mixed rows of 151,936 bf16 logits and small nuclei take 27 us without, 20 in sixteen parts each; 256 rows fill the
// chip.
int parts_of(int64_t n_rows, int32_t vocab) {
    if (n_rows < 1 || n_rows > 128 || vocab < 16384) return 1;
    int64_t n = 1024 / n_rows;
    n = n < vocab / 4096 ? n : vocab / 4096;
    return (int)(n < kMaxParts ? n : kMaxParts);
}

}  // namespace

size_t sample_ws_bytes(int64_t n_rows, int32_t vocab) {
    const int parts = parts_of(n_rows, vocab);
    return parts > 1 ? (size_t)n_rows * parts * sizeof(Part) : 256;
}


hipError_t launch_sample(int64_t n_rows, int32_t vocab, int64_t ld, int32_t dtype, const void *logits,
                         const float *noise, int64_t noise_ld, const float *temperature,
                         const int32_t *top_k, const float *top_p, const float *min_p,
                         int32_t *token_ids, uint32_t *flags, void *ws, hipStream_t stream) {
    if (n_rows == 0) return hipSuccess;
    SampleArgs a;
    a.logits = logits;
    a.noise = noise;
    a.noise_ld = noise_ld;
    a.temperature = temperature;
    a.top_k = top_k;
    a.top_p = top_p;
    a.min_p = min_p;
    a.ids = token_ids;
    a.flags = flags;
    a.n_rows = n_rows;
    a.ld = ld;
    a.vocab = vocab;
    a.n_parts = parts_of(n_rows, vocab);
    a.parts = a.n_parts > 1 ? static_cast<Part *>(ws) : nullptr;
    if (a.parts) {
        const dim3 grid = grid_of(n_rows * a.n_parts, kPartThreads);
        if (dtype == STRIDE_BF16) sample_parts_kernel<STRIDE_BF16><<<grid, kPartThreads, 0, stream>>>(a);
        else sample_parts_kernel<STRIDE_F32><<<grid, kPartThreads, 0, stream>>>(a);
        const hipError_t e = hipGetLastError();
        if (e != hipSuccess) return e;
    }
    const dim3 grid = grid_of(n_rows, kThreads);
    if (dtype == STRIDE_BF16) {
        if (a.parts) sample_kernel<STRIDE_BF16, true><<<grid, kThreads, 0, stream>>>(a);
        else sample_kernel<STRIDE_BF16, false><<<grid, kThreads, 0, stream>>>(a);
    } else {
        if (a.parts) sample_kernel<STRIDE_F32, true><<<grid, kThreads, 0, stream>>>(a);
        else sample_kernel<STRIDE_F32, false><<<grid, kThreads, 0, stream>>>(a);
    }
    return hipGetLastError();
}

}  // namespace stride
