// attend.hip -- attention of each sequence's newest tokens over the paged cache.
//
// For a row (token, query head): o = sum_j p_j v_j with p the softmax of scale * q . k_j over the keys that the
// row sees, in one pass over K and V with a running reference point m and sum l: o and l are kept relative to
// exp2(m) and rescaled only when a key passes m by more than 2^kSlack (so p stays below 2^kSlack, and a
// block without a new maximum needs no exchange between lanes).
//
// Layout.  The query heads of a group and a sequence's new tokens are the rows of one small matrix, which
// every byte of K and V serves at once.  A work item is (sequence, key head, tile of 16 or 32 rows); the four waves of
// a workgroup take its keys in turn, 16 T at a time, each wave with a running state of its own, and join them
// through LDS at the item's end, in a fixed order.  Items are cut into units of one round of the four
// waves; the workgroups take equal shares of all units, so a long sequence is split over many of them
// (their partial results meet in attend_merge_kernel) and short ones share one.  The shares follow from
// q_off and ctx_len alone, which every workgroup sums for itself: the host reads nothing.
//
// Products.  S^T = K Q^T, with Q in registers as the B operand.  The result has one row's scores of 4 keys in each
// lane of a column, and that is the B operand of O^T = V^T P^T as it stands, with the keys of a block in another
// order; V takes that order when it is read from LDS transposed, 4 keys of one column per lane.  So the weights never
// leave the registers, and a column's m and l belong to the lanes that hold its accumulators.  A wave reads a block of K
// and V as whole rows (16 bytes a lane), one block ahead, and puts it into LDS of its own without a barrier.
//
// What bounds it, and what it takes (bf16, 8 key heads of 128 elements, pages of 64 tokens; a chip-wide read reaches
// 7.0 TB/s and a library product 1.38 PFLOP/s):
//   one token of 64 sequences of 1,000 to 16,384 keys   418 to 421 us, 6.35 TB/s: memory
//   one token of 8 sequences of 100 to 2,000 keys       18 us: chains of dependent loads in two launches (14 + 5 us)
//   9 to 24 drafted tokens of 32 sequences, 4 heads a group   114 to 123 us, 3.9 TB/s: a workgroup has one tile on its way
//                                                       and waits for it before it asks for the next; 11 us of joining
//   129 to 1,024 tokens of 6 sequences                  132 to 150 us, 560 to 640 TFLOP/s: the softmax's vector work
//                                                       beside the products, and 16 us of joining
//   the same turns in float                             1.63 ms, 52 TFLOP/s (154 in a library product): products of
//                                                       16 x 16 x 4 and tiles of 32 rows, each of which reads all keys
#include <type_traits>

#include "common.hpp"

namespace stride {
namespace {

typedef uint32_t u32x4 __attribute__((ext_vector_type(4)));
typedef uint32_t u32x2 __attribute__((ext_vector_type(2)));
typedef __bf16 bf16x4 __attribute__((ext_vector_type(4)));
typedef __bf16 bf16x8 __attribute__((ext_vector_type(8)));
typedef short i16x4 __attribute__((ext_vector_type(4)));
typedef short i16x8 __attribute__((ext_vector_type(8)));
typedef float f32x4 __attribute__((ext_vector_type(4)));

#define LDS_PTR(p) ((__attribute__((address_space(3))) void *)(p))
#define GLOBAL_PTR(p) ((const __attribute__((address_space(1))) void *)(p))
#define LDS_I16X4(p) ((__attribute__((address_space(3))) i16x4 *)(p))

constexpr int kThreads = 256;
constexpr int kWaves = kThreads / kWave;
constexpr int kCUs = 256;
constexpr float kLog2e = 1.4426950408889634f;
constexpr float kLn2 = 0.69314718055994531f;
constexpr float kSlack = 8.0f;  // log2 of the largest weight before a rescale

struct Place;

struct AttendArgs {
    const void *q, *k, *v;
    void *out;
    float *lse, *part;
    Place *at;
    const int32_t *table, *q_off, *ctx;
    const uint64_t *mask;
    uint32_t *flags;
    int64_t q_tok, q_head, o_tok, o_head, k_page, k_slot, k_head, v_page, v_slot, v_head;
    int64_t table_ld, max_len;
    int32_t n_pages, n_q, page_shift, n_seqs, n_heads, n_heads_q, group, mask_words, workers, log_workers;
    float scale_log2;
};

// Per element type: keys per block of a wave, and the words of 8 elements.
template <int DT>
struct Type;
template <>
struct Type<STRIDE_BF16> {
    static constexpr int size = 2, T = 2, words = 1, pad = 16;
};
template <>
struct Type<STRIDE_F32> {
    static constexpr int size = 4, T = 1, words = 2, pad = 4;
};

template <int DT>
struct Vec8 {  // 8 elements
    u32x4 w[Type<DT>::words];
};

template <int DT>
__device__ __forceinline__ Vec8<DT> load8(const char *p) {
    Vec8<DT> r;
#pragma unroll
    for (int i = 0; i < Type<DT>::words; ++i) r.w[i] = reinterpret_cast<const u32x4 *>(p)[i];
    return r;
}

// acc += A B over 32 elements of the contraction, 8 per lane.
template <int DT>
__device__ __forceinline__ f32x4 product(const Vec8<DT> &a, const Vec8<DT> &b, f32x4 acc) {
    if (DT == STRIDE_BF16)
        return __builtin_amdgcn_mfma_f32_16x16x32_bf16(__builtin_bit_cast(bf16x8, a.w[0]),
                                                       __builtin_bit_cast(bf16x8, b.w[0]), acc, 0, 0, 0);
#pragma unroll
    for (int j = 0; j < 8; ++j)  // lane group g holds elements 8 g + j: any order of the contraction will do
        acc = __builtin_amdgcn_mfma_f32_16x16x4f32(__uint_as_float(a.w[(Type<DT>::words - 1) * (j / 4)][j % 4]),
                                                   __uint_as_float(b.w[(Type<DT>::words - 1) * (j / 4)][j % 4]),
                                                   acc, 0, 0, 0);
    return acc;
}

// Maximum and sum over the four lanes l, l ^ 16, l ^ 32, l ^ 48 of a column.
__device__ __forceinline__ float column_max(float x) {
    const u32x2 a = __builtin_bit_cast(u32x2, __builtin_amdgcn_permlane16_swap(__float_as_uint(x), __float_as_uint(x), false, false));
    x = fmaxf(__uint_as_float(a[0]), __uint_as_float(a[1]));
    const u32x2 b = __builtin_bit_cast(u32x2, __builtin_amdgcn_permlane32_swap(__float_as_uint(x), __float_as_uint(x), false, false));
    return fmaxf(__uint_as_float(b[0]), __uint_as_float(b[1]));
}
__device__ __forceinline__ float column_sum(float x) {
    const u32x2 a = __builtin_bit_cast(u32x2, __builtin_amdgcn_permlane16_swap(__float_as_uint(x), __float_as_uint(x), false, false));
    x = __uint_as_float(a[0]) + __uint_as_float(a[1]);
    const u32x2 b = __builtin_bit_cast(u32x2, __builtin_amdgcn_permlane32_swap(__float_as_uint(x), __float_as_uint(x), false, false));
    return __uint_as_float(b[0]) + __uint_as_float(b[1]);
}
__device__ __forceinline__ float ex2(float x) { return __builtin_amdgcn_exp2f(x); }
// exp2(x - m) where m may be -inf (nothing seen yet): 0 then.
__device__ __forceinline__ float weight_of(float x, float m) { return m == -INFINITY ? 0.0f : ex2(x - m); }

// Wait until at most N vector-memory operations of this wave are outstanding.
template <int N>
__device__ __forceinline__ void wait_vmem() {
    __builtin_amdgcn_s_waitcnt((N & 0xF) | (7 << 4) | (0xF << 8) | ((N >> 4) << 14));
}

// ---- the work and its shares ----

struct Seq {
    int off, n, ctx;
    bool bad;  // lengths that the page table cannot hold: all its rows are NaN
};

__device__ __forceinline__ Seq sequence(const AttendArgs &a, int s, uint32_t &flag) {
    const int o0 = a.q_off[s], o1 = a.q_off[s + 1], c = a.ctx[s];
    Seq r = {o0, o1 - o0, c, false};
    if (o0 < 0 || o1 < o0 || o1 > a.n_q) {
        r = {0, 0, 0, false};
        flag |= STRIDE_FLAG_BAD_OFFSETS;
    } else if (c < 0 || (int64_t)c + r.n > a.max_len) {
        r.ctx = 0;
        r.bad = true;
        flag |= STRIDE_FLAG_BAD_OFFSETS;
    }
    return r;
}

// One past the last key that any row of tile rt sees.
template <int Rows>
__device__ __forceinline__ int keys_of(const AttendArgs &a, const Seq &q, int rt) {
    if (q.bad) return 0;
    if (a.mask) return q.ctx + q.n;
    const int last = ((rt + 1) * Rows - 1) / a.group + 1;
    return q.ctx + (last < q.n ? last : q.n);
}
template <int Rows, int Unit>
__device__ __forceinline__ int units_of(const AttendArgs &a, const Seq &q, int rt) {
    const int u = (keys_of<Rows>(a, q, rt) + Unit - 1) / Unit;
    return u > 1 ? u : 1;
}
template <int Rows>
__device__ __forceinline__ int tiles_of(const AttendArgs &a, const Seq &q) {
    return (q.n * a.group + Rows - 1) / Rows;
}

// What an item costs, in keys, for the shares: the keys it reads and Extra ones for its beginning and end (queries,
// the first block's way from memory, the results).  Item rt of a sequence costs base + step * (rt + 1): a chain's
// later row tiles see more keys.  It only has to be near; where an item ends is keys_of's.
template <int Rows, int Extra>
struct Cost {
    int64_t base, step, last;  // last: of the sequence's last tile
    int tiles;
    __device__ __forceinline__ Cost(const AttendArgs &a, const Seq &q) {
        tiles = tiles_of<Rows>(a, q);
        base = Extra + (q.bad ? 0 : q.ctx) + (a.mask && !q.bad ? q.n : 0);
        step = a.mask || q.bad ? 0 : (Rows + a.group - 1) / a.group;
        last = base + (a.mask || q.bad ? 0 : q.n);
    }
    __device__ __forceinline__ int64_t before(int rt) const { return rt * base + step * ((int64_t)rt * (rt + 1) / 2); }
    __device__ __forceinline__ int64_t head() const { return tiles ? before(tiles - 1) + last : 0; }
};

struct Place {  // where a share begins: a unit of an item
    int seq, head, rt, unit;
    __device__ __forceinline__ bool same_item(const Place &o) const { return seq == o.seq && head == o.head && rt == o.rt; }
};

struct PlanShared {
    int64_t wave_sum[kWaves];
    Place at[2];
};

// Inclusive sum over the wave's lanes, by moves within rows of 16 lanes and then from row to row.
__device__ __forceinline__ uint64_t wave_scan(uint64_t x) {
#define STRIDE_SCAN_STEP(ctrl, rows)                                                                     \
    {                                                                                                    \
        const uint32_t lo = __builtin_amdgcn_update_dpp(0, (uint32_t)x, ctrl, rows, 0xF, true);          \
        const uint32_t hi = __builtin_amdgcn_update_dpp(0, (uint32_t)(x >> 32), ctrl, rows, 0xF, true);  \
        x += (uint64_t)hi << 32 | lo;                                                                    \
    }
    STRIDE_SCAN_STEP(0x111, 0xF)  // from the lane 1, 2, 4, 8 before in the row
    STRIDE_SCAN_STEP(0x112, 0xF)
    STRIDE_SCAN_STEP(0x114, 0xF)
    STRIDE_SCAN_STEP(0x118, 0xF)
    STRIDE_SCAN_STEP(0x142, 0xA)  // the last lane of rows 0 and 2 to rows 1 and 3
    STRIDE_SCAN_STEP(0x143, 0xC)  // lane 31 to rows 2 and 3
#undef STRIDE_SCAN_STEP
    return x;
}

// Unit u (in cost) of sequence s's items.
template <int Rows, int Unit, int Extra>
__device__ __forceinline__ Place place_of(const AttendArgs &a, int s, const Seq &q, const Cost<Rows, Extra> &c, int64_t u) {
    Place x;
    x.seq = s;
    const int64_t head = c.head();
    x.head = (u | head) >> 32 ? (int)(u / head) : (int)((uint32_t)u / (uint32_t)head);
    u -= x.head * head;
    int lo = 0, hi = c.tiles - 1;  // the last tile that begins at or before u
    while (lo < hi) {
        const int mid = (lo + hi + 1) / 2;
        if (c.before(mid) <= u) lo = mid;
        else hi = mid - 1;
    }
    x.rt = lo;
    const int64_t unit = (u - c.before(lo) - Extra + Unit / 2) / Unit;
    const int units = units_of<Rows, Unit>(a, q, lo);
    x.unit = unit < 0 ? 0 : unit < units ? (int)unit : units - 1;
    return x;
}

__device__ __forceinline__ Place uniform(const Place &p, int lane) {
    return Place{__builtin_amdgcn_readlane(p.seq, lane), __builtin_amdgcn_readlane(p.head, lane),
                 __builtin_amdgcn_readlane(p.rt, lane), __builtin_amdgcn_readlane(p.unit, lane)};
}

// Where workgroup w's share of the work begins and ends.  The shares are equal parts of the cost of all items; a
// border near an item's beginning is put there.  What the first kernel finds stays in the workspace for the second.
// Up to 64 sequences every wave sums for itself, without a barrier: for one token of 8 rollouts this part of the call
// took 1.9 us instead of 3.2.
template <int Rows, int Unit, int Extra>
__device__ __forceinline__ void make_plan(const AttendArgs &a, int w, Place &from, Place &to, PlanShared &sh, uint32_t &flag) {
    const int tid = threadIdx.x, lane = tid & (kWave - 1), wave = tid / kWave;
    const Place end = {a.n_seqs, 0, 0, 0};
    if (a.n_seqs <= kWave) {
        Seq q = {};
        if (lane < a.n_seqs) q = sequence(a, lane, flag);
        const Cost<Rows, Extra> c(a, q);
        const int64_t mine = c.head() * a.n_heads, upto = wave_scan(mine);
        const int64_t total = (int64_t)(uint32_t)__builtin_amdgcn_readlane((int)upto, kWave - 1) |
                              (int64_t)__builtin_amdgcn_readlane((int)(upto >> 32), kWave - 1) << 32;
#pragma unroll
        for (int b = 0; b < 2; ++b) {
            const int64_t u = (total * (w + b) >> a.log_workers) - (upto - mine);
            const bool here = u >= 0 && u < mine;
            Place x = end;
            if (here) x = place_of<Rows, Unit, Extra>(a, lane, q, c, u);
            const uint64_t who = __ballot(here);
            const Place p = who ? uniform(x, __builtin_ctzll(who)) : end;
            if (b == 0) from = p;
            else to = p;
        }
    } else {
        const int per = (a.n_seqs + kThreads - 1) / kThreads;
        const int s0 = tid * per, s1 = s0 + per < a.n_seqs ? s0 + per : a.n_seqs;
        int64_t mine = 0;
        for (int s = s0; s < s1; ++s) mine += Cost<Rows, Extra>(a, sequence(a, s, flag)).head() * a.n_heads;
        const int64_t upto = wave_scan(mine);
        if (lane == kWave - 1) sh.wave_sum[wave] = upto;
        if (tid < 2) sh.at[tid] = end;
        __syncthreads();
        int64_t before = 0, total = 0;
#pragma unroll
        for (int i = 0; i < kWaves; ++i) {
            if (i < wave) before += sh.wave_sum[i];
            total += sh.wave_sum[i];
        }
        before += upto - mine;
#pragma unroll
        for (int b = 0; b < 2; ++b) {
            int64_t u = (total * (w + b) >> a.log_workers) - before;
            if (u < 0 || u >= mine) continue;  // another thread's
            uint32_t ignore = 0;
            for (int s = s0; s < s1; ++s) {
                const Seq q = sequence(a, s, ignore);
                const Cost<Rows, Extra> c(a, q);
                if (u < c.head() * a.n_heads) {
                    sh.at[b] = place_of<Rows, Unit, Extra>(a, s, q, c, u);
                    break;
                }
                u -= c.head() * a.n_heads;
            }
        }
        __syncthreads();
        from = uniform(sh.at[0], 0);
        to = uniform(sh.at[1], 0);
    }
    if (w == 0) {
        if (tid == 0 && (a.q_off[0] != 0 || a.q_off[a.n_seqs] != a.n_q)) flag |= STRIDE_FLAG_BAD_OFFSETS;
        if (flag) raise_flag(a.flags, flag);
    }
    if (tid == 0) {
        a.at[w] = from;
        if (w == a.workers - 1) a.at[w + 1] = end;
    }
}

// The item after `at` of sequence s.
template <int Rows>
__device__ __forceinline__ void next_item(const AttendArgs &a, const Seq &s, Place &at) {
    at.unit = 0;
    if (++at.rt < tiles_of<Rows>(a, s)) return;
    at.rt = 0;
    if (++at.head < a.n_heads) return;
    at.head = 0;
    uint32_t ignore = 0;
    do {
        ++at.seq;
    } while (at.seq < a.n_seqs && sequence(a, at.seq, ignore).n == 0);
}
__device__ __forceinline__ bool at_end(const Place &at, const Place &to) {
    return at.same_item(to) && at.unit == to.unit;
}

// ---- one block of 16 T keys ----

// Keys and values, which a step of few rows reads once, go past the caches: 64 sequences of 1,000 to 16,384 keys take 417
// us, or 468 with ordinary loads, and sequences that share their pages gain as well (436 us, or 467).  A sequence of several
// row tiles in this form (float, or a turn beside many single tokens) reads them from memory for each.
__device__ __forceinline__ u32x4 once(const char *p) {
    return __builtin_nontemporal_load(reinterpret_cast<const u32x4 *>(p));
}

// 16-byte words of a wave's block, lane after lane: whole rows follow each other in every load.
template <int DT, int D>
struct Block {
    static constexpr int rows = 16 * Type<DT>::T, per_row = D * Type<DT>::size / 16, N = rows * per_row / kWave;
    static constexpr int ks = D * Type<DT>::size + 16;               // bytes between K's rows in LDS
    static constexpr int vs = (D + Type<DT>::pad) * Type<DT>::size;  // and V's
    static constexpr int bytes = rows * (ks + vs);
    u32x4 k[N], v[N];
};

// A page id by the scalar unit: its wait does not cover the vector loads in flight.
__device__ __forceinline__ int32_t scalar_load(const int32_t *p) {
    return *(const __attribute__((address_space(4))) int32_t *)p;
}

// The page id, or the first page in the place of one outside the cache.  The rows that see its keys are NaN and no others:
// all rows where a block is whole, else the keys are made NaN.  `lost`: whether any of the wave's was outside; which is
// looked up again where there is one.
__device__ __forceinline__ bool in_cache(const AttendArgs &a, int32_t page) { return page >= 0 && page < a.n_pages; }
template <bool Uniform>
__device__ __forceinline__ int32_t checked_page(const AttendArgs &a, int32_t page, bool &lost) {
    const bool ok = in_cache(a, page);
    lost |= Uniform ? !ok : __any(!ok) != 0;
    return ok ? page : 0;
}
__device__ __forceinline__ u32x4 nan_word() { return u32x4{~0u, ~0u, ~0u, ~0u}; }  // of bf16 or float

// Non-finite elements of a word become zeros; whether there were any.
template <int DT>
__device__ __forceinline__ bool scrub(u32x4 &w) {
    bool any = false;
#pragma unroll
    for (int i = 0; i < 4; ++i) {
        if (DT == STRIDE_BF16) {
            const bool lo = (w[i] & 0x7F80u) == 0x7F80u, hi = (w[i] & 0x7F800000u) == 0x7F800000u;
            any |= lo | hi;
            w[i] = (lo ? 0u : w[i] & 0xFFFFu) | (hi ? 0u : w[i] & 0xFFFF0000u);
        } else {
            const bool x = (w[i] & 0x7F800000u) == 0x7F800000u;
            any |= x;
            w[i] = x ? 0u : w[i];
        }
    }
    return any;
}

template <int DT, int D, int RT>
struct Wave {
    static constexpr int T = Type<DT>::T, C = D / 32, DV = D / 16;
    Vec8<DT> q[RT][C];
    f32x4 o[RT][DV];
    float m[RT], l[RT];  // reference point in units of log2, this lane's part of the sum
    int tok[RT];
};

constexpr int row_pad(int D) { return D + 4; }  // floats between rows of the join

template <int DT, int D>
constexpr int lds_bytes() {
    const int b = kWaves * Block<DT, D>::bytes, o = kWaves * 16 * row_pad(D) * 4;
    return b > o ? b : o;
}

// OnePage: pages hold whole blocks, so a block's addresses are one page's and the same offsets every time.
template <int DT, int D, int RT, int Occ, bool OnePage>
__global__ __launch_bounds__(kThreads, Occ) void attend_kernel(AttendArgs a) {
    typedef Type<DT> Ty;
    constexpr int T = Ty::T, C = D / 32, DV = D / 16, KB = 16 * T, Rows = 16 * RT, Unit = kWaves * KB, Extra = Unit;
    constexpr int P = Rows * (D + 2);  // floats of a partial result
    __shared__ __attribute__((aligned(16))) char lds[lds_bytes<DT, D>()];
    __shared__ PlanShared sh;
    __shared__ float s_m[kWaves][16], s_l[kWaves][16];
    const int tid = threadIdx.x, lane = tid & (kWave - 1), wave = __builtin_amdgcn_readfirstlane(tid / kWave);
    const int col = lane & 15, grp = lane >> 4;
    // neighbouring shares, which read the same keys where a sequence has several row tiles, go to one
    // XCD (workgroups are handed to the eight of them in turn)
    const int w = (int)(blockIdx.x & 7) * (a.workers >> 3) + (int)(blockIdx.x >> 3);
    uint32_t flag = 0;
    Place at, to;
    make_plan<Rows, Unit, Extra>(a, w, at, to, sh, flag);
    typedef Block<DT, D> B;
    char *klds = lds + wave * B::bytes, *vlds = klds + B::rows * B::ks;
    auto row_of = [&](int i) __attribute__((always_inline)) { return (lane + i * kWave) / B::per_row; };
    auto word_of = [&](int i) __attribute__((always_inline)) { return (lane + i * kWave) % B::per_row; };

    Seq s = {};
    for (int known = -1; !at_end(at, to);) {
        if (at.seq != known) s = sequence(a, known = at.seq, flag);
        const int n_rows = s.n * a.group, len = keys_of<Rows>(a, s, at.rt);
        const int units = units_of<Rows, Unit>(a, s, at.rt);
        const int u1 = at.same_item(to) ? to.unit : units;
        const int32_t *table = a.table + at.seq * a.table_ld;
        const char *kb = static_cast<const char *>(a.k) + at.head * a.k_head * Ty::size;
        const char *vb = static_cast<const char *>(a.v) + at.head * a.v_head * Ty::size;
        bool lost = false, any_lost = false, poison = s.bad;  // pages outside the cache: of the block on its way, of all

        Wave<DT, D, RT> x;
#pragma unroll
        for (int t = 0; t < RT; ++t) {
            const int r = at.rt * Rows + t * 16 + col;
            const bool in = r < n_rows;
            const int tok = in ? r / a.group : 0;
            x.tok[t] = tok;
            const char *qp = static_cast<const char *>(a.q) +
                             ((int64_t)(s.off + tok) * a.q_tok +
                              (int64_t)(at.head * a.group + r - tok * a.group) * a.q_head + grp * 8) * Ty::size;
#pragma unroll
            for (int c = 0; c < C; ++c) {
                x.q[t][c] = Vec8<DT>{};
                if (in) x.q[t][c] = load8<DT>(qp + c * 32 * Ty::size);
            }
#pragma unroll
            for (int d = 0; d < DV; ++d) x.o[t][d] = f32x4{};
            x.m[t] = -INFINITY;
            x.l[t] = 0.0f;
        }

        const int end = (len + KB - 1) / KB;  // blocks of the item
        const int stop = u1 * kWaves < end ? u1 * kWaves : end;
        int b = at.unit * kWaves + wave;
        uint32_t koff[B::N], voff[B::N];  // OnePage: bytes from the block's first key
        int32_t pg[OnePage ? 1 : B::N];
        if (OnePage) {
#pragma unroll
            for (int i = 0; i < B::N; ++i) {
                koff[i] = (uint32_t)(row_of(i) * a.k_slot * Ty::size + word_of(i) * 16);
                voff[i] = (uint32_t)(row_of(i) * a.v_slot * Ty::size + word_of(i) * 16);
            }
        }
        // the pages of a block's keys, one round ahead of its loads
        auto pages = [&](int blk) __attribute__((always_inline)) {
            if (OnePage) {
                pg[0] = scalar_load(table + ((blk * KB) >> a.page_shift));
            } else {
#pragma unroll
                for (int i = 0; i < B::N; ++i) {
                    const int key = blk * KB + row_of(i);
                    pg[i] = table[(key < len ? key : len - 1) >> a.page_shift];
                }
            }
        };
        auto fetch = [&](int blk, B &x) __attribute__((always_inline)) {
            lost = false;
            if (OnePage) {  // slots past the sequence's end are the page's own
                const int32_t page = checked_page<true>(a, pg[0], lost);
                const int64_t slot = (blk * KB) & ((1 << a.page_shift) - 1);
                const char *kp = kb + (page * a.k_page + slot * a.k_slot) * Ty::size;
                const char *vp = vb + (page * a.v_page + slot * a.v_slot) * Ty::size;
#pragma unroll
                for (int i = 0; i < B::N; ++i) x.k[i] = once(kp + koff[i]);
#pragma unroll
                for (int i = 0; i < B::N; ++i) x.v[i] = once(vp + voff[i]);
            } else {
#pragma unroll
                for (int i = 0; i < B::N; ++i) {
                    int key = blk * KB + row_of(i);
                    key = key < len ? key : len - 1;
                    const int32_t page = checked_page<false>(a, pg[i], lost);
                    const int64_t slot = key & ((1 << a.page_shift) - 1);
                    x.k[i] = once(kb + (page * a.k_page + slot * a.k_slot) * Ty::size + word_of(i) * 16);
                    x.v[i] = once(vb + (page * a.v_page + slot * a.v_slot) * Ty::size + word_of(i) * 16);
                }
            }
        };
        Block<DT, D> next;
        if (b < stop) {
            pages(b);
            fetch(b, next);
            if (b + kWaves < stop) pages(b + kWaves);
        }
        for (; b < stop; b += kWaves) {
            const int k0 = b * KB;
            const bool tail = k0 + KB > s.ctx;  // the same for the whole wave: some keys are not every row's
            bool dirty = false;
            any_lost |= lost;
            poison |= lost && !tail;
            if (tail) {
#pragma unroll
                for (int i = 0; i < B::N; ++i) {
                    const int key = k0 + row_of(i);
                    if (key >= len) next.v[i] = u32x4{};
                    else if (key >= s.ctx) dirty |= scrub<DT>(next.v[i]);
                    if (lost && (OnePage || !in_cache(a, table[(key < len ? key : len - 1) >> a.page_shift])))
                        next.k[i] = nan_word();
                }
            }
#pragma unroll
            for (int i = 0; i < B::N; ++i) {
                *reinterpret_cast<u32x4 *>(klds + row_of(i) * B::ks + word_of(i) * 16) = next.k[i];
                *reinterpret_cast<u32x4 *>(vlds + row_of(i) * B::vs + word_of(i) * 16) = next.v[i];
            }
            __builtin_amdgcn_wave_barrier();
            if (b + kWaves < stop) {
                fetch(b + kWaves, next);
                if (b + 2 * kWaves < stop) pages(b + 2 * kWaves);
            }
            Vec8<DT> kf[T][C];
#pragma unroll
            for (int j = 0; j < T; ++j)
#pragma unroll
                for (int c = 0; c < C; ++c)
                    kf[j][c] = load8<DT>(klds + (j * 16 + col) * B::ks + (c * 32 + grp * 8) * Ty::size);

            // scores: lane (col, grp) has row col of tile t and keys k0 + 16 j + 4 grp + r
            Vec8<STRIDE_BF16> pw[RT];  // weights as the second product's operand
            float pf[RT][4];
#pragma unroll
            for (int t = 0; t < RT; ++t) {
                f32x4 sc[T];
#pragma unroll
                for (int j = 0; j < T; ++j) {
                    sc[j] = f32x4{};
#pragma unroll
                    for (int c = 0; c < C; ++c) sc[j] = product<DT>(kf[j][c], x.q[t][c], sc[j]);
                }
                if (tail) {
                    const uint64_t *mk = a.mask ? a.mask + (int64_t)(s.off + x.tok[t]) * a.mask_words : nullptr;
#pragma unroll
                    for (int j = 0; j < T; ++j)
#pragma unroll
                        for (int r = 0; r < 4; ++r) {
                            const int key = k0 + j * 16 + grp * 4 + r, rel = key - s.ctx;
                            bool sees = key < len;
                            if (sees && rel >= 0)
                                sees = mk ? (rel >> 6) < a.mask_words && ((mk[rel >> 6] >> (rel & 63)) & 1)
                                          : rel <= x.tok[t];
                            sc[j][r] = sees ? sc[j][r] : -INFINITY;
                        }
                }
                float top = sc[0][0];
#pragma unroll
                for (int i = 1; i < 4 * T; ++i) top = fmaxf(top, sc[i / 4][i % 4]);
                top *= a.scale_log2;
                if (__any(top > x.m[t] + kSlack)) {
                    const float m = fmaxf(x.m[t], column_max(top));
                    const float f = x.m[t] == m ? 1.0f : weight_of(x.m[t], m);
                    x.m[t] = m;
                    x.l[t] *= f;
#pragma unroll
                    for (int d = 0; d < DV; ++d) x.o[t][d] *= f;
                }
                const float ref = x.m[t] == -INFINITY ? 0.0f : x.m[t];
                float sum = 0.0f;
                bf16x8 pb;
#pragma unroll
                for (int i = 0; i < 4 * T; ++i) {
                    const float p = ex2(__builtin_fmaf(sc[i / 4][i % 4], a.scale_log2, -ref));
                    sum += p;
                    // bf16 weights: the matrix cores' input; the sum l keeps 32 bits, and the roundings
                    // (at most 2^-8 of each weight) average out over the keys
                    if (DT == STRIDE_BF16) pb[i] = (__bf16)p;
                    else pf[t][i] = p;
                }
                if (DT == STRIDE_BF16) pw[t].w[0] = __builtin_bit_cast(u32x4, pb);
                x.l[t] += sum;
            }
            // O^T += V^T P^T
#pragma unroll
            for (int d = 0; d < DV; ++d) {
                if (DT == STRIDE_BF16) {
                    char *p = vlds + (4 * grp + (col >> 2)) * B::vs + (d * 16 + (col & 3) * 4) * 2;
                    const i16x4 lo = __builtin_amdgcn_ds_read_tr16_b64_v4i16(LDS_I16X4(p));
                    const i16x4 hi = __builtin_amdgcn_ds_read_tr16_b64_v4i16(LDS_I16X4(p + 16 * B::vs));
                    const i16x8 f = __builtin_shufflevector(lo, hi, 0, 1, 2, 3, 4, 5, 6, 7);
#pragma unroll
                    for (int t = 0; t < RT; ++t)
                        x.o[t][d] = __builtin_amdgcn_mfma_f32_16x16x32_bf16(
                            __builtin_bit_cast(bf16x8, f), __builtin_bit_cast(bf16x8, pw[t].w[0]), x.o[t][d], 0, 0, 0);
                } else {
#pragma unroll
                    for (int r = 0; r < 4; ++r) {
                        const float f = *reinterpret_cast<const float *>(vlds + (4 * grp + r) * B::vs + (d * 16 + col) * 4);
#pragma unroll
                        for (int t = 0; t < RT; ++t)
                            x.o[t][d] = __builtin_amdgcn_mfma_f32_16x16x4f32(f, pf[t][r], x.o[t][d], 0, 0, 0);
                    }
                }
            }
            __builtin_amdgcn_wave_barrier();
            if (tail && __any(dirty)) {
                // values that are infinite or NaN: zeros above, added here to the rows that see them
                for (int kk = 0; kk < KB; ++kk) {
                    const int key = k0 + kk;
                    if (key < s.ctx || key >= len) continue;
                    int64_t page = table[key >> a.page_shift];
                    if (page < 0 || page >= a.n_pages) page = 0;
                    const int64_t off = page * a.v_page + (key & ((1 << a.page_shift) - 1)) * a.v_slot + at.head * a.v_head;
                    const int src = col + 16 * ((kk & 15) >> 2);
#pragma unroll
                    for (int t = 0; t < RT; ++t) {
                        float p = 0.0f;
#pragma unroll
                        for (int i = 0; i < 4 * T; ++i) {
                            float y;
                            if (DT == STRIDE_BF16) y = (float)__builtin_bit_cast(bf16x8, pw[t].w[0])[i];
                            else y = pf[t][i & 3];
                            y = __shfl(y, src, kWave);
                            if (i == (kk >> 4) * 4 + (kk & 3)) p = y;
                        }
#pragma unroll
                        for (int d = 0; d < DV; ++d)
#pragma unroll
                            for (int e = 0; e < 4; ++e) {
                                const int64_t i = off + d * 16 + grp * 4 + e;
                                const float v = DT == STRIDE_BF16
                                                    ? __uint_as_float((uint32_t) static_cast<const uint16_t *>(a.v)[i] << 16)
                                                    : static_cast<const float *>(a.v)[i];
                                if (!(fabsf(v) < INFINITY) && p != 0.0f) x.o[t][d][e] += p * v;
                            }
                    }
                }
            }
        }

        // ---- join the waves, one row tile after the other ----
        if (any_lost) raise_flag(a.flags, STRIDE_FLAG_BAD_PAGE);
        if (poison) {
#pragma unroll
            for (int t = 0; t < RT; ++t) x.l[t] = __builtin_nanf("");
        }
        const bool whole = at.unit == 0 && u1 == units;
        float *part = a.part + (int64_t)(2 * w + (at.unit == 0 ? 1 : 0)) * P;
        float *buf = reinterpret_cast<float *>(lds);
#pragma unroll
        for (int t = 0; t < RT; ++t) {
            const float l = column_sum(x.l[t]);
            __syncthreads();  // V of all waves, or the tile before, has been read
            if (grp == 0) {
                s_m[wave][col] = x.m[t];
                s_l[wave][col] = l;
            }
#pragma unroll
            for (int d = 0; d < DV; ++d)
                *reinterpret_cast<f32x4 *>(buf + (wave * 16 + col) * row_pad(D) + d * 16 + grp * 4) = x.o[t][d];
            __syncthreads();
            // 16 threads per row
            const int row = tid >> 4, r = at.rt * Rows + t * 16 + row;
            if (r >= n_rows) continue;  // not past a barrier: those of the next tile and of the item's end are met by all
            float m = s_m[0][row], sum = 0.0f, f[kWaves];
#pragma unroll
            for (int i = 1; i < kWaves; ++i) m = fmaxf(m, s_m[i][row]);
#pragma unroll
            for (int i = 0; i < kWaves; ++i) {
                f[i] = s_m[i][row] == m ? (m == -INFINITY ? 0.0f : 1.0f) : weight_of(s_m[i][row], m);
                sum += s_l[i][row] * (m == -INFINITY ? 1.0f : f[i]);  // a NaN sum (a bad page) stays one
            }
            const int tok = r / a.group, head = at.head * a.group + r - tok * a.group;
            const float inv = whole ? (sum == 0.0f ? 0.0f : 1.0f / sum) : 1.0f;
            for (int d = (tid & 15) * 4; d < D; d += 64) {
                f32x4 y = {};
#pragma unroll
                for (int i = 0; i < kWaves; ++i)
                    y += f[i] * *reinterpret_cast<const f32x4 *>(buf + (i * 16 + row) * row_pad(D) + d);
                y *= inv;
                if (!whole) {
                    *reinterpret_cast<f32x4 *>(part + (t * 16 + row) * D + d) = y;
                } else {
                    const int64_t i = (int64_t)(s.off + tok) * a.o_tok + (int64_t)head * a.o_head + d;
                    if (DT == STRIDE_BF16) {
                        const bf16x4 z = {(__bf16)y[0], (__bf16)y[1], (__bf16)y[2], (__bf16)y[3]};
                        *reinterpret_cast<bf16x4 *>(static_cast<uint16_t *>(a.out) + i) = z;
                    } else {
                        *reinterpret_cast<f32x4 *>(static_cast<float *>(a.out) + i) = y;
                    }
                }
            }
            if ((tid & 15) == 0) {
                if (!whole) {
                    part[Rows * D + t * 16 + row] = m;
                    part[Rows * D + Rows + t * 16 + row] = sum;
                } else if (a.lse) {
                    a.lse[(int64_t)(s.off + tok) * a.n_heads_q + head] =
                        sum == 0.0f ? -INFINITY : (m + __builtin_amdgcn_logf(sum)) * kLn2;
                }
            }
        }
        __syncthreads();  // `buf` has been read: the next item's keys and values go there
        if (at.same_item(to)) break;
        next_item<Rows>(a, s, at);
    }
}

// ---- many rows ----
// The same with the parts of the chip the other way round: many rows of a key head, where products and not
// memory bound it.  The four waves take 32 rows each and share every tile of 64 keys, which goes from memory
// straight to LDS (two buffers of K and V, one barrier per tile: while a tile is multiplied the next one is on its
// way).  32 x 32 x 16 products read half as many operand registers and LDS bytes per flop as the 16 x 16 x 32 ones;
// two workgroups per CU let one wave's softmax run beside another's products.
typedef float f32x16 __attribute__((ext_vector_type(16)));

constexpr int kTile = 64;
// Third word of a raw buffer descriptor: 32-bit data format, no swizzle; accesses at or beyond num_records
// bytes return zeros.
constexpr int kBufferFlags = 0x00020000;

// A tile in LDS: rows of D elements one after the other, 16-byte words of a row in another order, so that neither
// the 16-byte reads of K (sixteen rows at the same word of each, in each of the read's cycles) nor the transposed ones
// of V (four rows at four words) meet in a bank: k_place(row, word) and v_place are where a word is, and back.
template <int D>
struct Wide {
    static constexpr int words = D / 8, row = D * 2, bytes = kTile * row, buf = 2 * bytes;
    static constexpr int N = kTile * words / kThreads;  // words per thread of each
    static __device__ __forceinline__ int k_place(int r, int c) {
        if (D == 96) return (c + ((r >> 2) & 3)) % 12;  // rows of 48 banks: four of them go round
        return c ^ (D == 64 ? (r >> 1) & 7 : r & 15);
    }
    static __device__ __forceinline__ int k_back(int r, int c) {
        if (D == 96) return (c + 12 - ((r >> 2) & 3)) % 12;
        return k_place(r, c);
    }
    static __device__ __forceinline__ int v_place(int r, int c) {
        if (D == 96) return c;
        return c ^ (D == 64 ? ((r >> 1) & 1) << 2 : (r & 3) << 2);
    }
};

// Maximum and sum over lanes l and l ^ 32.
[[maybe_unused]] __device__ __forceinline__ float half_max(float x) {
    const u32x2 b = __builtin_bit_cast(u32x2, __builtin_amdgcn_permlane32_swap(__float_as_uint(x), __float_as_uint(x), false, false));
    return fmaxf(__uint_as_float(b[0]), __uint_as_float(b[1]));
}
[[maybe_unused]] __device__ __forceinline__ float half_sum(float x) {
    const u32x2 b = __builtin_bit_cast(u32x2, __builtin_amdgcn_permlane32_swap(__float_as_uint(x), __float_as_uint(x), false, false));
    return __uint_as_float(b[0]) + __uint_as_float(b[1]);
}

// Bits of the 64 keys from k0 on: which of them row `tok` of sequence s sees.
[[maybe_unused]] __device__ __forceinline__ uint64_t seen_keys(const AttendArgs &a, const Seq &s, int tok, int k0, int len) {
    auto first = [](int n) { return n <= 0 ? 0ull : n >= 64 ? ~0ull : (1ull << n) - 1; };
    const uint64_t real = first(len - k0);
    if (!a.mask) return real & first(s.ctx + tok + 1 - k0);
    const int rel = k0 - s.ctx;  // the tile's first key as a new token's number
    const uint64_t *m = a.mask + (int64_t)(s.off + tok) * a.mask_words;
    if (rel <= -64) return real;
    if (rel < 0) return real & (m[0] << -rel | first(-rel));
    const int w = rel >> 6, b = rel & 63;
    uint64_t x = w < a.mask_words ? m[w] >> b : 0;
    if (b && w + 1 < a.mask_words) x |= m[w + 1] << (64 - b);
    return real & x;
}

// OnePage: pages hold whole tiles, so a tile's addresses are one page's and the same offsets every time.
template <int D, bool OnePage>
__device__ __forceinline__ void attend_wide(const AttendArgs &a) {
    typedef Wide<D> W;
    // an item's beginning and end take as long as five tiles; counted as two, turns of 129 to 1,024 tokens took 165 us, not 154
    constexpr int Rows = 128, Unit = kTile, Extra = 5 * kTile, P = Rows * (D + 2), C = D / 16, DB = D / 32;
    // two objects, so that the compiler knows a load into one of them apart from the reads of the other
    __shared__ __attribute__((aligned(1024))) char lds0[W::buf], lds1[W::buf];
    __shared__ PlanShared sh;
    __shared__ uint32_t s_dirty[2][kWaves];  // by the tile's parity: a wave may be one tile ahead of another
    const int tid = threadIdx.x, lane = tid & (kWave - 1), wave = __builtin_amdgcn_readfirstlane(tid / kWave);
    const int col = lane & 31, half = lane >> 5;
    const int w = (int)(blockIdx.x & 7) * (a.workers >> 3) + (int)(blockIdx.x >> 3);
    uint32_t flag = 0;
    Place at, to;
    make_plan<Rows, Unit, Extra>(a, w, at, to, sh, flag);

    // word x of a tile in LDS, this thread's i-th: its row, and the word of the row that is there
    auto word = [&](int i) __attribute__((always_inline)) { return tid + i * kThreads; };
    uint32_t koff[W::N], voff[W::N];  // OnePage: bytes from the tile's first key; else from the key
#pragma unroll
    for (int i = 0; i < W::N; ++i) {
        const int row = word(i) / W::words, c = word(i) % W::words;
        koff[i] = (uint32_t)((OnePage ? row * a.k_slot : 0) + W::k_back(row, c) * 8) * 2;
        voff[i] = (uint32_t)((OnePage ? row * a.v_slot : 0) + W::v_place(row, c) * 8) * 2;
    }
    // this lane's fragments: K of row col at words 2 c + half; V transposed, rows 4 half + {0 .. 3}
    int kfrag[C];
#pragma unroll
    for (int c = 0; c < C; ++c) kfrag[c] = col * W::row + W::k_place(col, 2 * c + half) * 16;
    const int vrow = 4 * half + ((lane & 15) >> 2);
    int vfrag[DB];
#pragma unroll
    for (int d = 0; d < DB; ++d)
        vfrag[d] = W::bytes + vrow * W::row +
                   W::v_place(vrow, d * 4 + ((lane >> 4) & 1) * 2 + ((lane & 3) >> 1)) * 16 + (lane & 1) * 8;

    Seq s = {};
    for (int known = -1; !at_end(at, to);) {
        if (at.seq != known) s = sequence(a, known = at.seq, flag);
        const int n_rows = s.n * a.group, len = keys_of<Rows>(a, s, at.rt);
        const int units = units_of<Rows, Unit>(a, s, at.rt);
        const int u1 = at.same_item(to) ? to.unit : units;
        const int32_t *table = a.table + at.seq * a.table_ld;
        const uint16_t *kb = static_cast<const uint16_t *>(a.k) + at.head * a.k_head;
        const uint16_t *vb = static_cast<const uint16_t *>(a.v) + at.head * a.v_head;
        const int r0 = at.rt * Rows + wave * 32, r = r0 + col;  // this wave's first row, this lane's
        const bool busy = r0 < n_rows;                          // the wave has rows
        const bool in = r < n_rows;
        const int tok = in ? r / a.group : 0;
        bool lost = false, any_lost = false, poison = s.bad;  // pages outside the cache: of the tile on its way, of all
        // keys that all rows of the workgroup see, and one past the last that a row of this wave sees
        int all_see = s.ctx, wave_end = len;
        if (!a.mask) {
            all_see = s.ctx + (at.rt * Rows) / a.group + 1;
            const int last = (r0 + 31) / a.group + 1;
            wave_end = s.ctx + (last < s.n ? last : s.n);
        }
        if (all_see > len) all_see = len;

        bf16x8 q[C];
        const int64_t qi = (int64_t)(s.off + tok) * a.q_tok + (int64_t)(at.head * a.group + r - tok * a.group) * a.q_head + half * 8;
#pragma unroll
        for (int c = 0; c < C; ++c) {
            u32x4 x = {};
            if (in) x = *reinterpret_cast<const u32x4 *>(static_cast<const uint16_t *>(a.q) + qi + c * 16);
            q[c] = __builtin_bit_cast(bf16x8, x);
        }
        f32x16 o[DB];
#pragma unroll
        for (int d = 0; d < DB; ++d) o[d] = f32x16{};
        float m = -INFINITY, l = 0.0f;

        const int end = (len + kTile - 1) / kTile;
        const int stop = u1 < end ? u1 : end;
        int32_t pg[OnePage ? 1 : W::N];
        auto pages = [&](int t) __attribute__((always_inline)) {
            if (OnePage) {
                pg[0] = scalar_load(table + ((t * kTile) >> a.page_shift));
            } else {
#pragma unroll
                for (int i = 0; i < W::N; ++i) {
                    const int key = t * kTile + word(i) / W::words;
                    pg[i] = table[(key < len ? key : len - 1) >> a.page_shift];
                }
            }
        };
        // a tile's words into LDS: 64 lanes' one after the other with each load, past the caches (Aux 2) where no other row
        // tile reads them: 9 to 24 drafted tokens of 32 sequences with pages of their own take 120 us, 134 through the
        // caches; turns of several tiles take 147 us through the caches, 173 past them
        auto load = [&](int t, char *buf, auto aux) __attribute__((always_inline)) {
            constexpr int Aux = decltype(aux)::value;
            char *dst = buf + wave * 1024;
            lost = false;
            if (OnePage) {  // slots past the sequence's end are the page's own
                const int32_t page = checked_page<true>(a, pg[0], lost);
                const int64_t slot = (t * kTile) & ((1 << a.page_shift) - 1);
                const __amdgpu_buffer_rsrc_t rk = __builtin_amdgcn_make_buffer_rsrc(
                    (void *)(kb + page * a.k_page + slot * a.k_slot), (short)0, (int)((63 * a.k_slot + D) * 2), kBufferFlags);
                const __amdgpu_buffer_rsrc_t rv = __builtin_amdgcn_make_buffer_rsrc(
                    (void *)(vb + page * a.v_page + slot * a.v_slot), (short)0, (int)((63 * a.v_slot + D) * 2), kBufferFlags);
#pragma unroll
                for (int i = 0; i < W::N; ++i) {
                    __builtin_amdgcn_raw_ptr_buffer_load_lds(rk, LDS_PTR(dst + i * kThreads * 16), 16, koff[i], 0, 0, Aux);
                    __builtin_amdgcn_raw_ptr_buffer_load_lds(rv, LDS_PTR(dst + W::bytes + i * kThreads * 16), 16, voff[i], 0, 0, Aux);
                }
            } else {
#pragma unroll
                for (int i = 0; i < W::N; ++i) {
                    int key = t * kTile + word(i) / W::words;
                    key = key < len ? key : len - 1;
                    const int32_t page = checked_page<false>(a, pg[i], lost);
                    const int64_t slot = key & ((1 << a.page_shift) - 1);
                    const char *kp = reinterpret_cast<const char *>(kb + page * a.k_page + slot * a.k_slot) + koff[i];
                    const char *vp = reinterpret_cast<const char *>(vb + page * a.v_page + slot * a.v_slot) + voff[i];
                    __builtin_amdgcn_global_load_lds(GLOBAL_PTR(kp), LDS_PTR(dst + i * kThreads * 16), 16, 0, Aux);
                    __builtin_amdgcn_global_load_lds(GLOBAL_PTR(vp), LDS_PTR(dst + W::bytes + i * kThreads * 16), 16, 0, Aux);
                }
            }
        };
        const bool alone = n_rows <= Rows;
        auto fetch = [&](int t, char *buf) __attribute__((always_inline)) {
            if (alone) load(t, buf, std::integral_constant<int, 2>{});
            else load(t, buf, std::integral_constant<int, 0>{});
        };
        // values that not every row sees lose their infinities and NaN, those past the end are zeros: by the
        // thread whose loads brought them
        auto clean = [&](int t, char *buf) __attribute__((always_inline)) {
            bool dirty = false;
#pragma unroll
            for (int i = 0; i < W::N; ++i) {
                u32x4 *p = reinterpret_cast<u32x4 *>(buf + W::bytes + word(i) * 16);
                const int key = t * kTile + word(i) / W::words;
                u32x4 x = *p;
                if (key >= len) x = u32x4{};
                else if (key >= s.ctx) dirty |= scrub<STRIDE_BF16>(x);
                *p = x;
            }
            const bool any = __any(dirty);
            if (lane == 0) s_dirty[t & 1][wave] = any;
        };
        int t = at.unit;
        __syncthreads();  // every wave is past the item before
        if (t < stop) {
            pages(t);
            fetch(t, lds0);
            if (t + 1 < stop) pages(t + 1);
        }
        // One tile: scores of 64 keys, their weights, the weighted sum of their values.  `Tail`: not every row sees
        // every key.  The fragments of a product are all read before its first step, and V's first ones before the
        // softmax, so that a wave waits for LDS once per product.
        auto step = [&](char *base, char *other, auto tail_tag) __attribute__((always_inline)) {
            constexpr bool Tail = decltype(tail_tag)::value;
            wait_vmem<0>();  // this thread's part of tile t
            any_lost |= lost;
            if (OnePage && !Tail) {  // the same page for all waves
                poison |= lost;
            } else if (lost) {
                for (int i = 0; i < W::N; ++i) {
                    const int key = t * kTile + word(i) / W::words;
                    if (OnePage || !in_cache(a, table[(key < len ? key : len - 1) >> a.page_shift]))
                        *reinterpret_cast<u32x4 *>(base + word(i) * 16) = nan_word();
                }
            }
            if (Tail) clean(t, base);
            __syncthreads();  // all of it, and tile t - 1 has been read
            if (t + 1 < stop) {
                fetch(t + 1, other);
                if (t + 2 < stop) pages(t + 2);
            }
            const int k0 = t * kTile;
            if (!busy || (Tail && k0 >= wave_end)) return;
            f32x16 sc[2];
            {
                bf16x8 f[2][C <= 8 ? C : 1];
                if (C <= 8) {
#pragma unroll
                    for (int j = 0; j < 2; ++j)
#pragma unroll
                        for (int c = 0; c < C; ++c) f[j][c % 8] = *reinterpret_cast<const bf16x8 *>(base + kfrag[c] + j * 32 * W::row);
                    __builtin_amdgcn_sched_barrier(0);
                }
#pragma unroll
                for (int j = 0; j < 2; ++j) {
                    sc[j] = f32x16{};
#pragma unroll
                    for (int c = 0; c < C; ++c) {
                        if (C > 8) f[0][0] = *reinterpret_cast<const bf16x8 *>(base + kfrag[c] + j * 32 * W::row);
                        sc[j] = __builtin_amdgcn_mfma_f32_32x32x16_bf16(f[C <= 8 ? j : 0][C <= 8 ? c % 8 : 0], q[c], sc[j], 0, 0, 0);
                    }
                }
            }
            i16x8 vf[2][DB];
            auto read_v = [&](int j) __attribute__((always_inline)) {  // keys 16 j + 4 half + {0 .. 3} and + 8, transposed
#pragma unroll
                for (int d = 0; d < DB; ++d) {
                    char *p = base + vfrag[d] + j * 16 * W::row;
                    const i16x4 lo = __builtin_amdgcn_ds_read_tr16_b64_v4i16(LDS_I16X4(p));
                    const i16x4 hi = __builtin_amdgcn_ds_read_tr16_b64_v4i16(LDS_I16X4(p + 8 * W::row));
                    vf[j & 1][d] = __builtin_shufflevector(lo, hi, 0, 1, 2, 3, 4, 5, 6, 7);
                }
            };
            read_v(0);
            __builtin_amdgcn_sched_barrier(0);
            // lane (col, half): row col, keys k0 + 32 j + 8 (i / 4) + 4 half + i % 4
            if (Tail) {
                const uint64_t see = seen_keys(a, s, tok, k0, len) >> (4 * half);
                const uint32_t part[2] = {(uint32_t)see, (uint32_t)(see >> 32)};
#pragma unroll
                for (int i = 0; i < 32; ++i)
                    if (!((part[i / 16] >> (8 * (i % 16 / 4) + i % 4)) & 1)) sc[i / 16][i % 16] = -INFINITY;
            }
            float top = sc[0][0];
#pragma unroll
            for (int i = 1; i < 32; ++i) top = fmaxf(top, sc[i / 16][i % 16]);
            top *= a.scale_log2;
            if (__any(top > m + kSlack)) {
                const float mn = fmaxf(m, half_max(top));
                const float f = m == mn ? 1.0f : weight_of(m, mn);
                m = mn;
                l *= f;
#pragma unroll
                for (int d = 0; d < DB; ++d) o[d] *= f;
            }
            const float ref = m == -INFINITY ? 0.0f : m;
            bf16x8 pw[4];
            float s0 = 0.0f, s1 = 0.0f;
#pragma unroll
            for (int i = 0; i < 32; ++i) {
                const float p = ex2(__builtin_fmaf(sc[i / 16][i % 16], a.scale_log2, -ref));
                if (i & 1) s1 += p;
                else s0 += p;
                pw[i / 8][i % 8] = (__bf16)p;
            }
            l += s0 + s1;
#pragma unroll
            for (int j = 0; j < 4; ++j) {
                if (j < 3) read_v(j + 1);
#pragma unroll
                for (int d = 0; d < DB; ++d)
                    o[d] = __builtin_amdgcn_mfma_f32_32x32x16_bf16(__builtin_bit_cast(bf16x8, vf[j & 1][d]), pw[j], o[d], 0, 0, 0);
            }
            const uint32_t *marks = s_dirty[t & 1];
            if (Tail && (marks[0] | marks[1] | marks[2] | marks[3])) {
                // values that are infinite or NaN: zeros above, added here to the rows that see them
                for (int kk = 0; kk < kTile; ++kk) {
                    const int key = k0 + kk;
                    if (key < s.ctx || key >= len) continue;
                    int64_t page = table[key >> a.page_shift];
                    if (page < 0 || page >= a.n_pages) page = 0;
                    const uint16_t *v = vb + page * a.v_page + (key & ((1 << a.page_shift) - 1)) * a.v_slot;
                    const int src = col + 32 * ((kk & 7) >> 2), idx = (kk >> 5) * 16 + ((kk & 31) >> 3) * 4 + (kk & 3);
                    uint32_t pair = 0;
#pragma unroll
                    for (int i = 0; i < 16; ++i) {
                        const uint32_t y = __shfl(__builtin_bit_cast(u32x4, pw[i / 4])[i % 4], src, kWave);
                        if (i == idx >> 1) pair = y;
                    }
                    const float p = __uint_as_float(idx & 1 ? pair & 0xFFFF0000u : pair << 16);
#pragma unroll
                    for (int d = 0; d < DB; ++d)
#pragma unroll
                        for (int i = 0; i < 16; ++i) {
                            const float y = __uint_as_float((uint32_t)v[d * 32 + 8 * (i / 4) + 4 * half + i % 4] << 16);
                            if (!(fabsf(y) < INFINITY) && p != 0.0f) o[d][i] += p * y;
                        }
                }
            }
        };
        // tiles that every row sees whole, in pairs, then the others
        const int full = all_see / kTile < stop ? all_see / kTile : stop;
        while (t + 2 <= full) {
            step(lds0, lds1, std::false_type());
            ++t;
            step(lds1, lds0, std::false_type());
            ++t;
        }
        for (int odd = 0; t < stop; ++t, odd ^= 1) step(odd ? lds1 : lds0, odd ? lds0 : lds1, std::true_type());

        // ---- results: a lane has 4 consecutive elements of its row at a time ----
        if (any_lost) raise_flag(a.flags, STRIDE_FLAG_BAD_PAGE);
        l = poison ? __builtin_nanf("") : half_sum(l);
        const bool whole = at.unit == 0 && u1 == units;
        if (in) {
            const int head = at.head * a.group + r - tok * a.group, row = wave * 32 + col;
            if (whole) {
                const float inv = l == 0.0f ? 0.0f : 1.0f / l;
                uint16_t *out = static_cast<uint16_t *>(a.out) + (int64_t)(s.off + tok) * a.o_tok + (int64_t)head * a.o_head;
#pragma unroll
                for (int d = 0; d < DB; ++d)
#pragma unroll
                    for (int i = 0; i < 16; i += 4) {
                        const bf16x4 z = {(__bf16)(o[d][i] * inv), (__bf16)(o[d][i + 1] * inv),
                                          (__bf16)(o[d][i + 2] * inv), (__bf16)(o[d][i + 3] * inv)};
                        *reinterpret_cast<bf16x4 *>(out + d * 32 + 2 * i + 4 * half) = z;
                    }
                if (half == 0 && a.lse)
                    a.lse[(int64_t)(s.off + tok) * a.n_heads_q + head] =
                        l == 0.0f ? -INFINITY : (m + __builtin_amdgcn_logf(l)) * kLn2;
            } else {
                float *part = a.part + (int64_t)(2 * w + (at.unit == 0 ? 1 : 0)) * P;
#pragma unroll
                for (int d = 0; d < DB; ++d)
#pragma unroll
                    for (int i = 0; i < 16; i += 4)
                        *reinterpret_cast<f32x4 *>(part + row * D + d * 32 + 2 * i + 4 * half) =
                            f32x4{o[d][i], o[d][i + 1], o[d][i + 2], o[d][i + 3]};
                if (half == 0) {
                    part[Rows * D + row] = m;
                    part[Rows * D + Rows + row] = l;
                }
            }
        }
        if (at.same_item(to)) break;
        next_item<Rows>(a, s, at);
    }
}

template <int D, int Occ, bool OnePage>
__global__ __launch_bounds__(kThreads, Occ) void attend_wide_kernel(AttendArgs a) {
    attend_wide<D, OnePage>(a);
}

// The rows of an item that several workgroups shared.  One column of workgroups per border between two shares: the
// first border inside an item is responsible for it.  G groups of sixteen lanes take a row: a lane first has a
// part's m and l, then four elements of every G-th part at a time.  Latency bounds it: what the first kernel found
// is read instead of summed again, and a row's parts are asked for eight at a time by each group.
template <int DT, int D, int Rows, int G>
__global__ __launch_bounds__(kThreads) void attend_merge_kernel(AttendArgs a) {
    constexpr int P = Rows * (D + 2), E = (D + 63) / 64, L = 16 * G;
    const int lane = threadIdx.x & (kWave - 1), mine = lane & (L - 1), sub = lane & 15, grp = mine >> 4;
    const int w = blockIdx.x + 1;
    const Place at = a.at[w], prev = a.at[w - 1];
    if (at.unit == 0 || (at.same_item(prev) && prev.unit > 0)) return;
    uint32_t flag = 0;
    const Seq s = sequence(a, at.seq, flag);
    // The item's shares: w - 1, whose partial result is its second (the item begins inside it), and w, w + 1, ... while
    // they begin inside the item; of those, the ones that are not empty.  Bit i of a round: share w - 1 + i0 + i.
    auto shares = [&](int i0, bool &more) __attribute__((always_inline)) {
        const int i = w - 1 + i0 + lane;
        bool in = i == w - 1, full = in;
        if (i >= w && i < a.workers) {
            const Place p = a.at[i], e = a.at[i + 1];
            in = p.same_item(at);
            full = in && !at_end(p, e);
        }
        const uint64_t all = __ballot(in);
        more = all == ~0ull;
        const int run = more ? kWave : __builtin_ctzll(~all);
        return __ballot(full && lane < run);
    };
    auto part = [&](int i) { return a.part + (int64_t)(2 * (w - 1 + i) + (i == 0 ? 1 : 0)) * P; };
    const int row = blockIdx.y * (kThreads / L) + threadIdx.x / L, r = at.rt * Rows + row;
    const bool real = r < s.n * a.group;  // all lanes take part in the rounds below
    float m = -INFINITY, sum = 0.0f;
    f32x4 y[E] = {};
    bool more = true;
    for (int i0 = 0; more; i0 += kWave) {
        const uint64_t todo = shares(i0, more);
        for (int k0 = 0; k0 < kWave && todo >> k0; k0 += L) {
            float pm = -INFINITY, pl = 0.0f;
            if (real && (todo >> (k0 + mine) & 1)) {
                const float *p = part(i0 + k0 + mine) + Rows * D + row;
                pm = p[0];
                pl = p[Rows];
            }
            float mn = fmaxf(m, pm);
#pragma unroll
            for (int o = L / 2; o > 0; o >>= 1) mn = fmaxf(mn, __shfl_xor(mn, o, kWave));
            const float old = m == mn ? 1.0f : weight_of(m, mn);
            const float f = pm == mn ? 1.0f : weight_of(pm, mn);
            m = mn;
            pl *= f;
#pragma unroll
            for (int o = L / 2; o > 0; o >>= 1) pl += __shfl_xor(pl, o, kWave);
            sum = sum * old + pl;
#pragma unroll
            for (int e = 0; e < E; ++e) y[e] *= old;
            constexpr int B = 8;  // parts asked for at once
#pragma unroll
            for (int b = 0; b < 16; b += B) {
                if (!(todo >> (k0 + b * G))) continue;
                f32x4 x[B][E];
#pragma unroll
                for (int i = 0; i < B; ++i) {
                    const int k = k0 + (b + i) * G + grp;
                    const float *p = part(i0 + k) + row * D + sub * 4;
#pragma unroll
                    for (int e = 0; e < E; ++e) {
                        x[i][e] = f32x4{};
                        if (real && (todo >> k & 1) && e * 64 + sub * 4 < D) x[i][e] = *reinterpret_cast<const f32x4 *>(p + e * 64);
                    }
                }
#pragma unroll
                for (int i = 0; i < B; ++i) {
                    const float g = __shfl(f, (lane & ~(L - 1)) + (b + i) * G + grp, kWave);
#pragma unroll
                    for (int e = 0; e < E; ++e) y[e] += g * x[i][e];
                }
            }
        }
    }
#pragma unroll
    for (int o = 16; o < L; o <<= 1)
#pragma unroll
        for (int e = 0; e < E; ++e)
#pragma unroll
            for (int k = 0; k < 4; ++k) y[e][k] += __shfl_xor(y[e][k], o, kWave);
    if (!real || grp != 0) return;
    const int tok = r / a.group, head = at.head * a.group + r - tok * a.group;
    const float inv = sum == 0.0f ? 0.0f : 1.0f / sum;
    const int64_t o = (int64_t)(s.off + tok) * a.o_tok + (int64_t)head * a.o_head + sub * 4;
#pragma unroll
    for (int e = 0; e < E; ++e) {
        if (e * 64 + sub * 4 >= D) continue;
        const f32x4 z = y[e] * inv;
        if (DT == STRIDE_BF16)
            *reinterpret_cast<bf16x4 *>(static_cast<uint16_t *>(a.out) + o + e * 64) = bf16x4{(__bf16)z[0], (__bf16)z[1], (__bf16)z[2], (__bf16)z[3]};
        else
            *reinterpret_cast<f32x4 *>(static_cast<float *>(a.out) + o + e * 64) = z;
    }
    if (sub == 0 && a.lse)
        a.lse[(int64_t)(s.off + tok) * a.n_heads_q + head] = sum == 0.0f ? -INFINITY : (m + __builtin_amdgcn_logf(sum)) * kLn2;
}

// ---- the choice of a form ----

struct Form {
    int rows, workers;  // rows of a tile: 16 or 32 with the keys split over the waves, 128 with the rows
};

// By the mean number of rows of a sequence's key head (tokens times the group of query heads), which the host knows; it
// decides for all of a call's sequences.  63 single tokens and a turn of 400, each over 8,000 keys, take 549 us in tiles of
// 16, and 340 and 57 in calls of their own.
// 32 sequences of 500 to 8,192 keys, 8 key heads of 128 elements, bf16:
//   16 rows                       113 us in tiles of 16, 120 in tiles of 128 (one token of 64 long sequences 447, or 499)
//   32 rows                       119 us in tiles of 128, 177 in tiles of 32 with the keys split
//   32 rows of 256 elements       371 us as two tiles of 16, 517 in one of 128 (one workgroup per CU, and registers
//                                 that do not hold its accumulators); 48 rows 620, or 526
// In float, where products of 16 x 16 x 4 bound it: 32 rows 271 us in tiles of 32, 378 in tiles of 16; of 256
// elements 760 in tiles of 16, 1,845 in tiles of 32, whose accumulators pass the registers.
// Two workgroups per CU where registers and LDS hold both.

Form form_of(const stride_kv_cache &c, int64_t n_q, int32_t n_heads_q) {
    const int64_t rows = (n_q * (n_heads_q / c.n_heads) + c.n_seqs - 1) / c.n_seqs;
    const bool bf16 = c.dtype == STRIDE_BF16, large = c.head_dim > 128;
    const int workers = kCUs * (bf16 && !large ? 2 : 1);
    if (bf16) return {rows > (large ? 32 : 16) ? 128 : 16, workers};
    return {rows <= 16 || large ? 16 : 32, workers};
}

size_t head_bytes(int workers) { return ((size_t)(workers + 1) * sizeof(Place) + 255) / 256 * 256; }

template <int DT, int D, int Rows>
hipError_t launch_merge(const AttendArgs &a, hipStream_t stream) {
    // few rows can have many parts each (a long sequence of one key head: as many as there are workgroups): a wave
    // per row then (one token of 8 sequences 18.1 us, 18.8 with sixteen lanes per row); of 128 rows every border has a
    // quarter as many workgroups with sixteen lanes per row (turns of 129 to 1,024 tokens 153 us, or 177)
    constexpr int G = Rows == 128 ? 1 : 4;
    attend_merge_kernel<DT, D, Rows, G><<<dim3(a.workers - 1, Rows * 16 * G / kThreads), kThreads, 0, stream>>>(a);
    return hipGetLastError();
}

template <int D, int Occ, bool OnePage>
hipError_t launch_wide(const AttendArgs &a, hipStream_t stream) {
    attend_wide_kernel<D, Occ, OnePage><<<a.workers, kThreads, 0, stream>>>(a);
    const hipError_t e = hipGetLastError();
    return e != hipSuccess ? e : launch_merge<STRIDE_BF16, D, 128>(a, stream);
}

template <int DT, int D, int RT, int Occ, bool OnePage>
hipError_t launch_form(const AttendArgs &a, hipStream_t stream) {
    attend_kernel<DT, D, RT, Occ, OnePage><<<a.workers, kThreads, 0, stream>>>(a);
    const hipError_t e = hipGetLastError();
    return e != hipSuccess ? e : launch_merge<DT, D, 16 * RT>(a, stream);
}

// Whether `keys` keys from a multiple of them on lie in one page, within 32 bits of bytes of each other.
bool one_page(const stride_kv_cache &c, int keys) {
    const int64_t size = c.dtype == STRIDE_BF16 ? 2 : 4, most = (int64_t)1 << 31;
    auto near = [&](int64_t stride) { return stride >= 0 && stride < most / (keys * size) - c.head_dim; };
    return c.page_size >= keys && near(c.k_slot) && near(c.v_slot);
}

template <int DT, int D>
hipError_t launch_rows(const AttendArgs &a, const stride_kv_cache &c, int rows, hipStream_t stream) {
    constexpr int Occ = DT == STRIDE_BF16 && D <= 128 ? 2 : 1;
    if constexpr (DT == STRIDE_BF16)
        if (rows == 128)
            return one_page(c, kTile) ? launch_wide<D, Occ, true>(a, stream) : launch_wide<D, Occ, false>(a, stream);
    const bool one = one_page(c, 16 * Type<DT>::T);
    if constexpr (DT == STRIDE_F32 && D <= 128)
        if (rows == 32) return one ? launch_form<DT, D, 2, Occ, true>(a, stream) : launch_form<DT, D, 2, Occ, false>(a, stream);
    return one ? launch_form<DT, D, 1, Occ, true>(a, stream) : launch_form<DT, D, 1, Occ, false>(a, stream);
}

template <int DT>
hipError_t launch_dim(const AttendArgs &a, const stride_kv_cache &c, int rows, hipStream_t stream) {
    switch (c.head_dim) {
        case 64: return launch_rows<DT, 64>(a, c, rows, stream);
        case 96: return launch_rows<DT, 96>(a, c, rows, stream);
        case 128: return launch_rows<DT, 128>(a, c, rows, stream);
        default: return launch_rows<DT, 256>(a, c, rows, stream);
    }
}

}  // namespace

size_t attention_ws_bytes(const stride_kv_cache &c, int64_t n_q, int32_t n_heads_q) {
    if (n_q == 0 || c.n_seqs == 0) return 256;
    const Form f = form_of(c, n_q, n_heads_q);
    return head_bytes(f.workers) + (size_t)f.workers * 2 * f.rows * (c.head_dim + 2) * sizeof(float);
}

hipError_t launch_tree_attention(const stride_kv_cache &c, int64_t n_q, int32_t n_heads_q, const void *q,
                                 int64_t q_tok, int64_t q_head, const int32_t *q_off,
                                 const int32_t *ctx_len, const uint64_t *tree_mask, int32_t mask_words,
                                 float scale, void *out, int64_t out_tok, int64_t out_head, float *lse,
                                 uint32_t *flags, void *ws, hipStream_t stream) {
    if (n_q == 0 || c.n_seqs == 0) return hipSuccess;
    const Form f = form_of(c, n_q, n_heads_q);
    AttendArgs a;
    a.q = q;
    a.k = c.k;
    a.v = c.v;
    a.out = out;
    a.lse = lse;
    a.at = static_cast<Place *>(ws);
    a.part = reinterpret_cast<float *>(static_cast<char *>(ws) + head_bytes(f.workers));
    a.table = c.page_table;
    a.q_off = q_off;
    a.ctx = ctx_len;
    a.mask = tree_mask;
    a.flags = flags;
    a.q_tok = q_tok;
    a.q_head = q_head;
    a.o_tok = out_tok;
    a.o_head = out_head;
    a.k_page = c.k_page;
    a.k_slot = c.k_slot;
    a.k_head = c.k_head;
    a.v_page = c.v_page;
    a.v_slot = c.v_slot;
    a.v_head = c.v_head;
    a.table_ld = c.table_ld;
    a.n_pages = c.n_pages < INT32_MAX ? (int32_t)c.n_pages : INT32_MAX;
    a.max_len = (int64_t)c.max_pages * c.page_size;
    a.n_q = (int32_t)n_q;
    a.page_shift = __builtin_ctz((unsigned)c.page_size);
    a.n_seqs = c.n_seqs;
    a.n_heads = c.n_heads;
    a.n_heads_q = n_heads_q;
    a.group = n_heads_q / c.n_heads;
    a.mask_words = mask_words;
    a.workers = f.workers;  // a power of two
    a.log_workers = __builtin_ctz((unsigned)f.workers);
    a.scale_log2 = scale * kLog2e;
    return c.dtype == STRIDE_BF16 ? launch_dim<STRIDE_BF16>(a, c, f.rows, stream)
                                  : launch_dim<STRIDE_F32>(a, c, f.rows, stream);
}

}  // namespace stride
