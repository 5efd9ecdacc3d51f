// Tokens drawn from logits with given uniforms: temperature, top-k, top-p, min-p.
//
// A row's tokens in descending order of their logits, ties by index; w_i = exp((z_i - z_max) / T), C_n = w_1 + ... + w_n:
//   n_k = min(top_k, F)          F: logits above -inf
//   n_p = least n with C_n >= top_p C_{n_k}
//   n_m = number of i with w_i >= min_p
//   n   = min(n_k, n_p, n_m);    token = first j with C_j > u C_n;    logp = (z_j - z_max) / T - ln C_n
//
// A draw lies next to one of up to a million borders, so the masses have to be right to far more digits than float32 holds if the token
// is to be the definition's, and the same whichever way the row is cut.  All masses are float64, or integers of which each weight has 43 bits
// and more (right to 1e-13 of it), and none depends on an order:
//
//   16-bit logits   A row holds at most 65536 different numbers: one pass counts them, by integer additions in shared memory, and all the
//                   rest is arithmetic on a few thousand (number, count) pairs.  Bound by those additions (one warp's 32 fall on the 32
//                   banks at random, 3 cycles) where the row's bytes take 2.7 of the same cycles.
//   short float32   Up to 2048 are sorted, and their masses added up in that order.
//   float32         A row holds any numbers, so they go into 2048 bins of equal depth below the maximum, each with its count and what its
//                   mass falls short of the count, in fixed point relative to the bin's top (integers again).  The few hundred elements of the bin that holds a border
//                   are listed, and dealt out over the keys in it until a part holds one element or one number; a bin of more than
//                   2048 (many equal ones) in passes over the row.  16-bit rows that the counting does not fit (very large or
//                   very small logits, more than 65535 equal ones) go the same way.
//
// A cluster of CTAs shares a row, each with a contiguous piece of it: one CTA when there are rows enough, up to eight for a few.
#include "ppow_checked.cuh"
#include "ppow_rows.cuh"

#include <algorithm>
#include <cooperative_groups.h>

namespace ppow {
namespace cg = cooperative_groups;

constexpr int SAMPLE_CTAS = 8, WARPS_MOST = 16;
constexpr int32_t SAMPLE_MAX_VOCAB = 1 << 22;
constexpr int GROUP = 128;               // numbers of one sign whose counts and masses are summed up together: four to a lane
constexpr int SEARCH_GROUP = 32;         // the same of the bins of a search
constexpr int SEARCH_BINS = 2048;
constexpr double SEARCH_NATS = 56.0;     // what lies deeper than this below the maximum has no mass: 2^22 exp(-56) is 2e-18
constexpr uint32_t LOWEST_FINITE = 0x00800000u;     // key of the lowest float32 above -inf
// What weights fall short of a bin's top is added up in fixed point, in three limbs of 13 bits, so that 2^19 elements to a CTA fit words of 32.
constexpr int LIMBS = 3, LIMB_BITS = 13;
constexpr double LIMBS_HOLD = 549755813888.0;        // 2^39
constexpr int32_t PIECE_MOST = 1 << 19;

struct SampleJob {
    const void *logits;
    int64_t stride;
    const float *uniforms;
    int32_t R, V, top_k;                 // top_k <= 0: off
    double temperature, top_p, min_p;    // top_p >= 1 and min_p <= 0: off
    int32_t *tokens;
    float *logp;
    int32_t *kept;                       // or null
};

// ---- formats ----------------------------------------------------------------------------------------
// Counting: a word for each of WORDS neighbouring magnitudes (by their bits) from LOW on; positive numbers in the low half, negative ones
// in the high half, so that neighbours lie in different banks.
//   bfloat16   64 exponents, 2^-51 <= |z| < 2^13.  A magnitude's word is its low 13 bits, whatever LOW is.  Zeros are counted apart.
//   float16    all magnitudes below 2^11; a magnitude's word is the magnitude.  -0 is added to +0 afterwards.
template <int DTYPE> struct Counted;
template <> struct Counted<PPOW_BF16> {
    static constexpr uint32_t INF = 0x7f80u, LOW = 76 * 128, WORDS = 64 * 128, MASK = WORDS - 1;
    static constexpr int THREADS = 256, CTAS = 4;            // of a block; blocks on an SM
    static constexpr double LIMIT = 8192.0;
    static __device__ __forceinline__ uint32_t most(uint32_t a, uint32_t b) { return max_bf16x2(a, b); }     // NaN is passed over
    static __device__ __forceinline__ uint32_t equal(uint32_t a, uint32_t b)
    {
        return __heq2_mask(*reinterpret_cast<const __nv_bfloat162 *>(&a), *reinterpret_cast<const __nv_bfloat162 *>(&b));
    }
};
template <> struct Counted<PPOW_F16> {
    static constexpr uint32_t INF = 0x7c00u, LOW = 0, WORDS = 26 * 1024, MASK = 0x7fffu;
    static constexpr int THREADS = 512, CTAS = 2;
    static constexpr double LIMIT = 2048.0;
    static __device__ __forceinline__ uint32_t most(uint32_t a, uint32_t b)
    {
        const __half2 m = __hmax2(UnitF16::h2(a), UnitF16::h2(b));
        return *reinterpret_cast<const uint32_t *>(&m);
    }
    static __device__ __forceinline__ uint32_t equal(uint32_t a, uint32_t b) { return __heq2_mask(UnitF16::h2(a), UnitF16::h2(b)); }
};
// Groups of one sign, by rising magnitude; positive ones first, then the zeros (where they are counted apart), then negative ones.
template <int DTYPE> struct Groups {
    using F = Counted<DTYPE>;
    static constexpr int SIDE = F::WORDS / GROUP, ZERO = SIDE, ALL = 2 * SIDE + 1;
    static_assert(F::WORDS % GROUP == 0 && F::LOW % GROUP == 0, "whole groups");
    static_assert(SIDE % SAMPLE_CTAS == 0, "equal shares");
    static __device__ __forceinline__ bool negative(int group) { return group > ZERO; }
    static __device__ __forceinline__ int side(int group) { return group > ZERO ? group - ZERO - 1 : group; }
    // first word of a group of either sign
    static __device__ __forceinline__ int word(int side) { return (int)(((uint32_t)side * GROUP + F::LOW) & F::MASK); }
    // the i-th group in descending order
    static __device__ __forceinline__ int at(int i) { return i < SIDE ? SIDE - 1 - i : i; }
    // the i-th number of a group, by rising magnitude
    static __device__ __forceinline__ float number(int group, int i)
    {
        return group == ZERO ? 0.0f : Storage<DTYPE>::get((uint16_t)(F::LOW + side(group) * GROUP + i + (negative(group) ? 0x8000 : 0)));
    }
};
constexpr int GROUPS_MOST = Groups<PPOW_F16>::ALL;
static_assert(GROUPS_MOST >= Groups<PPOW_BF16>::ALL && GROUPS_MOST >= SEARCH_BINS / SEARCH_GROUP * 5 / 4, "groups");

// Order-preserving key of a float32 (-0 is +0), and back.
__device__ __forceinline__ uint32_t key_of(float z)
{
    const uint32_t b = __float_as_uint(z + 0.0f);
    return b & 0x80000000u ? ~b : b | 0x80000000u;
}
__device__ __forceinline__ float float_of(uint32_t key) { return __uint_as_float(key & 0x80000000u ? key ^ 0x80000000u : ~key); }

// This CTA's piece of a row in 16-byte units; what lies around the row in its first and last unit reads as -inf.
template <int DTYPE> struct Piece {
    using S = Storage<DTYPE>;
    using T = typename S::type;
    static constexpr int E = S::PER_UNIT;
    const uint4 *base;
    int32_t head, span, units, begin, end;
    __device__ __forceinline__ Piece(const SampleJob &job, int64_t row, int rank, int ctas)
    {
        const uintptr_t a = reinterpret_cast<uintptr_t>(static_cast<const T *>(job.logits) + row * job.stride);
        base = reinterpret_cast<const uint4 *>(a & ~(uintptr_t)15);
        head = (int32_t)((a & 15) / sizeof(T));
        span = head + job.V;
        units = (span + E - 1) / E;
        begin = (int32_t)((int64_t)units * rank / ctas);
        end = (int32_t)((int64_t)units * (rank + 1) / ctas);
    }
    __device__ __forceinline__ uint4 load(int32_t u) const
    {
        uint4 w = __ldg(base + u);
        if (u == 0 || u == units - 1) {
            const int lo = u == 0 ? head : 0, hi = min(E, span - u * E);
            if constexpr (DTYPE == PPOW_F32) {
                if (0 < lo || 0 >= hi) w.x = 0xff800000u;
                if (1 < lo || 1 >= hi) w.y = 0xff800000u;
                if (2 < lo || 2 >= hi) w.z = 0xff800000u;
                if (3 < lo || 3 >= hi) w.w = 0xff800000u;
            } else {
                mask_halves(w, lo, hi, 0x8000u | Counted<DTYPE>::INF);
            }
        }
        return w;
    }
    __device__ __forceinline__ int32_t token(int32_t u, int e) const { return u * E + e - head; }
};

// ---- borders ----------------------------------------------------------------------------------------
struct Place {
    int item;
    uint32_t count;          // elements before it
    double mass;             // and their mass
};

// The first place where the count reaches `count`, the mass reaches `from` and passes `above`: one of the three is asked for, the
// others hold everywhere (no branches: each row runs through this in one warp).
struct Target {
    uint32_t count;
    double from, above;
    static __device__ __forceinline__ Target at_count(uint32_t n) { return {n, -INFINITY, -INFINITY}; }
    static __device__ __forceinline__ Target mass_from(double m) { return {0, m, -INFINITY}; }
    static __device__ __forceinline__ Target mass_above(double m) { return {0, -INFINITY, m}; }
    __device__ __forceinline__ bool by_count() const { return count > 0; }
    __device__ __forceinline__ bool met(uint32_t c, double m) const { return (c >= count) & (m >= from) & (m > above); }
};

// What lies up to each of the items 0 .. n-1 (n <= 32 PER, descending), PER neighbours to a lane, and the item that holds a border.  The
// whole warp calls, every lane has the result.
struct Part {
    uint32_t count;
    double mass;
};
template <int PER> struct Scan {
    uint32_t count[PER + 1];         // before the lane's first item; up to and with each
    double mass[PER + 1];

    // get(item): count and mass of one
    template <typename Get> __device__ __forceinline__ Scan(int n, const Place &before, Get &&get)
    {
        const int lane = threadIdx.x & 31;
        count[0] = 0;
        mass[0] = 0.0;
#pragma unroll
        for (int i = 0; i < PER; ++i) {
            Part part = {0, 0.0};
            if (lane * PER + i < n) part = get(lane * PER + i);
            count[i + 1] = count[i] + part.count;
            mass[i + 1] = mass[i] + part.mass;
        }
        uint32_t c = count[PER];
        double m = mass[PER];
#pragma unroll
        for (int o = 1; o < 32; o <<= 1) {
            const uint32_t c2 = __shfl_up_sync(0xffffffffu, c, o);
            const double m2 = __shfl_up_sync(0xffffffffu, m, o);
            if (lane >= o) c += c2, m += m2;
        }
        c = __shfl_up_sync(0xffffffffu, c, 1);
        m = __shfl_up_sync(0xffffffffu, m, 1);
        c = before.count + (lane ? c : 0);
        m = before.mass + (lane ? m : 0.0);
#pragma unroll
        for (int i = 0; i <= PER; ++i) {
            count[i] += c;
            mass[i] += m;
        }
    }
    __device__ __forceinline__ Part all() const { return {__shfl_sync(0xffffffffu, count[PER], 31), __shfl_sync(0xffffffffu, mass[PER], 31)}; }
    // Only items with elements: the lanes' sums are rounded in orders of their own, so behind the last element one may be the first to reach
    // a mass next to the whole.  If rounding leaves the border to none, the last item that adds some mass, or an element.
    __device__ __forceinline__ Place find(Target target) const
    {
        const int lane = threadIdx.x & 31;
        for (int again = 0;; ++again) {
            Place p = {-1, 0, 0.0};
#pragma unroll
            for (int i = PER - 1; i >= 0; --i) {
                const bool here = count[i + 1] > count[i] && target.met(count[i + 1], mass[i + 1]);
                p = {here ? lane * PER + i : p.item, here ? count[i] : p.count, here ? mass[i] : p.mass};
            }
            const uint32_t who = __ballot_sync(0xffffffffu, p.item >= 0);
            if (who || again == 2) {
                const int from = who ? __ffs(who) - 1 : 31;
                return {max(__shfl_sync(0xffffffffu, p.item, from), 0), __shfl_sync(0xffffffffu, p.count, from), __shfl_sync(0xffffffffu, p.mass, from)};
            }
            const Part sum = all();
            target = target.by_count() || again ? Target::at_count(sum.count) : Target::mass_from(sum.mass);
        }
    }
};

// An element: its number, its place in the order, the mass up to and with it.  Where its token is not known, it is the rank-th (from 0) of
// the `have` elements with that number, by index.
struct Element {
    float value;
    uint32_t n;
    double total;
    int32_t token;           // -1: not known
    uint32_t rank, have;
};

// Which of `have` equal elements of this weight, behind `before`, the border falls on.
__device__ __forceinline__ Element choose(const Target &target, const Place &before, float value, uint32_t have, double weight)
{
    uint32_t rank = 0;
    if (have <= 1) {
    } else if (target.by_count()) {
        rank = min(target.count - before.count, have) - 1;
    } else {
        // the quotient is right to a small part of 1, but for weights below 1e-13 of the mass, which no border can tell apart
        const double q = floor((fmax(target.from, target.above) - before.mass) / weight);
        rank = q >= (double)have ? have - 1 : q > 0.0 ? (uint32_t)q : 0;
        if (rank > 0 && target.met(0, before.mass + rank * weight)) --rank;
        if (rank < have - 1 && !target.met(0, before.mass + (rank + 1) * weight)) ++rank;
    }
    return {value, before.count + rank + 1, before.mass + (rank + 1) * weight, -1, rank, have};
}

struct SampleShared {
    uint32_t group_count[GROUPS_MOST];
    double group_mass[GROUPS_MOST];
    uint32_t warp_count[2][WARPS_MOST];
    uint32_t none, low, zeros;               // -inf; below the counted range; zeros that are counted apart
    uint32_t flags, within, top;             // SAMPLE_*; within min_p; key of the maximum
    uint32_t here;                           // elements of the drawn number in this piece
    uint32_t listed, only_key;
    int32_t only_token;
    Element drawn;
    Place place;
};
enum : uint32_t { SAMPLE_BAD = 1, SAMPLE_ODD = 2 };      // NaN or +inf; a row that counting does not fit

__device__ __forceinline__ void meet(const cg::cluster_group &cluster, int ctas)
{
    if (ctas == 1)
        __syncthreads();
    else
        cluster.sync();
}

// The whole distribution of a row from find(target), which gives the element on a border: what is kept, and the draw.
// F: elements above -inf, of which `massive` carry the mass `all`.
template <typename Find>
__device__ __forceinline__ void decide(const SampleJob &job, float u, uint32_t F, uint32_t massive, double all, uint32_t within, Find &&find,
                                       Element &drawn, uint32_t &n, double &total)
{
    n = job.top_k > 0 && (uint32_t)job.top_k < F ? (uint32_t)job.top_k : F;
    total = all;
    u = fminf(fmaxf(u, 0.0f), 0x1.fffffep-1f);               // NaN is 0
    // one copy of the code of `find` for all borders: it is long, and each row runs through it once
#pragma unroll 1
    for (int step = 0; step < 5; ++step) {
        Target target = Target::at_count(n);
        if (step == 0) {
            if (n >= massive) continue;
        } else if (step == 1) {
            if (!(job.top_p < 1.0)) continue;
            target = Target::mass_from(job.top_p * total);
        } else if (step == 2) {
            if (!(job.min_p > 0.0 && within < n)) continue;
            n = within;
            target = Target::at_count(n);
        } else if (step == 3) {
            target = Target::mass_above((double)u * total);
        } else if (drawn.n <= n) {
            continue;
        }
        const Element e = find(target);
        if (step >= 3)
            drawn = e;
        else if (step != 1 || e.n < n)
            n = e.n, total = e.total;
    }
}

// The index of an element of this piece that `matches` accepts and `behind` others follow, searched from the end, where the pass over the row
// was last and the L2 cache still holds most, in rounds: each warp a stretch of neighbouring units, the next round's on their way while
// this one's are counted.  matches: a byte with a bit for each of a unit's elements, that of element e at e / 2 + 4 (e % 2) where there are
// eight, at e where there are four.  Out of line: inlined, it takes registers from the rest (4096 x 128256 bf16: 471 us, so 420).
// From the row's start the same takes 428 us.
template <int THREADS, int DTYPE, typename Matches>
__device__ __noinline__ void locate(const Piece<DTYPE> piece, uint32_t behind, SampleShared &sh, int32_t *token, const Matches matches)
{
    constexpr int DEEP = 4;                  // 8: 13 % slower, what is read beyond the token costs more than the rounds
    const int lane = threadIdx.x & 31, warp = threadIdx.x >> 5;
    uint32_t seen = 0;
    int turn = 0;
    uint4 next[DEEP];
    auto unit = [&](int32_t base, int q) { return base - (warp * DEEP + q) * 32 - lane; };
    auto fetch = [&](int32_t base) {
#pragma unroll
        for (int q = 0; q < DEEP; ++q)
            if (unit(base, q) >= piece.begin) next[q] = piece.load(unit(base, q));
    };
    fetch(piece.end - 1);
    for (int32_t base = piece.end - 1; base >= piece.begin; base -= THREADS * DEEP, turn ^= 1) {
        uint32_t bits = 0;
#pragma unroll
        for (int q = 0; q < DEEP; ++q)
            if (unit(base, q) >= piece.begin) bits |= matches(next[q]) << (q * 8);
        fetch(base - THREADS * DEEP);
        const uint32_t mine = __reduce_add_sync(0xffffffffu, __popc(bits));
        if (lane == 0) sh.warp_count[turn][warp] = mine;
        __syncthreads();
        const uint32_t c = lane < (THREADS / 32) ? sh.warp_count[turn][lane] : 0u;
        uint32_t before = seen + __reduce_add_sync(0xffffffffu, lane < warp ? c : 0u);
        seen += __reduce_add_sync(0xffffffffu, c);
        if (before <= behind && behind < before + mine) {
            for (int q = 0; q < DEEP; ++q) {
                const uint32_t m = bits >> (q * 8) & 0xffu;
                uint32_t upto = __popc(m);
#pragma unroll
                for (int o = 1; o < 32; o <<= 1) {
                    const uint32_t v = __shfl_up_sync(0xffffffffu, upto, o);
                    if (lane >= o) upto += v;
                }
                uint32_t from = before + upto - __popc(m);
#pragma unroll
                for (int e = Piece<DTYPE>::E - 1; e >= 0; --e)
                    if (m >> (Piece<DTYPE>::E == 8 ? e / 2 + e % 2 * 4 : e) & 1) {
                        if (from == behind) *token = piece.token(unit(base, q), e);
                        ++from;
                    }
                before += __shfl_sync(0xffffffffu, upto, 31);
            }
        }
        if (seen > behind) return;           // the same for the whole CTA
    }
}

// Elements with the bits of one float32 key; elements of 16-bit units equal to a number (the zeros are one).
template <int DTYPE> struct HasKey {
    uint32_t key;
    __device__ __forceinline__ uint32_t operator()(const uint4 &w) const
    {
        constexpr int E = Storage<DTYPE>::PER_UNIT;
        float z[E];
        Storage<DTYPE>::unpack(w, z);
        uint32_t bits = 0;
#pragma unroll
        for (int e = 0; e < E; ++e) bits |= (z[e] > -INFINITY && key_of(z[e]) == key) ? 1u << (E == 8 ? e / 2 + e % 2 * 4 : e) : 0u;
        return bits;
    }
};
template <int DTYPE> struct Equals {
    uint32_t both;           // the number, twice
    __device__ __forceinline__ uint32_t operator()(const uint4 &w) const
    {
        using F = Counted<DTYPE>;
        const uint32_t m = (F::equal(w.x, both) & 0x00010001u) | (F::equal(w.y, both) & 0x00020002u) | (F::equal(w.z, both) & 0x00040004u) |
                           (F::equal(w.w, both) & 0x00080008u);
        return (m | m >> 12) & 0xffu;
    }
};

// ---- search: any row --------------------------------------------------------------------------------
// Counts of bins and what their masses fall short of them, in fixed point as limbs, of this CTA; counts and masses of the cluster.
template <int BINS> struct BinCounts {
    uint32_t count[BINS], limb[LIMBS][BINS];
};
template <int BINS> struct BinTotals {
    uint32_t count[BINS];
    double mass[BINS];
};
template <int BINS> struct SearchBins {
    static constexpr int SUB = BINS / 4, LIST = BINS;        // parts of a bin; elements that are listed
    union {
        BinCounts<BINS> depth;
        struct {
            BinCounts<SUB> sub;
            unsigned long long list[LIST];                   // of this piece: key << 32 | token
        };
    };
    BinTotals<BINS> depths;
    BinTotals<SUB> subs;
};

template <int DTYPE, int THREADS, int BINS> struct Search {
    using S = Storage<DTYPE>;
    using Bins = SearchBins<BINS>;
    static constexpr int E = S::PER_UNIT, SUB = Bins::SUB;
    static constexpr double STEP = SEARCH_NATS / (BINS - 1);         // depth of a bin, nats
    // A weight lies between exp(-STEP) and 1 of its bin's top, so only the small rest to 1 is held, 2^44 (2^43 of wider bins) to 1: off by
    // 2^-45 (2^-44) of the bin's top, and not at all at the maximum.  SLACK keeps it above 0 where the rounding of depth_bin puts a number
    // into the bin below its own, by up to 1e-5.
    static constexpr double SLACK = 0x1p-15, UNIT = (STEP + 2 * SLACK) * 0x1p44 < LIMBS_HOLD ? 0x1p44 : 0x1p43;
    static_assert((STEP + 2 * SLACK) * UNIT < LIMBS_HOLD, "limbs");
    const SampleJob &job;
    const Piece<DTYPE> &piece;
    const cg::cluster_group &cluster;
    int rank, ctas;
    SampleShared &sh;
    Bins &bins;
    double top, per_nat;                     // maximum; 1 / temperature
    float top32, scale;                      // the same maximum; bins per logit
    int listed;                              // the elements looked at: those of the list, so many, or, < 0, all of the piece

    template <typename T> __device__ __forceinline__ T *of(T *p, int r) const { return ctas == 1 ? p : cluster.map_shared_rank(p, r); }
    // f(z, token) for every logit; those around the row are -inf
    template <typename F> __device__ __forceinline__ void each(F &&f) const
    {
        if (listed >= 0) {
            for (int i = threadIdx.x; i < listed; i += THREADS) f(float_of((uint32_t)(bins.list[i] >> 32)), (int32_t)(uint32_t)bins.list[i]);
            return;
        }
        // one unit at a time: more of them in flight make the code longer and the kernel slower (4: 535 us, 1: 507, 512 x 152064)
        for (int32_t u = piece.begin + (int32_t)threadIdx.x; u < piece.end; u += THREADS) {
            float z[E];
            S::unpack(piece.load(u), z);
#pragma unroll
            for (int e = 0; e < E; ++e) f(z[e], piece.token(u, e));
        }
    }
    __device__ __forceinline__ double weight(float z) const { return exp(((double)z - top) * per_nat); }
    // In float32, whose differences and products keep the order: a bin is a stretch of numbers.  Its rounding moves a border by 1e-5 nats.
    __device__ __forceinline__ int depth_bin(float z) const { return (int)fminf((top32 - z) * scale, (float)(BINS - 1)); }
    // The lowest key in lo .. hi whose number `accepts`, which all above it are and hi's is: 32 places at a time, by each warp for itself.
    template <typename Accepts> __device__ uint32_t lowest_key(uint32_t lo, uint32_t hi, Accepts &&accepts) const
    {
        const uint32_t lane = threadIdx.x & 31;
        while (lo < hi) {
            const uint32_t step = (hi - lo) / 32 + 1, at = lo + lane * step;     // lane 0 is lo
            const uint32_t yes = __ballot_sync(0xffffffffu, at < hi ? accepts(float_of(at)) : true);
            const int first = __ffs(yes) - 1;                // 0: lo itself; none (step 1 and 32 places): hi
            if (first == 0) return lo;
            const uint32_t last_no = lo + (uint32_t)(first < 0 ? 31 : first - 1) * step, first_yes = first < 0 ? hi : lo + (uint32_t)first * step;
            lo = last_no + 1, hi = min(first_yes, hi);
        }
        return lo;
    }
    // Of a number in `bin` or above it, sought around where the bin ends but for rounding.
    __device__ uint32_t lowest_of(int bin) const
    {
        auto accepts = [&](float z) { return depth_bin(z) <= bin; };
        const float end = top32 - (float)(bin + 1) / scale, about = 1e-6f * (fabsf(top32) + fabsf(end));
        const uint32_t lo = max(key_of(end - about), LOWEST_FINITE), hi = min(key_of(end + about), key_of(top32));
        const bool inside = lo < hi && !accepts(float_of(lo)) && accepts(float_of(hi));
        return lowest_key(inside ? lo + 1 : LOWEST_FINITE, inside ? hi : key_of(top32), accepts);
    }
    // UNIT times what z's weight falls short of the top of its depth bin, rounded, and SLACK, above 2^52: the low bits are the integer.  By the
    // series of exp(x) - 1 (x lies in -STEP .. 1e-5 but for rounding; the term left out is below 1e-17, in wider bins below 3e-15).
    __device__ __forceinline__ double rest_of(float z, int bin) const
    {
        const double depth = __hiloint2double(0x43300000, bin) - 4503599627370496.0;
        const double x = fma(depth, STEP, ((double)z - top) * per_nat);
        double w = fma(x, 1.0 / 5040.0, 1.0 / 720.0);
        w = fma(x, w, 1.0 / 120.0);
        w = fma(x, w, 1.0 / 24.0);
        w = fma(x, w, 1.0 / 6.0);
        w = fma(x, w, 0.5);
        w = fma(x, w, 1.0);
        return fma(x * w, -UNIT, 4503599627370496.0 + SLACK * UNIT);
    }
    // z's weight as the masses are added up from it; top_weight: that of the bin's top
    __device__ __forceinline__ double weight_in(float z, int bin, double top_weight) const
    {
        return (1.0 - (rest_of(z, bin) - (4503599627370496.0 + SLACK * UNIT)) * (1.0 / UNIT)) * top_weight;
    }
    // One more element.
    template <int N> __device__ __forceinline__ void add(BinCounts<N> &to, int item, float z, int bin)
    {
        if (!PPOW_CHECK(item >= 0 && item < N, 801, nullptr)) return;
        const double w = rest_of(z, bin);
        const uint32_t lo = (uint32_t)__double2loint(w), hi = (uint32_t)__double2hiint(w) & 0xfffffu;
        static_assert(LIMBS == 3 && LIMB_BITS == 13, "limbs");
        atomicAdd(&to.count[item], 1u);
        atomicAdd(&to.limb[0][item], lo & 0x1fffu);
        atomicAdd(&to.limb[1][item], lo >> 13 & 0x1fffu);
        atomicAdd(&to.limb[2][item], lo >> 26 | hi << 6);
    }
    template <int N> __device__ void clear(BinCounts<N> &counts)
    {
        for (int i = threadIdx.x; i < (1 + LIMBS) * N; i += THREADS) counts.count[i] = 0;        // the limbs lie behind
        __syncthreads();
    }
    // Sums up the CTAs' bins, each CTA a share of them for all, and the groups.  top_weight(item): that of the bin's top.
    template <int N, typename TopWeight> __device__ void join(BinCounts<N> &counts, BinTotals<N> &totals, TopWeight &&top_weight)
    {
        meet(cluster, ctas);
        for (int i = rank * THREADS + (int)threadIdx.x; i < N; i += ctas * THREADS) {
            uint32_t count = 0;
            unsigned long long limbs[LIMBS] = {};
            for (int r = 0; r < ctas; ++r) {
                const BinCounts<N> *b = of(&counts, r);
                count += b->count[i];
#pragma unroll
                for (int l = 0; l < LIMBS; ++l) limbs[l] += b->limb[l][i];
            }
            long long rest = -(long long)count * (long long)(SLACK * UNIT);
#pragma unroll
            for (int l = 0; l < LIMBS; ++l) rest += (long long)(limbs[l] << (l * LIMB_BITS));
            const double m = count ? ((double)count - (double)rest * (1.0 / UNIT)) * top_weight(i) : 0.0;
            for (int r = 0; r < ctas; ++r) {
                BinTotals<N> *t = of(&totals, r);
                t->count[i] = count;
                t->mass[i] = m;
            }
        }
        meet(cluster, ctas);
    }
    // The groups' sums, from `first` on in sh.
    template <int N> __device__ void sum_bins(const BinTotals<N> &totals, int first)
    {
        for (int c = threadIdx.x >> 5; c < N / SEARCH_GROUP; c += THREADS / 32) {
            const int i = c * SEARCH_GROUP + (threadIdx.x & 31);
            const uint32_t count = __reduce_add_sync(0xffffffffu, totals.count[i]);
            const double mass = warp_sum_f64(totals.mass[i]);
            if ((threadIdx.x & 31) == 0) sh.group_count[first + c] = count, sh.group_mass[first + c] = mass;
        }
        __syncthreads();
    }
    // The bin that holds the border; all threads have the result.
    template <int N> __device__ Place find_bin(const BinTotals<N> &totals, int first, const Target &target, const Place &before)
    {
        constexpr int GROUPS = N / SEARCH_GROUP, PER = (GROUPS + 31) / 32;
        if (threadIdx.x < 32) {
            const Scan<PER> groups(GROUPS, before, [&](int i) { return Part{sh.group_count[first + i], sh.group_mass[first + i]}; });
            Place p = groups.find(target);
            if (!PPOW_CHECK(p.item < GROUPS, 804, nullptr)) p.item = 0;
            const int start = p.item * SEARCH_GROUP;
            const Scan<1> in_group(SEARCH_GROUP, p, [&](int i) { return Part{totals.count[start + i], totals.mass[start + i]}; });
            p = in_group.find(target);
            p.item += start;
            if (threadIdx.x == 0) sh.place = p;
        }
        __syncthreads();
        const Place p = sh.place;
        __syncthreads();
        return p;
    }
    // Lists the piece's elements with keys in lo .. hi, Bins::LIST at most.
    __device__ void make_list(uint32_t lo, uint32_t hi)
    {
        if (threadIdx.x == 0) sh.listed = 0;
        __syncthreads();
        const float low = float_of(lo), high = float_of(hi);
        each([&](float z, int32_t token) {
            if (!(z >= low && z <= high)) return;
            const uint32_t at = atomicAdd(&sh.listed, 1u);
            // they were counted, but in another reading: a row that changes meanwhile must not write past the list
            if (PPOW_CHECK(at < Bins::LIST, 803, nullptr) && at < Bins::LIST) bins.list[at] = (unsigned long long)key_of(z) << 32 | (uint32_t)token;
        });
        __syncthreads();
        listed = min((int)sh.listed, (int)Bins::LIST);
    }
    // The element on the border; the whole CTA, and the whole cluster in step.  The list, if there is one, is left.
    __device__ Element find(const Target &target, bool whole)
    {
        if (!whole) listed = -1;
        Place p = find_bin(bins.depths, 0, target, Place{0, 0, 0.0});
        const int bin = p.item;
        const bool massless = bin == BINS - 1;
        const double top_weight = massless ? 0.0 : exp(-bin * STEP);
        uint32_t lo = lowest_of(bin), hi = bin == 0 ? key_of(top32) : lowest_of(bin - 1) - 1;
        if (!whole && bins.depths.count[bin] <= Bins::LIST) make_list(lo, hi);
        for (;;) {
            int shift = 0;
            while (((hi - lo) >> shift) >= SUB) ++shift;
            clear(bins.sub);
            each([&](float z, int32_t) {
                const uint32_t k = key_of(z);
                if (k < lo || k > hi) return;
                const int item = (int)((hi - k) >> shift);
                if (!massless)
                    add(bins.sub, item, z, bin);
                else if (PPOW_CHECK(item < SUB, 802, nullptr))
                    atomicAdd(&bins.sub.count[item], 1u);
            });
            join(bins.sub, bins.subs, [&](int) { return top_weight; });
            sum_bins(bins.subs, BINS / SEARCH_GROUP);
            p = find_bin(bins.subs, BINS / SEARCH_GROUP, target, p);
            hi -= (uint32_t)p.item << shift;
            const uint32_t width = (1u << shift) - 1;
            lo = hi - lo > width ? hi - width : lo;
            if (shift == 0 || bins.subs.count[p.item] == 1) break;
        }
        const uint32_t have = bins.subs.count[p.item];
        if (lo < hi) {                       // one element: which?
            meet(cluster, ctas);
            each([&](float z, int32_t token) {
                const uint32_t k = key_of(z);
                if (k < lo || k > hi) return;
                for (int r = 0; r < ctas; ++r) of(&sh, r)->only_key = k, of(&sh, r)->only_token = token;
            });
            meet(cluster, ctas);
            const float value = float_of(sh.only_key);
            return {value, p.count + 1, p.mass + (massless ? 0.0 : weight_in(value, bin, top_weight)), sh.only_token, 0, 1};
        }
        const float value = float_of(hi);
        if (massless && !target.by_count()) return {value, p.count + 1, p.mass, -1, 0, have};
        // the weight that the masses were added up from: a border on a multiple of it stays there
        return choose(target, p, value, have, massless ? 0.0 : weight_in(value, bin, top_weight));
    }
    __device__ void run(int64_t row)
    {
        const bool lead = rank == 0 && threadIdx.x == 0;
        if (threadIdx.x == 0) sh.top = sh.none = sh.flags = sh.within = 0;
        if (lead) job.tokens[row] = -1;      // never left unwritten, even if the row changes between its readings
        meet(cluster, ctas);
        float most = -INFINITY;
        uint32_t none = 0, bad = 0;
        each([&](float z, int32_t) {
            bad |= !(z < INFINITY);
            none += z == -INFINITY;
            most = fmaxf(most, z);
        });
        const uint32_t key = __reduce_max_sync(0xffffffffu, key_of(most));
        none = __reduce_add_sync(0xffffffffu, none), bad = __reduce_or_sync(0xffffffffu, bad);
        if ((threadIdx.x & 31) == 0)
            for (int r = 0; r < ctas; ++r) {
                SampleShared *s = of(&sh, r);
                atomicMax(&s->top, key);
                atomicAdd(&s->none, none);
                if (bad) atomicOr(&s->flags, (uint32_t)SAMPLE_BAD);
            }
        meet(cluster, ctas);
        const uint32_t F = (uint32_t)piece.units * E - sh.none;
        if (sh.flags & SAMPLE_BAD || F == 0) {
            if (lead) {
                job.logp[row] = F == 0 && !(sh.flags & SAMPLE_BAD) ? -INFINITY : NAN;
                if (job.kept) job.kept[row] = 0;
            }
            return;
        }
        top32 = float_of(sh.top);
        top = (double)top32;
        per_nat = 1.0 / job.temperature;
        scale = (float)((BINS - 1) / (SEARCH_NATS * job.temperature));
        uint32_t floor_key = LOWEST_FINITE;  // of the lowest number within min_p
        if (job.min_p > 0.0) floor_key = lowest_key(LOWEST_FINITE, sh.top, [&](float z) { return weight(z) >= job.min_p; });
        const float floor = float_of(floor_key);
        clear(bins.depth);
        uint32_t within = 0;
        each([&](float z, int32_t) {
            if (z == -INFINITY) return;
            within += z >= floor;
            const int b = depth_bin(z);
            if (b < BINS - 1)
                add(bins.depth, b, z, b);
            else
                atomicAdd(&bins.depth.count[b], 1u);         // too deep for any mass
        });
        within = __reduce_add_sync(0xffffffffu, within);
        if ((threadIdx.x & 31) == 0)
            for (int r = 0; r < ctas; ++r) atomicAdd(&of(&sh, r)->within, within);
        join(bins.depth, bins.depths, [&](int i) { return i < BINS - 1 ? exp(-i * STEP) : 0.0; });
        const bool whole = F <= Bins::LIST;  // then the list holds the row once and for all
        if (whole) make_list(LOWEST_FINITE, sh.top);
        sum_bins(bins.depths, 0);
        double all = 0.0;
        for (int i = threadIdx.x & 31; i < BINS / SEARCH_GROUP; i += 32) all += sh.group_mass[i];
        all = warp_sum_f64(all);
        Element drawn;
        uint32_t n;
        double total;
        decide(job, job.uniforms[row], F, F - bins.depths.count[BINS - 1], all, sh.within, [&](const Target &t) { return find(t, whole); }, drawn, n,
               total);
        if (lead) {
            job.logp[row] = (float)(((double)drawn.value - top) * per_nat - log(total));
            if (job.kept) job.kept[row] = (int32_t)n;
            if (drawn.token >= 0) job.tokens[row] = drawn.token;
        }
        if (drawn.token >= 0) return;
        // one of several equal ones: which piece holds it, and where
        const uint32_t drawn_key = key_of(drawn.value);
        uint32_t skip = 0, have = drawn.have;
        if (ctas > 1) {
            if (threadIdx.x == 0) sh.here = 0;
            __syncthreads();
            uint32_t mine = 0;
            each([&](float z, int32_t) { mine += key_of(z) == drawn_key; });
            mine = __reduce_add_sync(0xffffffffu, mine);
            if ((threadIdx.x & 31) == 0 && mine) atomicAdd(&sh.here, mine);
            cluster.sync();
            for (int r = 0; r < rank; ++r) skip += of(&sh, r)->here;
            have = sh.here;
        }
        if (drawn.rank < skip || drawn.rank - skip >= have) return;
        if (listed < 0) {
            locate<THREADS>(piece, have - 1 - (drawn.rank - skip), sh, job.tokens + row, HasKey<DTYPE>{drawn_key});
            return;
        }
        each([&](float z, int32_t token) {
            if (key_of(z) != drawn_key) return;
            uint32_t before = 0;
            for (int i = 0; i < listed; ++i) before += (uint32_t)(bins.list[i] >> 32) == drawn_key && (int32_t)(uint32_t)bins.list[i] < token;
            if (before == drawn.rank - skip) job.tokens[row] = token;
        });
    }
};

template <int DTYPE, int THREADS, int BINS>
__device__ __forceinline__ void search_row(const SampleJob &job, int64_t row, int rank, int ctas, SampleShared &sh, void *smem)
{
    const Piece<DTYPE> piece(job, row, rank, ctas);
    const cg::cluster_group cluster = cg::this_cluster();
    Search<DTYPE, THREADS, BINS> s{job, piece, cluster, rank, ctas, sh, *static_cast<SearchBins<BINS> *>(smem), 0.0, 0.0, 0.0f, 0.0f, -1};
    s.run(row);
}

template <int THREADS>
__global__ void __launch_bounds__(THREADS, 1024 / THREADS) sample_search_kernel(const SampleJob job)
{
    wait_for_previous_kernel();
    extern __shared__ uint4 sample_smem[];
    __shared__ SampleShared sh;
    const cg::cluster_group cluster = cg::this_cluster();
    const int ctas = (int)cluster.num_blocks(), rank = (int)cluster.block_rank();
    search_row<PPOW_F32, THREADS, SEARCH_BINS>(job, blockIdx.x / ctas, rank, ctas, sh, sample_smem);
    if (ctas > 1) cluster.sync();            // no CTA leaves while another still reads its shared memory
}

// ---- sorting: short float32 rows --------------------------------------------------------------------
// A row of up to SORT_THREADS * PER logits, sorted in registers: thread t holds the elements PER t .. of the order.  An entry is key << 32 | ~index,
// so that descending entries are descending numbers, equal ones by index; 0 is none.  Exchanges within PER places stay in a thread, within
// 32 PER in a warp, and only the rest goes through shared memory (256 x 1000: 21 us by a search, 10 us so).
constexpr int SORT_THREADS = 256, SORT_WARPS = SORT_THREADS / 32;

template <int PER> __device__ __forceinline__ void sort_entries(unsigned long long (&v)[PER], unsigned long long *exchange)
{
    const int t = threadIdx.x;
#pragma unroll 1
    for (int k = 2; k <= SORT_THREADS * PER; k <<= 1) {
#pragma unroll 1
        for (int j = k >> 1; j >= PER; j >>= 1) {            // with the thread j / PER away, element by element
            const int other = j / PER;
            unsigned long long p[PER];
            if (other < 32) {
#pragma unroll
                for (int e = 0; e < PER; ++e) p[e] = __shfl_xor_sync(0xffffffffu, v[e], other);
            } else {
                __syncthreads();
#pragma unroll
                for (int e = 0; e < PER; ++e) exchange[e * SORT_THREADS + t] = v[e];
                __syncthreads();
#pragma unroll
                for (int e = 0; e < PER; ++e) p[e] = exchange[e * SORT_THREADS + (t ^ other)];
            }
            const bool larger = ((t * PER & k) == 0) == ((t & other) == 0);      // which of the two stays here
#pragma unroll
            for (int e = 0; e < PER; ++e) v[e] = (v[e] > p[e]) == larger ? v[e] : p[e];
        }
#pragma unroll
        for (int j = PER / 2; j > 0; j >>= 1) {
            if (j >= k) continue;
#pragma unroll
            for (int e = 0; e < PER; ++e)
                if ((e & j) == 0) {
                    const bool down = k >= PER ? (t * PER & k) == 0 : (e & k) == 0;
                    const unsigned long long a = v[e], b = v[e | j];
                    const bool swap = (a < b) == down;
                    v[e] = swap ? b : a;
                    v[e | j] = swap ? a : b;
                }
        }
    }
}

template <int PER> __global__ void __launch_bounds__(SORT_THREADS) sample_sort_kernel(const SampleJob job)
{
    __shared__ unsigned long long exchange[SORT_THREADS * PER];
    __shared__ double warp_mass[SORT_WARPS], at_mass;
    __shared__ uint32_t sums[5][SORT_WARPS];
    wait_for_previous_kernel();
    const int64_t row = blockIdx.x;
    const int t = threadIdx.x, lane = t & 31, warp = t >> 5;
    const float *logits = static_cast<const float *>(job.logits) + row * job.stride;
    unsigned long long v[PER];
    bool bad = false;
#pragma unroll
    for (int e = 0; e < PER; ++e) {
        const int i = t + e * SORT_THREADS;
        const float z = i < job.V ? __ldcs(logits + i) : -INFINITY;
        bad |= !(z < INFINITY);
        v[e] = z > -INFINITY ? (unsigned long long)key_of(z) << 32 | (uint32_t)~i : 0ull;
    }
    sort_entries<PER>(v, exchange);
    bad = __syncthreads_or(bad);
    // a sum over the CTA, `turn` once each
    auto sum = [&](int turn, uint32_t n) {
        n = __reduce_add_sync(0xffffffffu, n);
        if (lane == 0) sums[turn][warp] = n;
        __syncthreads();
        n = 0;
#pragma unroll
        for (int i = 0; i < SORT_WARPS; ++i) n += sums[turn][i];
        return n;
    };
    uint32_t some = 0;
#pragma unroll
    for (int e = 0; e < PER; ++e) some += v[e] != 0;
    if (t == 0) exchange[0] = v[0];
    const uint32_t F = sum(0, some);
    if (bad || F == 0) {
        if (t == 0) {
            job.tokens[row] = -1;
            job.logp[row] = bad ? NAN : -INFINITY;
            if (job.kept) job.kept[row] = 0;
        }
        return;
    }
    const double per_nat = 1.0 / job.temperature, top = (double)float_of((uint32_t)(exchange[0] >> 32));
    double w[PER], mass[PER], upto = 0.0;                    // weights; the mass up to and with each
#pragma unroll
    for (int e = 0; e < PER; ++e) w[e] = v[e] ? exp(((double)float_of((uint32_t)(v[e] >> 32)) - top) * per_nat) : 0.0;
#pragma unroll
    for (int e = 0; e < PER; ++e) mass[e] = upto += w[e];
#pragma unroll
    for (int o = 1; o < 32; o <<= 1) {
        const double m = __shfl_up_sync(0xffffffffu, upto, o);
        if (lane >= o) upto += m;
    }
    if (lane == 31) warp_mass[warp] = upto;
    upto = __shfl_up_sync(0xffffffffu, upto, 1);
    if (lane == 0) upto = 0.0;
    __syncthreads();
    double before = 0.0;
    for (int i = 0; i < warp; ++i) before += warp_mass[i];
#pragma unroll
    for (int e = 0; e < PER; ++e) mass[e] += before + upto;
    auto mass_at = [&](uint32_t n) {         // of the first n
        __syncthreads();
#pragma unroll
        for (int e = 0; e < PER; ++e)
            if (t * PER + e + 1 == n) at_mass = mass[e];
        __syncthreads();
        return at_mass;
    };
    uint32_t n = job.top_k > 0 && (uint32_t)job.top_k < F ? (uint32_t)job.top_k : F;
    double total = mass_at(n);
    if (job.top_p < 1.0) {
        uint32_t below = 0;
#pragma unroll
        for (int e = 0; e < PER; ++e) below += t * PER + e < n && mass[e] < job.top_p * total;
        n = min(sum(1, below) + 1, n);
    }
    if (job.min_p > 0.0) {
        uint32_t within = 0;
#pragma unroll
        for (int e = 0; e < PER; ++e) within += t * PER + e < F && w[e] >= job.min_p;
        n = min(sum(2, within), n);
    }
    if (job.top_p < 1.0 || job.min_p > 0.0) total = mass_at(n);
    const double at = (double)fminf(fmaxf(job.uniforms[row], 0.0f), 0x1.fffffep-1f) * total;        // NaN is 0
    uint32_t passed = 0;
#pragma unroll
    for (int e = 0; e < PER; ++e) passed += t * PER + e < n && mass[e] <= at;
    const uint32_t drawn = min(sum(3, passed), n - 1);
#pragma unroll
    for (int e = 0; e < PER; ++e)
        if (t * PER + e == drawn) {
            job.tokens[row] = (int32_t)~(uint32_t)v[e];
            job.logp[row] = (float)(((double)float_of((uint32_t)(v[e] >> 32)) - top) * per_nat - log(total));
            if (job.kept) job.kept[row] = (int32_t)n;
        }
}

// ---- counting: 16-bit rows --------------------------------------------------------------------------
template <int DTYPE> struct Count {
    using F = Counted<DTYPE>;
    static constexpr uint32_t NEG_INF = 0x8000u | F::INF;
    static constexpr bool ZEROS = F::LOW > 0;                // counted apart
    char *words;
    uint32_t none = 0, low = 0, zeros = 0, flags = 0, most = NEG_INF * 0x10001u;

    // 1 in the low half for a positive number, in the high half for a negative one: copies of the sign in two bytes, and 1.
    template <int SELECT> static __device__ __forceinline__ uint32_t one(uint32_t w)
    {
        uint32_t signs;
        asm("prmt.b32 %0, %1, 0, %2;" : "=r"(signs) : "r"(w), "n"(SELECT));
        return signs + 1u;
    }
    __device__ __forceinline__ void low_half(uint32_t w) { atomicAdd(reinterpret_cast<uint32_t *>(words + (w << 2 & F::MASK << 2)), one<0x4499>(w)); }
    __device__ __forceinline__ void high_half(uint32_t w) { atomicAdd(reinterpret_cast<uint32_t *>(words + (w >> 14 & F::MASK << 2)), one<0x44bb>(w)); }
    // Not zero in the halves that are beyond the counted range.  Nothing goes from one half to the other: above its magnitude a half has a 1,
    // which the difference with LOW leaves (its bits past WORDS are those of a borrow, or of what is too large), and a sum with
    // 2^15 - WORDS reaches 2^15 and stays below 2^16.
    static __device__ __forceinline__ uint32_t beyond(uint32_t w)
    {
        if constexpr (F::LOW > 0)
            return (((w | 0x80008000u) - F::LOW * 0x10001u) ^ 0x80008000u) & (0xffffu - F::MASK) * 0x10001u;
        else
            return ((w & 0x7fff7fffu) + (0x8000u - F::WORDS) * 0x10001u) & 0x80008000u;
    }

    // Eight logits; the whole warp calls.   Bound by the integer units (4 operations a logit) and the additions in shared memory: nothing
    // is looked at one by one where all are in range, or in range and -inf (one way for the warp: both would cost the sum).
    __device__ __forceinline__ void add(const uint4 &w)
    {
        most = F::most(most, F::most(F::most(w.x, w.y), F::most(w.z, w.w)));
        const uint32_t words[4] = {w.x, w.y, w.z, w.w};
        uint32_t out[4];
#pragma unroll
        for (int i = 0; i < 4; ++i) out[i] = beyond(words[i]);
        if (!__any_sync(0xffffffffu, out[0] | out[1] | out[2] | out[3])) {
#pragma unroll
            for (int i = 0; i < 4; ++i) low_half(words[i]), high_half(words[i]);
            return;
        }
        uint32_t odd = 0, count = 0;
#pragma unroll
        for (int i = 0; i < 4; ++i) {
            const uint32_t masked = F::equal(words[i], NEG_INF * 0x10001u);
            odd |= out[i] & ~masked;
            count += masked & 0x10001u;
            if (!(out[i] & 0xffffu)) low_half(words[i]);
            if (!(out[i] >> 16)) high_half(words[i]);
        }
        none += (count & 0xffffu) + (count >> 16);
        if (odd) {
#pragma unroll
            for (int i = 0; i < 4; ++i) {
                beyond_one(words[i] & 0xffffu, !(out[i] & 0xffffu));
                beyond_one(words[i] >> 16, !(out[i] >> 16));
            }
        }
    }
    // What has not been counted; -inf was counted already.
    __device__ __forceinline__ void beyond_one(uint32_t bits, bool counted)
    {
        const uint32_t magnitude = bits & 0x7fffu;
        if (counted || bits == NEG_INF) return;
        if (magnitude == 0)
            ++zeros;
        else if (magnitude >= F::INF)
            flags |= SAMPLE_BAD;
        else if (bits & 0x8000u && magnitude >= F::LOW + F::WORDS)
            ++low;
        else
            flags |= SAMPLE_ODD;
    }
};

// Weights of the four numbers of a group from `first` on, by rising magnitude.  A group lies within one power of two, so they are a step apart: one
// exp for the largest and one for the step, unless the step is more than a nat.  That of the maximum is 1.
template <int DTYPE> __device__ __forceinline__ void weights_of(int group, int first, double top, double per_nat, double (&w)[4])
{
    using G = Groups<DTYPE>;
    const double z0 = (double)G::number(group, first), z3 = (double)G::number(group, first + 3), step = fabs(z3 - z0) * (1.0 / 3.0) * per_nat;
    if (step > 1.0) {
#pragma unroll
        for (int i = 0; i < 4; ++i) w[i] = exp(((double)G::number(group, first + i) - top) * per_nat);
        return;
    }
    const double r = exp(-step), e = exp((fmax(z0, z3) - top) * per_nat), r2 = r * r;
    const double down[4] = {e, e * r, e * r2, e * (r2 * r)};
#pragma unroll
    for (int i = 0; i < 4; ++i) w[i] = (double)G::number(group, first + i) == top ? 1.0 : G::negative(group) ? down[i] : down[3 - i];
}

// The groups' counts and masses: each CTA adds up a share of the groups for all, in its own words (the others read none of those).
template <int DTYPE>
__device__ __forceinline__ void sum_groups(const SampleJob &job, int rank, int ctas, SampleShared &sh, uint4 *words)
{
    using F = Counted<DTYPE>;
    using G = Groups<DTYPE>;
    constexpr int THREADS = F::THREADS;
    const cg::cluster_group cluster = cg::this_cluster();
    const int lane = threadIdx.x & 31, warp = threadIdx.x >> 5;
    auto of = [&](auto *p, int r) { return ctas == 1 ? p : cluster.map_shared_rank(p, r); };
    const double per_nat = 1.0 / job.temperature, top = (double)float_of(sh.top);
    const int from = G::SIDE / ctas * rank, to = G::SIDE / ctas * (rank + 1);
    uint32_t over = 0, within = 0;
    for (int g = from + warp; g < to; g += THREADS / 32) {
        const int at = G::word(g) / 4 + lane;
        const uint4 own = words[at];
        if (ctas == 1 && !__any_sync(0xffffffffu, own.x | own.y | own.z | own.w)) continue;
        uint32_t b[2][4] = {{own.x & 0xffffu, own.y & 0xffffu, own.z & 0xffffu, own.w & 0xffffu}, {own.x >> 16, own.y >> 16, own.z >> 16, own.w >> 16}};
        uint4 others[SAMPLE_CTAS];       // all on their way at once
#pragma unroll
        for (int r = 1; r < SAMPLE_CTAS; ++r)
            if (r < ctas) others[r] = cluster.map_shared_rank(words, rank + r < ctas ? rank + r : rank + r - ctas)[at];
#pragma unroll
        for (int r = 1; r < SAMPLE_CTAS; ++r) {
            if (r >= ctas) break;
            const uint4 o = others[r];
            b[0][0] += o.x & 0xffffu, b[0][1] += o.y & 0xffffu, b[0][2] += o.z & 0xffffu, b[0][3] += o.w & 0xffffu;
            b[1][0] += o.x >> 16, b[1][1] += o.y >> 16, b[1][2] += o.z >> 16, b[1][3] += o.w >> 16;
        }
        if (!Count<DTYPE>::ZEROS && at == 0) b[0][0] += b[1][0], b[1][0] = 0;        // -0 is +0
        if (ctas > 1 || (!Count<DTYPE>::ZEROS && g == 0)) {
            words[at] = make_uint4(b[0][0] | b[1][0] << 16, b[0][1] | b[1][1] << 16, b[0][2] | b[1][2] << 16, b[0][3] | b[1][3] << 16);
            over |= b[0][0] | b[0][1] | b[0][2] | b[0][3] | b[1][0] | b[1][1] | b[1][2] | b[1][3];
        }
#pragma unroll
        for (int side = 0; side < 2; ++side) {
            const uint32_t have = b[side][0] + b[side][1] + b[side][2] + b[side][3];
            if (!__any_sync(0xffffffffu, have != 0)) continue;
            const int group = side ? G::ZERO + 1 + g : g;
            double mass = 0.0, weights[4];
            weights_of<DTYPE>(group, lane * 4, top, per_nat, weights);
#pragma unroll
            for (int i = 0; i < 4; ++i) {
                mass += b[side][i] ? b[side][i] * weights[i] : 0.0;      // beyond the maximum a weight may overflow, with nothing to count
                within += weights[i] >= job.min_p ? b[side][i] : 0u;
            }
            mass = warp_sum_f64(mass);
            const uint32_t counted = __reduce_add_sync(0xffffffffu, have);
            for (int r = lane; r < ctas; r += 32) {
                SampleShared *s = of(&sh, r);
                s->group_count[group] = counted;
                s->group_mass[group] = mass;
            }
        }
    }
    if (Count<DTYPE>::ZEROS && threadIdx.x == 0 && sh.zeros > 0) {       // every CTA for itself
        const double e = exp(-top * per_nat);
        sh.group_count[G::ZERO] = sh.zeros;
        sh.group_mass[G::ZERO] = sh.zeros * e;
        if (rank == 0 && e >= job.min_p) within += sh.zeros;
    }
    within = __reduce_add_sync(0xffffffffu, within);
    over = __reduce_or_sync(0xffffffffu, over) >> 16;
    if (lane == 0)
        for (int r = 0; r < ctas; ++r) {
            if (within) atomicAdd(&of(&sh, r)->within, within);
            if (over) atomicOr(&of(&sh, r)->flags, (uint32_t)SAMPLE_ODD);
        }
}

// What is kept of a row, and the draw, from the groups' counts and masses; sh.drawn.n is 0 where there is none (rank: the flags). One warp.
template <int DTYPE>
__device__ __forceinline__ void decide_counted(const SampleJob &job, int64_t row, float uniform, uint32_t logits, int rank, int ctas, SampleShared &sh, const uint4 *own)
{
    using F = Counted<DTYPE>;
    using G = Groups<DTYPE>;
    const cg::cluster_group cluster = cg::this_cluster();
    const int lane = threadIdx.x & 31;
    const double per_nat = 1.0 / job.temperature, top = (double)float_of(sh.top);
    constexpr int PER = (G::ALL + 31) / 32;
    const Scan<PER> groups(G::ALL, Place{0, 0, 0.0}, [&](int i) { return Part{sh.group_count[G::at(i)], sh.group_mass[G::at(i)]}; });
    const Part all = groups.all();
    uint32_t flags = sh.flags;
    const uint32_t low = sh.low;
    // a count that ran over left a sum that is short; numbers below the counted range have to be too deep for any mass
    if (all.count + sh.none + low != logits) flags |= SAMPLE_ODD;
    if (low > 0) {
        const double deep = (top + F::LIMIT) * per_nat;
        if (all.count == 0 || deep < SEARCH_NATS || (job.min_p > 0.0 && exp(-deep) >= job.min_p)) flags |= SAMPLE_ODD;
    }
    if (flags || all.count == 0) {
        if (lane == 0) {
            if (rank == 0 && (flags & SAMPLE_BAD || flags == 0)) {
                job.logp[row] = flags ? NAN : -INFINITY;
                if (job.kept) job.kept[row] = 0;
            }
            sh.drawn.n = 0;
            sh.drawn.rank = flags;
        }
        return;
    }
    auto find = [&](const Target &target) {
        Place p = groups.find(target);
        if (!PPOW_CHECK(p.item < G::ALL, 805, nullptr)) p.item = 0;
        const int group = G::at(p.item);
        if (group == G::ZERO) return choose(target, p, 0.0f, sh.zeros, exp(-top * per_nat));
        // four words a lane, of the group's numbers in descending order, from the CTA that added this group up
        const bool negative = G::negative(group);
        const int owner = G::side(group) / (G::SIDE / ctas), at = G::word(G::side(group)) / 4 + (negative ? lane : 31 - lane);
        const uint4 words = ctas == 1 ? own[at] : cluster.map_shared_rank(own, owner)[at];
        const uint32_t half = negative ? 16 : 0;
        const uint32_t have[4] = {(negative ? words.x : words.w) >> half & 0xffffu, (negative ? words.y : words.z) >> half & 0xffffu,
                                  (negative ? words.z : words.y) >> half & 0xffffu, (negative ? words.w : words.x) >> half & 0xffffu};
        auto number = [&](int i) { return G::number(group, negative ? i : GROUP - 1 - i); };
        double rising[4];
        weights_of<DTYPE>(group, negative ? lane * 4 : GROUP - 4 - lane * 4, top, per_nat, rising);
        const double falling[4] = {negative ? rising[0] : rising[3], negative ? rising[1] : rising[2], negative ? rising[2] : rising[1],
                                   negative ? rising[3] : rising[0]};
        const Scan<GROUP / 32> numbers(GROUP, p, [&](int i) {
            const uint32_t c = have[i % 4];
            return Part{c, c ? c * falling[i % 4] : 0.0};      // beyond the maximum a weight may overflow
        });
        p = numbers.find(target);
        const int at_lane = p.item / 4, slot = p.item % 4;
        const uint32_t mine = slot == 0 ? have[0] : slot == 1 ? have[1] : slot == 2 ? have[2] : have[3];
        const double weight = slot == 0 ? falling[0] : slot == 1 ? falling[1] : slot == 2 ? falling[2] : falling[3];
        // the weight that the masses were added up from: a border on a multiple of it stays there
        return choose(target, p, number(p.item), __shfl_sync(0xffffffffu, mine, at_lane), __shfl_sync(0xffffffffu, weight, at_lane));
    };
    Element drawn;
    uint32_t n;
    double total;
    decide(job, uniform, all.count + low, all.count, all.mass, sh.within, find, drawn, n, total);
    if (lane == 0) {
        if (rank == 0) {
            job.logp[row] = (float)(((double)drawn.value - top) * per_nat - log(total));
            if (job.kept) job.kept[row] = (int32_t)n;
        }
        sh.drawn = drawn;
    }
}

// A row that counting does not fit, in the same shared memory with half the bins.  Rare, and out of line: registers are the others'.
template <int DTYPE, int THREADS>
__device__ __noinline__ void search_odd_row(const SampleJob &job, int64_t row, int rank, int ctas, SampleShared &sh, void *smem)
{
    static_assert(sizeof(SearchBins<1024>) <= Counted<DTYPE>::WORDS * 4, "room for a search");
    search_row<DTYPE, THREADS, 1024>(job, row, rank, ctas, sh, smem);
}

template <int DTYPE>
__global__ void __launch_bounds__(Counted<DTYPE>::THREADS, Counted<DTYPE>::CTAS) sample_count_kernel(const SampleJob job)
{
    using F = Counted<DTYPE>;
    constexpr int THREADS = F::THREADS;
    using G = Groups<DTYPE>;
    extern __shared__ uint4 sample_smem[];
    __shared__ SampleShared sh;
    wait_for_previous_kernel();
    const cg::cluster_group cluster = cg::this_cluster();
    const int ctas = (int)cluster.num_blocks(), rank = (int)cluster.block_rank();
    const int lane = threadIdx.x & 31, warp = threadIdx.x >> 5;
    const int64_t row = blockIdx.x / ctas;
    const Piece<DTYPE> piece(job, row, rank, ctas);
    const float uniform = job.uniforms[row];                 // on its way early
    auto of = [&](auto *p, int r) { return ctas == 1 ? p : cluster.map_shared_rank(p, r); };
    constexpr int DEEP = 2;
    uint4 w[DEEP];
    auto fetch = [&](int32_t u0) {           // behind the piece's end, -inf
#pragma unroll
        for (int q = 0; q < DEEP; ++q) {
            constexpr uint32_t BEHIND = Count<DTYPE>::NEG_INF * 0x10001u;
            w[q] = make_uint4(BEHIND, BEHIND, BEHIND, BEHIND);
            if (u0 + q * THREADS < piece.end) w[q] = piece.load(u0 + q * THREADS);
        }
    };
    fetch(piece.begin + (int32_t)threadIdx.x);
    for (int i = threadIdx.x; i < (int)F::WORDS / 4; i += THREADS) sample_smem[i] = make_uint4(0, 0, 0, 0);
    for (int i = threadIdx.x; i < G::ALL; i += THREADS) sh.group_count[i] = 0, sh.group_mass[i] = 0.0;
    if (threadIdx.x == 0) sh.none = sh.low = sh.zeros = sh.flags = sh.within = sh.top = 0;
    if (rank == 0 && threadIdx.x == 0) job.tokens[row] = -1;     // never left unwritten, even if the row changes between its two readings
    meet(cluster, ctas);                     // the others write into these
    {
        Count<DTYPE> count{reinterpret_cast<char *>(sample_smem)};
        for (int32_t u0 = piece.begin + (int32_t)threadIdx.x; u0 - lane < piece.end; u0 += THREADS * DEEP) {
            uint4 now[DEEP];
#pragma unroll
            for (int q = 0; q < DEEP; ++q) now[q] = w[q];
            fetch(u0 + THREADS * DEEP);
#pragma unroll
            for (int q = 0; q < DEEP; ++q)
                if (u0 - lane + q * THREADS < piece.end) count.add(now[q]);
        }
        // without what fetch() put behind the piece
        const int32_t length = piece.end - piece.begin, behind = (32 - length % 32) % 32;
        const bool last = warp == (int)((uint32_t)(length / 32) % (THREADS / 32));       // the warp whose units the end divides
        const uint32_t none = __reduce_add_sync(0xffffffffu, count.none) - (last ? behind * 8u : 0u), low = __reduce_add_sync(0xffffffffu, count.low),
                       zeros = __reduce_add_sync(0xffffffffu, count.zeros), flags = __reduce_or_sync(0xffffffffu, count.flags);
        const uint32_t top = __reduce_max_sync(0xffffffffu, max(key_of(Storage<DTYPE>::get((uint16_t)count.most)),
                                                                key_of(Storage<DTYPE>::get((uint16_t)(count.most >> 16)))));
        if (lane == 0)
            for (int r = 0; r < ctas; ++r) {
                SampleShared *s = of(&sh, r);
                if (none) atomicAdd(&s->none, none);
                if (low) atomicAdd(&s->low, low);
                if (zeros) atomicAdd(&s->zeros, zeros);
                if (flags) atomicOr(&s->flags, flags);
                atomicMax(&s->top, top);
            }
    }
    meet(cluster, ctas);
    sum_groups<DTYPE>(job, rank, ctas, sh, sample_smem);
    meet(cluster, ctas);
    if (warp == 0) decide_counted<DTYPE>(job, row, uniform, (uint32_t)piece.units * 8, rank, ctas, sh, sample_smem);
    __syncthreads();
    const Element drawn = sh.drawn;
    if (drawn.n == 0) {                      // the same for all CTAs of the row
        const bool odd = drawn.rank == SAMPLE_ODD;
        meet(cluster, ctas);                 // everybody has read what the search writes over
        if (odd) {
            search_odd_row<DTYPE, THREADS>(job, row, rank, ctas, sh, sample_smem);
            meet(cluster, ctas);
        }
        return;
    }
    const uint32_t bits = Storage<DTYPE>::put(drawn.value);
    const Equals<DTYPE> matches{bits * 0x10001u};
    uint32_t skip = 0, have = drawn.have;
    if (ctas > 1 && Count<DTYPE>::ZEROS && drawn.value == 0.0f) {
        uint32_t mine = 0;                   // zeros have no word: counted here
        for (int32_t u = piece.begin + (int32_t)threadIdx.x; u < piece.end; u += THREADS) mine += __popc(matches(piece.load(u)));
        mine = __reduce_add_sync(0xffffffffu, mine);
        if (threadIdx.x == 0) sh.here = 0;
        __syncthreads();
        if (lane == 0 && mine) atomicAdd(&sh.here, mine);
        cluster.sync();
        for (int r = 0; r < rank; ++r) skip += cluster.map_shared_rank(&sh, r)->here;
        have = sh.here;
    } else if (ctas > 1) {
        // how many of them each piece holds: the other CTAs' words still tell; the owner's own are what is left of the sum
        const uint32_t magnitude = bits & 0x7fffu;
        const int own = (int)(magnitude - F::LOW) / GROUP / (G::SIDE / ctas);      // the CTA that added this group up
        uint32_t c = 0;
        if (lane < ctas && lane != own) {
            const uint32_t word = reinterpret_cast<const uint32_t *>(cluster.map_shared_rank(&sample_smem[0], lane))[magnitude & F::MASK];
            c = magnitude == 0 ? (word & 0xffffu) + (word >> 16) : bits & 0x8000u ? word >> 16 : word & 0xffffu;
        }
        const uint32_t others = __reduce_add_sync(0xffffffffu, c);
        if (lane == own) c = drawn.have - others;
        skip = __reduce_add_sync(0xffffffffu, lane < rank ? c : 0u);
        have = __shfl_sync(0xffffffffu, c, rank);
    }
    if (drawn.rank >= skip && drawn.rank - skip < have) locate<THREADS>(piece, have - 1 - (drawn.rank - skip), sh, job.tokens + row, matches);
    if (ctas > 1) cluster.sync();            // no CTA leaves while another still reads its shared memory
}

// ---- host side --------------------------------------------------------------------------------------
namespace {

template <auto kernel, int THREADS>
bool sample_launch(size_t smem, const SampleJob &job, int32_t units, cudaStream_t stream)
{
    static std::atomic<bool> ready[DEVICES];
    int dev = 0;
    if (cudaGetDevice(&dev) != cudaSuccess || dev < 0 || dev >= DEVICES) return false;
    if (!ready[dev].load(std::memory_order_relaxed)) {
        if (cudaFuncSetAttribute(kernel, cudaFuncAttributeMaxDynamicSharedMemorySize, (int)smem) != cudaSuccess) return false;
        ready[dev].store(true, std::memory_order_relaxed);
    }
    // Few rows are shared out, until 768 threads to an SM have work, each CTA with 1024 units or more: what a CTA does besides reading
    // its piece costs as much as 2000 units.  74 x 128256: bf16 25 us with 296 CTAs, 28 with 148, 38 with 592; f16 29 with 148, 50 with
    // 296; f32 68 with 148, 109 with 74, 87 with 296.  And no more than PIECE_MOST logits to a CTA.  (A float32 row is passed over four times:
    // shared by four CTAs the rows in work would stay in the L2 cache, but each pass ends in meetings.  512 x 152064: 561 us against 507.)
    int ctas = 1;
    while (ctas < SAMPLE_CTAS && (((int64_t)job.R * ctas * 2 * THREADS <= 148 * 768 && units / (ctas * 2) >= 1024) || job.V > (int64_t)PIECE_MOST * ctas)) ctas *= 2;
    cudaLaunchConfig_t config = {};
    config.gridDim = dim3((unsigned)(job.R * ctas));
    config.blockDim = dim3(THREADS);
    config.dynamicSmemBytes = smem;
    config.stream = stream;
    cudaLaunchAttribute attributes[2];
    attributes[0].id = cudaLaunchAttributeProgrammaticStreamSerialization;
    attributes[0].val.programmaticStreamSerializationAllowed = 1;
    attributes[1].id = cudaLaunchAttributeClusterDimension;
    attributes[1].val.clusterDim.x = (unsigned)ctas;
    attributes[1].val.clusterDim.y = attributes[1].val.clusterDim.z = 1;
    config.attrs = attributes;
    config.numAttrs = 2;
    return cudaLaunchKernelEx(&config, kernel, job) == cudaSuccess;
}

bool launch_search(const SampleJob &job, int32_t units, cudaStream_t stream)
{
    constexpr int THREADS = 512;
    return sample_launch<sample_search_kernel<THREADS>, THREADS>(sizeof(SearchBins<SEARCH_BINS>), job, units, stream);
}
template <int PER> bool launch_sort(const SampleJob &job, cudaStream_t stream)
{
    return launch_after(sample_sort_kernel<PER>, (unsigned)job.R, SORT_THREADS, 0, stream, job);
}
template <int DTYPE> bool launch_count(const SampleJob &job, int32_t units, cudaStream_t stream)
{
    using F = Counted<DTYPE>;
    return sample_launch<sample_count_kernel<DTYPE>, F::THREADS>(F::WORDS * 4, job, units, stream);
}

}  // namespace
}  // namespace ppow

#ifdef PPOW_CHECKED
namespace ppow { int read_check_counters_sample(unsigned int *f, unsigned int *s) { return read_check_counters(f, s); } }
#endif

using namespace ppow;

extern "C" ppow_status ppow_sample_tokens(const ppow_sample_params *params, const void *logits, const float *uniforms, int32_t *tokens, float *logp,
                                          int32_t *kept, void *cuda_stream)
{
    if (!params || params->R < 0 || params->R > (1 << 27) || params->V < 1 || !dtype_ok(params->dtype) || !stride_ok(params->logits_stride, params->V))
        return PPOW_ERR_INVALID_ARG;
    if (!(params->temperature >= 1e-30 && params->temperature <= 1e30) || params->top_k < 0 || !(params->top_p > 0.0 && params->top_p <= 1.0) ||
        !(params->min_p >= 0.0 && params->min_p <= 1.0))
        return PPOW_ERR_INVALID_ARG;
    if (params->V > SAMPLE_MAX_VOCAB) return PPOW_ERR_UNSUPPORTED;
    if (params->R == 0) return PPOW_OK;
    const size_t es = bytes_of(params->dtype);
    if (!logits || !uniforms || !tokens || !logp || (uintptr_t)logits % es || (uintptr_t)uniforms % 4 || (uintptr_t)tokens % 4 || (uintptr_t)logp % 4 ||
        (uintptr_t)kept % 4)
        return PPOW_ERR_INVALID_ARG;
    const SampleJob job = {logits,        params->logits_stride, uniforms, params->R, params->V, params->top_k, params->temperature,
                           params->top_p, params->min_p,         tokens,   logp,      kept};
    const int32_t units = (int32_t)((params->V * (int64_t)es + 15) / 16);
    cudaStream_t stream = (cudaStream_t)cuda_stream;
    const bool ok = params->dtype == PPOW_F32    ? (params->V <= SORT_THREADS * 4   ? launch_sort<4>(job, stream)
                                                    : params->V <= SORT_THREADS * 8 ? launch_sort<8>(job, stream)
                                                                                    : launch_search(job, units, stream))
                    : params->dtype == PPOW_BF16 ? launch_count<PPOW_BF16>(job, units, stream)
                                                 : launch_count<PPOW_F16>(job, units, stream);
    return ok ? PPOW_OK : PPOW_ERR_CUDA;
}
