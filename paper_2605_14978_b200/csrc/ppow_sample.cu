// Tokens drawn from logits with given uniforms: temperature, top-k, top-p, min-p.
//
// A row's tokens in descending order of their logits, ties by index; w_i = exp((z_i - z_max) / T), C_n = w_1 + ... + w_n:
//   n_k = min(top_k, F)          F: logits above -inf
//   n_p = least n with C_n >= top_p C_{n_k}
//   n_m = number of i with w_i >= min_p
//   n   = min(n_k, n_p, n_m);    token = first j with C_j > u C_n;    logp = (z_j - z_max) / T - ln C_n
//
// A draw lies next to one of up to a million borders, so the masses have to be right to far more digits than float32 holds if the token
// is to be the definition's, and the same whichever way the row is cut.  All masses are float64, and none depends on an order:
//
//   16-bit logits   A row holds at most 65536 different numbers: one pass counts them, by integer additions in shared memory, and all the
//                   rest is arithmetic on a few thousand (number, count) pairs.  Bound by those additions (one warp's 32 fall on the 32
//                   banks at random, 3.5 cycles) where the row's bytes take 2.2 of the same cycles.
//   float32         A row holds any numbers, so they go into 2048 bins of equal depth below the maximum, each with its count and its mass in
//                   64-bit fixed point relative to the bin's top (integers again).  A border is followed into its bin by further passes
//                   over the keys, 2048 to one, until a bin holds one number.  16-bit rows that the counting does not fit (logits
//                   of 2048 and more, more than 65535 equal ones) go the same way.
//
// A cluster of CTAs shares a row, each with a contiguous piece of it: one CTA when there are rows enough, up to eight for a few.
#include "ppow_checked.cuh"
#include "ppow_rows.cuh"

#include <cooperative_groups.h>

namespace ppow {
namespace cg = cooperative_groups;

constexpr int SAMPLE_THREADS = 512, SAMPLE_WARPS = SAMPLE_THREADS / 32, SAMPLE_CTAS = 8;
constexpr int32_t SAMPLE_MAX_VOCAB = 1 << 22;
constexpr int CHUNK = 256;               // bins whose counts and masses are summed up together
constexpr int CHUNKS_MOST = 256;
constexpr int SEARCH_BINS = 2048, SEARCH_CHUNK = 32, SEARCH_CHUNKS = SEARCH_BINS / SEARCH_CHUNK;
constexpr double SEARCH_NATS = 64.0;     // what lies deeper than this below the maximum has no mass: 2^22 exp(-64) is 1e-21
constexpr double MASS_ONE = 2199023255552.0;        // 2^41: a weight of 1; the 2^22 weights of a bin stay below 2^64

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
// Counting: keys (bits in the order of the numbers) from BASE on, BINS of them, hold every |z| < LIMIT.  ZERO, the bin of +0, is even
// and not a chunk's first, so that -0, the bin before it, can be added to it within the chunk.
template <int DTYPE> struct Counted;
template <> struct Counted<PPOW_BF16> {
    static constexpr uint32_t LOWEST = 0x007fu, HIGHEST = 0xff80u, NEG_INF = 0xff80u;   // keys of -inf, +inf; bits of -inf
    static constexpr uint32_t ZERO = 139 * 128, BINS = 2 * ZERO, BASE = 0x8000u - ZERO;
    static constexpr double LIMIT = 4096.0;
};
template <> struct Counted<PPOW_F16> {
    static constexpr uint32_t LOWEST = 0x03ffu, HIGHEST = 0xfc00u, NEG_INF = 0xfc00u;
    static constexpr uint32_t ZERO = 26 * 1024 + 128, BINS = 2 * ZERO, BASE = 0x8000u - ZERO;
    static constexpr double LIMIT = 2048.0;
};
static_assert(Counted<PPOW_BF16>::BINS % CHUNK == 0 && Counted<PPOW_F16>::BINS % CHUNK == 0, "whole chunks");
static_assert(Counted<PPOW_BF16>::ZERO % CHUNK != 0 && Counted<PPOW_F16>::ZERO % CHUNK != 0, "-0 beside +0");
static_assert(Counted<PPOW_F16>::BINS / CHUNK <= CHUNKS_MOST, "chunks");

template <int DTYPE> __device__ __forceinline__ float number_of(uint32_t bin)
{
    const uint32_t key = bin + Counted<DTYPE>::BASE;
    return Storage<DTYPE>::get((uint16_t)(key & 0x8000u ? key ^ 0x8000u : ~key));
}

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
                mask_halves(w, lo, hi, Counted<DTYPE>::NEG_INF);
            }
        }
        return w;
    }
    __device__ __forceinline__ int32_t token(int32_t u, int e) const { return u * E + e - head; }
};

// ---- borders ----------------------------------------------------------------------------------------
enum class Border { Count, MassFrom, MassAbove };    // the first place where the count, or the mass, reaches `target`; the mass passes it

struct Place {
    int item;
    uint32_t count;          // elements before it
    double mass;             // and their mass
};

struct Target {
    Border kind;
    uint32_t count;
    double mass;
    __device__ __forceinline__ bool met(uint32_t c, double m) const
    {
        return kind == Border::Count ? c >= count : kind == Border::MassFrom ? m >= mass : m > mass;
    }
};

// The item of 0 .. n-1 (n <= 256, descending) that holds the border; the last one that is not empty if rounding leaves it to
// none.  get(item, count, mass).  The whole warp calls, every lane has the result.
template <typename Get> __device__ Place warp_find(int n, const Target &target, const Place &before, Get &&get)
{
    constexpr int PER = CHUNKS_MOST / 32;
    const int lane = threadIdx.x & 31;
    uint32_t c[PER], count = 0;
    double m[PER], mass = 0.0;
#pragma unroll
    for (int i = 0; i < PER; ++i) {
        c[i] = 0;
        m[i] = 0.0;
        if (lane * PER + i < n) get(lane * PER + i, c[i], m[i]);
        count += c[i];
        mass += m[i];
    }
#pragma unroll
    for (int o = 1; o < 32; o <<= 1) {
        const uint32_t c2 = __shfl_up_sync(0xffffffffu, count, o);
        const double m2 = __shfl_up_sync(0xffffffffu, mass, o);
        if (lane >= o) count += c2, mass += m2;
    }
    count = __shfl_up_sync(0xffffffffu, count, 1);
    mass = __shfl_up_sync(0xffffffffu, mass, 1);
    if (lane == 0) count = 0, mass = 0.0;
    count += before.count;
    mass += before.mass;
    Place found = {-1, 0, 0.0}, last = {-1, 0, 0.0};
#pragma unroll
    for (int i = 0; i < PER; ++i) {
        if (target.kind == Border::Count ? c[i] > 0 : m[i] > 0.0) {
            last = {lane * PER + i, count, mass};
            if (found.item < 0 && target.met(count + c[i], mass + m[i])) found = last;
        }
        count += c[i];
        mass += m[i];
    }
    uint32_t who = __ballot_sync(0xffffffffu, found.item >= 0);
    int from = __ffs(who) - 1;
    if (who == 0) {
        who = __ballot_sync(0xffffffffu, last.item >= 0);
        from = who ? 31 - __clz(who) : 0;
        found = last;
    }
    return {__shfl_sync(0xffffffffu, found.item, from), __shfl_sync(0xffffffffu, found.count, from), __shfl_sync(0xffffffffu, found.mass, from)};
}

// A number, how many elements have it, what lies before them, and which of them is meant.
struct Number {
    float value;
    uint32_t have, before, rank;         // rank: 0 .. have - 1
    double weight, mass;                 // of one element; of those before
    __device__ __forceinline__ uint32_t n() const { return before + rank + 1; }
    __device__ __forceinline__ double total() const { return mass + (rank + 1) * weight; }
    __device__ __forceinline__ void choose(const Target &target)
    {
        if (target.kind == Border::Count) {
            rank = min(target.count - before, have) - 1;
            return;
        }
        // the quotient is right to a small part of 1, but for weights below 1e-13 of the mass, which no border can tell apart
        const double q = floor((target.mass - mass) / weight);
        rank = q >= (double)have ? have - 1 : q > 0.0 ? (uint32_t)q : 0;
        if (rank > 0 && target.met(0, mass + rank * weight)) --rank;
        if (rank < have - 1 && !target.met(0, mass + (rank + 1) * weight)) ++rank;
    }
};

struct SampleShared {
    uint32_t chunk_count[CHUNKS_MOST], chunk_within[CHUNKS_MOST];       // elements; those within min_p
    double chunk_mass[CHUNKS_MOST];
    int32_t chunk_top[CHUNKS_MOST];          // highest bin that is not empty
    uint32_t none, low, flags;               // -inf; below the counted range; SAMPLE_*
    uint32_t warp_count[2][SAMPLE_WARPS];
    uint32_t here;                           // elements of the drawn number in this piece
    // search
    uint32_t max_key, low_key, high_key, within;
    // results of warp 0
    Number drawn;
    uint32_t n;
    double total;
    Place place;
};
enum : uint32_t { SAMPLE_BAD = 1, SAMPLE_ODD = 2 };      // NaN or +inf; a row that counting does not fit

template <typename Cluster> __device__ __forceinline__ void meet(const Cluster &cluster, int ctas)
{
    if (ctas == 1)
        __syncthreads();
    else
        cluster.sync();
}

// The whole distribution of a row from find(target), which gives the number that holds a border: what is kept, and the draw.
// F: elements above -inf, of which `massive` carry the mass `all`.  One warp.
template <typename Find>
__device__ void decide(const SampleJob &job, float u, uint32_t F, uint32_t massive, double all, uint32_t within, Find &&find, Number &drawn,
                       uint32_t &n, double &total)
{
    n = job.top_k > 0 && (uint32_t)job.top_k < F ? (uint32_t)job.top_k : F;
    total = n < massive ? find(Target{Border::Count, n, 0.0}).total() : all;
    if (job.top_p < 1.0) {
        const Number border = find(Target{Border::MassFrom, 0, job.top_p * total});
        if (border.n() < n) n = border.n(), total = border.total();
    }
    if (job.min_p > 0.0 && within < n) {
        n = within;
        total = find(Target{Border::Count, n, 0.0}).total();
    }
    const double at = fminf(fmaxf(u, 0.0f), 0x1.fffffep-1f);        // NaN is 0
    drawn = find(Target{Border::MassAbove, 0, at * total});
    if (drawn.n() > n) drawn = find(Target{Border::Count, n, 0.0});
}

// The index of the rank-th element of this piece that `matches` accepts; searched in rounds, each warp a stretch of neighbouring units.
template <int DTYPE, typename Matches>
__device__ void locate(const Piece<DTYPE> &piece, uint32_t rank, SampleShared &sh, int32_t *token, Matches &&matches)
{
    using S = Storage<DTYPE>;
    constexpr int E = S::PER_UNIT, DEEP = 4;
    const int lane = threadIdx.x & 31, warp = threadIdx.x >> 5;
    uint32_t seen = 0;
    int turn = 0;
    for (int32_t base = piece.begin; base < piece.end; base += SAMPLE_THREADS * DEEP, turn ^= 1) {
        uint32_t bits[DEEP], mine = 0;
#pragma unroll
        for (int q = 0; q < DEEP; ++q) {
            const int32_t u = base + (warp * DEEP + q) * 32 + lane;
            bits[q] = 0;
            if (u < piece.end) bits[q] = matches(piece.load(u));
            mine += __popc(bits[q]);
        }
        mine = __reduce_add_sync(0xffffffffu, mine);
        if (lane == 0) sh.warp_count[turn][warp] = mine;
        __syncthreads();
        uint32_t before = seen;
        for (int i = 0; i < SAMPLE_WARPS; ++i) {
            const uint32_t c = sh.warp_count[turn][i];
            if (i < warp) before += c;
            seen += c;
        }
        if (before <= rank && rank < before + mine) {
#pragma unroll
            for (int q = 0; q < DEEP; ++q) {
                uint32_t upto = __popc(bits[q]);
#pragma unroll
                for (int o = 1; o < 32; o <<= 1) {
                    const uint32_t v = __shfl_up_sync(0xffffffffu, upto, o);
                    if (lane >= o) upto += v;
                }
                const uint32_t from = before + upto - __popc(bits[q]);
                if (from <= rank && rank < before + upto)
                    *token = piece.token(base + (warp * DEEP + q) * 32 + lane, (int)__fns(bits[q], 0, (int)(rank - from) + 1));
                before += __shfl_sync(0xffffffffu, upto, 31);
            }
        }
        if (seen > rank) return;             // the same for the whole CTA
    }
    static_assert(E <= 8, "a bit for each element");
}

// ---- search: any row --------------------------------------------------------------------------------
struct SearchBins {
    uint32_t count[SEARCH_BINS], low[SEARCH_BINS], high[SEARCH_BINS];       // of this CTA; mass in fixed point
    uint32_t all_count[SEARCH_BINS];                                        // of the cluster
    double all_mass[SEARCH_BINS];
};

template <int DTYPE> struct Search {
    using S = Storage<DTYPE>;
    static constexpr int E = S::PER_UNIT;
    const SampleJob &job;
    const Piece<DTYPE> &piece;
    const cg::cluster_group &cluster;
    int rank, ctas;
    SampleShared &sh;
    SearchBins &bins;
    double top, scale, per_nat;              // maximum; bins per logit; 1 / temperature

    template <typename F> __device__ __forceinline__ void each(F &&f) const
    {
        for (int32_t u = piece.begin + (int32_t)threadIdx.x; u < piece.end; u += SAMPLE_THREADS) {
            float z[E];
            S::unpack(piece.load(u), z);
#pragma unroll
            for (int e = 0; e < E; ++e) f(z[e]);
        }
    }
    __device__ __forceinline__ int depth_bin(double d) const { return (int)fmin(d * scale, (double)(SEARCH_BINS - 1)); }
    __device__ __forceinline__ double weight(double d) const { return exp(-d * per_nat); }

    __device__ void clear()
    {
        for (int i = threadIdx.x; i < SEARCH_BINS; i += SAMPLE_THREADS) bins.count[i] = bins.low[i] = bins.high[i] = 0;
        __syncthreads();
    }
    // mass relative to the top of a depth bin, 2^41 to the whole
    __device__ __forceinline__ void add(int item, double d, double bin_top)
    {
        const unsigned long long w = __double2ull_rn(exp((bin_top - d) * per_nat) * MASS_ONE);
        if (!PPOW_CHECK(item >= 0 && item < SEARCH_BINS, 801, nullptr)) return;
        atomicAdd(&bins.count[item], 1u);
        const uint32_t lo = (uint32_t)w, old = atomicAdd(&bins.low[item], lo);
        const uint32_t hi = (uint32_t)(w >> 32) + (old + lo < old ? 1u : 0u);
        if (hi) atomicAdd(&bins.high[item], hi);
    }
    // Sums up the CTAs' bins, each CTA a share of them for all, and the chunks.  unit(item): what a mass of 1 in this bin stands for.
    template <typename Unit> __device__ void join(Unit &&unit)
    {
        meet(cluster, ctas);
        for (int i = rank * SAMPLE_THREADS + (int)threadIdx.x; i < SEARCH_BINS; i += ctas * SAMPLE_THREADS) {
            uint32_t count = 0;
            unsigned long long mass = 0;
            for (int r = 0; r < ctas; ++r) {
                const SearchBins *b = ctas == 1 ? &bins : cluster.map_shared_rank(&bins, r);
                count += b->count[i];
                mass += b->low[i] + ((unsigned long long)b->high[i] << 32);
            }
            const double m = count ? (double)mass * (1.0 / MASS_ONE) * unit(i) : 0.0;
            for (int r = 0; r < ctas; ++r) {
                SearchBins *b = ctas == 1 ? &bins : cluster.map_shared_rank(&bins, r);
                b->all_count[i] = count;
                b->all_mass[i] = m;
            }
        }
        meet(cluster, ctas);
        for (int c = threadIdx.x >> 5; c < SEARCH_CHUNKS; c += SAMPLE_WARPS) {
            const int i = c * SEARCH_CHUNK + (threadIdx.x & 31);
            const uint32_t count = __reduce_add_sync(0xffffffffu, bins.all_count[i]);
            const double mass = warp_sum_f64(bins.all_mass[i]);
            if ((threadIdx.x & 31) == 0) sh.chunk_count[c] = count, sh.chunk_mass[c] = mass;
        }
        __syncthreads();
    }
    // The bin that holds the border; all threads have the result.
    __device__ Place find_bin(const Target &target, const Place &before)
    {
        if (threadIdx.x < 32) {
            Place p = warp_find(SEARCH_CHUNKS, target, before, [&](int i, uint32_t &c, double &m) { c = sh.chunk_count[i], m = sh.chunk_mass[i]; });
            const int chunk = p.item < 0 ? 0 : p.item;
            p = warp_find(SEARCH_CHUNK, target, p, [&](int i, uint32_t &c, double &m) {
                c = bins.all_count[chunk * SEARCH_CHUNK + i], m = bins.all_mass[chunk * SEARCH_CHUNK + i];
            });
            p.item = chunk * SEARCH_CHUNK + (p.item < 0 ? 0 : p.item);
            if (threadIdx.x == 0) sh.place = p;
        }
        __syncthreads();
        const Place p = sh.place;
        __syncthreads();
        return p;
    }
    __device__ void fill_depths()
    {
        clear();
        each([&](float z) {
            if (z == -INFINITY) return;
            const double d = top - (double)z;
            const int b = depth_bin(d);
            if (b < SEARCH_BINS - 1)
                add(b, d, b / scale);
            else
                atomicAdd(&bins.count[b], 1u);               // too deep for any mass
        });
        join([&](int i) { return exp(-(i / scale) * per_nat); });
    }
    // The number that holds the border; the whole CTA, and the whole cluster in step.
    __device__ Number find(const Target &target)
    {
        fill_depths();
        Place p = find_bin(target, Place{0, 0, 0.0});
        const int bin = p.item;
        const bool massless = bin == SEARCH_BINS - 1;
        const double bin_top = bin / scale, unit = massless ? 0.0 : exp(-bin_top * per_nat);
        // keys in the bin
        if (threadIdx.x == 0) sh.low_key = 0xffffffffu, sh.high_key = 0;
        meet(cluster, ctas);
        uint32_t lo = 0xffffffffu, hi = 0;
        each([&](float z) {
            if (z == -INFINITY || depth_bin(top - (double)z) != bin) return;
            const uint32_t k = key_of(z);
            lo = min(lo, k), hi = max(hi, k);
        });
        lo = __reduce_min_sync(0xffffffffu, lo), hi = __reduce_max_sync(0xffffffffu, hi);
        if ((threadIdx.x & 31) == 0) {
            for (int r = 0; r < ctas; ++r) {
                SampleShared *s = ctas == 1 ? &sh : cluster.map_shared_rank(&sh, r);
                atomicMin(&s->low_key, lo);
                atomicMax(&s->high_key, hi);
            }
        }
        meet(cluster, ctas);
        lo = sh.low_key, hi = sh.high_key;
        int shift = 0;
        while (((hi - lo) >> shift) >= SEARCH_BINS) ++shift;
        for (;;) {
            clear();
            each([&](float z) {
                if (z == -INFINITY) return;
                const uint32_t k = key_of(z);
                if (k < lo || k > hi) return;
                const int item = (int)((hi - k) >> shift);
                if (massless) {
                    if (PPOW_CHECK(item < SEARCH_BINS, 802, nullptr)) atomicAdd(&bins.count[item], 1u);
                } else {
                    add(item, top - (double)z, bin_top);
                }
            });
            join([&](int) { return unit; });
            p = find_bin(target, p);
            hi -= (uint32_t)p.item << shift;
            if (shift == 0) break;
            const uint32_t width = (1u << shift) - 1;
            lo = hi - lo > width ? hi - width : lo;
            shift = shift > 11 ? shift - 11 : 0;
        }
        Number found;
        found.value = float_of(hi);
        found.have = bins.all_count[p.item];
        found.before = p.count;
        found.mass = p.mass;
        found.weight = massless ? 0.0 : weight(top - (double)found.value);
        if (massless)
            found.rank = target.kind == Border::Count ? min(target.count - p.count, found.have) - 1 : 0;
        else
            found.choose(target);
        __syncthreads();
        return found;
    }
    __device__ void run(int64_t row)
    {
        if (threadIdx.x == 0) sh.max_key = sh.none = sh.flags = sh.within = 0;
        meet(cluster, ctas);
        uint32_t most = 0, none = 0, bad = 0;
        each([&](float z) {
            bad |= !(z < INFINITY);
            none += z == -INFINITY;
            most = max(most, key_of(z));
        });
        most = __reduce_max_sync(0xffffffffu, most), none = __reduce_add_sync(0xffffffffu, none), bad = __reduce_or_sync(0xffffffffu, bad);
        if ((threadIdx.x & 31) == 0) {
            for (int r = 0; r < ctas; ++r) {
                SampleShared *s = ctas == 1 ? &sh : cluster.map_shared_rank(&sh, r);
                atomicMax(&s->max_key, most);
                atomicAdd(&s->none, none);
                if (bad) atomicOr(&s->flags, (uint32_t)SAMPLE_BAD);
            }
        }
        meet(cluster, ctas);
        const uint32_t F = (uint32_t)piece.units * E - sh.none;
        const bool lead = rank == 0 && threadIdx.x == 0;
        if (sh.flags & SAMPLE_BAD || F == 0) {
            if (lead) {
                job.tokens[row] = -1;
                job.logp[row] = F == 0 && !(sh.flags & SAMPLE_BAD) ? -INFINITY : NAN;
                if (job.kept) job.kept[row] = 0;
            }
            return;
        }
        top = (double)float_of(sh.max_key);
        per_nat = 1.0 / job.temperature;
        scale = (SEARCH_BINS - 1) / (SEARCH_NATS * job.temperature);
        if (job.min_p > 0.0) {
            uint32_t within = 0;
            each([&](float z) { within += z > -INFINITY && weight(top - (double)z) >= job.min_p; });
            within = __reduce_add_sync(0xffffffffu, within);
            if ((threadIdx.x & 31) == 0)
                for (int r = 0; r < ctas; ++r) atomicAdd(&(ctas == 1 ? &sh : cluster.map_shared_rank(&sh, r))->within, within);
        }
        fill_depths();
        uint32_t massive = F - bins.all_count[SEARCH_BINS - 1];
        double all = 0.0;
        for (int c = 0; c < SEARCH_CHUNKS; ++c) all += sh.chunk_mass[c];
        const uint32_t within = sh.within;
        __syncthreads();
        Number drawn;
        uint32_t n;
        double total;
        decide(job, job.uniforms[row], F, massive, all, within, [&](const Target &t) { return find(t); }, drawn, n, total);
        if (lead) {
            job.logp[row] = (float)(((double)drawn.value - top) * per_nat - log(total));
            if (job.kept) job.kept[row] = (int32_t)n;
        }
        // which piece holds it
        const uint32_t key = key_of(drawn.value);
        auto matches = [&](const uint4 &w) {
            float z[E];
            S::unpack(w, z);
            uint32_t bits = 0;
#pragma unroll
            for (int e = 0; e < E; ++e) bits |= (z[e] > -INFINITY && key_of(z[e]) == key) ? 1u << e : 0u;
            return bits;
        };
        uint32_t skip = 0, have = 0xffffffffu;
        if (ctas > 1) {
            if (threadIdx.x == 0) sh.here = 0;
            __syncthreads();
            uint32_t mine = 0;
            for (int32_t u = piece.begin + (int32_t)threadIdx.x; u < piece.end; u += SAMPLE_THREADS) mine += __popc(matches(piece.load(u)));
            mine = __reduce_add_sync(0xffffffffu, mine);
            if ((threadIdx.x & 31) == 0 && mine) atomicAdd(&sh.here, mine);
            cluster.sync();
            for (int r = 0; r < rank; ++r) skip += cluster.map_shared_rank(&sh, r)->here;
            have = sh.here;
        }
        if (drawn.rank >= skip && drawn.rank - skip < have) locate(piece, drawn.rank - skip, sh, job.tokens + row, matches);
    }
};

template <int DTYPE>
__device__ __noinline__ void search_row(const SampleJob &job, int64_t row, int rank, int ctas, SampleShared &sh, void *smem)
{
    const Piece<DTYPE> piece(job, row, rank, ctas);
    const cg::cluster_group cluster = cg::this_cluster();
    Search<DTYPE> s{job, piece, cluster, rank, ctas, sh, *static_cast<SearchBins *>(smem), 0.0, 0.0, 0.0};
    s.run(row);
}

__global__ void __launch_bounds__(SAMPLE_THREADS) sample_search_kernel(const SampleJob job)
{
    wait_for_previous_kernel();
    extern __shared__ uint4 sample_smem[];
    __shared__ SampleShared sh;
    const cg::cluster_group cluster = cg::this_cluster();
    const int ctas = (int)cluster.num_blocks(), rank = (int)cluster.block_rank();
    search_row<PPOW_F32>(job, blockIdx.x / ctas, rank, ctas, sh, sample_smem);
    if (ctas > 1) cluster.sync();            // no CTA leaves while another still reads its shared memory
}

// ---- counting: 16-bit rows --------------------------------------------------------------------------
template <int DTYPE> struct Count {
    using F = Counted<DTYPE>;
    static constexpr int CHUNKS = F::BINS / CHUNK;
    uint32_t *words;         // two bins each

    __device__ __forceinline__ void add(uint32_t key, uint32_t &none, uint32_t &low, uint32_t &flags)
    {
        const uint32_t bin = key - F::BASE;
        if (bin < F::BINS) {
            atomicAdd(&words[bin >> 1], 1u << ((bin & 1) * 16));
        } else if (key == F::LOWEST) {
            ++none;
        } else if (key < F::LOWEST || key >= F::HIGHEST) {
            flags |= SAMPLE_BAD;
        } else if (key < F::BASE) {
            ++low;
        } else {
            flags |= SAMPLE_ODD;
        }
    }
    __device__ __forceinline__ void add_word(uint32_t w, uint32_t &none, uint32_t &low, uint32_t &flags)
    {
        const uint32_t sign = w & 0x80008000u, keys = w ^ (sign - (sign >> 15)) ^ 0x80008000u;
        add(keys & 0xffffu, none, low, flags);
        add(keys >> 16, none, low, flags);
    }
};

template <int DTYPE>
__global__ void __launch_bounds__(SAMPLE_THREADS) sample_count_kernel(const SampleJob job)
{
    using F = Counted<DTYPE>;
    using C = Count<DTYPE>;
    extern __shared__ uint4 sample_smem[];
    __shared__ SampleShared sh;
    wait_for_previous_kernel();
    const cg::cluster_group cluster = cg::this_cluster();
    const int ctas = (int)cluster.num_blocks(), rank = (int)cluster.block_rank();
    const int lane = threadIdx.x & 31, warp = threadIdx.x >> 5;
    const int64_t row = blockIdx.x / ctas;
    const Piece<DTYPE> piece(job, row, rank, ctas);
    C bins{reinterpret_cast<uint32_t *>(sample_smem)};
    for (int i = threadIdx.x; i < (int)F::BINS / 8; i += SAMPLE_THREADS) sample_smem[i] = make_uint4(0, 0, 0, 0);
    if (threadIdx.x == 0) sh.none = sh.low = sh.flags = 0;
    __syncthreads();
    {
        uint32_t none = 0, low = 0, flags = 0;
        constexpr int DEEP = 4;
        for (int32_t u0 = piece.begin + (int32_t)threadIdx.x; u0 < piece.end; u0 += SAMPLE_THREADS * DEEP) {
            uint4 w[DEEP];
#pragma unroll
            for (int q = 0; q < DEEP; ++q)
                if (u0 + q * SAMPLE_THREADS < piece.end) w[q] = piece.load(u0 + q * SAMPLE_THREADS);
#pragma unroll
            for (int q = 0; q < DEEP; ++q)
                if (u0 + q * SAMPLE_THREADS < piece.end) {
                    bins.add_word(w[q].x, none, low, flags);
                    bins.add_word(w[q].y, none, low, flags);
                    bins.add_word(w[q].z, none, low, flags);
                    bins.add_word(w[q].w, none, low, flags);
                }
        }
        none = __reduce_add_sync(0xffffffffu, none), low = __reduce_add_sync(0xffffffffu, low), flags = __reduce_or_sync(0xffffffffu, flags);
        if (lane == 0) {
            if (none) atomicAdd(&sh.none, none);
            if (low) atomicAdd(&sh.low, low);
            if (flags) atomicOr(&sh.flags, flags);
        }
    }
    meet(cluster, ctas);
    // Each CTA adds up a share of the chunks for all, in its own bins: the other CTAs read none of those.
    const int from = C::CHUNKS * rank / ctas, to = C::CHUNKS * (rank + 1) / ctas;
    for (int c = from + warp; c < to; c += SAMPLE_WARPS) {
        const int at = c * (CHUNK / 8) + lane;
        uint4 w = sample_smem[at];
        uint32_t b[8] = {w.x & 0xffffu, w.x >> 16, w.y & 0xffffu, w.y >> 16, w.z & 0xffffu, w.z >> 16, w.w & 0xffffu, w.w >> 16};
        for (int r = 1; r < ctas; ++r) {
            const uint4 o = cluster.map_shared_rank(sample_smem, (rank + r) % ctas)[at];
            b[0] += o.x & 0xffffu, b[1] += o.x >> 16, b[2] += o.y & 0xffffu, b[3] += o.y >> 16;
            b[4] += o.z & 0xffffu, b[5] += o.z >> 16, b[6] += o.w & 0xffffu, b[7] += o.w >> 16;
        }
        if (c == (int)F::ZERO / CHUNK) {                     // -0 to +0
            constexpr int LANE = F::ZERO % CHUNK / 8, SLOT = F::ZERO % 8;
            static_assert(SLOT == 0, "+0 is the first of its lane's bins, -0 the last of the lane before");
            const uint32_t minus = __shfl_sync(0xffffffffu, b[7], LANE - 1);
            if (lane == LANE) b[0] += minus;
            if (lane == LANE - 1) b[7] = 0;
        }
        uint32_t count = 0, over = 0;
        int32_t top = -1;
#pragma unroll
        for (int i = 0; i < 8; ++i) {
            count += b[i];
            over |= b[i] >> 16;
            if (b[i]) top = c * CHUNK + lane * 8 + i;
        }
        if (__any_sync(0xffffffffu, over != 0) && lane == 0) atomicOr(&sh.flags, (uint32_t)SAMPLE_ODD);
        if (ctas > 1 || c == (int)F::ZERO / CHUNK)
            sample_smem[at] = make_uint4(b[0] | (b[1] << 16), b[2] | (b[3] << 16), b[4] | (b[5] << 16), b[6] | (b[7] << 16));
        count = __reduce_add_sync(0xffffffffu, count);
        top = __reduce_max_sync(0xffffffffu, top);
        for (int r = lane; r < ctas; r += 32) {
            SampleShared *s = ctas == 1 ? &sh : cluster.map_shared_rank(&sh, r);
            s->chunk_count[c] = count;
            s->chunk_top[c] = top;
        }
    }
    meet(cluster, ctas);
    uint32_t none = 0, low = 0, flags = 0, counted = 0;
    int32_t top_bin = -1;
    for (int r = 0; r < ctas; ++r) {
        const SampleShared *s = ctas == 1 ? &sh : cluster.map_shared_rank(&sh, r);
        none += s->none, low += s->low, flags |= s->flags;
    }
    for (int c = lane; c < C::CHUNKS; c += 32) counted += sh.chunk_count[c], top_bin = max(top_bin, sh.chunk_top[c]);
    counted = __reduce_add_sync(0xffffffffu, counted);
    top_bin = __reduce_max_sync(0xffffffffu, top_bin);
    const double top = top_bin < 0 ? 0.0 : (double)number_of<DTYPE>((uint32_t)top_bin), per_nat = 1.0 / job.temperature;
    // a count that ran over left a sum that is short; numbers below the counted range have to be too deep for any mass
    if (counted + none + low != (uint32_t)piece.units * 8) flags |= SAMPLE_ODD;
    if (low > 0) {
        const double deep = (top + F::LIMIT) * per_nat;
        if (top_bin < 0 || deep < SEARCH_NATS || (job.min_p > 0.0 && exp(-deep) >= job.min_p)) flags |= SAMPLE_ODD;
    }
    if (flags || counted == 0) {                             // the same for all CTAs of the row
        if (flags & SAMPLE_BAD || (flags == 0 && counted == 0)) {
            if (rank == 0 && threadIdx.x == 0) {
                job.tokens[row] = -1;
                job.logp[row] = flags ? NAN : -INFINITY;
                if (job.kept) job.kept[row] = 0;
            }
            meet(cluster, ctas);
        } else {
            meet(cluster, ctas);             // everybody has read what the search writes over
            search_row<DTYPE>(job, row, rank, ctas, sh, sample_smem);
            meet(cluster, ctas);
        }
        return;
    }
    for (int c = from + warp; c < to; c += SAMPLE_WARPS) {
        if (sh.chunk_count[c] == 0) continue;
        const uint4 w = sample_smem[c * (CHUNK / 8) + lane];
        const uint32_t b[8] = {w.x & 0xffffu, w.x >> 16, w.y & 0xffffu, w.y >> 16, w.z & 0xffffu, w.z >> 16, w.w & 0xffffu, w.w >> 16};
        double mass = 0.0;
        uint32_t within = 0;
#pragma unroll
        for (int i = 0; i < 8; ++i)
            if (b[i]) {
                const double e = exp(((double)number_of<DTYPE>((uint32_t)(c * CHUNK + lane * 8 + i)) - top) * per_nat);
                mass += b[i] * e;
                if (e >= job.min_p) within += b[i];
            }
        mass = warp_sum_f64(mass);
        within = __reduce_add_sync(0xffffffffu, within);
        for (int r = lane; r < ctas; r += 32) {
            SampleShared *s = ctas == 1 ? &sh : cluster.map_shared_rank(&sh, r);
            s->chunk_mass[c] = mass;
            s->chunk_within[c] = within;
        }
    }
    meet(cluster, ctas);
    if (warp == 0) {
        uint32_t within = 0;
        double all = 0.0;
        for (int c = lane; c < C::CHUNKS; c += 32)
            if (sh.chunk_count[c]) within += sh.chunk_within[c], all += sh.chunk_mass[c];
        within = __reduce_add_sync(0xffffffffu, within);
        all = warp_sum_f64(all);
        auto owner = [&](int chunk) {        // the CTA that added this chunk up
            int r = 0;
            while (C::CHUNKS * (r + 1) / ctas <= chunk) ++r;
            return r;
        };
        auto find = [&](const Target &target) {
            Place p = warp_find(C::CHUNKS, target, Place{0, 0, 0.0}, [&](int i, uint32_t &c, double &m) {
                const int chunk = C::CHUNKS - 1 - i;
                c = sh.chunk_count[chunk];
                m = c ? sh.chunk_mass[chunk] : 0.0;
            });
            const int chunk = C::CHUNKS - 1 - max(p.item, 0);
            const uint4 *remote = ctas == 1 ? sample_smem : cluster.map_shared_rank(sample_smem, owner(chunk));
            const uint16_t *counts = reinterpret_cast<const uint16_t *>(remote + chunk * (CHUNK / 8));
            auto weight = [&](int bin) { return exp(((double)number_of<DTYPE>((uint32_t)bin) - top) * per_nat); };
            p = warp_find(CHUNK, target, p, [&](int i, uint32_t &c, double &m) {
                c = counts[CHUNK - 1 - i];
                m = c ? c * weight(chunk * CHUNK + CHUNK - 1 - i) : 0.0;
            });
            const int item = CHUNK - 1 - max(p.item, 0);
            Number found;
            found.value = number_of<DTYPE>((uint32_t)(chunk * CHUNK + item));
            found.have = counts[item];
            found.before = p.count;
            found.mass = p.mass;
            found.weight = weight(chunk * CHUNK + item);
            found.choose(target);
            return found;
        };
        Number drawn;
        uint32_t n;
        double total;
        decide(job, job.uniforms[row], counted + low, counted, all, within, find, drawn, n, total);
        if (lane == 0) {
            if (rank == 0) {
                job.logp[row] = (float)(((double)drawn.value - top) * per_nat - log(total));
                if (job.kept) job.kept[row] = (int32_t)n;
            }
            sh.drawn = drawn;
        }
    }
    __syncthreads();
    const Number drawn = sh.drawn;
    // bits to look for; the zeros are one number
    const uint32_t bits = drawn.value == 0.0f ? 0u : Storage<DTYPE>::put(drawn.value);
    const uint32_t mask = bits ? 0xffffu : 0x7fffu, both = bits * 0x10001u, masks = mask * 0x10001u;
    uint32_t skip = 0, have = drawn.have;
    if (ctas > 1) {
        // how many of them each piece holds: the other CTAs' bins still tell; the owner's own are what is left of the sum
        const uint32_t key = bits & 0x8000u ? 0xffffu - bits : bits | 0x8000u, bin = key - F::BASE;
        const int chunk = (int)bin / CHUNK;
        int owner = 0;
        while (C::CHUNKS * (owner + 1) / ctas <= chunk) ++owner;
        uint32_t others = 0, mine = 0, before = 0;
        for (int r = 0; r < ctas; ++r) {
            if (r == owner) continue;
            const uint16_t *counts = reinterpret_cast<const uint16_t *>(cluster.map_shared_rank(sample_smem, r));
            const uint32_t c = counts[bin] + (bin == F::ZERO ? counts[bin - 1] : 0u);
            others += c;
            if (r < rank) before += c;
            if (r == rank) mine = c;
        }
        if (owner == rank) mine = drawn.have - others;
        if (owner < rank) before += drawn.have - others;
        skip = before;
        have = mine;
    }
    if (drawn.rank >= skip && drawn.rank - skip < have)
        locate(piece, drawn.rank - skip, sh, job.tokens + row, [&](const uint4 &w) {
            const uint32_t x = (w.x & masks) ^ both, y = (w.y & masks) ^ both, z = (w.z & masks) ^ both, v = (w.w & masks) ^ both;
            uint32_t m = 0;
            m |= (x & 0xffffu) ? 0u : 1u;
            m |= (x >> 16) ? 0u : 2u;
            m |= (y & 0xffffu) ? 0u : 4u;
            m |= (y >> 16) ? 0u : 8u;
            m |= (z & 0xffffu) ? 0u : 16u;
            m |= (z >> 16) ? 0u : 32u;
            m |= (v & 0xffffu) ? 0u : 64u;
            m |= (v >> 16) ? 0u : 128u;
            return m;
        });
    if (ctas > 1) cluster.sync();            // no CTA leaves while another still reads its shared memory
}

// ---- host side --------------------------------------------------------------------------------------
namespace {

template <auto kernel>
bool sample_launch(size_t smem, int per_sm, const SampleJob &job, int32_t units, cudaStream_t stream)
{
    static std::atomic<bool> ready[DEVICES];
    int dev = 0;
    if (cudaGetDevice(&dev) != cudaSuccess || dev < 0 || dev >= DEVICES) return false;
    if (!ready[dev].load(std::memory_order_relaxed)) {
        if (cudaFuncSetAttribute(kernel, cudaFuncAttributeMaxDynamicSharedMemorySize, (int)smem) != cudaSuccess) return false;
        ready[dev].store(true, std::memory_order_relaxed);
    }
    // As many CTAs to a row as keep the device's places filled, each with 512 units or more.
    int ctas = 1;
    while (ctas < SAMPLE_CTAS && (int64_t)job.R * ctas * 2 <= 148 * per_sm && units / (ctas * 2) >= 512) ctas *= 2;
    cudaLaunchConfig_t config = {};
    config.gridDim = dim3((unsigned)(job.R * ctas));
    config.blockDim = dim3(SAMPLE_THREADS);
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
    if (!(params->temperature >= 1e-300 && params->temperature <= 1e300) || params->top_k < 0 || !(params->top_p > 0.0 && params->top_p <= 1.0) ||
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
    const bool ok = params->dtype == PPOW_F32    ? sample_launch<sample_search_kernel>(sizeof(SearchBins), 4, job, units, stream)
                    : params->dtype == PPOW_BF16 ? sample_launch<sample_count_kernel<PPOW_BF16>>(Counted<PPOW_BF16>::BINS * 2, 2, job, units, stream)
                                                 : sample_launch<sample_count_kernel<PPOW_F16>>(Counted<PPOW_F16>::BINS * 2, 2, job, units, stream);
    return ok ? PPOW_OK : PPOW_ERR_CUDA;
}
