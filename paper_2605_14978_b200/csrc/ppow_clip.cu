// Global norm of many gradients, and clipping: what a training step does between its gradients and the optimizer.
//
//   norm = sqrt(sum over all tensors of g^2),   factor = min(1, max_norm / norm),   out = round(g * factor)
//
// Two passes over the gradients, bound by memory.  A CTA owns a run of neighbouring chunks (32 KB each) of all tensors laid end to end; the second pass
// takes each run from its end, so that it starts with what the first pass read last and the L2 cache still holds.  The table of
// tensors travels as a kernel argument: no copy to the device, and a captured graph holds it.
//
// A thread's squares of a chunk, 64 of 16-bit types or 32 of float32, are added in float32, as four chains of 16 or 8 that are then joined,
// and from there on in float64.  In float64 from the start, where their float32 sum lies outside the range in which float32 squares
// are good (overflow, or below 2^-96, where squares of 2^-63 and less have lost bits).  The norm is right to 10 half steps of float32.
#include "ppow_checked.cuh"
#include "ppow_rows.cuh"

#include <algorithm>
#include <new>

namespace ppow {

constexpr int CLIP_THREADS = 256, CLIP_UNITS = 8;                  // 16-byte units of a chunk that a thread takes
constexpr int64_t CLIP_CHUNK = CLIP_THREADS * CLIP_UNITS;
// CTAs of a launch, each of which leaves a share of the sum: 148 SMs x 6.  Not by the device's own number, so that the order of the
// sum goes by the tensors alone.
constexpr int CLIP_SHARES = 148 * 6;

struct ClipEntry {
    const void *grad;
    void *out;
    int64_t size;            // elements
};
// Tensors of a launch.  Three sizes of table, for it is copied at every launch; the longest is just below the limit of kernel arguments
// (32764 bytes).
template <int N> struct ClipTable {
    static constexpr int MOST = N;
    ClipEntry at[N];
    int32_t chunk_end[N];    // chunks of this tensor and those before it
    uint8_t dtype[N];
    int32_t n, chunks;
};
using ShortTable = ClipTable<48>;
using MiddleTable = ClipTable<256>;
using LongTable = ClipTable<1024>;
static_assert(sizeof(LongTable) + 64 <= 32764, "kernel arguments");

// A tensor as 16-byte units from the aligned address at or below its start; the first and last may be partly its own.
template <int DTYPE> struct ClipSpan {
    using S = Storage<DTYPE>;
    using T = typename S::type;
    static constexpr int E = S::PER_UNIT;
    const uint4 *base;
    int32_t head;            // elements of unit 0 that lie before the tensor
    int64_t span, units;
    __device__ __forceinline__ ClipSpan(const void *p, int64_t size)
    {
        const uintptr_t a = reinterpret_cast<uintptr_t>(p);
        base = reinterpret_cast<const uint4 *>(a & ~(uintptr_t)15);
        head = (int32_t)((a & 15) / sizeof(T));
        span = head + size;
        units = (span + E - 1) / E;
    }
    // elements [lo, hi) of unit u are the tensor's
    __device__ __forceinline__ int lo(int64_t u) const { return u == 0 ? head : 0; }
    __device__ __forceinline__ int hi(int64_t u) const { return (int)min((int64_t)E, span - u * E); }
    __device__ __forceinline__ uint4 edge(int64_t u) const         // a unit at an end: element by element, zeros around
    {
        float f[E];
        const T *p = reinterpret_cast<const T *>(base + u);
#pragma unroll
        for (int e = 0; e < E; ++e) f[e] = e >= lo(u) && e < hi(u) ? S::get(p[e]) : 0.0f;
        return S::pack(f);
    }
    __device__ __forceinline__ bool whole(int64_t u) const { return lo(u) == 0 && hi(u) == E; }
};

// Sum of the squares of N units, in float64.  load(k): the k-th of them, asked again where float32 does not do.
template <int DTYPE, int N, typename Load> __device__ __forceinline__ double squares_of(const uint4 (&raw)[N], Load &&load)
{
    using S = Storage<DTYPE>;
    constexpr int E = S::PER_UNIT;
    float2 acc[2] = {make_float2(0.0f, 0.0f), make_float2(0.0f, 0.0f)};
    uint32_t any = 0;
#pragma unroll
    for (int k = 0; k < N; ++k) {
        float f[E];
        S::unpack(raw[k], f);
#pragma unroll
        for (int e = 0; e < E; e += 2) {
            const float2 v = make_float2(f[e], f[e + 1]);
            acc[(e / 2) & 1] = __ffma2_rn(v, v, acc[(e / 2) & 1]);
        }
        any |= raw[k].x | raw[k].y | raw[k].z | raw[k].w;
    }
    const float sum = (acc[0].x + acc[0].y) + (acc[1].x + acc[1].y);
    if (sum >= 0x1p-96f && sum < INFINITY) return (double)sum;
    // nothing but zeros is common (rows without a gradient)
    if ((any & (DTYPE == PPOW_F32 ? 0x7fffffffu : 0x7fff7fffu)) == 0) return 0.0;
    double exact = 0.0;
#pragma unroll 1
    for (int k = 0; k < N; ++k) {
        float f[E];
        S::unpack(load(k), f);
#pragma unroll
        for (int e = 0; e < E; ++e) exact = fma((double)f[e], (double)f[e], exact);
    }
    return exact;
}

__device__ __forceinline__ double cta_sum(double v)
{
    __shared__ double warps[CLIP_THREADS / 32];
    v = warp_sum_f64(v);
    if ((threadIdx.x & 31) == 0) warps[threadIdx.x >> 5] = v;
    __syncthreads();
    v = 0.0;
#pragma unroll
    for (int i = 0; i < CLIP_THREADS / 32; ++i) v += warps[i];
    return v;
}

// The tensor that holds chunk c (entries are never empty).
template <typename Table> __device__ __forceinline__ int tensor_of(const Table &table, int32_t c)
{
    int lo = 0, hi = table.n - 1;
    while (lo < hi) {
        const int mid = (lo + hi) / 2;
        if (table.chunk_end[mid] > c) hi = mid; else lo = mid + 1;
    }
    return lo;
}

template <int DTYPE> __device__ __forceinline__ double chunk_squares(const ClipEntry &entry, int64_t chunk)
{
    const ClipSpan<DTYPE> span(entry.grad, entry.size);
    const int64_t u0 = chunk * CLIP_CHUNK + threadIdx.x;
    auto load = [&](int k) {
        const int64_t u = u0 + k * CLIP_THREADS;
        return u >= span.units ? make_uint4(0, 0, 0, 0) : span.whole(u) ? span.base[u] : span.edge(u);
    };
    uint4 raw[CLIP_UNITS];
    if (chunk > 0 && (chunk + 1) * CLIP_CHUNK < span.units) {      // no unit at an end
#pragma unroll
        for (int k = 0; k < CLIP_UNITS; ++k) raw[k] = span.base[u0 + k * CLIP_THREADS];
    } else {
#pragma unroll
        for (int k = 0; k < CLIP_UNITS; ++k) raw[k] = load(k);
    }
    return squares_of<DTYPE>(raw, load);
}

template <typename Table>
__global__ void __launch_bounds__(CLIP_THREADS, 4) clip_norm_kernel(const __grid_constant__ Table table, double *__restrict__ shares)
{
    wait_for_previous_kernel();
    const int32_t first = (int32_t)((int64_t)table.chunks * blockIdx.x / gridDim.x), last = (int32_t)((int64_t)table.chunks * (blockIdx.x + 1) / gridDim.x);
    int i = tensor_of(table, first);
    double sum = 0.0;
    for (int32_t c = first; c < last; ++c) {
        while (table.chunk_end[i] <= c) ++i;
        if (!PPOW_CHECK(i < table.n, 901, nullptr)) return;
        const int64_t chunk = c - (i ? table.chunk_end[i - 1] : 0);
        const int dtype = table.dtype[i];
        sum += dtype == PPOW_F32    ? chunk_squares<PPOW_F32>(table.at[i], chunk)
               : dtype == PPOW_BF16 ? chunk_squares<PPOW_BF16>(table.at[i], chunk)
                                    : chunk_squares<PPOW_F16>(table.at[i], chunk);
    }
    sum = cta_sum(sum);
    if (threadIdx.x == 0) shares[blockIdx.x] = sum;
}

// A factor as a power of two and the rest.  Below 2^-100 float32 has no bits for it, or soon not, and the product may still be an ordinary
// number (1e35 clipped to 1e-5): the power of two takes 2^-100 of the exponent away.  The first product is exact, or so small that
// nothing is left after the second.  Loops of their own for the two, the rare one a unit at a time: with both products in one loop all calls
// pay (743 M bf16: 717 us, so 709), and with more than 128 registers one CTA is left on an SM (791 us).
struct ClipFactor {
    float power = 1.0f, rest = 1.0f;
    __device__ __forceinline__ bool small() const { return power != 1.0f; }
    __device__ __forceinline__ explicit ClipFactor(double factor)
    {
        if (factor > 0.0 && factor < 0x1p-100) power = ldexpf(1.0f, max(ilogb(factor) + 100, -149));
        rest = (float)(factor / power);
    }
};

template <int DTYPE, bool SMALL>
__device__ __forceinline__ void scale_unit(typename Storage<DTYPE>::type *out, const uint4 &raw, const ClipFactor &factor, int lo, int hi)
{
    using S = Storage<DTYPE>;
    constexpr int E = S::PER_UNIT;
    float f[E];
    S::unpack(raw, f);
#pragma unroll
    for (int e = 0; e < E; ++e) f[e] = SMALL ? f[e] * factor.power * factor.rest : f[e] * factor.rest;
    if (lo == 0 && hi == E && (uintptr_t)out % 16 == 0) {
        __stcs(reinterpret_cast<uint4 *>(out), S::pack(f));
    } else {
#pragma unroll
        for (int e = 0; e < E; ++e)
            if (e >= lo && e < hi) out[e] = S::put(f[e]);
    }
}

template <int DTYPE, bool SMALL> __device__ __forceinline__ void chunk_scale(const ClipEntry &entry, int64_t chunk, const ClipFactor &factor)
{
    using T = typename Storage<DTYPE>::type;
    constexpr int E = Storage<DTYPE>::PER_UNIT;
    const ClipSpan<DTYPE> span(entry.grad, entry.size);
    T *out = static_cast<T *>(entry.out) - span.head;              // where unit 0 begins on the other side
    const int64_t u0 = chunk * CLIP_CHUNK + threadIdx.x;
    uint4 raw[CLIP_UNITS];
    if (SMALL) {
#pragma unroll 1
        for (int k = 0; k < CLIP_UNITS; ++k) {
            const int64_t u = u0 + k * CLIP_THREADS;
            if (u < span.units) scale_unit<DTYPE, SMALL>(out + u * E, span.whole(u) ? span.base[u] : span.edge(u), factor, span.lo(u), span.hi(u));
        }
    } else if (chunk > 0 && (chunk + 1) * CLIP_CHUNK < span.units) {
#pragma unroll
        for (int k = 0; k < CLIP_UNITS; ++k) raw[k] = __ldcs(span.base + u0 + k * CLIP_THREADS);
#pragma unroll
        for (int k = 0; k < CLIP_UNITS; ++k) scale_unit<DTYPE, SMALL>(out + (u0 + k * CLIP_THREADS) * E, raw[k], factor, 0, E);
    } else {
#pragma unroll
        for (int k = 0; k < CLIP_UNITS; ++k) {
            const int64_t u = u0 + k * CLIP_THREADS;
            if (u < span.units) raw[k] = span.whole(u) ? __ldcs(span.base + u) : span.edge(u);
        }
#pragma unroll
        for (int k = 0; k < CLIP_UNITS; ++k) {
            const int64_t u = u0 + k * CLIP_THREADS;
            if (u < span.units) scale_unit<DTYPE, SMALL>(out + u * E, raw[k], factor, span.lo(u), span.hi(u));
        }
    }
}

// A CTA's run of chunks, from its end.
template <bool SMALL, typename Table>
__device__ __forceinline__ void scale_run(const Table &table, int32_t first, int32_t last, const ClipFactor &factor)
{
    int i = tensor_of(table, last - 1);
    for (int32_t c = last - 1; c >= first; --c) {
        while (i > 0 && table.chunk_end[i - 1] > c) --i;
        if (!PPOW_CHECK(i < table.n && c < table.chunk_end[i], 902, nullptr)) return;
        const int64_t chunk = c - (i ? table.chunk_end[i - 1] : 0);
        const int dtype = table.dtype[i];
        if (dtype == PPOW_F32)
            chunk_scale<PPOW_F32, SMALL>(table.at[i], chunk, factor);
        else if (dtype == PPOW_BF16)
            chunk_scale<PPOW_BF16, SMALL>(table.at[i], chunk, factor);
        else
            chunk_scale<PPOW_F16, SMALL>(table.at[i], chunk, factor);
    }
}

// Every CTA adds up all shares, in one order.  in_place: gradients that need no clipping are already where they belong.
template <typename Table>
__global__ void __launch_bounds__(CLIP_THREADS, 2) clip_scale_kernel(const __grid_constant__ Table table, const double *__restrict__ shares, int32_t n_shares,
                                                                  double max_norm, bool in_place, float *__restrict__ norm_out)
{
    wait_for_previous_kernel();
    double sum = 0.0;
    for (int32_t s = threadIdx.x; s < n_shares; s += CLIP_THREADS) sum += shares[s];
    const double norm = sqrt(cta_sum(sum));
    if (blockIdx.x == 0 && threadIdx.x == 0 && norm_out) *norm_out = (float)norm;
    if (table.n == 0) return;
    const bool within = norm <= max_norm;                          // false for NaN, which then goes into every gradient
    if (within && in_place) return;
    const ClipFactor factor(within ? 1.0 : max_norm / norm);
    const int32_t first = (int32_t)((int64_t)table.chunks * blockIdx.x / gridDim.x), last = (int32_t)((int64_t)table.chunks * (blockIdx.x + 1) / gridDim.x);
    if (factor.small())
        scale_run<true>(table, first, last, factor);
    else
        scale_run<false>(table, first, last, factor);
}

// ---- host side --------------------------------------------------------------------------------------
namespace {

constexpr int32_t CLIP_MOST_TENSORS = 1 << 16;
constexpr int64_t CLIP_MOST_ELEMENTS = (int64_t)1 << 40;

int32_t chunks_of(const void *grad, int64_t size, size_t es)
{
    const int64_t bytes = (int64_t)((uintptr_t)grad % 16) + size * (int64_t)es;
    return (int32_t)((bytes + CLIP_CHUNK * 16 - 1) / (CLIP_CHUNK * 16));
}

struct Range {
    uintptr_t lo, hi;
    int32_t tensor;
    bool written;
};

// Whether something that is written overlaps anything but, at the same address, the gradient that it is made from.
// 0 no, 1 yes, -1 out of memory.
int overlaps(int32_t n, const void *const *grads, void *const *outs, const int64_t *sizes, const int32_t *dtypes)
{
    const bool in_place = std::equal(grads, grads + n, outs);
    Range *all = new (std::nothrow) Range[(size_t)2 * n + 1];
    if (!all) return -1;
    size_t m = 0;
    for (int32_t i = 0; i < n; ++i) {
        if (sizes[i] == 0) continue;
        const size_t bytes = (size_t)sizes[i] * bytes_of(dtypes[i]);
        all[m++] = {(uintptr_t)outs[i], (uintptr_t)outs[i] + bytes, i, true};
        if (!in_place && grads[i] != outs[i]) all[m++] = {(uintptr_t)grads[i], (uintptr_t)grads[i] + bytes, i, false};
    }
    auto before = [](const Range &a, const Range &b) { return a.lo < b.lo; };
    if (!std::is_sorted(all, all + m, before)) std::sort(all, all + m, before);
    uintptr_t written = 0, read = 0;                               // ends of what was seen so far
    int found = 0;
    for (size_t k = 0; k < m && !found; ++k) {
        found = all[k].lo < written || (all[k].written && all[k].lo < read);
        uintptr_t &end = all[k].written ? written : read;
        end = std::max(end, all[k].hi);
    }
    delete[] all;
    return found;
}

// One table after the other; `launch` gets each when it is full, and the last one.
template <typename Table, typename Launch>
bool each_table(int32_t n, const void *const *grads, void *const *outs, const int64_t *sizes, const int32_t *dtypes, Launch &&launch)
{
    Table table;
    table.n = table.chunks = 0;
    for (int32_t i = 0; i < n; ++i) {
        if (sizes[i] == 0) continue;
        const int32_t more = chunks_of(grads[i], sizes[i], bytes_of(dtypes[i]));
        if (table.n == Table::MOST || (int64_t)table.chunks + more > INT32_MAX) {
            if (!launch(table)) return false;
            table.n = table.chunks = 0;
        }
        table.at[table.n] = {grads[i], outs ? outs[i] : nullptr, sizes[i]};
        table.dtype[table.n] = (uint8_t)dtypes[i];
        table.chunks += more;
        table.chunk_end[table.n++] = table.chunks;
    }
    return table.n == 0 || launch(table);
}

template <typename Table>
bool clip_launch(int32_t n, const void *const *grads, void *const *outs, const int64_t *sizes, const int32_t *dtypes, double max_norm, bool in_place,
                 float *norm, double *shares, cudaStream_t stream)
{
    int32_t n_shares = 0;
    if (!each_table<Table>(n, grads, outs, sizes, dtypes, [&](const Table &t) {
            const int grid = std::min<int32_t>(t.chunks, CLIP_SHARES);
            const bool ok = launch_after(clip_norm_kernel<Table>, (unsigned)grid, CLIP_THREADS, 0, stream, t, shares + n_shares);
            n_shares += grid;
            return ok;
        }))
        return false;
    if (!outs || n_shares == 0) {                                  // the norm alone
        ShortTable none;
        none.n = none.chunks = 0;
        return launch_after(clip_scale_kernel<ShortTable>, 1, CLIP_THREADS, 0, stream, none, shares, n_shares, max_norm, false, norm);
    }
    float *to = norm;
    return each_table<Table>(n, grads, outs, sizes, dtypes, [&](const Table &t) {
        const int grid = std::min<int32_t>(t.chunks, CLIP_SHARES);
        const bool ok = launch_after(clip_scale_kernel<Table>, (unsigned)grid, CLIP_THREADS, 0, stream, t, shares, n_shares, max_norm, in_place, to);
        to = nullptr;
        return ok;
    });
}

}  // namespace
}  // namespace ppow

#ifdef PPOW_CHECKED
namespace ppow { int read_check_counters_clip(unsigned int *f, unsigned int *s) { return read_check_counters(f, s); } }
#endif

using namespace ppow;

// Shares of every launch that n tensors can take: one a table, and one more for each table that is closed early because its
// chunks would pass 31 bits.
extern "C" size_t ppow_clip_workspace_bytes(int32_t n)
{
    if (n < 0 || n > CLIP_MOST_TENSORS) return 0;
    return ((size_t)n / ShortTable::MOST + 2) * CLIP_SHARES * sizeof(double);
}

extern "C" ppow_status ppow_clip_gradients(int32_t n, const void *const *grads, void *const *out, const int64_t *sizes, const int32_t *dtypes,
                                           double max_norm, float *norm, void *workspace, size_t workspace_bytes, void *cuda_stream)
{
    if (n < 0 || n > CLIP_MOST_TENSORS || !norm || (uintptr_t)norm % 4 || (n > 0 && (!grads || !sizes || !dtypes))) return PPOW_ERR_INVALID_ARG;
    if (out && !(max_norm >= 0.0 && max_norm < INFINITY)) return PPOW_ERR_INVALID_ARG;
    int64_t total = 0;
    bool in_place = out != nullptr;
    for (int32_t i = 0; i < n; ++i) {
        if (sizes[i] < 0 || sizes[i] > CLIP_MOST_ELEMENTS || !dtype_ok(dtypes[i])) return PPOW_ERR_INVALID_ARG;
        if (sizes[i] == 0) continue;
        const size_t es = bytes_of(dtypes[i]);
        if (!grads[i] || (uintptr_t)grads[i] % es || (out && (!out[i] || (uintptr_t)out[i] % es))) return PPOW_ERR_INVALID_ARG;
        total += sizes[i];
        in_place = in_place && out[i] == grads[i];
        if (total > CLIP_MOST_ELEMENTS) return PPOW_ERR_INVALID_ARG;
    }
    if (!workspace || (uintptr_t)workspace % 256 || workspace_bytes < ppow_clip_workspace_bytes(n)) return PPOW_ERR_WORKSPACE;
    if (out && n > 0) {
        const int found = overlaps(n, grads, out, sizes, dtypes);
        if (found) return found < 0 ? PPOW_ERR_CUDA : PPOW_ERR_INVALID_ARG;
    }
    double *shares = static_cast<double *>(workspace);
    cudaStream_t stream = static_cast<cudaStream_t>(cuda_stream);
    return (n <= ShortTable::MOST    ? clip_launch<ShortTable>(n, grads, out, sizes, dtypes, max_norm, in_place, norm, shares, stream)
            : n <= MiddleTable::MOST ? clip_launch<MiddleTable>(n, grads, out, sizes, dtypes, max_norm, in_place, norm, shares, stream)
                                     : clip_launch<LongTable>(n, grads, out, sizes, dtypes, max_norm, in_place, norm, shares, stream))
               ? PPOW_OK
               : PPOW_ERR_CUDA;
}
