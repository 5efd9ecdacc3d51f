// Layer normalisation and its gradient, and 8-bit checkpoints of activations: what stands in front of the head in a
// training step, and how the norm's input is kept between the passes.
//
//   y = (x - mean) rstd w + b                     mean, 1/rstd^2 - eps: mean and variance of the row, float32
//   a = gy w,  xh = (x - mean) rstd
//   dx = rstd (a - mean(a) - xh mean(a xh)),      dw = sum_rows gy xh,   db = sum_rows gy
//
// Checkpoint: blocks of 128 along a row share a factor 2^e, e the smallest integer with max|x| <= 448 * 2^e (>= -126);
// values are x / 2^e rounded to nearest even in e4m3.  A power of two costs at most one bit of range against max/448 and
// makes the division exact, so each value is rounded once and any implementation gives the same bits.
//
// Bound by memory, the backward pass by what a warp has to wait for between two passes over a row: one row at a time is held in
// registers by one warp or one CTA, read once; the sums over rows (dw, db) stay in registers of the thread that owns the column,
// are written once per CTA and added up by a second kernel in an order that is fixed for a device and build.
#include "ppow_checked.cuh"
#include "ppow_rows.cuh"

namespace ppow {

// ---- forward ----------------------------------------------------------------------------------------
struct NormJob {
    const void *x;
    int64_t x_stride;
    const void *weight, *bias;
    int32_t R, D, param_dtype, blocks;
    float eps;
    void *y;
    float *mean, *rstd;
    uint8_t *codes, *scales;     // null: no checkpoint
};

// Rows in flight: about 16 to 64 KB of shared memory per CTA.
template <int DTYPE, int TPR> __host__ __device__ constexpr int forward_slots() { return TPR <= 128 ? 4 : TPR == 256 ? 3 : 2; }
template <int DTYPE, bool VEC, int TPR> __host__ __device__ constexpr int backward_slots()
{
    return !VEC || DTYPE == PPOW_F32 ? (VEC && TPR > 256 ? 1 : 2) : TPR <= 128 ? 4 : 2;
}

template <int DTYPE, bool VEC, int TPR>
__global__ void __launch_bounds__(norm_threads<TPR>()) norm_forward_kernel(const NormJob job)
{
    wait_for_previous_kernel();
    using DealT = Deal<DTYPE, VEC>;
    using T = typename DealT::T;
    constexpr int E = DealT::E, U = norm_units<DTYPE, VEC>(), S = forward_slots<DTYPE, TPR>();
    constexpr int ROWS = norm_threads<TPR>() / TPR, WARPS = TPR / 32;
    using Ahead = RowAhead<DTYPE, VEC, TPR, U, S>;
    extern __shared__ uint4 slots[];
    __shared__ float2 part[2][WARPS];                        // per warp: sum, sum of squares about the warp's own mean
    __shared__ float2 counts[WARPS];                         // values that a warp holds, and one over that
    const int t = threadIdx.x % TPR, lane = threadIdx.x & 31, group = threadIdx.x / TPR;
    const int32_t D = job.D, units = DealT::units(D);
    if (!PPOW_CHECK(units <= TPR * U, 601, nullptr)) return;
    float w[U][E], b[U][E];                                  // weight and bias of the thread's columns
    int32_t mine = 0;                                        // columns that this thread holds
#pragma unroll
    for (int k = 0; k < U; ++k)
#pragma unroll
        for (int e = 0; e < E; ++e) {
            const int32_t c = DealT::column(t + k * TPR, e);
            const bool has = t + k * TPR < units && c < D;
            mine += has;
            w[k][e] = has ? load_param(job.weight, job.param_dtype, c) : 0.0f;
            b[k][e] = has && job.bias ? load_param(job.bias, job.param_dtype, c) : 0.0f;
        }
    const float in_warp = (float)__reduce_add_sync(0xffffffffu, mine);
    const float inv_warp = in_warp > 0.0f ? 1.0f / in_warp : 0.0f, inv_d = 1.0f / (float)D;
    if (WARPS > 1) {
        if (lane == 0) counts[t >> 5] = make_float2(in_warp, inv_warp);
        __syncthreads();
    }

    const int64_t step = (int64_t)gridDim.x * ROWS, first = (int64_t)blockIdx.x * ROWS + group;
    const T *x = static_cast<const T *>(job.x);
    Ahead ahead(reinterpret_cast<uint8_t *>(slots) + group * Ahead::BYTES, t);
    constexpr int LEAD = VEC ? S - 1 : 1;                    // rows that are on their way when one is worked on
#pragma unroll
    for (int i = 0; i < LEAD; ++i) {
        if (first + i * step < job.R) ahead.start(i, x + (first + i * step) * job.x_stride, t, units, D);
        if (VEC) copy_commit();
    }
    int slot = 0, turn = 0;
    for (int64_t row = first; row < job.R; row += step, turn ^= 1) {
        ahead.take();
        {
            const int64_t next = row + LEAD * step;
            const int to = slot == 0 ? S - 1 : slot - 1;     // the slot of the row before
            if (next < job.R) ahead.start(to, x + next * job.x_stride, t, units, D);
            if (VEC) {
                copy_commit();
                copy_wait<LEAD>();
            }
        }
        float f[U][E];
        float2 sum2[U];                                      // a chain of additions per unit
#pragma unroll
        for (int k = 0; k < U; ++k) {
            if (t + k * TPR < units) {
                ahead.get(slot, k, f[k]);
            } else {
#pragma unroll
                for (int e = 0; e < E; ++e) f[k][e] = 0.0f;
            }
            sum2[k] = make_float2(f[k][0], f[k][1]);
#pragma unroll
            for (int e = 2; e < E; e += 2) sum2[k] = __fadd2_rn(sum2[k], make_float2(f[k][e], f[k][e + 1]));
        }
        // sum of the warp's values, then squares about their mean: no difference of large sums
        const float sum = warp_sum(total_of(sum2)), m = sum * inv_warp;
        const float2 minus_m = make_float2(-m, -m);
        float2 sq2[U];
#pragma unroll
        for (int k = 0; k < U; ++k) {
            sq2[k] = make_float2(0.0f, 0.0f);
#pragma unroll
            for (int e = 0; e < E; e += 2) {
                const float2 d = __fadd2_rn(make_float2(f[k][e], f[k][e + 1]), minus_m);
                if constexpr (VEC) {
                    if (t + k * TPR < units) sq2[k] = __ffma2_rn(d, d, sq2[k]);
                } else if (DealT::whole(t + k * TPR, D)) {
                    sq2[k] = __ffma2_rn(d, d, sq2[k]);
                } else {
                    const int32_t u = t + k * TPR;
                    const float2 in = make_float2(DealT::has(u, e, D) ? d.x : 0.0f, DealT::has(u, e + 1, D) ? d.y : 0.0f);
                    sq2[k] = __ffma2_rn(in, in, sq2[k]);
                }
            }
        }
        const float sq = warp_sum(total_of(sq2));
        float mean = m, squares = sq;
        if (WARPS > 1) {
            // squares about the row's mean: each warp's squares about its own, plus its count times the gap squared
            if (lane == 0) part[turn][t >> 5] = make_float2(sum, sq);
            __syncthreads();
            float total = 0.0f;
#pragma unroll
            for (int i = 0; i < WARPS; ++i) total += part[turn][i].x;
            mean = total * inv_d;
            squares = 0.0f;
#pragma unroll
            for (int i = 0; i < WARPS; ++i) {
                const float2 n = counts[i], p = part[turn][i];
                const float gap = fmaf(p.x, n.y, -mean);
                squares += fmaf(n.x * gap, gap, p.y);
            }
        }
        const float rstd = inverse_root(fmaf(squares, inv_d, job.eps));
        const float2 minus_mean = make_float2(-mean, -mean), r2 = make_float2(rstd, rstd);
        T *dst = static_cast<T *>(job.y) + row * D;
#pragma unroll
        for (int k = 0; k < U; ++k) {
            const int32_t u = t + k * TPR;
            if (u < units) {
                float y[E];
#pragma unroll
                for (int e = 0; e < E; e += 2) {
                    const float2 xh = __fmul2_rn(__fadd2_rn(make_float2(f[k][e], f[k][e + 1]), minus_mean), r2);
                    const float2 o = __ffma2_rn(xh, make_float2(w[k][e], w[k][e + 1]), make_float2(b[k][e], b[k][e + 1]));
                    y[e] = o.x, y[e + 1] = o.y;
                }
                DealT::store(dst, u, D, y);
            }
        }
        if (t == 0) {
            job.mean[row] = mean;
            job.rstd[row] = rstd;
        }
        if (job.codes) {
            pack_units<DealT, U>(f, t, TPR, units, D, job.codes + row * D, job.scales + row * job.blocks);
        }
        slot = slot == S - 1 ? 0 : slot + 1;
    }
}

// ---- backward ---------------------------------------------------------------------------------------
struct NormGradJob {
    const void *grad_y;
    int64_t grad_y_stride;
    const void *x;                       // null: the checkpoint
    int64_t x_stride;
    const uint8_t *codes, *scales;
    const void *weight;
    const float *mean, *rstd;
    int32_t R, D, param_dtype, blocks;
    void *grad_x;
    float *partial;                      // [CTAs][2][D]: shares of dw, then of db
};

// Two passes over a row's values, both from the thread's own copies: sums first, then dx.  The column sums of dw and db stay in
// the registers of the thread that owns the column.
template <int DTYPE, bool VEC, bool PACKED, int TPR>
__global__ void __launch_bounds__(norm_threads<TPR>()) norm_backward_kernel(const NormGradJob job)
{
    wait_for_previous_kernel();
    using DealT = Deal<DTYPE, VEC>;
    using T = typename DealT::T;
    constexpr int E = DealT::E, U = norm_units<DTYPE, VEC>(), S = backward_slots<DTYPE, VEC, TPR>();
    constexpr int ROWS = norm_threads<TPR>() / TPR, WARPS = TPR / 32;
    using Grads = RowAhead<DTYPE, VEC, TPR, U, S>;
    using Inputs = std::conditional_t<PACKED, CodesAhead<DTYPE, VEC, TPR, U, S>, RowAhead<DTYPE, VEC, TPR, U, S>>;
    extern __shared__ uint4 slots[];
    __shared__ float2 part[2][WARPS];
    const int t = threadIdx.x % TPR, lane = threadIdx.x & 31, group = threadIdx.x / TPR;
    const int32_t D = job.D, units = DealT::units(D);
    if (!PPOW_CHECK(units <= TPR * U, 602, nullptr)) return;
    const float inv_d = 1.0f / (float)D;
    float w[U][E];
    float2 dw[U][E / 2], db[U][E / 2];
#pragma unroll
    for (int k = 0; k < U; ++k)
#pragma unroll
        for (int e = 0; e < E; ++e) {
            const int32_t c = DealT::column(t + k * TPR, e);
            w[k][e] = t + k * TPR < units && c < D ? load_param(job.weight, job.param_dtype, c) : 0.0f;
            dw[k][e / 2] = db[k][e / 2] = make_float2(0.0f, 0.0f);
        }
    const int64_t step = (int64_t)gridDim.x * ROWS, first = (int64_t)blockIdx.x * ROWS + group;
    using Scalars = ScalarsAhead<DealT, PACKED, TPR, U, S>;
    uint8_t *own = reinterpret_cast<uint8_t *>(slots) + group * (Grads::BYTES + Inputs::BYTES + Scalars::BYTES);
    Grads grads(own, t);
    Inputs inputs(own + Grads::BYTES, t);
    Scalars scalars(own + Grads::BYTES + Inputs::BYTES, t);
    constexpr int LEAD = S - 1;
    auto start = [&](int slot, int64_t row) {
        if (row < job.R) {
            grads.start(slot, static_cast<const T *>(job.grad_y) + row * job.grad_y_stride, t, units, D);
            if constexpr (PACKED)
                inputs.start(slot, job.codes + row * D, t, units, D);
            else
                inputs.start(slot, static_cast<const T *>(job.x) + row * job.x_stride, t, units, D);
            scalars.start(slot, job.mean + row, job.rstd + row, job.scales + row * job.blocks, t, units);
        }
        copy_commit();
    };
#pragma unroll
    for (int i = 0; i < LEAD; ++i) start(i, first + i * step);
    int slot = 0, turn = 0;
    for (int64_t row = first; row < job.R; row += step, turn ^= 1) {
        grads.take();
        inputs.take();
        start(slot == 0 ? S - 1 : slot - 1, row + LEAD * step);          // S == 1: the row itself
        copy_wait<LEAD>();
        __syncwarp();
        const float mean = scalars.get(slot, 0), rstd = scalars.get(slot, 1);
        const float2 minus_mean = make_float2(-mean, -mean), r2 = make_float2(rstd, rstd);
        float scale[U];
#pragma unroll
        for (int k = 0; k < U; ++k) scale[k] = scalars.scale(slot, k, job.scales + row * job.blocks, t);
        float2 c1[U], c2[U];
#pragma unroll
        for (int k = 0; k < U; ++k) {
            c1[k] = c2[k] = make_float2(0.0f, 0.0f);
            if (t + k * TPR < units) {
                float g[E];
                float2 xc[E / 2];
                inputs.centred(slot, k, scale[k], minus_mean, xc);
                grads.get(slot, k, g);
#pragma unroll
                for (int e = 0; e < E; e += 2) {
                    // columns that do not exist have g = 0 and w = 0
                    const float2 xh = __fmul2_rn(xc[e / 2], r2);
                    const float2 gy = make_float2(g[e], g[e + 1]), a = __fmul2_rn(gy, make_float2(w[k][e], w[k][e + 1]));
                    c1[k] = __fadd2_rn(c1[k], a);
                    c2[k] = __ffma2_rn(a, xh, c2[k]);
                    dw[k][e / 2] = __ffma2_rn(gy, xh, dw[k][e / 2]);
                    db[k][e / 2] = __fadd2_rn(db[k][e / 2], gy);
                }
            }
        }
        float s1 = warp_sum(total_of(c1)), s2 = warp_sum(total_of(c2));
        if (WARPS > 1) {
            if (lane == 0) part[turn][t >> 5] = make_float2(s1, s2);
            __syncthreads();
            s1 = s2 = 0.0f;
#pragma unroll
            for (int i = 0; i < WARPS; ++i) {
                s1 += part[turn][i].x;
                s2 += part[turn][i].y;
            }
        } else {
            __syncwarp();                                    // the next row's start writes over scalars that all lanes have read by now
        }
        s1 *= -inv_d;
        s2 *= -inv_d;
        const float2 m1 = make_float2(s1, s1), m2 = make_float2(s2, s2);
        T *dst = static_cast<T *>(job.grad_x) + row * D;
#pragma unroll
        for (int k = 0; k < U; ++k) {
            const int32_t u = t + k * TPR;
            if (u < units) {
                float g[E], o[E];
                float2 xc[E / 2];
                inputs.centred(slot, k, scale[k], minus_mean, xc);
                grads.get(slot, k, g);
#pragma unroll
                for (int e = 0; e < E; e += 2) {
                    const float2 xh = __fmul2_rn(xc[e / 2], r2);
                    const float2 a = __ffma2_rn(make_float2(g[e], g[e + 1]), make_float2(w[k][e], w[k][e + 1]), m1);
                    const float2 d = __fmul2_rn(__ffma2_rn(xh, m2, a), r2);
                    o[e] = d.x, o[e + 1] = d.y;
                }
                DealT::store(dst, u, D, o);
            }
        }
        slot = slot == S - 1 ? 0 : slot + 1;
    }
    // this CTA's share of the column sums
    float *out = job.partial + (size_t)blockIdx.x * 2 * D;
    auto each_column = [&](auto &&f) {
#pragma unroll
        for (int k = 0; k < U; ++k)
#pragma unroll
            for (int e = 0; e < E; ++e) {
                const int32_t u = t + k * TPR, c = DealT::column(u, e);
                if (u < units && c < D) f(c, e & 1 ? dw[k][e / 2].y : dw[k][e / 2].x, e & 1 ? db[k][e / 2].y : db[k][e / 2].x);
            }
    };
    if constexpr (ROWS == 1) {
        each_column([&](int32_t c, float sw, float sb) {
            out[c] = sw;
            out[D + c] = sb;
        });
    } else {
        // several rows at a time: the groups add their sums up one after the other
        __shared__ float joint[2][TPR * norm_values<VEC>()];
        for (int s = 0; s < ROWS; ++s) {
            if (group == s)
                each_column([&](int32_t c, float sw, float sb) {
                    sw += s ? joint[0][c] : 0.0f;
                    sb += s ? joint[1][c] : 0.0f;
                    joint[0][c] = sw;
                    joint[1][c] = sb;
                    if (s == ROWS - 1) {
                        out[c] = sw;
                        out[D + c] = sb;
                    }
                });
            __syncthreads();
        }
    }
}

// Column sums of dw and db over the CTAs' shares.
__global__ void __launch_bounds__(32 * JOIN_GROUPS) norm_join_kernel(const float *__restrict__ partial, int32_t shares, int32_t D,
                                                                     int32_t param_dtype, void *grad_weight, void *grad_bias)
{
    const int32_t c = blockIdx.x * 32 + (threadIdx.x & 31);        // column of dw, then of db
    wait_for_previous_kernel();
    const float sum = column_total(partial, shares, 2 * D, c);
    if (threadIdx.x < 32 && c < 2 * D) {
        if (c < D) {
            if (grad_weight) store_param(grad_weight, param_dtype, c, sum);
        } else if (grad_bias) {
            store_param(grad_bias, param_dtype, c - D, sum);
        }
    }
}

// ---- pack, unpack: a warp takes chunks of 32 units ----------------------------------------------------
constexpr int PACK_THREADS = 256, PACK_CHUNKS = 4;      // chunks in flight per warp

struct PackJob {
    const void *x;
    int64_t x_stride;
    void *out;
    uint8_t *codes, *scales;
    int32_t R, D, blocks;
};

// Chunks of 32 units, row by row; a warp takes PACK_CHUNKS neighbours.  One division per warp.
struct ChunkWalk {
    int64_t row;
    int32_t chunk;
    __device__ __forceinline__ ChunkWalk(int64_t warp, int32_t per_row)
    {
        const int64_t first = warp * PACK_CHUNKS;
        row = first / per_row;
        chunk = (int32_t)(first - row * per_row);
    }
    __device__ __forceinline__ void step(int32_t per_row)
    {
        if (++chunk == per_row) {
            chunk = 0;
            ++row;
        }
    }
};

template <int DTYPE, bool VEC>
__global__ void __launch_bounds__(PACK_THREADS) pack_kernel(const PackJob job)
{
    wait_for_previous_kernel();
    using DealT = Deal<DTYPE, VEC>;
    using T = typename DealT::T;
    const int lane = threadIdx.x & 31;
    const int32_t units = DealT::units(job.D), per_row = (units + 31) / 32;
    ChunkWalk at((int64_t)blockIdx.x * (PACK_THREADS / 32) + (threadIdx.x >> 5), per_row);
    DealT x[PACK_CHUNKS];
    ChunkWalk ahead = at;
#pragma unroll
    for (int i = 0; i < PACK_CHUNKS; ++i, ahead.step(per_row)) {
        const int32_t u = ahead.chunk * 32 + lane;
        x[i].zero();
        if (ahead.row < job.R && u < units) x[i].load(static_cast<const T *>(job.x) + ahead.row * job.x_stride, u, job.D);
    }
    if (at.row < job.R && at.chunk + PACK_CHUNKS <= per_row && PPOW_CHECK(at.chunk >= 0, 605, nullptr)) {
        // all in one row: their maxima go through the lanes together
        float f[PACK_CHUNKS][DealT::E];
#pragma unroll
        for (int i = 0; i < PACK_CHUNKS; ++i) x[i].get(f[i]);
        pack_units<DealT, PACK_CHUNKS>(f, at.chunk * 32 + lane, 32, units, job.D, job.codes + at.row * job.D, job.scales + at.row * job.blocks);
        return;
    }
#pragma unroll
    for (int i = 0; i < PACK_CHUNKS; ++i, at.step(per_row)) {
        const int32_t u = at.chunk * 32 + lane;
        if (at.row >= job.R || !PPOW_CHECK(at.chunk < per_row, 603, nullptr)) return;
        float f[1][DealT::E];
        x[i].get(f[0]);
        pack_units<DealT, 1>(f, u, 0, units, job.D, job.codes + at.row * job.D, job.scales + at.row * job.blocks);
    }
}

template <int DTYPE, bool VEC>
__global__ void __launch_bounds__(PACK_THREADS) unpack_kernel(const PackJob job)
{
    wait_for_previous_kernel();
    using DealT = Deal<DTYPE, VEC>;
    using T = typename DealT::T;
    const int lane = threadIdx.x & 31;
    const int32_t units = DealT::units(job.D), per_row = (units + 31) / 32;
    ChunkWalk at((int64_t)blockIdx.x * (PACK_THREADS / 32) + (threadIdx.x >> 5), per_row), ahead = at;
    uint32_t q[PACK_CHUNKS][DealT::E / 2];
    uint8_t scale[PACK_CHUNKS];
#pragma unroll
    for (int i = 0; i < PACK_CHUNKS; ++i, ahead.step(per_row)) {
        const int32_t u = ahead.chunk * 32 + lane;
        if (ahead.row < job.R && u < units) {
            DealT::load_codes(job.codes + ahead.row * job.D, u, job.D, q[i]);
            scale[i] = job.scales[ahead.row * job.blocks + u / DealT::BLOCK_LANES];
        }
    }
#pragma unroll
    for (int i = 0; i < PACK_CHUNKS; ++i, at.step(per_row)) {
        const int32_t u = at.chunk * 32 + lane;
        if (at.row >= job.R || !PPOW_CHECK(at.chunk < per_row, 604, nullptr)) return;
        if (u < units) {
            float f[DealT::E];
#pragma unroll
            for (int e = 0; e < DealT::E / 2; ++e) {
                const float2 v = values_of(q[i][e], scale_down(scale[i]));
                f[2 * e] = v.x, f[2 * e + 1] = v.y;
            }
            DealT::store(static_cast<T *>(job.out) + at.row * job.D, u, job.D, f);
        }
    }
}

// ---- host side --------------------------------------------------------------------------------------
namespace {

// CTAs of the backward pass: each leaves one share of the column sums.  148 SMs x 2 to 4, and no more than the device keeps resident:
// the order of the sums is fixed for a device and a build of the kernel, not across them.
constexpr int32_t SHARES_MAX = 148 * 4;

template <int DTYPE, bool VEC, int TPR>
bool forward_launch(const NormJob &job, cudaStream_t stream)
{
    constexpr int THREADS = norm_threads<TPR>(), ROWS = THREADS / TPR;
    constexpr size_t SMEM = ROWS * RowAhead<DTYPE, VEC, TPR, norm_units<DTYPE, VEC>(), forward_slots<DTYPE, TPR>()>::BYTES;
    auto kernel = norm_forward_kernel<DTYPE, VEC, TPR>;
    static Resident known;
    const int64_t need = ((int64_t)job.R + ROWS - 1) / ROWS, most = resident_ctas(known, kernel, THREADS, SMEM);
    if (most < 1) return false;
    return launch_after(kernel, (unsigned)(need < most ? need : most), THREADS, SMEM, stream, job);
}

// The fewest threads that hold a row.
template <int DTYPE, bool VEC>
bool forward_shape(const NormJob &job, cudaStream_t stream)
{
    constexpr int HELD = norm_values<VEC>();
    if (job.D <= 32 * HELD) return forward_launch<DTYPE, VEC, 32>(job, stream);
    if (job.D <= 128 * HELD) return forward_launch<DTYPE, VEC, 128>(job, stream);
    if (job.D <= 256 * HELD) return forward_launch<DTYPE, VEC, 256>(job, stream);
    if (512 * HELD >= NORM_MAX_WIDTH || job.D <= 512 * HELD) return forward_launch<DTYPE, VEC, 512>(job, stream);
    return forward_launch<DTYPE, VEC, 512 * HELD >= NORM_MAX_WIDTH ? 512 : 1024>(job, stream);
}

template <int DTYPE, bool VEC, bool PACKED, int TPR>
bool backward_launch(const NormGradJob &job, int32_t *shares, cudaStream_t stream)
{
    constexpr int THREADS = norm_threads<TPR>(), ROWS = THREADS / TPR, U = norm_units<DTYPE, VEC>(), S = backward_slots<DTYPE, VEC, TPR>();
    constexpr size_t ROW = RowAhead<DTYPE, VEC, TPR, U, S>::BYTES;
    constexpr size_t SMEM = ROWS * (ROW + (PACKED ? CodesAhead<DTYPE, VEC, TPR, U, S>::BYTES : ROW) +
                                    ScalarsAhead<Deal<DTYPE, VEC>, PACKED, TPR, U, S>::BYTES);
    auto kernel = norm_backward_kernel<DTYPE, VEC, PACKED, TPR>;
    static Resident known;
    const int64_t most = resident_ctas(known, kernel, THREADS, SMEM);
    if (most < 1) return false;
    int64_t n = ((int64_t)job.R + ROWS - 1) / ROWS;
    if (n > most) n = most;
    if (n > SHARES_MAX) n = SHARES_MAX;
    *shares = (int32_t)n;
    return launch_after(kernel, (unsigned)n, THREADS, SMEM, stream, job);
}

template <int DTYPE, bool VEC, bool PACKED>
bool backward_shape(const NormGradJob &job, int32_t *shares, cudaStream_t stream)
{
    constexpr int HELD = norm_values<VEC>();
    if (job.D <= 32 * HELD) return backward_launch<DTYPE, VEC, PACKED, 32>(job, shares, stream);
    if (job.D <= 128 * HELD) return backward_launch<DTYPE, VEC, PACKED, 128>(job, shares, stream);
    if (job.D <= 256 * HELD) return backward_launch<DTYPE, VEC, PACKED, 256>(job, shares, stream);
    if (512 * HELD >= NORM_MAX_WIDTH || job.D <= 512 * HELD) return backward_launch<DTYPE, VEC, PACKED, 512>(job, shares, stream);
    return backward_launch<DTYPE, VEC, PACKED, 512 * HELD >= NORM_MAX_WIDTH ? 512 : 1024>(job, shares, stream);
}

template <int DTYPE, bool VEC>
bool pack_launch(const PackJob &job, bool unpack, cudaStream_t stream)
{
    const int32_t units = VEC ? job.D / (16 / (int32_t)bytes_of(DTYPE)) : (job.D + CKPT_BLOCK - 1) / CKPT_BLOCK * 32;
    const int64_t chunks = (int64_t)job.R * ((units + 31) / 32), per_cta = PACK_THREADS / 32 * PACK_CHUNKS;
    const unsigned grid = (unsigned)((chunks + per_cta - 1) / per_cta);
    return launch_after(unpack ? unpack_kernel<DTYPE, VEC> : pack_kernel<DTYPE, VEC>, grid, PACK_THREADS, 0, stream, job);
}

}  // namespace
}  // namespace ppow

#ifdef PPOW_CHECKED
namespace ppow { int read_check_counters_norm(unsigned int *f, unsigned int *s) { return read_check_counters(f, s); } }
#endif

using namespace ppow;

extern "C" ppow_status ppow_layer_norm(const ppow_norm_params *params, const void *x, int64_t x_stride, const void *weight,
                                       const void *bias, void *y, float *mean, float *rstd, uint8_t *packed, uint8_t *scale,
                                       void *cuda_stream)
{
    if (!norm_ok(params) || !stride_ok(x_stride, params->D)) return PPOW_ERR_INVALID_ARG;
    if (params->D > NORM_MAX_WIDTH) return PPOW_ERR_UNSUPPORTED;
    if (params->R == 0) return PPOW_OK;
    const size_t es = bytes_of(params->dtype), ps = bytes_of(params->param_dtype);
    if (!x || !weight || !y || !mean || !rstd || !packed != !scale) return PPOW_ERR_INVALID_ARG;
    if ((uintptr_t)x % es || (uintptr_t)y % es || (uintptr_t)weight % ps || (uintptr_t)bias % ps || (uintptr_t)mean % 4 || (uintptr_t)rstd % 4)
        return PPOW_ERR_INVALID_ARG;
    NormJob job = {x, x_stride, weight, bias, params->R, params->D, params->param_dtype, (params->D + CKPT_BLOCK - 1) / CKPT_BLOCK,
                   params->eps, y, mean, rstd, packed, scale};
    const bool vec = vec_ok(x, x_stride, params->D, es) && (uintptr_t)y % 16 == 0 && (uintptr_t)packed % 8 == 0;
#define PPOW_CALL(DT, VEC) forward_shape<DT, VEC>(job, (cudaStream_t)cuda_stream)
    return PPOW_BY_TYPE(params->dtype, vec, PPOW_CALL) ? PPOW_OK : PPOW_ERR_CUDA;
#undef PPOW_CALL
}

extern "C" size_t ppow_layer_norm_workspace_bytes(const ppow_norm_params *params)
{
    if (!norm_ok(params) || params->D > NORM_MAX_WIDTH) return 0;
    const int64_t shares = params->R < SHARES_MAX ? (params->R > 0 ? params->R : 1) : SHARES_MAX;
    return (size_t)shares * 2 * params->D * 4;
}

extern "C" ppow_status ppow_layer_norm_backward(const ppow_norm_params *params, const void *grad_y, int64_t grad_y_stride, const void *x,
                                                int64_t x_stride, const uint8_t *packed, const uint8_t *scale, const void *weight,
                                                const float *mean, const float *rstd, void *grad_x, void *grad_weight, void *grad_bias,
                                                void *workspace, size_t workspace_bytes, void *cuda_stream)
{
    if (!norm_ok(params) || !stride_ok(grad_y_stride, params->D)) return PPOW_ERR_INVALID_ARG;
    if (params->D > NORM_MAX_WIDTH) return PPOW_ERR_UNSUPPORTED;
    cudaStream_t stream = (cudaStream_t)cuda_stream;
    const size_t es = bytes_of(params->dtype), ps = bytes_of(params->param_dtype);
    if ((uintptr_t)grad_weight % ps || (uintptr_t)grad_bias % ps) return PPOW_ERR_INVALID_ARG;
    if (params->R == 0) {
        for (void *p : {grad_weight, grad_bias})
            if (p && cudaMemsetAsync(p, 0, (size_t)params->D * ps, stream) != cudaSuccess) return PPOW_ERR_CUDA;
        return PPOW_OK;
    }
    if (!grad_y || !weight || !mean || !rstd || !grad_x || !packed != !scale || !x == !packed) return PPOW_ERR_INVALID_ARG;
    if (x && !stride_ok(x_stride, params->D)) return PPOW_ERR_INVALID_ARG;
    if ((uintptr_t)grad_y % es || (uintptr_t)x % es || (uintptr_t)grad_x % es || (uintptr_t)weight % ps || (uintptr_t)mean % 4 ||
        (uintptr_t)rstd % 4)
        return PPOW_ERR_INVALID_ARG;
    if (!workspace || (uintptr_t)workspace % 256 || workspace_bytes < ppow_layer_norm_workspace_bytes(params)) return PPOW_ERR_WORKSPACE;
    NormGradJob job = {grad_y, grad_y_stride, x, x_stride, packed, scale, weight, mean, rstd, params->R, params->D, params->param_dtype,
                       (params->D + CKPT_BLOCK - 1) / CKPT_BLOCK, grad_x, (float *)workspace};
    const bool vec = vec_ok(grad_y, grad_y_stride, params->D, es) && (uintptr_t)grad_x % 16 == 0 &&
                     (x ? vec_ok(x, x_stride, params->D, es) : (uintptr_t)packed % 8 == 0);
    int32_t shares = 0;
#define PPOW_CALL(DT, VEC) (x ? backward_shape<DT, VEC, false>(job, &shares, stream) : backward_shape<DT, VEC, true>(job, &shares, stream))
    if (!PPOW_BY_TYPE(params->dtype, vec, PPOW_CALL)) return PPOW_ERR_CUDA;
#undef PPOW_CALL
    if (grad_weight || grad_bias) {
        if (!launch_after(norm_join_kernel, (unsigned)((2 * params->D + 31) / 32), 32 * JOIN_GROUPS, 0, stream, job.partial, shares, params->D,
                          params->param_dtype, grad_weight, grad_bias))
            return PPOW_ERR_CUDA;
    }
    return PPOW_OK;
}

static bool pack_ok(int32_t R, int32_t D, int32_t dtype)
{
    return R >= 0 && R <= NORM_MAX_ROWS && D >= 1 && D <= (1 << 20) && (int64_t)R * ((D + 127) / 128) <= (int64_t)1 << 34 && dtype_ok(dtype);
}

extern "C" ppow_status ppow_pack_activation(const void *x, int64_t x_stride, int32_t R, int32_t D, int32_t dtype, uint8_t *packed,
                                            uint8_t *scale, void *cuda_stream)
{
    if (!pack_ok(R, D, dtype) || !stride_ok(x_stride, D)) return PPOW_ERR_INVALID_ARG;
    if (R == 0) return PPOW_OK;
    const size_t es = bytes_of(dtype);
    if (!x || !packed || !scale || (uintptr_t)x % es) return PPOW_ERR_INVALID_ARG;
    PackJob job = {x, x_stride, nullptr, packed, scale, R, D, (D + CKPT_BLOCK - 1) / CKPT_BLOCK};
    const bool vec = vec_ok(x, x_stride, D, es) && (uintptr_t)packed % 8 == 0;
#define PPOW_CALL(DT, VEC) pack_launch<DT, VEC>(job, false, (cudaStream_t)cuda_stream)
    return PPOW_BY_TYPE(dtype, vec, PPOW_CALL) ? PPOW_OK : PPOW_ERR_CUDA;
#undef PPOW_CALL
}

extern "C" ppow_status ppow_unpack_activation(const uint8_t *packed, const uint8_t *scale, int32_t R, int32_t D, int32_t dtype, void *x,
                                              void *cuda_stream)
{
    if (!pack_ok(R, D, dtype)) return PPOW_ERR_INVALID_ARG;
    if (R == 0) return PPOW_OK;
    const size_t es = bytes_of(dtype);
    if (!x || !packed || !scale || (uintptr_t)x % es) return PPOW_ERR_INVALID_ARG;
    PackJob job = {nullptr, 0, x, const_cast<uint8_t *>(packed), const_cast<uint8_t *>(scale), R, D, (D + CKPT_BLOCK - 1) / CKPT_BLOCK};
    const bool vec = vec_ok(x, D, D, es) && (uintptr_t)packed % 8 == 0;
#define PPOW_CALL(DT, VEC) pack_launch<DT, VEC>(job, true, (cudaStream_t)cuda_stream)
    return PPOW_BY_TYPE(dtype, vec, PPOW_CALL) ? PPOW_OK : PPOW_ERR_CUDA;
#undef PPOW_CALL
}
