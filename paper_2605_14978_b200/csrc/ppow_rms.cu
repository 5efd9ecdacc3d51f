// Root-mean-square norm with the residual's addition, and its gradient: the norm of the models whose drafters are trained here.
//
//   s = x + r, rounded to the storage type (without a residual s = x);  rstd = 1 / sqrt(mean(s^2) + eps);  y = s rstd w
//   a = gy w,  xh = s rstd
//   dx = rstd (a - xh mean(a xh)) + gs      (gs: what reaches s along the residual stream; dx is the gradient of x and of r alike)
//   dw = sum_rows gy xh
//
// The norm reads s as it is stored, so that the gradient, which has nothing else, is that of the forward pass.  y may leave in 8 bits,
// taken from its float32 values (one rounding), and s may be kept in 8 bits for the gradient.
//
// Bound by memory.  One row at a time is held in registers by a warp or a CTA and read once; dw stays in the registers of the
// thread that owns the column, is written once per CTA and added up by a second kernel in an order fixed for a device and build.
#include "ppow_checked.cuh"
#include "ppow_rows.cuh"

namespace ppow {

// Slots of rows in flight per CTA.  `bytes`: of one row in all its streams, times the rows that a CTA takes at a time.
//   many streams (x and residual; gradient, input and residual's gradient): one slot, the other CTAs' rows fill the wait.  16384 x 4096
//   bf16: forward 84 us with one slot, 95 with three; backward 91 with one, 99 with two
//   otherwise two at least, and what 40 KB hold.  8192 x 8192 bf16 without a residual: forward 44 us with two, 60 with one; backward 74 and 85
// Rows of a warp take more slots (16384 x 1024: 21.2 us with four, 22.4 with one), so do the widest (4096 x 16384: 42.6 us with three, 46.5
// with two); float32 rows, twice as long, what 56 KB hold.
template <int DTYPE, int TPR> __host__ __device__ constexpr int rms_slots(size_t bytes, bool many_streams)
{
    if (DTYPE == PPOW_F32 || TPR == 32) return 56 * 1024 / bytes >= 4 ? 4 : 56 * 1024 / bytes >= 1 ? (int)(56 * 1024 / bytes) : 1;
    if (many_streams) return 1;
    if (TPR == 512) return 112 * 1024 / bytes >= 3 ? 3 : 1;
    return 40 * 1024 / bytes >= 4 ? 4 : 40 * 1024 / bytes >= 2 ? (int)(40 * 1024 / bytes) : bytes <= 56 * 1024 ? 2 : 1;
}

// ---- forward ----------------------------------------------------------------------------------------
struct RmsJob {
    const void *x;
    int64_t x_stride;
    const void *residual;        // null: none
    int64_t residual_stride;
    const void *weight;
    int32_t R, D, param_dtype, blocks;
    float eps;
    void *sum;                   // s, written where there is a residual
    void *y;                     // null: y only in 8 bits
    float *rstd;
    uint8_t *y_codes, *y_scales; // null: y not in 8 bits
    uint8_t *codes, *scales;     // of s; null: no checkpoint
};

template <int DTYPE, bool VEC, bool RES, int TPR> struct RmsForward {
    using DealT = Deal<DTYPE, VEC>;
    static constexpr int U = norm_units<DTYPE, VEC>(), THREADS = norm_threads<TPR>(), ROWS = THREADS / TPR;
    static constexpr int S = rms_slots<DTYPE, TPR>((size_t)(RES ? 2 : 1) * U * THREADS * 16, RES);
    using Ahead = RowAhead<DTYPE, VEC, TPR, U, S>;
    static constexpr size_t SMEM = ROWS * (RES ? 2 : 1) * Ahead::BYTES;
};

template <int DTYPE, bool VEC, bool RES, int TPR>
__global__ void __launch_bounds__(norm_threads<TPR>()) rms_forward_kernel(const RmsJob job)
{
    wait_for_previous_kernel();
    using Shape = RmsForward<DTYPE, VEC, RES, TPR>;
    using DealT = typename Shape::DealT;
    using T = typename DealT::T;
    using St = Storage<DTYPE>;
    using Ahead = typename Shape::Ahead;
    constexpr int E = DealT::E, U = Shape::U, S = Shape::S, ROWS = Shape::ROWS, WARPS = TPR / 32;
    extern __shared__ uint4 slots[];
    __shared__ float part[2][WARPS];
    const int t = threadIdx.x % TPR, lane = threadIdx.x & 31, group = threadIdx.x / TPR;
    const int32_t D = job.D, units = DealT::units(D);
    if (!PPOW_CHECK(units <= TPR * U, 701, nullptr)) return;
    float w[U][E];
#pragma unroll
    for (int k = 0; k < U; ++k)
#pragma unroll
        for (int e = 0; e < E; ++e) {
            const int32_t c = DealT::column(t + k * TPR, e);
            w[k][e] = t + k * TPR < units && c < D ? load_param(job.weight, job.param_dtype, c) : 0.0f;
        }
    const float inv_d = 1.0f / (float)D;
    const int64_t step = (int64_t)gridDim.x * ROWS, first = (int64_t)blockIdx.x * ROWS + group;
    const T *x = static_cast<const T *>(job.x), *r = static_cast<const T *>(job.residual);
    uint8_t *own = reinterpret_cast<uint8_t *>(slots) + group * ((RES ? 2 : 1) * Ahead::BYTES);
    Ahead xs(own, t), rs(own + (RES ? Ahead::BYTES : 0), t);
    constexpr int LEAD = VEC ? S - 1 : 1;                    // rows that are on their way when one is worked on
    auto start = [&](int slot, int64_t row) {
        if (row < job.R) {
            xs.start(slot, x + row * job.x_stride, t, units, D);
            if constexpr (RES) rs.start(slot, r + row * job.residual_stride, t, units, D);
        }
        if (VEC) copy_commit();
    };
#pragma unroll
    for (int i = 0; i < LEAD; ++i) start(i, first + i * step);
    int slot = 0, turn = 0;
    for (int64_t row = first; row < job.R; row += step, turn ^= 1) {
        xs.take();
        if constexpr (RES) rs.take();
        start(slot == 0 ? S - 1 : slot - 1, row + LEAD * step);          // the slot of the row before; S == 1: the row itself
        if (VEC) copy_wait<LEAD>();
        float f[U][E];
        float2 sq2[U];                                       // a chain of additions per unit
        T *sum = static_cast<T *>(job.sum) + row * D;
#pragma unroll
        for (int k = 0; k < U; ++k) {
            const int32_t u = t + k * TPR;
            sq2[k] = make_float2(0.0f, 0.0f);
            if (u < units) {
                xs.get(slot, k, f[k]);
                if constexpr (RES) {
                    float g[E];
                    rs.get(slot, k, g);
#pragma unroll
                    for (int e = 0; e < E; e += 2) {
                        const float2 v = __fadd2_rn(make_float2(f[k][e], f[k][e + 1]), make_float2(g[e], g[e + 1]));
                        f[k][e] = St::get(St::put(v.x)), f[k][e + 1] = St::get(St::put(v.y));
                    }
                    DealT::store(sum, u, D, f[k]);
                }
#pragma unroll
                for (int e = 0; e < E; e += 2) {             // columns that do not exist were read as 0
                    const float2 v = make_float2(f[k][e], f[k][e + 1]);
                    sq2[k] = __ffma2_rn(v, v, sq2[k]);
                }
            } else {
#pragma unroll
                for (int e = 0; e < E; ++e) f[k][e] = 0.0f;
            }
        }
        float squares = warp_sum(total_of(sq2));
        if (WARPS > 1) {
            if (lane == 0) part[turn][t >> 5] = squares;
            __syncthreads();
            squares = 0.0f;
#pragma unroll
            for (int i = 0; i < WARPS; ++i) squares += part[turn][i];
        }
        const float rstd = inverse_root(fmaf(squares, inv_d, job.eps));
        if (t == 0) job.rstd[row] = rstd;
        if (job.codes) pack_units<DealT, U>(f, t, TPR, units, D, job.codes + row * D, job.scales + row * job.blocks);
        const float2 r2 = make_float2(rstd, rstd);
#pragma unroll
        for (int k = 0; k < U; ++k)
#pragma unroll
            for (int e = 0; e < E; e += 2) {
                const float2 v = __fmul2_rn(__fmul2_rn(make_float2(f[k][e], f[k][e + 1]), r2), make_float2(w[k][e], w[k][e + 1]));
                f[k][e] = v.x, f[k][e + 1] = v.y;
            }
        if (job.y) {
            T *dst = static_cast<T *>(job.y) + row * D;
#pragma unroll
            for (int k = 0; k < U; ++k)
                if (t + k * TPR < units) DealT::store(dst, t + k * TPR, D, f[k]);
        }
        if (job.y_codes) pack_units<DealT, U>(f, t, TPR, units, D, job.y_codes + row * D, job.y_scales + row * job.blocks);
        slot = slot == S - 1 ? 0 : slot + 1;
    }
}

// ---- backward ---------------------------------------------------------------------------------------
struct RmsGradJob {
    const void *grad_y;
    int64_t grad_y_stride;
    const void *grad_sum;                // null: nothing reaches s along the residual stream
    int64_t grad_sum_stride;
    const void *x;                       // s; null: its checkpoint
    int64_t x_stride;
    const uint8_t *codes, *scales;
    const void *weight;
    const float *rstd;
    int32_t R, D, param_dtype, blocks;
    void *grad_x;
    float *partial;                      // [CTAs][D]: shares of dw
};

template <int DTYPE, bool VEC, bool PACKED, bool RES, int TPR> struct RmsBackward {
    using DealT = Deal<DTYPE, VEC>;
    static constexpr int U = norm_units<DTYPE, VEC>(), THREADS = norm_threads<TPR>(), ROWS = THREADS / TPR;
    static constexpr size_t UNIT = (RES ? 32 : 16) + (PACKED ? DealT::E : 16);       // bytes of a unit in all streams
    static constexpr int S = VEC ? rms_slots<DTYPE, TPR>(UNIT * U * THREADS, RES && !PACKED) : 1;      // the scalar deal's rows sit in registers
    using Grads = RowAhead<DTYPE, VEC, TPR, U, S>;
    using Inputs = std::conditional_t<PACKED, CodesAhead<DTYPE, VEC, TPR, U, S>, RowAhead<DTYPE, VEC, TPR, U, S>>;
    using Scalars = ScalarsAhead<DealT, PACKED, TPR, U, S>;
    static constexpr size_t ROW = (RES ? 2 : 1) * Grads::BYTES + Inputs::BYTES + Scalars::BYTES;
    static constexpr size_t SMEM = ROWS * ROW;
};

// Blocks on an SM that registers have to leave room for.  Left to itself the compiler gives the scalar deal of an 8-bit input so many (for
// addresses of single bytes) that few warps are left: 8192 x 4095 with a residual 240 us, with two blocks 136.
template <bool VEC, bool PACKED, int TPR> __host__ __device__ constexpr int rms_blocks() { return VEC || !PACKED || TPR >= 512 ? 1 : TPR <= 128 ? 4 : 2; }

// Two passes over a row's values, both from the thread's own copies: sums first, then dx.
template <int DTYPE, bool VEC, bool PACKED, bool RES, int TPR>
__global__ void __launch_bounds__(norm_threads<TPR>(), rms_blocks<VEC, PACKED, TPR>()) rms_backward_kernel(const RmsGradJob job)
{
    wait_for_previous_kernel();
    using Shape = RmsBackward<DTYPE, VEC, PACKED, RES, TPR>;
    using DealT = typename Shape::DealT;
    using T = typename DealT::T;
    using Grads = typename Shape::Grads;
    using Inputs = typename Shape::Inputs;
    constexpr int E = DealT::E, U = Shape::U, S = Shape::S, ROWS = Shape::ROWS, WARPS = TPR / 32;
    extern __shared__ uint4 slots[];
    __shared__ float part[2][WARPS];
    const int t = threadIdx.x % TPR, lane = threadIdx.x & 31, group = threadIdx.x / TPR;
    const int32_t D = job.D, units = DealT::units(D);
    if (!PPOW_CHECK(units <= TPR * U, 702, nullptr)) return;
    const float inv_d = 1.0f / (float)D;
    float w[U][E];
    float2 dw[U][E / 2];
#pragma unroll
    for (int k = 0; k < U; ++k)
#pragma unroll
        for (int e = 0; e < E; ++e) {
            const int32_t c = DealT::column(t + k * TPR, e);
            w[k][e] = t + k * TPR < units && c < D ? load_param(job.weight, job.param_dtype, c) : 0.0f;
            dw[k][e / 2] = make_float2(0.0f, 0.0f);
        }
    const int64_t step = (int64_t)gridDim.x * ROWS, first = (int64_t)blockIdx.x * ROWS + group;
    uint8_t *own = reinterpret_cast<uint8_t *>(slots) + group * Shape::ROW;
    Grads grads(own, t), more(own + (RES ? Grads::BYTES : 0), t);
    own += (RES ? 2 : 1) * Grads::BYTES;
    Inputs inputs(own, t);
    typename Shape::Scalars scalars(own + Inputs::BYTES, t);
    constexpr int LEAD = S - 1;
    auto start = [&](int slot, int64_t row) {
        if (row < job.R) {
            grads.start(slot, static_cast<const T *>(job.grad_y) + row * job.grad_y_stride, t, units, D);
            if constexpr (PACKED)
                inputs.start(slot, job.codes + row * D, t, units, D);
            else
                inputs.start(slot, static_cast<const T *>(job.x) + row * job.x_stride, t, units, D);
            if constexpr (RES) more.start(slot, static_cast<const T *>(job.grad_sum) + row * job.grad_sum_stride, t, units, D);
            scalars.start(slot, job.rstd + row, job.rstd + row, job.scales + row * job.blocks, t, units);
        }
        copy_commit();
    };
#pragma unroll
    for (int i = 0; i < LEAD; ++i) start(i, first + i * step);
    int slot = 0, turn = 0;
    const float2 zero = make_float2(0.0f, 0.0f);
    for (int64_t row = first; row < job.R; row += step, turn ^= 1) {
        start(slot == 0 ? S - 1 : slot - 1, row + LEAD * step);          // S == 1: the row itself
        grads.take();
        inputs.take();
        if constexpr (RES) more.take();
        copy_wait<LEAD>();
        __syncwarp();
        const float rstd = scalars.get(slot, 1);
        const float2 r2 = make_float2(rstd, rstd);
        float scale[U];
#pragma unroll
        for (int k = 0; k < U; ++k) scale[k] = scalars.scale(slot, k, job.scales + row * job.blocks, t);
        float2 c2[U];
#pragma unroll
        for (int k = 0; k < U; ++k) {
            c2[k] = zero;
            if (t + k * TPR < units) {
                float g[E];
                float2 x[E / 2];
                inputs.centred(slot, k, scale[k], zero, x);
                grads.get(slot, k, g);
#pragma unroll
                for (int e = 0; e < E; e += 2) {
                    // columns that do not exist have g = 0 and w = 0
                    const float2 xh = __fmul2_rn(x[e / 2], r2);
                    const float2 gy = make_float2(g[e], g[e + 1]);
                    c2[k] = __ffma2_rn(__fmul2_rn(gy, make_float2(w[k][e], w[k][e + 1])), xh, c2[k]);
                    dw[k][e / 2] = __ffma2_rn(gy, xh, dw[k][e / 2]);
                }
            }
        }
        float s2 = warp_sum(total_of(c2));
        if (WARPS > 1) {
            if (lane == 0) part[turn][t >> 5] = s2;
            __syncthreads();
            s2 = 0.0f;
#pragma unroll
            for (int i = 0; i < WARPS; ++i) s2 += part[turn][i];
        } else {
            __syncwarp();                                    // the next row's start writes over scalars that all lanes have read by now
        }
        s2 *= -inv_d;
        const float2 m2 = make_float2(s2, s2);
        T *dst = static_cast<T *>(job.grad_x) + row * D;
#pragma unroll
        for (int k = 0; k < U; ++k) {
            const int32_t u = t + k * TPR;
            if (u < units) {
                float g[E], o[E], h[E];
                float2 x[E / 2];
                inputs.centred(slot, k, scale[k], zero, x);
                grads.get(slot, k, g);
                if constexpr (RES) more.get(slot, k, h);
#pragma unroll
                for (int e = 0; e < E; e += 2) {
                    const float2 xh = __fmul2_rn(x[e / 2], r2);
                    const float2 a = __fmul2_rn(make_float2(g[e], g[e + 1]), make_float2(w[k][e], w[k][e + 1]));
                    float2 d = __ffma2_rn(xh, m2, a);
                    if constexpr (RES)
                        d = __ffma2_rn(d, r2, make_float2(h[e], h[e + 1]));
                    else
                        d = __fmul2_rn(d, r2);
                    o[e] = d.x, o[e + 1] = d.y;
                }
                DealT::store(dst, u, D, o);
            }
        }
        slot = slot == S - 1 ? 0 : slot + 1;
    }
    // this CTA's share of the column sums
    float *out = job.partial + (size_t)blockIdx.x * D;
    auto each_column = [&](auto &&f) {
#pragma unroll
        for (int k = 0; k < U; ++k)
#pragma unroll
            for (int e = 0; e < E; ++e) {
                const int32_t u = t + k * TPR, c = DealT::column(u, e);
                if (u < units && c < D) f(c, e & 1 ? dw[k][e / 2].y : dw[k][e / 2].x);
            }
    };
    if constexpr (ROWS == 1) {
        each_column([&](int32_t c, float v) { out[c] = v; });
    } else {
        // several rows at a time: the groups add their sums up one after the other
        __shared__ float joint[TPR * norm_values<VEC>()];
        for (int s = 0; s < ROWS; ++s) {
            if (group == s)
                each_column([&](int32_t c, float v) {
                    v += s ? joint[c] : 0.0f;
                    joint[c] = v;
                    if (s == ROWS - 1) out[c] = v;
                });
            __syncthreads();
        }
    }
}

__global__ void __launch_bounds__(32 * JOIN_GROUPS) rms_join_kernel(const float *__restrict__ partial, int32_t shares, int32_t D,
                                                                    int32_t param_dtype, void *grad_weight)
{
    const int32_t c = blockIdx.x * 32 + (threadIdx.x & 31);
    wait_for_previous_kernel();
    const float sum = column_total(partial, shares, D, c);
    if (threadIdx.x < 32 && c < D) store_param(grad_weight, param_dtype, c, sum);
}

// ---- host side --------------------------------------------------------------------------------------
namespace {

// Shares of the column sums: 148 SMs x up to 6 CTAs, and no more than the device keeps resident.
constexpr int32_t RMS_SHARES_MAX = 148 * 6;

template <int DTYPE, bool VEC, bool RES, int TPR>
bool rms_forward_launch(const RmsJob &job, cudaStream_t stream)
{
    using Shape = RmsForward<DTYPE, VEC, RES, TPR>;
    auto kernel = rms_forward_kernel<DTYPE, VEC, RES, TPR>;
    static Resident known;
    const int64_t need = ((int64_t)job.R + Shape::ROWS - 1) / Shape::ROWS, most = resident_ctas(known, kernel, Shape::THREADS, Shape::SMEM);
    if (most < 1) return false;
    return launch_after(kernel, (unsigned)(need < most ? need : most), Shape::THREADS, Shape::SMEM, stream, job);
}

template <int DTYPE, bool VEC, bool PACKED, bool RES, int TPR>
bool rms_backward_launch(const RmsGradJob &job, int32_t *shares, cudaStream_t stream)
{
    using Shape = RmsBackward<DTYPE, VEC, PACKED, RES, TPR>;
    auto kernel = rms_backward_kernel<DTYPE, VEC, PACKED, RES, TPR>;
    static Resident known;
    const int64_t most = resident_ctas(known, kernel, Shape::THREADS, Shape::SMEM);
    if (most < 1) return false;
    int64_t n = ((int64_t)job.R + Shape::ROWS - 1) / Shape::ROWS;
    if (n > most) n = most;
    if (n > RMS_SHARES_MAX) n = RMS_SHARES_MAX;
    *shares = (int32_t)n;
    return launch_after(kernel, (unsigned)n, Shape::THREADS, Shape::SMEM, stream, job);
}

// The fewest threads that hold a row.
template <typename Launch> bool by_width(int32_t D, int32_t held, Launch &&launch)
{
    return D <= 32 * held    ? launch(std::integral_constant<int, 32>())
           : D <= 128 * held ? launch(std::integral_constant<int, 128>())
           : D <= 256 * held ? launch(std::integral_constant<int, 256>())
           : D <= 512 * held ? launch(std::integral_constant<int, 512>())
                             : launch(std::integral_constant<int, 1024>());
}

template <int DTYPE, bool VEC> bool rms_forward(const RmsJob &job, cudaStream_t stream)
{
    return by_width(job.D, norm_values<VEC>(), [&](auto tpr) {
        constexpr int TPR = VEC && tpr() == 1024 ? 512 : tpr();          // 512 threads hold the widest row of whole units
        return job.residual ? rms_forward_launch<DTYPE, VEC, true, TPR>(job, stream) : rms_forward_launch<DTYPE, VEC, false, TPR>(job, stream);
    });
}

template <int DTYPE, bool VEC> bool rms_backward(const RmsGradJob &job, int32_t *shares, cudaStream_t stream)
{
    return by_width(job.D, norm_values<VEC>(), [&](auto tpr) {
        constexpr int TPR = VEC && tpr() == 1024 ? 512 : tpr();
        if (job.x)
            return job.grad_sum ? rms_backward_launch<DTYPE, VEC, false, true, TPR>(job, shares, stream)
                                : rms_backward_launch<DTYPE, VEC, false, false, TPR>(job, shares, stream);
        return job.grad_sum ? rms_backward_launch<DTYPE, VEC, true, true, TPR>(job, shares, stream)
                            : rms_backward_launch<DTYPE, VEC, true, false, TPR>(job, shares, stream);
    });
}

}  // namespace
}  // namespace ppow

#ifdef PPOW_CHECKED
namespace ppow { int read_check_counters_rms(unsigned int *f, unsigned int *s) { return read_check_counters(f, s); } }
#endif

using namespace ppow;

extern "C" ppow_status ppow_rms_norm(const ppow_norm_params *params, const void *x, int64_t x_stride, const void *residual,
                                     int64_t residual_stride, const void *weight, void *sum, void *y, float *rstd, uint8_t *y_packed,
                                     uint8_t *y_scale, uint8_t *packed, uint8_t *scale, void *cuda_stream)
{
    if (!norm_ok(params) || !stride_ok(x_stride, params->D) || (residual && !stride_ok(residual_stride, params->D))) return PPOW_ERR_INVALID_ARG;
    if (params->D > NORM_MAX_WIDTH) return PPOW_ERR_UNSUPPORTED;
    if (params->R == 0) return PPOW_OK;
    const size_t es = bytes_of(params->dtype), ps = bytes_of(params->param_dtype);
    if (!x || !weight || !rstd || !residual != !sum || (!y && !y_packed) || !y_packed != !y_scale || !packed != !scale) return PPOW_ERR_INVALID_ARG;
    if ((uintptr_t)x % es || (uintptr_t)residual % es || (uintptr_t)sum % es || (uintptr_t)y % es || (uintptr_t)weight % ps || (uintptr_t)rstd % 4)
        return PPOW_ERR_INVALID_ARG;
    const RmsJob job = {x, x_stride, residual, residual_stride, weight, params->R, params->D, params->param_dtype,
                        (params->D + CKPT_BLOCK - 1) / CKPT_BLOCK, params->eps, sum, y, rstd, y_packed, y_scale, packed, scale};
    const bool vec = vec_ok(x, x_stride, params->D, es) && (!residual || vec_ok(residual, residual_stride, params->D, es)) &&
                     (uintptr_t)sum % 16 == 0 && (uintptr_t)y % 16 == 0 && (uintptr_t)y_packed % 8 == 0 && (uintptr_t)packed % 8 == 0;
#define PPOW_CALL(DT, VEC) rms_forward<DT, VEC>(job, (cudaStream_t)cuda_stream)
    return PPOW_BY_TYPE(params->dtype, vec, PPOW_CALL) ? PPOW_OK : PPOW_ERR_CUDA;
#undef PPOW_CALL
}

extern "C" size_t ppow_rms_norm_workspace_bytes(const ppow_norm_params *params)
{
    if (!norm_ok(params) || params->D > NORM_MAX_WIDTH) return 0;
    const int64_t shares = params->R < RMS_SHARES_MAX ? (params->R > 0 ? params->R : 1) : RMS_SHARES_MAX;
    return (size_t)shares * params->D * 4;
}

extern "C" ppow_status ppow_rms_norm_backward(const ppow_norm_params *params, const void *grad_y, int64_t grad_y_stride, const void *grad_sum,
                                              int64_t grad_sum_stride, const void *x, int64_t x_stride, const uint8_t *packed,
                                              const uint8_t *scale, const void *weight, const float *rstd, void *grad_x, void *grad_weight,
                                              void *workspace, size_t workspace_bytes, void *cuda_stream)
{
    if (!norm_ok(params) || !stride_ok(grad_y_stride, params->D)) return PPOW_ERR_INVALID_ARG;
    if (params->D > NORM_MAX_WIDTH) return PPOW_ERR_UNSUPPORTED;
    cudaStream_t stream = (cudaStream_t)cuda_stream;
    const size_t es = bytes_of(params->dtype), ps = bytes_of(params->param_dtype);
    if ((uintptr_t)grad_weight % ps) return PPOW_ERR_INVALID_ARG;
    if (params->R == 0)
        return grad_weight && cudaMemsetAsync(grad_weight, 0, (size_t)params->D * ps, stream) != cudaSuccess ? PPOW_ERR_CUDA : PPOW_OK;
    if (!grad_y || !weight || !rstd || !grad_x || !packed != !scale || !x == !packed) return PPOW_ERR_INVALID_ARG;
    if ((x && !stride_ok(x_stride, params->D)) || (grad_sum && !stride_ok(grad_sum_stride, params->D))) return PPOW_ERR_INVALID_ARG;
    if ((uintptr_t)grad_y % es || (uintptr_t)grad_sum % es || (uintptr_t)x % es || (uintptr_t)grad_x % es || (uintptr_t)weight % ps ||
        (uintptr_t)rstd % 4)
        return PPOW_ERR_INVALID_ARG;
    if (!workspace || (uintptr_t)workspace % 256 || workspace_bytes < ppow_rms_norm_workspace_bytes(params)) return PPOW_ERR_WORKSPACE;
    const RmsGradJob job = {grad_y, grad_y_stride, grad_sum, grad_sum_stride, x, x_stride, packed, scale, weight, rstd, params->R, params->D,
                            params->param_dtype, (params->D + CKPT_BLOCK - 1) / CKPT_BLOCK, grad_x, (float *)workspace};
    const bool vec = vec_ok(grad_y, grad_y_stride, params->D, es) && (!grad_sum || vec_ok(grad_sum, grad_sum_stride, params->D, es)) &&
                     (uintptr_t)grad_x % 16 == 0 && (x ? vec_ok(x, x_stride, params->D, es) : (uintptr_t)packed % 8 == 0);
    int32_t shares = 0;
#define PPOW_CALL(DT, VEC) rms_backward<DT, VEC>(job, &shares, stream)
    if (!PPOW_BY_TYPE(params->dtype, vec, PPOW_CALL)) return PPOW_ERR_CUDA;
#undef PPOW_CALL
    if (grad_weight && !launch_after(rms_join_kernel, (unsigned)((params->D + 31) / 32), 32 * JOIN_GROUPS, 0, stream, job.partial, shares,
                                     params->D, params->param_dtype, grad_weight))
        return PPOW_ERR_CUDA;
    return PPOW_OK;
}
