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
// All of it is bound by memory: one row at a time is held in registers by one warp or one CTA, read once; the sums over
// rows (dw, db) stay in registers of the thread that owns the column, are written once per CTA and added up in a fixed
// order by a second kernel.
#include "../../include/ppow.h"
#include "ppow_checked.cuh"
#include "ppow_device.cuh"

#include <cuda_bf16.h>
#include <cuda_fp8.h>
#include <atomic>
#include <math.h>

namespace ppow {

constexpr int CKPT_BLOCK = 128;          // values that share a scale
constexpr int32_t NORM_MAX_WIDTH = 16384;
constexpr int32_t NORM_MAX_ROWS = 1 << 28;

// ---- storage types ----------------------------------------------------------------------------------
template <int DTYPE> struct Storage;
template <> struct Storage<PPOW_F32> {
    using type = float;
    static constexpr int PER_UNIT = 4;
    static __device__ __forceinline__ float get(float x) { return x; }
    static __device__ __forceinline__ float put(float x) { return x; }
    static __device__ __forceinline__ void unpack(const uint4 &w, float (&f)[4]) { UnitF32::unpack(w, f); }
    static __device__ __forceinline__ uint4 pack(const float (&f)[4])
    {
        return make_uint4(__float_as_uint(f[0]), __float_as_uint(f[1]), __float_as_uint(f[2]), __float_as_uint(f[3]));
    }
};
template <> struct Storage<PPOW_BF16> {
    using type = uint16_t;
    static constexpr int PER_UNIT = 8;
    static __device__ __forceinline__ float get(uint16_t x) { return __uint_as_float((uint32_t)x << 16); }
    static __device__ __forceinline__ uint16_t put(float x) { return __bfloat16_as_ushort(__float2bfloat16_rn(x)); }
    static __device__ __forceinline__ void unpack(const uint4 &w, float (&f)[8]) { UnitBf16::unpack(w, f); }
    static __device__ __forceinline__ uint32_t two(float a, float b)
    {
        const __nv_bfloat162 h = __floats2bfloat162_rn(a, b);
        return *reinterpret_cast<const uint32_t *>(&h);
    }
    static __device__ __forceinline__ uint4 pack(const float (&f)[8])
    {
        return make_uint4(two(f[0], f[1]), two(f[2], f[3]), two(f[4], f[5]), two(f[6], f[7]));
    }
};
template <> struct Storage<PPOW_F16> {
    using type = uint16_t;
    static constexpr int PER_UNIT = 8;
    static __device__ __forceinline__ float get(uint16_t x) { return f16_to_f32(x); }
    static __device__ __forceinline__ uint16_t put(float x) { return __half_as_ushort(__float2half_rn(x)); }
    static __device__ __forceinline__ void unpack(const uint4 &w, float (&f)[8]) { UnitF16::unpack(w, f); }
    static __device__ __forceinline__ uint32_t two(float a, float b)
    {
        const __half2 h = __floats2half2_rn(a, b);
        return *reinterpret_cast<const uint32_t *>(&h);
    }
    static __device__ __forceinline__ uint4 pack(const float (&f)[8])
    {
        return make_uint4(two(f[0], f[1]), two(f[2], f[3]), two(f[4], f[5]), two(f[6], f[7]));
    }
};

// How a row is dealt out.  Unit u belongs to lane u % 32 of some warp.
//   VEC     a unit is 16 aligned bytes; a checkpoint block is 16 lanes (16-bit types) or 32 lanes (f32)
//   scalar  any width, stride and alignment: 32 units are a block of 128 columns, a lane takes columns lane, lane + 32, ...
template <int DTYPE, bool VEC> struct Deal;
template <int DTYPE> struct Deal<DTYPE, true> {
    using S = Storage<DTYPE>;
    using T = typename S::type;
    static constexpr int E = S::PER_UNIT;
    static constexpr int BLOCK_LANES = CKPT_BLOCK / E;
    uint4 raw;
    static __device__ __forceinline__ int32_t units(int32_t D) { return D / E; }
    static __device__ __forceinline__ int32_t column(int32_t u, int e) { return u * E + e; }
    static __device__ __forceinline__ bool has(int32_t, int, int32_t) { return true; }
    __device__ __forceinline__ void load(const T *row, int32_t u, int32_t) { raw = __ldcs(reinterpret_cast<const uint4 *>(row) + u); }
    __device__ __forceinline__ void zero() { raw = make_uint4(0, 0, 0, 0); }
    __device__ __forceinline__ void get(float (&f)[E]) const { S::unpack(raw, f); }
    static __device__ __forceinline__ void store(T *row, int32_t u, int32_t, const float (&f)[E])
    {
        reinterpret_cast<uint4 *>(row)[u] = S::pack(f);
    }
    static __device__ __forceinline__ void store_codes(uint8_t *row, int32_t u, int32_t, const uint32_t (&q)[E / 2])
    {
        if (E == 8)
            reinterpret_cast<uint2 *>(row)[u] = make_uint2(q[0] | (q[1] << 16), q[E / 2 - 2] | (q[E / 2 - 1] << 16));
        else
            reinterpret_cast<uint32_t *>(row)[u] = q[0] | (q[1] << 16);
    }
    static __device__ __forceinline__ void load_codes(const uint8_t *row, int32_t u, int32_t, uint32_t (&q)[E / 2])
    {
        if (E == 8) {
            const uint2 w = __ldcs(reinterpret_cast<const uint2 *>(row) + u);
            q[0] = w.x & 0xffffu, q[1] = w.x >> 16, q[E / 2 - 2] = w.y & 0xffffu, q[E / 2 - 1] = w.y >> 16;
        } else {
            const uint32_t w = __ldcs(reinterpret_cast<const uint32_t *>(row) + u);
            q[0] = w & 0xffffu, q[1] = w >> 16;
        }
    }
};
template <int DTYPE> struct Deal<DTYPE, false> {
    using S = Storage<DTYPE>;
    using T = typename S::type;
    static constexpr int E = 4;
    static constexpr int BLOCK_LANES = 32;
    T raw[4];
    static __device__ __forceinline__ int32_t units(int32_t D) { return (D + CKPT_BLOCK - 1) / CKPT_BLOCK * 32; }
    static __device__ __forceinline__ int32_t column(int32_t u, int e) { return (u >> 5) * CKPT_BLOCK + e * 32 + (u & 31); }
    static __device__ __forceinline__ bool has(int32_t u, int e, int32_t D) { return column(u, e) < D; }
    __device__ __forceinline__ void load(const T *row, int32_t u, int32_t D)
    {
#pragma unroll
        for (int e = 0; e < 4; ++e) raw[e] = has(u, e, D) ? __ldcs(row + column(u, e)) : T(0);
    }
    __device__ __forceinline__ void zero() { raw[0] = raw[1] = raw[2] = raw[3] = T(0); }
    __device__ __forceinline__ void get(float (&f)[4]) const
    {
#pragma unroll
        for (int e = 0; e < 4; ++e) f[e] = S::get(raw[e]);
    }
    static __device__ __forceinline__ void store(T *row, int32_t u, int32_t D, const float (&f)[4])
    {
#pragma unroll
        for (int e = 0; e < 4; ++e)
            if (has(u, e, D)) row[column(u, e)] = S::put(f[e]);
    }
    static __device__ __forceinline__ void store_codes(uint8_t *row, int32_t u, int32_t D, const uint32_t (&q)[2])
    {
#pragma unroll
        for (int e = 0; e < 4; ++e)
            if (has(u, e, D)) row[column(u, e)] = (uint8_t)(q[e >> 1] >> (8 * (e & 1)));
    }
    static __device__ __forceinline__ void load_codes(const uint8_t *row, int32_t u, int32_t D, uint32_t (&q)[2])
    {
        q[0] = q[1] = 0;
#pragma unroll
        for (int e = 0; e < 4; ++e)
            if (has(u, e, D)) q[e >> 1] |= (uint32_t)__ldcs(row + column(u, e)) << (8 * (e & 1));
    }
};

// ---- the 8-bit format -------------------------------------------------------------------------------
// e + 127 for a block whose largest finite magnitude is `top`.
__device__ __forceinline__ uint32_t scale_code(float top)
{
    const uint32_t b = __float_as_uint(top);
    const int32_t e = (int32_t)(b >> 23) - 127 - 8 + ((b & 0x7fffffu) > 0x600000u ? 1 : 0);   // 448 = 1.75 * 2^8
    return (uint32_t)(max(e, -126) + 127);
}
__device__ __forceinline__ float scale_up(uint32_t code) { return __uint_as_float((254u - code) << 23); }     // 2^-e
__device__ __forceinline__ float scale_down(uint32_t code) { return __uint_as_float(code << 23); }            // 2^e

__device__ __forceinline__ float finite_magnitude(float x)
{
    const float a = fabsf(x);
    return a < INFINITY ? a : 0.0f;
}
// two values; an infinity becomes NaN (the format has none), as NaN does
__device__ __forceinline__ uint32_t codes_of(float a, float b, float up)
{
    return (uint32_t)__nv_cvt_float2_to_fp8x2(make_float2(fmaf(a, 0.0f, a) * up, fmaf(b, 0.0f, b) * up), __NV_SATFINITE, __NV_E4M3);
}
__device__ __forceinline__ float2 values_of(uint32_t codes, float down)
{
    const __half2_raw h = __nv_cvt_fp8x2_to_halfraw2((__nv_fp8x2_storage_t)codes, __NV_E4M3);
    const float2 f = __half22float2(__half2(h));
    return make_float2(f.x * down, f.y * down);
}

template <int LANES> __device__ __forceinline__ float lanes_max(float v)
{
#pragma unroll
    for (int o = LANES / 2; o > 0; o >>= 1) v = fmaxf(v, __shfl_xor_sync(0xffffffffu, v, o));
    return v;
}
__device__ __forceinline__ float warp_sum(float v)
{
#pragma unroll
    for (int o = 16; o > 0; o >>= 1) v += __shfl_xor_sync(0xffffffffu, v, o);
    return v;
}

// Packs one unit per lane (the whole warp calls; `valid` lanes hold a unit).
template <typename DealT>
__device__ __forceinline__ void pack_unit(const float (&f)[DealT::E], bool valid, int32_t u, int32_t D, uint8_t *codes, uint8_t *scales)
{
    float top = 0.0f;
#pragma unroll
    for (int e = 0; e < DealT::E; ++e) top = fmaxf(top, finite_magnitude(f[e]));
    top = lanes_max<DealT::BLOCK_LANES>(valid ? top : 0.0f);
    if (!valid) return;
    const uint32_t code = scale_code(top);
    const float up = scale_up(code);
    uint32_t q[DealT::E / 2];
#pragma unroll
    for (int e = 0; e < DealT::E / 2; ++e) q[e] = codes_of(f[2 * e], f[2 * e + 1], up);
    DealT::store_codes(codes, u, D, q);
    if (u % DealT::BLOCK_LANES == 0) scales[u / DealT::BLOCK_LANES] = (uint8_t)code;
}

template <typename DealT>
__device__ __forceinline__ void unpack_unit(const uint8_t *codes, const uint8_t *scales, int32_t u, int32_t D, float (&f)[DealT::E])
{
    uint32_t q[DealT::E / 2];
    DealT::load_codes(codes, u, D, q);
    const float down = scale_down(scales[u / DealT::BLOCK_LANES]);
#pragma unroll
    for (int e = 0; e < DealT::E / 2; ++e) {
        const float2 v = values_of(q[e], down);
        f[2 * e] = v.x, f[2 * e + 1] = v.y;
    }
}

__device__ __forceinline__ float load_param(const void *p, int32_t dtype, int32_t i)
{
    if (dtype == PPOW_F32) return static_cast<const float *>(p)[i];
    const uint16_t b = static_cast<const uint16_t *>(p)[i];
    return dtype == PPOW_BF16 ? Storage<PPOW_BF16>::get(b) : Storage<PPOW_F16>::get(b);
}
__device__ __forceinline__ void store_param(void *p, int32_t dtype, int32_t i, float v)
{
    if (dtype == PPOW_F32)
        static_cast<float *>(p)[i] = v;
    else
        static_cast<uint16_t *>(p)[i] = dtype == PPOW_BF16 ? Storage<PPOW_BF16>::put(v) : Storage<PPOW_F16>::put(v);
}

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

// TPR threads hold one row, U units each.
template <int TPR> __host__ __device__ constexpr int norm_threads() { return TPR < 128 ? 128 : TPR; }

template <int DTYPE, bool VEC, int TPR, int U>
__global__ void __launch_bounds__(norm_threads<TPR>()) norm_forward_kernel(const NormJob job)
{
    using DealT = Deal<DTYPE, VEC>;
    using T = typename DealT::T;
    constexpr int E = DealT::E, THREADS = norm_threads<TPR>(), ROWS = THREADS / TPR, WARPS = TPR / 32;
    constexpr bool HOLD = TPR <= 256;                        // weight and bias of the thread's columns stay in registers
    __shared__ float2 part[2][WARPS];                        // per warp: mean, sum of squares about it
    const int t = threadIdx.x % TPR, lane = threadIdx.x & 31;
    const int32_t D = job.D, units = DealT::units(D);
    float w[HOLD ? U : 1][E], b[HOLD ? U : 1][E];
    if constexpr (HOLD) {
#pragma unroll
        for (int k = 0; k < U; ++k)
#pragma unroll
            for (int e = 0; e < E; ++e) {
                const int32_t c = DealT::column(t + k * TPR, e);
                w[k][e] = c < D ? load_param(job.weight, job.param_dtype, c) : 0.0f;
                b[k][e] = c < D && job.bias ? load_param(job.bias, job.param_dtype, c) : 0.0f;
            }
    }
    // columns that this thread and this warp hold
    int32_t mine = 0;
#pragma unroll
    for (int k = 0; k < U; ++k)
#pragma unroll
        for (int e = 0; e < E; ++e) mine += t + k * TPR < units && DealT::column(t + k * TPR, e) < D;
    const float in_warp = (float)__reduce_add_sync(0xffffffffu, mine);
    const float inv_warp = in_warp > 0.0f ? 1.0f / in_warp : 0.0f, inv_d = 1.0f / (float)D;
    int turn = 0;

    for (int64_t row = (int64_t)blockIdx.x * ROWS + threadIdx.x / TPR; row < job.R; row += (int64_t)gridDim.x * ROWS, turn ^= 1) {
        if (!PPOW_CHECK(units <= TPR * U, 601, nullptr)) return;
        DealT x[U];
        const T *src = static_cast<const T *>(job.x) + row * job.x_stride;
#pragma unroll
        for (int k = 0; k < U; ++k) {
            const int32_t u = t + k * TPR;
            if (u < units)
                x[k].load(src, u, D);
            else
                x[k].zero();
        }
        // mean of the warp's values, then squares about it: no difference of large sums
        float sum = 0.0f;
#pragma unroll
        for (int k = 0; k < U; ++k) {
            float f[E];
            x[k].get(f);
#pragma unroll
            for (int e = 0; e < E; ++e) sum += f[e];
        }
        const float m = warp_sum(sum) * inv_warp;
        float sq = 0.0f;
#pragma unroll
        for (int k = 0; k < U; ++k) {
            const int32_t u = t + k * TPR;
            float f[E];
            x[k].get(f);
#pragma unroll
            for (int e = 0; e < E; ++e) {
                const float d = u < units && DealT::has(u, e, D) ? f[e] - m : 0.0f;
                sq = fmaf(d, d, sq);
            }
        }
        sq = warp_sum(sq);
        float mean = m, squares = sq;
        if (WARPS > 1) {
            // every warp's count follows from the deal: recompute it instead of sending it
            if (lane == 0) part[turn][t >> 5] = make_float2(m * in_warp, in_warp > 0.0f ? sq : 0.0f);
            __syncthreads();
            float total = 0.0f;
#pragma unroll
            for (int i = 0; i < WARPS; ++i) total += part[turn][i].x;
            mean = total * inv_d;
            // squares about the row's mean: each warp's squares about its own, plus its count times the gap squared
            const float gap = m - mean;
            float own = sq + in_warp * gap * gap;
            __shared__ float spread[2][WARPS];
            if (lane == 0) spread[turn][t >> 5] = in_warp > 0.0f ? own : 0.0f;
            __syncthreads();
            squares = 0.0f;
#pragma unroll
            for (int i = 0; i < WARPS; ++i) squares += spread[turn][i];
        }
        const float rstd = 1.0f / sqrtf(squares * inv_d + job.eps);
        T *dst = static_cast<T *>(job.y) + row * D;
#pragma unroll
        for (int k = 0; k < U; ++k) {
            const int32_t u = t + k * TPR;
            if (u < units) {
                float f[E], y[E];
                x[k].get(f);
#pragma unroll
                for (int e = 0; e < E; ++e) {
                    float we, be;
                    if constexpr (HOLD) {
                        we = w[k][e], be = b[k][e];
                    } else {
                        const int32_t c = min(DealT::column(u, e), D - 1);
                        we = load_param(job.weight, job.param_dtype, c);
                        be = job.bias ? load_param(job.bias, job.param_dtype, c) : 0.0f;
                    }
                    y[e] = fmaf((f[e] - mean) * rstd, we, be);
                }
                DealT::store(dst, u, D, y);
            }
        }
        if (t == 0) {
            job.mean[row] = mean;
            job.rstd[row] = rstd;
        }
        if (job.codes) {
#pragma unroll
            for (int k = 0; k < U; ++k) {
                const int32_t u = t + k * TPR;
                float f[E];
                x[k].get(f);
                pack_unit<DealT>(f, u < units, u, D, job.codes + row * D, job.scales + row * job.blocks);
            }
        }
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

template <int DTYPE, bool VEC, bool PACKED, int TPR, int U>
__global__ void __launch_bounds__(norm_threads<TPR>()) norm_backward_kernel(const NormGradJob job)
{
    using DealT = Deal<DTYPE, VEC>;
    using T = typename DealT::T;
    constexpr int E = DealT::E, THREADS = norm_threads<TPR>(), ROWS = THREADS / TPR, WARPS = TPR / 32;
    constexpr bool HOLD = TPR <= 256;    // the column sums and the weight stay in registers; else the sums in shared memory
    extern __shared__ float sums[];      // !HOLD: [2][D]
    __shared__ float2 part[2][WARPS];
    const int t = threadIdx.x % TPR, lane = threadIdx.x & 31;
    const int32_t D = job.D, units = DealT::units(D);
    const float inv_d = 1.0f / (float)D;
    float w[HOLD ? U : 1][E], dw[HOLD ? U : 1][E], db[HOLD ? U : 1][E];
#pragma unroll
    for (int k = 0; k < (HOLD ? U : 1); ++k)
#pragma unroll
        for (int e = 0; e < E; ++e) {
            const int32_t c = DealT::column(t + k * TPR, e);
            w[k][e] = HOLD && c < D ? load_param(job.weight, job.param_dtype, c) : 0.0f;
            dw[k][e] = db[k][e] = 0.0f;
        }
    if (!HOLD) {
        for (int32_t i = threadIdx.x; i < 2 * D; i += THREADS) sums[i] = 0.0f;
        __syncthreads();
    }
    int turn = 0;
    for (int64_t row = (int64_t)blockIdx.x * ROWS + threadIdx.x / TPR; row < job.R; row += (int64_t)gridDim.x * ROWS, turn ^= 1) {
        if (!PPOW_CHECK(units <= TPR * U, 602, nullptr)) return;
        DealT g[U], x[PACKED ? 1 : U];
        float xp[PACKED ? U : 1][E];
        const T *gsrc = static_cast<const T *>(job.grad_y) + row * job.grad_y_stride;
        const T *xsrc = static_cast<const T *>(job.x) + row * job.x_stride;
#pragma unroll
        for (int k = 0; k < U; ++k) {
            const int32_t u = t + k * TPR;
            if (u < units) {
                g[k].load(gsrc, u, D);
                if (PACKED)
                    unpack_unit<DealT>(job.codes + row * D, job.scales + row * job.blocks, u, D, xp[PACKED ? k : 0]);
                else
                    x[PACKED ? 0 : k].load(xsrc, u, D);
            } else {
                g[k].zero();
                if (PACKED) {
#pragma unroll
                    for (int e = 0; e < E; ++e) xp[PACKED ? k : 0][e] = 0.0f;
                } else {
                    x[PACKED ? 0 : k].zero();
                }
            }
        }
        const float mean = job.mean[row], rstd = job.rstd[row];
        auto weight_at = [&](int k, int e) {
            if constexpr (HOLD) {
                return w[k][e];
            } else {
                const int32_t c = DealT::column(t + k * TPR, e);
                return c < D ? load_param(job.weight, job.param_dtype, c) : 0.0f;
            }
        };
        auto input = [&](int k, float (&f)[E]) {
            if (PACKED) {
#pragma unroll
                for (int e = 0; e < E; ++e) f[e] = xp[PACKED ? k : 0][e];
            } else {
                x[PACKED ? 0 : k].get(f);
            }
        };
        float c1 = 0.0f, c2 = 0.0f;
#pragma unroll
        for (int k = 0; k < U; ++k) {
            float f[E], gy[E];
            input(k, f);
            g[k].get(gy);
#pragma unroll
            for (int e = 0; e < E; ++e) {
                // columns that do not exist have gy = 0 and w = 0
                const float xh = (f[e] - mean) * rstd, a = gy[e] * weight_at(k, e);
                c1 += a;
                c2 = fmaf(a, xh, c2);
                if constexpr (HOLD) {
                    dw[k][e] = fmaf(gy[e], xh, dw[k][e]);
                    db[k][e] += gy[e];
                } else {
                    const int32_t c = DealT::column(t + k * TPR, e);
                    if (t + k * TPR < units && c < D) {
                        sums[c] = fmaf(gy[e], xh, sums[c]);
                        sums[D + c] += gy[e];
                    }
                }
            }
        }
        c1 = warp_sum(c1);
        c2 = warp_sum(c2);
        if (WARPS > 1) {
            if (lane == 0) part[turn][t >> 5] = make_float2(c1, c2);
            __syncthreads();
            c1 = c2 = 0.0f;
#pragma unroll
            for (int i = 0; i < WARPS; ++i) {
                c1 += part[turn][i].x;
                c2 += part[turn][i].y;
            }
        }
        c1 *= inv_d;
        c2 *= inv_d;
        T *dst = static_cast<T *>(job.grad_x) + row * D;
#pragma unroll
        for (int k = 0; k < U; ++k) {
            const int32_t u = t + k * TPR;
            if (u < units) {
                float f[E], gy[E], o[E];
                input(k, f);
                g[k].get(gy);
#pragma unroll
                for (int e = 0; e < E; ++e) {
                    const float xh = (f[e] - mean) * rstd;
                    o[e] = (gy[e] * weight_at(k, e) - c1 - xh * c2) * rstd;
                }
                DealT::store(dst, u, D, o);
            }
        }
    }
    // this CTA's share of the column sums
    float *out = job.partial + (size_t)blockIdx.x * 2 * D;
    if constexpr (!HOLD) {
        __syncthreads();
        for (int32_t i = threadIdx.x; i < 2 * D; i += THREADS) out[i] = sums[i];
    }
    if constexpr (HOLD && ROWS == 1) {
#pragma unroll
        for (int k = 0; k < U; ++k)
#pragma unroll
            for (int e = 0; e < E; ++e) {
                const int32_t u = t + k * TPR, c = DealT::column(u, e);
                if (u < units && c < D) {
                    out[c] = dw[k][e];
                    out[D + c] = db[k][e];
                }
            }
    }
    if constexpr (ROWS > 1) {
        // several rows at a time: the warps add their sums up one after the other
        __shared__ float joint[2][TPR * U * E];
        for (int s = 0; s < ROWS; ++s) {
            if (threadIdx.x / TPR == s) {
#pragma unroll
                for (int k = 0; k < U; ++k)
#pragma unroll
                    for (int e = 0; e < E; ++e) {
                        const int i = (k * E + e) * TPR + t;
                        const float sw = (s ? joint[0][i] : 0.0f) + dw[k][e], sb = (s ? joint[1][i] : 0.0f) + db[k][e];
                        joint[0][i] = sw;
                        joint[1][i] = sb;
                        const int32_t u = t + k * TPR, c = DealT::column(u, e);
                        if (s == ROWS - 1 && u < units && c < D) {
                            out[c] = sw;
                            out[D + c] = sb;
                        }
                    }
            }
            __syncthreads();
        }
    }
}

// Column sums over the CTAs' shares, in a fixed order: 32 columns by 8 groups of shares per CTA.
constexpr int JOIN_GROUPS = 8;
__global__ void __launch_bounds__(32 * JOIN_GROUPS) norm_join_kernel(const float *__restrict__ partial, int32_t shares, int32_t D,
                                                                     int32_t param_dtype, void *grad_weight, void *grad_bias)
{
    __shared__ float group[JOIN_GROUPS][32];
    const int lane = threadIdx.x & 31, g = threadIdx.x >> 5;
    const int32_t c = blockIdx.x * 32 + lane;        // column of dw, then of db
    float sum = 0.0f;
    if (c < 2 * D)
        for (int32_t s = g; s < shares; s += JOIN_GROUPS) sum += partial[(size_t)s * 2 * D + c];
    group[g][lane] = sum;
    __syncthreads();
    if (g == 0 && c < 2 * D) {
        sum = 0.0f;
#pragma unroll
        for (int i = 0; i < JOIN_GROUPS; ++i) sum += group[i][lane];
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

template <int DTYPE, bool VEC>
__global__ void __launch_bounds__(PACK_THREADS) pack_kernel(const PackJob job)
{
    using DealT = Deal<DTYPE, VEC>;
    using T = typename DealT::T;
    const int lane = threadIdx.x & 31;
    const int32_t units = DealT::units(job.D), per_row = (units + 31) / 32;
    const int64_t chunks = (int64_t)job.R * per_row, first = ((int64_t)blockIdx.x * (PACK_THREADS / 32) + (threadIdx.x >> 5)) * PACK_CHUNKS;
    DealT x[PACK_CHUNKS];
#pragma unroll
    for (int i = 0; i < PACK_CHUNKS; ++i) {
        const int64_t c = first + i, row = c / per_row;
        const int32_t u = (int32_t)(c % per_row) * 32 + lane;
        x[i].zero();
        if (c < chunks && u < units) x[i].load(static_cast<const T *>(job.x) + row * job.x_stride, u, job.D);
    }
#pragma unroll
    for (int i = 0; i < PACK_CHUNKS; ++i) {
        const int64_t c = first + i, row = c / per_row;
        const int32_t u = (int32_t)(c % per_row) * 32 + lane;
        if (c >= chunks || !PPOW_CHECK(row < job.R, 603, nullptr)) return;
        float f[DealT::E];
        x[i].get(f);
        pack_unit<DealT>(f, u < units, u, job.D, job.codes + row * job.D, job.scales + row * job.blocks);
    }
}

template <int DTYPE, bool VEC>
__global__ void __launch_bounds__(PACK_THREADS) unpack_kernel(const PackJob job)
{
    using DealT = Deal<DTYPE, VEC>;
    using T = typename DealT::T;
    const int lane = threadIdx.x & 31;
    const int32_t units = DealT::units(job.D), per_row = (units + 31) / 32;
    const int64_t chunks = (int64_t)job.R * per_row, first = ((int64_t)blockIdx.x * (PACK_THREADS / 32) + (threadIdx.x >> 5)) * PACK_CHUNKS;
#pragma unroll
    for (int i = 0; i < PACK_CHUNKS; ++i) {
        const int64_t c = first + i, row = c / per_row;
        const int32_t u = (int32_t)(c % per_row) * 32 + lane;
        if (c >= chunks || !PPOW_CHECK(row < job.R, 604, nullptr)) return;
        if (u < units) {
            float f[DealT::E];
            unpack_unit<DealT>(job.codes + row * job.D, job.scales + row * job.blocks, u, job.D, f);
            DealT::store(static_cast<T *>(job.out) + row * job.D, u, job.D, f);
        }
    }
}

// ---- host side --------------------------------------------------------------------------------------
namespace {

size_t bytes_of(int32_t dtype) { return dtype == PPOW_F32 ? 4 : 2; }
bool dtype_ok(int32_t d) { return d == PPOW_F32 || d == PPOW_BF16 || d == PPOW_F16; }

bool norm_ok(const ppow_norm_params *p)
{
    return p && p->R >= 0 && p->R <= NORM_MAX_ROWS && p->D >= 1 && dtype_ok(p->dtype) &&
           (p->param_dtype == PPOW_F32 || p->param_dtype == p->dtype) && p->eps >= 0.0f && isfinite(p->eps);
}
bool stride_ok(int64_t stride, int32_t D) { return stride >= D && stride <= (int64_t)1 << 40; }

// rows in whole 16-byte units
bool vec_ok(const void *p, int64_t stride, int32_t D, size_t es)
{
    return (uintptr_t)p % 16 == 0 && (size_t)D * es % 16 == 0 && (size_t)stride * es % 16 == 0;
}

// CTAs of a kernel that one launch keeps resident on the current device; asked once per device and kernel.
constexpr int DEVICES = 64;
struct Resident {
    std::atomic<int> ctas[DEVICES];
};
template <typename Kernel>
int resident_ctas(Resident &known, Kernel kernel, int threads, size_t smem)
{
    int dev = 0;
    if (cudaGetDevice(&dev) != cudaSuccess || dev < 0 || dev >= DEVICES) return 0;
    int n = known.ctas[dev].load(std::memory_order_relaxed);
    if (n > 0) return n;
    int sms = 0, per_sm = 0;
    if (smem > 0 && cudaFuncSetAttribute(kernel, cudaFuncAttributeMaxDynamicSharedMemorySize, (int)smem) != cudaSuccess) return 0;
    if (cudaDeviceGetAttribute(&sms, cudaDevAttrMultiProcessorCount, dev) != cudaSuccess ||
        cudaOccupancyMaxActiveBlocksPerMultiprocessor(&per_sm, kernel, threads, smem) != cudaSuccess)
        return 0;
    n = sms * per_sm;
    known.ctas[dev].store(n, std::memory_order_relaxed);
    return n;
}

// CTAs of the backward pass: each leaves one share of the column sums.  148 SMs x 2 to 4; a function of the sizes alone.
constexpr int32_t SHARES_MAX = 148 * 4;

template <int DTYPE, bool VEC, int TPR, int U>
bool forward_launch(const NormJob &job, cudaStream_t stream)
{
    constexpr int THREADS = norm_threads<TPR>(), ROWS = THREADS / TPR;
    static Resident known;
    const int64_t need = ((int64_t)job.R + ROWS - 1) / ROWS, most = resident_ctas(known, norm_forward_kernel<DTYPE, VEC, TPR, U>, THREADS, 0);
    if (most < 1) return false;
    norm_forward_kernel<DTYPE, VEC, TPR, U><<<(unsigned)(need < most ? need : most), THREADS, 0, stream>>>(job);
    return cudaGetLastError() == cudaSuccess;
}

template <int DTYPE, bool VEC>
bool forward_shape(const NormJob &job, cudaStream_t stream)
{
    const int32_t units = VEC ? job.D / (16 / (int32_t)bytes_of(DTYPE)) : (job.D + CKPT_BLOCK - 1) / CKPT_BLOCK * 32;
    if (units <= 32 * 4) return forward_launch<DTYPE, VEC, 32, 4>(job, stream);
    if (units <= 128 * 4) return forward_launch<DTYPE, VEC, 128, 4>(job, stream);
    if (units <= 256 * 4) return forward_launch<DTYPE, VEC, 256, 4>(job, stream);
    return forward_launch<DTYPE, VEC, 1024, 4>(job, stream);
}

template <int DTYPE, bool VEC, bool PACKED, int TPR, int U>
bool backward_launch(const NormGradJob &job, int32_t *shares, cudaStream_t stream)
{
    constexpr int THREADS = norm_threads<TPR>(), ROWS = THREADS / TPR;
    constexpr size_t SMEM = TPR <= 256 ? 0 : (size_t)NORM_MAX_WIDTH * 8;
    auto kernel = norm_backward_kernel<DTYPE, VEC, PACKED, TPR, U>;
    static Resident known;
    const int64_t most = resident_ctas(known, kernel, THREADS, SMEM);
    if (most < 1) return false;
    int64_t n = ((int64_t)job.R + ROWS - 1) / ROWS;
    if (n > most) n = most;
    if (n > SHARES_MAX) n = SHARES_MAX;
    *shares = (int32_t)n;
    kernel<<<(unsigned)n, THREADS, SMEM, stream>>>(job);
    return cudaGetLastError() == cudaSuccess;
}

template <int DTYPE, bool VEC, bool PACKED>
bool backward_shape(const NormGradJob &job, int32_t *shares, cudaStream_t stream)
{
    const int32_t units = VEC ? job.D / (16 / (int32_t)bytes_of(DTYPE)) : (job.D + CKPT_BLOCK - 1) / CKPT_BLOCK * 32;
    if (units <= 32 * 4) return backward_launch<DTYPE, VEC, PACKED, 32, 4>(job, shares, stream);
    if (units <= 128 * 4) return backward_launch<DTYPE, VEC, PACKED, 128, 4>(job, shares, stream);
    if (units <= 256 * 4) return backward_launch<DTYPE, VEC, PACKED, 256, 4>(job, shares, stream);
    return backward_launch<DTYPE, VEC, PACKED, 1024, 4>(job, shares, stream);
}

template <int DTYPE, bool VEC>
bool pack_launch(const PackJob &job, bool unpack, cudaStream_t stream)
{
    const int32_t units = VEC ? job.D / (16 / (int32_t)bytes_of(DTYPE)) : (job.D + CKPT_BLOCK - 1) / CKPT_BLOCK * 32;
    const int64_t chunks = (int64_t)job.R * ((units + 31) / 32), per_cta = PACK_THREADS / 32 * PACK_CHUNKS;
    const unsigned grid = (unsigned)((chunks + per_cta - 1) / per_cta);
    if (unpack)
        unpack_kernel<DTYPE, VEC><<<grid, PACK_THREADS, 0, stream>>>(job);
    else
        pack_kernel<DTYPE, VEC><<<grid, PACK_THREADS, 0, stream>>>(job);
    return cudaGetLastError() == cudaSuccess;
}

#define PPOW_BY_TYPE(dtype, vec, CALL)                                                                          \
    ((dtype) == PPOW_F32    ? ((vec) ? CALL(PPOW_F32, true) : CALL(PPOW_F32, false))                             \
     : (dtype) == PPOW_BF16 ? ((vec) ? CALL(PPOW_BF16, true) : CALL(PPOW_BF16, false))                           \
                            : ((vec) ? CALL(PPOW_F16, true) : CALL(PPOW_F16, false)))

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
        norm_join_kernel<<<(unsigned)((2 * params->D + 31) / 32), 32 * JOIN_GROUPS, 0, stream>>>(job.partial, shares, params->D,
                                                                                             params->param_dtype, grad_weight, grad_bias);
        if (cudaGetLastError() != cudaSuccess) return PPOW_ERR_CUDA;
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
