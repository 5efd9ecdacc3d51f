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
#include "../../include/ppow.h"
#include "ppow_checked.cuh"
#include "ppow_device.cuh"
#include "ppow_mma.cuh"

#include <cuda_bf16.h>
#include <cuda_fp8.h>
#include <atomic>
#include <math.h>
#include <type_traits>

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
    static __device__ __forceinline__ bool whole(int32_t u, int32_t D) { return ((u >> 5) + 1) * CKPT_BLOCK <= D; }   // of the warp's block
    __device__ __forceinline__ void load(const T *row, int32_t u, int32_t D)
    {
        if (whole(u, D)) {
#pragma unroll
            for (int e = 0; e < 4; ++e) raw[e] = __ldcs(row + column(u, 0) + 32 * e);
        } else {
#pragma unroll
            for (int e = 0; e < 4; ++e) raw[e] = has(u, e, D) ? __ldcs(row + column(u, e)) : T(0);
        }
    }
    __device__ __forceinline__ void zero() { raw[0] = raw[1] = raw[2] = raw[3] = T(0); }
    __device__ __forceinline__ void get(float (&f)[4]) const
    {
#pragma unroll
        for (int e = 0; e < 4; ++e) f[e] = S::get(raw[e]);
    }
    static __device__ __forceinline__ void store(T *row, int32_t u, int32_t D, const float (&f)[4])
    {
        T *to = row + column(u, 0);
        if (whole(u, D)) {
#pragma unroll
            for (int e = 0; e < 4; ++e) to[32 * e] = S::put(f[e]);
        } else {
#pragma unroll
            for (int e = 0; e < 4; ++e)
                if (has(u, e, D)) to[32 * e] = S::put(f[e]);
        }
    }
    static __device__ __forceinline__ void store_codes(uint8_t *row, int32_t u, int32_t D, const uint32_t (&q)[2])
    {
        uint8_t *to = row + column(u, 0);
        if (whole(u, D)) {
#pragma unroll
            for (int e = 0; e < 4; ++e) to[32 * e] = (uint8_t)(q[e >> 1] >> (8 * (e & 1)));
        } else {
#pragma unroll
            for (int e = 0; e < 4; ++e)
                if (has(u, e, D)) to[32 * e] = (uint8_t)(q[e >> 1] >> (8 * (e & 1)));
        }
    }
    static __device__ __forceinline__ void load_codes(const uint8_t *row, int32_t u, int32_t D, uint32_t (&q)[2])
    {
        uint32_t c[4];
#pragma unroll
        for (int e = 0; e < 4; ++e) c[e] = whole(u, D) || has(u, e, D) ? __ldcs(row + column(u, 0) + 32 * e) : 0u;
        q[0] = c[0] | (c[1] << 8);
        q[1] = c[2] | (c[3] << 8);
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
__device__ __forceinline__ float nan_for_inf(float x) { return fmaf(x, 0.0f, x); }     // the format has no infinity
// two scaled values, to nearest even; NaN stays NaN
__device__ __forceinline__ uint32_t codes_of(float a, float b)
{
    return (uint32_t)__nv_cvt_float2_to_fp8x2(make_float2(a, b), __NV_SATFINITE, __NV_E4M3);
}
// two codes as float16 pairs (exact)
__device__ __forceinline__ float2 halves_of(uint32_t codes)
{
    const __half2_raw h = __nv_cvt_fp8x2_to_halfraw2((__nv_fp8x2_storage_t)codes, __NV_E4M3);
    return __half22float2(__half2(h));
}
__device__ __forceinline__ float2 values_of(uint32_t codes, float down) { return __fmul2_rn(halves_of(codes), make_float2(down, down)); }

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

// 1 / sqrt(v): the approximation and one step of Newton's method, exact to about a step of float32
__device__ __forceinline__ float inverse_root(float v)
{
    const float r = rsqrtf(v), h = 0.5f * v * r;
    return v > 0.0f && v < INFINITY ? fmaf(r, fmaf(-h, r, 0.5f), r) : r;
}

template <int U> __device__ __forceinline__ float total_of(float2 (&v)[U])
{
#pragma unroll
    for (int h = U / 2; h > 0; h >>= 1)
#pragma unroll
        for (int k = 0; k < h; ++k) v[k] = __fadd2_rn(v[k], v[k + h]);
    return v[0].x + v[0].y;
}

// Packs N units per lane, `step` units apart (the whole warp calls; lanes with no unit bring any finite values).
template <typename DealT, int N>
__device__ __forceinline__ void pack_units(const float (&f)[N][DealT::E], int32_t u0, int32_t step, int32_t units, int32_t D, uint8_t *codes,
                                           uint8_t *scales)
{
    constexpr int E = DealT::E, LANES = DealT::BLOCK_LANES;
    float top[N];
    bool infinite = false;
#pragma unroll
    for (int k = 0; k < N; ++k) {
        float a = 0.0f, b = 0.0f;
#pragma unroll
        for (int e = 0; e < E; e += 2) a = fmaxf(a, fabsf(f[k][e])), b = fmaxf(b, fabsf(f[k][e + 1]));     // pass NaN over
        top[k] = u0 + k * step < units ? fmaxf(a, b) : 0.0f;
    }
#pragma unroll
    for (int o = LANES / 2; o > 0; o >>= 1)
#pragma unroll
        for (int k = 0; k < N; ++k) top[k] = fmaxf(top[k], __shfl_xor_sync(0xffffffffu, top[k], o));
#pragma unroll
    for (int k = 0; k < N; ++k) infinite = infinite || top[k] == INFINITY;
    infinite = __any_sync(0xffffffffu, infinite);
#pragma unroll
    for (int k = 0; k < N; ++k) {
        const int32_t u = u0 + k * step;
        uint32_t q[E / 2], code = scale_code(top[k]);
        if (infinite) {                                                   // the scale goes by the finite values
            float finite = 0.0f;
#pragma unroll
            for (int e = 0; e < E; ++e) finite = fmaxf(finite, finite_magnitude(f[k][e]));
            code = scale_code(lanes_max<LANES>(u < units ? finite : 0.0f));
        }
        const float2 up = make_float2(scale_up(code), scale_up(code));
#pragma unroll
        for (int e = 0; e < E / 2; ++e) {
            float2 v = make_float2(f[k][2 * e], f[k][2 * e + 1]);
            if (infinite) v = make_float2(nan_for_inf(v.x), nan_for_inf(v.y));
            v = __fmul2_rn(v, up);
            q[e] = codes_of(v.x, v.y);
        }
        if (u < units) {
            DealT::store_codes(codes, u, D, q);
            if (u % LANES == 0) scales[u / LANES] = (uint8_t)code;
        }
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

// ---- rows ahead of their use ------------------------------------------------------------------------
__device__ __forceinline__ uint32_t smem_address(const void *p) { return (uint32_t)__cvta_generic_to_shared(p); }
template <int BYTES> __device__ __forceinline__ void copy_async(uint32_t dst, const void *src)
{
    if constexpr (BYTES == 16)
        asm volatile("cp.async.cg.shared.global [%0], [%1], 16;" ::"r"(dst), "l"(src) : "memory");
    else
        asm volatile("cp.async.ca.shared.global [%0], [%1], %2;" ::"r"(dst), "l"(src), "n"(BYTES) : "memory");
}
__device__ __forceinline__ void copy_commit() { asm volatile("cp.async.commit_group;" ::: "memory"); }
template <int LEFT> __device__ __forceinline__ void copy_wait() { asm volatile("cp.async.wait_group %0;" ::"n"(LEFT) : "memory"); }

// The thread's own units of the next rows.  VEC: S slots in shared memory, filled by asynchronous copies; a thread reads what
// it copied itself, so no barrier is needed and the bytes in flight cost no registers.  Scalar: registers, one row ahead.
template <int DTYPE, bool VEC, int TPR, int U, int S> struct RowAhead;
template <int DTYPE, int TPR, int U, int S> struct RowAhead<DTYPE, true, TPR, U, S> {
    using DealT = Deal<DTYPE, true>;
    using T = typename DealT::T;
    static constexpr size_t BYTES = (size_t)S * U * TPR * 16;       // per row group
    uint8_t *own;                                                   // this thread's first unit in slot 0
    uint32_t base;
    __device__ __forceinline__ RowAhead(uint8_t *smem, int t) : own(smem + t * 16), base(smem_address(own)) {}
    __device__ __forceinline__ void start(int slot, const T *row, int t, int32_t units, int32_t)
    {
#pragma unroll
        for (int k = 0; k < U; ++k)
            if (t + k * TPR < units) copy_async<16>(base + (slot * U + k) * (TPR * 16), reinterpret_cast<const uint4 *>(row) + t + k * TPR);
    }
    __device__ __forceinline__ void take() {}
    // units behind the row's end read as whatever the slot holds: callers use them only where t + k * TPR < units
    __device__ __forceinline__ void get(int slot, int k, float (&f)[DealT::E]) const
    {
        const uint4 w = *reinterpret_cast<const uint4 *>(own + (slot * U + k) * (TPR * 16));
        DealT::S::unpack(w, f);
    }
    __device__ __forceinline__ void centred(int slot, int k, float, float2 minus_mean, float2 (&c)[DealT::E / 2]) const
    {
        float f[DealT::E];
        get(slot, k, f);
#pragma unroll
        for (int e = 0; e < DealT::E / 2; ++e) c[e] = __fadd2_rn(make_float2(f[2 * e], f[2 * e + 1]), minus_mean);
    }
};
template <int DTYPE, int TPR, int U, int S> struct RowAhead<DTYPE, false, TPR, U, S> {
    using DealT = Deal<DTYPE, false>;
    using T = typename DealT::T;
    static constexpr size_t BYTES = 0;
    DealT next[U], now[U];
    __device__ __forceinline__ RowAhead(uint8_t *, int) {}
    __device__ __forceinline__ void start(int, const T *row, int t, int32_t units, int32_t D)
    {
#pragma unroll
        for (int k = 0; k < U; ++k)
            if (t + k * TPR < units) next[k].load(row, t + k * TPR, D);
    }
    __device__ __forceinline__ void take()
    {
#pragma unroll
        for (int k = 0; k < U; ++k) now[k] = next[k];
    }
    __device__ __forceinline__ void get(int, int k, float (&f)[4]) const { now[k].get(f); }
    __device__ __forceinline__ void centred(int, int k, float, float2 minus_mean, float2 (&c)[2]) const
    {
        float f[4];
        now[k].get(f);
        c[0] = __fadd2_rn(make_float2(f[0], f[1]), minus_mean);
        c[1] = __fadd2_rn(make_float2(f[2], f[3]), minus_mean);
    }
};
// The 8-bit form of the next rows, and the scales of the thread's units.
template <int DTYPE, bool VEC, int TPR, int U, int S> struct CodesAhead {
    using DealT = Deal<DTYPE, VEC>;
    static constexpr int E = DealT::E;
    static constexpr size_t BYTES = VEC ? (size_t)S * U * TPR * E : 0;
    uint8_t *own;
    uint32_t base;
    uint32_t next[VEC ? 1 : U][E / 2], now[VEC ? 1 : U][E / 2];
    __device__ __forceinline__ CodesAhead(uint8_t *smem, int t) : own(smem + t * E), base(smem_address(own)) {}
    __device__ __forceinline__ void start(int slot, const uint8_t *row, int t, int32_t units, int32_t D)
    {
#pragma unroll
        for (int k = 0; k < U; ++k)
            if (t + k * TPR < units) {
                if constexpr (VEC)
                    copy_async<E>(base + (slot * U + k) * (TPR * E), row + (size_t)(t + k * TPR) * E);
                else
                    DealT::load_codes(row, t + k * TPR, D, next[k]);
            }
    }
    __device__ __forceinline__ void take()
    {
#pragma unroll
        for (int k = 0; k < (VEC ? 0 : U); ++k)
#pragma unroll
            for (int e = 0; e < E / 2; ++e) now[k][e] = next[k][e];
    }
    __device__ __forceinline__ void centred(int slot, int k, float scale, float2 minus_mean, float2 (&c)[E / 2]) const
    {
        uint32_t q[E / 2];
        if constexpr (!VEC) {
#pragma unroll
            for (int e = 0; e < E / 2; ++e) q[e] = now[k][e];
        } else {
            const uint32_t *at = reinterpret_cast<const uint32_t *>(own + (slot * U + k) * (TPR * E));
            uint32_t lo, hi = 0;
            if constexpr (E == 8) {
                const uint2 both = *reinterpret_cast<const uint2 *>(at);
                lo = both.x, hi = both.y;
            } else {
                lo = *at;
            }
            q[0] = lo & 0xffffu, q[1] = lo >> 16;
            if constexpr (E == 8) q[2] = hi & 0xffffu, q[3] = hi >> 16;
        }
        // a code times a power of two is exact: one rounding, that of the difference
        const float2 down = make_float2(scale, scale);
#pragma unroll
        for (int e = 0; e < E / 2; ++e) c[e] = __ffma2_rn(halves_of(q[e]), down, minus_mean);
    }
};

// Mean, rstd and the scales of a warp's blocks, for the next rows: one four-byte copy per word and warp, each by a lane of its own
// (loaded into registers a row ahead they held the loop up; copied by every lane for itself each copy takes 32 shared-memory
// cycles.  16384 x 4096: 28 us more either way).  A scale is a byte: the aligned word around it is copied.
template <typename DealT, bool PACKED, int TPR, int U, int S> struct ScalarsAhead {
    static constexpr int LANES = DealT::BLOCK_LANES, PER_UNIT = 32 / LANES;      // blocks that a warp's 32 units span
    static constexpr int WORDS = 2 + (PACKED ? U * PER_UNIT : 0);
    static_assert(WORDS <= 32, "one lane per word");
    static constexpr size_t BYTES = ((size_t)S * (TPR / 32) * WORDS * 4 + 15) / 16 * 16;      // what follows starts on 16 bytes again
    uint32_t *own;                   // the warp's words in slot 0
    __device__ __forceinline__ ScalarsAhead(uint8_t *smem, int t) : own(reinterpret_cast<uint32_t *>(smem) + t / 32 * WORDS) {}
    static __device__ __forceinline__ int32_t block_of(int t, int k, int j) { return ((t & ~31) + k * TPR) / LANES + j; }
    __device__ __forceinline__ uint32_t *word(int slot, int i) const { return own + slot * (TPR / 32 * WORDS) + i; }
    __device__ __forceinline__ void start(int slot, const float *mean, const float *rstd, const uint8_t *scales, int t, int32_t units)
    {
        const int lane = t & 31;
        const void *src = lane == 0 ? mean : rstd;
        bool has = lane < 2;
        if (PACKED && lane >= 2 && lane < WORDS) {
            const int32_t block = block_of(t, (lane - 2) / PER_UNIT, (lane - 2) % PER_UNIT);
            has = block * LANES < units;
            src = reinterpret_cast<const void *>((uintptr_t)(scales + block) & ~(uintptr_t)3);
        }
        if (has) copy_async<4>(smem_address(word(slot, lane)), src);
    }
    // after the copies have been waited for and the warp has met
    __device__ __forceinline__ float get(int slot, int i) const { return __uint_as_float(*word(slot, i)); }
    __device__ __forceinline__ float scale(int slot, int k, const uint8_t *scales, int t) const
    {
        if constexpr (PACKED) {
            const int j = (t & 31) / LANES;
            const uint32_t at = (uint32_t)(uintptr_t)(scales + block_of(t, k, j)) & 3u;
            return scale_down(__byte_perm(*word(slot, 2 + k * PER_UNIT + j), 0, 0x4440u | at));
        }
        return 1.0f;
    }
};

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

// TPR threads hold one row, 32 values each (16 in the scalar deal, whose rows ahead sit in registers); below 128 threads a CTA
// takes several rows at a time.
template <int TPR> __host__ __device__ constexpr int norm_threads() { return TPR < 128 ? 128 : TPR; }
template <bool VEC> __host__ __device__ constexpr int norm_values() { return VEC ? 32 : 16; }
template <int DTYPE, bool VEC> __host__ __device__ constexpr int norm_units() { return norm_values<VEC>() / (VEC && DTYPE != PPOW_F32 ? 8 : 4); }
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

// Column sums over the CTAs' shares, in a fixed order: 32 columns by JOIN_GROUPS groups of shares per CTA.
constexpr int JOIN_GROUPS = 16;
__global__ void __launch_bounds__(32 * JOIN_GROUPS) norm_join_kernel(const float *__restrict__ partial, int32_t shares, int32_t D,
                                                                     int32_t param_dtype, void *grad_weight, void *grad_bias)
{
    __shared__ float group[JOIN_GROUPS][32];
    const int lane = threadIdx.x & 31, g = threadIdx.x >> 5;
    const int32_t c = blockIdx.x * 32 + lane;        // column of dw, then of db
    wait_for_previous_kernel();
    float sum = 0.0f;
    if (c < 2 * D) {
        const float *p = partial + c;
        int32_t s = g;
        for (; s + 7 * JOIN_GROUPS < shares; s += 8 * JOIN_GROUPS) {
            float v[8];
#pragma unroll
            for (int i = 0; i < 8; ++i) v[i] = p[(size_t)(s + i * JOIN_GROUPS) * 2 * D];
#pragma unroll
            for (int i = 0; i < 8; ++i) sum += v[i];
        }
        for (; s < shares; s += JOIN_GROUPS) sum += p[(size_t)s * 2 * D];
    }
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
