// What kernels over the rows of an activation share: storage types, how a row is dealt out to threads, the 8-bit form of a row,
// and rows on their way into shared memory ahead of their use.
#pragma once

#include "../../include/ppow.h"
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

// TPR threads hold one row, 32 values each (16 in the scalar deal, whose rows ahead sit in registers); below 128 threads a CTA
// takes several rows at a time.
template <int TPR> __host__ __device__ constexpr int norm_threads() { return TPR < 128 ? 128 : TPR; }
template <bool VEC> __host__ __device__ constexpr int norm_values() { return VEC ? 32 : 16; }
template <int DTYPE, bool VEC> __host__ __device__ constexpr int norm_units() { return norm_values<VEC>() / (VEC && DTYPE != PPOW_F32 ? 8 : 4); }

// Column sums over the CTAs' shares [shares][columns], in a fixed order: a CTA takes 32 columns by JOIN_GROUPS groups of shares.
// The total of the lane's column, valid in group 0.
constexpr int JOIN_GROUPS = 16;
__device__ __forceinline__ float column_total(const float *__restrict__ partial, int32_t shares, int32_t columns, int32_t c)
{
    __shared__ float group[JOIN_GROUPS][32];
    const int lane = threadIdx.x & 31, g = threadIdx.x >> 5;
    float sum = 0.0f;
    if (c < columns) {
        const float *p = partial + c;
        int32_t s = g;
        for (; s + 7 * JOIN_GROUPS < shares; s += 8 * JOIN_GROUPS) {
            float v[8];
#pragma unroll
            for (int i = 0; i < 8; ++i) v[i] = p[(size_t)(s + i * JOIN_GROUPS) * columns];
#pragma unroll
            for (int i = 0; i < 8; ++i) sum += v[i];
        }
        for (; s < shares; s += JOIN_GROUPS) sum += p[(size_t)s * columns];
    }
    group[g][lane] = sum;
    __syncthreads();
    sum = 0.0f;
    if (g == 0) {
#pragma unroll
        for (int i = 0; i < JOIN_GROUPS; ++i) sum += group[i][lane];
    }
    return sum;
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

}  // namespace

#define PPOW_BY_TYPE(dtype, vec, CALL)                                                                          \
    ((dtype) == PPOW_F32    ? ((vec) ? CALL(PPOW_F32, true) : CALL(PPOW_F32, false))                             \
     : (dtype) == PPOW_BF16 ? ((vec) ? CALL(PPOW_BF16, true) : CALL(PPOW_BF16, false))                           \
                            : ((vec) ? CALL(PPOW_F16, true) : CALL(PPOW_F16, false)))


}  // namespace ppow
