// Log-probability of given tokens straight from hidden states and the head's weight, and its gradient, without keeping
// the logits (the token terms of the objective of Sec. 4.1 and of the supervised loss of App. C.2):
//   z = h W^T / T,   lse = log sum_v exp z_v,   logp = z_y - lse,
//   dz_v = g/T ([v = y] - exp(z_v - lse)),   dh = dz W,   dW = dz^T h      (g: the gradient that arrives at logp).
//
// Steps of a call:
//   gather    live rows of `hidden` are copied to the front of a workspace array, in order, for dW in the order of their tokens
//             (masked rows may hold anything and cost no products, but the shares of a call's work are planned for all of its rows;
//             rows of any stride and alignment become tiles)
//   forward   logits by tiles of 256 tokens x 256 vocabulary entries; each tile leaves a maximum and a sum of exponentials
//             per row; `merge` joins them in float64
//   backward  per piece of the vocabulary: logits again, dz rounded to the operands' 16-bit type; dW of the piece, and the
//             piece's share of dh added to float32 sums; `finish` rounds dh once
// All products run in one kernel template on tcgen05 (ppow_mma.cuh).
#include "../../include/ppow.h"
#include "ppow_checked.cuh"
#include "ppow_device.cuh"
#include "ppow_mma.cuh"

#include <cuda_bf16.h>

#include <atomic>
#include <math.h>

namespace ppow {

constexpr float LOG2E = 1.4426950408889634f;
constexpr int TILE = 256;            // rows and columns of an output tile (a pair of CTAs)
constexpr int HALF_TILE = 128;       // rows of A that one CTA holds
constexpr int BK = 64;               // products' inner step per pipeline stage: one 128-byte swizzle row
constexpr uint32_t A_BYTES = HALF_TILE * BK * 2;           // 16 KB
constexpr int MMA_THREADS = 320;     // producer warp, issuing warp, eight epilogue warps; for dW one more, for the remainders
constexpr int PAIRS = 74;            // pairs of SMs that the shares of an inner axis are planned for
constexpr int MAX_PAIRS = 128;       // pairs that a launch uses at most

// Columns of a tile: 256, or for few tokens the tokens themselves (16, 32, 64 or 128), with W taking the 256 rows.
template <int N> __host__ __device__ constexpr uint32_t stage_bytes() { return A_BYTES + N / 2 * BK * 2; }
template <int N> __host__ __device__ constexpr int stage_count()
{
    return N == 256 ? 6 : N == 128 ? 8 : N == 64 ? 10 : N == 32 ? 11 : 12;    // 192 to 204 KB
}
enum Product {
    LOGITS_SUM,   // rows x W^T: maximum and sum of exponentials per row and tile
    LOGITS_GRAD,  // rows x W^T: dz of a piece of the vocabulary
    GRAD_HIDDEN,  // dz x W: the piece's share of dh
    GRAD_WEIGHT   // dz^T x rows: dW of the piece
};

// Steps that a product is summed over in Tensor Memory before the sum moves on to registers: the tensor cores' additions cut off
// what does not fit, and logp and lse show it (with 16 steps 1.4e-6 of logp in bf16, twice that in f16; with 4 a quarter).
//   Logits of the forward pass: up to 1024 wide half of the steps, then a third, 4 to 16; few tokens 8 at most, or 4.  That keeps
//   logp about as exact as a float32 product has it: 300 tokens x 1024 in bf16 at T = 0.7 1.2e-6 (in one sum 2.1e-6, by a float32
//   product 0.8e-6), and costs 2048 x 1024 x 32000 112 -> 119 us, x 2048 214 -> 220; 4096 wide it is 16 steps, 3.6 % (8: 8 %).
//   dW: its sum runs over the tokens, and where its terms have one sign (every softmax's has, so the states' mean is enough) each
//   65536 of them took 4e-4 off it, of 2^20 0.7 %; with parts of 8192 tokens it is under 1e-4.  (Gradient of 262144 x 1024 x 4096:
//   12.5 ms either way.)
constexpr int32_t WEIGHT_PART_STEPS = 128;
inline int32_t logit_part_steps(int32_t width, int32_t columns)
{
    const int32_t steps = (width + BK - 1) / BK, share = steps <= 16 ? (steps + 1) / 2 : (steps + 2) / 3;
    const int32_t most = columns == 256 ? 16 : columns == 128 ? 8 : 4;
    return share < 4 ? 4 : share < most ? share : most;
}
// Tiles of 16-bit results leave through shared memory: a box of 128 rows x 64 columns for each half of the columns.
constexpr uint32_t BOX_BYTES = HALF_TILE * 128;
template <int N> __host__ __device__ constexpr size_t mma_smem()
{
    return 1024 + (size_t)stage_count<N>() * stage_bytes<N>() + (N == 256 ? 2 * BOX_BYTES : 0) + 512;
}

constexpr int GATHER_THREADS = 256, EARLY = 4;
constexpr int GATHER_ROWS_MAX = 1024, GATHER_CTAS = 1024;
constexpr size_t HEADER_BYTES = 256;
constexpr size_t DZ_BYTES = 512u << 20;      // a piece of dz holds at most this much
constexpr int32_t PIECE_TILES = 1024;        // and this many vocabulary tiles: dh is summed over a piece (see below)
constexpr int32_t MAX_TOKENS = 1 << 20, MAX_VOCAB = 1 << 22, MAX_WIDTH = 1 << 16;

// First bytes of the workspace; error_flags sits where ppow_read_error_flags looks for it.
struct HeadHeader {
    unsigned int unused;
    unsigned int error_flags;
    int32_t live;          // live rows
    float out_scale;       // factor of dW (f16: undoes the power of two that the rows were brought to)
    int32_t splits;        // shares of the inner axis of dh
};

// The live rows, from `first` to before `end`, whose tokens lie in one tile of the vocabulary (both 0: none).
struct TokenRows {
    int32_t first, end;
};

// Arrays of the workspace, all indexed by live row.
struct HeadRows {
    HeadHeader *header;
    int32_t *source;       // row of `hidden`; null: the same
    int32_t *token;
    float *mult;           // dz = mult * (softmax - onehot)
    float *lse2;           // normaliser in log2 units
    float *row_scale;      // dh = row_scale * (dz W)
    float *target;         // p - 1 at the token
    float *residual;       // what the rounding of dz at the token left over
    TokenRows *rows_of;    // backward, per tile of the vocabulary
    void *rows;            // [padded, D] hidden states
    void *scaled;          // f16 backward: the same times a power of two per row
};

__device__ __forceinline__ void fault(HeadHeader *h, unsigned int bit) { atomicOr(&h->error_flags, bit); }
// A kernel of this call gave a wait up: its results are not there, and what is made of them is NaN.
__device__ __forceinline__ bool gave_up(const HeadHeader *h) { return h->error_flags & PPOW_FLAG_DEVICE_TIMEOUT; }

template <bool BF16>
__device__ __forceinline__ uint32_t pack2(float a, float b)
{
    if (BF16) {
        const __nv_bfloat162 h = __floats2bfloat162_rn(a, b);
        return *reinterpret_cast<const uint32_t *>(&h);
    }
    const __half2 h = __floats2half2_rn(a, b);
    return *reinterpret_cast<const uint32_t *>(&h);
}

template <bool BF16>
__device__ __forceinline__ float2 unpack2(uint32_t w)
{
    if (BF16) return make_float2(bf16_lo(w), bf16_hi(w));
    return __half22float2(*reinterpret_cast<const __half2 *>(&w));
}

// x minus x rounded to 16 bits
template <bool BF16>
__device__ __forceinline__ float rounding_of(float x)
{
    return x - (BF16 ? __bfloat162float(__float2bfloat16_rn(x)) : __half2float(__float2half_rn(x)));
}

// ---- the token's own product ---------------------------------------------------------------------------
// 1 - p of a token that the drafter is nearly sure of is a small difference, and log p close to 0 too: an error d of the token's
// logit appears in them as d / (1 - p).  Tensor cores cut sums off towards zero, and over a product whose terms have one sign that
// adds up (4096 wide, logits near 14: 1e-4, of the gradient of a token with p = 0.9995 a third to all).  So the token's logit is
// computed apart: float32 over the 8 products of a unit, float64 from there on.  The calling lane's share: units first, first + step, ...
template <bool BF16>
__device__ __forceinline__ double token_product(const uint16_t *h, const uint16_t *w, int32_t units, int32_t first, int32_t step)
{
    double sum = 0.0;
#pragma unroll 4
    for (int32_t u = first; u < units; u += step) {
        const uint4 a = *(reinterpret_cast<const uint4 *>(h) + u), b = *(reinterpret_cast<const uint4 *>(w) + u);
        const uint32_t x[4] = {a.x, a.y, a.z, a.w}, y[4] = {b.x, b.y, b.z, b.w};
        float s = 0.0f;
#pragma unroll
        for (int i = 0; i < 4; ++i) {
            const float2 p = unpack2<BF16>(x[i]), q = unpack2<BF16>(y[i]);
            s = fmaf(p.x, q.x, s);
            s = fmaf(p.y, q.y, s);
        }
        sum += (double)s;
    }
    return sum;
}

// ---- the order of the gradient's rows ----------------------------------------------------------------
// By token, and with the same token as they come: what dW needs of the rows of an entry then lies side by side, and neither
// depends on the order in which threads get there.  A row's place is the number of live rows with a smaller token, or with the same
// one and a smaller index.  Up to ORDER_COUNTED tokens every gather CTA counts that for its rows over all tokens; that is T^2
// comparisons, so behind it four small kernels make lists of each token's rows, in any order, in which a row then counts its
// predecessors.  (Whole gradients of T x 64 x 1000 by lists: 1.5 us more at T = 4096, 12 us less at 8192.)
constexpr int32_t ORDER_COUNTED = 4096;
struct RowOrder {
    int32_t *count, *first;         // per vocabulary entry: live rows, and the place of the first
    int32_t *slot;                  // per row: its place in the token's list
    int32_t *list;                  // rows, by token
};
__device__ __forceinline__ bool grad_live(int32_t y, float g, int32_t V) { return y >= 0 && y < V && !(g == 0.0f); }

constexpr int ORDER_THREADS = 256;
__global__ void __launch_bounds__(ORDER_THREADS) head_order_clear_kernel(RowOrder order, int32_t V)
{
    allow_next_kernel();
    wait_for_previous_kernel();
    for (int32_t v = blockIdx.x * ORDER_THREADS + threadIdx.x; v < V; v += gridDim.x * ORDER_THREADS) order.count[v] = 0;
}
__global__ void __launch_bounds__(ORDER_THREADS) head_order_count_kernel(RowOrder order, const int32_t *tokens, const float *grad, int32_t T, int32_t V)
{
    allow_next_kernel();
    wait_for_previous_kernel();
    for (int32_t r = blockIdx.x * ORDER_THREADS + threadIdx.x; r < T; r += gridDim.x * ORDER_THREADS)
        if (grad_live(tokens[r], grad[r], V)) order.slot[r] = atomicAdd(order.count + tokens[r], 1);
}
// A CTA takes `share` entries, a multiple of its threads; it adds up all counts before them itself instead of waiting for its neighbour.
constexpr int SCAN_THREADS = 512;
__global__ void __launch_bounds__(SCAN_THREADS) head_order_scan_kernel(RowOrder order, int32_t V, int32_t share)
{
    __shared__ int32_t sums[SCAN_THREADS / 32];
    const int tid = threadIdx.x, lane = tid & 31, warp = tid >> 5;
    allow_next_kernel();
    wait_for_previous_kernel();
    const int32_t begin = blockIdx.x * share, end = min(begin + share, V);
    int32_t carry = 0;
#pragma unroll 8
    for (int32_t v = tid; v < begin; v += SCAN_THREADS) carry += order.count[v];
    carry = __reduce_add_sync(0xffffffffu, carry);
    if (lane == 0) sums[warp] = carry;
    __syncthreads();
    carry = 0;
#pragma unroll
    for (int i = 0; i < SCAN_THREADS / 32; ++i) carry += sums[i];
    for (int32_t v0 = begin; v0 < end; v0 += SCAN_THREADS) {
        const int32_t v = v0 + tid, own = v < end ? order.count[v] : 0;
        int32_t upto = own;
#pragma unroll
        for (int o = 1; o < 32; o <<= 1) {
            const int32_t x = __shfl_up_sync(0xffffffffu, upto, o);
            if (lane >= o) upto += x;
        }
        __syncthreads();
        if (lane == 31) sums[warp] = upto;
        __syncthreads();
        int32_t before = 0, all = 0;
#pragma unroll
        for (int i = 0; i < SCAN_THREADS / 32; ++i) {
            before += i < warp ? sums[i] : 0;
            all += sums[i];
        }
        if (v < end) order.first[v] = carry + before + upto - own;
        carry += all;
    }
}
__global__ void __launch_bounds__(ORDER_THREADS) head_order_list_kernel(RowOrder order, const int32_t *tokens, const float *grad, int32_t T, int32_t V)
{
    allow_next_kernel();
    wait_for_previous_kernel();
    for (int32_t r = blockIdx.x * ORDER_THREADS + threadIdx.x; r < T; r += gridDim.x * ORDER_THREADS)
        if (grad_live(tokens[r], grad[r], V)) order.list[order.first[tokens[r]] + order.slot[r]] = r;
}

// ---- gather -----------------------------------------------------------------------------------------
struct GatherJob {
    const uint16_t *hidden;
    const int32_t *tokens;
    const float *lse, *grad;
    float *logp_out, *lse_out;      // forward: masked rows receive 0
    uint16_t *grad_hidden;          // backward: masked rows receive 0 (may be null)
    int64_t stride;
    int32_t T, D, V, rows_per_cta;
    int32_t few;                    // token columns of a call of few tokens, else 0
    bool by_token;                  // backward: rows in the order of their tokens, for dW
    RowOrder order;                 // of many tokens; null: counted here
    int32_t d_tiles, piece_steps;   // backward: what the shares of dh follow from; steps of the shortest piece
    const uint16_t *weight;         // backward
    int64_t weight_stride;
    double exact_inv_temperature;
    float inv_temperature;
    bool vec;                       // rows start on 16-byte boundaries
};

// Shares of the inner axis of dh: `tiles` output tiles times the shares should fill whole rounds of the pairs.  A share is
// at least eight steps long, and each one costs a pass over its sums (2 % of a round is about what that measures).  `steps`
// are those of the shortest piece of the vocabulary, so that no share of any piece is empty.  The host runs the same rule.
constexpr int32_t SPLIT_TILES = 8 * PAIRS;      // tiles x shares where there is more than one share
__host__ __device__ __forceinline__ bool split_allowed(int32_t s, int64_t tiles, int32_t steps)
{
    return s == 1 || (s <= PAIRS && s * 8 <= steps && s * tiles <= SPLIT_TILES);
}
__host__ __device__ __forceinline__ float split_cost(int32_t s, int64_t tiles)
{
    return (float)((tiles * s + PAIRS - 1) / PAIRS) / (float)s * fmaf(0.02f, (float)(s < 11 ? s - 1 : 10), 1.0f);
}
__device__ __forceinline__ int32_t split_count(int64_t tiles, int32_t steps)      // one warp, a candidate per lane and turn
{
    float best_cost = INFINITY;
    uint32_t best = 1;
    for (int32_t s = 1 + (int32_t)(threadIdx.x & 31); split_allowed(s, tiles, steps); s += 32) {
        const float cost = split_cost(s, tiles);
        if (cost < best_cost) {
            best_cost = cost;
            best = (uint32_t)s;
        }
    }
    const uint32_t lowest = __reduce_min_sync(0xffffffffu, __float_as_uint(best_cost));        // costs are positive
    return (int32_t)__reduce_min_sync(0xffffffffu, __float_as_uint(best_cost) == lowest ? best : ~0u);
}

// mult of a row, and for f16 the split into a factor near 2^15 and a power of two: dz of a row whose gradient is small
// would fall below f16's smallest values.
// (The states that dW multiplies are brought down by the row's power against the largest's instead: a row 2^14 and more below the
// largest loses bits of its share of dW, which is as far below the largest rows' shares.)
__device__ __forceinline__ float row_mult(float g, float inv_temperature) { return -g * inv_temperature; }
__device__ __forceinline__ int row_exponent(float mult, int top)
{
    int e = top;
    if (isfinite(mult) && mult != 0.0f) frexpf(mult, &e);
    return e;
}

// Every CTA looks at all T tokens (4 bytes each, from L2) to learn where its rows go, instead of waiting for a scan kernel.
template <bool BACKWARD, bool SCALED>
__global__ void __launch_bounds__(GATHER_THREADS) head_gather_kernel(GatherJob job, HeadRows out)
{
    constexpr int COUNTED = ORDER_COUNTED / GATHER_CTAS;         // rows of a CTA that counts their places
    __shared__ int32_t part[4 + COUNTED][GATHER_THREADS / 32];
    __shared__ int32_t dest[GATHER_ROWS_MAX];
    const int tid = threadIdx.x, lane = tid & 31, warp = tid >> 5;
    wait_for_previous_kernel();
    const int32_t r0 = (int32_t)min((int64_t)blockIdx.x * job.rows_per_cta, (int64_t)job.T);
    const int32_t n = min(job.rows_per_cta, job.T - r0);
    // rows that start on 16-byte boundaries are on their way before it is known where they go
    const int32_t units = job.D / 8, all = n * units;
    uint4 early[EARLY];
    if (job.vec) {
#pragma unroll
        for (int j = 0; j < EARLY; ++j) {
            const int32_t i = tid + j * GATHER_THREADS;
            if (i < all) early[j] = __ldg(reinterpret_cast<const uint4 *>(job.hidden + (size_t)(r0 + i / units) * job.stride) + i % units);
        }
    }
    if (BACKWARD)
        for (int32_t i = blockIdx.x * GATHER_THREADS + tid; i < (job.V + TILE - 1) / TILE; i += gridDim.x * GATHER_THREADS)
            out.rows_of[i] = {0, 0};
    auto live = [&](int32_t y, float g) { return BACKWARD ? grad_live(y, g, job.V) : y >= 0; };
    const bool counts = BACKWARD && job.by_token && !job.order.count;
    int32_t own[COUNTED], less[COUNTED] = {};                    // the CTA's rows' tokens, -1: masked; live rows in front of them
#pragma unroll
    for (int k = 0; k < COUNTED; ++k) own[k] = counts && k < n && live(job.tokens[r0 + k], job.grad[r0 + k]) ? job.tokens[r0 + k] : -1;
    int32_t before = 0, total = 0, top = -1000, range = 0;
    for (int32_t i = tid; i < job.T; i += GATHER_THREADS) {
        const int32_t y = job.tokens[i];
        const float g = BACKWARD ? job.grad[i] : 1.0f;
        const bool ok = live(y, g);
        total += ok;
        before += ok && i < r0;
        if (counts) {
#pragma unroll
            for (int k = 0; k < COUNTED; ++k) less[k] += ok && y < own[k] + (i < r0 + k ? 1 : 0);
        }
        range |= y >= job.V;
        if (SCALED && ok) {
            const float m = row_mult(g, job.inv_temperature);
            if (isfinite(m) && m != 0.0f) top = max(top, row_exponent(m, 0));
        }
    }
    before = __reduce_add_sync(0xffffffffu, before);
    total = __reduce_add_sync(0xffffffffu, total);
    top = __reduce_max_sync(0xffffffffu, top);
    range = __reduce_or_sync(0xffffffffu, range);
    if (lane == 0) {
        part[0][warp] = before;
        part[1][warp] = total;
        part[2][warp] = top;
        part[3][warp] = range;
    }
    if (counts) {
#pragma unroll
        for (int k = 0; k < COUNTED; ++k) {
            less[k] = __reduce_add_sync(0xffffffffu, less[k]);
            if (lane == 0) part[4 + k][warp] = less[k];
        }
    }
    __syncthreads();
    before = total = range = 0;
    top = -1000;
#pragma unroll
    for (int w = 0; w < GATHER_THREADS / 32; ++w) {
        before += part[0][w];
        total += part[1][w];
        top = max(top, part[2][w]);
        range |= part[3][w];
    }
    if (top == -1000) top = 0;
    if (blockIdx.x == 0 && tid == 0) {
        out.header->error_flags = range ? (unsigned)PPOW_FLAG_TOKEN_RANGE : 0u;
        out.header->live = total;
        out.header->out_scale = SCALED ? ldexpf(1.0f, top - 15) : 1.0f;
    }
    if (BACKWARD && blockIdx.x == 0 && warp == 1) {
        const int64_t tiles = (int64_t)(job.few ? 1 : max(1, (total + TILE - 1) / TILE)) * job.d_tiles;
        const int32_t splits = split_count(tiles, job.piece_steps);
        if (lane == 0) out.header->splits = splits;
    }
    if (BACKWARD && job.by_token && !counts) {
        for (int32_t k = warp; k < n; k += GATHER_THREADS / 32) {
            const int32_t r = r0 + k, y = job.tokens[r];
            int32_t place = -1;
            if (live(y, job.grad[r])) {
                const int32_t first = job.order.first[y], rows = job.order.count[y];
                int32_t less = 0;
                for (int32_t i = lane; i < rows; i += 32) less += job.order.list[first + i] < r;
                place = first + __reduce_add_sync(0xffffffffu, less);
            }
            if (lane == 0) dest[k] = place;
        }
    } else if (counts) {
#pragma unroll
        for (int k = 0; k < COUNTED; ++k)
            if (tid == 0 && k < n) {
                int32_t place = 0;
#pragma unroll
                for (int w = 0; w < GATHER_THREADS / 32; ++w) place += part[4 + k][w];
                dest[k] = own[k] < 0 ? -1 : place;
            }
    } else if (warp == 0) {
        int32_t next = before;
        for (int32_t k = 0; k < n; k += 32) {
            const int32_t r = min(r0 + k + lane, job.T - 1);
            const bool ok = k + lane < n && live(job.tokens[r], BACKWARD ? job.grad[r] : 1.0f);
            const unsigned m = __ballot_sync(0xffffffffu, ok);
            if (k + lane < n) dest[k + lane] = ok ? next + __popc(m & ((1u << lane) - 1u)) : -1;
            next += __popc(m);
        }
    }
    __syncthreads();

    allow_next_kernel();
    // per row: what the products need to know of it
    for (int32_t k = tid; k < n; k += GATHER_THREADS) {
        const int32_t r = r0 + k, d = dest[k];
        if (d < 0) {
            if (!BACKWARD) job.logp_out[r] = job.lse_out[r] = 0.0f;
            continue;
        }
        if (!PPOW_CHECK(d < total && (BACKWARD || d <= r), 501, nullptr)) continue;
        out.source[d] = r;
        out.token[d] = job.tokens[r];
        if (BACKWARD) {
            float m = row_mult(job.grad[r], job.inv_temperature), scale = 1.0f;
            if (SCALED) {
                const int e = row_exponent(m, top);
                m = ldexpf(m, 15 - e);
                scale = ldexpf(1.0f, e - 15);
            }
            out.mult[d] = m;
            out.row_scale[d] = scale;
            out.lse2[d] = job.lse[r] * LOG2E;
        }
    }
    // the rows themselves, by 16-byte units
    auto put = [&](int32_t i, uint4 x) {
        const int32_t k = i / units, u = i % units, r = r0 + k, d = dest[k];
        if (d < 0) {
            if (BACKWARD && job.grad_hidden) reinterpret_cast<uint4 *>(job.grad_hidden + (size_t)r * job.D)[u] = make_uint4(0, 0, 0, 0);
            return;
        }
        reinterpret_cast<uint4 *>((uint16_t *)out.rows + (size_t)d * job.D)[u] = x;
        if (SCALED) {
            const float down = ldexpf(1.0f, row_exponent(row_mult(job.grad[r], job.inv_temperature), top) - top);
            uint32_t w[4] = {x.x, x.y, x.z, x.w};
#pragma unroll
            for (int q = 0; q < 4; ++q) {
                const __half2 h = *reinterpret_cast<__half2 *>(&w[q]);
                const __half2 s = __floats2half2_rn(__low2float(h) * down, __high2float(h) * down);
                w[q] = *reinterpret_cast<const uint32_t *>(&s);
            }
            reinterpret_cast<uint4 *>((uint16_t *)out.scaled + (size_t)d * job.D)[u] = make_uint4(w[0], w[1], w[2], w[3]);
        }
    };
    if (job.vec) {
#pragma unroll
        for (int j = 0; j < EARLY; ++j)
            if (tid + j * GATHER_THREADS < all) put(tid + j * GATHER_THREADS, early[j]);
        for (int32_t i = tid + EARLY * GATHER_THREADS; i < all; i += GATHER_THREADS)
            put(i, __ldg(reinterpret_cast<const uint4 *>(job.hidden + (size_t)(r0 + i / units) * job.stride) + i % units));
    } else {
        for (int32_t i = tid; i < all; i += GATHER_THREADS) {
            const uint16_t *src = job.hidden + (size_t)(r0 + i / units) * job.stride + i % units * 8;
            uint32_t w[4];
#pragma unroll
            for (int q = 0; q < 4; ++q) w[q] = (uint32_t)src[2 * q] | ((uint32_t)src[2 * q + 1] << 16);
            put(i, make_uint4(w[0], w[1], w[2], w[3]));
        }
    }
    if (BACKWARD) {
        // p - 1 at the token; of a few rows by all warps together, else a warp per row
        __shared__ double shares[COUNTED][GATHER_THREADS / 32];
        const bool together = n <= COUNTED;
        __syncthreads();
        for (int32_t k = together ? 0 : warp; k < n; k += together ? 1 : GATHER_THREADS / 32) {
            const int32_t d = dest[k];
            if (d < 0) continue;
            const int32_t r = r0 + k;
            const double z = warp_sum_f64(token_product<!SCALED>((const uint16_t *)out.rows + (size_t)d * job.D,
                                                                 job.weight + (size_t)job.tokens[r] * job.weight_stride, units,
                                                                 together ? tid : lane, together ? GATHER_THREADS : 32));
            if (lane != 0) continue;
            if (together)
                shares[k][warp] = z;
            else
                out.target[d] = expm1f((float)(z * job.exact_inv_temperature - (double)job.lse[r]));
        }
        if (together) {
            __syncthreads();
            if (tid < n && dest[tid] >= 0) {
                double z = 0.0;
#pragma unroll
                for (int w = 0; w < GATHER_THREADS / 32; ++w) z += shares[tid][w];
                out.target[dest[tid]] = expm1f((float)(z * job.exact_inv_temperature - (double)job.lse[r0 + tid]));
            }
        }
    }
    // the last tile's rows behind the live ones are zeros: they are products' operands too
    const int32_t padded = job.few ? job.few : max(TILE, (total + TILE - 1) / TILE * TILE);
    for (int32_t p = total + blockIdx.x; p < padded; p += gridDim.x) {
        if (tid == 0) {
            out.token[p] = -1;
            out.mult[p] = 0.0f;
            out.lse2[p] = 0.0f;
        }
        for (int32_t u = tid; u < units; u += GATHER_THREADS) {
            reinterpret_cast<uint4 *>((uint16_t *)out.rows + (size_t)p * job.D)[u] = make_uint4(0, 0, 0, 0);
            if (SCALED) reinterpret_cast<uint4 *>((uint16_t *)out.scaled + (size_t)p * job.D)[u] = make_uint4(0, 0, 0, 0);
        }
    }
}

// ---- the products -----------------------------------------------------------------------------------
struct ProductJob {
    HeadRows rows;
    float scale;            // log2(e) / temperature
    int32_t D, V;
    int32_t tokens;         // GRAD_WEIGHT: rows at most, masked ones with them
    int32_t part_steps;     // LOGITS_SUM, GRAD_WEIGHT: steps of a part of the sum
    int32_t v0, columns;    // the piece: vocabulary entries v0 .. v0 + columns - 1
    int32_t v_tiles, d_tiles;
    int32_t piece;          // row length of dz
    int32_t direct;         // LOGITS_SUM, few tokens: that many tokens, read where they lie (0: gathered)
    bool add;               // GRAD_HIDDEN: add to what the pieces before left
    int32_t parts;          // LOGITS_SUM: entries of `partial` per row
    float2 *partial;        // LOGITS_SUM: [live row][parts] maximum, sum (log2 units), without the token
    uint16_t *dz;           // [padded rows][piece]
    float *grad_rows;       // GRAD_HIDDEN: [splits][padded live rows][D]
};

struct Tile {
    int32_t row, col;       // first row of A and column of B, in elements of the product's own axes
    int32_t k0, k1;         // inner steps of BK
    int32_t index, split;   // tile along the vocabulary or the width; share of the inner axis
};

// What a launch works on: sizes that follow from the number of live rows.
struct Extent {
    int32_t live, row_tiles, splits;
};

template <int PRODUCT>
__device__ __forceinline__ int64_t tile_count(const ProductJob &job, const Extent &x)
{
    if (PRODUCT == GRAD_HIDDEN) return (int64_t)x.row_tiles * job.d_tiles * x.splits;
    if (PRODUCT == GRAD_WEIGHT) return (int64_t)job.v_tiles * job.d_tiles;
    return (int64_t)x.row_tiles * job.v_tiles;
}

// Logit tiles go through all rows for one strip of W, then the next strip: W comes from HBM once, the rows stay in L2.
// With few tokens there is one tile of them, the columns, and the rows are the vocabulary's or the width's.
template <int PRODUCT, bool FEW>
__device__ __forceinline__ Tile tile_at(const ProductJob &job, const Extent &e, int64_t t)
{
    Tile x;
    x.split = 0;
    if (PRODUCT == LOGITS_SUM || PRODUCT == LOGITS_GRAD) {
        x.index = (int32_t)(FEW ? t : t / e.row_tiles);
        const int32_t rows = (int32_t)(FEW ? 0 : t % e.row_tiles) * TILE, vocab = job.v0 + x.index * TILE;
        x.row = FEW ? vocab : rows;
        x.col = FEW ? 0 : vocab;
        x.k0 = 0;
        x.k1 = (job.D + BK - 1) / BK;
    } else if (PRODUCT == GRAD_HIDDEN) {
        x.index = (int32_t)(t % job.d_tiles);
        const int32_t u = (int32_t)(t / job.d_tiles);
        x.split = u / e.row_tiles;
        x.row = FEW ? x.index * TILE : (u % e.row_tiles) * TILE;
        x.col = FEW ? 0 : x.index * TILE;
        const int32_t steps = (job.columns + BK - 1) / BK;
        x.k0 = (int32_t)((int64_t)steps * x.split / e.splits);
        x.k1 = (int32_t)((int64_t)steps * (x.split + 1) / e.splits);
    } else {
        x.index = (int32_t)(t % job.d_tiles);
        x.row = (int32_t)(t / job.d_tiles) * TILE;
        x.col = x.index * TILE;
        x.k0 = 0;
        x.k1 = max(1, (e.live + BK - 1) / BK);    // no live row: one step over rows of zeros
    }
    return x;
}

// Accumulators that a tile's sum passes through, one after the other.  The issuing thread and the epilogue warps both count by
// it: every tile takes one at least, so that the two sides agree on buffer and phase whatever its steps are.
template <bool PARTS> __device__ __forceinline__ int32_t part_count(const ProductJob &job, const Tile &x)
{
    return PARTS ? max(1, (x.k1 - x.k0 + job.part_steps - 1) / job.part_steps) : 1;
}

// ---- epilogues: one warp, 32 rows of the tile's accumulator (its Tensor Memory lanes), half of the columns --------
// Loads run one step ahead of the arithmetic; `release` hands the accumulator back as soon as the last one is in.
template <int CHUNKS, int WIDTH, typename R, typename F>
__device__ __forceinline__ void for_chunks(uint32_t src, R &&release, F &&f)
{
    uint32_t w[2][WIDTH];
    tmem_load(src, w[0]);
#pragma unroll
    for (int i = 0; i < CHUNKS; ++i) {
        tmem_wait(w[i & 1]);
        if (i + 1 < CHUNKS)
            tmem_load(src + (i + 1) * WIDTH, w[(i + 1) & 1]);
        else
            release();
        f(i * WIDTH, w[i & 1]);
    }
}

// What a row's epilogue needs of its token, loaded before the tile is waited for.
struct RowData {
    int32_t token;
    float mult, lse2, target;
};

// 32 columns (from column c of the half's 128) of the calling thread's row into the half's box, in the 128-byte swizzle: the
// 16-byte unit i of row r sits at i ^ (r & 7), so that the 32 rows of a warp's store spread over all banks.  Every second
// call the box is full and one thread hands it to the copy engine, at column x0 + 64 * (c / 64) and row y of `map`.
__device__ __forceinline__ void put_box(uint32_t box, int32_t in_tile, int half, int c, const uint32_t (&o)[16], const CUtensorMap *map,
                                        int32_t x0, int32_t y, bool inside)
{
    const uint32_t r = in_tile % HALF_TILE, threads = 128, id = 1 + half;
    const bool first = r == 0;
    const uint32_t row = box + half * BOX_BYTES + r * 128;
    if (c % 64 == 0) {
        if (first) tma_store_wait_read();
        named_barrier(id, threads);
    }
#pragma unroll
    for (int i = 0; i < 4; ++i)
        store_shared16(row + ((((c % 64) / 8 + i) ^ (r & 7)) << 4), o[4 * i], o[4 * i + 1], o[4 * i + 2], o[4 * i + 3]);
    if (c % 64 == 32) {
        fence_for_copy_engine();
        named_barrier(id, threads);
        if (first && inside) tma_store(map, box + half * BOX_BYTES, x0 + c / 64 * 64, y);
    }
}

// The gradient's rows lie in the order of their tokens: those at either end of a tile's rows say so.
__device__ __forceinline__ void note_token(const ProductJob &job, const Extent &e, int32_t token, int32_t row)
{
    const int32_t before = row > 0 ? job.rows.token[row - 1] : -1, behind = row + 1 < e.live ? job.rows.token[row + 1] : -1;
    if (before < token / TILE * TILE) job.rows.rows_of[token / TILE].first = row;
    if (behind < 0 || behind / TILE > token / TILE) job.rows.rows_of[token / TILE].end = row + 1;
}

// rows: tokens, columns: vocabulary
template <int PRODUCT, bool BF16, bool PARTS, typename R>
__device__ __forceinline__ void epilogue_many(const ProductJob &job, const Extent &e, const Tile &x, const RowData &own, uint32_t src,
                                              int32_t in_tile, int half, const CUtensorMap *map_out, uint32_t box,
                                              uint32_t (&w)[TILE / 64][32], R &&release)
{
    constexpr int COLS = TILE / 2;
    const int32_t row = x.row + in_tile;                     // a live row, or for GRAD_WEIGHT an entry of the piece
    const int32_t first = half * COLS;                       // this warp's columns of the tile
    [[maybe_unused]] const int lane = threadIdx.x & 31;
    src += first;
    [[maybe_unused]] unsigned int *flags = &job.rows.header->error_flags;
    if (PRODUCT == LOGITS_SUM) {
        const int32_t left = min(TILE, job.V - x.col) - first;   // columns that exist
        const int32_t at = own.token - x.col - first;            // padded rows hold a negative token
        // all 128 columns at once: one maximum, no rescaling; the token's term comes from elsewhere
        if (left < COLS || (at >= 0 && at < COLS)) {
#pragma unroll
            for (int j = 0; j < COLS; ++j)
                if (j >= left || j == at) w[j / 32][j % 32] = 0xff800000u;
        }
        float hi[4];
#pragma unroll
        for (int j = 0; j < 4; ++j) hi[j] = __uint_as_float(w[0][j]);
#pragma unroll
        for (int j = 4; j < COLS; ++j) hi[j & 3] = fmaxf(hi[j & 3], __uint_as_float(w[j / 32][j % 32]));
        const float most = fmaxf(fmaxf(hi[0], hi[1]), fmaxf(hi[2], hi[3]));
        const float top = most * job.scale;
        const float2 scale2 = make_float2(job.scale, job.scale), minus = make_float2(-top, -top);
        float2 add[4] = {};
#pragma unroll
        for (int j = 0; j < COLS; j += 2) {
            const float2 a = __ffma2_rn(make_float2(__uint_as_float(w[j / 32][j % 32]), __uint_as_float(w[j / 32][j % 32 + 1])), scale2, minus);
            add[(j >> 1) & 3] = __fadd2_rn(add[(j >> 1) & 3], make_float2(ex2_approx(a.x), ex2_approx(a.y)));
        }
        const float2 s01 = __fadd2_rn(add[0], add[1]), s23 = __fadd2_rn(add[2], add[3]);
        // a half may have no terms: behind the vocabulary's end, or but for the token
        const float sum = most > -INFINITY ? (s01.x + s01.y) + (s23.x + s23.y) : 0.0f;
        if (row < e.live && PPOW_CHECK(2 * x.index + half < job.parts, 502, flags))
            job.partial[(size_t)row * job.parts + 2 * x.index + half] = make_float2(top, sum);
    } else if (PRODUCT == LOGITS_GRAD) {
        const int32_t left = min(TILE, job.V - x.col) - first;
        const int32_t at = own.token - x.col - first;
        const float mult = own.mult, lse2 = own.lse2;
        if (at >= 0 && at < COLS && row < e.live) note_token(job, e, own.token, row);
        for_chunks<COLS / 32, 32>(src, release, [&](int c, uint32_t (&w)[32]) {
            float p[32];
#pragma unroll
            for (int j = 0; j < 32; ++j) p[j] = ex2_approx(fmaf(__uint_as_float(w[j]), job.scale, -lse2));
            if (at >= c && at < c + 32) {
#pragma unroll
                for (int j = 0; j < 32; ++j)
                    if (at == c + j) p[j] = own.target;
                if (row < e.live) job.rows.residual[row] = rounding_of<BF16>(own.target * mult);
            }
            if (row >= e.live || c + 32 > left) {
#pragma unroll
                for (int j = 0; j < 32; ++j)
                    if (row >= e.live || c + j >= left) p[j] = 0.0f;
            }
            uint32_t o[16];
#pragma unroll
            for (int j = 0; j < 16; ++j) o[j] = pack2<BF16>(p[2 * j] * mult, p[2 * j + 1] * mult);
            put_box(box, in_tile, half, c, o, map_out, x.index * TILE + first, x.row + in_tile / HALF_TILE * HALF_TILE,
                    PPOW_CHECK(x.index * TILE + first + c < job.piece, 503, flags));
        });
    } else if (PRODUCT == GRAD_HIDDEN) {
        float *to = job.grad_rows + ((size_t)x.split * e.row_tiles * TILE + row) * job.D + x.col + first;
        const int32_t left = min(TILE, job.D - x.col) - first;   // a multiple of 8
        for_chunks<COLS / 32, 32>(src, release, [&](int c, uint32_t (&w)[32]) {
#pragma unroll
            for (int h = 0; h < 4; ++h) {
                if (c + 8 * h < left && row < e.live && PPOW_CHECK(x.split < e.splits && x.k0 < x.k1, 504, flags)) {
                    uint32_t o[8];
#pragma unroll
                    for (int j = 0; j < 8; ++j) o[j] = w[8 * h + j];
                    if (job.add) {
                        const float4 *old = reinterpret_cast<const float4 *>(to + c + 8 * h);
                        const float4 p = old[0], q = old[1];
                        const float f[8] = {p.x, p.y, p.z, p.w, q.x, q.y, q.z, q.w};
#pragma unroll
                        for (int j = 0; j < 8; ++j) o[j] = __float_as_uint(__uint_as_float(o[j]) + f[j]);
                    }
                    store32(to + c + 8 * h, o);
                }
            }
        });
    } else {
        const float out_scale = gave_up(job.rows.header) ? NAN : job.rows.header->out_scale;
        const int32_t v = x.row + in_tile / HALF_TILE * HALF_TILE;       // the box's first row within the piece
        auto store = [&](int c, uint32_t (&w)[32]) {
            uint32_t o[16];
#pragma unroll
            for (int j = 0; j < 16; ++j)
                o[j] = pack2<BF16>(__uint_as_float(w[2 * j]) * out_scale, __uint_as_float(w[2 * j + 1]) * out_scale);
            put_box(box, in_tile, half, c, o, map_out, x.col + first, job.v0 + v, x.col + first + (c & 64) < job.D && v < job.columns);
        };
        if constexpr (PARTS) {
#pragma unroll
            for (int c = 0; c < COLS; c += 32) store(c, w[c / 32]);
        } else {
            for_chunks<COLS / 32, 32>(src, release, store);
        }
    }
}

// Combines column j of the 32 lanes for every j: lane l ends with the result of column l % WIDTH in v[0].  Each step halves the
// columns that a lane still carries (31 exchanges in all, not 5 for each column).
template <int WIDTH, typename Op>
__device__ __forceinline__ void across_lanes(float (&v)[WIDTH], Op op)
{
    const int lane = threadIdx.x & 31;
#pragma unroll
    for (int o = 16; o > 0; o >>= 1) {
        if (o >= WIDTH) {
#pragma unroll
            for (int j = 0; j < WIDTH; ++j) v[j] = op(v[j], __shfl_xor_sync(0xffffffffu, v[j], o));
        } else {
#pragma unroll
            for (int j = 0; j < o; ++j) {
                const float give = lane & o ? v[j] : v[j + o], keep = lane & o ? v[j + o] : v[j];
                v[j] = op(keep, __shfl_xor_sync(0xffffffffu, give, o));
            }
        }
    }
}

// A warp's columns of a tile, in registers: chunks of at most 32.
template <int N> __host__ __device__ constexpr int sum_width() { return N / 2 < 32 ? N / 2 : 32; }
template <int N> __host__ __device__ constexpr int sum_chunks() { return N / 2 / sum_width<N>(); }

// Maximum and sum of exponentials, over the tiles that a warp has seen, of column lane % 32 of a chunk of 32.
struct RunningSum {
    float top, sum;
};

// rows: the vocabulary's entries, for GRAD_HIDDEN the width's; columns: tokens.  Sums over the rows run across the lanes.
template <int PRODUCT, bool BF16, int N, typename R>
__device__ __forceinline__ void epilogue_few(const ProductJob &job, const Extent &e, const Tile &x, uint32_t src, int32_t in_tile, int half,
                                             RunningSum (&run)[2], const int32_t (&token)[2], uint32_t (&z)[sum_chunks<N>()][sum_width<N>()],
                                             R &&release)
{
    constexpr int COLS = N / 2, WIDTH = sum_width<N>();
    const int lane = threadIdx.x & 31;
    const int32_t row = x.row + in_tile, first = half * COLS;
    src += first;
    [[maybe_unused]] unsigned int *flags = &job.rows.header->error_flags;
    if (PRODUCT == LOGITS_SUM) {
        const bool inside = row < job.V;
#pragma unroll
        for (int c = 0; c < COLS; c += WIDTH) {
            if (first + c >= e.live) break;
            uint32_t (&w)[WIDTH] = z[c / WIDTH];
            // the term of a token that lies in this warp's 32 rows, if any does, comes from elsewhere
            const int32_t at = token[c / 32] - (row - lane);
            const unsigned hits = __ballot_sync(0xffffffffu, at >= 0 && at < 32);
            if (hits) {
#pragma unroll
                for (int j = 0; j < WIDTH; ++j)
                    if ((hits >> j & 1u) && __shfl_sync(0xffffffffu, at, j) == lane) w[j] = 0xff800000u;
            }
            float r[WIDTH];
#pragma unroll
            for (int j = 0; j < WIDTH; ++j) r[j] = inside ? __uint_as_float(w[j]) : -INFINITY;
            across_lanes<WIDTH>(r, [](float a, float b) { return fmaxf(a, b); });
            RunningSum &seen = run[c / 32];
            const float top = fmaxf(seen.top, r[0] * job.scale);     // of column lane % WIDTH; rounded, and taken as it is from here on
#pragma unroll
            for (int j = 0; j < WIDTH; ++j) {
                const float hi = __shfl_sync(0xffffffffu, top, j);
                r[j] = inside ? ex2_approx(fmaf(__uint_as_float(w[j]), job.scale, -hi)) : 0.0f;
            }
            across_lanes<WIDTH>(r, [](float a, float b) { return a + b; });
            seen.sum = top > -INFINITY ? fmaf(seen.sum, ex2_approx(seen.top - top), r[0]) : 0.0f;
            seen.top = top;
        }
    } else if (PRODUCT == LOGITS_GRAD) {
        const bool inside = row < job.V;
        uint16_t *to = job.dz + x.index * TILE + in_tile;
        for_chunks<COLS / WIDTH, WIDTH>(src, release, [&](int c, uint32_t (&w)[WIDTH]) {
            // lane j holds what column j needs of its token; columns behind the live ones get zeros
            const int32_t mine = first + c + lane;
            const bool live = lane < WIDTH && mine < e.live;
            const float lse2 = live ? job.rows.lse2[mine] : 0.0f, mult = live ? job.rows.mult[mine] : 0.0f;
            const int32_t token = live ? job.rows.token[mine] : -1;
            if (token >= row - lane && token < row - lane + 32) note_token(job, e, token, mine);
#pragma unroll
            for (int j = 0; j < WIDTH; ++j) {
                const float l = __shfl_sync(0xffffffffu, lse2, j), m = __shfl_sync(0xffffffffu, mult, j);
                float d = ex2_approx(fmaf(__uint_as_float(w[j]), job.scale, -l));
                const bool target = __shfl_sync(0xffffffffu, token, j) == row;
                if (target) d = job.rows.target[first + c + j];
                d = inside && first + c + j < e.live ? d * m : 0.0f;
                if (target) job.rows.residual[first + c + j] = rounding_of<BF16>(d);
                if (PPOW_CHECK(x.index * TILE + in_tile < job.piece, 507, flags))
                    to[(size_t)(first + c + j) * job.piece] = (uint16_t)pack2<BF16>(d, 0.0f);
            }
        });
    } else {
        float *to = job.grad_rows + (size_t)x.split * N * job.D + row;
        const bool inside = row < job.D;
        for_chunks<COLS / WIDTH, WIDTH>(src, release, [&](int c, uint32_t (&w)[WIDTH]) {
#pragma unroll
            for (int j = 0; j < WIDTH; ++j) {
                const int32_t token = first + c + j;
                if (inside && token < e.live && PPOW_CHECK(x.split < e.splits && x.k0 < x.k1, 508, flags)) {
                    float *p = to + (size_t)token * job.D;
                    const float v = __uint_as_float(w[j]);
                    *p = job.add ? *p + v : v;
                }
            }
        });
    }
}

// ---- remainders ---------------------------------------------------------------------------------------
// dz at its token is most of the row of dW that it falls into, and rounded alone it is off by as much as the result's own rounding
// (4096 x 4096 x 128256 bf16: 0.0023 of dW, 0.0017 without that error).  What the rounding left over is added as further steps of the
// tile's sum: the tile's rows lie side by side, and for 64 of them the operand in dz's place is zero but for one entry each, their
// remainders.  A warp of its own writes it into the stage (done by the producer warp it held the copies up, and the tensor pipe was 79 %
// active at 2048 x 4096 x 32000, not 95), where TMA brings the rows' hidden states beside it, in slices of the 16
// rows that one instruction multiplies, since a tile has few rows more often than not (552 tokens x 776 x 68450: 6 us less than by
// whole steps; 222 us in all, without remainders 217).
constexpr uint32_t SLICE_BYTES = 16 * 128;
// A step takes the 64 rows from `row` on, of those of the tile.  The hidden states read with them end with the last row tile at the
// latest, because behind it the workspace holds anything: `row` is row `skip` of what is read.
struct RemainderStep {
    int32_t box_row, skip;
    uint32_t slices;
};
__device__ __forceinline__ RemainderStep remainder_step(const Extent &e, TokenRows rows, int32_t row)
{
    const int32_t box_row = min(row, e.row_tiles * TILE - BK);
    return {box_row, row - box_row, (uint32_t)(row - box_row + min(BK, rows.end - row) + 15) / 16};
}
template <bool REMAINDERS>
__device__ __forceinline__ TokenRows tile_rows(const ProductJob &job, int64_t tiles, int64_t t, int64_t other)     // of tile t, if there is one
{
    if (!REMAINDERS) return {0, 0};
    const int2 r = *reinterpret_cast<const int2 *>(job.rows.rows_of + job.v0 / TILE + (int32_t)(t < tiles ? t : other) / job.d_tiles);
    return {r.x, r.y};
}
struct RemainderRows {
    int32_t token[BK / 32];          // of rows `from` + lane + 32 i, negative: none
    float rest[BK / 32];
};
__device__ __forceinline__ RemainderRows remainder_rows(const ProductJob &job, TokenRows rows, int32_t from)
{
    RemainderRows r;
#pragma unroll
    for (int i = 0; i < BK / 32; ++i) {
        const int32_t row = from + 32 * i + (int32_t)(threadIdx.x & 31);
        r.token[i] = row < rows.end ? job.rows.token[row] : -1;
        r.rest[i] = row < rows.end ? job.rows.residual[row] : 0.0f;
    }
    return r;
}
// A step's slices of the half tile from vocabulary entry `base` on, rows by 128 entries, laid out as TMA would: blocks of 64 entries, a
// row 128 bytes, its 16-byte unit u at u ^ (row & 7).
template <bool BF16> __device__ __forceinline__ void put_remainders(uint32_t a, const RemainderRows &r, const RemainderStep &step, int32_t base)
{
    const uint32_t lane = threadIdx.x & 31;
#pragma unroll 4
    for (uint32_t i = lane; i < step.slices * (SLICE_BYTES / 16); i += 32) {
        store_shared16(a + 16 * i, 0u, 0u, 0u, 0u);
        store_shared16(a + BK * 128 + 16 * i, 0u, 0u, 0u, 0u);
    }
    __syncwarp();
#pragma unroll
    for (int i = 0; i < BK / 32; ++i) {
        const uint32_t k = step.skip + 32 * i + lane, m = (uint32_t)(r.token[i] - base);
        if (r.token[i] >= 0 && m < HALF_TILE && PPOW_CHECK(k < BK, 510, nullptr))
            store_shared2(a + m / 64 * (BK * 128) + k * 128 + ((m % 64 / 8 ^ (k & 7)) << 4) + m % 8 * 2, pack2<BF16>(r.rest[i], 0.0f));
    }
    fence_for_copy_engine();
    __syncwarp();
}

// Persistent: one CTA per SM, pair p takes tiles p, p + pairs, ...  Warp 0 keeps the operand ring full, one thread of
// the leader's warp 1 issues the products into one of two accumulators, warps 2..9 read the other one out.
template <int PRODUCT> __host__ __device__ constexpr int mma_threads() { return MMA_THREADS + (PRODUCT == GRAD_WEIGHT ? 32 : 0); }
template <int PRODUCT, bool BF16, int N, bool PARTS>
__global__ void __cluster_dims__(2, 1, 1) __launch_bounds__(mma_threads<PRODUCT>(), 1)
    head_product_kernel(const __grid_constant__ CUtensorMap map_a, const __grid_constant__ CUtensorMap map_b,
                        const __grid_constant__ CUtensorMap map_out, const __grid_constant__ CUtensorMap map_rest, const ProductJob job)
{
    constexpr bool FEW = N < TILE;
    constexpr bool A_K = FEW ? PRODUCT != GRAD_HIDDEN : PRODUCT != GRAD_WEIGHT;     // the inner axis is contiguous in A
    constexpr bool B_K = FEW || PRODUCT == LOGITS_SUM || PRODUCT == LOGITS_GRAD;
    constexpr uint32_t INSTRUCTION = mma_instruction(BF16, A_K, B_K, TILE, N);
    constexpr uint32_t BLOCK_BYTES = BK * 128;                                      // 64 wide x BK rows
    constexpr uint32_t STAGES = stage_count<N>(), STAGE_BYTES = stage_bytes<N>();
    constexpr bool REMAINDERS = PRODUCT == GRAD_WEIGHT;                             // steps behind the product's own

    extern __shared__ uint8_t smem_raw[];
    const uint32_t smem = (smem_addr(smem_raw) + 1023u) & ~1023u;
    const uint32_t box = smem + STAGES * STAGE_BYTES, bars = box + (FEW ? 0 : 2 * BOX_BYTES);
    auto full = [&](uint32_t s) { return bars + 8 * s; };                       // the leader's count, for both CTAs
    auto empty = [&](uint32_t s) { return bars + 8 * (STAGES + s); };
    auto acc_full = [&](uint32_t b) { return bars + 8 * (2 * STAGES + b); };
    auto acc_empty = [&](uint32_t b) { return bars + 8 * (2 * STAGES + 2 + b); };   // the leader's count, for both CTAs
    // Steps of remainders: the producer warp, which passes every step of the ring, says that the step's stage is free; the leader's
    // count of both CTAs says that the remainders are written.  The producer is no more steps ahead of the products than the ring has
    // stages, so of more barriers than that, taken by turns, none completes a second time before the first has been waited for.
    constexpr uint32_t TURNS = 8;
    static_assert(STAGES < TURNS || !REMAINDERS, "a barrier must not complete twice before it is waited for");
    [[maybe_unused]] auto free_stage = [&](uint32_t step) { return bars + 8 * (2 * STAGES + 5 + step % TURNS); };
    [[maybe_unused]] auto written = [&](uint32_t step) { return bars + 8 * (2 * STAGES + 5 + TURNS + step % TURNS); };
    const uint32_t tmem_slot = bars + 8 * (2 * STAGES + 4);

    const int warp = threadIdx.x >> 5, lane = threadIdx.x & 31;
    const uint32_t rank = cluster_rank();
    const int32_t pair = blockIdx.x >> 1, pairs = gridDim.x >> 1;
    HeadHeader *header = job.rows.header;

    if (threadIdx.x == 0) {
        prefetch_tensor_map(&map_a);
        prefetch_tensor_map(&map_b);
        for (uint32_t s = 0; s < STAGES; ++s) {
            mbar_init(full(s), 1);
            mbar_init(empty(s), 1);
        }
        for (uint32_t b = 0; b < 2; ++b) {
            mbar_init(acc_full(b), 1);
            mbar_init(acc_empty(b), 16);     // eight epilogue warps of each CTA
        }
        if (REMAINDERS)
            for (uint32_t i = 0; i < TURNS; ++i) {
                mbar_init(free_stage(i), 1);
                mbar_init(written(i), 2);
            }
        mbar_init_fence();
    }
    if (warp == 1) tmem_alloc_pair(tmem_slot);
    tcgen05_fence_before();
    __syncthreads();
    cluster_barrier();
    tcgen05_fence_after();
    uint32_t tmem;
    asm volatile("ld.shared.b32 %0, [%1];" : "=r"(tmem) : "r"(tmem_slot));
    wait_for_previous_kernel();

    Extent e;
    const bool direct = FEW && PRODUCT == LOGITS_SUM && job.direct;
    e.live = direct ? job.direct : header->live;
    if (direct && blockIdx.x == 0 && warp == 0) {
        // no gather has written the header.  (A wait that runs out adds its flag two seconds from here at the earliest.)
        bool range = false;
        for (int32_t i = lane; i < job.direct; i += 32) range = range || job.rows.token[i] >= job.V;
        range = __any_sync(0xffffffffu, range);
        if (lane == 0) {
            header->error_flags = range ? (unsigned)PPOW_FLAG_TOKEN_RANGE : 0u;
            header->live = job.direct;
        }
    }
    e.row_tiles = (e.live + TILE - 1) / TILE;
    if (FEW || PRODUCT != LOGITS_SUM) e.row_tiles = max(1, e.row_tiles);
    e.splits = PRODUCT == GRAD_HIDDEN ? header->splits : 1;
    const int64_t tiles = tile_count<PRODUCT>(job, e);

    if (warp == 0) {
        if (lane == 0) {
            uint32_t it = 0;
            [[maybe_unused]] uint32_t step = 0;              // of remainders
            bool ok = true;
            [[maybe_unused]] TokenRows rows = tile_rows<REMAINDERS>(job, tiles, pair, pair);
            for (int64_t t = pair; t < tiles && ok; t += pairs) {
                const Tile x = tile_at<PRODUCT, FEW>(job, e, t);
                const int32_t n = x.col + (int32_t)rank * (N / 2);
                [[maybe_unused]] const TokenRows next = tile_rows<REMAINDERS>(job, tiles, t + pairs, t);
                for (int32_t k = x.k0; k < x.k1 && ok; ++k, ++it) {
                    const uint32_t s = it % STAGES, phase = (it / STAGES) & 1u;
                    ok = mbar_wait_ns(empty(s), phase ^ 1u);
                    if (!ok) break;
                    if (rank == 0) mbar_arrive_expect_tx(full(s), 2 * STAGE_BYTES);
                    const uint32_t bar = peer_addr(full(s), 0);
                    const uint32_t a = smem + s * STAGE_BYTES, b = a + A_BYTES;
                    const int32_t m = x.row + (int32_t)rank * HALF_TILE;
                    // the vocabulary is the inner axis of dh: its coordinate in W starts at the piece
                    const int32_t k_weight = k * BK + (PRODUCT == GRAD_HIDDEN ? job.v0 : 0);
                    if (A_K) {
                        tma_load_pair(a, &map_a, k * BK, m, bar);
                    } else {
                        tma_load_pair(a, &map_a, m, k_weight, bar);
                        tma_load_pair(a + BLOCK_BYTES, &map_a, m + 64, k_weight, bar);
                    }
                    if (B_K) {
                        tma_load_pair(b, &map_b, k * BK, n, bar);
                    } else {
                        tma_load_pair(b, &map_b, n, k_weight, bar);
                        tma_load_pair(b + BLOCK_BYTES, &map_b, n + 64, k_weight, bar);
                    }
                }
                if constexpr (REMAINDERS) {
                    for (int32_t row = rows.first; row < rows.end && ok; row += BK, ++it, ++step) {
                        const uint32_t s = it % STAGES, b = smem + s * STAGE_BYTES + A_BYTES;
                        ok = mbar_wait_ns(empty(s), ((it / STAGES) & 1u) ^ 1u);
                        if (!ok) break;
                        mbar_arrive(free_stage(step));
                        const RemainderStep r = remainder_step(e, rows, row);
                        if (rank == 0) mbar_arrive_expect_tx(full(s), r.slices * (2 * 2 * SLICE_BYTES));
                        const uint32_t bar = peer_addr(full(s), 0);
#pragma unroll 1
                        for (uint32_t q = 0; q < r.slices; ++q) {
                            tma_load_pair(b + q * SLICE_BYTES, &map_rest, n, r.box_row + 16 * q, bar);
                            tma_load_pair(b + BLOCK_BYTES + q * SLICE_BYTES, &map_rest, n + 64, r.box_row + 16 * q, bar);
                        }
                    }
                    rows = next;
                }
            }
            // the leader's last commits land on this CTA's barriers: stay until they have
            for (uint32_t j = it > STAGES ? it - STAGES : 0; j < it && ok; ++j) ok = mbar_wait_ns(empty(j % STAGES), (j / STAGES) & 1u);
            if (!ok) fault(header, PPOW_FLAG_DEVICE_TIMEOUT);
        }
    } else if (REMAINDERS && warp == MMA_THREADS / 32) {
        if constexpr (REMAINDERS) {
            uint32_t it = 0, step = 0;
            bool ok = true;
            TokenRows rows = tile_rows<REMAINDERS>(job, tiles, pair, pair);
            RemainderRows ahead = remainder_rows(job, rows, rows.first);
            for (int64_t t = pair; t < tiles && ok; t += pairs) {
                const Tile x = tile_at<PRODUCT, FEW>(job, e, t);
                const TokenRows next = tile_rows<REMAINDERS>(job, tiles, t + pairs, t);
                it += x.k1 - x.k0;
                for (int32_t row = rows.first; row < rows.end && ok; row += BK, ++it, ++step) {
                    const uint32_t s = it % STAGES;
                    const RemainderRows here = ahead;
                    if (row + BK < rows.end) ahead = remainder_rows(job, rows, row + BK);
                    if (lane == 0) ok = mbar_wait_ns(free_stage(step), (step / TURNS) & 1u);
                    ok = __shfl_sync(0xffffffffu, ok, 0);
                    __syncwarp();
                    if (!ok) break;
                    put_remainders<BF16>(smem + s * STAGE_BYTES, here, remainder_step(e, rows, row), job.v0 + x.row + (int32_t)rank * HALF_TILE);
                    if (lane == 0) mbar_arrive_release_cluster(peer_addr(written(step), 0));
                }
                rows = next;
                ahead = remainder_rows(job, rows, rows.first);
            }
            if (!ok && lane == 0) fault(header, PPOW_FLAG_DEVICE_TIMEOUT);
        }
    } else if (warp == 1) {
        if (rank == 0 && lane == 0) {
            uint32_t it = 0, acc = 0;
            [[maybe_unused]] uint32_t step = 0;              // of remainders
            bool ok = true;
            for (int64_t t = pair; t < tiles && ok; t += pairs) {
                const Tile x = tile_at<PRODUCT, FEW>(job, e, t);
                const int32_t parts = part_count<PARTS>(job, x);
                [[maybe_unused]] const TokenRows rows = tile_rows<REMAINDERS>(job, tiles, t, t);
                for (int32_t part = 0; part < parts && ok; ++part, ++acc) {
                    const int32_t k0 = PARTS ? x.k0 + part * job.part_steps : x.k0, k1 = PARTS ? min(k0 + job.part_steps, x.k1) : x.k1;
                    const uint32_t b = acc & 1u, d = tmem + b * TILE;
                    ok = mbar_wait_ns(acc_empty(b), ((acc >> 1) & 1u) ^ 1u);
                    tcgen05_fence_after();
                    for (int32_t k = k0; k < k1 && ok; ++k, ++it) {
                        const uint32_t s = it % STAGES;
                        ok = mbar_wait_ns(full(s), (it / STAGES) & 1u);
                        if (!ok) break;
                        tcgen05_fence_after();
                        const uint32_t a = smem + s * STAGE_BYTES;
                        const uint64_t da = operand_descriptor(a, A_K, BLOCK_BYTES), db = operand_descriptor(a + A_BYTES, B_K, BLOCK_BYTES);
#pragma unroll
                        for (int q = 0; q < BK / 16; ++q)
                            mma_pair(d, da + (uint64_t)(q * (A_K ? 32 : 2048) >> 4), db + (uint64_t)(q * (B_K ? 32 : 2048) >> 4), INSTRUCTION,
                                     k > k0 || q > 0);
                        mma_commit_pair(empty(s));
                    }
                    if constexpr (REMAINDERS) {
                        for (int32_t row = part + 1 < parts ? rows.end : rows.first; row < rows.end && ok; row += BK, ++it, ++step) {
                            const uint32_t s = it % STAGES;
                            ok = mbar_wait_ns(full(s), (it / STAGES) & 1u) && mbar_wait_ns(written(step), (step / TURNS) & 1u) &&
                                 mbar_acquire_cluster(written(step), (step / TURNS) & 1u);
                            if (!ok) break;
                            tcgen05_fence_after();
                            const uint32_t a = smem + s * STAGE_BYTES;
                            const uint64_t da = operand_descriptor(a, A_K, BLOCK_BYTES), db = operand_descriptor(a + A_BYTES, B_K, BLOCK_BYTES);
                            const uint32_t slices = remainder_step(e, rows, row).slices;
#pragma unroll 1
                            for (uint32_t q = 0; q < slices; ++q)
                                mma_pair(d, da + (uint64_t)(q * SLICE_BYTES >> 4), db + (uint64_t)(q * SLICE_BYTES >> 4), INSTRUCTION, true);
                            mma_commit_pair(empty(s));
                        }
                    }
                    if (ok) mma_commit_pair(acc_full(b));
                }
            }
            if (!ok) fault(header, PPOW_FLAG_DEVICE_TIMEOUT);
        }
    } else {
        const uint32_t quarter = warp & 3;                       // the 32 Tensor Memory lanes that this warp may read
        const int half = (warp - 2) >> 2;
        const int32_t in_tile = (int32_t)(rank * HALF_TILE + quarter * 32 + lane);
        uint32_t acc = 0;
        bool ok = true;
        RunningSum run[2] = {{-INFINITY, 0.0f}, {-INFINITY, 0.0f}};
        int32_t token[2] = {-1, -1};                             // LOGITS_SUM, few tokens: those of columns lane % 32 of the chunks
        if (FEW && PRODUCT == LOGITS_SUM) {
#pragma unroll
            for (int c = 0; c < N / 2; c += 32)
                if (c + lane < N / 2 && half * (N / 2) + c + lane < e.live) token[c / 32] = max(job.rows.token[half * (N / 2) + c + lane], -1);
        }
        uint32_t z[sum_chunks<N>()][sum_width<N>()] = {};        // LOGITS_SUM, GRAD_WEIGHT in parts: the warp's columns
        for (int64_t t = pair; t < tiles && ok; t += pairs) {
            const Tile x = tile_at<PRODUCT, FEW>(job, e, t);
            RowData own = {};
            if (!FEW && (PRODUCT == LOGITS_SUM || PRODUCT == LOGITS_GRAD)) {
                own.token = job.rows.token[x.row + in_tile];
                if (PRODUCT == LOGITS_GRAD) {
                    own.mult = job.rows.mult[x.row + in_tile];
                    own.lse2 = job.rows.lse2[x.row + in_tile];
                    own.target = job.rows.target[x.row + in_tile];
                }
            }
            const int32_t parts = part_count<PARTS>(job, x);
            for (int32_t part = 0; part < parts; ++part, ++acc) {
                const uint32_t b = acc & 1u;
                // all four warps of a half go on or none does: they meet at barriers further down
                ok = named_barrier_all(1 + half, 128, mbar_wait_ns(acc_full(b), (acc >> 1) & 1u));
                if (!ok) break;
                tcgen05_fence_after();
                const uint32_t src = tmem + b * TILE + (quarter * 32u << 16);
                auto release = [&] {
                    tcgen05_fence_before();
                    __syncwarp();
                    if (lane == 0) mbar_arrive_cluster(peer_addr(acc_empty(b), 0));
                };
                if constexpr (PRODUCT == LOGITS_SUM || (PRODUCT == GRAD_WEIGHT && PARTS)) {
                    constexpr int CHUNKS = sum_chunks<N>(), WIDTH = sum_width<N>(), ADD = WIDTH < 16 ? WIDTH : 16;
                    const uint32_t from = src + half * (N / 2);
                    if (!PARTS || part == 0) {
#pragma unroll
                        for (int i = 0; i < CHUNKS; ++i) tmem_load(from + i * WIDTH, z[i]);
#pragma unroll
                        for (int i = 0; i < CHUNKS; ++i) tmem_wait(z[i]);
                    } else {
                        // few registers are left beside the sums: 16 columns at a time, behind the products of the next steps
#pragma unroll
                        for (int c = 0; c < N / 2; c += ADD) {
                            uint32_t w[ADD];
                            tmem_load(from + c, w);
                            tmem_wait(w);
#pragma unroll
                            for (int j = 0; j < ADD; ++j) {
                                uint32_t &sum = z[(c + j) / WIDTH][(c + j) % WIDTH];
                                sum = __float_as_uint(__uint_as_float(sum) + __uint_as_float(w[j]));
                            }
                        }
                    }
                    release();
                    if (part + 1 < parts) continue;
                }
                if constexpr (FEW)
                    epilogue_few<PRODUCT, BF16, N>(job, e, x, src, in_tile, half, run, token, z, release);
                else
                    epilogue_many<PRODUCT, BF16, PARTS>(job, e, x, own, src, in_tile, half, &map_out, box, z, release);
            }
        }
        if (FEW && PRODUCT == LOGITS_SUM) {
            constexpr int COLS = N / 2;
            const int32_t part = (int32_t)blockIdx.x * 4 + (int32_t)quarter;
#pragma unroll
            for (int c = 0; c < COLS; c += 32) {
                const int32_t token = half * COLS + c + lane;
                if (c + lane < COLS && token < e.live && PPOW_CHECK(part < job.parts, 506, &header->error_flags))
                    job.partial[(size_t)token * job.parts + part] = make_float2(run[c / 32].top, run[c / 32].sum);
            }
        }
        if (!FEW && (PRODUCT == LOGITS_GRAD || PRODUCT == GRAD_WEIGHT) && in_tile % HALF_TILE == 0) tma_store_wait();
        if (!ok && lane == 0) fault(header, PPOW_FLAG_DEVICE_TIMEOUT);
    }
    __syncwarp();
    tcgen05_fence_before();
    __syncthreads();
    cluster_barrier();
    if (warp == 1) {
        tcgen05_fence_after();
        tmem_free_pair(tmem);
    }
}

// ---- merge: one CTA per row ----------------------------------------------------------------------
constexpr int MERGE_THREADS = 128;
struct MergeJob {
    HeadRows rows;
    const float2 *partial;
    const uint16_t *hidden, *weight;      // hidden: by live row
    int64_t hidden_stride, weight_stride;
    int32_t parts, V, D;
    double exact_scale, rescale;          // log2(e) / temperature; that over the float32 value that the sums were taken with
    float *logp, *lse;
};
template <bool BF16>
__global__ void __launch_bounds__(MERGE_THREADS) head_merge_kernel(const MergeJob job)
{
    constexpr int HELD = 16;                             // entries per thread that are read once; more are read twice
    __shared__ float tops[MERGE_THREADS / 32];
    __shared__ double sums[MERGE_THREADS / 32], products[MERGE_THREADS / 32];
    const int tid = threadIdx.x, lane = tid & 31, warp = tid >> 5;
    const int32_t row = blockIdx.x, parts = job.parts;
    const HeadRows &rows = job.rows;
    allow_next_kernel();
    wait_for_previous_kernel();
    if (row >= rows.header->live) return;
    const int32_t r = rows.source ? rows.source[row] : row, y = rows.token[row];
    if (y < 0) {                                         // tokens that were not gathered: the masked ones are among them
        if (tid == 0) job.logp[r] = job.lse[r] = 0.0f;
        return;
    }
    const float2 *p = job.partial + (size_t)row * parts;
    float2 held[HELD];
    float top = -INFINITY;
#pragma unroll
    for (int i = 0; i < HELD; ++i) {
        const int32_t k = tid + i * MERGE_THREADS;
        held[i] = k < parts ? p[k] : make_float2(-INFINITY, 0.0f);
    }
#pragma unroll
    for (int i = 0; i < HELD; ++i) top = fmaxf(top, held[i].x);
#pragma unroll 8
    for (int32_t k = tid + HELD * MERGE_THREADS; k < parts; k += MERGE_THREADS) top = fmaxf(top, p[k].x);
    const double product = y < job.V ? token_product<BF16>(job.hidden + (size_t)row * job.hidden_stride, job.weight + (size_t)y * job.weight_stride,
                                                           job.D / 8, tid, MERGE_THREADS)
                                     : 0.0;
    top = warp_max(top);
    if (lane == 0) tops[warp] = top;
    __syncthreads();
#pragma unroll
    for (int i = 0; i < MERGE_THREADS / 32; ++i) top = fmaxf(top, tops[i]);
    double sum = 0.0, z2 = warp_sum_f64(product);
#pragma unroll
    for (int i = 0; i < HELD; ++i) sum += (double)(held[i].y * ex2_approx(held[i].x - top));
#pragma unroll 8
    for (int32_t k = tid + HELD * MERGE_THREADS; k < parts; k += MERGE_THREADS) sum += (double)(p[k].y * ex2_approx(p[k].x - top));
    sum = warp_sum_f64(sum);
    if (lane == 0) {
        sums[warp] = sum;
        products[warp] = z2;
    }
    __syncthreads();
    if (tid == 0) {
        sum = z2 = 0.0;
#pragma unroll
        for (int i = 0; i < MERGE_THREADS / 32; ++i) {
            sum += sums[i];
            z2 += products[i];
        }
        const double ln2 = 0.69314718055994530942;
        z2 *= job.exact_scale;
        if (gave_up(rows.header)) sum = NAN;
        // the sums' reference was scaled by a rounded number: 6e-8 of a logit of 60 would be in the result undamped
        const double others2 = (double)top * job.rescale + log2(sum);
        if (y >= job.V) {                                // no such token: the sums are whole without it
            job.lse[r] = (float)(others2 * ln2);
            job.logp[r] = -INFINITY;
        } else {
            // the others' share against the token's: log p = -log(1 + others / token), exact for p near 1 too
            const double ratio2 = others2 - z2;
            const double nats = ratio2 < 60.0 ? log1p(exp2(ratio2)) : ratio2 * ln2;
            job.logp[r] = (float)-nats;
            job.lse[r] = (float)(z2 * ln2 + nats);
        }
    }
}

// ---- finish: dh of the live rows, rounded once ------------------------------------------------------
constexpr int FINISH_THREADS = 128;
template <bool BF16>
__global__ void __launch_bounds__(FINISH_THREADS) head_finish_kernel(HeadRows rows, const float *__restrict__ parts, int32_t few,
                                                                     int32_t D, const uint16_t *__restrict__ weight,
                                                                     int64_t weight_stride, uint16_t *__restrict__ grad_hidden)
{
    allow_next_kernel();
    wait_for_previous_kernel();
    const int32_t units = D / 4, splits = rows.header->splits, live = rows.header->live;
    const size_t split_units = (size_t)(few ? few : (live + TILE - 1) / TILE * TILE) * units;
    const int64_t all = (int64_t)live * units;
    const bool lost = gave_up(rows.header);
    for (int64_t i = (int64_t)blockIdx.x * FINISH_THREADS + threadIdx.x; i < all; i += (int64_t)gridDim.x * FINISH_THREADS) {
        const int32_t row = (int32_t)(i / units), u = (int32_t)(i % units);
        const float4 *p = reinterpret_cast<const float4 *>(parts) + i;
        float4 f = make_float4(0.0f, 0.0f, 0.0f, 0.0f);
        int32_t s = 0;
        for (; s + 8 <= splits; s += 8) {
            float4 a[8];
#pragma unroll
            for (int j = 0; j < 8; ++j) a[j] = p[(s + j) * split_units];
#pragma unroll
            for (int j = 0; j < 8; ++j) f.x += a[j].x, f.y += a[j].y, f.z += a[j].z, f.w += a[j].w;
        }
        for (; s < splits; ++s) {
            const float4 a = p[s * split_units];
            f.x += a.x, f.y += a.y, f.z += a.z, f.w += a.w;
        }
        // the token's entry of dz is most of the row: what its rounding left over comes back here, in float32
        const uint2 wy = *(reinterpret_cast<const uint2 *>(weight + (size_t)rows.token[row] * weight_stride) + u);
        const float rest = rows.residual[row];
        const float2 w01 = unpack2<BF16>(wy.x), w23 = unpack2<BF16>(wy.y);
        f.x = fmaf(rest, w01.x, f.x), f.y = fmaf(rest, w01.y, f.y), f.z = fmaf(rest, w23.x, f.z), f.w = fmaf(rest, w23.y, f.w);
        const float k = lost ? NAN : rows.row_scale[row];
        reinterpret_cast<uint2 *>(grad_hidden + (size_t)rows.source[row] * D)[u] =
            make_uint2(pack2<BF16>(f.x * k, f.y * k), pack2<BF16>(f.z * k, f.w * k));
    }
}

// ---- host side --------------------------------------------------------------------------------------
namespace {

bool params_ok(const ppow_head_params *p)
{
    if (!p || p->T < 0 || p->T > MAX_TOKENS || p->V < 2 || p->V > MAX_VOCAB || p->D < 8 || p->D > MAX_WIDTH || p->D % 8) return false;
    if (p->dtype != PPOW_BF16 && p->dtype != PPOW_F16) return false;
    if (!(p->temperature > 0.0f) || !isfinite(p->temperature)) return false;
    if (p->hidden_stride < p->D || p->weight_stride < p->D || p->weight_stride % 8) return false;
    if (p->hidden_stride > (int64_t)1 << 40 || p->weight_stride > (int64_t)1 << 32) return false;
    return true;
}

// Columns of a tile for this many tokens.  Up to 128 the tokens are the columns and W the rows: 8 tokens x 4096 x 128256
// would spend as much on loading and multiplying 256 rows, 248 of them zeros, as W takes to come from HBM (222 us, like this 169).
// At 100 tokens it is 211 us against 231, at 128 x 4096 x 32000 62 against 69.
int32_t tile_columns(int32_t T) { return T <= 16 ? 16 : T <= 32 ? 32 : T <= 64 ? 64 : T <= 128 ? 128 : TILE; }

struct Layout {
    size_t source, token, mult, lse2, row_scale, target, residual, rows_of, rows, scaled, partial, dz, grad_rows, order, total;
    int32_t columns, few, padded, v_tiles, d_tiles, parts;
    int32_t pieces, piece;          // backward: pieces of the vocabulary, entries of the longest (the row length of dz)
};

// First vocabulary entry of piece i; piece `pieces` would start at or behind the vocabulary's end.
int64_t piece_start(const Layout &L, int32_t i) { return (int64_t)L.v_tiles * i / L.pieces * TILE; }
int32_t piece_columns(const Layout &L, int32_t V, int32_t i)
{
    const int64_t end = piece_start(L, i + 1);
    return (int32_t)((end < V ? end : V) - piece_start(L, i));
}
// Steps of the inner axis of dh in the shortest piece: a whole one, or the last one, whose end may lie inside a tile.
int32_t shortest_steps(const Layout &L, int32_t V)
{
    const int32_t whole = L.v_tiles / L.pieces * (TILE / BK), last = (piece_columns(L, V, L.pieces - 1) + BK - 1) / BK;
    return last < whole ? last : whole;
}
// Output tiles of dh for this many live rows, and the shares that head_gather_kernel plans for them.
int64_t hidden_tiles(const Layout &L, int32_t live) { return (int64_t)(L.few || live < 1 ? 1 : (live + TILE - 1) / TILE) * L.d_tiles; }
int32_t planned_splits(int64_t tiles, int32_t steps)
{
    int32_t best = 1;
    for (int32_t s = 2; split_allowed(s, tiles, steps); ++s)
        if (split_cost(s, tiles) < split_cost(best, tiles)) best = s;
    return best;
}

Layout layout_of(const ppow_head_params *p, bool backward)
{
    Layout L = {};
    size_t off = HEADER_BYTES;
    auto take = [&](size_t bytes) {
        const size_t o = off;
        off = (off + bytes + 255) & ~(size_t)255;
        return o;
    };
    L.columns = tile_columns(p->T);
    L.few = L.columns < TILE ? L.columns : 0;
    L.padded = L.few ? L.few : (p->T + TILE - 1) / TILE * TILE;
    L.v_tiles = (p->V + TILE - 1) / TILE;
    L.d_tiles = (p->D + TILE - 1) / TILE;
    const size_t rows = (size_t)L.padded;
    L.source = take(rows * 4);
    L.token = take(rows * 4);
    L.mult = take(rows * 4);
    L.lse2 = take(rows * 4);
    L.row_scale = take(rows * 4);
    L.target = take(rows * 4);
    L.residual = take(rows * 4);
    L.rows = take(rows * p->D * 2);
    if (!backward) {
        // few tokens: four warps of each CTA; there are at most as many pairs as tiles
        L.parts = L.few ? 8 * (L.v_tiles < MAX_PAIRS ? L.v_tiles : MAX_PAIRS) : 2 * L.v_tiles;
        L.partial = take(rows * L.parts * sizeof(float2));
    } else {
        if (p->T > ORDER_COUNTED) L.order = take(((size_t)p->V * 2 + rows * 2) * 4);
        if (p->dtype == PPOW_F16) L.scaled = take(rows * p->D * 2);
        const size_t strip = rows * TILE * 2;                      // one column tile of dz
        int32_t fit = (int32_t)(DZ_BYTES / strip);
        if (fit < 1) fit = 1;
        if (fit > PIECE_TILES) fit = PIECE_TILES;
        L.pieces = (L.v_tiles + fit - 1) / fit;
        L.piece = (L.v_tiles + L.pieces - 1) / L.pieces * TILE;    // lengths differ by one tile at most
        L.dz = take(rows * L.piece * 2);
        // sums of dh: all rows once, or as many shares as SPLIT_TILES allows
        size_t sums = rows, split = (size_t)(SPLIT_TILES / L.d_tiles) * (L.few ? L.few : TILE);
        if (split > sums) sums = split;
        L.grad_rows = take(sums * p->D * 4);
        L.rows_of = take((size_t)L.v_tiles * sizeof(TokenRows));
    }
    L.total = off;
    return L;
}

using EncodeTiled = CUresult (*)(CUtensorMap *, CUtensorMapDataType, cuuint32_t, void *, const cuuint64_t *, const cuuint64_t *,
                                 const cuuint32_t *, const cuuint32_t *, CUtensorMapInterleave, CUtensorMapSwizzle,
                                 CUtensorMapL2promotion, CUtensorMapFloatOOBfill);

EncodeTiled encode_tiled()
{
    static EncodeTiled fn = [] {
        void *p = nullptr;
        cudaDriverEntryPointQueryResult found;
        if (cudaGetDriverEntryPointByVersion("cuTensorMapEncodeTiled", &p, 12000, cudaEnableDefault, &found) != cudaSuccess ||
            found != cudaDriverEntryPointSuccess)
            p = nullptr;
        return (EncodeTiled)p;
    }();
    return fn;
}

// [height, width] 16-bit elements, rows `stride` elements apart; boxes of 64 x `box_rows`, what lies outside reads as 0.
bool make_map(CUtensorMap *map, const void *base, bool bf16, int64_t width, int64_t height, int64_t stride, uint32_t box_rows)
{
    const EncodeTiled encode = encode_tiled();
    if (!encode) return false;
    const cuuint64_t dims[2] = {(cuuint64_t)width, (cuuint64_t)height}, strides[1] = {(cuuint64_t)stride * 2};
    const cuuint32_t box[2] = {BK, box_rows}, step[2] = {1, 1};
    return encode(map, bf16 ? CU_TENSOR_MAP_DATA_TYPE_BFLOAT16 : CU_TENSOR_MAP_DATA_TYPE_FLOAT16, 2, const_cast<void *>(base), dims,
                  strides, box, step, CU_TENSOR_MAP_INTERLEAVE_NONE, CU_TENSOR_MAP_SWIZZLE_128B, CU_TENSOR_MAP_L2_PROMOTION_L2_256B,
                  CU_TENSOR_MAP_FLOAT_OOB_FILL_NONE) == CUDA_SUCCESS;
}

// Pairs of SMs of the current device, asked once per device; the kernels' shared-memory limit is raised at the same time.
constexpr int DEVICES = 64;
template <int PRODUCT> constexpr bool in_parts() { return PRODUCT == LOGITS_SUM || PRODUCT == GRAD_WEIGHT; }
template <int PRODUCT, bool BF16, int N> bool allow_smem()
{
    constexpr int BYTES = (int)mma_smem<N>();
    return cudaFuncSetAttribute(head_product_kernel<PRODUCT, BF16, N, false>, cudaFuncAttributeMaxDynamicSharedMemorySize, BYTES) == cudaSuccess &&
           (!in_parts<PRODUCT>() || cudaFuncSetAttribute(head_product_kernel<PRODUCT, BF16, N, in_parts<PRODUCT>()>,
                                                         cudaFuncAttributeMaxDynamicSharedMemorySize, BYTES) == cudaSuccess);
}
template <int PRODUCT, bool BF16> bool allow_smem_few()
{
    return allow_smem<PRODUCT, BF16, 16>() && allow_smem<PRODUCT, BF16, 32>() && allow_smem<PRODUCT, BF16, 64>() &&
           allow_smem<PRODUCT, BF16, 128>() && allow_smem<PRODUCT, BF16, TILE>();
}
template <bool BF16> int pair_count()
{
    static std::atomic<int> known[DEVICES];
    int dev = 0, sms = 0;
    if (cudaGetDevice(&dev) != cudaSuccess || dev < 0 || dev >= DEVICES) return 0;
    int n = known[dev].load(std::memory_order_relaxed);
    if (n > 0) return n;
    if (!allow_smem_few<LOGITS_SUM, BF16>() || !allow_smem_few<LOGITS_GRAD, BF16>() || !allow_smem_few<GRAD_HIDDEN, BF16>() ||
        !allow_smem<GRAD_WEIGHT, BF16, TILE>() || cudaDeviceGetAttribute(&sms, cudaDevAttrMultiProcessorCount, dev) != cudaSuccess)
        return 0;
    n = sms / 2 < MAX_PAIRS ? sms / 2 : MAX_PAIRS;
    known[dev].store(n, std::memory_order_relaxed);
    return n;
}

template <int PRODUCT, bool BF16, int N>
bool launch_tiles(const CUtensorMap &a, const CUtensorMap &b, const CUtensorMap &out, const CUtensorMap &rest, const ProductJob &job,
                  int64_t most_tiles, int pairs, cudaStream_t stream)
{
    const int n = (int)(most_tiles < pairs ? most_tiles : pairs);
    // one part is a kernel of its own: the loop over parts costs the forward pass a third (2048 x 128 x 128256: 106 us, with it 140)
    if (in_parts<PRODUCT>() && (PRODUCT == LOGITS_SUM ? job.D : job.tokens) > job.part_steps * BK)
        return launch_after(head_product_kernel<PRODUCT, BF16, N, in_parts<PRODUCT>()>, 2 * n, mma_threads<PRODUCT>(), mma_smem<N>(), stream, a, b, out, rest, job);
    return launch_after(head_product_kernel<PRODUCT, BF16, N, false>, 2 * n, mma_threads<PRODUCT>(), mma_smem<N>(), stream, a, b, out, rest, job);
}

// `rows` and `weight`: the operand maps of the token side and of W's side.  With few tokens the two change places.  `out`: the
// map of 16-bit results, where there are any.
template <int PRODUCT, bool BF16>
bool launch_product(const CUtensorMap &rows, const CUtensorMap &weight, const CUtensorMap &out, const ProductJob &job, int32_t columns,
                    int64_t most_tiles, int pairs, cudaStream_t stream)
{
    switch (columns) {
    case 16: return launch_tiles<PRODUCT, BF16, 16>(weight, rows, out, out, job, most_tiles, pairs, stream);
    case 32: return launch_tiles<PRODUCT, BF16, 32>(weight, rows, out, out, job, most_tiles, pairs, stream);
    case 64: return launch_tiles<PRODUCT, BF16, 64>(weight, rows, out, out, job, most_tiles, pairs, stream);
    case 128: return launch_tiles<PRODUCT, BF16, 128>(weight, rows, out, out, job, most_tiles, pairs, stream);
    }
    return launch_tiles<PRODUCT, BF16, TILE>(rows, weight, out, out, job, most_tiles, pairs, stream);
}

// Rows on 16-byte boundaries, within the strides that a tensor map can hold.
bool rows_aligned(const void *hidden, int64_t stride)
{
    return (uintptr_t)hidden % 16 == 0 && stride % 8 == 0 && stride <= (int64_t)1 << 32;
}

HeadRows rows_of(char *ws, const Layout &L)
{
    HeadRows r = {};
    r.header = (HeadHeader *)ws;
    r.source = (int32_t *)(ws + L.source);
    r.token = (int32_t *)(ws + L.token);
    r.mult = (float *)(ws + L.mult);
    r.lse2 = (float *)(ws + L.lse2);
    r.row_scale = (float *)(ws + L.row_scale);
    r.target = (float *)(ws + L.target);
    r.residual = (float *)(ws + L.residual);
    r.rows_of = (TokenRows *)(ws + L.rows_of);
    r.rows = ws + L.rows;
    r.scaled = ws + L.scaled;
    return r;
}

template <bool BACKWARD, bool SCALED>
bool launch_gather(const ppow_head_params *p, const Layout &L, const GatherJob &base, const HeadRows &rows, const void *hidden,
                   cudaStream_t stream)
{
    GatherJob job = base;
    job.stride = p->hidden_stride;
    job.T = p->T;
    job.D = p->D;
    job.V = p->V;
    job.few = L.few;
    job.d_tiles = L.d_tiles;
    job.piece_steps = L.pieces ? shortest_steps(L, p->V) : 0;
    job.exact_inv_temperature = 1.0 / (double)p->temperature;
    job.inv_temperature = (float)job.exact_inv_temperature;
    job.vec = rows_aligned(hidden, p->hidden_stride);
    job.hidden = (const uint16_t *)hidden;
    // a row per CTA, more where that would be over a thousand CTAs: each of them looks at all tokens
    job.rows_per_cta = (L.padded + GATHER_CTAS - 1) / GATHER_CTAS;
    const unsigned grid = (unsigned)((L.padded + job.rows_per_cta - 1) / job.rows_per_cta);
    return launch_after(head_gather_kernel<BACKWARD, SCALED>, grid, GATHER_THREADS, 0, stream, job, rows);
}

template <bool BF16>
ppow_status forward(const ppow_head_params *p, const void *hidden, const void *weight, const int32_t *tokens, float *logp, float *lse,
                    char *ws, cudaStream_t stream)
{
    const Layout L = layout_of(p, false);
    HeadRows rows = rows_of(ws, L);
    // Few tokens on 16-byte boundaries are read where they lie: they are the columns of one tile, and a masked one's column touches
    // no other.  That saves the gather, a quarter of a small call (77 x 520 x 1001: 12.6 us with it).
    const bool direct = L.few && rows_aligned(hidden, p->hidden_stride);
    if (direct) {
        rows.source = nullptr;
        rows.token = const_cast<int32_t *>(tokens);
    }
    CUtensorMap map_rows, map_weight;
    if (!make_map(&map_rows, direct ? hidden : rows.rows, BF16, p->D, direct ? p->T : L.padded, direct ? p->hidden_stride : p->D, L.columns / 2) ||
        !make_map(&map_weight, weight, BF16, p->D, p->V, p->weight_stride, HALF_TILE))
        return PPOW_ERR_CUDA;
    const int pairs = pair_count<BF16>();
    if (pairs < 1) return PPOW_ERR_CUDA;
    if (!direct) {
        GatherJob g = {};
        g.tokens = tokens;
        g.logp_out = logp;
        g.lse_out = lse;
        if (!launch_gather<false, false>(p, L, g, rows, hidden, stream)) return PPOW_ERR_CUDA;
    }
    ProductJob job = {};
    job.rows = rows;
    job.scale = (float)(1.4426950408889634074 / (double)p->temperature);
    job.D = p->D;
    job.V = job.columns = p->V;
    job.direct = direct ? p->T : 0;
    job.part_steps = logit_part_steps(p->D, L.columns);
    job.v_tiles = L.v_tiles;
    job.d_tiles = L.d_tiles;
    job.parts = L.few ? 8 * (L.v_tiles < pairs ? L.v_tiles : pairs) : L.parts;
    job.partial = (float2 *)(ws + L.partial);
    const int64_t tiles = (int64_t)((L.padded + TILE - 1) / TILE) * L.v_tiles;
    if (!launch_product<LOGITS_SUM, BF16>(map_rows, map_weight, map_rows, job, L.columns, tiles, pairs, stream)) return PPOW_ERR_CUDA;
    MergeJob merge = {};
    merge.rows = rows;
    merge.partial = job.partial;
    merge.hidden = (const uint16_t *)(direct ? hidden : rows.rows);
    merge.hidden_stride = direct ? p->hidden_stride : p->D;
    merge.weight = (const uint16_t *)weight;
    merge.weight_stride = p->weight_stride;
    merge.parts = job.parts;
    merge.V = p->V;
    merge.D = p->D;
    merge.exact_scale = 1.4426950408889634074 / (double)p->temperature;
    merge.rescale = merge.exact_scale / (double)job.scale;
    merge.logp = logp;
    merge.lse = lse;
    return launch_after(head_merge_kernel<BF16>, (unsigned)p->T, MERGE_THREADS, 0, stream, merge) ? PPOW_OK : PPOW_ERR_CUDA;
}

template <bool BF16>
ppow_status backward(const ppow_head_params *p, const void *hidden, const void *weight, const int32_t *tokens, const float *lse,
                     const float *grad_logp, void *grad_hidden, void *grad_weight, char *ws, cudaStream_t stream)
{
    const Layout L = layout_of(p, true);
    const HeadRows rows = rows_of(ws, L);
    uint16_t *dz = (uint16_t *)(ws + L.dz);
    CUtensorMap map_rows, map_rows_t, map_weight, map_weight_t, map_dz, map_dz_t, map_grad, map_rest;
    if (!make_map(&map_rows, rows.rows, BF16, p->D, L.padded, p->D, L.columns / 2) ||
        !make_map(&map_rows_t, BF16 ? rows.rows : rows.scaled, BF16, p->D, L.padded, p->D, BK) ||
        !make_map(&map_weight, weight, BF16, p->D, p->V, p->weight_stride, HALF_TILE) ||
        !make_map(&map_weight_t, weight, BF16, p->D, p->V, p->weight_stride, BK) ||
        !make_map(&map_dz, dz, BF16, L.piece, L.padded, L.piece, L.columns / 2) || !make_map(&map_dz_t, dz, BF16, L.piece, L.padded, L.piece, BK) ||
        (grad_weight && (!make_map(&map_grad, grad_weight, BF16, p->D, p->V, p->D, HALF_TILE) ||
                         !make_map(&map_rest, BF16 ? rows.rows : rows.scaled, BF16, p->D, L.padded, p->D, 16))))
        return PPOW_ERR_CUDA;
    const int pairs = pair_count<BF16>();
    if (pairs < 1) return PPOW_ERR_CUDA;
    GatherJob g = {};
    g.tokens = tokens;
    g.lse = lse;
    g.grad = grad_logp;
    g.grad_hidden = (uint16_t *)grad_hidden;
    g.by_token = grad_weight != nullptr;
    g.weight = (const uint16_t *)weight;
    g.weight_stride = p->weight_stride;
    if (L.order && grad_weight) {
        g.order.count = (int32_t *)(ws + L.order);
        g.order.first = g.order.count + p->V;
        g.order.slot = g.order.first + p->V;
        g.order.list = g.order.slot + L.padded;
        const int32_t most = 148 * 8, share = (p->V / 148 / SCAN_THREADS + 1) * SCAN_THREADS;
        auto grid = [&](int32_t n) { return (unsigned)((n - 1) / ORDER_THREADS + 1 < most ? (n - 1) / ORDER_THREADS + 1 : most); };
        if (!launch_after(head_order_clear_kernel, grid(p->V), ORDER_THREADS, 0, stream, g.order, p->V) ||
            !launch_after(head_order_count_kernel, grid(p->T), ORDER_THREADS, 0, stream, g.order, tokens, grad_logp, p->T, p->V) ||
            !launch_after(head_order_scan_kernel, (unsigned)((p->V + share - 1) / share), SCAN_THREADS, 0, stream, g.order, p->V, share) ||
            !launch_after(head_order_list_kernel, grid(p->T), ORDER_THREADS, 0, stream, g.order, tokens, grad_logp, p->T, p->V))
            return PPOW_ERR_CUDA;
    }
    if (!launch_gather<true, !BF16>(p, L, g, rows, hidden, stream)) return PPOW_ERR_CUDA;
    ProductJob job = {};
    job.rows = rows;
    job.scale = (float)(1.4426950408889634074 / (double)p->temperature);
    job.D = p->D;
    job.V = p->V;
    job.d_tiles = L.d_tiles;
    job.piece = L.piece;
    job.tokens = p->T;
    job.part_steps = WEIGHT_PART_STEPS;
    job.dz = dz;
    job.grad_rows = (float *)(ws + L.grad_rows);
    const int64_t row_tiles = (L.padded + TILE - 1) / TILE;
    for (int32_t i = 0; i < L.pieces; ++i) {
        job.v0 = (int32_t)piece_start(L, i);
        job.columns = piece_columns(L, p->V, i);
        job.v_tiles = (job.columns + TILE - 1) / TILE;
        job.add = i > 0;
        if (!launch_product<LOGITS_GRAD, BF16>(map_rows, map_weight, map_dz, job, L.columns, row_tiles * job.v_tiles, pairs, stream))
            return PPOW_ERR_CUDA;
        if (grad_hidden && !launch_product<GRAD_HIDDEN, BF16>(map_dz, map_weight_t, map_dz, job, L.columns, pairs, pairs, stream)) return PPOW_ERR_CUDA;
        if (grad_weight && !launch_tiles<GRAD_WEIGHT, BF16, TILE>(map_dz_t, map_rows_t, map_grad, map_rest, job, (int64_t)job.v_tiles * L.d_tiles, pairs, stream))
            return PPOW_ERR_CUDA;
    }
    if (grad_hidden) {
        const int64_t blocks = ((int64_t)p->T * (p->D / 4) + FINISH_THREADS - 1) / FINISH_THREADS;
        if (!launch_after(head_finish_kernel<BF16>, (unsigned)(blocks < 148 * 16 ? blocks : 148 * 16), FINISH_THREADS, 0, stream, rows,
                          job.grad_rows, L.few, p->D, (const uint16_t *)weight, p->weight_stride, (uint16_t *)grad_hidden))
            return PPOW_ERR_CUDA;
    }
    return PPOW_OK;
}

// Without tokens nothing is launched that would; a workspace is not needed then.
ppow_status clear_header(void *workspace, size_t bytes, cudaStream_t stream)
{
    if (!workspace || bytes < sizeof(HeadHeader)) return PPOW_OK;
    return cudaMemsetAsync(workspace, 0, sizeof(HeadHeader), stream) == cudaSuccess ? PPOW_OK : PPOW_ERR_CUDA;
}

}  // namespace
}  // namespace ppow

#ifdef PPOW_CHECKED
namespace ppow { int read_check_counters_head(unsigned int *f, unsigned int *s) { return read_check_counters(f, s); } }
#endif

using namespace ppow;

extern "C" size_t ppow_head_workspace_bytes(const ppow_head_params *params, int backward)
{
    return params_ok(params) ? layout_of(params, backward != 0).total : 0;
}

extern "C" int ppow_head_plan(const ppow_head_params *params, int32_t live, int32_t piece, int32_t *first, int32_t *columns, int32_t *shares)
{
    if (!params_ok(params) || live < 0 || live > params->T || piece < 0) return 0;
    const Layout L = layout_of(params, true);
    if (piece < L.pieces) {
        if (first) *first = (int32_t)piece_start(L, piece);
        if (columns) *columns = piece_columns(L, params->V, piece);
        if (shares) *shares = planned_splits(hidden_tiles(L, live), shortest_steps(L, params->V));
    }
    return L.pieces;
}

extern "C" ppow_status ppow_head_logprob(const ppow_head_params *params, const void *hidden, const void *weight, const int32_t *tokens,
                                         float *logp, float *lse, void *workspace, size_t workspace_bytes, void *cuda_stream)
{
    if (!params_ok(params)) return PPOW_ERR_INVALID_ARG;
    if (params->T == 0) return clear_header(workspace, workspace_bytes, (cudaStream_t)cuda_stream);
    if (!hidden || !weight || !tokens || !logp || !lse) return PPOW_ERR_INVALID_ARG;
    if ((uintptr_t)hidden % 2 || (uintptr_t)weight % 16 || (uintptr_t)tokens % 4 || (uintptr_t)logp % 4 || (uintptr_t)lse % 4)
        return PPOW_ERR_INVALID_ARG;
    if (!workspace || (uintptr_t)workspace % 256 || workspace_bytes < layout_of(params, false).total) return PPOW_ERR_WORKSPACE;
    return params->dtype == PPOW_BF16
               ? forward<true>(params, hidden, weight, tokens, logp, lse, (char *)workspace, (cudaStream_t)cuda_stream)
               : forward<false>(params, hidden, weight, tokens, logp, lse, (char *)workspace, (cudaStream_t)cuda_stream);
}

extern "C" ppow_status ppow_head_logprob_backward(const ppow_head_params *params, const void *hidden, const void *weight,
                                                  const int32_t *tokens, const float *lse, const float *grad_logp, void *grad_hidden,
                                                  void *grad_weight, void *workspace, size_t workspace_bytes, void *cuda_stream)
{
    if (!params_ok(params)) return PPOW_ERR_INVALID_ARG;
    if ((uintptr_t)grad_hidden % 16 || (uintptr_t)grad_weight % 16) return PPOW_ERR_INVALID_ARG;
    if (params->T == 0) {
        if (grad_weight && cudaMemsetAsync(grad_weight, 0, (size_t)params->V * params->D * 2, (cudaStream_t)cuda_stream) != cudaSuccess)
            return PPOW_ERR_CUDA;
        return clear_header(workspace, workspace_bytes, (cudaStream_t)cuda_stream);
    }
    if ((!grad_hidden && !grad_weight) || !hidden || !weight || !tokens || !lse || !grad_logp) return PPOW_ERR_INVALID_ARG;
    if ((uintptr_t)hidden % 2 || (uintptr_t)weight % 16 || (uintptr_t)tokens % 4 || (uintptr_t)lse % 4 || (uintptr_t)grad_logp % 4)
        return PPOW_ERR_INVALID_ARG;
    if (!workspace || (uintptr_t)workspace % 256 || workspace_bytes < layout_of(params, true).total) return PPOW_ERR_WORKSPACE;
    return params->dtype == PPOW_BF16 ? backward<true>(params, hidden, weight, tokens, lse, grad_logp, grad_hidden, grad_weight,
                                                       (char *)workspace, (cudaStream_t)cuda_stream)
                                      : backward<false>(params, hidden, weight, tokens, lse, grad_logp, grad_hidden, grad_weight,
                                                        (char *)workspace, (cudaStream_t)cuda_stream);
}
