// dropout, layer norm, and dropout + residual sum + layer norm on [n, rows, h] activations: forward and backward, with the
// gradient of the weight and the bias kept apart by worker.
//
//   s = residual + dropout(x)             (or s = x)        kept in the residual's type
//   y = (s - mean) rstd w + b,            mean and variance over the h columns, rstd = 1 / sqrt(var + eps)
//   backward:  g = dy w,  xhat = (s - mean) rstd,
//   ds_all = rstd (g - mean(g) - xhat mean(g xhat)) + ds,   dresidual = ds_all,  dx = dropout(ds_all) with the same mask
//   dw_i = sum over the rows of worker i of dy xhat,        db_i = sum of dy
//
// All bound by memory. Sums and statistics are fp32, the variance is summed over differences from the mean (the row stays in
// registers), weights, biases and their gradients are fp32 as the optimizer keeps them.
#include <string.h>

#include <algorithm>
#include <atomic>
#include <type_traits>

#include "context.h"
#include "rows.cuh"

namespace compams {
namespace {

struct NormArgs {
    const void* x;         // forward: x; backward: dy
    const void* residual;  // forward: the residual; backward: ds (may be null)
    const void* v;         // backward: the normalised values (x or s)
    void* y;               // forward: y; backward: dx (may be null)
    void* s;               // forward: s; backward: dresidual (may be null)
    float2* stats;         // mean and rstd of every row; forward: may be null
    const float* weight;   // may be null: ones
    const float* bias;     // may be null: zeros
    float* partial;        // backward: [n, chunks, 2, h] sums over the rows of a chunk; null: not wanted
    int64_t x_ws, x_rs, r_ws, r_rs, v_ws, v_rs, weight_ws, bias_ws;
    uint32_t rows;         // per worker
    uint32_t total;        // n * rows
    int32_t h;
    uint32_t chunks;       // backward: CTAs per worker
    float eps;
    Drop drop;
};

__device__ __forceinline__ float warp_sum(float x) {
#pragma unroll
    for (int o = 16; o > 0; o >>= 1) x += __shfl_xor_sync(0xffffffffu, x, o);
    return x;
}
// Over W neighbouring lanes.
template <int W>
__device__ __forceinline__ float few_sum(float x) {
#pragma unroll
    for (int o = W / 2; o > 0; o >>= 1) x += __shfl_xor_sync(0xffffffffu, x, o);
    return x;
}
// The sum over the W warps of a row; the same order on every warp. `scratch`: W floats that no one reads any more.
template <int W>
__device__ __forceinline__ float row_sum(float x, float* scratch, int warp) {
    x = warp_sum(x);
    if (W == 1) return x;
    if ((threadIdx.x & 31) == 0) scratch[warp] = x;
    __syncthreads();
    float s = 0.0f;
#pragma unroll
    for (int w = 0; w < W; ++w) s += scratch[w];
    return s;
}

constexpr int kRowsOfOneWarp = 8;  // warps of a CTA whose warps share no row
// Rows of such a CTA, L lanes to a row: 32, or as many as the eights of an aligned short row need.
template <int W, int L>
__host__ __device__ constexpr int norm_rows() { return W == 1 ? kRowsOfOneWarp * (32 / L) : 1; }

template <int W>
__host__ __device__ constexpr int norm_threads() { return W == 1 ? 32 * kRowsOfOneWarp : 32 * W; }

// CTAs that the registers of an SM have to hold, so that their barriers fall at different times: 24 warps' (16 where the backward
// pass with its third input would not fit 80 registers a thread, and where rows are read element by element). One CTA of 16 warps; two in
// the forward pass, where 64 registers a thread nearly do, but for aligned rows with a residual: 16384 bfloat16 rows of 4097 219 us
// with one and 147 with two, with the residual, some of whose values spill then, 367 and 263; aligned rows of 8192 120 and 97, with the
// residual 207 and 222; backward, with spills, 155 and 221.
template <int W, int NG, bool VEC, bool MORE, bool ADD>
__host__ __device__ constexpr int norm_ctas() {
    return W == 16 ? (!MORE && NG <= 2 && !(ADD && VEC) ? 2 : 1) : (VEC && !(MORE && NG > 1) ? 24 : 16) / (W == 1 ? kRowsOfOneWarp : W);
}

// ---- a CTA's rows ----------------------------------------------------------------------------------------------------------

// A CTA goes through the rows of one chunk of one worker, W warps to a row, NG spans to a warp, and keeps in registers what all rows share.
// Where rows are aligned (VEC) every lane copies what it will need of the next rows into places of shared memory that it
// alone reads, kStages - 1 rows ahead, so that the sums that a row waits for (one barrier) do not stop the loads. Place:
// [stage][slot][thread], 16 bytes each; SLOTS: of a lane in a stage. Three stages where an SM has the room, or two; none for
// the longest rows of fp32, which are read where they are used.
template <int W, int SLOTS, bool VEC>
__host__ __device__ constexpr int row_stages() {
    const int bytes = SLOTS * 16 * norm_threads<W>();
    return !VEC || 2 * bytes > 200 * 1024 ? 0 : 3 * bytes > 200 * 1024 ? 2 : 3;
}
template <int W, int SLOTS, bool VEC>
__host__ __device__ constexpr int row_shared() { return row_stages<W, SLOTS, VEC>() * SLOTS * 16 * norm_threads<W>(); }
template <typename T>
__host__ __device__ constexpr int raw_slots() { return (int)sizeof(Raw8<T>) / 16; }

template <int W, int SLOTS>
__device__ __forceinline__ uint4* row_place(char* smem, int stage, int slot) {
    return reinterpret_cast<uint4*>(smem) + (stage * SLOTS + slot) * norm_threads<W>() + threadIdx.x;
}
template <typename T, int W, int SLOTS>
__device__ __forceinline__ void row_copy(char* smem, int stage, int slot, const T* from) {
#pragma unroll
    for (int k = 0; k < raw_slots<T>(); ++k) copy16(row_place<W, SLOTS>(smem, stage, slot + k), reinterpret_cast<const char*>(from) + 16 * k);
}
// A lane's values of the span from column c0 on, `beyond` in the columns from h on.
template <typename T, int W, int SLOTS, bool VEC, bool RING>
__device__ __forceinline__ void row_take(char* smem, int stage, int slot, const T* row, int c0, int h, int lane, float beyond, Pair (&to)[4]) {
    if constexpr (RING) {
        if (c0 + lane * 8 < h) {
            Raw8<T> r;
            uint4 u[raw_slots<T>()];
#pragma unroll
            for (int k = 0; k < raw_slots<T>(); ++k) u[k] = *row_place<W, SLOTS>(smem, stage, slot + k);
            memcpy(&r, u, sizeof(r));
            raw_pairs<T>(r, to);
        } else {
#pragma unroll
            for (int p = 0; p < 4; ++p) to[p] = pair(beyond);
        }
    } else {
        span_load<T, VEC>(row, c0, h, lane, to, beyond);
    }
}

// ---- forward ---------------------------------------------------------------------------------------------------------------

template <typename TX, typename TR, int NG, bool ADD>
__host__ __device__ constexpr int forward_slots() { return NG * (raw_slots<TX>() + (ADD ? raw_slots<TR>() : 0)); }

// Every warp finds the mean and the sum of squares about it of its own columns; the barrier passes these on, and each warp
// joins them (Chan, Golub, LeVeque 1979: the squares about the common mean are those about the parts' means and n_w (mean_w -
// mean)^2 more), so a row costs one barrier and its values stay in registers. Bound by memory: 16384 rows of 4096 in bfloat16, 268 MB,
// 48 us (5.6 TB/s; a plain copy takes 42); with dropout and the residual, 32768 rows, 1.07 GB, 198 us (5.4 TB/s). One row of 4096 takes
// 3 us, which is the latency of its loads and the barrier.
template <typename TX, typename TR, int W, int NG, int L, bool VEC, bool ADD>
__global__ void __launch_bounds__(norm_threads<W>(), norm_ctas<W, NG, VEC, false, ADD>()) norm_forward_kernel(const __grid_constant__ NormArgs a) {
    extern __shared__ __align__(16) char smem[];
    constexpr int kRows = norm_rows<W, L>(), SLOTS = forward_slots<TX, TR, NG, ADD>(), kStages = row_stages<W, SLOTS, VEC>();
    constexpr bool RING = kStages > 0, kHold = NG <= 2;
    __shared__ float2 scratch[2][W];
    const int lane = (int)threadIdx.x % L, warp = W == 1 ? 0 : (int)(threadIdx.x >> 5), slot = W == 1 ? (int)threadIdx.x / L : 0;
    const uint32_t i = blockIdx.x / a.chunks, chunk = blockIdx.x - i * a.chunks;
    const uint32_t j0 = (uint32_t)((uint64_t)a.rows * chunk / a.chunks), j1 = (uint32_t)((uint64_t)a.rows * (chunk + 1) / a.chunks);
    const uint32_t call = drop_call(a.drop);
    const TX* x = (const TX*)a.x + (int64_t)i * a.x_ws;
    const TR* residual = ADD ? (const TR*)a.residual + (int64_t)i * a.r_ws : nullptr;
    const float* weight = a.weight ? a.weight + (int64_t)i * a.weight_ws : nullptr;
    const float* bias = a.bias ? a.bias + (int64_t)i * a.bias_ws : nullptr;
    auto affine = [&](int q, Pair (&w)[4], Pair (&b)[4]) {
        const int c0 = (q * W + warp) * kSpan;
#pragma unroll
        for (int p = 0; p < 4; ++p) b[p] = pair(0.0f), w[p] = pair(1.0f);
        if (weight) span_load<float, VEC>(weight, c0, a.h, lane, w);
        if (bias) span_load<float, VEC>(bias, c0, a.h, lane, b);
    };
    auto fetch = [&](uint32_t j, int stage) {
        if constexpr (RING) {
#pragma unroll
            for (int q = 0; q < NG; ++q) {
                const int c = (q * W + warp) * kSpan + lane * 8;
                if (j < j1 && c < a.h) {
                    row_copy<TX, W, SLOTS>(smem, stage, q * raw_slots<TX>(), x + (int64_t)j * a.x_rs + c);
                    if (ADD) row_copy<TR, W, SLOTS>(smem, stage, NG * raw_slots<TX>() + q * raw_slots<TR>(), residual + (int64_t)j * a.r_rs + c);
                }
            }
            copies_commit();
        }
    };
    for (int k = 0; k + 1 < kStages; ++k) fetch(j0 + slot + k * kRows, k);
    Pair w[kHold ? NG : 1][4], b[kHold ? NG : 1][4];
    if (kHold)
#pragma unroll
        for (int q = 0; q < NG; ++q) affine(q, w[kHold ? q : 0], b[kHold ? q : 0]);
    // columns of this warp's own, and of warp k
    auto columns = [&](int k) {
        int c = 0;
#pragma unroll
        for (int q = 0; q < NG; ++q) c += min(max(a.h - (q * W + k) * kSpan, 0), kSpan);
        return (float)c;
    };
    const float own = columns(warp), per_own = own > 0.0f ? 1.0f / own : 0.0f, per_row = 1.0f / (float)a.h;
    const float lane_columns = columns(lane % W);
    int turn = 0, stage = 0;
    for (uint32_t j = j0 + slot; j - slot % (32 / L) < j1; j += kRows, turn ^= 1) {
        const uint32_t m = i * a.rows + j;
        const int h = L == 32 || j < j1 ? a.h : 0;  // a warp's rows go on together; the ones behind the chunk's last are empty
        if constexpr (RING) {
            fetch(j + (kStages - 1) * kRows, stage == 0 ? kStages - 1 : stage - 1);
            copies_wait<kStages - 1>();  // a lane's own
        }
        Pair v[NG][4], sum = pair(0.0f);
#pragma unroll
        for (int q = 0; q < NG; ++q) {
            const int c0 = (q * W + warp) * kSpan;
            row_take<TX, W, SLOTS, VEC, RING>(smem, stage, q * raw_slots<TX>(), x + (int64_t)j * a.x_rs, c0, h, lane, 0.0f, v[q]);
            if (ADD && c0 < h) {
                Pair more[4];
                row_take<TR, W, SLOTS, VEC, RING>(smem, stage, NG * raw_slots<TX>() + q * raw_slots<TR>(), residual + (int64_t)j * a.r_rs, c0,
                                                  h, lane, 0.0f, more);
                if (a.drop.on) span_drop<VEC>(a.drop, c0, j, a.drop.worker + i, call, lane, v[q]);
#pragma unroll
                for (int p = 0; p < 4; ++p) v[q][p] = add(v[q][p], more[p]);
                span_store<TR, VEC, true>((TR*)a.s + (int64_t)m * a.h, c0, h, lane, v[q]);
            }
#pragma unroll
            for (int p = 0; p < 4; ++p) sum = add(sum, v[q][p]);  // 0 beyond h
        }
        stage = stage + 1 == kStages ? 0 : stage + 1;
        const float mean = few_sum<L>(joint(sum)) * per_own;
        Pair squares = pair(0.0f);
#pragma unroll
        for (int q = 0; q < NG; ++q) {
            const int c0 = (q * W + warp) * kSpan;
#pragma unroll
            for (int p = 0; p < 4; ++p) {
                if (VEC) {
                    v[q][p] = add(v[q][p], pair(c0 + lane * 8 < h ? -mean : 0.0f));
                } else {
                    v[q][p] = add(v[q][p], pair(c0 + 64 * p + lane < a.h ? -mean : 0.0f, c0 + 64 * p + 32 + lane < a.h ? -mean : 0.0f));
                }
                squares = fma(v[q][p], v[q][p], squares);
            }
        }
        float square = few_sum<L>(joint(squares)), off = 0.0f, centre = mean;  // off: of the warp's mean from the row's
        if (W > 1) {
            if (lane == 0) scratch[turn][warp] = make_float2(mean, square);
            __syncthreads();  // the next row writes the other half, and the one after it only behind the next row's barrier
            const float2 part = scratch[turn][lane % W];  // every W lanes join the W warps' in the same way
            centre = few_sum<W>(lane_columns * part.x) * per_row;
            const float d = part.x - centre;
            square = few_sum<W>(fmaf(lane_columns * d, d, part.y));
            off = mean - centre;
        }
        const float rstd = 1.0f / sqrtf(square * per_row + a.eps);
        if (a.stats && warp == 0 && lane == 0 && h) a.stats[m] = make_float2(centre, rstd);
        const Pair factor = pair(rstd), offset = pair(off * rstd);
#pragma unroll
        for (int q = 0; q < NG; ++q) {
            const int c0 = (q * W + warp) * kSpan;
            if (c0 >= h) break;
            if (!kHold) affine(q, w[0], b[0]);
#pragma unroll
            for (int p = 0; p < 4; ++p) v[q][p] = fma(fma(v[q][p], factor, offset), w[kHold ? q : 0][p], b[kHold ? q : 0][p]);
            span_store<TX, VEC>((TX*)a.y + (int64_t)m * a.h, c0, h, lane, v[q]);
        }
    }
}

// Rows too long for registers (above 16384 columns): a CTA to a row, which is read again for each sum, from the L2 as a rule.
template <typename TX, typename TR, bool ADD>
__global__ void __launch_bounds__(512) norm_forward_long_kernel(const __grid_constant__ NormArgs a) {
    constexpr int W = 16;
    __shared__ float scratch[2][W];
    const int lane = threadIdx.x & 31, warp = threadIdx.x >> 5;
    const uint32_t m = blockIdx.x, i = m / a.rows, j = m - i * a.rows;
    const TX* x = (const TX*)a.x + (int64_t)i * a.x_ws + (int64_t)j * a.x_rs;
    // where there is a sum s it is written first, and read again by the thread that wrote it
    TR* s = (TR*)a.s + (int64_t)m * a.h;
    const TR* r = (const TR*)a.residual + (int64_t)i * a.r_ws + (int64_t)j * a.r_rs;
    const uint32_t call = drop_call(a.drop);
    float sum = 0.0f;
    for (int c0 = warp * kSpan; c0 < a.h; c0 += W * kSpan) {
        float v[8], add[8];
        span_load<TX, false>(x, c0, a.h, lane, v);
        if (ADD) {
            span_load<TR, false>(r, c0, a.h, lane, add);
            if (a.drop.on) span_drop<false>(a.drop, c0, j, a.drop.worker + i, call, lane, v);
#pragma unroll
            for (int k = 0; k < 8; ++k) v[k] = to_float(from_float<TR>(v[k] + add[k]));
            span_store<TR, false>(s, c0, a.h, lane, v);
        }
#pragma unroll
        for (int k = 0; k < 8; ++k) sum += v[k];
    }
    const float mean = row_sum<W>(sum, scratch[0], warp) / (float)a.h;
    float square = 0.0f;
    for (int c = warp * kSpan + lane; c < a.h; c += (c - lane) % kSpan == kSpan - 32 ? (W - 1) * kSpan + 32 : 32) {
        const float v = (ADD ? to_float(s[c]) : to_float(__ldg(x + c))) - mean;
        square = fmaf(v, v, square);
    }
    const float rstd = 1.0f / sqrtf(row_sum<W>(square, scratch[1], warp) / (float)a.h + a.eps);
    if (a.stats && threadIdx.x == 0) a.stats[m] = make_float2(mean, rstd);
    const float* weight = a.weight ? a.weight + (int64_t)i * a.weight_ws : nullptr;
    const float* bias = a.bias ? a.bias + (int64_t)i * a.bias_ws : nullptr;
    TX* y = (TX*)a.y + (int64_t)m * a.h;
    for (int c = warp * kSpan + lane; c < a.h; c += (c - lane) % kSpan == kSpan - 32 ? (W - 1) * kSpan + 32 : 32) {
        const float v = (ADD ? to_float(s[c]) : to_float(__ldg(x + c))) - mean;
        y[c] = from_float<TX>(fmaf(v * rstd, weight ? __ldg(weight + c) : 1.0f, bias ? __ldg(bias + c) : 0.0f));
    }
}

// ---- backward --------------------------------------------------------------------------------------------------------------

template <typename TX, typename TR, int NG, bool ADD>
__host__ __device__ constexpr int backward_slots() { return NG * (raw_slots<TX>() + (ADD ? 2 : 1) * raw_slots<TR>()); }

// The sums of dy xhat and dy of a chunk's rows stay in registers, the weight too. With several spans to a warp the values are taken
// a second time behind the barrier instead of being held, and with four the weight is read again for each row: registers are what
// bounds the CTAs of an SM. 16384 rows of 4096 in bfloat16, 403 MB, take 79 us (5.1 TB/s); with dropout, the second incoming gradient
// and the residual's, 32768 rows, 1.34 GB, 237 us (5.7 TB/s). 8192 rows of 16000, four spans to a warp, take 427 us with the forward
// pass, 2.6 times the bytes' time: the weights are read again from the L2 for each row.
template <typename TX, typename TR, int W, int NG, int L, bool VEC, bool ADD>
__global__ void __launch_bounds__(norm_threads<W>(), norm_ctas<W, NG, VEC, true, ADD>()) norm_backward_kernel(const __grid_constant__ NormArgs a) {
    extern __shared__ __align__(16) char smem[];
    constexpr int kSlots = norm_rows<W, L>(), SX = raw_slots<TX>(), SR = raw_slots<TR>();
    constexpr int SLOTS = backward_slots<TX, TR, NG, ADD>(), kStages = row_stages<W, SLOTS, VEC>();
    constexpr bool RING = kStages > 0;
    __shared__ float2 scratch[2][W];
    __shared__ float joined[W == 1 ? NG * kSpan : 1];
    const int lane = (int)threadIdx.x % L, warp = W == 1 ? 0 : (int)(threadIdx.x >> 5), slot = W == 1 ? (int)threadIdx.x / L : 0;
    const uint32_t i = blockIdx.x / a.chunks, chunk = blockIdx.x - i * a.chunks;
    const uint32_t j0 = (uint32_t)((uint64_t)a.rows * chunk / a.chunks), j1 = (uint32_t)((uint64_t)a.rows * (chunk + 1) / a.chunks);
    const uint32_t call = drop_call(a.drop);
    const TX* dy = (const TX*)a.x + (int64_t)i * a.x_ws;
    const TR* v = (const TR*)a.v + (int64_t)i * a.v_ws;
    const TR* more = ADD && a.residual ? (const TR*)a.residual + (int64_t)i * a.r_ws : nullptr;
    constexpr bool kHold = NG == 1, kHoldWeight = NG <= 2;
    Pair held[kHoldWeight ? NG : 1][4], dw[NG][4], db[NG][4];
    auto weight = [&](int q, Pair (&w)[4]) {
#pragma unroll
        for (int p = 0; p < 4; ++p) w[p] = pair(1.0f);
        if (a.weight) span_load<float, VEC>(a.weight + (int64_t)i * a.weight_ws, (q * W + warp) * kSpan, a.h, lane, w);
    };
#pragma unroll
    for (int q = 0; q < NG; ++q) {
#pragma unroll
        for (int p = 0; p < 4; ++p) dw[q][p] = db[q][p] = pair(0.0f);
        if (kHoldWeight) weight(q, held[kHoldWeight ? q : 0]);
    }
    auto fetch = [&](uint32_t j, int stage) {
        if constexpr (RING) {
#pragma unroll
            for (int q = 0; q < NG; ++q) {
                const int c = (q * W + warp) * kSpan + lane * 8;
                if (j < j1 && c < a.h) {
                    row_copy<TX, W, SLOTS>(smem, stage, q * SX, dy + (int64_t)j * a.x_rs + c);
                    row_copy<TR, W, SLOTS>(smem, stage, NG * SX + q * SR, v + (int64_t)j * a.v_rs + c);
                    if (ADD && more) row_copy<TR, W, SLOTS>(smem, stage, NG * (SX + SR) + q * SR, more + (int64_t)j * a.r_rs + c);
                }
            }
            copies_commit();
        }
    };
    for (int k = 0; k + 1 < kStages; ++k) fetch(j0 + slot + k * kSlots, k);
    int turn = 0, stage = 0;
    const float per_row = 1.0f / (float)a.h;
    float2 next = j0 + slot < j1 ? a.stats[i * a.rows + j0 + slot] : make_float2(0.0f, 0.0f);
    for (uint32_t j = j0 + slot; j - slot % (32 / L) < j1; j += kSlots, turn ^= 1) {
        const uint32_t m = i * a.rows + j;
        const int h = L == 32 || j < j1 ? a.h : 0;  // as in the forward pass: empty, so all its sums and terms are zeros
        const float2 st = next;
        if (j + kSlots < j1) next = a.stats[m + kSlots];
        if constexpr (RING) {
            fetch(j + (kStages - 1) * kSlots, stage == 0 ? kStages - 1 : stage - 1);
            copies_wait<kStages - 1>();  // a lane's own
        }
        Pair g[4], xhat[4], sum1 = pair(0.0f), sum2 = pair(0.0f);
        const Pair rstd = pair(st.y), less_mean = pair(-st.x);
        // dy w and xhat of span q; the first time its share of the sums
        auto values = [&](int q, bool first) {
            const int c0 = (q * W + warp) * kSpan;
            row_take<TX, W, SLOTS, VEC, RING>(smem, stage, q * SX, dy + (int64_t)j * a.x_rs, c0, h, lane, 0.0f, g);
            row_take<TR, W, SLOTS, VEC, RING>(smem, stage, NG * SX + q * SR, v + (int64_t)j * a.v_rs, c0, h, lane, st.x, xhat);
            Pair w[4];
            if (!kHoldWeight) weight(q, w);
#pragma unroll
            for (int p = 0; p < 4; ++p) {
                xhat[p] = mul(add(xhat[p], less_mean), rstd);  // (a product with the mean would leave its rounding in rows far from zero)
                if (first) {
                    db[q][p] = add(db[q][p], g[p]);
                    dw[q][p] = fma(g[p], xhat[p], dw[q][p]);
                }
                g[p] = mul(g[p], kHoldWeight ? held[kHoldWeight ? q : 0][p] : w[p]);
                if (first) {
                    sum1 = add(sum1, g[p]);
                    sum2 = fma(g[p], xhat[p], sum2);
                }
            }
        };
#pragma unroll
        for (int q = 0; q < NG; ++q) values(q, true);
        if (a.y || (ADD && a.s)) {
            float c1 = few_sum<L>(joint(sum1)), c2 = few_sum<L>(joint(sum2));
            if (W > 1) {
                if (lane == 0) scratch[turn][warp] = make_float2(c1, c2);
                __syncthreads();  // the next row writes the other half, and the one after it only behind the next row's barrier
                const float2 part = scratch[turn][lane % W];
                c1 = few_sum<W>(part.x);
                c2 = few_sum<W>(part.y);
            }
            // rstd (g - c1 - xhat c2)
            const Pair less = pair(-c1 * per_row * st.y), along = pair(-c2 * per_row * st.y);
#pragma unroll
            for (int q = 0; q < NG; ++q) {
                const int c0 = (q * W + warp) * kSpan;
                if (c0 >= h) break;
                if (!kHold) values(q, false);
#pragma unroll
                for (int p = 0; p < 4; ++p) g[p] = fma(xhat[p], along, fma(g[p], rstd, less));
                if (ADD && more) {
                    Pair r[4];
                    row_take<TR, W, SLOTS, VEC, RING>(smem, stage, NG * (SX + SR) + q * SR, more + (int64_t)j * a.r_rs, c0, h, lane, 0.0f, r);
#pragma unroll
                    for (int p = 0; p < 4; ++p) g[p] = add(g[p], r[p]);
                }
                if (ADD && a.s) span_store<TR, VEC>((TR*)a.s + (int64_t)m * a.h, c0, h, lane, g);
                if (ADD && a.drop.on && a.y) span_drop<VEC>(a.drop, c0, j, a.drop.worker + i, call, lane, g);
                if (a.y) span_store<TX, VEC>((TX*)a.y + (int64_t)m * a.h, c0, h, lane, g);
            }
        }
        stage = stage + 1 == kStages ? 0 : stage + 1;
    }
    if (!a.partial) return;
    float* out = a.partial + (int64_t)blockIdx.x * 2 * a.h;
    if constexpr (W > 1) {
#pragma unroll
        for (int q = 0; q < NG; ++q) {
            span_store<float, VEC>(out, (q * W + warp) * kSpan, a.h, lane, dw[q]);
            span_store<float, VEC>(out + a.h, (q * W + warp) * kSpan, a.h, lane, db[q]);
        }
    } else {  // warps with rows of their own: their sums joined, those of a warp's rows first, then one warp after the other
#pragma unroll
        for (int o = L; o < 32; o <<= 1)
#pragma unroll
            for (int p = 0; p < 4; ++p)
#pragma unroll
                for (int q = 0; q < NG; ++q) {
                    float x[2], y[2];
                    halves(dw[q][p], x[0], x[1]);
                    halves(db[q][p], y[0], y[1]);
#pragma unroll
                    for (int k = 0; k < 2; ++k) {
                        x[k] += __shfl_xor_sync(0xffffffffu, x[k], o);
                        y[k] += __shfl_xor_sync(0xffffffffu, y[k], o);
                    }
                    dw[q][p] = pair(x[0], x[1]);
                    db[q][p] = pair(y[0], y[1]);
                }
#pragma unroll
        for (int which = 0; which < 2; ++which) {
            for (int s = 0; s < kRowsOfOneWarp; ++s) {
                if ((int)threadIdx.x / 32 == s && (int)threadIdx.x % 32 < L) {
#pragma unroll
                    for (int q = 0; q < NG; ++q)
#pragma unroll
                        for (int p = 0; p < 4; ++p) {
                            float x[2];
                            halves(which ? db[q][p] : dw[q][p], x[0], x[1]);
#pragma unroll
                            for (int k = 0; k < 2; ++k) {
                                const int at = span_column<VEC>(q * kSpan, lane, 2 * p + k);
                                joined[at] = s == 0 ? x[k] : joined[at] + x[k];
                            }
                        }
                }
                __syncthreads();
            }
            for (int c = threadIdx.x; c < a.h; c += blockDim.x) out[which * a.h + c] = joined[c];
            __syncthreads();
        }
    }
}

// Rows too long for registers: one kernel for the rows' sums and dx, one for the columns' sums.
template <typename TX, typename TR, bool ADD>
__global__ void __launch_bounds__(512) norm_backward_long_kernel(const __grid_constant__ NormArgs a) {
    constexpr int W = 16;
    __shared__ float scratch[2][W];
    const int lane = threadIdx.x & 31, warp = threadIdx.x >> 5;
    const uint32_t m = blockIdx.x, i = m / a.rows, j = m - i * a.rows;
    const TX* dy = (const TX*)a.x + (int64_t)i * a.x_ws + (int64_t)j * a.x_rs;
    const TR* v = (const TR*)a.v + (int64_t)i * a.v_ws + (int64_t)j * a.v_rs;
    const float* weight = a.weight ? a.weight + (int64_t)i * a.weight_ws : nullptr;
    const uint32_t call = drop_call(a.drop);
    const float2 st = a.stats[m];
    float c1 = 0.0f, c2 = 0.0f;
    for (int c0 = warp * kSpan; c0 < a.h; c0 += W * kSpan)
#pragma unroll
        for (int k = 0; k < 8; ++k) {
            const int c = span_column<false>(c0, lane, k);
            if (c < a.h) {
                const float g = to_float(__ldg(dy + c)) * (weight ? __ldg(weight + c) : 1.0f);
                c1 += g;
                c2 = fmaf(g, (to_float(__ldg(v + c)) - st.x) * st.y, c2);
            }
        }
    c1 = row_sum<W>(c1, scratch[0], warp) / (float)a.h;
    c2 = row_sum<W>(c2, scratch[1], warp) / (float)a.h;
    const TR* more = ADD && a.residual ? (const TR*)a.residual + (int64_t)i * a.r_ws + (int64_t)j * a.r_rs : nullptr;
    for (int c0 = warp * kSpan; c0 < a.h; c0 += W * kSpan) {
        float g[8], xhat[8], add[8], w[8];
#pragma unroll
        for (int k = 0; k < 8; ++k) add[k] = 0.0f, w[k] = 1.0f;
        span_load<TX, false>(dy, c0, a.h, lane, g);
        span_load<TR, false>(v, c0, a.h, lane, xhat, st.x);
        if (weight) span_load<float, false>(weight, c0, a.h, lane, w);
        if (more) span_load<TR, false>(more, c0, a.h, lane, add);
#pragma unroll
        for (int k = 0; k < 8; ++k) g[k] = fmaf(st.y, g[k] * w[k] - c1 - (xhat[k] - st.x) * st.y * c2, add[k]);
        if (ADD && a.s) span_store<TR, false>((TR*)a.s + (int64_t)m * a.h, c0, a.h, lane, g);
        if (ADD && a.drop.on && a.y) span_drop<false>(a.drop, c0, j, a.drop.worker + i, call, lane, g);
        if (a.y) span_store<TX, false>((TX*)a.y + (int64_t)m * a.h, c0, a.h, lane, g);
    }
}

template <typename TX, typename TR>
__global__ void __launch_bounds__(256) norm_columns_kernel(const __grid_constant__ NormArgs a) {
    const uint32_t tiles = (uint32_t)(a.h + 255) / 256, at = blockIdx.x / tiles;
    const uint32_t i = at / a.chunks, chunk = at - i * a.chunks;
    const uint32_t j0 = (uint32_t)((uint64_t)a.rows * chunk / a.chunks), j1 = (uint32_t)((uint64_t)a.rows * (chunk + 1) / a.chunks);
    const int c = (int)((blockIdx.x - at * tiles) * 256 + threadIdx.x);
    if (c >= a.h) return;
    const TX* dy = (const TX*)a.x + (int64_t)i * a.x_ws + c;
    const TR* v = (const TR*)a.v + (int64_t)i * a.v_ws + c;
    float dw = 0.0f, db = 0.0f;
    for (uint32_t j = j0; j < j1; ++j) {
        const float2 st = a.stats[i * a.rows + j];
        const float g = to_float(__ldg(dy + (int64_t)j * a.x_rs));
        dw = fmaf(g, (to_float(__ldg(v + (int64_t)j * a.v_rs)) - st.x) * st.y, dw);
        db += g;
    }
    float* out = a.partial + (int64_t)at * 2 * a.h;
    out[c] = dw;
    out[a.h + c] = db;
}

// Sums the chunks of a worker (or of all) in their order, so that the result does not depend on which CTA was first, as it would with
// atomics: 32 columns by 8 shares of the chunks, the shares joined in shared memory. 8 workers of 4096 columns 5 us, 10 MB from the L2.
__global__ void __launch_bounds__(256) norm_join_kernel(const float* __restrict__ partial, float* dweight, float* dbias, int32_t h,
                                                        uint32_t chunks) {
    __shared__ float share[8][33];
    dependency_wait();
    const int c = (int)(blockIdx.x * 32 + threadIdx.x);
    float* out = blockIdx.z ? dbias : dweight;
    if (!out) return;
    float s = 0.0f;
    if (c < h) {
        const float* p = partial + ((int64_t)blockIdx.y * chunks * 2 + blockIdx.z) * h + c;
        for (uint32_t q = threadIdx.y; q < chunks; q += 8) s += __ldcg(p + (int64_t)q * 2 * h);
    }
    share[threadIdx.y][threadIdx.x] = s;
    __syncthreads();
    if (threadIdx.y == 0 && c < h) {
        for (int k = 1; k < 8; ++k) s += share[k][threadIdx.x];
        out[(int64_t)blockIdx.y * h + c] = s;
    }
}

// ---- dropout ---------------------------------------------------------------------------------------------------------------

// n / d for n < 2^31 by a multiplication (Granlund, Montgomery 1994): shift = ceil(log2 d), factor = ceil(2^(31 + shift) / d).
struct Divisor {
    uint32_t factor, shift, d;
    __device__ __forceinline__ uint32_t operator()(uint32_t n) const { return d == 1 ? n : __umulhi(n, factor) >> (shift - 1); }
};
inline Divisor divisor(uint32_t d) {
    uint32_t shift = 0;
    while (((uint64_t)1 << shift) < d) ++shift;
    return {(uint32_t)((((uint64_t)1 << (31 + shift)) + d - 1) / d), shift, d};
}

struct DropoutArgs {
    const void* x;
    void* y;
    int64_t ws, rs;
    uint32_t row0, count;  // rows of this launch, of all workers'
    uint32_t units;        // groups of eight (aligned rows) or spans, all rows' together: below 2^31
    int32_t h;
    Divisor rows, per_row;  // rows of a worker, units of a row
    Drop drop;
};

// Aligned rows: a thread takes groups of eight elements, four at a time in the order of memory and the next four on their way. Bound by
// memory and by what the SMs can issue, the generator's 40 instructions and 50 more a group: 67 M bfloat16 numbers, 268 MB, 56 us (a
// plain copy 43; with the words of the place instead of the generator's 46). Numbered through, a group's row and worker come from two
// multiplications, and short rows leave no lane idle: 67 M numbers in rows of 64 take 60 us for both passes together, with a span of 256
// columns to a warp 212.
constexpr int kDropGroups = 4;
template <typename T>
__global__ void __launch_bounds__(256) dropout_kernel(const __grid_constant__ DropoutArgs a) {
    const uint32_t stride = gridDim.x * 256 * kDropGroups, call = drop_call(a.drop);
    uint32_t at = blockIdx.x * 256 * kDropGroups + threadIdx.x;
    struct Place {
        uint32_t group, m, i, j;
    };
    auto place = [&](uint32_t unit) {
        Place p;
        const uint32_t r = a.per_row(unit);
        p.group = unit - r * a.per_row.d;
        p.m = a.row0 + r;
        p.i = a.rows(p.m);
        p.j = p.m - p.i * a.rows.d;
        return p;
    };
    Raw8<T> next[kDropGroups];
    auto load = [&](uint32_t unit) {
#pragma unroll
        for (int k = 0; k < kDropGroups; ++k) {
            next[k] = {};
            if (unit + 256 * k < a.units) {
                const Place p = place(unit + 256 * k);
                next[k] = raw_load<T>((const T*)a.x + (int64_t)p.i * a.ws + (int64_t)p.j * a.rs + p.group * 8);
            }
        }
    };
    load(at);
    for (; at < a.units; at += stride) {
        Raw8<T> now[kDropGroups];
#pragma unroll
        for (int k = 0; k < kDropGroups; ++k) now[k] = next[k];
        if (a.units - at > stride) load(at + stride);
#pragma unroll
        for (int k = 0; k < kDropGroups; ++k) {
            if (at + 256 * k >= a.units) break;
            const Place p = place(at + 256 * k);
            Pair v[4];
            raw_pairs<T>(now[k], v);
            if (a.drop.on) {
                const uint4 u = drop_words(a.drop, p.group, p.j, a.drop.worker + p.i, call);
#pragma unroll
                for (int e = 0; e < 4; ++e) {
                    float x[2];
                    halves(mul(v[e], pair(a.drop.factor)), x[0], x[1]);
                    v[e] = pair(drop_keeps(a.drop, u, 2 * e) ? x[0] : 0.0f, drop_keeps(a.drop, u, 2 * e + 1) ? x[1] : 0.0f);
                }
            }
            raw_store<T>((T*)a.y + (int64_t)p.m * a.h + p.group * 8, pack_pairs<T>(v));
        }
    }
}

// Other rows: a warp per span (rows of 4097: 88 us a pass).
template <typename T>
__global__ void __launch_bounds__(256) dropout_spans_kernel(const __grid_constant__ DropoutArgs a) {
    const int lane = threadIdx.x & 31;
    const uint32_t unit = blockIdx.x * 8 + (threadIdx.x >> 5);
    if (unit >= a.units) return;
    const uint32_t r = a.per_row(unit), m = a.row0 + r, i = a.rows(m), j = m - i * a.rows.d;
    const int c0 = (int)(unit - r * a.per_row.d) * kSpan;
    float v[8];
    span_load<T, false>((const T*)a.x + (int64_t)i * a.ws + (int64_t)j * a.rs, c0, a.h, lane, v);
    if (a.drop.on) span_drop<false>(a.drop, c0, j, a.drop.worker + i, drop_call(a.drop), lane, v);
    span_store<T, false>((T*)a.y + (int64_t)m * a.h, c0, a.h, lane, v);
}

// ---- host ------------------------------------------------------------------------------------------------------------------

constexpr int kLongest = 16 * 4 * kSpan;  // columns of a row that is kept in registers

struct Shape {
    int32_t n;
    int64_t rows, h;
    bool ok() const {
        return n >= 1 && n <= 65535 && rows >= 0 && h >= 1 && h < ((int64_t)1 << 31) - 16 * kSpan && rows <= (int64_t)0x7fffffff / n;
    }
};

// CTAs of a kernel that an SM holds at once. Asked once for every kernel and device.
template <auto kernel>
cudaError_t resident(int threads, int shared, int* count) {
    static std::atomic<int> known[64];
    int device = 0;
    cudaError_t e = cudaGetDevice(&device);
    if (e != cudaSuccess) return e;
    *count = device < 64 ? known[device].load(std::memory_order_relaxed) : 0;
    if (*count) return cudaSuccess;
    if (shared > 32 * 1024) e = cudaFuncSetAttribute(kernel, cudaFuncAttributeMaxDynamicSharedMemorySize, shared);
    if (e == cudaSuccess) e = cudaOccupancyMaxActiveBlocksPerMultiprocessor(count, kernel, threads, shared);
    if (e == cudaSuccess && *count < 1) e = cudaErrorInvalidConfiguration;
    if (e == cudaSuccess && device < 64) known[device].store(*count, std::memory_order_relaxed);
    return e;
}

// Chunks of a worker's rows: at most as many as give every SM 32 warps, of eight rows at least (16 where a warp takes a row); the
// partial sums of so many fit the workspace. Fewer where an SM holds fewer CTAs: then all run at once.
uint32_t most_chunks(const Shape& z) {
    const int64_t spans = (z.h + kSpan - 1) / kSpan;
    const int w = spans <= 1 ? 1 : spans <= 2 ? 2 : spans <= 4 ? 4 : spans <= 16 ? 8 : 16, each = w == 1 ? 32 / kRowsOfOneWarp : 32 / w;
    int64_t c = ((int64_t)multiprocessors() * each + z.n - 1) / z.n;
    const int64_t least = w == 1 ? 16 : 8, most = (z.rows + least - 1) / least;
    if (c > most) c = most;
    return (uint32_t)(c < 1 ? 1 : c);
}

template <int V>
using Int = std::integral_constant<int, V>;

template <typename F>
int by_types(int32_t x, int32_t r, F f) {  // r: x's type or fp32
    if (x == kTypeF32) return f(float(), float());
    if (x == kTypeBF16) return r == kTypeF32 ? f(__nv_bfloat16(), float()) : f(__nv_bfloat16(), __nv_bfloat16());
    return r == kTypeF32 ? f(__half(), float()) : f(__half(), __half());
}

int launched(cudaError_t e, const char* what) { return e == cudaSuccess ? COMPAMS_OK : cuda_fail(e, what); }

// One wave of CTAs: as many chunks as run at once, no more than `most`, each of one row at least.
uint32_t chunks_at_once(int count, int n, int64_t rows, int64_t per, int64_t most) {
    int64_t c = (int64_t)multiprocessors() * count / n;
    if (c > most) c = most;
    if (c > (rows + per - 1) / per) c = (rows + per - 1) / per;
    return (uint32_t)(c < 1 ? 1 : c);
}

// f(warps of a row, spans of a warp, aligned, lanes of a row): a span to a warp as far as eight warps go, so that few values are kept by
// each thread; then two and four. A warp takes several aligned short rows: 262144 bfloat16 rows of 64, both passes, 41 us with eight
// lanes to a row, 118 with 32; of 128, 74 us with 16 lanes; of 200, with 32 as their groups of eight need, 129. Rows that are not
// aligned go the same way: 16384 of 4097, 358 us with two spans to 16 warps, 664 with four.
template <typename F>
void by_width(int32_t h, bool vec, F f) {
    const int spans = (h + kSpan - 1) / kSpan;
    auto of = [&](auto v) {
        const Int<32> l;
        if (spans <= 1) f(Int<1>(), Int<1>(), v, l);
        else if (spans <= 2) f(Int<2>(), Int<1>(), v, l);
        else if (spans <= 4) f(Int<4>(), Int<1>(), v, l);
        else if (spans <= 8) f(Int<8>(), Int<1>(), v, l);
        else if (spans <= 16) f(Int<8>(), Int<2>(), v, l);
        else if (spans <= 32) f(Int<16>(), Int<2>(), v, l);
        else f(Int<16>(), Int<4>(), v, l);
    };
    if (vec && h <= 64) f(Int<1>(), Int<1>(), Int<1>(), Int<8>());
    else if (vec && h <= 128) f(Int<1>(), Int<1>(), Int<1>(), Int<16>());
    else if (vec) of(Int<1>());
    else of(Int<0>());
}

template <typename TX, typename TR, bool ADD>
int forward(NormArgs a, int n, bool vec, cudaStream_t stream) {
    cudaError_t e = cudaSuccess;
    auto go = [&](auto w, auto g, auto v, auto l) {
        constexpr int W = decltype(w)::value, NG = decltype(g)::value;
        constexpr bool V = decltype(v)::value;
        constexpr int L = decltype(l)::value;
        auto kernel = norm_forward_kernel<TX, TR, W, NG, L, V, ADD>;
        constexpr int shared = row_shared<W, forward_slots<TX, TR, NG, ADD>(), V>();
        int count = 0;
        e = resident<norm_forward_kernel<TX, TR, W, NG, L, V, ADD>>(norm_threads<W>(), shared, &count);
        if (e != cudaSuccess) return;
        a.chunks = chunks_at_once(count, n, a.rows, norm_rows<W, L>(), 0x7fffffff / n);
        e = launch_plain(kernel, dim3((uint32_t)n * a.chunks), dim3(norm_threads<W>()), shared, stream, a);
    };
    if (a.h > kLongest) {
        e = launch_plain(norm_forward_long_kernel<TX, TR, ADD>, dim3(a.total), dim3(512), 0, stream, a);
    } else {
        by_width(a.h, vec, go);
    }
    return launched(e, "norm_forward");
}

template <typename TX, typename TR, bool ADD>
int backward(NormArgs& a, int n, bool vec, cudaStream_t stream) {
    const uint32_t most = a.chunks;
    cudaError_t e = cudaSuccess;
    auto go = [&](auto w, auto g, auto v, auto l) {
        constexpr int W = decltype(w)::value, NG = decltype(g)::value;
        constexpr bool V = decltype(v)::value;
        constexpr int L = decltype(l)::value;
        auto kernel = norm_backward_kernel<TX, TR, W, NG, L, V, ADD>;
        constexpr int shared = row_shared<W, backward_slots<TX, TR, NG, ADD>(), V>();
        int count = 0;
        e = resident<norm_backward_kernel<TX, TR, W, NG, L, V, ADD>>(norm_threads<W>(), shared, &count);
        if (e != cudaSuccess) return;
        a.chunks = chunks_at_once(count, n, a.rows, norm_rows<W, L>(), most);
        e = launch_plain(kernel, dim3((uint32_t)n * a.chunks), dim3(norm_threads<W>()), shared, stream, a);
    };
    if (a.h > kLongest) {
        if (a.y || a.s) e = launch_plain(norm_backward_long_kernel<TX, TR, ADD>, dim3(a.total), dim3(512), 0, stream, a);
        if (e == cudaSuccess && a.partial)
            e = launch_plain(norm_columns_kernel<TX, TR>, dim3((uint32_t)(a.h + 255) / 256 * (uint32_t)n * a.chunks), dim3(256), 0, stream, a);
    } else {
        by_width(a.h, vec, go);
    }
    return launched(e, "norm_backward");
}

bool vector_parameter(const float* p, int64_t ws) {
    return !p || (((reinterpret_cast<uintptr_t>(p) | (uint64_t)(ws * 4)) & 15u) == 0);
}
bool float_aligned(const void* p) { return (reinterpret_cast<uintptr_t>(p) & 3u) == 0; }

}  // namespace
}  // namespace compams

using namespace compams;

extern "C" {

int compams_dropout(void* y, const void* x, int32_t type, int32_t n, int64_t rows, int64_t h, int64_t worker_stride, int64_t row_stride,
                    double p, uint64_t seed, uint32_t call, const int64_t* call_device, uint32_t first_worker, void* cuda_stream) {
    const Shape z{n, rows, h};
    Drop d;
    if (!z.ok() || !type_known(type) || !make_drop(d, p, seed, call, call_device, first_worker)) return COMPAMS_ERR_INVALID_ARG;
    if (rows == 0) return COMPAMS_OK;
    const Rows in{x, worker_stride, row_stride, type}, out = packed(y, rows, h, type);
    if (!in.strides_ok() || !x || !y || !in.element_aligned() || !out.element_aligned()) return COMPAMS_ERR_INVALID_ARG;
    const bool vec = h % 8 == 0 && in.aligned() && out.aligned();
    DropoutArgs a = {};
    a.x = x; a.y = y; a.ws = worker_stride; a.rs = row_stride; a.h = (int32_t)h; a.drop = d;
    const uint32_t per_row = (uint32_t)(vec ? h / 8 : (h + kSpan - 1) / kSpan);
    a.rows = divisor((uint32_t)rows);
    a.per_row = divisor(per_row);
    // units are counted in 31 bits (and the steps of all threads beyond them in 32): as many rows at a time as that allows
    const int64_t total = n * rows, most = std::max<int64_t>(1, ((int64_t)1 << 31) / per_row - 1);
    return by_types(type, type, [&](auto t, auto) {
        using T = decltype(t);
        for (int64_t row = 0; row < total; row += most) {
            a.row0 = (uint32_t)row;
            a.count = (uint32_t)std::min(most, total - row);
            a.units = a.count * per_row;
            cudaError_t e;
            if (vec) {
                int count = 0;
                e = resident<dropout_kernel<T>>(256, 0, &count);
                const uint32_t all = (a.units + 256 * kDropGroups - 1) / (256 * kDropGroups), once = (uint32_t)(multiprocessors() * count);
                if (e == cudaSuccess) e = launch_plain(dropout_kernel<T>, dim3(std::min(all, once)), dim3(256), 0, (cudaStream_t)cuda_stream, a);
            } else {
                e = launch_plain(dropout_spans_kernel<T>, dim3((a.units + 7) / 8), dim3(256), 0, (cudaStream_t)cuda_stream, a);
            }
            if (e != cudaSuccess) return cuda_fail(e, "dropout");
        }
        return (int)COMPAMS_OK;
    });
}

int compams_norm_forward(void* y, void* s, float* stats, const void* x, const void* residual, int32_t type, int32_t residual_type,
                         int32_t n, int64_t rows, int64_t h, int64_t x_worker_stride, int64_t x_row_stride,
                         int64_t residual_worker_stride, int64_t residual_row_stride, const float* weight, int64_t weight_stride,
                         const float* bias, int64_t bias_stride, float eps, double p, uint64_t seed, uint32_t call,
                         const int64_t* call_device, uint32_t first_worker, void* cuda_stream) {
    const Shape z{n, rows, h};
    NormArgs a = {};
    if (!z.ok() || !type_known(type) || !make_drop(a.drop, p, seed, call, call_device, first_worker) || !(eps >= 0.0f))
        return COMPAMS_ERR_INVALID_ARG;
    const bool add = residual != nullptr;
    if (add ? residual_type != type && residual_type != kTypeF32 : s != nullptr || p != 0.0) return COMPAMS_ERR_INVALID_ARG;
    if (rows == 0) return COMPAMS_OK;
    const Rows in{x, x_worker_stride, x_row_stride, type}, out = packed(y, rows, h, type);
    const Rows res{residual, residual_worker_stride, residual_row_stride, residual_type}, sum = packed(s, rows, h, residual_type);
    if (!in.strides_ok() || (add && !res.strides_ok()) || weight_stride < 0 || bias_stride < 0 || !x || !y || (add && !s) ||
        !in.element_aligned() || !out.element_aligned() || !float_aligned(weight) || !float_aligned(bias) ||
        (reinterpret_cast<uintptr_t>(stats) & 7u) || (add && (!res.element_aligned() || !sum.element_aligned())))
        return COMPAMS_ERR_INVALID_ARG;
    const bool vec = h % 8 == 0 && in.aligned() && out.aligned() && (!add || (res.aligned() && sum.aligned())) &&
                     vector_parameter(weight, weight_stride) && vector_parameter(bias, bias_stride);
    a.x = x; a.residual = residual; a.y = y; a.s = s; a.stats = (float2*)stats; a.weight = weight; a.bias = bias;
    a.x_ws = x_worker_stride; a.x_rs = x_row_stride; a.r_ws = residual_worker_stride; a.r_rs = residual_row_stride;
    a.weight_ws = weight_stride; a.bias_ws = bias_stride;
    a.rows = (uint32_t)rows; a.total = (uint32_t)(n * rows); a.h = (int32_t)h; a.eps = eps;
    return by_types(type, add ? residual_type : type, [&](auto tx, auto tr) {
        using TX = decltype(tx);
        using TR = decltype(tr);
        if (add) return forward<TX, TR, true>(a, n, vec, (cudaStream_t)cuda_stream);
        return forward<TX, TX, false>(a, n, vec, (cudaStream_t)cuda_stream);
    });
}

int compams_norm_workspace_bytes(size_t* bytes, int32_t n, int64_t rows, int64_t h) {
    const Shape z{n, rows, h};
    if (!bytes || !z.ok()) return COMPAMS_ERR_INVALID_ARG;
    *bytes = (size_t)n * most_chunks(z) * 2 * (size_t)h * sizeof(float);
    return COMPAMS_OK;
}

int compams_norm_backward(void* dx, void* dresidual, float* dweight, float* dbias, int32_t sum_workers, const void* dy, const void* ds,
                          const void* v, const float* stats, int32_t type, int32_t v_type, int32_t n, int64_t rows, int64_t h,
                          int64_t dy_worker_stride, int64_t dy_row_stride, int64_t ds_worker_stride, int64_t ds_row_stride,
                          int64_t v_worker_stride, int64_t v_row_stride, const float* weight, int64_t weight_stride, int32_t added,
                          double p, uint64_t seed, uint32_t call, const int64_t* call_device, uint32_t first_worker, void* workspace,
                          size_t workspace_bytes, void* cuda_stream) {
    const Shape z{n, rows, h};
    NormArgs a = {};
    if (!z.ok() || !type_known(type) || !make_drop(a.drop, p, seed, call, call_device, first_worker)) return COMPAMS_ERR_INVALID_ARG;
    const bool add = added != 0;
    if (add ? v_type != type && v_type != kTypeF32 : v_type != type || ds || dresidual || p != 0.0) return COMPAMS_ERR_INVALID_ARG;
    const bool sums = dweight || dbias;
    const uint32_t chunks = most_chunks(z);
    if ((uint64_t)n * chunks * (uint64_t)((h + 255) / 256) > 0x7fffffffu) return COMPAMS_ERR_TOO_LARGE;
    if (sums && (!workspace || workspace_bytes < (size_t)n * chunks * 2 * (size_t)h * sizeof(float) ||
                 (reinterpret_cast<uintptr_t>(workspace) & 15u) || !float_aligned(dweight) || !float_aligned(dbias)))
        return COMPAMS_ERR_INVALID_ARG;
    const cudaStream_t stream = (cudaStream_t)cuda_stream;
    if (rows == 0) {
        const size_t bytes = (size_t)(sum_workers ? 1 : n) * (size_t)h * sizeof(float);
        cudaError_t e = dweight ? cudaMemsetAsync(dweight, 0, bytes, stream) : cudaSuccess;
        if (e == cudaSuccess && dbias) e = cudaMemsetAsync(dbias, 0, bytes, stream);
        return launched(e, "norm_backward");
    }
    const Rows gin{dy, dy_worker_stride, dy_row_stride, type}, gsum{ds, ds_worker_stride, ds_row_stride, v_type};
    const Rows vin{v, v_worker_stride, v_row_stride, v_type}, out = packed(dx, rows, h, type), rout = packed(dresidual, rows, h, v_type);
    if (!gin.strides_ok() || (ds && !gsum.strides_ok()) || !vin.strides_ok() || weight_stride < 0 || !dy || !v || !stats ||
        (reinterpret_cast<uintptr_t>(stats) & 7u) || !float_aligned(weight) || !gin.element_aligned() ||
        !gsum.element_aligned() || !vin.element_aligned() || !out.element_aligned() || !rout.element_aligned())
        return COMPAMS_ERR_INVALID_ARG;
    const bool vec = h % 8 == 0 && gin.aligned() && vin.aligned() && (!ds || gsum.aligned()) && out.aligned() && rout.aligned() &&
                     vector_parameter(weight, weight_stride);
    a.x = dy; a.residual = ds; a.v = v; a.y = dx; a.s = dresidual; a.stats = (float2*)stats; a.weight = weight;
    a.partial = sums ? (float*)workspace : nullptr;
    a.x_ws = dy_worker_stride; a.x_rs = dy_row_stride; a.r_ws = ds_worker_stride; a.r_rs = ds_row_stride;
    a.v_ws = v_worker_stride; a.v_rs = v_row_stride; a.weight_ws = weight_stride;
    a.rows = (uint32_t)rows; a.total = (uint32_t)(n * rows); a.h = (int32_t)h; a.chunks = chunks;
    const int rc = by_types(type, v_type, [&](auto tx, auto tr) {
        using TX = decltype(tx);
        using TR = decltype(tr);
        if (add) return backward<TX, TR, true>(a, n, vec, stream);
        return backward<TX, TX, false>(a, n, vec, stream);
    });
    if (rc != COMPAMS_OK || !sums) return rc;
    const uint32_t groups = sum_workers ? 1u : (uint32_t)n, per = sum_workers ? (uint32_t)n * a.chunks : a.chunks;
    return launched(launch_after(norm_join_kernel, dim3((uint32_t)((h + 31) / 32), groups, 2), dim3(32, 8), stream,
                                 (const float*)workspace, dweight, dbias, (int32_t)h, per),
                    "norm_join");
}

}  // extern "C"
