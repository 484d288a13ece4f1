// The head of a language model with the n workers' micro-batches in one batch: logits z = x W^T over a vocabulary, softmax cross entropy
// with a target for each row, and the gradients of x and W, without the logits ever being in memory as a whole.
//
//   lse_j = log sum_v exp(z_jv)           loss_j = lse_j - z_j,target(j)     (0 where the target is ignored)
//   d_jv  = (exp(z_jv - lse_j) - [v = target(j)]) g_j          g_j: the loss's gradient, for a mean divided by the worker's counted rows
//   dx_j  = sum_v d_jv W_v                dW_v = sum_j d_jv x_j
//
// Forward: the products (head_tensor.cuh) leave a row's maximum and sum of exponentials for every 128 columns, 8 bytes in the place of
// 512, which `join` brings together. Backward: the vocabulary goes by in pieces; a piece's logits are formed again and leave as d in 16
// bits, as far as it fits a workspace that does not grow with the vocabulary, and the two products that read d follow. So a training
// step does four products of 2 m h V operations where three would do for someone who keeps the logits: with m = 8192 rows, V = 100000 and
// fp32 they would be 3.3 GB.
//
// A few rows (kFew) read W once, a warp taking rows of W whole, in fp32 arithmetic: bound by memory; backward for d as well, so that the logits
// of both passes are the same.
//
// Precision. Products of 16-bit numbers of one type are exact and their sums fp32. Beside an fp32 weight everything is bf16 planes: an fp32
// number is three (each the rest of those before it, rounded), fp16 two; pairs of planes i + j <= 2 are formed, which leaves out at most
// 2^-24 of a product. d is one plane (2^-9 of it at most left out) where the result has 8 bits, two for fp16 beside an fp32 weight, three
// for an fp32 result. The rows' factors g are taken relative to their worker's: a mean's and a sum's g, the same for all rows of a worker,
// stays out of d altogether and joins in fp32, so that d of the target, p - 1, is not rounded the same way in every row (8192 rows,
// 100000 columns: 2.9e-3 off with g inside, 2.2e-3 now, of which rounding the result is 1.7e-3); without a reduction it is taken relative
// to a power of two above the worker's largest, and where d is fp16, which could not hold rows far below it, to one of the row's own: dx
// then has its row's, and d is brought to the worker's before the sum over the rows. For dx of 8 bits beside an fp32 weight two
// planes of W are taken. lse is one fp32 number, so every p, and the target's p - 1, is off by up to half a step of it (1e-6 for 16 to 32).
// No atomics: results do not change from run to run.
#include <string.h>

#include <algorithm>
#include <atomic>
#include <type_traits>

#include "context.h"
#include "head_tensor.cuh"

namespace compams {
namespace {

using head::power2;
using head::kLog2e;

constexpr float kInf = __builtin_inff();
constexpr int kVocab = 128;  // columns of a statistic of head_tensor.cuh

// (m, s) stands for s exp(m).
__device__ __forceinline__ float2 merged(float2 a, float2 b) {
    const float m = fmaxf(a.x, b.x), base = m == -kInf ? 0.0f : m;
    return make_float2(m, fmaf(a.y, power2((a.x - base) * kLog2e), b.y * power2((b.x - base) * kLog2e)));
}

// ---- operands as 16-bit planes ---------------------------------------------------------------------------------------------

struct PackArgs {
    const void* src;
    int64_t ws, rs;       // of src
    int64_t rows, row0;   // rows of a batch that are taken, from row0 on
    int64_t chunks;       // of all batches: eight columns each
    int32_t h, per_row;   // columns; chunks of a row, the last padded with zeros
    uint16_t* out;        // [plane][batch][rows][8 per_row]
    int64_t plane;        // elements
};
// Of up to two tensors of a type: the second's chunks are numbered behind the first's.
template <typename T, int P, bool VEC>
__global__ void __launch_bounds__(256) pack_kernel(const __grid_constant__ PackArgs first, const __grid_constant__ PackArgs second) {
    dependency_wait();
    int64_t at = (int64_t)blockIdx.x * 256 + threadIdx.x;
    if (at >= first.chunks + second.chunks) return;
    const bool behind = at >= first.chunks;
    const PackArgs& a = behind ? second : first;
    if (behind) at -= first.chunks;
    const int64_t row = at / a.per_row, batch = row / a.rows;
    const int c = (int)(at - row * a.per_row) * 8;
    const T* x = (const T*)a.src + batch * a.ws + (a.row0 + row - batch * a.rows) * a.rs + c;
    Raw8<T> raw;
    float v[8];
    if (VEC) {
        raw = raw_load<T>(x);
        raw_floats<T>(raw, v);
    } else {
#pragma unroll
        for (int k = 0; k < 8; ++k) v[k] = c + k < a.h ? to_float(x[k]) : 0.0f;
    }
    uint4 out[P];
    if constexpr (P == 1) {  // a copy: the type's own bits
        out[0] = make_uint4(pack(v[0], v[1], T()), pack(v[2], v[3], T()), pack(v[4], v[5], T()), pack(v[6], v[7], T()));
    } else {
        uint32_t w[4][P];
#pragma unroll
        for (int q = 0; q < 4; ++q) split2<P>(v[2 * q], v[2 * q + 1], w[q]);
#pragma unroll
        for (int p = 0; p < P; ++p) out[p] = make_uint4(w[0][p], w[1][p], w[2][p], w[3][p]);
    }
#pragma unroll
    for (int p = 0; p < P; ++p) *reinterpret_cast<uint4*>(a.out + p * a.plane + at * 8) = out[p];
}

// ---- a few rows ------------------------------------------------------------------------------------------------------------

constexpr int kFew = 4;                   // rows of a batch
constexpr int64_t kFewShared = 96 * 1024;  // bytes that they take in shared memory: two CTAs to an SM

struct FewArgs {
    const void *x, *weight;
    int64_t x_ws, x_rs, w_ws, w_rs;
    int32_t h, vocab, rows, worker_rows;  // rows of a batch, and of a worker
    int64_t all_rows;
    const int64_t* target;
    float* target_logit;
    float2* stats;  // [CTA][all rows]
    // PROBS: of the columns from `first` on, the first `vocab` (weight is that of `first`)
    const float *lse, *row_gradient;
    int64_t ignored;
    int32_t first, all_columns, probs, f16;
    uint16_t* d;           // [plane][all rows][width]; zeros behind the last column up to a multiple of 64
    int64_t width;
};
// A warp takes a share of the rows of W, for one row of x a row at a time and eight CTAs to an SM (32000 rows of 4096 bfloat16 columns, 262 MB:
// 46 us; four rows at a time and four CTAs 49, two and six 51), for more of them four, so that x is read once for four; a lane has eight
// columns (or every 32nd) of each. Two to four rows of x: shares for four CTAs to an SM, of which the registers let two (two rows of x) or one
// be there at a time. 32000 rows of W in shares for four / three / two: two rows of 4096 65 / 76 / 61 us, of 8192 110 / 137 / 113, four of 1024
// 46 / 48 / 42, of 4096 113 / 117 / 105, of 6144 155 / 159 / 141.
constexpr int staged_rows(int rows) { return rows == 3 ? 4 : rows; }  // the kernel's MR: three rows are taken as four
__host__ __device__ constexpr int rows_at_once(int rows) { return rows == 1 ? 1 : 4; }
__host__ __device__ constexpr int ctas_at_once(int rows) { return rows == 1 ? 8 : 4; }
// PROBS: the same logits, to the last bit, and d from them: a target that is nearly certain has d = p - 1, which another order of the sums
// would be in the place of.
template <typename TX, typename TW, int MR, bool VEC, bool PROBS>
__global__ void __launch_bounds__(256, MR == 1 ? ctas_at_once(MR) : 1) few_kernel(const __grid_constant__ FewArgs a) {
    extern __shared__ __align__(16) float xs[];  // [MR][h up to a multiple of 8]
    __shared__ float2 joint[8][MR];
    constexpr int kRows = rows_at_once(MR);
    const int warp = threadIdx.x >> 5, lane = threadIdx.x & 31, pitch = (a.h + 7) & ~7;
    const int64_t batch = blockIdx.y, number0 = batch * a.rows;
    const TW* weight = (const TW*)a.weight + batch * a.w_ws;
    // a warp's rows, as many as any other's but for one
    const int64_t warps = (int64_t)gridDim.x * 8, mine = (int64_t)blockIdx.x * 8 + warp;
    const int last = (int)(a.vocab * (mine + 1) / warps);
    const int start = (int)(a.vocab * mine / warps);
    for (int r = 0; r < MR; ++r) {
        const TX* x = (const TX*)a.x + (batch + r / a.worker_rows) * a.x_ws + r % a.worker_rows * a.x_rs;
        for (int c = threadIdx.x; c < pitch; c += 256) xs[r * pitch + c] = r < a.rows && c < a.h ? to_float(x[c]) : 0.0f;
    }
    __syncthreads();
    int64_t target[MR];
    float2 state[MR];
#pragma unroll
    for (int r = 0; r < MR; ++r) {
        target[r] = r < a.rows ? a.target[number0 + r] : -1;
        state[r] = make_float2(-kInf, 0.0f);
    }
    // PROBS: a lane's row of x, and which of the rows of W it writes
    const int own = lane % MR, own_j = lane / MR;
    const bool writes = PROBS && own < a.rows && own_j < kRows;
    float lse = 0.0f, g = 0.0f;
    int64_t own_target = -1;
    uint16_t* d = nullptr;
    if (writes) {
        const int64_t number = number0 + own;
        own_target = a.target[number];
        lse = a.lse[number];
        g = a.row_gradient ? a.row_gradient[number]
                           : own_target == a.ignored ? 0.0f : own_target >= 0 && own_target < a.all_columns ? 1.0f : __int_as_float(0x7fffffff);
        d = a.d + number * a.width;
        if (blockIdx.x == 0 && warp == 0 && own_j == 0)
            for (int p = 0; p < a.probs; ++p)
                for (int c = a.vocab; c < (a.vocab + 63) / 64 * 64; ++c) d[p * a.all_rows * a.width + c] = 0;
    }
    for (int v0 = start; v0 < last; v0 += kRows) {
        float acc[kRows][MR] = {};
        const TW* row[kRows];
#pragma unroll
        for (int j = 0; j < kRows; ++j) row[j] = weight + (int64_t)min(v0 + j, last - 1) * a.w_rs;
        if constexpr (VEC) {
#pragma unroll 2
            for (int c = lane * 8; c < a.h; c += kSpan) {
                Raw8<TW> raw[kRows];
#pragma unroll
                for (int j = 0; j < kRows; ++j) raw[j] = raw_load<TW>(row[j] + c);
                float w[kRows][8];
#pragma unroll
                for (int j = 0; j < kRows; ++j) raw_floats<TW>(raw[j], w[j]);
#pragma unroll
                for (int r = 0; r < MR; ++r) {
                    float v[8];
                    *reinterpret_cast<float4*>(v) = *reinterpret_cast<const float4*>(xs + r * pitch + c);
                    *reinterpret_cast<float4*>(v + 4) = *reinterpret_cast<const float4*>(xs + r * pitch + c + 4);
#pragma unroll
                    for (int j = 0; j < kRows; ++j)
#pragma unroll
                        for (int k = 0; k < 8; ++k) acc[j][r] = fmaf(w[j][k], v[k], acc[j][r]);
                }
            }
        } else {
#pragma unroll 4
            for (int c = lane; c < a.h; c += 32) {
                float w[kRows];
#pragma unroll
                for (int j = 0; j < kRows; ++j) w[j] = to_float(__ldg(row[j] + c));
#pragma unroll
                for (int r = 0; r < MR; ++r)
#pragma unroll
                    for (int j = 0; j < kRows; ++j) acc[j][r] = fmaf(w[j], xs[r * pitch + c], acc[j][r]);
            }
        }
        float mine = 0.0f;
#pragma unroll
        for (int j = 0; j < kRows; ++j)
#pragma unroll
            for (int r = 0; r < MR; ++r) {
                float z = acc[j][r];
#pragma unroll
                for (int o = 16; o; o >>= 1) z += __shfl_xor_sync(0xffffffffu, z, o);
                const int v = v0 + j;
                if (PROBS) {
                    if (lane == j * MR + r) mine = z;
                } else if (v < last) {
                    state[r] = merged(state[r], make_float2(z, 1.0f));
                    if (lane == 0 && v == target[r]) a.target_logit[number0 + r] = z;
                }
            }
        if (PROBS && writes && v0 + own_j < last) {
            const int v = v0 + own_j;
            float rest = 0.0f;
            if (g != 0.0f) rest = (power2((mine - lse) * kLog2e) - (a.first + v == own_target ? 1.0f : 0.0f)) * (a.f16 ? g * head::kF16Scale : g);
            for (int p = 0; p < a.probs; ++p) {
                float none = 0.0f;
                d[p * a.all_rows * a.width + v] = (uint16_t)head::plane_of(rest, none, a.f16 != 0, p + 1 == a.probs);
            }
        }
    }
    if (PROBS) return;
#pragma unroll
    for (int r = 0; r < MR; ++r)
        if (lane == 0) joint[warp][r] = state[r];
    __syncthreads();
    if (threadIdx.x < a.rows) {
        float2 v = joint[0][threadIdx.x];
#pragma unroll
        for (int w = 1; w < 8; ++w) v = merged(v, joint[w][threadIdx.x]);
        a.stats[blockIdx.x * a.all_rows + number0 + threadIdx.x] = v;
    }
}

// ---- losses ----------------------------------------------------------------------------------------------------------------

enum Reduction : int32_t { kNone = 0, kMean = 1, kSum = 2 };

struct JoinArgs {
    const float2* stats;  // [part][all rows]
    const float* target_logit;
    const int64_t* target;
    int64_t all_rows, rows, parts, ignored, vocab;
    int32_t lanes;      // rows of a CTA, a power of two up to 256
    int32_t whole;      // a CTA has a worker's rows, all of them
    int32_t reduction;
    float *lse, *row_loss, *loss, *inverse;  // the last: a mean's 1 / counted rows, a sum's 1
};
__device__ __forceinline__ float sum_of_warp(float v) {
#pragma unroll
    for (int o = 16; o; o >>= 1) v += __shfl_xor_sync(0xffffffffu, v, o);
    return v;
}
// 32 rows (fewer where there are fewer, a worker's up to 256 where the parts are few) by 1024 / rows shares of the parts.
__global__ void __launch_bounds__(1024) join_kernel(const __grid_constant__ JoinArgs a) {
    __shared__ float2 shares[1024], joint[8];
    dependency_wait();
    const int r = threadIdx.x & (a.lanes - 1), share = threadIdx.x / a.lanes, count = 1024 / a.lanes;
    const int64_t row = (int64_t)blockIdx.x * (a.whole ? a.rows : a.lanes) + r;
    const bool there = a.whole ? r < a.rows : row < a.all_rows;
    float2 v = make_float2(-kInf, 0.0f);
    if (there)
#pragma unroll 4
        for (int64_t p = share; p < a.parts; p += count) v = merged(v, a.stats[p * a.all_rows + row]);
    shares[threadIdx.x] = v;
    for (int o = count / 2; o; o >>= 1) {
        __syncthreads();
        if (share < o) shares[threadIdx.x] = merged(shares[threadIdx.x], shares[threadIdx.x + o * a.lanes]);
    }
    if (threadIdx.x >= 32 && (int)threadIdx.x >= a.lanes) return;  // (whole warps)
    __syncwarp();
    float loss = 0.0f, counted = 0.0f;
    if (there && (int)threadIdx.x < a.lanes) {
        v = shares[threadIdx.x];
        const float log_sum = logf(v.y), lse = v.x + log_sum;
        const int64_t t = a.target[row];
        a.lse[row] = lse;
        if (t != a.ignored) {
            counted = 1.0f;
            // (the logits' difference first: where the target is nearly certain lse has rounded away what the loss is)
            loss = t >= 0 && t < a.vocab ? (v.x - a.target_logit[row]) + log_sum : __int_as_float(0x7fffffff);  // no such column
        }
        if (a.reduction == kNone) a.loss[row] = loss;
        else if (!a.whole) a.row_loss[row] = loss;
    }
    if (a.reduction == kNone || !a.whole) return;
    loss = sum_of_warp(loss);
    counted = sum_of_warp(counted);
    const int warps = (a.lanes + 31) / 32;
    if (warps > 1) {
        if ((threadIdx.x & 31) == 0) joint[threadIdx.x >> 5] = make_float2(loss, counted);
        asm volatile("bar.sync 1, %0;" ::"r"(warps * 32) : "memory");
        loss = counted = 0.0f;
        for (int w = 0; w < warps; ++w) {
            loss += joint[w].x;
            counted += joint[w].y;
        }
    }
    if (threadIdx.x == 0) {
        const float inverse = a.reduction == kMean ? 1.0f / fmaxf(counted, 1.0f) : 1.0f;
        a.inverse[blockIdx.x] = inverse;
        a.loss[blockIdx.x] = a.reduction == kMean ? loss / fmaxf(counted, 1.0f) : loss;
    }
}
// A worker's loss from its rows'.
__global__ void __launch_bounds__(256) reduce_kernel(const float* __restrict__ row_loss, const int64_t* __restrict__ target, int64_t rows,
                                                     int64_t ignored, int32_t reduction, float* __restrict__ loss, float* __restrict__ inverse) {
    __shared__ float sums[8], counts[8];
    dependency_wait();
    const int64_t row0 = blockIdx.x * rows;
    float sum = 0.0f, count = 0.0f;
    for (int64_t j = threadIdx.x; j < rows; j += 256) {
        sum += row_loss[row0 + j];
        count += target[row0 + j] != ignored ? 1.0f : 0.0f;
    }
    sum = sum_of_warp(sum);
    count = sum_of_warp(count);
    if ((threadIdx.x & 31) == 0) {
        sums[threadIdx.x >> 5] = sum;
        counts[threadIdx.x >> 5] = count;
    }
    __syncthreads();
    if (threadIdx.x == 0) {
        for (int w = 1; w < 8; ++w) {
            sum += sums[w];
            count += counts[w];
        }
        loss[blockIdx.x] = reduction == kMean ? sum / fmaxf(count, 1.0f) : sum;
        inverse[blockIdx.x] = reduction == kMean ? 1.0f / fmaxf(count, 1.0f) : 1.0f;
    }
}

// ---- the rows' gradients ---------------------------------------------------------------------------------------------------

struct RowsArgs {
    const float* dloss;
    int64_t ws, rs;
    const int64_t* target;
    int64_t rows, ignored, vocab;
    float *g, *scale;         // [all rows], [n]
    float *row_scale, *back;  // [all rows], where d is fp16; else null
};
// The exponent of the power of two above v, as far as it and its inverse are finite.
__device__ __forceinline__ int exponent_above(float v) {
    int e = 0;
    if (v > 0.0f && v < kInf) frexpf(v, &e);
    return min(max(e, -100), 127);
}
// Without a reduction: a CTA per worker, its rows' g relative to the power of two above the largest; where d is fp16, to that above the row's
// own, with what takes it from there to the result and to the worker's.
__global__ void __launch_bounds__(256) rows_kernel(const __grid_constant__ RowsArgs a) {
    __shared__ float tops[8];
    dependency_wait();
    const int64_t i = blockIdx.x;
    const int64_t* target = a.target + i * a.rows;
    const float* dloss = a.dloss + i * a.ws;
    float top = 0.0f;
    for (int64_t j = threadIdx.x; j < a.rows; j += 256)
        if (target[j] != a.ignored) top = fmaxf(top, fabsf(dloss[j * a.rs]));
#pragma unroll
    for (int o = 16; o; o >>= 1) top = fmaxf(top, __shfl_xor_sync(0xffffffffu, top, o));
    if ((threadIdx.x & 31) == 0) tops[threadIdx.x >> 5] = top;
    __syncthreads();
#pragma unroll
    for (int w = 0; w < 8; ++w) top = fmaxf(top, tops[w]);
    const int e = exponent_above(top);
    const float inverse = ldexpf(1.0f, -e), result = a.row_scale ? 1.0f / head::kF16Scale : 1.0f;
    if (threadIdx.x == 0) a.scale[i] = ldexpf(result, e);
    for (int64_t j = threadIdx.x; j < a.rows; j += 256) {
        const int64_t t = target[j], number = i * a.rows + j;
        const float v = t == a.ignored ? 0.0f : dloss[j * a.rs];
        float by = inverse;
        if (a.row_scale) {
            const int own = v != 0.0f ? exponent_above(fabsf(v)) : e;
            by = ldexpf(1.0f, -own);
            a.row_scale[number] = ldexpf(result, own);
            a.back[number] = ldexpf(1.0f, own - e);
        }
        a.g[number] = t == a.ignored ? 0.0f : t >= 0 && t < a.vocab ? by * v : __int_as_float(0x7fffffff);  // no such column
    }
}
// A piece's d from the rows' own powers of two to their workers'.
__global__ void __launch_bounds__(256) back_kernel(uint4* __restrict__ d, const float* __restrict__ back, int64_t chunks, int32_t per_row, int64_t pitch) {
    dependency_wait();
    const int64_t at = (int64_t)blockIdx.x * 256 + threadIdx.x;
    if (at >= chunks) return;
    const int64_t row = at / per_row;
    const float by = back[row];
    if (by == 1.0f) return;
    uint4& place = d[row * pitch + (at - row * per_row)];
    float v[8];
    raw_floats<__half>(Raw8<__half>{place}, v);
#pragma unroll
    for (int k = 0; k < 8; ++k) v[k] *= by;
    store8<__half>(reinterpret_cast<__half*>(&place), v);
}

// dx from the parts' sums.
struct PartsArgs {
    const float* parts;  // [parts][all rows][pitch]
    int64_t part, all_rows, chunks;
    int32_t count, h, per_row, pitch;
    head::Scale scale;   // of a worker
    int64_t worker_rows;
    void* out;           // [all rows][h]
};
template <typename T, bool VEC>
__global__ void __launch_bounds__(256) parts_kernel(const __grid_constant__ PartsArgs a) {
    dependency_wait();
    const int64_t at = (int64_t)blockIdx.x * 256 + threadIdx.x;
    if (at >= a.chunks) return;
    const int64_t row = at / a.per_row;
    const int c = (int)(at - row * a.per_row) * 8;
    float v[8] = {};
    for (int s = 0; s < a.count; ++s) {
        const float* from = a.parts + s * a.part + row * a.pitch + c;
        const float4 p = *reinterpret_cast<const float4*>(from), q = *reinterpret_cast<const float4*>(from + 4);
        v[0] += p.x; v[1] += p.y; v[2] += p.z; v[3] += p.w;
        v[4] += q.x; v[5] += q.y; v[6] += q.z; v[7] += q.w;
    }
    const float scale = head::scale_of(a.scale, row / a.worker_rows);
#pragma unroll
    for (int k = 0; k < 8; ++k) v[k] *= scale;
    T* out = (T*)a.out + row * a.h + c;
    if (VEC) {
        store8<T>(out, v);
    } else {
#pragma unroll
        for (int k = 0; k < 8; ++k)
            if (c + k < a.h) out[k] = from_float<T>(v[k]);
    }
}

// ---- host ------------------------------------------------------------------------------------------------------------------

std::atomic<uint32_t> wait_tries{tensor::kTries};

struct HeadShape {
    int32_t n;
    int64_t rows, h, vocab;
    int32_t type, weight_type;
    bool shared;  // one weight for all workers
    bool ok() const {
        return n >= 1 && n <= 65535 && rows >= 0 && rows <= (int64_t)0x7fffffff / n && h >= 1 && h < ((int64_t)1 << 31) - 4096 && vocab >= 1 &&
               vocab < ((int64_t)1 << 31) - 4096 && type_known(type) && type_known(weight_type) && (type == weight_type || weight_type == kTypeF32);
    }
    bool copies() const { return weight_type == kTypeF32; }  // operands are planes, never the caller's own memory
    bool f16() const { return type == kTypeF16 && !copies(); }
    int x_planes() const { return !copies() || type == kTypeBF16 ? 1 : type == kTypeF16 ? 2 : 3; }
    int w_planes() const { return copies() ? 3 : 1; }
    int64_t batches() const { return shared ? 1 : n; }
    int64_t batch_rows() const { return shared ? n * rows : rows; }
    int64_t all_rows() const { return n * rows; }
    int64_t pitch() const { return (h + 7) / 8 * 8; }
    bool few() const { return batch_rows() <= kFew && staged_rows((int)batch_rows()) * pitch() * 4 <= kFewShared; }
    // planes of d: for dx, for dW
    int x_probs() const { return type == kTypeF32 ? 3 : type == kTypeF16 && copies() ? 2 : 1; }
    int w_probs() const { return copies() ? 3 : 1; }
};

// Rows on 16-byte boundaries and one behind the other, as TMA takes them; where there is but one row or batch its stride does not count.
struct Matrix {
    const void* p;
    int64_t row_stride, batch_stride;  // elements
};
bool lies_well(const Matrix& m, int64_t rows, int64_t batches, int64_t h) {
    return ((reinterpret_cast<uintptr_t>(m.p) & 15u) == 0) && (rows == 1 || (m.row_stride % 8 == 0 && m.row_stride >= h && m.row_stride < (int64_t)1 << 38)) &&
           (batches == 1 || (m.batch_stride % 8 == 0 && m.batch_stride >= 1 && m.batch_stride < (int64_t)1 << 38));
}
// x as one batch of all workers' rows; false where the workers do not lie so.
bool flat(const HeadShape& z, int64_t ws, int64_t rs, int64_t& stride) {
    stride = z.rows == 1 ? ws : rs;
    return z.rows == 1 || z.n == 1 || ws == z.rows * rs;
}
bool x_lies_well(const HeadShape& z, const void* x, int64_t ws, int64_t rs, Matrix& m) {
    if (z.x_planes() > 1) return false;
    int64_t stride = rs;
    if (z.shared) {
        if (!flat(z, ws, rs, stride)) return false;
        m = {x, stride, 0};
        return lies_well(m, z.all_rows(), 1, z.h);
    }
    m = {x, rs, ws};
    return lies_well(m, z.rows, z.n, z.h);
}
bool w_lies_well(const HeadShape& z, const void* w, int64_t ws, int64_t rs, Matrix& m) {
    if (z.copies()) return false;
    m = {w, rs, ws};
    return lies_well(m, z.vocab, z.batches(), z.h);
}

// How the vocabulary goes by, and where things lie in the workspace.
struct Plan {
    int64_t piece, pieces;  // columns, a multiple of 256 unless it is all of them
    int64_t width;          // columns of d
    int32_t probs, parts;   // planes of d; parts of the vocabulary's sum of dx
    bool sums;              // dx is added up in fp32
    int64_t x_copy, w_copy, stats, stat_parts, target_logit, row_loss, g, row_scale, back, scale, d, dx_sums, bytes;
};
constexpr int64_t kCopyBytes = 64ll << 20;   // of a piece's copy of W: it stays in the L2 between its writing and its reading
constexpr int64_t kProbsBytes = 512ll << 20;  // of a piece's d
constexpr int64_t kSumsBytes = 256ll << 20;   // of the parts' sums of dx

int64_t up_to(int64_t v, int64_t to) { return (v + to - 1) / to * to; }
int64_t few_ctas(const HeadShape& z, int64_t columns) {
    return std::max<int64_t>(1, std::min<int64_t>((columns + 31) / 32, ((int64_t)multiprocessors() * ctas_at_once((int)z.batch_rows()) + z.batches() - 1) / z.batches()));
}

// Parts of the vocabulary's sum of dx: as many as take the pairs of CTAs the shortest time, in tiles of 64 (0.3 us), with what adding up
// the parts costs.
int32_t parts_of(const HeadShape& z, int64_t steps, int pairs) {
    const int64_t m = z.batch_rows(), tiles = (m + 255) / 256 * ((z.h + 255) / 256) * z.batches(), at_once = std::max(1, multiprocessors() / 2);
    int32_t best = 1;
    double least = 1e30;
    for (int32_t s = 1; s <= 32 && s * 4 <= std::max<int64_t>(steps, 4) && (s == 1 || s * z.all_rows() * z.pitch() * 4 <= kSumsBytes); ++s) {
        const double waves = (double)((tiles * s + at_once - 1) / at_once);
        const double t = waves * (0.3 * pairs * (double)((steps + s - 1) / s) + 2.0) +
                         (s > 1 ? 3.0 + s * (double)z.all_rows() * z.pitch() * 8e-6 / 5.0 : 0.0);
        if (t < 0.98 * least) {
            least = t;
            best = s;
        }
    }
    return best;
}

Plan plan_of(const HeadShape& z, bool x_copied, bool w_copied, int wanted) {  // wanted: 0 forward, else 1 dx + 2 dW
    Plan p = {};
    const int64_t m = z.all_rows();
    p.probs = std::max(wanted & 1 ? z.x_probs() : 0, wanted & 2 ? z.w_probs() : 0);
    p.piece = z.vocab;
    const bool few = !wanted && z.few();
    if (!few) {
        int64_t most = up_to(z.vocab, 256);
        if (w_copied) most = std::min(most, std::max<int64_t>(256, kCopyBytes / (z.w_planes() * z.batches() * z.pitch() * 2) / 256 * 256));
        if (wanted) most = std::min(most, std::max<int64_t>(256, kProbsBytes / (p.probs * m * 2) / 256 * 256));
        p.pieces = (z.vocab + most - 1) / most;
        p.piece = std::min(z.vocab, up_to((z.vocab + p.pieces - 1) / p.pieces, 256));
    }
    p.pieces = (z.vocab + p.piece - 1) / p.piece;
    p.width = up_to(p.piece, 256);
    int64_t at = 0;
    auto take = [&](int64_t bytes) {
        const int64_t here = at;
        at += up_to(bytes, 256);
        return here;
    };
    if (x_copied && !few) p.x_copy = take(z.x_planes() * m * z.pitch() * 2);
    if (w_copied && !few) p.w_copy = take(z.w_planes() * z.batches() * p.piece * z.pitch() * 2);
    if (!wanted) {
        p.stat_parts = few ? few_ctas(z, z.vocab) : (z.vocab + kVocab - 1) / kVocab;
        p.stats = take(p.stat_parts * m * 8);
        p.target_logit = take(m * 4);
        p.row_loss = take(m * 4);
    } else {
        p.g = take(m * 4);
        if (z.f16()) {
            p.row_scale = take(m * 4);
            p.back = take(m * 4);
        }
        p.scale = take(z.n * 4);
        p.d = take(p.probs * m * p.width * 2);
        p.parts = wanted & 1 ? parts_of(z, (p.piece + 63) / 64, z.x_probs() == 3 ? 6 : z.x_probs() == 2 ? 3 : z.copies() ? 2 : 1) : 1;
        p.sums = (wanted & 1) && (p.parts > 1 || p.pieces > 1);
        if (p.sums) p.dx_sums = take(p.parts * m * z.pitch() * 4);
    }
    p.bytes = at;
    return p;
}

// An operand: 16-bit planes, [plane][batch][rows][columns].
struct Operand {
    const void* p;
    int64_t columns, rows, batches, planes;
    int64_t row_stride, batch_stride;  // elements; plane after plane
};
bool operand_map(CUtensorMap* map, const Operand& o, bool f16, uint32_t box_rows) {
    const Encode encode = map_encoder();
    if (!encode) return false;
    const int64_t row = o.rows > 1 ? o.row_stride : up_to(o.columns, 8), batch = o.batches * o.planes > 1 ? o.batch_stride : row * o.rows;
    const cuuint64_t size[3] = {(cuuint64_t)o.columns, (cuuint64_t)o.rows, (cuuint64_t)(o.batches * o.planes)};
    const cuuint64_t stride[2] = {(cuuint64_t)row * 2, (cuuint64_t)batch * 2};
    const cuuint32_t extent[3] = {64, box_rows, 1}, every[3] = {1, 1, 1};
    return encode(map, f16 ? CU_TENSOR_MAP_DATA_TYPE_FLOAT16 : CU_TENSOR_MAP_DATA_TYPE_BFLOAT16, 3, const_cast<void*>(o.p), size, stride, extent,
                  every, CU_TENSOR_MAP_INTERLEAVE_NONE, CU_TENSOR_MAP_SWIZZLE_128B, CU_TENSOR_MAP_L2_PROMOTION_L2_256B,
                  CU_TENSOR_MAP_FLOAT_OOB_FILL_NONE) == CUDA_SUCCESS;
}

// Pairs of planes whose indices together are at most `order`, small ones first.
void pairs_of(head::Args& a, int left, int right, int order) {
    a.pairs = 0;
    for (int both = order; both >= 0; --both)
        for (int i = 0; i <= both; ++i)
            if (i < left && both - i < right) {
                a.left_plane[a.pairs] = (uint8_t)i;
                a.right_plane[a.pairs++] = (uint8_t)(both - i);
            }
}

// What a form writes: fp32 or 16-bit rows [batches][rows][columns] for boxes of 64 bytes and 32 rows; false where TMA cannot address them.
bool result_map(CUtensorMap* map, void* p, int32_t type, int64_t columns, int64_t rows, int64_t batches, int64_t row, int64_t batch) {
    const Encode encode = map_encoder();
    const int64_t e = type_bytes(type);
    if (!encode || (reinterpret_cast<uintptr_t>(p) & 15u) || (row * e) % 16 || (batch * e) % 16 || row * e >= (int64_t)1 << 40 || batch * e >= (int64_t)1 << 40)
        return false;
    const cuuint64_t size[3] = {(cuuint64_t)columns, (cuuint64_t)rows, (cuuint64_t)batches};
    const cuuint64_t stride[2] = {(cuuint64_t)(row * e), (cuuint64_t)(batch * e)};
    const cuuint32_t extent[3] = {(cuuint32_t)(64 / e), 32, 1}, every[3] = {1, 1, 1};
    const auto kind = type == kTypeF32 ? CU_TENSOR_MAP_DATA_TYPE_FLOAT32 : type == kTypeBF16 ? CU_TENSOR_MAP_DATA_TYPE_BFLOAT16 : CU_TENSOR_MAP_DATA_TYPE_FLOAT16;
    return encode(map, kind, 3, p, size, stride, extent, every, CU_TENSOR_MAP_INTERLEAVE_NONE, CU_TENSOR_MAP_SWIZZLE_64B,
                  CU_TENSOR_MAP_L2_PROMOTION_NONE, CU_TENSOR_MAP_FLOAT_OOB_FILL_NONE) == CUDA_SUCCESS;
}

template <int FORM>
int product(head::Args& a, const Operand& left, const Operand& right, const CUtensorMap& out, bool f16, cudaStream_t stream, const char* what) {
    using O = head::Order<FORM>;
    CUtensorMap l = {}, r = {};
    if (!operand_map(&l, left, f16, O::kLeftAcross ? 64 : 128) || !operand_map(&r, right, f16, O::kRightAcross ? 64 : 128))
        return COMPAMS_ERR_INVALID_ARG;
    a.left_planes = (int32_t)left.batches;
    a.right_planes = (int32_t)right.batches;
    a.left_batch = left.batches > 1;
    a.right_batch = right.batches > 1;
    for (int k = 0; k < a.pairs; ++k) {
        a.left_count = std::max(a.left_count, a.left_plane[k] + 1);
        a.right_count = std::max(a.right_count, a.right_plane[k] + 1);
    }
    a.stages = std::min(head::kMostStages, head::kHalves / (a.left_count + a.right_count));
    a.stretch = std::max(1, head::flush_after(a.pairs) / a.pairs);
    a.f16 = f16;
    a.tries = wait_tries.load(std::memory_order_relaxed);
    const int64_t tiles = (int64_t)a.tiles_m * a.tiles_n * a.batches * a.parts;
    if (tiles > 0x3fffffff) return COMPAMS_ERR_TOO_LARGE;
    const int64_t at_once = std::max(1, multiprocessors() / 2);
    return launched(launch_sized(head::head_kernel<FORM>, dim3((uint32_t)(2 * std::min(tiles, at_once))), head::kThreads, 2, head::kShared, false,
                                 stream, a, l, r, out),
                    what);
}

// What is to be brought into planes: rows row0 ... row0 + rows of every batch of a matrix.
struct Job {
    Matrix m;
    int64_t rows, row0, batches;
    void* out;
};
template <typename T, int P>
int pack(const Job* jobs, int count, int64_t h, cudaStream_t stream) {
    PackArgs a[2] = {};
    bool vec = h % 8 == 0;
    for (int k = 0; k < count; ++k) {
        const Job& j = jobs[k];
        a[k].src = j.m.p; a[k].ws = j.m.batch_stride; a[k].rs = j.m.row_stride; a[k].rows = j.rows; a[k].row0 = j.row0; a[k].h = (int32_t)h;
        a[k].per_row = (int32_t)((h + 7) / 8);
        a[k].chunks = j.batches * j.rows * a[k].per_row;
        a[k].out = (uint16_t*)j.out; a[k].plane = a[k].chunks * 8;
        vec = vec && ((reinterpret_cast<uintptr_t>(j.m.p) | (uint64_t)(j.m.row_stride * (int64_t)sizeof(T)) |
                       (uint64_t)(j.m.batch_stride * (int64_t)sizeof(T))) & 15u) == 0;
    }
    const int64_t ctas = (a[0].chunks + a[1].chunks + 255) / 256;
    if (ctas > 0x7fffffff) return COMPAMS_ERR_TOO_LARGE;
    const auto kernel = vec ? pack_kernel<T, P, true> : pack_kernel<T, P, false>;
    return launched(launch_sized(kernel, dim3((uint32_t)ctas), 256, 1, 0, false, stream, a[0], a[1]), "head_pack");
}
int pack(int32_t type, int planes, const Job* jobs, int count, int64_t h, cudaStream_t stream) {
    if (type == kTypeF32) return pack<float, 3>(jobs, count, h, stream);
    if (type == kTypeBF16) return pack<__nv_bfloat16, 1>(jobs, count, h, stream);
    return planes == 2 ? pack<__half, 2>(jobs, count, h, stream) : pack<__half, 1>(jobs, count, h, stream);
}

// x and the piece of the weight from row v0 on as operands: the caller's memory, or copies, [plane][batch][rows][columns]. The weight's piece
// starts at row `first` of its operand. x_too: x has not been copied yet.
int operands(const HeadShape& z, const void* x, int64_t x_ws, int64_t x_rs, const void* w, int64_t w_ws, int64_t w_rs, const Plan& p, int64_t v0,
             int64_t count, bool x_too, char* work, Operand& xo, Operand& wo, int32_t& first, cudaStream_t stream) {
    Job jobs[2];
    int much = 0;
    Matrix m;
    xo = {nullptr, z.h, z.batch_rows(), z.batches(), z.x_planes(), 0, 0};
    if (x_lies_well(z, x, x_ws, x_rs, m)) {
        xo.p = m.p; xo.row_stride = m.row_stride; xo.batch_stride = m.batch_stride;
    } else {
        xo.p = work + p.x_copy; xo.row_stride = z.pitch(); xo.batch_stride = z.batch_rows() * z.pitch(); xo.columns = z.pitch();
        if (x_too) jobs[much++] = {{x, x_rs, x_ws}, z.rows, 0, z.n, work + p.x_copy};
    }
    wo = {nullptr, z.h, z.vocab, z.batches(), z.w_planes(), 0, 0};
    first = (int32_t)v0;
    if (w_lies_well(z, w, w_ws, w_rs, m)) {
        wo.p = m.p; wo.row_stride = m.row_stride; wo.batch_stride = m.batch_stride;
        return much ? pack(z.type, z.x_planes(), jobs, 1, z.h, stream) : (int)COMPAMS_OK;
    }
    first = 0;
    wo.p = work + p.w_copy; wo.rows = count; wo.columns = z.pitch(); wo.row_stride = z.pitch(); wo.batch_stride = count * z.pitch();
    const Job weight{{w, w_rs, w_ws}, count, v0, z.batches(), work + p.w_copy};
    if (much && z.type == z.weight_type) {  // both at once
        jobs[much++] = weight;
        return pack(z.type, z.x_planes(), jobs, 2, z.h, stream);
    }
    const int rc = much ? pack(z.type, z.x_planes(), jobs, 1, z.h, stream) : (int)COMPAMS_OK;
    return rc == COMPAMS_OK ? pack(z.weight_type, z.w_planes(), &weight, 1, z.h, stream) : rc;
}

template <typename TX, typename TW, int MR>
int few_rows(const HeadShape& z, const FewArgs& a, bool vec, int64_t ctas, cudaStream_t stream) {
    const auto kernel = a.d ? (vec ? few_kernel<TX, TW, MR, true, true> : few_kernel<TX, TW, MR, false, true>)
                            : (vec ? few_kernel<TX, TW, MR, true, false> : few_kernel<TX, TW, MR, false, false>);
    return launched(launch_sized(kernel, dim3((uint32_t)ctas, (uint32_t)z.batches()), 256, 1, Shared((size_t)(MR * z.pitch() * 4), kFewShared), true,
                                 stream, a),
                    "head_few");
}
template <typename TX, typename TW>
int few_rows(const HeadShape& z, const FewArgs& a, int64_t ctas, cudaStream_t stream) {
    const bool vec = z.h % 8 == 0 && ((reinterpret_cast<uintptr_t>(a.weight) | (uint64_t)(a.w_rs * (int64_t)sizeof(TW)) |
                                       (uint64_t)(a.w_ws * (int64_t)sizeof(TW))) & 15u) == 0;
    const int staged = staged_rows(a.rows);
    return staged == 1 ? few_rows<TX, TW, 1>(z, a, vec, ctas, stream)
                       : staged == 2 ? few_rows<TX, TW, 2>(z, a, vec, ctas, stream) : few_rows<TX, TW, 4>(z, a, vec, ctas, stream);
}

// The logits of a few rows for `columns` rows of the weight, a.weight on.
int few_rows(const HeadShape& z, FewArgs& a, const void* x, int64_t x_ws, int64_t x_rs, int64_t w_ws, int64_t w_rs, int64_t columns, cudaStream_t stream) {
    a.x = x; a.x_ws = x_ws; a.x_rs = x_rs; a.w_ws = z.shared ? 0 : w_ws; a.w_rs = w_rs; a.h = (int32_t)z.h; a.vocab = (int32_t)columns;
    a.rows = (int32_t)z.batch_rows(); a.worker_rows = (int32_t)z.rows; a.all_rows = z.all_rows();
    const int64_t ctas = few_ctas(z, columns);
    const bool wide = z.weight_type == kTypeF32;
    return z.type == kTypeF32 ? few_rows<float, float>(z, a, ctas, stream)
           : z.type == kTypeBF16 ? (wide ? few_rows<__nv_bfloat16, float>(z, a, ctas, stream) : few_rows<__nv_bfloat16, __nv_bfloat16>(z, a, ctas, stream))
                                 : (wide ? few_rows<__half, float>(z, a, ctas, stream) : few_rows<__half, __half>(z, a, ctas, stream));
}

bool float_aligned(const void* p) { return (reinterpret_cast<uintptr_t>(p) & 3u) == 0; }
bool element_aligned(const void* p, int32_t type) { return (reinterpret_cast<uintptr_t>(p) & (uintptr_t)(type_bytes(type) - 1)) == 0; }

}  // namespace
}  // namespace compams

using namespace compams;

extern "C" {

int compams_head_status(int32_t* gave_up) {
    if (!gave_up) return COMPAMS_ERR_INVALID_ARG;
    int32_t none = 0;
    cudaError_t e = cudaMemcpyFromSymbol(gave_up, head::gave_up, sizeof(int32_t));
    if (e == cudaSuccess && *gave_up) e = cudaMemcpyToSymbol(head::gave_up, &none, sizeof(int32_t));
    return launched(e, "head_status");
}

int compams_head_wait_tries(int32_t tries) {
    if (tries < 0 || tries > (int32_t)tensor::kTries) return COMPAMS_ERR_INVALID_ARG;
    wait_tries.store((uint32_t)tries, std::memory_order_relaxed);
    return COMPAMS_OK;
}

int compams_head_workspace_bytes(size_t* bytes, int32_t n, int64_t rows, int64_t h, int64_t vocab, int32_t type, int32_t weight_type,
                                 int32_t shared, int32_t x_copied, int32_t weight_copied, int32_t wanted) {
    const HeadShape z{n, rows, h, vocab, type, weight_type, shared != 0 || n == 1};
    if (!bytes || !z.ok() || wanted < 0 || wanted > 3) return COMPAMS_ERR_INVALID_ARG;
    *bytes = 0;
    if (rows == 0) return COMPAMS_OK;
    // Who says "copied" may find that a call reads it where it lies: a weight's copy makes pieces smaller, and with them d, so that either may
    // take more. (x's copy only adds to the others.)
    const bool x = x_copied || z.x_planes() > 1;
    int64_t most = plan_of(z, x, weight_copied || z.copies(), wanted).bytes;
    if (weight_copied && !z.copies()) most = std::max(most, plan_of(z, x, false, wanted).bytes);
    *bytes = (size_t)most;
    return COMPAMS_OK;
}

int compams_head_forward(float* loss, float* lse, const void* x, int32_t type, const void* weight, int32_t weight_type, const int64_t* target,
                         int32_t n, int64_t rows, int64_t h, int64_t vocab, int64_t x_worker_stride, int64_t x_row_stride,
                         int64_t weight_worker_stride, int64_t weight_row_stride, int64_t ignored, int32_t reduction, void* workspace,
                         size_t workspace_bytes, void* cuda_stream) {
    const HeadShape z{n, rows, h, vocab, type, weight_type, weight_worker_stride == 0 || n == 1};
    if (!z.ok() || reduction < kNone || reduction > kSum || x_worker_stride < 0 || x_row_stride < 0 || weight_worker_stride < 0 ||
        weight_row_stride < 0 || !float_aligned(loss) || (!loss && (rows || reduction)))
        return COMPAMS_ERR_INVALID_ARG;
    const cudaStream_t stream = (cudaStream_t)cuda_stream;
    if (rows == 0) return reduction == kNone ? COMPAMS_OK : launched(cudaMemsetAsync(loss, 0, (size_t)n * 4, stream), "head_forward");
    Matrix m;
    const Plan p = plan_of(z, !x_lies_well(z, x, x_worker_stride, x_row_stride, m),
                           !w_lies_well(z, weight, weight_worker_stride, weight_row_stride, m), 0);
    if (!lse || !x || !weight || !target || !workspace || workspace_bytes < (size_t)p.bytes || (reinterpret_cast<uintptr_t>(workspace) & 255u) ||
        !float_aligned(lse) || !element_aligned(x, type) || !element_aligned(weight, weight_type) || (reinterpret_cast<uintptr_t>(target) & 7u))
        return COMPAMS_ERR_INVALID_ARG;
    char* work = (char*)workspace;
    float2* stats = (float2*)(work + p.stats);
    float* target_logit = (float*)(work + p.target_logit);
    int rc = COMPAMS_OK;
    if (z.few()) {
        FewArgs a = {};
        a.weight = weight; a.target = target; a.target_logit = target_logit; a.stats = stats;
        rc = few_rows(z, a, x, x_worker_stride, x_row_stride, weight_worker_stride, weight_row_stride, vocab, stream);
    } else {
        Operand xo, wo;
        for (int64_t v0 = 0; v0 < vocab && rc == COMPAMS_OK; v0 += p.piece) {
            const int64_t count = std::min(p.piece, vocab - v0);
            head::Args a = {};
            rc = operands(z, x, x_worker_stride, x_row_stride, weight, weight_worker_stride, weight_row_stride, p, v0, count, v0 == 0, work, xo, wo,
                          a.right_row, stream);
            if (rc != COMPAMS_OK) break;
            a.tiles_m = (int32_t)((z.batch_rows() + 255) / 256); a.tiles_n = (int32_t)((count + 255) / 256);
            a.batches = (int32_t)z.batches(); a.parts = 1;
            a.segments = 1; a.steps = a.part_steps = (int32_t)((h + 63) / 64);
            pairs_of(a, z.x_planes(), z.w_planes(), 2);
            a.rows = z.batch_rows(); a.columns = (int32_t)vocab; a.first = (int32_t)v0;
            a.target = target; a.target_logit = target_logit; a.stats = stats; a.all_rows = z.all_rows();
            rc = product<head::kForward>(a, xo, wo, {}, z.f16(), stream, "head_forward");
        }
    }
    if (rc != COMPAMS_OK) return rc;
    JoinArgs j = {};
    j.stats = stats; j.target_logit = target_logit; j.target = target; j.all_rows = z.all_rows(); j.rows = rows; j.parts = p.stat_parts;
    j.ignored = ignored; j.vocab = vocab; j.reduction = reduction; j.lse = lse; j.row_loss = (float*)(work + p.row_loss); j.loss = loss;
    j.inverse = lse + j.all_rows;
    // (256 rows of 250 parts: 16 us by one CTA a worker, 6 + 2 by two kernels; 100 of 63: 4.5, and a launch less)
    j.whole = reduction != kNone && (rows <= 32 || (rows <= 256 && rows * p.stat_parts <= 16384));
    const int64_t most = j.whole ? rows : std::min<int64_t>(32, j.all_rows);
    for (j.lanes = 1; j.lanes < most;) j.lanes *= 2;
    const int64_t ctas = j.whole ? n : (j.all_rows + j.lanes - 1) / j.lanes;
    rc = launched(launch_sized(join_kernel, dim3((uint32_t)ctas), 1024, 1, 0, false, stream, j), "head_join");
    if (rc != COMPAMS_OK || j.whole || reduction == kNone) return rc;
    return launched(launch_sized(reduce_kernel, dim3((uint32_t)n), 256, 1, 0, false, stream, (const float*)j.row_loss, target, rows, ignored,
                                 reduction, loss, j.inverse),
                    "head_reduce");
}

int compams_head_backward(void* dx, void* dweight, int32_t sum_workers, const float* dloss, int64_t dloss_worker_stride, int64_t dloss_row_stride,
                          const void* x, int32_t type, const void* weight, int32_t weight_type, const int64_t* target, const float* lse, int32_t n,
                          int64_t rows, int64_t h, int64_t vocab, int64_t x_worker_stride, int64_t x_row_stride, int64_t weight_worker_stride,
                          int64_t weight_row_stride, int64_t ignored, int32_t reduction, void* workspace, size_t workspace_bytes,
                          void* cuda_stream) {
    const HeadShape z{n, rows, h, vocab, type, weight_type, weight_worker_stride == 0 || n == 1};
    const bool together = sum_workers != 0;
    if (!z.ok() || reduction < kNone || reduction > kSum || x_worker_stride < 0 || x_row_stride < 0 || weight_worker_stride < 0 ||
        weight_row_stride < 0 || dloss_worker_stride < 0 || dloss_row_stride < 0 || (together && dweight && !z.shared) ||
        !element_aligned(dx, type) || !element_aligned(dweight, weight_type))
        return COMPAMS_ERR_INVALID_ARG;
    const cudaStream_t stream = (cudaStream_t)cuda_stream;
    const int64_t gradients = together ? 1 : n;
    if (rows == 0)
        return dweight ? launched(cudaMemsetAsync(dweight, 0, (size_t)(gradients * vocab * h * type_bytes(weight_type)), stream), "head_backward")
                       : COMPAMS_OK;
    const int wanted = (dx ? 1 : 0) | (dweight ? 2 : 0);
    if (!wanted) return COMPAMS_OK;
    Matrix m;
    const Plan p = plan_of(z, !x_lies_well(z, x, x_worker_stride, x_row_stride, m),
                           !w_lies_well(z, weight, weight_worker_stride, weight_row_stride, m), wanted);
    if (!dloss || !lse || !x || !weight || !target || !workspace || workspace_bytes < (size_t)p.bytes ||
        (reinterpret_cast<uintptr_t>(workspace) & 255u) || !float_aligned(lse) || !float_aligned(dloss) || !element_aligned(x, type) ||
        !element_aligned(weight, weight_type) || (reinterpret_cast<uintptr_t>(target) & 7u))
        return COMPAMS_ERR_INVALID_ARG;
    char* work = (char*)workspace;
    const int64_t all = z.all_rows();
    // a mean's and a sum's rows have d by itself, and the worker's factor is found where it is needed; without a reduction each has its own
    head::Scale scale = {nullptr, dloss, lse + all, dloss_worker_stride, z.f16() ? 1.0f / head::kF16Scale : 1.0f};
    const float* row_gradient = nullptr;
    int rc = COMPAMS_OK;
    if (reduction == kNone) {
        RowsArgs r = {};
        r.dloss = dloss; r.ws = dloss_worker_stride; r.rs = dloss_row_stride; r.target = target; r.rows = rows; r.ignored = ignored; r.vocab = vocab;
        r.g = (float*)(work + p.g); r.scale = (float*)(work + p.scale);
        if (z.f16()) { r.row_scale = (float*)(work + p.row_scale); r.back = (float*)(work + p.back); }
        rc = launched(launch_sized(rows_kernel, dim3((uint32_t)n), 256, 1, 0, true, stream, r), "head_rows");
        scale.own = r.scale;
        row_gradient = r.g;
    }
    head::Scale scale_x = scale;  // of dx: a worker's, or a row's own
    int64_t scale_rows = rows;
    const float* back = nullptr;
    if (reduction == kNone && z.f16()) {
        scale_x.own = (const float*)(work + p.row_scale);
        scale_rows = 1;
        back = (const float*)(work + p.back);
    }
    Operand xo, wo;
    uint16_t* d = (uint16_t*)(work + p.d);
    const int32_t tiles_h = (int32_t)((h + 255) / 256), tiles_rows = (int32_t)((z.batch_rows() + 255) / 256);
    for (int64_t v0 = 0; v0 < vocab && rc == COMPAMS_OK; v0 += p.piece) {
        const int64_t count = std::min(p.piece, vocab - v0);
        int32_t first = 0;
        rc = operands(z, x, x_worker_stride, x_row_stride, weight, weight_worker_stride, weight_row_stride, p, v0, count, v0 == 0, work, xo, wo, first,
                      stream);
        if (rc != COMPAMS_OK) break;
        if (z.few()) {  // (launched behind what still reads the last piece's d, all of it)
            FewArgs a = {};
            a.weight = (const char*)weight + v0 * weight_row_stride * type_bytes(weight_type); a.target = target;
            a.lse = lse; a.row_gradient = row_gradient; a.ignored = ignored; a.first = (int32_t)v0; a.all_columns = (int32_t)vocab;
            a.probs = p.probs; a.f16 = z.f16(); a.d = d; a.width = p.width;
            rc = few_rows(z, a, x, x_worker_stride, x_row_stride, weight_worker_stride, weight_row_stride, count, stream);
        } else {
            head::Args a = {};
            a.tiles_m = tiles_rows; a.tiles_n = (int32_t)((count + 255) / 256); a.batches = (int32_t)z.batches(); a.parts = 1;
            a.segments = 1; a.steps = a.part_steps = (int32_t)((h + 63) / 64);
            pairs_of(a, z.x_planes(), z.w_planes(), 2);
            a.right_row = first; a.rows = z.batch_rows(); a.columns = (int32_t)vocab; a.first = (int32_t)v0; a.target = target;
            a.all_rows = all; a.lse = lse; a.row_gradient = row_gradient; a.ignored = ignored; a.probs_planes = p.probs;
            CUtensorMap out = {};
            if (!result_map(&out, d, z.f16() ? kTypeF16 : kTypeBF16, p.width, z.batch_rows(), z.batches() * p.probs, p.width, z.batch_rows() * p.width))
                return COMPAMS_ERR_INVALID_ARG;
            rc = product<head::kProbs>(a, xo, wo, out, z.f16(), stream, "head_probs");
        }
        const Operand by_batch{d, p.width, z.batch_rows(), z.batches(), p.probs, p.width, z.batch_rows() * p.width};
        if (rc == COMPAMS_OK && dx) {
            head::Args a = {};
            a.tiles_m = tiles_rows; a.tiles_n = tiles_h; a.batches = (int32_t)z.batches(); a.parts = p.parts;
            a.segments = 1; a.steps = (int32_t)((count + 63) / 64); a.part_steps = (a.steps + p.parts - 1) / p.parts;
            // 8 bits beside an fp32 weight: two of its planes; 11 bits: to the same order
            pairs_of(a, z.x_probs(), z.copies() && type != kTypeF32 ? 2 : z.w_planes(), type == kTypeF32 ? 2 : 1);
            a.right_sum = first; a.rows = z.batch_rows();
            void* to = p.sums ? (void*)(work + p.dx_sums) : dx;
            a.out_row = p.sums ? z.pitch() : h;
            a.columns = (int32_t)a.out_row; a.out_type = p.sums ? kTypeF32 : type; a.out_batch = z.batch_rows() * a.out_row;
            a.add = p.sums && v0 > 0;
            a.scale = scale_x; a.worker_rows = scale_rows;
            if (p.sums) a.scale.factor = 0.0f;  // later
            CUtensorMap out = {};
            if (!result_map(&out, to, a.out_type, a.out_row, z.batch_rows(), z.batches() * p.parts, a.out_row, a.out_batch)) a.out = to;
            rc = product<head::kInput>(a, by_batch, wo, out, z.f16(), stream, "head_input");
        }
        if (rc == COMPAMS_OK && dweight && back) {
            const int32_t per_row = (int32_t)(up_to(count, 256) / 8);
            const int64_t ctas = (all * per_row + 255) / 256;
            if (ctas > 0x7fffffff) return COMPAMS_ERR_TOO_LARGE;
            rc = launched(launch_sized(back_kernel, dim3((uint32_t)ctas), 256, 1, 0, false, stream, (uint4*)d, back, all * per_row, per_row, p.width / 8),
                          "head_back");
        }
        if (rc == COMPAMS_OK && dweight) {
            // together: the workers are segments of one sum; else each is a batch
            head::Args a = {};
            a.tiles_m = (int32_t)((count + 255) / 256); a.tiles_n = tiles_h; a.batches = together ? 1 : n; a.parts = 1;
            a.segments = together ? n : 1; a.steps = a.part_steps = (int32_t)((rows + 63) / 64);
            pairs_of(a, z.w_probs(), z.x_planes(), 2);
            a.rows = count; a.columns = (int32_t)h; a.out_type = weight_type; a.out_row = h; a.out_batch = vocab * h; a.out_first = (int32_t)v0;
            a.scale = scale;
            CUtensorMap out = {};
            if (!result_map(&out, dweight, weight_type, h, vocab, together ? 1 : n, h, vocab * h)) a.out = dweight;
            const Operand left{d, p.width, rows, n, p.probs, p.width, rows * p.width};
            Operand right = xo;
            right.rows = rows; right.batches = n;
            if (z.shared) right.batch_stride = rows * (all > 1 ? xo.row_stride : z.pitch());
            rc = product<head::kWeight>(a, left, right, out, z.f16(), stream, "head_weight");
        }
    }
    if (rc != COMPAMS_OK || !p.sums || !dx) return rc;
    PartsArgs a = {};
    a.parts = (const float*)(work + p.dx_sums); a.part = all * z.pitch(); a.all_rows = all; a.count = p.parts; a.h = (int32_t)h;
    a.per_row = (int32_t)(z.pitch() / 8); a.pitch = (int32_t)z.pitch(); a.chunks = all * a.per_row; a.scale = scale_x; a.worker_rows = scale_rows; a.out = dx;
    const int64_t ctas = (a.chunks + 255) / 256;
    if (ctas > 0x7fffffff) return COMPAMS_ERR_TOO_LARGE;
    const bool vec = h % 8 == 0 && (reinterpret_cast<uintptr_t>(dx) & 15u) == 0;
    auto go = [&](auto t) {
        using T = decltype(t);
        const auto kernel = vec ? parts_kernel<T, true> : parts_kernel<T, false>;
        return launched(launch_sized(kernel, dim3((uint32_t)ctas), 256, 1, 0, false, stream, a), "head_parts");
    };
    return type == kTypeF32 ? go(float()) : type == kTypeBF16 ? go(__nv_bfloat16()) : go(__half());
}

}  // extern "C"
