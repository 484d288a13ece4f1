// Root-mean-square norms around a model's blocks, on [n, rows, h] activations:
//
//   norm:   y = x r w                                   r = 1 / sqrt(mean(x^2) + eps)
//   gated:  s = alpha residual + gate x r w             the norm behind a block, its gate, the residual's scale
//           y = s q v                                   q = 1 / sqrt(mean(s^2) + eps), the norm before the next block
//
//   backward:  b = dy v,   ds' = ds + q (b - s q^2 mean(b s)),   dv = sum_j dy s q
//              dresidual = alpha ds'
//              a = ds' gate w,   dx = r (a - x r^2 mean(a x)),   c = sum_j ds' x r,   dw = gate c,   dgate = w c
//
// Bound by memory. A row's threads keep it in registers (eight columns each, or sixteen), from the reading to the writing, and have the
// next row on its way meanwhile; they walk a chunk of a worker's rows and add up its part of the weights' gradients as they go, so that
// these cost no reading of their own. Rows above kLongest are read again instead, and their sums grow in the workspace.
//
// Precision. Everything is fp32 between the reading and the writing. s is kept in the residual's type and normalised as it is kept. In a
// 16-bit type a difference in the last bit of fp32 may put s on the other side of a border between two of its values: a row's squares are
// summed in binary64, and an s that is nearer to a border than the fp32 error is formed again in binary64; so s is the exact sum,
// rounded to fp32 and then to 16 bits, but for one in a million, and with it what the backward pass reads (with fp32 alone one s in 30000
// differs, and dv by 1.3e-5 of its length).
#include <algorithm>
#include <atomic>
#include <type_traits>

#include "context.h"
#include "rows.cuh"

namespace compams {
namespace {

constexpr float kInf = __builtin_inff();
constexpr int kMostThreads = 512;                      // of a row
constexpr int kForwardBytes = 96 * 1024, kBackwardBytes = 200 * 1024;  // of the rows that come ahead, for 512 threads
// Columns up to which a thread keeps eight of them, else sixteen. us forward and backward, eight / sixteen, of 33 million bfloat16 elements: aligned
// norm of 512 columns 28 43 / 26 37, of 1024 28 43 / 27 38, of 1536 36 47 / 30 55, of 2048 29 44 / 26 40; gated of 512 88 75 / 61 77, of 1024
// 91 77 / 70 79, of 1536 112 87 / 112 108, of 2048 100 80 / 72 84; beside an fp32 stream of 1024 87 143 / 92 149. Off 16-byte boundaries, where
// sixteen leave no registers for the next row: norm of 1001 64 138 / 92 149, of 2047 66 146 / 93 153, gated of 1001 185 312 / 199 641, of
// 1025 408 665 / 494 1226, of 2047 196 327 / 212 665.
constexpr int kNarrow = 1024;
constexpr int64_t kLongest = 16 * (int64_t)kMostThreads;  // columns that they keep

struct BlockArgs {
    const void *x, *residual, *dy, *ds, *s_in;
    void *y, *s, *dx, *dresidual;
    float2* stats;  // of a row: r, q; may be null going forward
    const float *weight, *gate, *next;  // may be null: ones
    int64_t weight_ws, gate_ws, next_ws;
    int64_t x_ws, x_rs, r_ws, r_rs, dy_ws, dy_rs, ds_ws, ds_rs;  // r: of the residual
    uint32_t rows, groups;  // of a worker; that walk them
    int32_t h;
    float alpha, eps;
    double alpha64;
    float* partial;  // [n][groups][2][h]: dv, c; may be null
};

// A thread's eight columns of a row, part k of several: neighbours on a 16-byte boundary (VEC), or every blockDim.x-th.
template <bool VEC> __device__ __forceinline__ int cell_column(int k, int e) {
    return VEC ? (k * (int)blockDim.x + (int)threadIdx.x) * 8 + e : (k * 8 + e) * (int)blockDim.x + (int)threadIdx.x;
}
// Rows come ahead. VEC: by asynchronous copies into places of a thread's own in shared memory, `depth` rows of them, of which it waits for
// the oldest; a row's cells stand there until its turn is over. Elsewhere the next row waits in registers.
template <typename T> constexpr int kChunks = (int)sizeof(T) / 2;  // of 16 bytes, for eight columns
__host__ __device__ constexpr int depth_of(int chunks, int bytes) {  // of rows whose threads hold so many chunks each
    const int d = bytes / (chunks * 16 * kMostThreads);
    return d < 1 ? 1 : d > 4 ? 4 : d;
}
// A tensor's cells of a row: `first` chunks stand in front of them in a thread's place.
template <typename T>
__device__ __forceinline__ void cell_fetch(uint4* place, int first, const T* row, int k, int h, bool there, int pitch) {
    const int at = cell_column<true>(k, 0);
    const bool in = there && at < h;
#pragma unroll
    for (int c = 0; c < kChunks<T>; ++c)
        copy16(place + (first + k * kChunks<T> + c) * pitch, in ? (const void*)(row + at + c * (8 / kChunks<T>)) : (const void*)row, in);
}
template <typename T>
__device__ __forceinline__ void cell_take(const uint4* place, int first, int k, int pitch, Pair (&v)[4]) {
    Raw8<T> raw;
    const uint4* at = place + (first + k * kChunks<T>) * pitch;
    if constexpr (std::is_same_v<T, float>) {
        raw.a = *reinterpret_cast<const float4*>(at);
        raw.b = *reinterpret_cast<const float4*>(at + pitch);
    } else {
        raw.q = *at;
    }
    raw_pairs<T>(raw, v);
}
template <typename T>
__device__ __forceinline__ void cell_load(const T* row, int k, int h, bool there, Pair (&v)[4]) {
#pragma unroll
    for (int p = 0; p < 4; ++p) {
        const int at = cell_column<false>(k, 2 * p), next = cell_column<false>(k, 2 * p + 1);
        v[p] = pair(there && at < h ? to_float(__ldg(row + at)) : 0.0f, there && next < h ? to_float(__ldg(row + next)) : 0.0f);
    }
}
// Rounds to T and stores; v becomes what was stored where KEEP.
template <typename T, bool VEC, bool KEEP = false>
__device__ __forceinline__ void cell_store(T* row, int k, int h, bool there, Pair (&v)[4]) {
    const Raw8<T> raw = pack_pairs<T>(v);
    if constexpr (VEC) {
        if (there && cell_column<VEC>(k, 0) < h) raw_store<T>(row + cell_column<VEC>(k, 0), raw);
    } else {
#pragma unroll
        for (int p = 0; p < 4; ++p) {
            float x[2];
            halves(v[p], x[0], x[1]);
#pragma unroll
            for (int e = 0; e < 2; ++e) {
                const int at = cell_column<VEC>(k, 2 * p + e);
                if (there && at < h) row[at] = from_float<T>(x[e]);
            }
        }
    }
    if (KEEP) raw_pairs<T>(raw, v);
}
template <bool VEC>
__device__ __forceinline__ void parameter_load(const float* p, int k, int h, Pair (&v)[4]) {
    auto one = [&](int at) { return at >= h ? 0.0f : p ? __ldg(p + at) : 1.0f; };
#pragma unroll
    for (int q = 0; q < 4; ++q) v[q] = pair(one(cell_column<VEC>(k, 2 * q)), one(cell_column<VEC>(k, 2 * q + 1)));
}
__device__ __forceinline__ Pair minus(Pair a, Pair b) { return fma(b, pair(-1.0f), a); }  // exact where a - b is
// 1 / sqrt(v), to the last bit or the one before: a step of Newton's behind the fast one.
__device__ __forceinline__ float root(float v) {
    const float r = rsqrtf(v), off = fmaf(-v * r, r, 1.0f);
    return v < kInf && v > 0.0f ? fmaf(0.5f * r, off, r) : r;
}

// The sum over a row's threads: 8, 16 or 32 lanes, or warps that meet at a barrier of their own. `turn` alternates between two places.
constexpr int kScratch = 4 * 2 * 16;  // rows of a CTA that need it (64 threads each at least), turns, warps
template <typename V>
__device__ __forceinline__ V row_sum(V v, V* scratch, int& turn) {
    const int threads = (int)blockDim.x;
#pragma unroll
    for (int o = 16; o; o >>= 1)
        if (o < threads) v += __shfl_xor_sync(0xffffffffu, v, o);
    if (threads <= 32) return v;
    V* place = scratch + (threadIdx.y * 2 + turn) * 16;
    turn ^= 1;
    if ((threadIdx.x & 31) == 0) place[threadIdx.x >> 5] = v;
    asm volatile("bar.sync %0, %1;" ::"r"((int)threadIdx.y + 1), "r"(threads) : "memory");
    V some[4];  // (places without a warp hold zeros)
#pragma unroll
    for (int k = 0; k < 4; ++k) some[k] = (place[4 * k] + place[4 * k + 1]) + (place[4 * k + 2] + place[4 * k + 3]);
    return (some[0] + some[1]) + (some[2] + some[3]);
}
template <typename V>
__device__ __forceinline__ void clear_scratch(V* scratch) {
    for (int k = threadIdx.y * blockDim.x + threadIdx.x; k < kScratch; k += blockDim.x * blockDim.y) scratch[k] = V(0);
}

// Whether the fp32 sum s of p and q, which is s + off in the 16-bit type, is so near to a border between two of its values that its error,
// 6.5 2^-24 of |p| + |q| at most (5.5 of q: the root 2.5, three products; 2 of p: alpha and a product; the sum), may have carried it over:
// off is then half a step.
template <typename T>
__device__ __forceinline__ bool near_border(float s, float off, float p, float q) {
    constexpr bool kHalfType = std::is_same_v<T, __half>;
    float half_step = __uint_as_float(__float_as_uint(s) & 0x7f800000u) * (kHalfType ? 0x1p-11f : 0x1p-8f);
    if (kHalfType) half_step = fmaxf(half_step, 0x1p-25f);
    // (less, not also equal: 0 + 0 is no sum to form again, of a row of zeros and of the threads behind a row's end)
    return fabsf(fabsf(off) - half_step) < 0x1.ap-22f * (fabsf(p) + fabsf(q));
}

// 1 / sqrt(v) in binary64 from its fp32 approximation, by a step of Newton's: off by about 2^-46. (Of an infinity it is 0 and of 0 infinite, as in
// fp32: the step would make either NaN.)
__device__ __forceinline__ double root64(double v, float r) {
    return r > 0.0f && r < kInf ? (double)r * (1.5 - 0.5 * v * ((double)r * (double)r)) : (double)r;
}
// The sum of eight squares of 16-bit numbers, which are exact in fp32, in binary64. (Pairs of bf16's in fp32, which halves the conversions,
// are off by 2^-33 of the sum: enough for three of 4 million s.)
__device__ __forceinline__ double squares8(const Pair (&v)[4]) {
    double s[4];
#pragma unroll
    for (int k = 0; k < 4; ++k) {
        float a, b;
        halves(mul(v[k], v[k]), a, b);
        s[k] = (double)a + (double)b;
    }
    return (s[0] + s[1]) + (s[2] + s[3]);
}

// 16384 bfloat16 rows: norm of 2048 columns 23.5 us (5.7 TB/s) with registers for 1024 threads to an SM, 28 with them for 768; gated of 4096
// 144 us (3.7 TB/s) with registers for 512, 219 and spills for 768: the two sums, one in binary64, and what a row's rounding takes are 300
// instructions a thread, and 16 warps do not cover the barriers between them.
template <typename T, typename R, bool GATED, bool VEC, int K>
__global__ void __launch_bounds__(K == 1 ? 256 : kMostThreads, GATED ? (K == 1 ? 2 : 1) : (K == 1 ? 4 : 2)) block_forward_kernel(const __grid_constant__ BlockArgs a) {
    constexpr bool kWide = GATED && !std::is_same_v<R, float>;  // s is rounded to 16 bits
    using Sum = std::conditional_t<kWide, double, float>;
    __shared__ __align__(16) Sum scratch[kScratch];
    __shared__ __align__(16) float scratch2[kScratch];
    const uint32_t worker = blockIdx.y, group = blockIdx.x * blockDim.y + threadIdx.y, rounds = (a.rows + a.groups - 1) / a.groups;
    const T* x = (const T*)a.x + (int64_t)worker * a.x_ws;
    const R* residual = GATED ? (const R*)a.residual + (int64_t)worker * a.r_ws : nullptr;
    const float *weight = a.weight ? a.weight + worker * a.weight_ws : nullptr, *gate = a.gate ? a.gate + worker * a.gate_ws : nullptr;
    const float* next = a.next ? a.next + worker * a.next_ws : nullptr;
    constexpr int kRowChunks = K * (kChunks<T> + (GATED ? kChunks<R> : 0)), kDepth = depth_of(kRowChunks, kForwardBytes);
    extern __shared__ __align__(16) uint4 ring[];
    const int pitch = (int)(blockDim.x * blockDim.y), tid = (int)(threadIdx.y * blockDim.x + threadIdx.x);
    // a thread's weights and gates, for what is formed in binary64
    float2* parameters = reinterpret_cast<float2*>(ring + (VEC ? kDepth * kRowChunks * pitch : 0)) + tid;
    Pair w[K][4], v[K][4];  // weight * gate, next
#pragma unroll
    for (int k = 0; k < K; ++k) {
        parameter_load<VEC>(weight, k, a.h, w[k]);
        if (GATED) {
            Pair g[4];
            parameter_load<VEC>(gate, k, a.h, g);
#pragma unroll
            for (int p = 0; p < 4; ++p) {
                if (kWide) {
                    float x0, x1, g0, g1;
                    halves(w[k][p], x0, x1);
                    halves(g[p], g0, g1);
                    parameters[(k * 8 + 2 * p) * pitch] = make_float2(x0, g0);
                    parameters[(k * 8 + 2 * p + 1) * pitch] = make_float2(x1, g1);
                }
                w[k][p] = mul(w[k][p], g[p]);
            }
            parameter_load<VEC>(next, k, a.h, v[k]);
        }
    }
    const float inverse = 1.0f / (float)a.h;
    const double inverse64 = 1.0 / (double)a.h;
    const Pair alpha = pair(a.alpha);
    int turn = 0, turn2 = 0;
    clear_scratch(scratch);
    clear_scratch(scratch2);
    __syncthreads();
    Pair nx[K][4], nr[K][4];  // the next row, where it waits in registers
    auto fetch = [&](uint32_t round) {
        const uint32_t j = group + round * a.groups;
        const bool there = round < rounds && j < a.rows;
        const T* from = x + (there ? (int64_t)j * a.x_rs : 0);
        const R* also = GATED ? residual + (there ? (int64_t)j * a.r_rs : 0) : nullptr;
        uint4* place = ring + (round % kDepth) * kRowChunks * pitch + tid;
#pragma unroll
        for (int k = 0; k < K; ++k) {
            if constexpr (VEC) {
                cell_fetch<T>(place, 0, from, k, a.h, there, pitch);
                if (GATED) cell_fetch<R>(place, K * kChunks<T>, also, k, a.h, there, pitch);
            } else {
                cell_load<T>(from, k, a.h, there, nx[k]);
                if (GATED) cell_load<R>(also, k, a.h, there, nr[k]);
            }
        }
        if (VEC) copies_commit();
    };
    for (uint32_t round = 0; round < (VEC ? kDepth - 1 : 1); ++round) fetch(round);
    for (uint32_t round = 0, j = group; round < rounds; ++round, j += a.groups) {
        const bool there = j < a.rows;
        Pair xs[K][4], rs[K][4];
        const uint4* place = ring + (round % kDepth) * kRowChunks * pitch + tid;
        if (VEC) {
            fetch(round + kDepth - 1);
            copies_wait<kDepth - 1>();
#pragma unroll
            for (int k = 0; k < K; ++k) cell_take<T>(place, 0, k, pitch, xs[k]);
        } else {
#pragma unroll
            for (int k = 0; k < K; ++k)
#pragma unroll
                for (int p = 0; p < 4; ++p) {
                    xs[k][p] = nx[k][p];
                    if (GATED) rs[k][p] = nr[k][p];
                }
            fetch(round + 1);
        }
        Sum sum = 0;
        if constexpr (kWide) {
#pragma unroll
            for (int k = 0; k < K; ++k) sum += squares8(xs[k]);
        } else {
            Pair some = pair(0.0f);
#pragma unroll
            for (int k = 0; k < K; ++k)
#pragma unroll
                for (int p = 0; p < 4; ++p) some = fma(xs[k][p], xs[k][p], some);
            sum = joint(some);
        }
        const Sum all = row_sum<Sum>(sum, scratch, turn);
        double exact = 0.0;
        float r;
        if constexpr (kWide) {
            exact = all * inverse64 + (double)a.eps;
            r = root((float)exact);
        } else {
            r = root(all * inverse + a.eps);
        }
        const int64_t number = (int64_t)worker * a.rows + j;
        T* y = (T*)a.y + number * a.h;
        if constexpr (!GATED) {
#pragma unroll
            for (int k = 0; k < K; ++k) {
#pragma unroll
                for (int p = 0; p < 4; ++p) xs[k][p] = mul(mul(xs[k][p], pair(r)), w[k][p]);
                cell_store<T, VEC>(y, k, a.h, there, xs[k]);
            }
            if (a.stats && there && threadIdx.x == 0) a.stats[number] = make_float2(r, 0.0f);
        } else {
            R* s = (R*)a.s + number * a.h;
            Pair squares = pair(0.0f);
#pragma unroll
            for (int k = 0; k < K; ++k) {
                if (VEC) cell_take<R>(place, K * kChunks<T>, k, pitch, rs[k]);
                Pair one[4], other[4], t[4];
#pragma unroll
                for (int p = 0; p < 4; ++p) {
                    one[p] = mul(alpha, rs[k][p]);
                    other[p] = mul(mul(xs[k][p], pair(r)), w[k][p]);
                    t[p] = add(one[p], other[p]);
                }
                if constexpr (kWide) {
                    Pair off[4];
                    raw_pairs<R>(pack_pairs<R>(t), off);
                    float sv[8], ov[8], pv[8], qv[8];
                    bool any = false;
#pragma unroll
                    for (int p = 0; p < 4; ++p) {
                        halves(t[p], sv[2 * p], sv[2 * p + 1]);
                        halves(minus(off[p], t[p]), ov[2 * p], ov[2 * p + 1]);
                        halves(one[p], pv[2 * p], pv[2 * p + 1]);
                        halves(other[p], qv[2 * p], qv[2 * p + 1]);
                    }
#pragma unroll
                    for (int e = 0; e < 8; ++e) any = any || near_border<R>(sv[e], ov[e], pv[e], qv[e]);
                    if (any) {  // one thread in a hundred, where neither x nor the residual is 0
                        uint32_t which = 0;
#pragma unroll
                        for (int e = 0; e < 8; ++e) which |= near_border<R>(sv[e], ov[e], pv[e], qv[e]) ? 1u << e : 0u;
                        const double r64 = root64(exact, r);
                        while (which) {
                            const int e = __ffs(which) - 1;
                            which &= which - 1;
                            const float2 factors = parameters[(k * 8 + e) * pitch];
                            double xv, rv;
                            if (VEC) {
                                xv = to_float(reinterpret_cast<const T*>(place + k * pitch)[e]);
                                rv = to_float(reinterpret_cast<const R*>(place + (K + k) * pitch)[e]);
                            } else {
                                const int at = cell_column<VEC>(k, e);
                                xv = there && at < a.h ? to_float(x[(int64_t)j * a.x_rs + at]) : 0.0f;
                                rv = there && at < a.h ? to_float(residual[(int64_t)j * a.r_rs + at]) : 0.0f;
                            }
                            const float exactly = (float)(a.alpha64 * rv + xv * r64 * ((double)factors.x * (double)factors.y));
#pragma unroll
                            for (int c = 0; c < 8; ++c) sv[c] = c == e ? exactly : sv[c];
                        }
#pragma unroll
                        for (int p = 0; p < 4; ++p) t[p] = pair(sv[2 * p], sv[2 * p + 1]);
                    }
                }
                cell_store<R, VEC, true>(s, k, a.h, there, t);
#pragma unroll
                for (int p = 0; p < 4; ++p) {
                    rs[k][p] = t[p];
                    squares = fma(t[p], t[p], squares);
                }
            }
            const float q = root(row_sum<float>(joint(squares), scratch2, turn2) * inverse + a.eps);
#pragma unroll
            for (int k = 0; k < K; ++k) {
#pragma unroll
                for (int p = 0; p < 4; ++p) rs[k][p] = mul(mul(rs[k][p], pair(q)), v[k][p]);
                cell_store<T, VEC>(y, k, a.h, there, rs[k]);
            }
            if (a.stats && there && threadIdx.x == 0) a.stats[number] = make_float2(r, q);
        }
    }
}

// The same rows: norm of 2048 columns 40 us (5.0 TB/s), gated of 4096 158 us (5.1 TB/s); more threads to an SM spill (47, 247).
template <typename T, typename R, bool GATED, bool VEC, int K>
__global__ void __launch_bounds__(K == 1 ? 256 : kMostThreads, K == 1 ? 2 : 1) block_backward_kernel(const __grid_constant__ BlockArgs a) {
    __shared__ __align__(16) float scratch[kScratch];
    clear_scratch(scratch);
    __syncthreads();
    const uint32_t worker = blockIdx.y, group = blockIdx.x * blockDim.y + threadIdx.y, rounds = (a.rows + a.groups - 1) / a.groups;
    const T* x = (const T*)a.x + (int64_t)worker * a.x_ws;
    const T* dy = (const T*)a.dy + (int64_t)worker * a.dy_ws;
    const R* ds = GATED && a.ds ? (const R*)a.ds + (int64_t)worker * a.ds_ws : nullptr;
    const R* s = GATED ? (const R*)a.s_in + (int64_t)worker * a.rows * a.h : nullptr;
    const float *weight = a.weight ? a.weight + worker * a.weight_ws : nullptr, *gate = a.gate ? a.gate + worker * a.gate_ws : nullptr;
    const float* next = a.next ? a.next + worker * a.next_ws : nullptr;
    Pair w[K][4], v[K][4], sums[2][K][4];  // weight * gate, next; dv, c
#pragma unroll
    for (int k = 0; k < K; ++k) {
        parameter_load<VEC>(weight, k, a.h, w[k]);
        if (GATED) {
            Pair g[4];
            parameter_load<VEC>(gate, k, a.h, g);
#pragma unroll
            for (int p = 0; p < 4; ++p) w[k][p] = mul(w[k][p], g[p]);
            parameter_load<VEC>(next, k, a.h, v[k]);
        }
#pragma unroll
        for (int p = 0; p < 4; ++p) sums[0][k][p] = sums[1][k][p] = pair(0.0f);
    }
    const float inverse = 1.0f / (float)a.h;
    int turn = 0;
    // chunks of a row: dy, x, then s and ds
    constexpr int kY = 0, kX = K * kChunks<T>, kS = 2 * kX, kD = kS + K * kChunks<R>;
    constexpr int kRowChunks = GATED ? kD + K * kChunks<R> : kS, kDepth = depth_of(kRowChunks, kBackwardBytes);
    extern __shared__ __align__(16) uint4 ring[];
    const int pitch = (int)(blockDim.x * blockDim.y), tid = (int)(threadIdx.y * blockDim.x + threadIdx.x);
    Pair nx[K][4], ny[K][4], ns[K][4], nd[K][4];  // the next row, where it waits in registers
    float2 next_stats = {};
    auto stats_of = [&](uint32_t j) { return j < a.rows ? __ldg(a.stats + (int64_t)worker * a.rows + j) : make_float2(0.0f, 0.0f); };
    auto fetch = [&](uint32_t round) {
        const uint32_t j = group + round * a.groups;
        const bool there = round < rounds && j < a.rows;
        const int64_t at = there ? j : 0;
        uint4* place = ring + (round % kDepth) * kRowChunks * pitch + tid;
#pragma unroll
        for (int k = 0; k < K; ++k) {
            if constexpr (VEC) {
                cell_fetch<T>(place, kY, dy + at * a.dy_rs, k, a.h, there, pitch);
                cell_fetch<T>(place, kX, x + at * a.x_rs, k, a.h, there, pitch);
                if (GATED) {
                    cell_fetch<R>(place, kS, s + at * a.h, k, a.h, there, pitch);
                    cell_fetch<R>(place, kD, ds ? ds + at * a.ds_rs : s, k, a.h, there && ds, pitch);
                }
            } else {
                cell_load<T>(dy + at * a.dy_rs, k, a.h, there, ny[k]);
                cell_load<T>(x + at * a.x_rs, k, a.h, there, nx[k]);
                if (GATED) {
                    cell_load<R>(s + at * a.h, k, a.h, there, ns[k]);
                    cell_load<R>(ds ? ds + at * a.ds_rs : s, k, a.h, there && ds, nd[k]);
                }
            }
        }
        if (VEC) copies_commit();
    };
    for (uint32_t round = 0; round < (VEC ? kDepth - 1 : 1); ++round) fetch(round);
    next_stats = stats_of(group);
    for (uint32_t round = 0, j = group; round < rounds; ++round, j += a.groups) {
        const bool there = j < a.rows;
        const float r = next_stats.x, q = next_stats.y;
        next_stats = stats_of(j + a.groups);
        Pair xs[K][4], g[K][4], ss[K][4], dd[K][4];  // x; the gradient of what the norm behind x gives; s; ds
        const uint4* place = ring + (round % kDepth) * kRowChunks * pitch + tid;
        if (VEC) {
            fetch(round + kDepth - 1);
            copies_wait<kDepth - 1>();
#pragma unroll
            for (int k = 0; k < K; ++k) {
                cell_take<T>(place, kY, k, pitch, g[k]);
                if (GATED) cell_take<R>(place, kS, k, pitch, ss[k]);
                else cell_take<T>(place, kX, k, pitch, xs[k]);
            }
        } else {
#pragma unroll
            for (int k = 0; k < K; ++k)
#pragma unroll
                for (int p = 0; p < 4; ++p) {
                    xs[k][p] = nx[k][p], g[k][p] = ny[k][p];
                    if (GATED) ss[k][p] = ns[k][p], dd[k][p] = nd[k][p];
                }
            fetch(round + 1);
        }
        const int64_t number = (int64_t)worker * a.rows + j;
        if constexpr (GATED) {
            Pair dot = pair(0.0f);
#pragma unroll
            for (int k = 0; k < K; ++k)
#pragma unroll
                for (int p = 0; p < 4; ++p) {
                    ss[k][p] = mul(ss[k][p], pair(q));
                    sums[0][k][p] = fma(g[k][p], ss[k][p], sums[0][k][p]);
                    g[k][p] = mul(g[k][p], v[k][p]);
                    dot = fma(g[k][p], ss[k][p], dot);
                }
            const float mean = row_sum<float>(joint(dot), scratch, turn) * inverse;
#pragma unroll
            for (int k = 0; k < K; ++k) {
                if (VEC) {
                    cell_take<R>(place, kD, k, pitch, dd[k]);
                    cell_take<T>(place, kX, k, pitch, xs[k]);
                }
#pragma unroll
                for (int p = 0; p < 4; ++p) {
                    g[k][p] = fma(pair(q), fma(pair(-mean), ss[k][p], g[k][p]), dd[k][p]);
                    dd[k][p] = mul(pair(a.alpha), g[k][p]);
                }
                if (a.dresidual) cell_store<R, VEC>((R*)a.dresidual + number * a.h, k, a.h, there, dd[k]);
            }
        }
        Pair dot = pair(0.0f);
#pragma unroll
        for (int k = 0; k < K; ++k)
#pragma unroll
            for (int p = 0; p < 4; ++p) {
                xs[k][p] = mul(xs[k][p], pair(r));
                sums[1][k][p] = fma(g[k][p], xs[k][p], sums[1][k][p]);
                g[k][p] = mul(g[k][p], w[k][p]);
                dot = fma(g[k][p], xs[k][p], dot);
            }
        if (a.dx) {
            const float mean = row_sum<float>(joint(dot), scratch, turn) * inverse;
#pragma unroll
            for (int k = 0; k < K; ++k) {
#pragma unroll
                for (int p = 0; p < 4; ++p) g[k][p] = mul(pair(r), fma(pair(-mean), xs[k][p], g[k][p]));
                cell_store<T, VEC>((T*)a.dx + number * a.h, k, a.h, there, g[k]);
            }
        }
    }
    if (!a.partial) return;
    float* out = a.partial + ((int64_t)worker * a.groups + group) * 2 * a.h;
#pragma unroll
    for (int k = 0; k < K; ++k)
#pragma unroll
        for (int p = 0; p < 4; ++p) {
            float dv[2], c[2];
            halves(sums[0][k][p], dv[0], dv[1]);
            halves(sums[1][k][p], c[0], c[1]);
#pragma unroll
            for (int e = 0; e < 2; ++e) {
                const int at = cell_column<VEC>(k, 2 * p + e);
                if (at < a.h) {
                    if (GATED) out[at] = dv[e];
                    out[a.h + at] = c[e];
                }
            }
        }
}

// Rows that registers do not hold: a CTA of 512 threads walks its rows' columns again for every sum, one element an access, and nothing comes
// ahead. bfloat16, 16384 rows of 12288 columns: norm 331 us forward (2.4 TB/s) and 2068 backward (0.6), where the weights' sums also grow in memory
// row by row; 8192 rows gated 922 and 2356.
template <typename T, typename R, bool GATED>
__global__ void __launch_bounds__(kMostThreads) long_forward_kernel(const __grid_constant__ BlockArgs a) {
    constexpr bool kWide = GATED && !std::is_same_v<R, float>;
    __shared__ __align__(16) double scratch[kScratch];
    __shared__ __align__(16) float scratch2[kScratch];
    clear_scratch(scratch);
    clear_scratch(scratch2);
    __syncthreads();
    const uint32_t worker = blockIdx.y;
    const float *weight = a.weight ? a.weight + worker * a.weight_ws : nullptr, *gate = a.gate ? a.gate + worker * a.gate_ws : nullptr;
    const float* next = a.next ? a.next + worker * a.next_ws : nullptr;
    const float inverse = 1.0f / (float)a.h;
    int turn = 0, turn2 = 0;
    for (uint32_t j = blockIdx.x; j < a.rows; j += a.groups) {
        const T* x = (const T*)a.x + (int64_t)worker * a.x_ws + (int64_t)j * a.x_rs;
        const R* residual = GATED ? (const R*)a.residual + (int64_t)worker * a.r_ws + (int64_t)j * a.r_rs : nullptr;
        const int64_t number = (int64_t)worker * a.rows + j;
        T* y = (T*)a.y + number * a.h;
        R* s = GATED ? (R*)a.s + number * a.h : nullptr;
        double sum = 0.0;
        for (int c0 = threadIdx.x; c0 < a.h; c0 += 8 * kMostThreads) {
            Pair v[4];
            auto one = [&](int c) { return c < a.h ? to_float(__ldg(x + c)) : 0.0f; };
#pragma unroll
            for (int p = 0; p < 4; ++p) v[p] = pair(one(c0 + 2 * p * kMostThreads), one(c0 + (2 * p + 1) * kMostThreads));
            sum += squares8(v);
        }
        const double exact = row_sum<double>(sum, scratch, turn) / a.h + (double)a.eps;
        const float r = root((float)exact);
        float squares = 0.0f, q = 0.0f;
        for (int c = threadIdx.x; c < a.h; c += kMostThreads) {
            const float w = weight ? __ldg(weight + c) : 1.0f, v = to_float(__ldg(x + c));
            if constexpr (!GATED) {
                y[c] = from_float<T>(v * r * w);
            } else {
                const float p = a.alpha * to_float(__ldg(residual + c)), u = v * r * (w * (gate ? __ldg(gate + c) : 1.0f));
                float t = p + u;
                if constexpr (kWide)
                    if (near_border<R>(t, to_float(from_float<R>(t)) - t, p, u))
                        t = (float)(a.alpha64 * (double)to_float(__ldg(residual + c)) + (double)v * root64(exact, r) * ((double)w * (gate ? (double)gate[c] : 1.0)));
                s[c] = from_float<R>(t);
                t = to_float(from_float<R>(t));
                squares = fmaf(t, t, squares);
            }
        }
        if constexpr (GATED) {
            q = root(row_sum<float>(squares, scratch2, turn2) * inverse + a.eps);
            for (int c = threadIdx.x; c < a.h; c += kMostThreads)  // (its own: a thread reads what it wrote)
                y[c] = from_float<T>(to_float(s[c]) * q * (next ? __ldg(next + c) : 1.0f));
        }
        if (a.stats && threadIdx.x == 0) a.stats[number] = make_float2(r, q);
    }
}
template <typename T, typename R, bool GATED>
__global__ void __launch_bounds__(kMostThreads) long_backward_kernel(const __grid_constant__ BlockArgs a) {
    __shared__ __align__(16) float scratch[kScratch];
    clear_scratch(scratch);
    __syncthreads();
    const uint32_t worker = blockIdx.y;
    const float *weight = a.weight ? a.weight + worker * a.weight_ws : nullptr, *gate = a.gate ? a.gate + worker * a.gate_ws : nullptr;
    const float* next = a.next ? a.next + worker * a.next_ws : nullptr;
    const float inverse = 1.0f / (float)a.h;
    float* out = a.partial ? a.partial + ((int64_t)worker * a.groups + blockIdx.x) * 2 * a.h : nullptr;
    int turn = 0;
    for (uint32_t j = blockIdx.x; j < a.rows; j += a.groups) {
        const T* x = (const T*)a.x + (int64_t)worker * a.x_ws + (int64_t)j * a.x_rs;
        const T* dy = (const T*)a.dy + (int64_t)worker * a.dy_ws + (int64_t)j * a.dy_rs;
        const R* ds = GATED && a.ds ? (const R*)a.ds + (int64_t)worker * a.ds_ws + (int64_t)j * a.ds_rs : nullptr;
        const int64_t number = (int64_t)worker * a.rows + j;
        const R* s = GATED ? (const R*)a.s_in + number * a.h : nullptr;
        const float2 stats = __ldg(a.stats + number);
        const float r = stats.x, q = stats.y;
        const bool first = j == blockIdx.x;
        float mean = 0.0f;
        if constexpr (GATED) {
            float dot = 0.0f;
            for (int c = threadIdx.x; c < a.h; c += kMostThreads) {
                const float g = to_float(__ldg(dy + c)), shat = to_float(__ldg(s + c)) * q;
                dot = fmaf(g * (next ? __ldg(next + c) : 1.0f), shat, dot);
                if (out) out[c] = fmaf(g, shat, first ? 0.0f : out[c]);
            }
            mean = row_sum<float>(dot, scratch, turn) * inverse;
        }
        auto gradient = [&](int c) {  // of what the norm behind x gives, gate included
            const float g = to_float(__ldg(dy + c));
            if constexpr (!GATED) return g;
            else return fmaf(q, fmaf(-mean, to_float(__ldg(s + c)) * q, g * (next ? __ldg(next + c) : 1.0f)), ds ? to_float(__ldg(ds + c)) : 0.0f);
        };
        auto factor = [&](int c) { return (weight ? __ldg(weight + c) : 1.0f) * (GATED && gate ? __ldg(gate + c) : 1.0f); };
        float dot = 0.0f;
        for (int c = threadIdx.x; c < a.h; c += kMostThreads) {
            const float g = gradient(c), xhat = to_float(__ldg(x + c)) * r;
            if (GATED && a.dresidual) ((R*)a.dresidual)[number * a.h + c] = from_float<R>(a.alpha * g);
            if (out) out[a.h + c] = fmaf(g, xhat, first ? 0.0f : out[a.h + c]);
            dot = fmaf(g * factor(c), xhat, dot);
        }
        if (a.dx) {
            const float mean2 = row_sum<float>(dot, scratch, turn) * inverse;
            for (int c = threadIdx.x; c < a.h; c += kMostThreads)
                ((T*)a.dx)[number * a.h + c] = from_float<T>(r * fmaf(-mean2, to_float(__ldg(x + c)) * r, gradient(c) * factor(c)));
        }
    }
}

struct SumsArgs {
    const float* partial;
    const float *weight, *gate;
    int64_t weight_ws, gate_ws;
    float *dweight, *dgate, *dnext;
    int32_t h, n, gated;
    uint32_t groups;
    int32_t together;
};
// The groups' sums, eight shares of them for 32 columns, and the weights' gradients from them. together: over all workers.
__global__ void __launch_bounds__(256) block_sums_kernel(const __grid_constant__ SumsArgs a) {
    __shared__ float shares[2][8][33];
    dependency_wait();
    const int c = blockIdx.x * 32 + threadIdx.x;
    float dv = 0.0f, dw = 0.0f, dg = 0.0f;
    for (int i = a.together ? 0 : blockIdx.y; i < (a.together ? a.n : (int)blockIdx.y + 1); ++i) {
        const float* from = a.partial + (int64_t)i * a.groups * 2 * a.h + c;
        float v = 0.0f, q = 0.0f;
        if (c < a.h)
#pragma unroll 4
            for (uint32_t g = threadIdx.y; g < a.groups; g += 8) {
                if (a.gated) v += from[(int64_t)g * 2 * a.h];
                q += from[(int64_t)g * 2 * a.h + a.h];
            }
        __syncthreads();
        shares[0][threadIdx.y][threadIdx.x] = v;
        shares[1][threadIdx.y][threadIdx.x] = q;
        __syncthreads();
        if (threadIdx.y == 0 && c < a.h) {
            v = q = 0.0f;
#pragma unroll
            for (int k = 0; k < 8; ++k) {
                v += shares[0][k][threadIdx.x];
                q += shares[1][k][threadIdx.x];
            }
            dv += v;
            dw += (a.gate ? a.gate[i * a.gate_ws + c] : 1.0f) * q;
            dg += (a.weight ? a.weight[i * a.weight_ws + c] : 1.0f) * q;
        }
    }
    if (threadIdx.y || c >= a.h) return;
    const int64_t at = (int64_t)blockIdx.y * a.h + c;
    if (a.dnext) a.dnext[at] = dv;
    if (a.dweight) a.dweight[at] = dw;
    if (a.dgate) a.dgate[at] = dg;
}

// ---- host ------------------------------------------------------------------------------------------------------------------

struct BlockShape {
    int32_t n;
    int64_t rows, h;
    bool ok() const {
        return n >= 1 && n <= 65535 && rows >= 0 && h >= 1 && h < ((int64_t)1 << 31) - 16 * kSpan && rows <= (int64_t)0x7fffffff / n;
    }
    // Threads of a row: eight columns each, then sixteen; at least 8. Rows of a CTA: 256 threads, or one row.
    int parts() const { return h <= kNarrow ? 1 : 2; }
    int threads() const {
        if (h > kLongest) return kMostThreads;
        const int64_t cells = (h + 8 * parts() - 1) / (8 * parts());
        return cells <= 8 ? 8 : cells <= 16 ? 16 : (int)((cells + 31) / 32 * 32);
    }
    int rows_of_cta() const { return threads() >= 256 ? 1 : 256 / threads(); }
    // Groups of threads that walk a worker's rows: what the SMs hold at once with so many threads, of four rows at least.
    uint32_t groups(int resident = 512) const {
        const int64_t all = (int64_t)multiprocessors() * std::max(1, resident / threads());
        const int64_t most = (rows + 3) / 4, per = rows_of_cta();
        int64_t g = (all + n - 1) / n;
        g = std::min(std::max<int64_t>(1, g), std::max<int64_t>(1, most));
        return (uint32_t)((g + per - 1) / per * per);
    }
};

template <typename F>
int by_block_types(int32_t x, int32_t r, F f) {
    if (x == kTypeF32) return f(float(), float());
    if (x == kTypeBF16) return r == kTypeF32 ? f(__nv_bfloat16(), float()) : f(__nv_bfloat16(), __nv_bfloat16());
    return r == kTypeF32 ? f(__half(), float()) : f(__half(), __half());
}
int launched(cudaError_t e, const char* what) { return e == cudaSuccess ? COMPAMS_OK : cuda_fail(e, what); }
bool float_aligned(const void* p) { return (reinterpret_cast<uintptr_t>(p) & 3u) == 0; }
bool vector_parameter(const float* p, int64_t ws) { return !p || (((reinterpret_cast<uintptr_t>(p) | (uint64_t)(ws * 4)) & 15u) == 0); }

// Shared memory for rows of so many 16-byte chunks a thread.
int ring_bytes(const BlockShape& z, bool vec, int chunks, int bytes) {
    return vec ? depth_of(chunks, bytes) * chunks * 16 * z.threads() * z.rows_of_cta() : 0;
}
template <auto kernel>
cudaError_t allow(int bytes) {  // more than 48 KB, the static part included: asked once for every device
    static std::atomic<uint64_t> known{0};
    int device = 0;
    cudaError_t e = cudaGetDevice(&device);
    if (e != cudaSuccess || bytes <= 40 * 1024 || (device < 64 && known.load(std::memory_order_relaxed) >> device & 1u)) return e;
    e = cudaFuncSetAttribute(kernel, cudaFuncAttributeMaxDynamicSharedMemorySize, 220 * 1024);
    if (e == cudaSuccess && device < 64) known.fetch_or((uint64_t)1 << device, std::memory_order_relaxed);
    return e;
}
template <typename T, typename R, bool GATED, bool VEC, int K>
int block_forward(BlockArgs& a, const BlockShape& z, cudaStream_t stream) {
    constexpr auto kernel = block_forward_kernel<T, R, GATED, VEC, K>;
    const int bytes = ring_bytes(z, VEC, K * (kChunks<T> + (GATED ? kChunks<R> : 0)), kForwardBytes) +
                      (GATED && !std::is_same_v<R, float> ? K * 64 * z.threads() * z.rows_of_cta() : 0);
    cudaError_t e = allow<kernel>(bytes);
    if (e == cudaSuccess)
        e = launch_plain(kernel, dim3(a.groups / z.rows_of_cta(), (uint32_t)z.n), dim3((uint32_t)z.threads(), (uint32_t)z.rows_of_cta()), bytes, stream, a);
    return launched(e, "block_forward");
}
template <typename T, typename R, bool GATED, bool VEC, int K>
int block_backward(BlockArgs& a, const BlockShape& z, cudaStream_t stream) {
    constexpr auto kernel = block_backward_kernel<T, R, GATED, VEC, K>;
    const int bytes = ring_bytes(z, VEC, 2 * K * (kChunks<T> + (GATED ? kChunks<R> : 0)), kBackwardBytes);
    cudaError_t e = allow<kernel>(bytes);
    if (e == cudaSuccess)
        e = launch_plain(kernel, dim3(a.groups / z.rows_of_cta(), (uint32_t)z.n), dim3((uint32_t)z.threads(), (uint32_t)z.rows_of_cta()), bytes, stream, a);
    return launched(e, "block_backward");
}
template <typename T, typename R, bool GATED>
int block_forward(BlockArgs& a, const BlockShape& z, bool vec, cudaStream_t stream) {
    if (z.h > kLongest)
        return launched(launch_plain(long_forward_kernel<T, R, GATED>, dim3(a.groups, (uint32_t)z.n), dim3(kMostThreads), 0, stream, a), "block_forward");
    if (z.parts() == 1) return vec ? block_forward<T, R, GATED, true, 1>(a, z, stream) : block_forward<T, R, GATED, false, 1>(a, z, stream);
    return vec ? block_forward<T, R, GATED, true, 2>(a, z, stream) : block_forward<T, R, GATED, false, 2>(a, z, stream);
}
template <typename T, typename R, bool GATED>
int block_backward(BlockArgs& a, const BlockShape& z, bool vec, cudaStream_t stream) {
    if (z.h > kLongest)
        return launched(launch_plain(long_backward_kernel<T, R, GATED>, dim3(a.groups, (uint32_t)z.n), dim3(kMostThreads), 0, stream, a), "block_backward");
    if (z.parts() == 1) return vec ? block_backward<T, R, GATED, true, 1>(a, z, stream) : block_backward<T, R, GATED, false, 1>(a, z, stream);
    return vec ? block_backward<T, R, GATED, true, 2>(a, z, stream) : block_backward<T, R, GATED, false, 2>(a, z, stream);
}

}  // namespace
}  // namespace compams

using namespace compams;

extern "C" {

int compams_rms_norm_forward(void* y, void* s, float* stats, const void* x, const void* residual, int32_t type, int32_t residual_type,
                             int32_t n, int64_t rows, int64_t h, int64_t x_worker_stride, int64_t x_row_stride, int64_t residual_worker_stride,
                             int64_t residual_row_stride, const float* weight, int64_t weight_stride, const float* gate, int64_t gate_stride,
                             const float* next, int64_t next_stride, double residual_scale, float eps, void* cuda_stream) {
    const BlockShape z{n, rows, h};
    const bool gated = residual != nullptr;
    if (!z.ok() || !type_known(type) || !(eps >= 0.0f) || (gated ? residual_type != type && residual_type != kTypeF32 : s || gate || next))
        return COMPAMS_ERR_INVALID_ARG;
    if (rows == 0) return COMPAMS_OK;
    const Rows in{x, x_worker_stride, x_row_stride, type}, out = packed(y, rows, h, type);
    const Rows res{residual, residual_worker_stride, residual_row_stride, residual_type}, sum = packed(s, rows, h, residual_type);
    if (!in.strides_ok() || (gated && !res.strides_ok()) || weight_stride < 0 || gate_stride < 0 || next_stride < 0 || !x || !y || (gated && !s) ||
        !in.element_aligned() || !out.element_aligned() || !float_aligned(weight) || !float_aligned(gate) || !float_aligned(next) ||
        (reinterpret_cast<uintptr_t>(stats) & 7u) || (gated && (!res.element_aligned() || !sum.element_aligned())))
        return COMPAMS_ERR_INVALID_ARG;
    const bool vec = h % 8 == 0 && in.aligned() && out.aligned() && (!gated || (res.aligned() && sum.aligned())) &&
                     vector_parameter(weight, weight_stride) && vector_parameter(gate, gate_stride) && vector_parameter(next, next_stride);
    BlockArgs a = {};
    a.x = x; a.residual = residual; a.y = y; a.s = s; a.stats = (float2*)stats; a.weight = weight; a.gate = gate; a.next = next;
    a.weight_ws = weight_stride; a.gate_ws = gate_stride; a.next_ws = next_stride;
    a.x_ws = x_worker_stride; a.x_rs = x_row_stride; a.r_ws = residual_worker_stride; a.r_rs = residual_row_stride;
    a.rows = (uint32_t)rows; a.groups = z.groups(gated ? 512 : 1024); a.h = (int32_t)h; a.alpha = (float)residual_scale; a.alpha64 = residual_scale; a.eps = eps;
    return by_block_types(type, gated ? residual_type : type, [&](auto t, auto r) {
        using T = decltype(t);
        using R = decltype(r);
        if (gated) return block_forward<T, R, true>(a, z, vec, (cudaStream_t)cuda_stream);
        return block_forward<T, T, false>(a, z, vec, (cudaStream_t)cuda_stream);
    });
}

int compams_rms_norm_workspace_bytes(size_t* bytes, int32_t n, int64_t rows, int64_t h) {
    const BlockShape z{n, rows, h};
    if (!bytes || !z.ok()) return COMPAMS_ERR_INVALID_ARG;
    *bytes = (size_t)n * z.groups() * 2 * (size_t)h * sizeof(float);
    return COMPAMS_OK;
}

int compams_rms_norm_backward(void* dx, void* dresidual, float* dweight, float* dgate, float* dnext, int32_t sum_workers, const void* dy,
                              const void* ds, const void* x, const void* s, const float* stats, int32_t type, int32_t residual_type, int32_t n,
                              int64_t rows, int64_t h, int64_t dy_worker_stride, int64_t dy_row_stride, int64_t ds_worker_stride,
                              int64_t ds_row_stride, int64_t x_worker_stride, int64_t x_row_stride, const float* weight, int64_t weight_stride,
                              const float* gate, int64_t gate_stride, const float* next, int64_t next_stride, double residual_scale,
                              void* workspace, size_t workspace_bytes, void* cuda_stream) {
    const BlockShape z{n, rows, h};
    const bool gated = s != nullptr, sums = dweight || dgate || dnext;
    if (!z.ok() || !type_known(type) || (gated ? residual_type != type && residual_type != kTypeF32 : ds || dresidual || gate || next || dgate || dnext))
        return COMPAMS_ERR_INVALID_ARG;
    if (!float_aligned(dweight) || !float_aligned(dgate) || !float_aligned(dnext)) return COMPAMS_ERR_INVALID_ARG;
    const cudaStream_t stream = (cudaStream_t)cuda_stream;
    if (rows == 0) {
        const size_t bytes = (size_t)(sum_workers ? 1 : n) * (size_t)h * sizeof(float);
        cudaError_t e = dweight ? cudaMemsetAsync(dweight, 0, bytes, stream) : cudaSuccess;
        if (e == cudaSuccess && dgate) e = cudaMemsetAsync(dgate, 0, bytes, stream);
        if (e == cudaSuccess && dnext) e = cudaMemsetAsync(dnext, 0, bytes, stream);
        return launched(e, "block_backward");
    }
    const size_t need = (size_t)n * z.groups() * 2 * (size_t)h * sizeof(float);
    const Rows gin{dy, dy_worker_stride, dy_row_stride, type}, gsum{ds, ds_worker_stride, ds_row_stride, residual_type};
    const Rows xin{x, x_worker_stride, x_row_stride, type}, sin = packed(s, rows, h, residual_type), out = packed(dx, rows, h, type),
               rout = packed(dresidual, rows, h, residual_type);
    if ((sums && (!workspace || workspace_bytes < need || (reinterpret_cast<uintptr_t>(workspace) & 15u))) || !gin.strides_ok() ||
        (ds && !gsum.strides_ok()) || !xin.strides_ok() || weight_stride < 0 || gate_stride < 0 || next_stride < 0 || !dy || !x || !stats ||
        (reinterpret_cast<uintptr_t>(stats) & 7u) || !float_aligned(weight) || !float_aligned(gate) || !float_aligned(next) ||
        !gin.element_aligned() || !xin.element_aligned() || !out.element_aligned() ||
        (gated && (!gsum.element_aligned() || !sin.element_aligned() || !rout.element_aligned())))
        return COMPAMS_ERR_INVALID_ARG;
    if (!dx && !dresidual && !sums) return COMPAMS_OK;
    const bool vec = h % 8 == 0 && gin.aligned() && xin.aligned() && out.aligned() &&
                     (!gated || ((!ds || gsum.aligned()) && sin.aligned() && rout.aligned())) && vector_parameter(weight, weight_stride) &&
                     vector_parameter(gate, gate_stride) && vector_parameter(next, next_stride);
    BlockArgs a = {};
    a.x = x; a.dy = dy; a.ds = ds; a.s_in = s; a.dx = dx; a.dresidual = dresidual; a.stats = (float2*)const_cast<float*>(stats);
    a.weight = weight; a.gate = gate; a.next = next; a.weight_ws = weight_stride; a.gate_ws = gate_stride; a.next_ws = next_stride;
    a.x_ws = x_worker_stride; a.x_rs = x_row_stride; a.dy_ws = dy_worker_stride; a.dy_rs = dy_row_stride; a.ds_ws = ds_worker_stride;
    a.ds_rs = ds_row_stride; a.rows = (uint32_t)rows; a.groups = z.groups(); a.h = (int32_t)h; a.alpha = (float)residual_scale;
    a.partial = sums ? (float*)workspace : nullptr;
    const int rc = by_block_types(type, gated ? residual_type : type, [&](auto t, auto r) {
        using T = decltype(t);
        using R = decltype(r);
        if (gated) return block_backward<T, R, true>(a, z, vec, stream);
        return block_backward<T, T, false>(a, z, vec, stream);
    });
    if (rc != COMPAMS_OK || !sums) return rc;
    SumsArgs j = {};
    j.partial = a.partial; j.weight = weight; j.gate = gate; j.weight_ws = weight_stride; j.gate_ws = gate_stride; j.dweight = dweight; j.dgate = dgate;
    j.dnext = dnext; j.h = (int32_t)h; j.n = n; j.gated = gated; j.groups = a.groups; j.together = sum_workers != 0;
    return launched(launch_after(block_sums_kernel, dim3((uint32_t)((h + 31) / 32), sum_workers ? 1u : (uint32_t)n), dim3(32, 8), stream, j),
                    "block_sums");
}

}  // extern "C"
