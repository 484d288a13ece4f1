// Low-rank adapters beside a projection, on [n, rows, .] activations, every worker (or request) with its own or all with one:
//
//   t_i = dropout(x_i) A_i^T                       [rows, rank]      "down"
//   y_i = base_i + scale t_i B_i^T                 [rows, out]       "up"
//   backward:  dt_i = scale dy_i B_i               down, from the other side
//              dA_i = dt_i^T dropout(x_i)          [rank, in]        "outer"
//              dB_i = scale dy_i^T t_i             [out, rank]       outer
//              dx_i = dropout(dt_i A_i)            up, onto nothing
//
// A, B, t and the gradients of A and B are fp32. A factor's element (j, c), rank index j and column c, lies at j * sj + c * sc, so
// the three kernels serve both directions: A is (in, 1), B^T is (1, rank).
//
// A product with an activation costs 2 rank operations for each element that is read once, so at the usual ranks it is bound by
// memory, and the kernels are built around 16-byte loads of the activation that become matrix operands where they arrive, in
// registers: a sum's terms and a product's columns may be numbered as one likes, so the eight neighbours that a lane loads are taken as
// the places of the operand that this lane has to hold. No shared memory stands between memory and mma.sync; the factors wait in the
// order of the lanes' registers ("frag") and come through the L1.
//
// Precision. mma.sync multiplies bf16 exactly and adds in fp32. An fp32 number is the sum of three bf16 numbers, its planes (8 bits
// each, cut, not rounded: the rest after each cut is exact, nothing overflows); fp16 needs two and bf16 is one. Products of planes
// i and j are formed for i + j <= 2, which leaves out less than 3 * 2^-24 of a product: as fp32 arithmetic does. Where the result is
// a 16-bit number (y, dx) i + j <= 1 suffice: 3 * 2^-16 of a product, an eighth of half a step of fp16, 2^-6 of one of bf16.
#include "context.h"
#include "rows.cuh"

namespace compams {
namespace {

struct Factor {  // A or B^T
    const float* p;
    int64_t ws, sj, sc;
};

struct AdapterArgs {
    const void* x;  // down, outer: the rows; up: the base (may be null)
    void* y;        // up: the result
    const float* t;
    float* out;     // down: t; outer: the result, or the partial sums [n, chunks, rank * h]
    const uint4* frag;
    Factor f;
    int64_t x_ws, x_rs;
    int64_t frag_ws;   // 16-byte words of a group's fragments
    uint32_t rows, total;
    uint32_t group_rows;  // rows that share a factor: a worker's, or all
    uint32_t tiles;       // down: row tiles of a group; up: row chunks of a group
    int32_t h, rank;
    uint32_t chunks;
    float scale;
    Drop drop;
};

// The kernels behind the first of a call are programmatic dependents of the one before: they read nothing before dependency_wait(), and
// what that call's kernels wrote (t, fragments) by plain loads.

// ---- operands --------------------------------------------------------------------------------------------------------------

__device__ __forceinline__ void mma(float (&c)[4], uint32_t a0, uint32_t a1, uint32_t a2, uint32_t a3, uint32_t b0, uint32_t b1) {
    asm("mma.sync.aligned.m16n8k16.row.col.f32.bf16.bf16.f32 {%0,%1,%2,%3}, {%4,%5,%6,%7}, {%8,%9}, {%0,%1,%2,%3};"
        : "+f"(c[0]), "+f"(c[1]), "+f"(c[2]), "+f"(c[3])
        : "r"(a0), "r"(a1), "r"(a2), "r"(a3), "r"(b0), "r"(b1));
}

// As above onto nothing. The tensor cores cut their sums instead of rounding them, so a sum grows there for a few products only, the
// small planes' first, and joins the others by an fp32 addition: with one running sum in mma.sync dA of 4096 columns and rank 16 was
// 4e-6 off, this way as near as fp32 arithmetic comes.
__device__ __forceinline__ void mma_first(float (&c)[4], uint32_t a0, uint32_t a1, uint32_t a2, uint32_t a3, uint32_t b0, uint32_t b1) {
    asm("mma.sync.aligned.m16n8k16.row.col.f32.bf16.bf16.f32 {%0,%1,%2,%3}, {%4,%5,%6,%7}, {%8,%9}, {%10,%10,%10,%10};"
        : "=f"(c[0]), "=f"(c[1]), "=f"(c[2]), "=f"(c[3])
        : "r"(a0), "r"(a1), "r"(a2), "r"(a3), "r"(b0), "r"(b1), "f"(0.0f));
}

// The first P planes of two numbers, packed. The rest of an infinity is 0, of what is not a number itself.
template <int P>
__device__ __forceinline__ void split2(float a, float b, uint32_t (&planes)[P]) {
#pragma unroll
    for (int p = 0; p < P; ++p) {
        planes[p] = __byte_perm(__float_as_uint(a), __float_as_uint(b), 0x7632);
        if (p + 1 < P) {
            const float ha = __uint_as_float(__float_as_uint(a) & 0xffff0000u), hb = __uint_as_float(__float_as_uint(b) & 0xffff0000u);
            a = a == ha ? 0.0f : a - ha;
            b = b == hb ? 0.0f : b - hb;
        }
    }
}

template <typename T> struct Planes { static constexpr int count = 3; };
template <> struct Planes<__nv_bfloat16> { static constexpr int count = 1; };
template <> struct Planes<__half> { static constexpr int count = 2; };

// A lane's eight neighbours of a row from column c on, 0 beyond h.
template <typename T, bool VEC>
__device__ __forceinline__ Raw8<T> raw_columns(const T* __restrict__ row, int c, int h) {
    Raw8<T> r = {};
    if (VEC) {
        if (c < h) r = raw_load<T>(row + c);
    } else {
        T v[8];
#pragma unroll
        for (int k = 0; k < 8; ++k) v[k] = c + k < h ? __ldg(row + c + k) : from_float<T>(0.0f);
        memcpy(&r, v, sizeof(r));
    }
    return r;
}
// Their planes, as pairs; elements whose bit is 0 are 0.
template <typename T>
__device__ __forceinline__ void raw_planes(const Raw8<T>& r, bool drop, uint32_t bits, uint32_t (&w)[Planes<T>::count][4]) {
    float v[8];
    raw_floats<T>(r, v);
    if (drop)
#pragma unroll
        for (int k = 0; k < 8; ++k)
            if (!((bits >> k) & 1u)) v[k] = 0.0f;
#pragma unroll
    for (int q = 0; q < 4; ++q) {
        uint32_t p[Planes<T>::count];
        split2<Planes<T>::count>(v[2 * q], v[2 * q + 1], p);
#pragma unroll
        for (int k = 0; k < Planes<T>::count; ++k) w[k][q] = p[k];
    }
}
template <>
__device__ __forceinline__ void raw_planes<__nv_bfloat16>(const Raw8<__nv_bfloat16>& r, bool drop, uint32_t bits, uint32_t (&w)[1][4]) {
    w[0][0] = r.q.x; w[0][1] = r.q.y; w[0][2] = r.q.z; w[0][3] = r.q.w;
    if (drop)
#pragma unroll
        for (int q = 0; q < 4; ++q)
            w[0][q] &= ((bits >> (2 * q)) & 1u ? 0xffffu : 0u) | ((bits >> (2 * q + 1)) & 1u ? 0xffff0000u : 0u);
}

// ---- the factors as operands -----------------------------------------------------------------------------------------------

constexpr int kPlanes = 3;
constexpr int kDownColumns = 32;  // columns of a fragment of "down": 8 per lane of a quad
constexpr int kUpColumns = 32;    // columns of a fragment of "up": four 8-column products, whose columns interleave by pairs

__host__ __device__ inline int64_t down_frag_words(int64_t h, int rank) {  // of 16 bytes
    return (h + kDownColumns - 1) / kDownColumns * ((rank + 7) / 8) * kPlanes * 32;
}
__host__ __device__ inline int64_t up_frag_words(int64_t h, int rank) {
    return (h + kUpColumns - 1) / kUpColumns * ((rank + 15) / 16) * kPlanes * 64;
}

// A block per 8 fragments; one lane writes its share of the planes of one fragment.
//   down: [column block][8 ranks][plane][lane g, t] = rank 8 b + g, columns 8 t ... 8 t + 7
//   up:   [column block][16 ranks][plane][half][lane g, t] = for two of the four products q, column 8 (g / 2) + 2 q + g % 2, ranks 4 t ... 4 t + 3
struct PrepareArgs {
    Factor down, up;
    uint4 *down_frag, *up_frag;
    int32_t down_h, up_h, rank;
    uint32_t down_count, up_count;  // fragments of a group
};
__global__ void __launch_bounds__(256) adapter_prepare_kernel(const __grid_constant__ PrepareArgs a) {
    const int lane = threadIdx.x & 31, g = lane >> 2, t = lane & 3;
    uint32_t at = blockIdx.x * 8 + (threadIdx.x >> 5);
    if (at < a.down_count) {
        const int ranks = (a.rank + 7) / 8, j = (int)(at % ranks) * 8 + g, c = (int)(at / ranks) * kDownColumns + 8 * t;
        const float* f = a.down.p + (int64_t)blockIdx.y * a.down.ws;
        uint32_t w[4][kPlanes];
#pragma unroll
        for (int q = 0; q < 4; ++q) {
            float v[2];
#pragma unroll
            for (int k = 0; k < 2; ++k)
                v[k] = j < a.rank && c + 2 * q + k < a.down_h ? __ldg(f + j * a.down.sj + (c + 2 * q + k) * a.down.sc) : 0.0f;
            split2<kPlanes>(v[0], v[1], w[q]);
        }
        uint4* out = a.down_frag + (int64_t)blockIdx.y * down_frag_words(a.down_h, a.rank) + (int64_t)at * kPlanes * 32 + lane;
#pragma unroll
        for (int p = 0; p < kPlanes; ++p) out[p * 32] = make_uint4(w[0][p], w[1][p], w[2][p], w[3][p]);
        return;
    }
    at -= a.down_count;
    if (at >= a.up_count) return;
    const int ranks = (a.rank + 15) / 16, j = (int)(at % ranks) * 16 + 4 * t, c0 = (int)(at / ranks) * kUpColumns + 8 * (g >> 1) + (g & 1);
    const float* f = a.up.p + (int64_t)blockIdx.y * a.up.ws;
    uint32_t w[4][2][kPlanes];
#pragma unroll
    for (int q = 0; q < 4; ++q)
#pragma unroll
        for (int pair = 0; pair < 2; ++pair) {
            float v[2];
#pragma unroll
            for (int k = 0; k < 2; ++k)
                v[k] = j + 2 * pair + k < a.rank && c0 + 2 * q < a.up_h ? __ldg(f + (j + 2 * pair + k) * a.up.sj + (c0 + 2 * q) * a.up.sc) : 0.0f;
            split2<kPlanes>(v[0], v[1], w[q][pair]);
        }
    uint4* out = a.up_frag + (int64_t)blockIdx.y * up_frag_words(a.up_h, a.rank) + (int64_t)at * kPlanes * 64 + lane;
#pragma unroll
    for (int p = 0; p < kPlanes; ++p) {
        out[p * 64] = make_uint4(w[0][0][p], w[0][1][p], w[1][0][p], w[1][1][p]);
        out[p * 64 + 32] = make_uint4(w[2][0][p], w[2][1][p], w[3][0][p], w[3][1][p]);
    }
}

// ---- down ------------------------------------------------------------------------------------------------------------------

// A CTA per 16 MT rows and 8 NT rank indices; its warps take every eighth block of 32 columns, so that the CTA reads 512 bytes of a row
// at a time, and join their sums at the end, in order.
template <typename T, bool VEC, int MT, int NT>
__global__ void __launch_bounds__(256) adapter_down_kernel(const __grid_constant__ AdapterArgs a) {
    __shared__ float joined[8][16][NT * 8 + 1];
    dependency_wait();
    constexpr int PX = Planes<T>::count;
    const int lane = threadIdx.x & 31, warp = threadIdx.x >> 5, g = lane >> 2, t = lane & 3;
    const uint32_t group = blockIdx.x / a.tiles, row0 = (blockIdx.x - group * a.tiles) * 16 * MT;
    const int n0 = blockIdx.y * NT, ntiles = (a.rank + 7) / 8;
    const uint32_t call = drop_call(a.drop);
    const T* row[MT][2];
    uint32_t wi[MT][2], wj[MT][2];
    bool in[MT][2];
#pragma unroll
    for (int q = 0; q < MT; ++q)
#pragma unroll
        for (int half = 0; half < 2; ++half) {
            const uint32_t r = row0 + q * 16 + half * 8 + g;
            in[q][half] = r < a.group_rows;
            const uint32_t m = group * a.group_rows + (in[q][half] ? r : 0);
            wi[q][half] = m / a.rows;
            wj[q][half] = m - wi[q][half] * a.rows;
            row[q][half] = (const T*)a.x + (int64_t)wi[q][half] * a.x_ws + (int64_t)wj[q][half] * a.x_rs;
        }
    const uint4* frag = a.frag + (int64_t)group * a.frag_ws + lane;
    const int blocks = (a.h + kDownColumns - 1) / kDownColumns;
    float acc[MT][NT][4] = {};
    Raw8<T> next[MT][2];
#pragma unroll
    for (int q = 0; q < MT; ++q)
#pragma unroll
        for (int half = 0; half < 2; ++half)
            next[q][half] = raw_columns<T, VEC>(row[q][half], warp * kDownColumns + 8 * t, in[q][half] ? a.h : 0);
    for (int b = warp; b < blocks; b += 8) {
        uint32_t w[MT][2][PX][4];
#pragma unroll
        for (int q = 0; q < MT; ++q)
#pragma unroll
            for (int half = 0; half < 2; ++half) {
                const Raw8<T> now = next[q][half];
                next[q][half] = raw_columns<T, VEC>(row[q][half], (b + 8) * kDownColumns + 8 * t, in[q][half] ? a.h : 0);
                uint32_t bits = 0xffu;
                if (a.drop.on) bits = drop_bits(a.drop, b * (kDownColumns / 8) + t, wj[q][half], a.drop.worker + wi[q][half], call);
                raw_planes<T>(now, a.drop.on, bits, w[q][half]);
            }
#pragma unroll
        for (int j = 0; j < NT; ++j) {
            if (n0 + j >= ntiles) break;
            uint4 f[kPlanes];
#pragma unroll
            for (int p = 0; p < kPlanes; ++p) f[p] = frag[((int64_t)(b * ntiles + n0 + j) * kPlanes + p) * 32];
#pragma unroll
            for (int q = 0; q < MT; ++q) {
                float c[4];
                bool first = true;
#pragma unroll
                for (int sum = kPlanes - 1; sum >= 0; --sum)  // the planes' indices together: the smallest products first
#pragma unroll
                    for (int px = 0; px < PX; ++px) {
                        const int p = sum - px;
                        if (p < 0) break;
                        if (first) mma_first(c, w[q][0][px][0], w[q][1][px][0], w[q][0][px][1], w[q][1][px][1], f[p].x, f[p].y);
                        else mma(c, w[q][0][px][0], w[q][1][px][0], w[q][0][px][1], w[q][1][px][1], f[p].x, f[p].y);
                        mma(c, w[q][0][px][2], w[q][1][px][2], w[q][0][px][3], w[q][1][px][3], f[p].z, f[p].w);
                        first = false;
                    }
#pragma unroll
                for (int k = 0; k < 4; ++k) acc[q][j][k] += c[k];
            }
        }
    }
    const float scale = a.scale * (a.drop.on ? a.drop.factor : 1.0f);
#pragma unroll
    for (int q = 0; q < MT; ++q) {
        if (q) __syncthreads();
#pragma unroll
        for (int j = 0; j < NT; ++j)
#pragma unroll
            for (int k = 0; k < 4; ++k) joined[warp][g + (k >> 1) * 8][j * 8 + 2 * t + (k & 1)] = acc[q][j][k];
        __syncthreads();
        for (int e = threadIdx.x; e < 16 * NT * 8; e += 256) {
            const int r = e / (NT * 8), j = e - r * (NT * 8);
            const uint32_t at = row0 + q * 16 + r;
            if (at < a.group_rows && n0 * 8 + j < a.rank) {
                float s = 0.0f;
#pragma unroll
                for (int w = 0; w < 8; ++w) s += joined[w][r][j];
                a.out[((int64_t)group * a.group_rows + at) * a.rank + n0 * 8 + j] = scale * s;
            }
        }
    }
}

// A few rows that share a factor: bound by the factor, which is read once, in fp32 as it lies. A CTA per rank index.
constexpr int kFewRows = 4;
template <typename T, bool VEC>
__global__ void __launch_bounds__(256) adapter_down_few_kernel(const __grid_constant__ AdapterArgs a) {
    __shared__ float joined[8][kFewRows];
    dependency_wait();
    const int lane = threadIdx.x & 31, warp = threadIdx.x >> 5, j = blockIdx.x;
    const uint32_t group = blockIdx.y, call = drop_call(a.drop);
    const float* f = a.f.p + (int64_t)group * a.f.ws + j * a.f.sj;
    float acc[kFewRows] = {};
    for (int c0 = warp * kSpan; c0 < a.h; c0 += 8 * kSpan) {
        float w[8];
#pragma unroll
        for (int k = 0; k < 8; ++k) {
            const int c = span_column<VEC>(c0, lane, k);
            w[k] = c < a.h ? __ldg(f + c * a.f.sc) : 0.0f;
        }
#pragma unroll
        for (int r = 0; r < kFewRows; ++r) {
            if (r >= (int)a.group_rows) break;
            const uint32_t m = group * a.group_rows + r, i = m / a.rows, jr = m - i * a.rows;
            float v[8];
            span_load<T, VEC>((const T*)a.x + (int64_t)i * a.x_ws + (int64_t)jr * a.x_rs, c0, a.h, lane, v);
            if (a.drop.on) span_drop<VEC>(a.drop, c0, jr, a.drop.worker + i, call, lane, v);
#pragma unroll
            for (int k = 0; k < 8; ++k)
                if (span_column<VEC>(c0, lane, k) < a.h) acc[r] = fmaf(v[k], w[k], acc[r]);
        }
    }
#pragma unroll
    for (int r = 0; r < kFewRows; ++r) {
#pragma unroll
        for (int o = 16; o > 0; o >>= 1) acc[r] += __shfl_xor_sync(0xffffffffu, acc[r], o);
        if (lane == 0) joined[warp][r] = acc[r];
    }
    __syncthreads();
    if (threadIdx.x < kFewRows && threadIdx.x < a.group_rows) {
        float s = 0.0f;
#pragma unroll
        for (int w = 0; w < 8; ++w) s += joined[w][threadIdx.x];
        a.out[((int64_t)group * a.group_rows + threadIdx.x) * a.rank + j] = a.scale * s;
    }
}

// ---- up --------------------------------------------------------------------------------------------------------------------

// A warp per 32 columns goes through the rows of a chunk, 16 MT at a time; the eight warps of a CTA are neighbours and meet at the
// same rows of t in the L1. PT: planes of t and of the factor.
template <typename T, bool VEC, int MT, int PT>
__global__ void __launch_bounds__(256) adapter_up_kernel(const __grid_constant__ AdapterArgs a) {
    dependency_wait();
    const int lane = threadIdx.x & 31, g = lane >> 2, t = lane & 3;
    const uint32_t group = blockIdx.y / a.tiles, chunk = blockIdx.y - group * a.tiles;
    const int cb = blockIdx.x * 8 + (threadIdx.x >> 5), c = cb * kUpColumns + 8 * t;
    if (cb * kUpColumns >= a.h) return;
    const int ranks = (a.rank + 15) / 16;
    const uint32_t steps = (a.group_rows + 16 * MT - 1) / (16 * MT);
    const uint32_t s0 = (uint32_t)((uint64_t)steps * chunk / a.tiles), s1 = (uint32_t)((uint64_t)steps * (chunk + 1) / a.tiles);
    const uint32_t call = drop_call(a.drop);
    const uint4* frag = a.frag + (int64_t)group * a.frag_ws + (int64_t)cb * ranks * kPlanes * 64 + lane;
    const bool four = (a.rank & 3) == 0 && (reinterpret_cast<uintptr_t>(a.t) & 15u) == 0;
    for (uint32_t s = s0; s < s1; ++s) {
        uint32_t m[MT][2], wi[MT][2], wj[MT][2];
        bool in[MT][2];
        Raw8<T> base[MT][2];
#pragma unroll
        for (int q = 0; q < MT; ++q)
#pragma unroll
            for (int half = 0; half < 2; ++half) {
                const uint32_t r = (s * MT + q) * 16 + half * 8 + g;
                in[q][half] = r < a.group_rows;
                m[q][half] = group * a.group_rows + (in[q][half] ? r : 0);
                wi[q][half] = m[q][half] / a.rows;
                wj[q][half] = m[q][half] - wi[q][half] * a.rows;
                base[q][half] = raw_columns<T, VEC>((const T*)a.x + (int64_t)wi[q][half] * a.x_ws + (int64_t)wj[q][half] * a.x_rs, c,
                                                    a.x && in[q][half] ? a.h : 0);
            }
        float acc[MT][4][4] = {};
        for (int b = 0; b < ranks; ++b) {
            uint32_t w[MT][2][2][PT];
#pragma unroll
            for (int q = 0; q < MT; ++q)
#pragma unroll
                for (int half = 0; half < 2; ++half) {
                    const float* p = a.t + (int64_t)m[q][half] * a.rank + b * 16 + 4 * t;
                    float v[4];
                    if (four) {
                        const float4 f = in[q][half] && b * 16 + 4 * t < a.rank ? *reinterpret_cast<const float4*>(p) : make_float4(0.f, 0.f, 0.f, 0.f);
                        v[0] = f.x; v[1] = f.y; v[2] = f.z; v[3] = f.w;
                    } else {
#pragma unroll
                        for (int k = 0; k < 4; ++k) v[k] = in[q][half] && b * 16 + 4 * t + k < a.rank ? p[k] : 0.0f;
                    }
                    split2<PT>(v[0], v[1], w[q][half][0]);
                    split2<PT>(v[2], v[3], w[q][half][1]);
                }
            uint4 f[PT][2];
#pragma unroll
            for (int p = 0; p < PT; ++p) {
                f[p][0] = frag[((int64_t)b * kPlanes + p) * 64];
                f[p][1] = frag[((int64_t)b * kPlanes + p) * 64 + 32];
            }
#pragma unroll
            for (int q = 0; q < MT; ++q)
#pragma unroll
                for (int k = 0; k < 4; ++k) {
                    float d[4] = {};
                    float(&sum)[4] = PT == 3 ? d : acc[q][k];  // a 16-bit result can stand one running sum
#pragma unroll
                    for (int both = PT - 1; both >= 0; --both)
#pragma unroll
                        for (int pt = 0; pt <= both; ++pt) {
                            const uint4 e = f[both - pt][k >> 1];
                            mma(sum, w[q][0][0][pt], w[q][1][0][pt], w[q][0][1][pt], w[q][1][1][pt], k & 1 ? e.z : e.x, k & 1 ? e.w : e.y);
                        }
                    if (PT == 3)
#pragma unroll
                        for (int v = 0; v < 4; ++v) acc[q][k][v] += d[v];
                }
        }
#pragma unroll
        for (int q = 0; q < MT; ++q)
#pragma unroll
            for (int half = 0; half < 2; ++half) {
                if (!in[q][half] || c >= a.h) continue;
                float v[8];
                raw_floats<T>(base[q][half], v);
#pragma unroll
                for (int k = 0; k < 8; ++k) v[k] = fmaf(a.scale, acc[q][k >> 1][half * 2 + (k & 1)], v[k]);
                if (a.drop.on) {
                    const uint32_t bits = drop_bits(a.drop, (uint32_t)c >> 3, wj[q][half], a.drop.worker + wi[q][half], call);
#pragma unroll
                    for (int k = 0; k < 8; ++k) v[k] = (bits >> k) & 1u ? v[k] * a.drop.factor : 0.0f;
                }
                T* y = (T*)a.y + (int64_t)m[q][half] * a.h + c;
                if (VEC) {
                    store8<T>(y, v);
                } else {
#pragma unroll
                    for (int k = 0; k < 8; ++k)
                        if (c + k < a.h) y[k] = from_float<T>(v[k]);
                }
            }
    }
}

// A few rows that share a factor: a warp per span of the columns, the factor read once in fp32.
template <typename T, bool VEC>
__global__ void __launch_bounds__(256) adapter_up_few_kernel(const __grid_constant__ AdapterArgs a) {
    dependency_wait();
    const int lane = threadIdx.x & 31, c0 = (blockIdx.x * 8 + (int)(threadIdx.x >> 5)) * 32;
    const uint32_t group = blockIdx.y;
    const int c = c0 + lane;
    if (c0 >= a.h) return;
    const float* f = a.f.p + (int64_t)group * a.f.ws + c * a.f.sc;
    const float* t = a.t + (int64_t)group * a.group_rows * a.rank;
    float acc[kFewRows] = {};
    const bool four = a.f.sj == 1 && ((reinterpret_cast<uintptr_t>(a.f.p) | (uint64_t)a.f.ws * 4 | (uint64_t)a.f.sc * 4) & 15u) == 0 && (a.rank & 3) == 0;
    if (c < a.h) {
        for (int j = 0; j < a.rank; j += 4) {
            float w[4];
            if (four) {
                const float4 q = __ldg(reinterpret_cast<const float4*>(f + j));
                w[0] = q.x; w[1] = q.y; w[2] = q.z; w[3] = q.w;
            } else {
#pragma unroll
                for (int k = 0; k < 4; ++k) w[k] = j + k < a.rank ? __ldg(f + (j + k) * a.f.sj) : 0.0f;
            }
#pragma unroll
            for (int r = 0; r < kFewRows; ++r)
#pragma unroll
                for (int k = 0; k < 4; ++k)
                    if (r < (int)a.group_rows && j + k < a.rank) acc[r] = fmaf(t[r * a.rank + j + k], w[k], acc[r]);
        }
    }
    const uint32_t call = drop_call(a.drop);
#pragma unroll
    for (int r = 0; r < kFewRows; ++r) {
        if (r >= (int)a.group_rows) break;
        const uint32_t m = group * a.group_rows + r, i = m / a.rows, j = m - i * a.rows;
        float v = a.scale * acc[r];
        if (c < a.h && a.x) v += to_float(__ldg((const T*)a.x + (int64_t)i * a.x_ws + (int64_t)j * a.x_rs + c));
        if (a.drop.on) {
            const uint32_t bits = drop_bits(a.drop, (uint32_t)c >> 3, j, a.drop.worker + i, call);
            v = (bits >> (c & 7)) & 1u ? v * a.drop.factor : 0.0f;
        }
        if (c < a.h) ((T*)a.y)[(int64_t)m * a.h + c] = from_float<T>(v);
    }
}

// ---- outer -----------------------------------------------------------------------------------------------------------------

// A CTA per 128 columns, 8 NT rank indices and chunk of a worker's rows: two warps side by side, four that share out the rows and
// join their sums in order. A lane loads eight neighbours of four rows; pairs of rows become the operand's pairs by byte permutes.
constexpr int kOuterColumns = 128;
template <typename T, bool VEC, int NT>
__global__ void __launch_bounds__(256) adapter_outer_kernel(const __grid_constant__ AdapterArgs a) {
    constexpr int PX = Planes<T>::count;
    __shared__ float joined[kOuterColumns][NT * 8 + 1];
    dependency_wait();
    const int lane = threadIdx.x & 31, warp = threadIdx.x >> 5, g = lane >> 2, t = lane & 3, side = warp & 1, turn = warp >> 1;
    const uint32_t i = blockIdx.y / a.chunks, chunk = blockIdx.y - i * a.chunks;
    const int groups = (a.rank + NT * 8 - 1) / (NT * 8), column = blockIdx.x / groups, n0 = (blockIdx.x - column * groups) * NT * 8;
    const int cc = column * kOuterColumns, c = cc + side * 64 + 8 * g;
    const uint32_t steps = (a.rows + 15) / 16;
    const uint32_t s0 = (uint32_t)((uint64_t)steps * chunk / a.chunks), s1 = (uint32_t)((uint64_t)steps * (chunk + 1) / a.chunks);
    const uint32_t call = drop_call(a.drop);
    const T* x = (const T*)a.x + (int64_t)i * a.x_ws;
    const float* tt = a.t + (int64_t)i * a.rows * a.rank + n0 + g;
    float acc[4][NT][4] = {};
    Raw8<T> next[4];
    float tnext[NT][4];
    auto fetch = [&](uint32_t s) {
#pragma unroll
        for (int r = 0; r < 4; ++r) {
            const uint32_t j = s * 16 + 4 * t + r;
            const bool in = s < s1 && j < a.rows;
            next[r] = raw_columns<T, VEC>(x + (int64_t)(in ? j : 0) * a.x_rs, c, in ? a.h : 0);
#pragma unroll
            for (int q = 0; q < NT; ++q) tnext[q][r] = in && n0 + q * 8 + g < a.rank ? tt[(int64_t)j * a.rank + q * 8] : 0.0f;
        }
    };
    fetch(s0 + turn);
    for (uint32_t s = s0 + turn; s < s1; s += 4) {
        uint32_t w[4][PX][4], f[NT][2][kPlanes];
#pragma unroll
        for (int r = 0; r < 4; ++r) {
            uint32_t bits = 0xffu;
            if (a.drop.on) bits = drop_bits(a.drop, (uint32_t)c >> 3, s * 16 + 4 * t + r, a.drop.worker + i, call);
            raw_planes<T>(next[r], a.drop.on, bits, w[r]);
        }
#pragma unroll
        for (int q = 0; q < NT; ++q) {
            split2<kPlanes>(tnext[q][0], tnext[q][1], f[q][0]);
            split2<kPlanes>(tnext[q][2], tnext[q][3], f[q][1]);
        }
        fetch(s + 4);
#pragma unroll
        for (int k = 0; k < 4; ++k) {
            uint32_t e[PX][4];
#pragma unroll
            for (int px = 0; px < PX; ++px)
#pragma unroll
                for (int pair = 0; pair < 4; ++pair)
                    e[px][pair] = __byte_perm(w[pair & 2][px][k], w[(pair & 2) + 1][px][k], pair & 1 ? 0x7632 : 0x5410);
#pragma unroll
            for (int q = 0; q < NT; ++q) {
                float d[4];
                bool first = true;
#pragma unroll
                for (int both = kPlanes - 1; both >= 0; --both)
#pragma unroll
                    for (int px = 0; px < PX; ++px) {
                        const int p = both - px;
                        if (p < 0) break;
                        if (first) mma_first(d, e[px][0], e[px][1], e[px][2], e[px][3], f[q][0][p], f[q][1][p]);
                        else mma(d, e[px][0], e[px][1], e[px][2], e[px][3], f[q][0][p], f[q][1][p]);
                        first = false;
                    }
#pragma unroll
                for (int v = 0; v < 4; ++v) acc[k][q][v] += d[v];
            }
        }
    }
    for (int w = 0; w < 4; ++w) {
        if (turn == w) {
#pragma unroll
            for (int k = 0; k < 4; ++k)
#pragma unroll
                for (int q = 0; q < NT; ++q)
#pragma unroll
                    for (int e = 0; e < 4; ++e) {
                        float& at = joined[side * 64 + 8 * g + 2 * k + (e >> 1)][q * 8 + 2 * t + (e & 1)];
                        at = w == 0 ? acc[k][q][e] : at + acc[k][q][e];
                    }
        }
        __syncthreads();
    }
    const float scale = a.scale * (a.drop.on ? a.drop.factor : 1.0f);
    float* out = a.out + (int64_t)blockIdx.y * a.rank * a.h;
    const bool ranks_packed = a.f.sj == 1;
    for (int e = threadIdx.x; e < kOuterColumns * NT * 8; e += 256) {
        const int k = ranks_packed ? e / (NT * 8) : e % kOuterColumns, j = ranks_packed ? e % (NT * 8) : e / kOuterColumns;
        if (cc + k < a.h && n0 + j < a.rank) out[(n0 + j) * a.f.sj + (cc + k) * a.f.sc] = scale * joined[k][j];
    }
}

// Sums the chunks of a worker (or of all) in their order.
__global__ void __launch_bounds__(256) adapter_join_kernel(const float* __restrict__ partial, float* out, int64_t len, uint32_t chunks) {
    dependency_wait();
    const int64_t at = (int64_t)blockIdx.x * 256 + threadIdx.x;
    if (at >= len) return;
    const float* p = partial + (int64_t)blockIdx.y * chunks * len + at;
    float s = 0.0f;
    for (uint32_t q = 0; q < chunks; ++q) s += __ldcg(p + q * len);
    out[(int64_t)blockIdx.y * len + at] = s;
}

// ---- host ------------------------------------------------------------------------------------------------------------------

constexpr int kMostRank = 1024;

struct AdapterShape {
    int32_t n;
    int64_t rows, in, out;
    int32_t rank;
    bool ok() const {
        const int64_t most = ((int64_t)1 << 31) - 16 * kSpan;
        return n >= 1 && n <= 65535 && rows >= 0 && rows <= (int64_t)0x7fffffff / n && in >= 1 && in < most && out >= 1 && out < most &&
               rank >= 1 && rank <= kMostRank;
    }
    uint32_t total() const { return (uint32_t)(n * rows); }
};

// Whether the rows that share a factor are few enough for the kernels that read the factor as it lies: with a tile of 16 rows of which
// four are there, three quarters of the products are of zeros, and the fragments are written and read again for them.
bool few(const AdapterShape& z, bool shared) { return (shared ? (int64_t)z.n * z.rows : z.rows) <= kFewRows; }

int outer_ranks(int rank) { return rank <= 8 ? 1 : rank <= 16 ? 2 : 4; }  // NT

// Chunks of a worker's rows: as many as give each SM about four CTAs, of 64 rows at least.
uint32_t outer_chunks(const AdapterShape& z, int64_t h) {
    const int nt = outer_ranks(z.rank) * 8;
    const int64_t tiles = (h + kOuterColumns - 1) / kOuterColumns * ((z.rank + nt - 1) / nt) * z.n;
    int64_t c = 148 * 4 / tiles;
    const int64_t most = (z.rows + 63) / 64;
    if (c > most) c = most;
    if (c > 65535 / z.n) c = 65535 / z.n;
    return (uint32_t)(c < 1 ? 1 : c);
}
int64_t outer_floats(const AdapterShape& z, int64_t h, bool sum_workers) {
    const uint32_t c = outer_chunks(z, h);
    return c == 1 && (!sum_workers || z.n == 1) ? 0 : (int64_t)z.n * c * z.rank * h;
}

template <typename F>
int by_type(int32_t type, F f) {
    return type == kTypeF32 ? f(float()) : type == kTypeBF16 ? f(__nv_bfloat16()) : f(__half());
}
int launched(cudaError_t e, const char* what) { return e == cudaSuccess ? COMPAMS_OK : cuda_fail(e, what); }

AdapterArgs arguments(const AdapterShape& z, Rows x, int64_t h, bool shared, float scale, const Drop& d) {
    AdapterArgs a = {};
    a.x = x.p; a.x_ws = x.worker_stride; a.x_rs = x.row_stride; a.rows = (uint32_t)z.rows; a.total = z.total();
    a.group_rows = shared ? a.total : a.rows;
    a.h = (int32_t)h; a.rank = z.rank; a.scale = scale; a.drop = d;
    return a;
}

int prepare(const AdapterShape& z, bool shared, Factor down, int64_t down_h, uint4* down_frag, Factor up, int64_t up_h, uint4* up_frag,
            cudaStream_t stream) {
    PrepareArgs p = {down, up, down_frag, up_frag, (int32_t)down_h, (int32_t)up_h, z.rank, 0, 0};
    if (down_frag) p.down_count = (uint32_t)((down_h + kDownColumns - 1) / kDownColumns * ((z.rank + 7) / 8));
    if (up_frag) p.up_count = (uint32_t)((up_h + kUpColumns - 1) / kUpColumns * ((z.rank + 15) / 16));
    const uint64_t ctas = ((uint64_t)p.down_count + p.up_count + 7) / 8;
    if (ctas > 0x0fffffffu) return COMPAMS_ERR_TOO_LARGE;
    return launched(launch_plain(adapter_prepare_kernel, dim3((uint32_t)ctas, shared ? 1 : (uint32_t)z.n), dim3(256), 0, stream, p),
                    "adapter_prepare");
}

int down(float* out, Rows x, const AdapterShape& z, int64_t h, bool shared, Factor f, const uint4* frag, float scale, const Drop& d,
         cudaStream_t stream) {
    AdapterArgs a = arguments(z, x, h, shared, scale, d);
    a.out = out; a.f = f; a.frag = frag; a.frag_ws = shared ? 0 : down_frag_words(h, z.rank);
    const uint32_t groups = shared ? 1 : (uint32_t)z.n;
    const bool vec = h % 8 == 0 && x.aligned();
    return by_type(x.type, [&](auto t) {
        using T = decltype(t);
        if (!frag) {
            auto kernel = vec ? adapter_down_few_kernel<T, true> : adapter_down_few_kernel<T, false>;
            return launched(launch_plain(kernel, dim3((uint32_t)z.rank, groups), dim3(256), 0, stream, a), "adapter_down");
        }
        const int ntiles = (z.rank + 7) / 8;
        auto go = [&](auto kernel, int mt, int nt) {
            a.tiles = (a.group_rows + 16 * mt - 1) / (16 * mt);
            const uint64_t ctas = (uint64_t)a.tiles * groups;
            if (ctas > 0x7fffffffu) return (int)COMPAMS_ERR_TOO_LARGE;
            return launched(launch_after(kernel, dim3((uint32_t)ctas, (ntiles + nt - 1) / nt), dim3(256), stream, a), "adapter_down");
        };
        if (ntiles <= 1) return vec ? go(adapter_down_kernel<T, true, 1, 1>, 1, 1) : go(adapter_down_kernel<T, false, 1, 1>, 1, 1);
        if (ntiles <= 2) return vec ? go(adapter_down_kernel<T, true, 1, 2>, 1, 2) : go(adapter_down_kernel<T, false, 1, 2>, 1, 2);
        if (ntiles <= 4) return vec ? go(adapter_down_kernel<T, true, 1, 4>, 1, 4) : go(adapter_down_kernel<T, false, 1, 4>, 1, 4);
        return vec ? go(adapter_down_kernel<T, true, 2, 8>, 2, 8) : go(adapter_down_kernel<T, false, 2, 8>, 2, 8);
    });
}

int up(void* y, Rows base, const float* t, const AdapterShape& z, int64_t h, bool shared, Factor f, const uint4* frag, float scale,
       const Drop& d, cudaStream_t stream) {
    AdapterArgs a = arguments(z, base, h, shared, scale, d);
    a.y = y; a.t = t; a.f = f; a.frag = frag; a.frag_ws = shared ? 0 : up_frag_words(h, z.rank);
    const uint32_t groups = shared ? 1 : (uint32_t)z.n;
    const bool vec = h % 8 == 0 && (!base.p || base.aligned()) && packed(y, z.rows, h, base.type).aligned();
    return by_type(base.type, [&](auto tt) {
        using T = decltype(tt);
        if (!frag) {
            auto kernel = vec ? adapter_up_few_kernel<T, true> : adapter_up_few_kernel<T, false>;
            return launched(launch_after(kernel, dim3((uint32_t)((h + 255) / 256), groups), dim3(256), stream, a), "adapter_up");
        }
        constexpr int MT = sizeof(T) == 4 ? 1 : 2, PT = sizeof(T) == 4 ? 3 : 2;
        // row chunks: as many as give each SM about eight CTAs
        const uint32_t columns = (uint32_t)((h + 8 * kUpColumns - 1) / (8 * kUpColumns)), steps = (a.group_rows + 16 * MT - 1) / (16 * MT);
        uint64_t c = 148 * 8 / ((uint64_t)columns * groups) + 1;
        if (c > steps) c = steps;
        if (c > 65535 / groups) c = 65535 / groups;
        a.tiles = (uint32_t)c;
        auto kernel = vec ? adapter_up_kernel<T, true, MT, PT> : adapter_up_kernel<T, false, MT, PT>;
        return launched(launch_after(kernel, dim3(columns, groups * a.tiles), dim3(256), stream, a), "adapter_up");
    });
}

// out(j, c) at j * sj + c * sc of every worker's rank * h floats.
int outer(float* out, bool sum_workers, Rows x, const float* t, const AdapterShape& z, int64_t h, int64_t sj, int64_t sc, float scale,
          const Drop& d, float* partial, bool first, cudaStream_t stream) {
    AdapterArgs a = arguments(z, x, h, false, scale, d);
    a.t = t; a.f = {nullptr, 0, sj, sc}; a.chunks = outer_chunks(z, h);
    const bool straight = outer_floats(z, h, sum_workers) == 0;
    a.out = straight ? out : partial;
    const int nt = outer_ranks(z.rank);
    const uint64_t tiles = (uint64_t)((h + kOuterColumns - 1) / kOuterColumns) * ((z.rank + 8 * nt - 1) / (8 * nt));
    if (tiles > 0x7fffffffu) return COMPAMS_ERR_TOO_LARGE;
    const int rc = by_type(x.type, [&](auto tt) {
        using T = decltype(tt);
        const bool vec = h % 8 == 0 && x.aligned();
        auto kernel = nt == 1 ? (vec ? adapter_outer_kernel<T, true, 1> : adapter_outer_kernel<T, false, 1>)
                    : nt == 2 ? (vec ? adapter_outer_kernel<T, true, 2> : adapter_outer_kernel<T, false, 2>)
                              : (vec ? adapter_outer_kernel<T, true, 4> : adapter_outer_kernel<T, false, 4>);
        const dim3 grid((uint32_t)tiles, (uint32_t)z.n * a.chunks);
        return launched(first ? launch_plain(kernel, grid, dim3(256), 0, stream, a) : launch_after(kernel, grid, dim3(256), stream, a),
                        "adapter_outer");
    });
    if (rc != COMPAMS_OK || straight) return rc;
    const int64_t len = z.rank * h;
    return launched(launch_after(adapter_join_kernel, dim3((uint32_t)((len + 255) / 256), sum_workers ? 1 : (uint32_t)z.n), dim3(256),
                                 stream, (const float*)partial, out, len, sum_workers ? z.n * a.chunks : a.chunks),
                    "adapter_join");
}

bool float_aligned(const void* p) { return (reinterpret_cast<uintptr_t>(p) & 3u) == 0; }
int64_t padded(int64_t floats) { return (floats + 63) / 64 * 64; }

// The workspace: fragments of the two factors, and, for the backward pass, dt and the partial sums.
struct Places {
    int64_t down, up, dt, partial, bytes;  // offsets in bytes
};
Places places(const AdapterShape& z, bool shared, bool backward, bool sum_workers) {
    const int64_t groups = shared ? 1 : z.n;
    const bool frags = !few(z, shared);
    Places p = {};
    p.up = p.down + (frags ? groups * down_frag_words(backward ? z.out : z.in, z.rank) * 16 : 0);
    p.dt = p.up + (frags ? groups * up_frag_words(backward ? z.in : z.out, z.rank) * 16 : 0);
    p.partial = p.dt + (backward ? padded((int64_t)z.total() * z.rank) * 4 : 0);
    const int64_t fa = backward ? outer_floats(z, z.in, sum_workers) : 0, fb = backward ? outer_floats(z, z.out, sum_workers) : 0;
    p.bytes = p.partial + (fa > fb ? fa : fb) * 4;
    return p;
}

}  // namespace
}  // namespace compams

using namespace compams;

extern "C" {

int compams_adapter_workspace_bytes(size_t* bytes, int32_t n, int64_t rows, int64_t in, int64_t out, int32_t rank, int32_t shared,
                                    int32_t backward, int32_t sum_workers) {
    const AdapterShape z{n, rows, in, out, rank};
    if (!bytes || !z.ok()) return COMPAMS_ERR_INVALID_ARG;
    *bytes = (size_t)places(z, shared != 0, backward != 0, sum_workers != 0).bytes;
    return COMPAMS_OK;
}

int compams_adapter_forward(void* y, float* t, const void* x, const void* base, int32_t type, int32_t n, int64_t rows, int64_t in,
                            int64_t out, int32_t rank, int64_t x_worker_stride, int64_t x_row_stride, int64_t base_worker_stride,
                            int64_t base_row_stride, const float* a, int64_t a_worker_stride, int64_t a_row_stride, const float* b,
                            int64_t b_worker_stride, int64_t b_row_stride, float scale, double p, uint64_t seed, uint32_t call,
                            const int64_t* call_device, uint32_t first_worker, void* workspace, size_t workspace_bytes,
                            void* cuda_stream) {
    const AdapterShape z{n, rows, in, out, rank};
    Drop d, none;
    if (!z.ok() || !type_known(type) || !make_drop(d, p, seed, call, call_device, first_worker) ||
        !make_drop(none, 0.0, 0, 0, nullptr, 0))
        return COMPAMS_ERR_INVALID_ARG;
    if (rows == 0) return COMPAMS_OK;
    const Rows xin{x, x_worker_stride, x_row_stride, type}, bin{base, base_worker_stride, base_row_stride, type};
    const bool shared = n == 1 || (a_worker_stride == 0 && b_worker_stride == 0);
    const Places at = places(z, shared, false, false);
    if (!x || !y || !t || !a || !b || !float_aligned(t) || !float_aligned(a) || !float_aligned(b) || !xin.element_aligned() ||
        !bin.element_aligned() || !packed(y, rows, out, type).element_aligned() || workspace_bytes < (size_t)at.bytes ||
        (at.bytes && !workspace) || (reinterpret_cast<uintptr_t>(workspace) & 15u))
        return COMPAMS_ERR_INVALID_ARG;
    const cudaStream_t stream = (cudaStream_t)cuda_stream;
    const Factor fa{a, a_worker_stride, a_row_stride, 1}, fb{b, b_worker_stride, 1, b_row_stride};
    uint4 *down_frag = nullptr, *up_frag = nullptr;
    int rc = COMPAMS_OK;
    if (!few(z, shared)) {
        down_frag = (uint4*)((char*)workspace + at.down);
        up_frag = (uint4*)((char*)workspace + at.up);
        rc = prepare(z, shared, fa, in, down_frag, fb, out, up_frag, stream);
    }
    if (rc == COMPAMS_OK) rc = down(t, xin, z, in, shared, fa, down_frag, 1.0f, d, stream);
    if (rc == COMPAMS_OK) rc = up(y, bin, t, z, out, shared, fb, up_frag, scale, none, stream);
    return rc;
}

int compams_adapter_backward(void* dx, float* da, float* db, int32_t sum_workers, const void* dy, const void* x, const float* t,
                             int32_t type, int32_t n, int64_t rows, int64_t in, int64_t out, int32_t rank, int64_t dy_worker_stride,
                             int64_t dy_row_stride, int64_t x_worker_stride, int64_t x_row_stride, const float* a,
                             int64_t a_worker_stride, int64_t a_row_stride, const float* b, int64_t b_worker_stride,
                             int64_t b_row_stride, float scale, double p, uint64_t seed, uint32_t call, const int64_t* call_device,
                             uint32_t first_worker, void* workspace, size_t workspace_bytes, void* cuda_stream) {
    const AdapterShape z{n, rows, in, out, rank};
    Drop d, none;
    if (!z.ok() || !type_known(type) || !make_drop(d, p, seed, call, call_device, first_worker) ||
        !make_drop(none, 0.0, 0, 0, nullptr, 0))
        return COMPAMS_ERR_INVALID_ARG;
    const cudaStream_t stream = (cudaStream_t)cuda_stream;
    if (rows == 0) {
        const size_t many = sum_workers ? 1 : n;
        cudaError_t e = da ? cudaMemsetAsync(da, 0, many * rank * in * sizeof(float), stream) : cudaSuccess;
        if (e == cudaSuccess && db) e = cudaMemsetAsync(db, 0, many * rank * out * sizeof(float), stream);
        return launched(e, "adapter_backward");
    }
    const Rows xin{x, x_worker_stride, x_row_stride, type}, gin{dy, dy_worker_stride, dy_row_stride, type};
    const bool shared = n == 1 || (a_worker_stride == 0 && b_worker_stride == 0);
    const Places at = places(z, shared, true, sum_workers != 0);
    if (!dy || !a || !b || (da && !x) || (db && !t) || !workspace || workspace_bytes < (size_t)at.bytes ||
        (reinterpret_cast<uintptr_t>(workspace) & 15u) || !float_aligned(t) || !float_aligned(a) || !float_aligned(b) ||
        !float_aligned(da) || !float_aligned(db) || !xin.element_aligned() || !gin.element_aligned() ||
        !packed(dx, rows, in, type).element_aligned())
        return COMPAMS_ERR_INVALID_ARG;
    const Factor fa{a, a_worker_stride, a_row_stride, 1}, fb{b, b_worker_stride, 1, b_row_stride};
    float* dt = (float*)((char*)workspace + at.dt);
    float* partial = (float*)((char*)workspace + at.partial);
    uint4 *down_frag = nullptr, *up_frag = nullptr;
    int rc = COMPAMS_OK;
    if (!few(z, shared) && (dx || da)) {
        down_frag = (uint4*)((char*)workspace + at.down);
        up_frag = dx ? (uint4*)((char*)workspace + at.up) : nullptr;
        rc = prepare(z, shared, fb, out, down_frag, fa, in, up_frag, stream);
    }
    if (rc == COMPAMS_OK && (dx || da)) rc = down(dt, gin, z, out, shared, fb, down_frag, scale, none, stream);
    if (rc == COMPAMS_OK && db) rc = outer(db, sum_workers, gin, t, z, out, 1, rank, scale, none, partial, !(dx || da), stream);
    if (rc == COMPAMS_OK && da) rc = outer(da, sum_workers, xin, dt, z, in, in, 1, 1.0f, d, partial, false, stream);
    if (rc == COMPAMS_OK && dx) rc = up(dx, {nullptr, 0, 0, type}, dt, z, in, shared, fa, up_frag, 1.0f, d, stream);
    return rc;
}

}  // extern "C"
