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
// the places of the operand that this lane has to hold. No exchange between lanes stands between memory and mma.sync; the factors and t
// wait in the order of the lanes' registers and come through the L1.
//
// Precision. mma.sync multiplies bf16 exactly and adds in fp32. An fp32 number is the sum of three bf16 numbers, its planes: each is the
// rest of those before it, rounded, and every rest is exact (of numbers below 2^-110 what lies under 2^-133 is lost); fp16 needs two and
// bf16 is one. Products of planes i and j are formed for i + j <= 2, which leaves out at most 2^-24 of a product, of either sign: as fp32
// arithmetic does. (Planes that are cut instead of rounded leave out up to 2^-21, always towards zero.) So also where the result is a
// 16-bit number (y, dx): base and adapter may cancel, and a result near the border of two roundings should fall where fp32 arithmetic
// lets it fall.
#include <cooperative_groups.h>
#include <string.h>

#include <algorithm>
#include <atomic>
#include <type_traits>

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
    const float* t; // the kernels for a few rows: t
    float* out;     // down: t (may be null); outer: the result, or the partial sums [n, chunks, rank * h]
    const uint4* frag;       // down, up: the factor's fragments
    uint4* t_up;             // t as an operand of up: written by down, read by up
    uint2* t_outer;          // t as an operand of outer: written by down (may be null), read by outer
    Factor f;
    int64_t x_ws, x_rs;
    int64_t frag_ws;   // 16-byte words of a worker's fragments; 0: one factor for all
    uint32_t rows;
    uint32_t tiles;    // down: row tiles of a worker; up: row chunks of a worker
    int32_t h, rank;
    uint32_t chunks;   // outer: row chunks of a worker
    int32_t split;     // down: CTAs of a cluster, which share out the columns
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
// small planes' first, and joins the others by an fp32 addition: 300 rows of fp32, 1000 columns, rank 8: the largest error of dA is 1.3e-7
// of its largest value (torch's fp32 product: 7.6e-7); with one running sum it was 1.8e-6.
__device__ __forceinline__ void mma_first(float (&c)[4], uint32_t a0, uint32_t a1, uint32_t a2, uint32_t a3, uint32_t b0, uint32_t b1) {
    asm("mma.sync.aligned.m16n8k16.row.col.f32.bf16.bf16.f32 {%0,%1,%2,%3}, {%4,%5,%6,%7}, {%8,%9}, {%10,%10,%10,%10};"
        : "=f"(c[0]), "=f"(c[1]), "=f"(c[2]), "=f"(c[3])
        : "r"(a0), "r"(a1), "r"(a2), "r"(a3), "r"(b0), "r"(b1), "f"(0.0f));
}

// The first P planes of two numbers, packed. All but the last are held to finite numbers, so that the largest numbers are not rounded to an
// infinity, whose rest would be the other; an infinity arrives in the last plane.
template <int P>
__device__ __forceinline__ void split2(float a, float b, uint32_t (&planes)[P]) {
#pragma unroll
    for (int p = 0; p < P; ++p) {
        if (p + 1 < P) {
            asm("cvt.rn.satfinite.bf16x2.f32 %0, %1, %2;" : "=r"(planes[p]) : "f"(b), "f"(a));
            a -= __uint_as_float(planes[p] << 16);
            b -= __uint_as_float(planes[p] & 0xffff0000u);
        } else {
            asm("cvt.rn.bf16x2.f32 %0, %1, %2;" : "=r"(planes[p]) : "f"(b), "f"(a));
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
// Their planes, as pairs; dropped elements are 0.
template <typename T>
__device__ __forceinline__ void raw_planes(const Raw8<T>& r, const Drop& d, const uint4& u, uint32_t (&w)[Planes<T>::count][4]) {
    float v[8];
    raw_floats<T>(r, v);
    if (d.on)
#pragma unroll
        for (int k = 0; k < 8; ++k)
            if (!drop_keeps(d, u, k)) v[k] = 0.0f;
#pragma unroll
    for (int q = 0; q < 4; ++q) {
        uint32_t p[Planes<T>::count];
        split2<Planes<T>::count>(v[2 * q], v[2 * q + 1], p);
#pragma unroll
        for (int k = 0; k < Planes<T>::count; ++k) w[k][q] = p[k];
    }
}
template <>
__device__ __forceinline__ void raw_planes<__nv_bfloat16>(const Raw8<__nv_bfloat16>& r, const Drop& d, const uint4& u, uint32_t (&w)[1][4]) {
    w[0][0] = r.q.x; w[0][1] = r.q.y; w[0][2] = r.q.z; w[0][3] = r.q.w;
    if (d.on)
#pragma unroll
        for (int q = 0; q < 4; ++q) {
            if (!drop_keeps(d, u, 2 * q)) w[0][q] &= 0xffff0000u;
            if (!drop_keeps(d, u, 2 * q + 1)) w[0][q] &= 0xffffu;
        }
}

// ---- the factors as operands -----------------------------------------------------------------------------------------------

constexpr int kPlanes = 3;
constexpr int kDownColumns = 32;  // columns of a fragment of "down": 8 per lane of a quad
constexpr int kUpColumns = 32;    // columns of a fragment of "up": four 8-column products, whose columns interleave by pairs

// Rank indices are taken in groups of NT tiles of 8: all of them up to 64, 64 at a time beyond. Fragments of a group are padded to whole
// groups and an even number of column blocks, so that the loops over them have no ends to look for; what is padded is 0.
__host__ __device__ inline int group_tiles(int rank) { return rank <= 8 ? 1 : rank <= 16 ? 2 : rank <= 32 ? 4 : 8; }  // NT
__host__ __device__ inline int rank_groups(int rank) { return rank <= 64 ? 1 : (rank + 63) / 64; }
__host__ __device__ inline int rank_tiles(int rank) { return rank_groups(rank) * group_tiles(rank); }
__host__ __device__ inline int down_blocks(int64_t h) { return (int)((h + 2 * kDownColumns - 1) / (2 * kDownColumns) * 2); }

// Words of 16 bytes, a worker's:
//   down: [group][column block][tile][plane][lane g, t] = rank 8 tile + g, columns 8 t ... 8 t + 7
//   up:   [column block][16 ranks][plane][half][lane g, t] = for two of the four products q, column 8 (g / 2) + 2 q + g % 2, ranks 4 t ... 4 t + 3
__host__ __device__ inline int64_t down_frag_words(int64_t h, int rank) { return (int64_t)down_blocks(h) * rank_tiles(rank) * kPlanes * 32; }
__host__ __device__ inline int64_t up_frag_words(int64_t h, int rank) {
    return (h + kUpColumns - 1) / kUpColumns * ((rank + 15) / 16) * kPlanes * 64;
}
// t as an operand, 16 rows of a worker at a time:
//   up:    [16 rows][16 ranks][plane][lane g, t] = rows g and g + 8, ranks 4 t ... 4 t + 3 (16 bytes)
//   outer: [group][16 rows][tile][plane][lane g, t] = rows 4 t ... 4 t + 3, rank g (8 bytes)
__host__ __device__ inline int64_t t_up_words(int64_t rows, int rank) { return (rows + 15) / 16 * ((rank + 15) / 16) * kPlanes * 32; }
__host__ __device__ inline int64_t t_outer_words(int64_t rows, int rank) { return (rows + 15) / 16 * rank_tiles(rank) * kPlanes * 16; }
// Four numbers of t as an operand of outer.
__device__ __forceinline__ void store_t_outer(uint2* at, const float (&v)[4]) {
    uint32_t lo[kPlanes], hi[kPlanes];
    split2<kPlanes>(v[0], v[1], lo);
    split2<kPlanes>(v[2], v[3], hi);
#pragma unroll
    for (int p = 0; p < kPlanes; ++p) at[p * 32] = make_uint2(lo[p], hi[p]);
}

// A warp per fragment; a lane writes its share of the planes. In the backward pass the forward pass's t becomes an operand of outer too.
struct PrepareArgs {
    Factor down, up;
    uint4 *down_frag, *up_frag;
    const float* t;
    uint2* t_outer;
    int32_t down_h, up_h, rank;
    uint32_t rows;
    uint32_t down_count, up_count, t_count;  // fragments of a worker
    int32_t shared;  // the factors' fragments are those of worker 0
};
__global__ void __launch_bounds__(256) adapter_prepare_kernel(const __grid_constant__ PrepareArgs a) {
    const int lane = threadIdx.x & 31, g = lane >> 2, t = lane & 3;
    uint32_t at = blockIdx.x * 8 + (threadIdx.x >> 5);
    if (at < a.t_count) {
        const uint32_t nt = group_tiles(a.rank), blocks = (a.rows + 15) / 16, tile = at % nt, block = at / nt % blocks, group = at / nt / blocks;
        const int j = (int)(group * nt + tile) * 8 + g;
        const uint32_t row = block * 16 + 4 * t;
        float v[4];
#pragma unroll
        for (int k = 0; k < 4; ++k)
            v[k] = row + k < a.rows && j < a.rank ? __ldg(a.t + ((int64_t)blockIdx.y * a.rows + row + k) * a.rank + j) : 0.0f;
        store_t_outer(a.t_outer + blockIdx.y * t_outer_words(a.rows, a.rank) * 2 + (int64_t)at * kPlanes * 32 + lane, v);
        return;
    }
    at -= a.t_count;
    if (a.shared && blockIdx.y) return;
    if (at < a.down_count) {
        const uint32_t nt = group_tiles(a.rank), blocks = down_blocks(a.down_h), tile = at % nt, block = at / nt % blocks, group = at / nt / blocks;
        const int j = (int)(group * nt + tile) * 8 + g;
        const int64_t c = (int64_t)block * kDownColumns + 8 * t;
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

}  // namespace
}  // namespace compams

#include "adapter_tensor.cuh"

namespace compams {
namespace {

// ---- rings of asynchronous copies ------------------------------------------------------------------------------------------

// Every lane copies what it will need of an activation into places of shared memory that it alone reads, kStages - 1 steps ahead, so
// that no registers wait for memory; place: [stage][slot][thread], 16 bytes each. What the warps of a CTA share (the factor's fragments,
// t's) is copied by all of them into a stage of the same step. Per step: wait for the step's copies, a barrier, behind which the stage of
// the step before is free and is filled again, then the products.
constexpr int kStages = 3;
template <int SLOTS>
__device__ __forceinline__ uint4* ring_at(char* smem, int stage, int slot) {
    return reinterpret_cast<uint4*>(smem) + (stage * SLOTS + slot) * 256 + threadIdx.x;
}
template <int N, typename T>
__device__ __forceinline__ Raw8<T> ring_raw(char* smem, int stage, int slot) {  // slot: of the first 16 bytes
    Raw8<T> r;
    uint4 q[sizeof(r) / 16];
#pragma unroll
    for (int k = 0; k < (int)sizeof(r) / 16; ++k) q[k] = *ring_at<N>(smem, stage, slot + k);
    memcpy(&r, q, sizeof(r));
    return r;
}

// ---- down ------------------------------------------------------------------------------------------------------------------

// A warp takes MT blocks of 16 rows and 8 NT rank indices; WK warps of a CTA share out the columns of their rows, and so do the CTAs of a
// cluster. WK is 8, and every warp fetches fragments of its own, or 1: then the eight warps, of different rows, share the fragments, which
// pass through shared memory. The sums of the warps and of the CTAs are
// joined in their order, through the CTAs' shared memory, and leave as t and as the operands that up and outer take. Bound by the
// instructions that make operands of the activation, not by memory: 8 workers of 2048 rows of 4096 in fp16, rank 16, 134 MB, 58 us
// (2.3 TB/s), 72 with dropout; of 1024 rows in fp32, 134 MB too, 58 and 63. 8 workers of 48 rows in bfloat16 7 us.
template <typename T>
__host__ __device__ constexpr int down_step() { return sizeof(T) == 4 ? 1 : 2; }  // blocks of 32 columns in a step
template <typename T, bool VEC, int NT, int WK, int MT>
__host__ __device__ constexpr int down_ring() { return VEC ? kStages * 2 * MT * down_step<T>() * (int)sizeof(Raw8<T>) * 256 : 0; }
template <typename T, bool VEC, int NT, int WK, int MT>
__host__ __device__ constexpr int down_shared() {
    const int rings = down_ring<T, VEC, NT, WK, MT>() + (WK == 1 ? kStages * down_step<T>() * NT * kPlanes * 512 : 0);
    const int join = (8 * MT + 1) * 16 * (NT * 8 + 1) * 4;
    return rings > join ? rings : join;
}

template <typename T, bool VEC, int NT, int WK, int MT>
__global__ void __launch_bounds__(256, MT == 1 ? 2 : 1) adapter_down_kernel(const __grid_constant__ AdapterArgs a) {
    extern __shared__ __align__(16) char smem[];
    dependency_wait();
    constexpr int PX = Planes<T>::count, KB = down_step<T>(), S16 = (int)sizeof(Raw8<T>) / 16, SLOTS = 2 * MT * KB * S16;
    constexpr int BLOCKS = 8 * MT / WK;  // of 16 rows, a CTA's
    uint4* stages = reinterpret_cast<uint4*>(smem + down_ring<T, VEC, NT, WK, MT>());
    const int lane = threadIdx.x & 31, warp = threadIdx.x >> 5, g = lane >> 2, t = lane & 3;
    const uint32_t tile = blockIdx.x / a.split, i = tile / a.tiles;
    const int part = (int)(blockIdx.x - tile * a.split);
    const uint32_t block0 = (tile - i * a.tiles) * BLOCKS;  // the first block of rows
    const uint32_t row0 = (block0 + warp / WK * MT) * 16;
    const int n0 = blockIdx.y * NT;
    const uint32_t call = drop_call(a.drop);
    const T* row[MT][2];
    bool in[MT][2];
#pragma unroll
    for (int q = 0; q < MT; ++q)
#pragma unroll
        for (int half = 0; half < 2; ++half) {
            const uint32_t r = row0 + q * 16 + half * 8 + g;
            in[q][half] = r < a.rows;
            row[q][half] = (const T*)a.x + (int64_t)i * a.x_ws + (int64_t)(in[q][half] ? r : 0) * a.x_rs;
        }
    const int steps = down_blocks(a.h) / KB, stride = a.split * WK;
    const uint4* frag = a.frag + (int64_t)i * a.frag_ws + (int64_t)blockIdx.y * steps * (KB * NT * kPlanes * 32);
    float acc[MT][NT][4] = {};
    Raw8<T> next[MT][2][KB];
    auto fetch = [&](int step, int stage) {
#pragma unroll
        for (int q = 0; q < MT; ++q)
#pragma unroll
            for (int half = 0; half < 2; ++half)
#pragma unroll
                for (int k = 0; k < KB; ++k) {
                    const int c = (step * KB + k) * kDownColumns + 8 * t;
                    const bool there = step < steps && in[q][half] && c < a.h;
                    if constexpr (VEC) {
#pragma unroll
                        for (int v = 0; v < S16; ++v)
                            copy16(ring_at<SLOTS>(smem, stage, ((q * 2 + half) * KB + k) * S16 + v),
                                   there ? reinterpret_cast<const char*>(row[q][half] + c) + 16 * v : a.x, there);
                    } else {
                        next[q][half][k] = raw_columns<T, false>(row[q][half], c, there ? a.h : 0);
                    }
                }
    };
    auto fetch_shared = [&](int step, int stage) {
        if constexpr (WK == 1) {
            uint4* to = stages + stage * (KB * NT * kPlanes * 32);
            const uint4* from = frag + (int64_t)step * (KB * NT * kPlanes * 32);
            if (step < steps)
#pragma unroll
                for (int e = threadIdx.x; e < KB * NT * kPlanes * 32; e += 256) copy16(to + e, from + e, true);
        }
        copies_commit();
    };
    const int first = part * WK + warp % WK;
    if constexpr (VEC) {
        for (int s = 0; s < kStages - 1; ++s) {
            fetch(first + s * stride, s);
            fetch_shared(first + s * stride, s);
        }
    } else {
        fetch(first, 0);
        for (int s = 0; s < kStages - 1; ++s) fetch_shared(first + s * stride, s);
    }
    int stage = 0;
    for (int step = first; step < steps; step += stride) {
        copies_wait<kStages - 2>();
        if constexpr (WK == 1) __syncthreads();  // (the steps of all warps are the same)
        else __syncwarp();
        const int behind = stage == 0 ? kStages - 1 : stage - 1;
        uint32_t w[MT][2][KB][PX][4];
#pragma unroll
        for (int q = 0; q < MT; ++q)
#pragma unroll
            for (int half = 0; half < 2; ++half)
#pragma unroll
                for (int k = 0; k < KB; ++k) {
                    Raw8<T> now;
                    if constexpr (VEC) now = ring_raw<SLOTS, T>(smem, stage, ((q * 2 + half) * KB + k) * S16);
                    else now = next[q][half][k];
                    uint4 u = {};
                    if (a.drop.on)
                        u = drop_words(a.drop, (step * KB + k) * (kDownColumns / 8) + t, row0 + q * 16 + half * 8 + g, a.drop.worker + i, call);
                    raw_planes<T>(now, a.drop, u, w[q][half][k]);
                }
        if constexpr (VEC) fetch(step + (kStages - 1) * stride, behind);
        else fetch(step + stride, 0);
        fetch_shared(step + (kStages - 1) * stride, behind);
        const uint4 *here = stages + stage * (KB * NT * kPlanes * 32) + lane, *mine = frag + (int64_t)step * (KB * NT * kPlanes * 32) + lane;
        stage = stage + 1 == kStages ? 0 : stage + 1;
#pragma unroll
        for (int k = 0; k < KB; ++k) {
#pragma unroll
            for (int j = 0; j < NT; ++j) {
                uint4 f[kPlanes];
#pragma unroll
                for (int p = 0; p < kPlanes; ++p)
                    f[p] = WK == 1 ? here[((k * NT + j) * kPlanes + p) * 32] : mine[((k * NT + j) * kPlanes + p) * 32];
#pragma unroll
                for (int q = 0; q < MT; ++q) {
                    float c[4];
                    bool start = true;
#pragma unroll
                    for (int sum = kPlanes - 1; sum >= 0; --sum)  // the planes' indices together: the smallest products first
#pragma unroll
                        for (int px = 0; px < PX; ++px) {
                            const int p = sum - px;
                            if (p < 0) break;
                            if (start) mma_first(c, w[q][0][k][px][0], w[q][1][k][px][0], w[q][0][k][px][1], w[q][1][k][px][1], f[p].x, f[p].y);
                            else mma(c, w[q][0][k][px][0], w[q][1][k][px][0], w[q][0][k][px][1], w[q][1][k][px][1], f[p].x, f[p].y);
                            mma(c, w[q][0][k][px][2], w[q][1][k][px][2], w[q][0][k][px][3], w[q][1][k][px][3], f[p].z, f[p].w);
                            start = false;
                        }
#pragma unroll
                    for (int e = 0; e < 4; ++e) acc[q][j][e] += c[e];
                }
            }
        }
    }
    // joined[warp][MT][row][rank], then whole[row][rank] of one block of rows
    constexpr int L = NT * 8 + 1, B = 16 * L;
    float* joined = reinterpret_cast<float*>(smem);
    float* whole = joined + 8 * MT * B;
    copies_wait<0>();
    __syncthreads();  // the rings' memory is taken over
#pragma unroll
    for (int q = 0; q < MT; ++q)
#pragma unroll
        for (int j = 0; j < NT; ++j)
#pragma unroll
            for (int e = 0; e < 4; ++e) joined[(warp * MT + q) * B + (g + (e >> 1) * 8) * L + j * 8 + 2 * t + (e & 1)] = acc[q][j][e];
    __syncthreads();
    if (WK > 1) {
        static_assert(WK == 1 || MT == 1, "");
        for (int e = threadIdx.x; e < B; e += 256) {
            float v = joined[e];
#pragma unroll
            for (int w = 1; w < WK; ++w) v += joined[w * B + e];
            joined[e] = v;
        }
    }
    cooperative_groups::cluster_group cluster = cooperative_groups::this_cluster();
    cluster.sync();
    const float scale = a.scale * (a.drop.on ? a.drop.factor : 1.0f);
    const int ranks = (a.rank + 15) / 16;
    for (int b = part; b < BLOCKS; b += a.split) {
        const uint32_t block = block0 + b;
        if (block * 16 >= a.rows) break;
        for (int e = threadIdx.x; e < B; e += 256) {
            float v = 0.0f;
            for (int s = 0; s < a.split; ++s) v += cluster.map_shared_rank(joined, s)[b * WK * B + e];
            whole[e] = scale * v;
        }
        __syncthreads();
        if (a.out)
            for (int e = threadIdx.x; e < 16 * NT * 8; e += 256) {
                const int r = e / (NT * 8), j = e - r * (NT * 8);
                if (block * 16 + r < a.rows && n0 * 8 + j < a.rank)
                    a.out[((int64_t)i * a.rows + block * 16 + r) * a.rank + n0 * 8 + j] = whole[r * L + j];
            }
        for (int q = warp; q < (NT + 1) / 2; q += 8) {  // 16 rank indices each
            if (n0 / 2 + q >= ranks) break;
            uint32_t v[2][2][kPlanes];  // [rows g, g + 8][pair of ranks]
#pragma unroll
            for (int half = 0; half < 2; ++half)
#pragma unroll
                for (int pair = 0; pair < 2; ++pair) {
                    const int j = q * 16 + 4 * t + 2 * pair;
                    const float* at = whole + (g + half * 8) * L + j;
                    split2<kPlanes>(j < NT * 8 ? at[0] : 0.0f, j < NT * 8 ? at[1] : 0.0f, v[half][pair]);
                }
            uint4* out = a.t_up + i * t_up_words(a.rows, a.rank) + ((int64_t)block * ranks + n0 / 2 + q) * kPlanes * 32 + lane;
#pragma unroll
            for (int p = 0; p < kPlanes; ++p) out[p * 32] = make_uint4(v[0][0][p], v[1][0][p], v[0][1][p], v[1][1][p]);
        }
        if (a.t_outer)
            for (int q = warp; q < NT; q += 8) {
                float v[4];
#pragma unroll
                for (int k = 0; k < 4; ++k) v[k] = whole[(4 * t + k) * L + q * 8 + g];
                store_t_outer(a.t_outer + i * t_outer_words(a.rows, a.rank) * 2 +
                                  (((int64_t)blockIdx.y * ((a.rows + 15) / 16) + block) * NT + q) * kPlanes * 32 + lane,
                              v);
            }
        __syncthreads();
    }
    cluster.sync();  // the others may still be reading
}

// A few rows to a worker: bound by the factor, which is read once, in fp32 as it lies. A CTA per worker and rank index. 32 workers of one
// row of 4096, rank 16, 8.4 MB of factors: 5.4 us, of which the launch and two trips to memory take most.
constexpr int kFewRows = 4;
template <typename T, bool VEC>
__global__ void __launch_bounds__(256) adapter_down_few_kernel(const __grid_constant__ AdapterArgs a) {
    __shared__ float joined[8][kFewRows];
    const int lane = threadIdx.x & 31, warp = threadIdx.x >> 5, j = blockIdx.x;
    const uint32_t i = blockIdx.y, call = drop_call(a.drop);
    const float* f = a.f.p + (int64_t)i * a.f.ws + j * a.f.sj;
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
            if (r >= (int)a.rows) break;
            float v[8];
            span_load<T, VEC>((const T*)a.x + (int64_t)i * a.x_ws + (int64_t)r * a.x_rs, c0, a.h, lane, v);
            if (a.drop.on) span_drop<VEC>(a.drop, c0, r, a.drop.worker + i, call, lane, v);
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
    if (threadIdx.x < kFewRows && threadIdx.x < a.rows) {
        float s = 0.0f;
#pragma unroll
        for (int w = 0; w < 8; ++w) s += joined[w][threadIdx.x];
        a.out[((int64_t)i * a.rows + threadIdx.x) * a.rank + j] = a.scale * s;
    }
}

// ---- up --------------------------------------------------------------------------------------------------------------------

// A warp per 32 columns goes through the blocks of 16 rows of a chunk, MB at a time; the eight warps of a CTA are neighbours and share
// t, which passes through shared memory. RB: blocks of 16 rank indices, whose fragments of the factor stay in registers (0: any number;
// fragments and t are fetched again for each block of rows). 8 workers of 2048 rows of 4096 in fp16, rank 16, 268 MB with the base, take
// 61 us (4.4 TB/s), 80 for dx with dropout, 134 MB; rank 32 89 and 118. Bound by the six products of planes from rank 64 on: 175 and 197 us,
// with one CTA to an SM, whose registers hold the fragments (fetched again for each block of rows: 248 and 260). Rank 128, where the
// fragments' way through the L1 is the limit: 431 and 448 us.
template <typename T, int RB>
__host__ __device__ constexpr int up_rows() { return RB == 1 && sizeof(T) == 2 ? 2 : 1; }  // MB
template <typename T, bool VEC, int RB>
__host__ __device__ constexpr int up_ring() { return VEC ? kStages * 2 * up_rows<T, RB>() * (int)sizeof(Raw8<T>) * 256 : 0; }
template <typename T, bool VEC, int RB>
__host__ __device__ constexpr int up_shared() { return up_ring<T, VEC, RB>() + kStages * up_rows<T, RB>() * RB * kPlanes * 512; }

template <typename T, bool VEC, int RB>
__global__ void __launch_bounds__(256, RB == 4 ? 1 : 2) adapter_up_kernel(const __grid_constant__ AdapterArgs a) {
    extern __shared__ __align__(16) char smem[];
    constexpr int S16 = (int)sizeof(Raw8<T>) / 16, MB = up_rows<T, RB>(), SLOTS = 2 * MB * S16, STAGE = MB * RB * kPlanes * 32;
    dependency_wait();
    uint4* stages = reinterpret_cast<uint4*>(smem + up_ring<T, VEC, RB>());
    const int lane = threadIdx.x & 31, g = lane >> 2, t = lane & 3;
    const uint32_t i = blockIdx.y / a.tiles, chunk = blockIdx.y - i * a.tiles;
    const int cb = blockIdx.x * 8 + (threadIdx.x >> 5), c = cb * kUpColumns + 8 * t;
    const bool mine = cb * kUpColumns < a.h;  // a whole warp
    const int ranks = RB ? RB : (a.rank + 15) / 16;
    const uint32_t blocks = (a.rows + 15) / 16;
    const uint32_t b0 = (uint32_t)((uint64_t)blocks * chunk / a.tiles), b1 = (uint32_t)((uint64_t)blocks * (chunk + 1) / a.tiles);
    const uint32_t call = drop_call(a.drop);
    const uint4* frag = a.frag + (int64_t)i * a.frag_ws + (int64_t)(mine ? cb : 0) * ranks * kPlanes * 64 + lane;
    const uint4* tt = a.t_up + i * t_up_words(a.rows, a.rank);
    uint4 f[RB ? RB : 1][kPlanes][2];
    auto factor = [&](int r, uint4 (&to)[kPlanes][2]) {
#pragma unroll
        for (int p = 0; p < kPlanes; ++p) {
            to[p][0] = frag[((int64_t)r * kPlanes + p) * 64];
            to[p][1] = frag[((int64_t)r * kPlanes + p) * 64 + 32];
        }
    };
    if constexpr (RB > 0)
#pragma unroll
        for (int r = 0; r < RB; ++r) factor(r, f[r]);
    const T* x = (const T*)a.x + (int64_t)i * a.x_ws + c;
    T* y = (T*)a.y + (int64_t)i * a.rows * a.h + c;
    Raw8<T> next[MB][2];
    auto fetch = [&](uint32_t b, int stage) {
        if constexpr (RB > 0) {
            const uint4* from = tt + (int64_t)b * (RB * kPlanes * 32);
            const int have = b < b1 ? (b + MB <= b1 ? STAGE : RB * kPlanes * 32) : 0;
#pragma unroll
            for (int e = threadIdx.x; e < STAGE; e += 256)
                if (e < have) copy16(stages + stage * STAGE + e, from + e, true);
        }
        if (a.x) {
#pragma unroll
            for (int q = 0; q < MB; ++q)
#pragma unroll
                for (int half = 0; half < 2; ++half) {
                    const uint32_t j = (b + q) * 16 + half * 8 + g;
                    const bool in = b + q < b1 && j < a.rows && c < a.h;
                    const T* from = in ? x + (int64_t)j * a.x_rs : (const T*)a.x;
                    if constexpr (VEC) {
#pragma unroll
                        for (int v = 0; v < S16; ++v)
                            copy16(ring_at<SLOTS>(smem, stage, (q * 2 + half) * S16 + v), reinterpret_cast<const char*>(from) + 16 * v, in);
                    } else {
                        next[q][half] = raw_columns<T, false>(from - c, c, in ? a.h : 0);
                    }
                }
        }
        copies_commit();
    };
    if constexpr (VEC) {
        for (int s = 0; s < kStages - 1; ++s) fetch(b0 + s * MB, s);
    } else {
        fetch(b0, 0);
    }
    int stage = 0;
    for (uint32_t b = b0; b < b1; b += MB) {
        copies_wait<VEC ? kStages - 2 : 0>();
        __syncthreads();
        Raw8<T> base[MB][2] = {};
        if (a.x)
#pragma unroll
            for (int q = 0; q < MB; ++q)
#pragma unroll
                for (int half = 0; half < 2; ++half) {
                    if constexpr (VEC) base[q][half] = ring_raw<SLOTS, T>(smem, stage, (q * 2 + half) * S16);
                    else base[q][half] = next[q][half];
                }
        const uint4* here = stages + stage * STAGE + lane;
        if constexpr (VEC) fetch(b + (kStages - 1) * MB, stage == 0 ? kStages - 1 : stage - 1);
        else fetch(b + MB, stage + 1 == kStages ? 0 : stage + 1);
        stage = stage + 1 == kStages ? 0 : stage + 1;
        if (!mine) continue;
        float acc[MB][4][4] = {};
#pragma unroll(RB ? RB : 1)
        for (int r = 0; r < ranks; ++r) {
            uint4 w[MB][kPlanes];
            if constexpr (RB == 0) factor(r, f[0]);
#pragma unroll
            for (int q = 0; q < MB; ++q)
#pragma unroll
                for (int p = 0; p < kPlanes; ++p) w[q][p] = RB ? here[((q * RB + r) * kPlanes + p) * 32] : tt[((int64_t)(b * ranks + r) * kPlanes + p) * 32 + lane];
            float d[MB][4][4] = {};
            auto& sum = RB == 1 ? acc : d;  // (a sum grows for the products of 16 rank indices only)
#pragma unroll
            for (int both = kPlanes - 1; both >= 0; --both)
#pragma unroll
                for (int pt = 0; pt <= both; ++pt)
#pragma unroll
                    for (int q = 0; q < MB; ++q)
#pragma unroll
                        for (int k = 0; k < 4; ++k) {
                            const uint4 e = f[RB ? r : 0][both - pt][k >> 1];
                            mma(sum[q][k], w[q][pt].x, w[q][pt].y, w[q][pt].z, w[q][pt].w, k & 1 ? e.z : e.x, k & 1 ? e.w : e.y);
                        }
            if (RB != 1)
#pragma unroll
                for (int q = 0; q < MB; ++q)
#pragma unroll
                    for (int k = 0; k < 4; ++k)
#pragma unroll
                        for (int v = 0; v < 4; ++v) acc[q][k][v] += d[q][k][v];
        }
#pragma unroll
        for (int q = 0; q < MB; ++q)
#pragma unroll
            for (int half = 0; half < 2; ++half) {
                const uint32_t j = (b + q) * 16 + half * 8 + g;
                if ((MB > 1 && b + q >= b1) || j >= a.rows || c >= a.h) continue;
                float v[8];
                raw_floats<T>(base[q][half], v);
#pragma unroll
                for (int k = 0; k < 8; ++k) v[k] = fmaf(a.scale, acc[q][k >> 1][half * 2 + (k & 1)], v[k]);
                if (a.drop.on) drop8(a.drop, drop_words(a.drop, (uint32_t)c >> 3, j, a.drop.worker + i, call), v);
                T* to = y + (int64_t)j * a.h;
                if (VEC) {
                    store8<T>(to, v);
                } else {
#pragma unroll
                    for (int k = 0; k < 8; ++k)
                        if (c + k < a.h) to[k] = from_float<T>(v[k]);
                }
            }
    }
}

// A few rows to a worker: a lane per column, the factor read once in fp32 (32 workers of one row of 4096, rank 16: 3.7 us).
template <typename T, bool VEC>
__global__ void __launch_bounds__(256) adapter_up_few_kernel(const __grid_constant__ AdapterArgs a) {
    dependency_wait();
    const int lane = threadIdx.x & 31, c0 = (blockIdx.x * 8 + (int)(threadIdx.x >> 5)) * 32;
    const uint32_t i = blockIdx.y;
    const int c = c0 + lane;
    if (c0 >= a.h) return;
    const float* f = a.f.p + (int64_t)i * a.f.ws + c * a.f.sc;
    const float* t = a.t + (int64_t)i * a.rows * a.rank;
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
                    if (r < (int)a.rows && j + k < a.rank) acc[r] = fmaf(t[r * a.rank + j + k], w[k], acc[r]);
        }
    }
    const uint32_t call = drop_call(a.drop);
#pragma unroll
    for (int r = 0; r < kFewRows; ++r) {
        if (r >= (int)a.rows) break;
        float v = a.scale * acc[r];
        if (c < a.h && a.x) v += to_float(__ldg((const T*)a.x + (int64_t)i * a.x_ws + (int64_t)r * a.x_rs + c));
        if (a.drop.on) {
            const uint32_t bits = drop_bits(a.drop, (uint32_t)c >> 3, r, a.drop.worker + i, call);
            v = (bits >> (c & 7)) & 1u ? v * a.drop.factor : 0.0f;
        }
        if (c < a.h) ((T*)a.y)[((int64_t)i * a.rows + r) * a.h + c] = from_float<T>(v);
    }
}

// ---- outer -----------------------------------------------------------------------------------------------------------------

// A CTA per 256 columns, 8 NT rank indices and chunk of a worker's rows: four warps side by side, two that share out the blocks of 16 rows
// and join their sums. A lane takes eight neighbours of four rows; pairs of rows become the operand's pairs by byte permutes. The side by
// side warps share t, which passes through shared memory. Bound by instructions, as down: 8 workers of 2048 rows of 4096 in fp16, rank 16,
// 134 MB, 77 us, 98 with dropout; of 1024 rows in fp32 70 and 84.
constexpr int kOuterColumns = 256;
template <typename T, bool VEC, int NT>
__host__ __device__ constexpr int outer_ring() { return VEC ? kStages * 4 * (int)sizeof(Raw8<T>) * 256 : 0; }
template <typename T, bool VEC, int NT>
__host__ __device__ constexpr int outer_shared() {
    const int rings = outer_ring<T, VEC, NT>() + kStages * 2 * NT * kPlanes * 256, join = 4 * 4 * NT * 4 * 32 * 4;
    return rings > join ? rings : join;
}
template <typename T, bool VEC, int NT>
__global__ void __launch_bounds__(256) adapter_outer_kernel(const __grid_constant__ AdapterArgs a) {
    extern __shared__ __align__(16) char smem[];
    constexpr int PX = Planes<T>::count, S16 = (int)sizeof(Raw8<T>) / 16, SLOTS = 4 * S16;
    dependency_wait();
    const int lane = threadIdx.x & 31, warp = threadIdx.x >> 5, g = lane >> 2, t = lane & 3, side = warp & 3, turn = warp >> 2;
    const uint32_t i = blockIdx.y / a.chunks, chunk = blockIdx.y - i * a.chunks;
    const int groups = rank_groups(a.rank), column = blockIdx.x / groups, group = blockIdx.x - column * groups, n0 = group * NT;
    const int c = column * kOuterColumns + side * 64 + 8 * g;
    const uint32_t blocks = (a.rows + 15) / 16;
    const uint32_t s0 = (uint32_t)((uint64_t)blocks * chunk / a.chunks), s1 = (uint32_t)((uint64_t)blocks * (chunk + 1) / a.chunks);
    const uint32_t call = drop_call(a.drop);
    const T* x = (const T*)a.x + (int64_t)i * a.x_ws;
    const uint4* tt = reinterpret_cast<const uint4*>(a.t_outer) + i * t_outer_words(a.rows, a.rank) + (int64_t)group * blocks * (NT * kPlanes * 16);
    uint4* stages = reinterpret_cast<uint4*>(smem + outer_ring<T, VEC, NT>());
    constexpr int STAGE = 2 * NT * kPlanes * 16;  // words of 16 bytes: the fragments of the two blocks of rows of a step
    float acc[4][NT][4] = {};
    Raw8<T> next[4];
    auto fetch = [&](uint32_t s, int stage) {  // s: the warp's block of rows
#pragma unroll
        for (int r = 0; r < 4; ++r) {
            const uint32_t j = s * 16 + 4 * t + r;
            const bool there = s < s1 && j < a.rows && c < a.h;
            const T* from = x + (int64_t)(there ? j : 0) * a.x_rs;
            if constexpr (VEC) {
#pragma unroll
                for (int q = 0; q < S16; ++q)
                    copy16(ring_at<SLOTS>(smem, stage, r * S16 + q), there ? reinterpret_cast<const char*>(from + c) + 16 * q : a.x, there);
            } else {
                next[r] = raw_columns<T, false>(from, c, there ? a.h : 0);
            }
        }
    };
    auto fetch_shared = [&](uint32_t s, int stage) {  // s: the first block of rows of the step
        const uint4* from = tt + (int64_t)s * (STAGE / 2);
        const int have = s < s1 ? (s + 2 <= s1 ? STAGE : STAGE / 2) : 0;
#pragma unroll
        for (int e = threadIdx.x; e < STAGE; e += 256)
            if (e < have) copy16(stages + stage * STAGE + e, from + e, true);
        copies_commit();
    };
    if constexpr (VEC) {
        for (int s = 0; s < kStages - 1; ++s) {
            fetch(s0 + turn + 2 * s, s);
            fetch_shared(s0 + 2 * s, s);
        }
    } else {
        fetch(s0 + turn, 0);
        for (int s = 0; s < kStages - 1; ++s) fetch_shared(s0 + 2 * s, s);
    }
    int stage = 0;
    for (uint32_t first = s0; first < s1; first += 2) {
        copies_wait<kStages - 2>();
        __syncthreads();
        const uint32_t s = first + turn;
        const int behind = stage == 0 ? kStages - 1 : stage - 1;
        uint32_t w[4][PX][4];
#pragma unroll
        for (int r = 0; r < 4; ++r) {
            Raw8<T> now;
            if constexpr (VEC) now = ring_raw<SLOTS, T>(smem, stage, r * S16);
            else now = next[r];
            uint4 u = {};
            if (a.drop.on) u = drop_words(a.drop, (uint32_t)c >> 3, s * 16 + 4 * t + r, a.drop.worker + i, call);
            raw_planes<T>(now, a.drop, u, w[r]);
        }
        if constexpr (VEC) fetch(s + 2 * (kStages - 1), behind);
        else fetch(s + 2, 0);
        fetch_shared(first + 2 * (kStages - 1), behind);
        const uint2* here = reinterpret_cast<const uint2*>(stages + stage * STAGE + turn * (STAGE / 2)) + lane;
        stage = stage + 1 == kStages ? 0 : stage + 1;
        if (s >= s1) continue;
        uint32_t e[4][PX][4];
#pragma unroll
        for (int k = 0; k < 4; ++k)
#pragma unroll
            for (int px = 0; px < PX; ++px)
#pragma unroll
                for (int pair = 0; pair < 4; ++pair)
                    e[k][px][pair] = __byte_perm(w[pair & 2][px][k], w[(pair & 2) + 1][px][k], pair & 1 ? 0x7632 : 0x5410);
#pragma unroll
        for (int q = 0; q < NT; ++q) {
            uint2 f[kPlanes];
#pragma unroll
            for (int p = 0; p < kPlanes; ++p) f[p] = here[(q * kPlanes + p) * 32];
#pragma unroll
            for (int k = 0; k < 4; ++k) {
                float d[4];
                bool start = true;
#pragma unroll
                for (int both = kPlanes - 1; both >= 0; --both)
#pragma unroll
                    for (int px = 0; px < PX; ++px) {
                        const int p = both - px;
                        if (p < 0) break;
                        if (start) mma_first(d, e[k][px][0], e[k][px][1], e[k][px][2], e[k][px][3], f[p].x, f[p].y);
                        else mma(d, e[k][px][0], e[k][px][1], e[k][px][2], e[k][px][3], f[p].x, f[p].y);
                        start = false;
                    }
#pragma unroll
                for (int v = 0; v < 4; ++v) acc[k][q][v] += d[v];
            }
        }
    }
    copies_wait<0>();
    __syncthreads();  // the rings' memory is taken over
    float* joined = reinterpret_cast<float*>(smem) + side * 4 * NT * 4 * 32 + lane;
    if (turn == 1)
#pragma unroll
        for (int k = 0; k < 4; ++k)
#pragma unroll
            for (int q = 0; q < NT; ++q)
#pragma unroll
                for (int v = 0; v < 4; ++v) joined[((k * NT + q) * 4 + v) * 32] = acc[k][q][v];
    __syncthreads();
    if (turn == 1) return;
    const float scale = a.scale * (a.drop.on ? a.drop.factor : 1.0f);
#pragma unroll
    for (int k = 0; k < 4; ++k)
#pragma unroll
        for (int q = 0; q < NT; ++q)
#pragma unroll
            for (int v = 0; v < 4; ++v) acc[k][q][v] = scale * (acc[k][q][v] + joined[((k * NT + q) * 4 + v) * 32]);
    // a lane holds columns c ... c + 7 of two neighbouring rank indices
    float* out = a.out + (int64_t)blockIdx.y * a.rank * a.h;
    const bool ranks_packed = a.f.sj == 1, aligned = (reinterpret_cast<uintptr_t>(out) & 15u) == 0;
#pragma unroll
    for (int q = 0; q < NT; ++q) {
        const int j = (n0 + q) * 8 + 2 * t;
        if (j >= a.rank) break;
        if (ranks_packed) {
#pragma unroll
            for (int k = 0; k < 8; ++k) {
                if (c + k >= a.h) break;
                float* at = out + (int64_t)(c + k) * a.f.sc + j;
                if (aligned && !(a.rank & 1)) {
                    *reinterpret_cast<float2*>(at) = make_float2(acc[k >> 1][q][(k & 1) * 2], acc[k >> 1][q][(k & 1) * 2 + 1]);
                } else {
                    at[0] = acc[k >> 1][q][(k & 1) * 2];
                    if (j + 1 < a.rank) at[1] = acc[k >> 1][q][(k & 1) * 2 + 1];
                }
            }
        } else {
#pragma unroll
            for (int r = 0; r < 2; ++r) {
                if (j + r >= a.rank) break;
                float* at = out + (int64_t)(j + r) * a.f.sj + c;
                if (aligned && !(a.h & 3)) {
#pragma unroll
                    for (int k = 0; k < 8; k += 4)
                        if (c + k < a.h)
                            *reinterpret_cast<float4*>(at + k) = make_float4(acc[k >> 1][q][r], acc[k >> 1][q][2 + r], acc[(k >> 1) + 1][q][r],
                                                                             acc[(k >> 1) + 1][q][2 + r]);
                } else {
#pragma unroll
                    for (int k = 0; k < 8; ++k)
                        if (c + k < a.h) at[k] = acc[k >> 1][q][(k & 1) * 2 + r];
                }
            }
        }
    }
}

// A few rows to a worker: a lane per column, bound by the gradient that it writes (8 workers of four rows of 4096, rank 16, 2.1 MB each: 4 us).
template <typename T>
__global__ void __launch_bounds__(256) adapter_outer_few_kernel(const __grid_constant__ AdapterArgs a) {
    dependency_wait();
    const int c = blockIdx.x * 256 + threadIdx.x;
    const uint32_t i = blockIdx.y, call = drop_call(a.drop);
    if (c >= a.h) return;
    float v[kFewRows] = {};
#pragma unroll
    for (int r = 0; r < kFewRows; ++r) {
        if (r >= (int)a.rows) break;
        v[r] = to_float(__ldg((const T*)a.x + (int64_t)i * a.x_ws + (int64_t)r * a.x_rs + c));
        if (a.drop.on) {
            const uint32_t bits = drop_bits(a.drop, (uint32_t)c >> 3, r, a.drop.worker + i, call);
            v[r] = (bits >> (c & 7)) & 1u ? v[r] * a.drop.factor : 0.0f;
        }
    }
    const float* t = a.t + (int64_t)i * a.rows * a.rank;
    float* out = a.out + (int64_t)i * a.rank * a.h;
    for (int j = 0; j < a.rank; ++j) {
        float s = 0.0f;
#pragma unroll
        for (int r = 0; r < kFewRows; ++r)
            if (r < (int)a.rows) s = fmaf(t[r * a.rank + j], v[r], s);
        out[j * a.f.sj + c * a.f.sc] = a.scale * s;
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
constexpr int kSms = 148;  // SMs of a B200, for which launches are laid out

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

// Whether a worker's rows are few enough for the kernels that read the factor as it lies: with a tile of 16 rows of which four are
// there, three quarters of the products are of zeros, and the fragments are written and read again for them. 32 workers, 4096 x 4096, rank
// 16, each its own factors: 9 us for one row, 15 for four; with fragments 23 for five.
bool few(const AdapterShape& z) { return z.rows <= kFewRows; }

// Whether the products run on tcgen05.mma, whose tiles are of 128 rows. Forward and backward of 8 workers' 4096 x 4096 in bfloat16, device time in
// us with it and without: rank 16 and 64 rows 55 and 44, 128 rows 59 and 65, 512 rows 101 and 148; rank 32 and 64 rows 66 and 54, 96 rows 69
// and 77, 512 rows 118 and 199; rank 64 and 64 rows 98 and 116, 512 rows 155 and 361; rank 128 and 64 rows 122 and 141, 512 rows 224 and 643.
// With few tiles on the whole device mma.sync stays ahead for longer: one worker's 128 rows at rank 16 take 52 and 40.
bool on_tensor(const AdapterShape& z, int32_t type) {
    const int r = tensor::padded_rank(z.rank);
    return type == kTypeBF16 && z.rows >= (r == 16 ? 128 : r == 32 ? 96 : 64);
}

// The number of parts, of 1 ... most, at which the slowest of `slots` places ends first: waves of tiles * parts CTAs, each a part's
// share of `work` and `fixed` more. join: what a part more of a tile costs the whole device afterwards, if there are several (and a
// launch, 3); all in steps of a CTA.
int64_t parts_of(int64_t tiles, int64_t slots, int64_t work, double fixed, int64_t most, bool powers, double join = 0.0) {
    int64_t best = 1;
    double least = 0.0;
    for (int64_t c = 1; c <= most && c <= work; c = powers ? 2 * c : c + 1) {
        const double cost = (double)((tiles * c + slots - 1) / slots) * ((double)((work + c - 1) / c) + fixed) +
                            (join > 0.0 && c > 1 ? 3.0 + join * (double)(tiles * c) : 0.0);
        if (c == 1 || cost < least * 0.999) best = c, least = cost;
    }
    return best;
}

// Chunks of a worker's rows: as many as give each SM about two CTAs, of 64 rows at least.
uint32_t outer_chunks(const AdapterShape& z, int64_t h, int32_t type) {
    if (few(z)) return 1;
    // (partial sums of 64 ranks and 256 columns, 64 KB written and read: 26 ns at 5 TB/s, here 0.05 steps; a step takes 0.7 us at rank 16 and
    // 0.9 at rank 64, so chunks are few rather than many. 16384 rows of 8192 at rank 128: 117 us with one chunk, 127 and 43 for the join with
    // two; one worker's 512 rows of 1024 at rank 64: 11, 7.4 and 2.3 with eight)
    if (on_tensor(z, type))
        return (uint32_t)parts_of((h + 255) / 256 * z.n * tensor::groups_of(z.rank), kSms, (z.rows + 63) / 64, 4.0,
                                  std::min<int64_t>(65535 / z.n, 8), false, 0.05 * std::min(z.rank, 64) / 64);
    const int64_t tiles = (h + kOuterColumns - 1) / kOuterColumns * rank_groups(z.rank) * z.n;
    int64_t c = (kSms * 2 + tiles - 1) / tiles;
    const int64_t most = (z.rows + 63) / 64;
    if (c > most) c = most;
    if (c > 65535 / z.n) c = 65535 / z.n;
    return (uint32_t)(c < 1 ? 1 : c);
}
int64_t outer_floats(const AdapterShape& z, int64_t h, bool sum_workers, int32_t type) {
    const uint32_t c = outer_chunks(z, h, type);
    return c == 1 && (!sum_workers || z.n == 1) ? 0 : (int64_t)z.n * c * z.rank * h;
}

template <int V>
using Int = std::integral_constant<int, V>;
template <typename F>
int by_type(int32_t type, F f) {
    return type == kTypeF32 ? f(float()) : type == kTypeBF16 ? f(__nv_bfloat16()) : f(__half());
}
int launched(cudaError_t e, const char* what) { return e == cudaSuccess ? COMPAMS_OK : cuda_fail(e, what); }

// Lets a kernel have more than 48 KB of shared memory: asked once for every kernel and device (a kernel's size is always the same).
cudaError_t allow_shared(const void* kernel, size_t bytes) {
    static std::atomic<uint64_t> known[1024];
    int device = 0;
    cudaError_t e = cudaGetDevice(&device);
    if (e != cudaSuccess) return e;
    const uint64_t key = (uint64_t)(uintptr_t)kernel ^ (uint64_t)(device + 1) << 56;
    std::atomic<uint64_t>& slot = known[(key * 0x9E3779B97F4A7C15ull) >> 54];
    if (slot.load(std::memory_order_relaxed) == key) return cudaSuccess;
    e = cudaFuncSetAttribute(kernel, cudaFuncAttributeMaxDynamicSharedMemorySize, (int)bytes);
    if (e == cudaSuccess) slot.store(key, std::memory_order_relaxed);
    return e;
}

// A launch behind another of the same call (or the first), with dynamic shared memory and a cluster along x.
template <typename... KArgs, typename... Args>
cudaError_t launch_sized(void (*kernel)(KArgs...), dim3 grid, int threads, int cluster, size_t shared, bool first, cudaStream_t stream,
                         Args... args) {
    if (shared > 48 * 1024) {
        const cudaError_t e = allow_shared((const void*)kernel, shared);
        if (e != cudaSuccess) return e;
    }
    cudaLaunchConfig_t cfg = {};
    cfg.gridDim = grid;
    cfg.blockDim = dim3(threads);
    cfg.dynamicSmemBytes = shared;
    cfg.stream = stream;
    cudaLaunchAttribute attr[2];
    int count = 0;
    if (!first) {
        attr[count].id = cudaLaunchAttributeProgrammaticStreamSerialization;
        attr[count++].val.programmaticStreamSerializationAllowed = 1;
    }
    if (cluster > 1) {
        attr[count].id = cudaLaunchAttributeClusterDimension;
        attr[count].val.clusterDim.x = (unsigned)cluster;
        attr[count].val.clusterDim.y = 1;
        attr[count++].val.clusterDim.z = 1;
    }
    cfg.attrs = attr;
    cfg.numAttrs = count;
    return cudaLaunchKernelEx(&cfg, kernel, static_cast<KArgs>(args)...);
}

template <typename... KArgs, typename... Args>
cudaError_t launch_next(void (*kernel)(KArgs...), dim3 grid, int cluster, size_t shared, bool first, cudaStream_t stream, Args... args) {
    return launch_sized(kernel, grid, 256, cluster, shared, first, stream, args...);
}

// Where t goes to and comes from: fp32, and the operands of up and outer.
struct Low {
    float* t;
    uint4* up;
    uint2* outer;
};

AdapterArgs arguments(const AdapterShape& z, Rows x, int64_t h, const Low& low, float scale, const Drop& d) {
    AdapterArgs a = {};
    a.x = x.p; a.x_ws = x.worker_stride; a.x_rs = x.row_stride; a.rows = (uint32_t)z.rows;
    a.t = low.t; a.t_up = low.up; a.t_outer = low.outer;
    a.h = (int32_t)h; a.rank = z.rank; a.scale = scale; a.drop = d;
    return a;
}

template <typename F>
int by_rank(const AdapterShape& z, F f) {
    const int r = tensor::padded_rank(z.rank);
    return r == 16 ? f(Int<16>()) : r == 32 ? f(Int<32>()) : f(Int<64>());
}

// A map of x for boxes of 64 columns and `box` rows, in the 128-byte swizzle; false where TMA cannot address x.
bool box_map(CUtensorMap* map, Rows x, const AdapterShape& z, int64_t h, uint32_t box) {
    *map = {};
    if (h % 8 != 0 || !x.aligned() || x.row_stride < h || (z.n > 1 && x.worker_stride < 1) || x.row_stride >= (int64_t)1 << 38 ||
        x.worker_stride >= (int64_t)1 << 38)
        return false;
    // the encoder is the driver's; it is asked for once
    using Encode = decltype(&cuTensorMapEncodeTiled);
    static const Encode encode = [] {
        void* f = nullptr;
        cudaDriverEntryPointQueryResult found;
        if (cudaGetDriverEntryPoint("cuTensorMapEncodeTiled", &f, cudaEnableDefault, &found) != cudaSuccess || found != cudaDriverEntryPointSuccess)
            f = nullptr;
        return (Encode)f;
    }();
    if (!encode) return false;
    const cuuint64_t size[3] = {(cuuint64_t)h, (cuuint64_t)z.rows, (cuuint64_t)z.n};
    const cuuint64_t stride[2] = {(cuuint64_t)x.row_stride * 2, (cuuint64_t)(z.n > 1 ? x.worker_stride : x.row_stride * z.rows) * 2};
    const cuuint32_t extent[3] = {64, box, 1}, every[3] = {1, 1, 1};
    return encode(map, CU_TENSOR_MAP_DATA_TYPE_BFLOAT16, 3, const_cast<void*>(x.p), size, stride, extent, every, CU_TENSOR_MAP_INTERLEAVE_NONE,
                  CU_TENSOR_MAP_SWIZZLE_128B, CU_TENSOR_MAP_L2_PROMOTION_L2_256B, CU_TENSOR_MAP_FLOAT_OOB_FILL_NONE) == CUDA_SUCCESS;
}

// Tries of a wait in the kernels on tcgen05.mma.
std::atomic<uint32_t> wait_tries{tensor::kTries};

// The three products on tcgen05.mma; the images stand where the fragments do.
int tensor_prepare(const AdapterShape& z, bool shared, Factor down, int64_t down_h, void* down_image, Factor up, int64_t up_h, void* up_image,
                   const float* t, void* t_image, cudaStream_t stream) {
    tensor::PrepareArgs p = {down, up, (char*)down_image, (char*)up_image, t, (char*)t_image, (int32_t)down_h, (int32_t)up_h, z.rank,
                             (uint32_t)z.rows, 0, 0, 0, 0, 0, 0, shared};
    const int64_t r = tensor::padded_rank(z.rank), groups = tensor::groups_of(z.rank);
    p.down_blocks = (uint32_t)((down_h + 127) / 128 * 2); p.up_blocks = (uint32_t)((up_h + 127) / 128); p.t_blocks = (uint32_t)((z.rows + 63) / 64);
    const int64_t down_count = down_image ? groups * p.down_blocks * 8 * r : 0, up_count = up_image ? groups * p.up_blocks * 16 * r : 0;
    const int64_t t_count = t_image ? groups * p.t_blocks * 8 * r : 0;
    const int64_t ctas = (down_count + up_count + t_count + 255) / 256;
    if (ctas > 0x00ffffff) return COMPAMS_ERR_TOO_LARGE;
    p.down_count = (uint32_t)down_count; p.up_count = (uint32_t)up_count; p.t_count = (uint32_t)t_count;
    const uint32_t workers = shared && !t_image ? 1 : (uint32_t)z.n;
    return by_rank(z, [&](auto v) {
        return launched(launch_next(tensor::prepare_kernel<decltype(v)::value>, dim3((uint32_t)ctas, workers), 1, 0, true, stream, p),
                        "adapter_prepare");
    });
}

int tensor_down(Low low, Rows x, const AdapterShape& z, int64_t h, bool shared, const uint4* image, float scale, const Drop& d,
                cudaStream_t stream) {
    tensor::Args a = {};
    a.x = x.p; a.x_ws = x.worker_stride; a.x_rs = x.row_stride; a.image = (const char*)image; a.image_ws = shared ? 0 : tensor::down_image(h, z.rank);
    a.t_up = (char*)low.up; a.t_outer = (char*)low.outer; a.out = low.t; a.rows = (uint32_t)z.rows; a.h = (int32_t)h; a.rank = z.rank;
    a.tries = wait_tries.load(std::memory_order_relaxed); a.scale = scale; a.drop = d;
    return by_rank(z, [&](auto v) {
        constexpr int R = decltype(v)::value;
        using P = tensor::Pipe<R, false>;
        a.tiles = (a.rows + P::kRows - 1) / P::kRows;
        const uint32_t groups = (uint32_t)tensor::groups_of(z.rank);
        a.split = (int32_t)parts_of((int64_t)a.tiles * z.n * groups, kSms, (h + P::kStep - 1) / P::kStep, 4.0, tensor::kMostSplit, true);
        const uint64_t ctas = (uint64_t)a.tiles * z.n * a.split;
        if (ctas > 0x7fffffffu) return (int)COMPAMS_ERR_TOO_LARGE;
        CUtensorMap map;
        auto kernel = box_map(&map, x, z, h, 128) ? tensor::down_kernel<R, true> : tensor::down_kernel<R, false>;
        return launched(launch_sized(kernel, dim3((uint32_t)ctas, groups), tensor::kThreads, a.split, P::kShared, false, stream, a, map),
                        "adapter_down");
    });
}

int tensor_up(void* y, Rows base, Low low, const AdapterShape& z, int64_t h, bool shared, const uint4* image, float scale, const Drop& d,
              cudaStream_t stream) {
    tensor::UpArgs a = {};
    a.base = base.p; a.y = y; a.image = (const char*)image; a.t_up = (const char*)low.up; a.base_ws = base.worker_stride;
    a.base_rs = base.row_stride; a.image_ws = shared ? 0 : tensor::up_image(h, z.rank); a.rows = (uint32_t)z.rows; a.h = (int32_t)h; a.rank = z.rank;
    a.tries = wait_tries.load(std::memory_order_relaxed); a.scale = scale; a.drop = d;
    const bool several = tensor::groups_of(z.rank) > 1, vec = h % 8 == 0 && (!base.p || base.aligned()) && packed(y, z.rows, h, base.type).aligned();
    return by_rank(z, [&](auto v) {
        constexpr int R = decltype(v)::value;
        auto go = [&](auto g) {
            constexpr bool GROUPS = decltype(g)::value;
            using U = tensor::Up<R, GROUPS>;
            const int64_t columns = (h + U::kColumns - 1) / U::kColumns, blocks = (z.rows + 127) / 128;
            a.chunks = (uint32_t)parts_of(columns * z.n, GROUPS ? kSms : 2 * kSms, blocks, 0.5, 65535 / z.n, false);
            auto kernel = vec ? tensor::up_kernel<R, true, GROUPS> : tensor::up_kernel<R, false, GROUPS>;
            return launched(launch_next(kernel, dim3((uint32_t)columns, (uint32_t)z.n * a.chunks), 1, U::kShared, false, stream, a), "adapter_up");
        };
        if constexpr (R == 64)
            if (several) return go(Int<1>());
        return go(Int<0>());
    });
}

int tensor_outer(const AdapterArgs& b, Rows x, Low low, const AdapterShape& z, int64_t h, bool first, cudaStream_t stream) {
    tensor::Args a = {};
    a.x = b.x; a.x_ws = b.x_ws; a.x_rs = b.x_rs; a.image = (const char*)low.outer; a.image_ws = tensor::t_outer_image(z.rows, z.rank); a.out = b.out;
    a.sj = b.f.sj; a.sc = b.f.sc; a.rows = b.rows; a.h = b.h; a.rank = b.rank; a.chunks = b.chunks; a.scale = b.scale; a.drop = b.drop;
    a.tries = wait_tries.load(std::memory_order_relaxed);
    return by_rank(z, [&](auto v) {
        constexpr int R = decltype(v)::value;
        CUtensorMap map;
        auto kernel = box_map(&map, x, z, h, 64) ? tensor::outer_kernel<R, true> : tensor::outer_kernel<R, false>;
        const dim3 grid((uint32_t)((h + 255) / 256), (uint32_t)z.n * a.chunks, (uint32_t)tensor::groups_of(z.rank));
        return launched(launch_sized(kernel, grid, tensor::kThreads, 1, tensor::Pipe<R, true>::kShared, first, stream, a, map),
                        "adapter_outer");
    });
}

int prepare(const AdapterShape& z, bool shared, Factor down, int64_t down_h, uint4* down_frag, Factor up, int64_t up_h, uint4* up_frag,
            const float* t, uint2* t_outer, int32_t type, cudaStream_t stream) {
    if (on_tensor(z, type)) return tensor_prepare(z, shared, down, down_h, down_frag, up, up_h, up_frag, t, t_outer, stream);
    PrepareArgs p = {down, up, down_frag, up_frag, t, t_outer, (int32_t)down_h, (int32_t)up_h, z.rank, (uint32_t)z.rows, 0, 0, 0, shared};
    if (down_frag) p.down_count = (uint32_t)(down_blocks(down_h) * rank_tiles(z.rank));
    if (up_frag) p.up_count = (uint32_t)((up_h + kUpColumns - 1) / kUpColumns * ((z.rank + 15) / 16));
    if (t_outer) p.t_count = (uint32_t)((z.rows + 15) / 16 * rank_tiles(z.rank));
    const uint64_t ctas = ((uint64_t)p.down_count + p.up_count + p.t_count + 7) / 8;
    if (ctas > 0x0fffffffu) return COMPAMS_ERR_TOO_LARGE;
    const uint32_t workers = shared && !t_outer ? 1 : (uint32_t)z.n;
    return launched(launch_next(adapter_prepare_kernel, dim3((uint32_t)ctas, workers), 1, 0, true, stream, p), "adapter_prepare");
}

int down(Low low, Rows x, const AdapterShape& z, int64_t h, bool shared, Factor f, const uint4* frag, float scale, const Drop& d,
         cudaStream_t stream) {
    if (on_tensor(z, x.type)) return tensor_down(low, x, z, h, shared, frag, scale, d, stream);
    AdapterArgs a = arguments(z, x, h, low, scale, d);
    a.out = low.t; a.f = f; a.frag = frag; a.frag_ws = shared ? 0 : down_frag_words(h, z.rank);
    const bool vec = h % 8 == 0 && x.aligned();
    return by_type(x.type, [&](auto t) {
        using T = decltype(t);
        if (!frag) {
            auto kernel = vec ? adapter_down_few_kernel<T, true> : adapter_down_few_kernel<T, false>;
            return launched(launch_next(kernel, dim3((uint32_t)z.rank, (uint32_t)z.n), 1, 0, true, stream, a), "adapter_down");
        }
        const uint32_t groups = rank_groups(z.rank);
        auto go = [&](auto kernel, int wk, int mt, int shared_bytes) {
            const int per = 16 * 8 * mt / wk;
            a.tiles = (a.rows + per - 1) / per;
            // columns shared out over as many CTAs (of a cluster) as give each SM two, four steps each at least
            const uint64_t tiles = (uint64_t)a.tiles * z.n * groups;
            const int64_t steps = (h + 32 * down_step<T>() - 1) / (32 * down_step<T>()) / wk;
            a.split = 1;
            while (a.split < 8 && tiles * a.split < 2 * kSms / mt && steps >= 8 * a.split) a.split *= 2;
            const uint64_t ctas = (uint64_t)a.tiles * z.n * a.split;
            if (ctas > 0x7fffffffu) return (int)COMPAMS_ERR_TOO_LARGE;
            return launched(launch_next(kernel, dim3((uint32_t)ctas, groups), a.split, shared_bytes, false, stream, a),
                            "adapter_down");
        };
        auto pick = [&](auto v, auto k, auto n, auto m) {
            constexpr bool V = decltype(v)::value;
            constexpr int WK = decltype(k)::value, NT = decltype(n)::value, MT = decltype(m)::value;
            return go(adapter_down_kernel<T, V, NT, WK, MT>, WK, MT, down_shared<T, V, NT, WK, MT>());
        };
        auto by_ranks = [&](auto v) {
            const int nt = group_tiles(z.rank);
            // Warps that share the rows' columns keep more loads on their way; warps of different rows share the fragments, which pays
            // for several groups of ranks in 16 bits and many rows. Both passes' kernels of 8 workers, 4096 columns, eight warps to the
            // rows / one: fp16, rank 128, 1024 rows 371 / 321 us, 512 rows 190 / 254 (of 1024 columns 117 / 114 and 63 / 59, of 8192 836 /
            // 596 and 420 / 459; rank 80 as 128); fp16, rank 16, 2048 rows 137 / 152, 512 rows 50 / 45; fp32, rank 64, 1024 rows 228 / 402.
            if constexpr (sizeof(T) == 2)
                if (z.rank > 64 && z.total() >= 8192) return pick(v, Int<1>(), Int<8>(), Int<2>());
            if (nt == 1) return pick(v, Int<8>(), Int<1>(), Int<1>());
            if (nt == 2) return pick(v, Int<8>(), Int<2>(), Int<1>());
            if (nt == 4) return pick(v, Int<8>(), Int<4>(), Int<1>());
            return pick(v, Int<8>(), Int<8>(), Int<1>());
        };
        return vec ? by_ranks(Int<1>()) : by_ranks(Int<0>());
    });
}

int up(void* y, Rows base, Low low, const AdapterShape& z, int64_t h, bool shared, Factor f, const uint4* frag, float scale, const Drop& d,
       cudaStream_t stream) {
    if (on_tensor(z, base.type)) return tensor_up(y, base, low, z, h, shared, frag, scale, d, stream);
    AdapterArgs a = arguments(z, base, h, low, scale, d);
    a.y = y; a.f = f; a.frag = frag; a.frag_ws = shared ? 0 : up_frag_words(h, z.rank);
    const bool vec = h % 8 == 0 && (!base.p || base.aligned()) && packed(y, z.rows, h, base.type).aligned();
    return by_type(base.type, [&](auto tt) {
        using T = decltype(tt);
        const uint32_t columns = (uint32_t)((h + 8 * kUpColumns - 1) / (8 * kUpColumns));
        if (!frag) {
            auto kernel = vec ? adapter_up_few_kernel<T, true> : adapter_up_few_kernel<T, false>;
            return launched(launch_next(kernel, dim3(columns, (uint32_t)z.n), 1, 0, false, stream, a), "adapter_up");
        }
        // row chunks: as many as give each SM about four CTAs
        const uint32_t blocks = (a.rows + 15) / 16, n = (uint32_t)z.n;
        uint64_t c = kSms * 4 / ((uint64_t)columns * n) + 1;
        if (c > blocks) c = blocks;
        if (c > 65535 / n) c = 65535 / n;
        a.tiles = (uint32_t)c;
        auto go = [&](auto v, auto r) {
            constexpr bool V = decltype(v)::value;
            constexpr int RB = decltype(r)::value;
            return launched(launch_next(adapter_up_kernel<T, V, RB>, dim3(columns, n * a.tiles), 1, up_shared<T, V, RB>(), false,
                                        stream, a),
                            "adapter_up");
        };
        auto by_ranks = [&](auto v) {
            const int ranks = (z.rank + 15) / 16;
            if (ranks == 1) return go(v, Int<1>());
            if (ranks == 2) return go(v, Int<2>());
            if constexpr (sizeof(T) == 2)
                if (ranks == 4) return go(v, Int<4>());
            return go(v, Int<0>());
        };
        return vec ? by_ranks(Int<1>()) : by_ranks(Int<0>());
    });
}

// out(j, c) at j * sj + c * sc of every worker's rank * h floats.
int outer(float* out, bool sum_workers, Rows x, Low low, const AdapterShape& z, int64_t h, int64_t sj, int64_t sc, float scale,
          const Drop& d, float* partial, bool first, cudaStream_t stream) {
    AdapterArgs a = arguments(z, x, h, low, scale, d);
    a.f = {nullptr, 0, sj, sc}; a.chunks = outer_chunks(z, h, x.type);
    const bool straight = outer_floats(z, h, sum_workers, x.type) == 0;
    a.out = straight ? out : partial;
    const int rc = by_type(x.type, [&](auto tt) {
        using T = decltype(tt);
        if (few(z))
            return launched(launch_next(adapter_outer_few_kernel<T>, dim3((uint32_t)((h + 255) / 256), (uint32_t)z.n), 1, 0, first, stream, a),
                            "adapter_outer");
        if (on_tensor(z, x.type)) return tensor_outer(a, x, low, z, h, first, stream);
        const int nt = group_tiles(z.rank);
        const uint64_t tiles = (uint64_t)((h + kOuterColumns - 1) / kOuterColumns) * rank_groups(z.rank);
        if (tiles > 0x7fffffffu) return (int)COMPAMS_ERR_TOO_LARGE;
        const bool vec = h % 8 == 0 && x.aligned();
        auto go = [&](auto v, auto m) {
            constexpr bool V = decltype(v)::value;
            constexpr int NT = decltype(m)::value;
            return launched(launch_next(adapter_outer_kernel<T, V, NT>, dim3((uint32_t)tiles, (uint32_t)z.n * a.chunks), 1,
                                        outer_shared<T, V, NT>(), first, stream, a),
                            "adapter_outer");
        };
        auto by_ranks = [&](auto v) {
            return nt == 1 ? go(v, Int<1>()) : nt == 2 ? go(v, Int<2>()) : nt == 4 ? go(v, Int<4>()) : go(v, Int<8>());
        };
        return vec ? by_ranks(Int<1>()) : by_ranks(Int<0>());
    });
    if (rc != COMPAMS_OK || straight) return rc;
    const int64_t len = z.rank * h;
    return launched(launch_next(adapter_join_kernel, dim3((uint32_t)((len + 255) / 256), sum_workers ? 1 : (uint32_t)z.n), 1, 0, false,
                                stream, (const float*)partial, out, len, sum_workers ? z.n * a.chunks : a.chunks),
                    "adapter_join");
}

bool float_aligned(const void* p) { return (reinterpret_cast<uintptr_t>(p) & 3u) == 0; }

// The workspace: fragments of the two factors, t (dt in the backward pass) as operands, and, in the backward pass, the forward pass's t
// as an operand of outer and the partial sums; offsets in bytes.
struct Places {
    int64_t down, up, t, t_up, t_outer, saved, partial, bytes;
};
Places places(const AdapterShape& z, bool shared, bool backward, bool sum_workers) {
    const int64_t factors = shared ? 1 : z.n;
    const bool frags = !few(z);
    Places p = {};
    int64_t at = 0;
    auto take = [&](int64_t bytes) {
        const int64_t here = at;
        at += (bytes + 255) / 256 * 256;
        return here;
    };
    // (the larger of the fragments and the images, so that the size does not depend on the type)
    auto either = [&](int64_t words, int64_t image) { return words * 16 > image ? words * 16 : image; };
    const int64_t dh = backward ? z.out : z.in, uh = backward ? z.in : z.out;
    if (frags) {
        p.down = take(factors * either(down_frag_words(dh, z.rank), tensor::down_image(dh, z.rank)));
        p.up = take(factors * either(up_frag_words(uh, z.rank), tensor::up_image(uh, z.rank)));
        p.t_up = take(z.n * either(t_up_words(z.rows, z.rank), tensor::t_up_image(z.rows, z.rank)));
    }
    if (frags && backward) {
        p.t_outer = take(z.n * either(t_outer_words(z.rows, z.rank), tensor::t_outer_image(z.rows, z.rank)));
        p.saved = take(z.n * either(t_outer_words(z.rows, z.rank), tensor::t_outer_image(z.rows, z.rank)));
    }
    p.t = take(backward && !frags ? (int64_t)z.total() * z.rank * 4 : 0);
    int64_t most = 0;
    if (backward)
        for (int32_t type : {kTypeF32, kTypeBF16})
            for (int64_t h : {z.in, z.out}) most = std::max(most, outer_floats(z, h, sum_workers, type));
    p.partial = take(most * 4);
    p.bytes = at;
    return p;
}

}  // namespace
}  // namespace compams

using namespace compams;

extern "C" {

int compams_adapter_status(int32_t* gave_up) {
    if (!gave_up) return COMPAMS_ERR_INVALID_ARG;
    cudaError_t e = cudaMemcpyFromSymbol(gave_up, tensor::gave_up, sizeof(int32_t));
    if (e == cudaSuccess && *gave_up) {
        const int32_t none = 0;
        e = cudaMemcpyToSymbol(tensor::gave_up, &none, sizeof(none));
    }
    return launched(e, "adapter_status");
}

int compams_adapter_wait_tries(int32_t tries) {
    if (tries < 0 || tries > (int32_t)tensor::kTries) return COMPAMS_ERR_INVALID_ARG;
    wait_tries.store((uint32_t)tries, std::memory_order_relaxed);
    return COMPAMS_OK;
}

int compams_adapter_workspace_bytes(size_t* bytes, int32_t n, int64_t rows, int64_t in, int64_t out, int32_t rank, int32_t shared,
                                    int32_t backward, int32_t sum_workers) {
    const AdapterShape z{n, rows, in, out, rank};
    if (!bytes || !z.ok()) return COMPAMS_ERR_INVALID_ARG;
    *bytes = (size_t)places(z, shared != 0 || n == 1, backward != 0, sum_workers != 0).bytes;
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
    if (!xin.strides_ok() || (base && !bin.strides_ok()) || a_worker_stride < 0 || a_row_stride < 0 || b_worker_stride < 0 || b_row_stride < 0 ||
        !x || !y || !t || !a || !b || !float_aligned(t) || !float_aligned(a) || !float_aligned(b) || !xin.element_aligned() ||
        !bin.element_aligned() || !packed(y, rows, out, type).element_aligned() || workspace_bytes < (size_t)at.bytes ||
        (at.bytes && !workspace) || (reinterpret_cast<uintptr_t>(workspace) & 15u))
        return COMPAMS_ERR_INVALID_ARG;
    const cudaStream_t stream = (cudaStream_t)cuda_stream;
    const Factor fa{a, a_worker_stride, a_row_stride, 1}, fb{b, b_worker_stride, 1, b_row_stride};
    char* work = (char*)workspace;
    Low low = {t, nullptr, nullptr};
    uint4 *down_frag = nullptr, *up_frag = nullptr;
    int rc = COMPAMS_OK;
    if (!few(z)) {
        down_frag = (uint4*)(work + at.down);
        up_frag = (uint4*)(work + at.up);
        low.up = (uint4*)(work + at.t_up);
        rc = prepare(z, shared, fa, in, down_frag, fb, out, up_frag, nullptr, nullptr, type, stream);
    }
    if (rc == COMPAMS_OK) rc = down(low, xin, z, in, shared, fa, down_frag, 1.0f, d, stream);
    if (rc == COMPAMS_OK) rc = up(y, bin, low, z, out, shared, fb, up_frag, scale, none, stream);
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
    if (!gin.strides_ok() || (x && !xin.strides_ok()) || a_worker_stride < 0 || a_row_stride < 0 || b_worker_stride < 0 || b_row_stride < 0 ||
        !dy || !a || !b || (da && !x) || (db && !t) || !workspace || workspace_bytes < (size_t)at.bytes ||
        (reinterpret_cast<uintptr_t>(workspace) & 15u) || !float_aligned(t) || !float_aligned(a) || !float_aligned(b) ||
        !float_aligned(da) || !float_aligned(db) || !xin.element_aligned() || !gin.element_aligned() ||
        !packed(dx, rows, in, type).element_aligned())
        return COMPAMS_ERR_INVALID_ARG;
    if (!dx && !da && !db) return COMPAMS_OK;
    const Factor fa{a, a_worker_stride, a_row_stride, 1}, fb{b, b_worker_stride, 1, b_row_stride};
    char* work = (char*)workspace;
    float* partial = (float*)(work + at.partial);
    Low low = {few(z) ? (float*)(work + at.t) : nullptr, nullptr, nullptr}, saved = {const_cast<float*>(t), nullptr, nullptr};
    uint4 *down_frag = nullptr, *up_frag = nullptr;
    int rc = COMPAMS_OK;
    bool first = true;
    if (!few(z)) {
        if (dx || da) down_frag = (uint4*)(work + at.down);
        if (dx) up_frag = (uint4*)(work + at.up);
        low.up = (uint4*)(work + at.t_up);
        if (da) low.outer = (uint2*)(work + at.t_outer);
        if (db) saved.outer = (uint2*)(work + at.saved);
        rc = prepare(z, shared, fb, out, down_frag, fa, in, up_frag, t, saved.outer, type, stream);
        first = false;
    }
    if (rc == COMPAMS_OK && (dx || da)) {
        rc = down(low, gin, z, out, shared, fb, down_frag, scale, none, stream);
        first = false;
    }
    if (rc == COMPAMS_OK && db) rc = outer(db, sum_workers, gin, saved, z, out, 1, rank, scale, none, partial, first, stream);
    if (rc == COMPAMS_OK && da) rc = outer(da, sum_workers, xin, low, z, in, in, 1, 1.0f, d, partial, false, stream);
    if (rc == COMPAMS_OK && dx) rc = up(dx, {nullptr, 0, 0, type}, low, z, in, shared, fa, up_frag, 1.0f, d, stream);
    return rc;
}

}  // extern "C"
