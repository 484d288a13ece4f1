// The adapters' three products on tcgen05.mma, for bfloat16 activations and ranks from 33 to 64, where mma.sync is bound by its own
// rate (550 TFLOP/s measured, a third of tcgen05's) instead of by memory.
//
// The planes of an fp32 operand are stacked along N: a tile of an activation, 128 x 64, is multiplied by [3 x 64] rows of planes at once, so
// it is an operand once and the planes' sums stand beside each other in tensor memory. Operands lie in shared memory in the
// 128-byte swizzle: rows of 128 bytes (64 elements), whose 16-byte chunk c lies at chunk c ^ (row % 8). down: the rows are the activation's
// and the sum runs along them (K-major); outer: the sum runs over the rows, the tile is read across them (MN-major), and t
// comes turned, [plane, rank][row].
//
// 256 threads copy (cp.async straight into the swizzle; where dropout masks an activation the thread that copied a chunk does so in place), a
// thread of a ninth warp copies the planes in bulk and issues the products; mbarriers pass the stages between them. The tensor cores cut
// their sums, so after every kFlush tiles of 64 the sums go to fp32 registers by rounded additions.
#pragma once

#include "rows.cuh"

namespace compams {
namespace {
namespace tensor {

constexpr int kRank = 64;                  // rank indices, padded
constexpr int kN = 3 * kRank;              // planes side by side
constexpr int kTileBytes = 128 * 128;      // 128 rows of 64 elements, or 64 rows of 128
constexpr int kPlanesBytes = kN * 128;     // planes: 192 rows of 64 elements
constexpr int kStageBytes = 2 * kTileBytes + kPlanesBytes;
constexpr int kStages = 4;
constexpr int kFlush = 8;                  // tiles between two additions to the registers
constexpr int kShared = 1024 + kStages * kStageBytes;
constexpr uint32_t kColumns = 512;         // of tensor memory: 2 x 192 used, a power of two taken

// ---- images of the fp32 operands in global memory, in the order of shared memory --------------------------------------------

// A factor for down: [64 columns][plane, rank][64 columns]; for up: [128 columns][plane 0, 1][column][rank]; bytes of a worker's.
__host__ __device__ inline int64_t down_image(int64_t h) { return (h + 63) / 64 * kPlanesBytes; }
__host__ __device__ inline int64_t up_image(int64_t h) { return (h + 127) / 128 * (2 * kTileBytes); }
// t for outer: [64 rows][plane, rank][row]; for up: [128 rows][plane 0, 1][row][rank].
__host__ __device__ inline int64_t t_outer_image(int64_t rows) { return (rows + 63) / 64 * kPlanesBytes; }
__host__ __device__ inline int64_t t_up_image(int64_t rows) { return (rows + 127) / 128 * (2 * kTileBytes); }

__device__ __forceinline__ uint32_t swizzled(uint32_t row, uint32_t chunk) { return row * 128u + ((chunk ^ (row & 7u)) << 4); }

// ---- instructions ----------------------------------------------------------------------------------------------------------

__device__ __forceinline__ uint32_t shared_address(const void* p) { return (uint32_t)__cvta_generic_to_shared(p); }

__device__ __forceinline__ void barrier_init(uint32_t bar, uint32_t count) {
    asm volatile("mbarrier.init.shared::cta.b64 [%0], %1;" ::"r"(bar), "r"(count) : "memory");
}
__device__ __forceinline__ void barrier_arrive(uint32_t bar) { asm volatile("mbarrier.arrive.shared::cta.b64 _, [%0];" ::"r"(bar) : "memory"); }
// Waits for the phase of this parity to end; gives up after a number of tries, each of which the hardware may hold for a while.
__device__ __forceinline__ bool barrier_wait(uint32_t bar, uint32_t parity) {
    uint32_t there = 0;
    for (int tries = 0; tries < (1 << 14) && !there; ++tries)
        asm volatile("{\n.reg .pred p;\nmbarrier.try_wait.parity.shared::cta.b64 p, [%1], %2;\nselp.u32 %0, 1, 0, p;\n}"
                     : "=r"(there)
                     : "r"(bar), "r"(parity)
                     : "memory");
    return there != 0u;
}
__device__ __forceinline__ void memory_alloc(uint32_t to, uint32_t columns) {  // a whole warp
    asm volatile("tcgen05.alloc.cta_group::1.sync.aligned.shared::cta.b32 [%0], %1;" ::"r"(to), "r"(columns) : "memory");
    asm volatile("tcgen05.relinquish_alloc_permit.cta_group::1.sync.aligned;" ::: "memory");
}
__device__ __forceinline__ void memory_free(uint32_t at, uint32_t columns) {
    asm volatile("tcgen05.dealloc.cta_group::1.sync.aligned.b32 %0, %1;" ::"r"(at), "r"(columns) : "memory");
}
__device__ __forceinline__ void fence_before() { asm volatile("tcgen05.fence::before_thread_sync;" ::: "memory"); }
__device__ __forceinline__ void fence_after() { asm volatile("tcgen05.fence::after_thread_sync;" ::: "memory"); }
__device__ __forceinline__ void fence_shared() { asm volatile("fence.proxy.async.shared::cta;" ::: "memory"); }

// Of an operand in the 128-byte swizzle that starts at a shared address. `along`: bytes to the next 64 elements along M or N of an
// MN-major operand; 8 rows of 128 bytes lie behind one another.
__device__ __forceinline__ uint64_t operand(uint32_t at, uint32_t along) {
    return (uint64_t)((at >> 4) & 0x3fffu) | (uint64_t)(along >> 4) << 16 | (uint64_t)(1024u >> 4) << 32 | (uint64_t)1 << 46 | (uint64_t)2 << 61;
}
// bf16 x bf16 -> fp32; M = 128; which operands are MN-major.
__host__ __device__ constexpr uint32_t instruction(int n, bool a_across, bool b_across) {
    return 1u << 4 | 1u << 7 | 1u << 10 | (a_across ? 1u : 0u) << 15 | (b_across ? 1u : 0u) << 16 | (uint32_t)(n >> 3) << 17 | (128u >> 4) << 24;
}
__device__ __forceinline__ void product(uint32_t d, uint64_t a, uint64_t b, uint32_t what, bool onto) {
    asm volatile("{\n.reg .pred p;\nsetp.ne.u32 p, %4, 0;\ntcgen05.mma.cta_group::1.kind::f16 [%0], %1, %2, %3, p;\n}" ::"r"(d), "l"(a), "l"(b),
                 "r"(what), "r"((uint32_t)onto)
                 : "memory");
}
__device__ __forceinline__ void products_done(uint32_t bar) {
    asm volatile("tcgen05.commit.cta_group::1.mbarrier::arrive::one.shared::cluster.b64 [%0];" ::"r"(bar) : "memory");
}
// 32 columns of a lane's row.
__device__ __forceinline__ void columns32(uint32_t at, float (&v)[32]) {
    uint32_t r[32];
    asm volatile(
        "tcgen05.ld.sync.aligned.32x32b.x32.b32 {%0,%1,%2,%3,%4,%5,%6,%7,%8,%9,%10,%11,%12,%13,%14,%15,%16,%17,%18,%19,%20,%21,%22,%23,%24,%25,"
        "%26,%27,%28,%29,%30,%31}, [%32];"
        : "=r"(r[0]), "=r"(r[1]), "=r"(r[2]), "=r"(r[3]), "=r"(r[4]), "=r"(r[5]), "=r"(r[6]), "=r"(r[7]), "=r"(r[8]), "=r"(r[9]), "=r"(r[10]),
          "=r"(r[11]), "=r"(r[12]), "=r"(r[13]), "=r"(r[14]), "=r"(r[15]), "=r"(r[16]), "=r"(r[17]), "=r"(r[18]), "=r"(r[19]), "=r"(r[20]),
          "=r"(r[21]), "=r"(r[22]), "=r"(r[23]), "=r"(r[24]), "=r"(r[25]), "=r"(r[26]), "=r"(r[27]), "=r"(r[28]), "=r"(r[29]), "=r"(r[30]),
          "=r"(r[31])
        : "r"(at));
#pragma unroll
    for (int k = 0; k < 32; ++k) v[k] = __uint_as_float(r[k]);
}
// Behind it the values are there.
__device__ __forceinline__ void columns_wait(float (&v)[32]) {
    asm volatile("tcgen05.wait::ld.sync.aligned;" ::: "memory");
#pragma unroll
    for (int k = 0; k < 32; ++k) asm volatile("" : "+f"(v[k]));
}

// Set where a wait gave up, which no size or input should bring about; the results of that call are then worthless.
__device__ int32_t gave_up;

// Eight planes' neighbours as a chunk of 16 bytes each.
__device__ __forceinline__ void planes8(const float (&v)[8], uint4 (&out)[3]) {
    uint32_t w[4][3];
#pragma unroll
    for (int q = 0; q < 4; ++q) split2<3>(v[2 * q], v[2 * q + 1], w[q]);
#pragma unroll
    for (int p = 0; p < 3; ++p) out[p] = make_uint4(w[0][p], w[1][p], w[2][p], w[3][p]);
}

// ---- prepare ---------------------------------------------------------------------------------------------------------------

struct PrepareArgs {
    Factor down, up;
    char *down_image, *up_image;  // may be null
    const float* t;
    char* t_image;  // t for outer; may be null
    int32_t down_h, up_h, rank;
    uint32_t rows, down_count, up_count, t_count;  // chunks of a worker's images, of one plane
    int32_t shared;
};
// A thread per chunk of 16 bytes.
__global__ void __launch_bounds__(256) prepare_kernel(const __grid_constant__ PrepareArgs a) {
    uint32_t at = blockIdx.x * 256 + threadIdx.x;
    float v[8];
    uint4 w[3];
    if (at < a.t_count) {  // [64 rows][8 rows][rank]: neighbouring threads read neighbouring ranks
        const uint32_t rank = at & 63u, c = at >> 6 & 7u, block = at >> 9;
#pragma unroll
        for (int k = 0; k < 8; ++k) {
            const uint32_t row = block * 64 + c * 8 + k;
            v[k] = row < a.rows && (int)rank < a.rank ? __ldg(a.t + ((int64_t)blockIdx.y * a.rows + row) * a.rank + rank) : 0.0f;
        }
        planes8(v, w);
        char* out = a.t_image + blockIdx.y * t_outer_image(a.rows) + (int64_t)block * kPlanesBytes;
#pragma unroll
        for (int p = 0; p < 3; ++p) *reinterpret_cast<uint4*>(out + swizzled(p * kRank + rank, c)) = w[p];
        return;
    }
    at -= a.t_count;
    if (a.shared && blockIdx.y) return;
    if (at < a.down_count) {
        // the faster index is the one along which the factor is packed
        const bool ranks_packed = a.down.sj == 1;
        const uint32_t rank = ranks_packed ? at & 63u : at >> 3 & 63u, c = ranks_packed ? at >> 6 & 7u : at & 7u, block = at >> 9;
        const float* f = a.down.p + (int64_t)blockIdx.y * a.down.ws;
#pragma unroll
        for (int k = 0; k < 8; ++k) {
            const int64_t col = (int64_t)block * 64 + c * 8 + k;
            v[k] = (int)rank < a.rank && col < a.down_h ? __ldg(f + rank * a.down.sj + col * a.down.sc) : 0.0f;
        }
        planes8(v, w);
        char* out = a.down_image + blockIdx.y * down_image(a.down_h) + (int64_t)block * kPlanesBytes;
#pragma unroll
        for (int p = 0; p < 3; ++p) *reinterpret_cast<uint4*>(out + swizzled(p * kRank + rank, c)) = w[p];
        return;
    }
    at -= a.down_count;
    if (at >= a.up_count) return;
    const bool ranks_packed = a.up.sj == 1;
    const uint32_t col = ranks_packed ? at >> 3 & 127u : at & 127u, c = ranks_packed ? at & 7u : at >> 7 & 7u, block = at >> 10;
    const float* f = a.up.p + (int64_t)blockIdx.y * a.up.ws;
    const int64_t column = (int64_t)block * 128 + col;
#pragma unroll
    for (int k = 0; k < 8; ++k) {
        const int rank = c * 8 + k;
        v[k] = rank < a.rank && column < a.up_h ? __ldg(f + rank * a.up.sj + column * a.up.sc) : 0.0f;
    }
    planes8(v, w);
    char* out = a.up_image + blockIdx.y * up_image(a.up_h) + (int64_t)block * (2 * kTileBytes);
#pragma unroll
    for (int p = 0; p < 2; ++p) *reinterpret_cast<uint4*>(out + p * kTileBytes + swizzled(col, c)) = w[p];
}

// ---- down and outer --------------------------------------------------------------------------------------------------------

struct Args {
    const void* x;
    int64_t x_ws, x_rs;
    const char* image;   // of the factor, or of t
    int64_t image_ws;    // bytes from worker to worker
    char *t_up, *t_outer;  // down: images of t to write (t_outer may be null)
    float* out;            // down: t (may be null); outer: as in AdapterArgs
    int64_t sj, sc;        // outer: of an element of out
    uint32_t rows;
    int32_t h, rank;
    uint32_t tiles;        // down: of 256 rows, a worker's
    int32_t split;         // down: CTAs of a cluster, which share out the columns
    uint32_t chunks;       // outer: of a worker's rows
    float scale;
    Drop drop;
};

// The barriers: a stage is full (256 threads' chunks and the planes), a stage is empty (its products are done); the sums are ready, the
// sums are drained.
enum : int { kFull = 0, kEmpty = kStages, kReady = 2 * kStages, kDrained = 2 * kStages + 1, kBars = 2 * kStages + 2 };
constexpr int kThreads = 288;

// Shared memory from its first 1024-byte boundary on, tensor memory and the barriers. The shared word that takes the address is the
// caller's.
__device__ __forceinline__ char* tensor_begin(char* smem, uint64_t* bars, uint32_t* word, uint32_t columns, uint32_t& memory) {
    if (threadIdx.x < 32) memory_alloc(shared_address(word), columns);
    if (threadIdx.x == 0) {
        for (int k = 0; k < kBars; ++k)
            barrier_init(shared_address(bars + k), k < kEmpty ? 257u : k == kDrained ? 256u : 1u);
        fence_shared();
        asm volatile("fence.mbarrier_init.release.cluster;" ::: "memory");
    }
    fence_before();
    __syncthreads();
    fence_after();
    memory = *word;
    return smem + ((1024u - (shared_address(smem) & 1023u)) & 1023u);
}
__device__ __forceinline__ void tensor_end(uint32_t memory, uint32_t columns) {
    fence_before();
    __syncthreads();
    fence_after();
    if (threadIdx.x < 32) memory_free(memory, columns);
}

// The ninth warp's part: planes and products of the steps first, first + stride, ... below last.
template <bool ACROSS>
__device__ __forceinline__ void issue_products_alone(const char* image, int first, int stride, int last, char* smem, uint32_t memory, uint32_t bars) {
    bool lost = false;
    auto planes = [&](int step, int stage) {
        if (step >= last) return;
        const uint32_t bar = bars + 8 * (kFull + stage);
        mbar_expect(bar, kPlanesBytes);
        bulk_load(smem + stage * kStageBytes + 2 * kTileBytes, image + (int64_t)step * kPlanesBytes, kPlanesBytes, bar);
    };
    for (int s = 0; s < kStages - 1; ++s) planes(first + s * stride, s);
    int stage = 0, since = 0;
    uint32_t full = 0, empty = 0, drained = 1;  // phases; nothing is to be drained at first
    for (int step = first, turn = 0; step < last && !lost; step += stride, ++turn) {
        if (since == 0) {
            if (turn > 0) lost = !barrier_wait(bars + 8 * kDrained, drained);
            drained ^= 1u;
        }
        lost = lost || !barrier_wait(bars + 8 * (kFull + stage), full >> stage & 1u);
        full ^= 1u << stage;
        if (lost) break;
        fence_after();
        const uint32_t tiles = shared_address(smem + stage * kStageBytes), right = tiles + 2 * kTileBytes;
#pragma unroll
        for (int m = 0; m < 2; ++m)
#pragma unroll
            for (int k = 0; k < 4; ++k) {  // 16 of the 64
                const uint64_t left = ACROSS ? operand(tiles + m * kTileBytes + k * 2048, 8192) : operand(tiles + m * kTileBytes + k * 32, 16);
                product(memory + m * kN, left, operand(right + k * 32, 16), instruction(kN, ACROSS, false), since > 0 || k > 0);
            }
        products_done(bars + 8 * (kEmpty + stage));
        if (++since == kFlush || step + stride >= last) {
            since = 0;
            products_done(bars + 8 * kReady);
        }
        const int behind = stage == 0 ? kStages - 1 : stage - 1;
        if (turn > 0) {
            lost = !barrier_wait(bars + 8 * (kEmpty + behind), empty >> behind & 1u);
            empty ^= 1u << behind;
        }
        if (!lost) planes(step + (kStages - 1) * stride, behind);
        stage = stage + 1 == kStages ? 0 : stage + 1;
    }
    if (lost) gave_up = 1;
}

template <bool ACROSS>
__device__ __forceinline__ void issue_products(const char* image, int first, int stride, int last, char* smem, uint32_t memory, uint32_t bars) {
    if (threadIdx.x == 256) issue_products_alone<ACROSS>(image, first, stride, last, smem, memory, bars);
    __syncwarp();
}

// The first eight warps' part: the sums of two tiles along the steps; sums[r] of a thread is rank r of row 128 (warp / 4) + 32 (warp % 4) +
// lane of the 256. ACROSS = false: 256 rows from row0 on, steps of 64 along the columns; true: 256 columns from column0 on, steps of
// 64 along the rows. A thread has a column of eight chunks, every 32nd row's (or 8th row's): its addresses are a start and a stride.
template <bool VEC, bool ACROSS>
__device__ __forceinline__ void sum_tiles(const Args& a, uint32_t worker, uint32_t row0, int column0, int first, int stride, int last, char* smem,
                                          uint32_t memory, uint32_t bars, float (&sums)[kRank]) {
    constexpr uint32_t kRows = ACROSS ? 8 : 32, kPlace = ACROSS ? 1024 : 4096;  // from one of a thread's chunks to the next
    const int warp = threadIdx.x >> 5;
    const uint32_t r0 = ACROSS ? threadIdx.x >> 5 : threadIdx.x >> 3, c0 = ACROSS ? threadIdx.x & 31u : threadIdx.x & 7u;
    char* at0 = smem + (ACROSS ? (c0 >> 3) * 8192u + swizzled(r0, c0 & 7u) : swizzled(r0, c0));
    const int64_t step_rows = ACROSS ? 64 : 0, step_columns = ACROSS ? 0 : 64;
    const uint32_t row1 = (ACROSS ? 0 : row0) + r0;        // of step 0 and the first chunk
    const int64_t column1 = (ACROSS ? column0 : 0) + (int64_t)c0 * 8;
    const __nv_bfloat16* x = (const __nv_bfloat16*)a.x + (int64_t)worker * a.x_ws;
    const uint32_t call = drop_call(a.drop);
    bool lost = false;  // a wait gave up
    auto fetch = [&](int step, int stage) {
        if (step < last) {
            const int64_t column = column1 + step * step_columns;
            const uint32_t row = row1 + (uint32_t)(step * step_rows);
            const __nv_bfloat16* from = x + (int64_t)row * a.x_rs + column;
            const bool in = column < a.h;
#pragma unroll
            for (int k = 0; k < 8; ++k) {
                const bool there = in && row + k * kRows < a.rows;
                char* to = at0 + stage * kStageBytes + k * kPlace;
                if constexpr (VEC) {
                    copy16(to, there ? (const void*)(from + k * kRows * a.x_rs) : a.x, there);
                } else {
                    *reinterpret_cast<uint4*>(to) = raw_columns<__nv_bfloat16, false>(
                        there ? from + k * kRows * a.x_rs - column : (const __nv_bfloat16*)a.x, (int)column, there ? a.h : 0).q;
                }
            }
        }
        copies_commit();
    };
    auto mask = [&](int step, int stage) {  // the chunks that this thread copied
        const uint32_t row = row1 + (uint32_t)(step * step_rows), group = (uint32_t)((column1 + step * step_columns) >> 3);
#pragma unroll
        for (int k = 0; k < 8; ++k) {
            const uint4 u = drop_words(a.drop, group, row + k * kRows, a.drop.worker + worker, call);
            uint4* place = reinterpret_cast<uint4*>(at0 + stage * kStageBytes + k * kPlace);
            const Raw8<__nv_bfloat16> raw = {*place};
            uint32_t w[1][4];
            raw_planes<__nv_bfloat16>(raw, a.drop, u, w);
            *place = make_uint4(w[0][0], w[0][1], w[0][2], w[0][3]);
        }
    };
    // the tiles' sums go from tensor memory to the registers, the planes' together
    auto flush = [&]() {
        const uint32_t at = memory + ((uint32_t)(warp & 3) << 21) + (uint32_t)(warp >> 2) * kN;
#pragma unroll
        for (int half = 0; half < 2; ++half) {
            float v[32], w[32];
            columns32(at + 2 * kRank + half * 32, v);
            columns32(at + kRank + half * 32, w);
            columns_wait(v);
            columns_wait(w);
#pragma unroll
            for (int k = 0; k < 32; ++k) w[k] += v[k];
            columns32(at + half * 32, v);
            columns_wait(v);
#pragma unroll
            for (int k = 0; k < 32; ++k) sums[half * 32 + k] += v[k] + w[k];
        }
    };
#pragma unroll
    for (int r = 0; r < kRank; ++r) sums[r] = 0.0f;
    for (int s = 0; s < kStages - 1; ++s) fetch(first + s * stride, s);
    int stage = 0, since = 0;
    uint32_t empty = 0, ready = 0;  // phases
    for (int step = first, turn = 0; step < last; step += stride, ++turn) {
        copies_wait<kStages - 2>();
        if (a.drop.on) mask(step, stage);
        fence_shared();
        barrier_arrive(bars + 8 * (kFull + stage));
        // the stage before is free once its products are done
        const int behind = stage == 0 ? kStages - 1 : stage - 1;
        if (turn > 0) {
            lost = lost || !barrier_wait(bars + 8 * (kEmpty + behind), empty >> behind & 1u);
            empty ^= 1u << behind;
        }
        fetch(step + (kStages - 1) * stride, behind);
        if (++since == kFlush || step + stride >= last) {
            since = 0;
            lost = lost || !barrier_wait(bars + 8 * kReady, ready);
            ready ^= 1u;
            fence_after();
            flush();
            fence_before();
            barrier_arrive(bars + 8 * kDrained);
        }
        stage = stage + 1 == kStages ? 0 : stage + 1;
    }
    copies_wait<0>();
    if (lost) gave_up = 1;
}

// A CTA takes 256 rows of a worker and its share of the columns.
template <bool VEC>
__global__ void __launch_bounds__(kThreads, 1) down_kernel(const __grid_constant__ Args a) {
    extern __shared__ __align__(16) char dynamic[];
    __shared__ uint64_t bars[kBars];
    __shared__ uint32_t word;
    dependency_wait();
    uint32_t memory;
    char* smem = tensor_begin(dynamic, bars, &word, kColumns, memory);
    const uint32_t tile = blockIdx.x / a.split, i = tile / a.tiles, row0 = (tile - i * a.tiles) * 256;
    const int part = (int)(blockIdx.x - tile * a.split), steps = (a.h + 63) / 64;
    const bool main = threadIdx.x < 256;
    float sums[kRank];
    if (main) sum_tiles<VEC, false>(a, i, row0, 0, part, a.split, steps, smem, memory, shared_address(bars), sums);
    else issue_products<false>(a.image + (int64_t)i * a.image_ws, part, a.split, steps, smem, memory, shared_address(bars));
    tensor_end(memory, kColumns);
    // this CTA's sums, then its share of the rows, joined over the cluster in order
    constexpr int L = kRank + 1;
    float *mine = reinterpret_cast<float*>(smem), *whole = mine + 256 * L;
    if (main)
#pragma unroll
        for (int r = 0; r < kRank; ++r) mine[threadIdx.x * L + r] = sums[r];
    cooperative_groups::cluster_group cluster = cooperative_groups::this_cluster();
    cluster.sync();
    const float scale = a.scale * (a.drop.on ? a.drop.factor : 1.0f);
    const int share = 256 / a.split, from = part * share;  // split is a power of two up to 4: a share is 64 rows at least
    for (int e = threadIdx.x; e < share * kRank; e += kThreads) {
        const int r = e / kRank, j = e % kRank;
        float v = 0.0f;
        for (int s = 0; s < a.split; ++s) v += cluster.map_shared_rank(mine, s)[(from + r) * L + j];
        whole[r * L + j] = scale * v;
    }
    __syncthreads();
    const uint32_t first = row0 + from;  // a multiple of 64
    if (a.out)
        for (int e = threadIdx.x; e < share * kRank; e += kThreads) {
            const int r = e / kRank, j = e % kRank;
            if (first + r < a.rows && j < a.rank) a.out[((int64_t)i * a.rows + first + r) * a.rank + j] = whole[r * L + j];
        }
    for (int e = threadIdx.x; e < share * 8; e += kThreads) {  // a row's eight ranks
        const int r = e >> 3, c = e & 7;
        const uint32_t row = first + r;
        if (row >= (a.rows + 127) / 128 * 128) break;
        float v[8];
#pragma unroll
        for (int k = 0; k < 8; ++k) v[k] = whole[r * L + c * 8 + k];
        uint4 w[3];
        planes8(v, w);
        char* out = a.t_up + i * t_up_image(a.rows) + (int64_t)(row >> 7) * (2 * kTileBytes) + swizzled(row & 127u, c);
        *reinterpret_cast<uint4*>(out) = w[0];
        *reinterpret_cast<uint4*>(out + kTileBytes) = w[1];
    }
    if (a.t_outer)
        for (int e = threadIdx.x; e < share * 8; e += kThreads) {  // a rank's eight rows
            const int j = e & 63, r = (e >> 6) * 8;
            const uint32_t row = first + r;
            if (row >= (a.rows + 63) / 64 * 64) break;
            float v[8];
#pragma unroll
            for (int k = 0; k < 8; ++k) v[k] = whole[(r + k) * L + j];
            uint4 w[3];
            planes8(v, w);
            char* out = a.t_outer + i * t_outer_image(a.rows) + (int64_t)(row >> 6) * kPlanesBytes;
#pragma unroll
            for (int p = 0; p < 3; ++p) *reinterpret_cast<uint4*>(out + swizzled(p * kRank + j, (row >> 3) & 7u)) = w[p];
        }
    cluster.sync();  // the others may still be reading
}

// A CTA takes 256 columns and a chunk of a worker's rows.
template <bool VEC>
__global__ void __launch_bounds__(kThreads, 1) outer_kernel(const __grid_constant__ Args a) {
    extern __shared__ __align__(16) char dynamic[];
    __shared__ uint64_t bars[kBars];
    __shared__ uint32_t word;
    dependency_wait();
    uint32_t memory;
    char* smem = tensor_begin(dynamic, bars, &word, kColumns, memory);
    const uint32_t i = blockIdx.y / a.chunks, chunk = blockIdx.y - i * a.chunks, blocks = (a.rows + 63) / 64;
    const int s0 = (int)((uint64_t)blocks * chunk / a.chunks), s1 = (int)((uint64_t)blocks * (chunk + 1) / a.chunks);
    float sums[kRank];
    if (threadIdx.x < 256) sum_tiles<VEC, true>(a, i, 0, (int)blockIdx.x * 256, s0, 1, s1, smem, memory, shared_address(bars), sums);
    else issue_products<true>(a.image + (int64_t)i * a.image_ws, s0, 1, s1, smem, memory, shared_address(bars));
    tensor_end(memory, kColumns);
    const int64_t c = (int64_t)blockIdx.x * 256 + threadIdx.x;
    if (threadIdx.x >= 256 || c >= a.h) return;
    const float scale = a.scale * (a.drop.on ? a.drop.factor : 1.0f);
    float* out = a.out + (int64_t)blockIdx.y * a.rank * a.h + c * a.sc;
    if (a.sj == 1 && (a.rank & 3) == 0 && (reinterpret_cast<uintptr_t>(a.out) & 15u) == 0) {
#pragma unroll
        for (int r = 0; r < kRank; r += 4)
            if (r < a.rank)
                *reinterpret_cast<float4*>(out + r) = make_float4(scale * sums[r], scale * sums[r + 1], scale * sums[r + 2], scale * sums[r + 3]);
    } else {
#pragma unroll
        for (int r = 0; r < kRank; ++r)
            if (r < a.rank) out[r * a.sj] = scale * sums[r];
    }
}

// ---- up --------------------------------------------------------------------------------------------------------------------

// A CTA takes 128 columns, whose planes of the factor stay in shared memory, and goes through the 128-row tiles of a chunk: the tile's
// planes of t and of the base by copies, 12 products of 16 rank indices (the planes' indices together at most 1), the
// result into the base's place in shared memory and from there to memory by rows. Behind the products t's place is free for the next base,
// which is on its way during the rest of the tile, and behind the stores the tile's place for the next t. Two CTAs to an SM.
constexpr int kUpShared = 1024 + 2 * 2 * kTileBytes + 2 * kTileBytes;
constexpr uint32_t kUpColumns = 128;

struct UpArgs {
    const void* base;  // may be null
    void* y;
    const char *image, *t_up;
    int64_t base_ws, base_rs, image_ws;
    uint32_t rows, chunks;
    int32_t h;
    float scale;
    Drop drop;
};

template <bool VEC>
__global__ void __launch_bounds__(256, 2) up_kernel(const __grid_constant__ UpArgs a) {
    extern __shared__ __align__(16) char dynamic[];
    __shared__ uint64_t bars[kBars];
    __shared__ uint32_t word;
    bool lost = false;  // a wait gave up
    dependency_wait();
    uint32_t memory;
    char* smem = tensor_begin(dynamic, bars, &word, kUpColumns, memory);
    // tile: 128 rows of 16 chunks, chunk c at c ^ (row % 8)
    char *planes = smem, *t = smem + 2 * kTileBytes, *tile = smem + 4 * kTileBytes;
    const uint32_t i = blockIdx.y / a.chunks, chunk = blockIdx.y - i * a.chunks, blocks = (a.rows + 127) / 128;
    const uint32_t b0 = (uint32_t)((uint64_t)blocks * chunk / a.chunks), b1 = (uint32_t)((uint64_t)blocks * (chunk + 1) / a.chunks);
    const int c0 = (int)blockIdx.x * 128, warp = threadIdx.x >> 5, lane = threadIdx.x & 31;
    const uint32_t call = drop_call(a.drop), bar = shared_address(bars + kReady);
    auto linear = [&](char* to, const char* from) {  // two planes
#pragma unroll
        for (int k = 0; k < 2 * kTileBytes / 16 / 256; ++k) copy16(to + (threadIdx.x + 256 * k) * 16, from + (threadIdx.x + 256 * k) * 16);
    };
    // a thread has a column of eight chunks of a tile, every 16th row's
    const uint32_t r0 = threadIdx.x >> 4, at0 = r0 * 256u + (((threadIdx.x & 15u) ^ (r0 & 7u)) << 4);
    const int column = c0 + (int)(threadIdx.x & 15u) * 8;
    const __nv_bfloat16* base = (const __nv_bfloat16*)a.base + (int64_t)i * a.base_ws + column;
    __nv_bfloat16* y = (__nv_bfloat16*)a.y + (int64_t)i * a.rows * a.h + column;
    auto fetch_base = [&](uint32_t b, char* tile) {
        if (!a.base) return;
        const __nv_bfloat16* from = base + (int64_t)(b * 128 + r0) * a.base_rs;
#pragma unroll
        for (int k = 0; k < 8; ++k) {
            const bool in = column < a.h && b * 128 + r0 + 16 * k < a.rows;
            if constexpr (VEC) copy16(tile + at0 + k * 4096, in ? (const void*)(from + k * 16 * a.base_rs) : a.base, in);
            else *reinterpret_cast<uint4*>(tile + at0 + k * 4096) = raw_columns<__nv_bfloat16, false>(
                     in ? from + k * 16 * a.base_rs - column : (const __nv_bfloat16*)a.base, column, in ? a.h : 0).q;
        }
    };
    const char* t_image = a.t_up + i * t_up_image(a.rows);
    linear(planes, a.image + (int64_t)i * a.image_ws + (int64_t)blockIdx.x * (2 * kTileBytes));
    if (b0 < b1) {
        linear(t, t_image + (int64_t)b0 * (2 * kTileBytes));
        fetch_base(b0, tile);
    }
    copies_commit();
    uint32_t phase = 0;
    for (uint32_t b = b0; b < b1; ++b) {
        copies_wait<0>();
        fence_shared();
        fence_before();
        __syncthreads();
        if (threadIdx.x == 0) {
            fence_after();
            const uint32_t left = shared_address(t), right = shared_address(planes);
#pragma unroll
            for (int q = 0; q < 3; ++q) {  // (0, 1), (1, 0), (0, 0): the smallest first
                const uint32_t l = left + (q == 1 ? kTileBytes : 0), r = right + (q == 0 ? kTileBytes : 0);
#pragma unroll
                for (int k = 0; k < 4; ++k)
                    product(memory, operand(l + k * 32, 16), operand(r + k * 32, 16), instruction(128, false, false), q > 0 || k > 0);
            }
            products_done(bar);
        }
        lost |= !barrier_wait(bar, phase);
        phase ^= 1u;
        fence_after();
        if (b + 1 < b1) fetch_base(b + 1, t);
        // a lane's row: 64 columns from 64 (warp / 4) on
        const uint32_t r = (uint32_t)(warp & 3) * 32 + lane, row = b * 128 + r;
#pragma unroll
        for (int half = 0; half < 2; ++half) {
            const int first = (warp >> 2) * 64 + half * 32;
            float v[32];
            columns32(memory + ((uint32_t)(warp & 3) << 21) + first, v);
            columns_wait(v);
#pragma unroll
            for (int k = 0; k < 4; ++k) {
                const uint32_t c = (uint32_t)(first >> 3) + k;
                uint4* at = reinterpret_cast<uint4*>(tile + r * 256u + ((c ^ (r & 7u)) << 4));
                float x[8] = {};
                if (a.base) raw_floats<__nv_bfloat16>({*at}, x);
#pragma unroll
                for (int e = 0; e < 8; ++e) x[e] = fmaf(a.scale, v[k * 8 + e], x[e]);
                if (a.drop.on) drop8(a.drop, drop_words(a.drop, (uint32_t)(c0 >> 3) + c, row, a.drop.worker + i, call), x);
                *at = make_uint4(pack(x[0], x[1], __nv_bfloat16()), pack(x[2], x[3], __nv_bfloat16()), pack(x[4], x[5], __nv_bfloat16()),
                                 pack(x[6], x[7], __nv_bfloat16()));
            }
        }
        fence_before();
        if (__syncthreads_or(lost)) {
            if (threadIdx.x == 0) gave_up = 1;
            break;
        }
        __nv_bfloat16* to = y + (int64_t)(b * 128 + r0) * a.h;
#pragma unroll
        for (int k = 0; k < 8; ++k) {
            const uint4 u = *reinterpret_cast<const uint4*>(tile + at0 + k * 4096);
            if (b * 128 + r0 + 16 * k >= a.rows || column >= a.h) continue;
            if (VEC) {
                *reinterpret_cast<uint4*>(to + (int64_t)k * 16 * a.h) = u;
            } else {
                __nv_bfloat16 s[8];
                memcpy(s, &u, sizeof(s));
#pragma unroll
                for (int e = 0; e < 8; ++e)
                    if (column + e < a.h) to[(int64_t)k * 16 * a.h + e] = s[e];
            }
        }
        __syncthreads();
        if (b + 1 < b1) linear(tile, t_image + (int64_t)(b + 1) * (2 * kTileBytes));
        copies_commit();
        char* other = t;
        t = tile;
        tile = other;
    }
    copies_wait<0>();
    tensor_end(memory, kUpColumns);
}

}  // namespace tensor
}  // namespace
}  // namespace compams
