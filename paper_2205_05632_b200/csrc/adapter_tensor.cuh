// The adapters' three products on tcgen05.mma, for bfloat16 activations. mma.sync is bound by its own rate (550 TFLOP/s measured, a third
// of tcgen05's) from about rank 32 on, and below by the instructions that bring operands to registers. (fp16 would need two tiles of bf16
// planes for each tile of the activation, which the eight warps would have to write, and fp32 three: both stay on mma.sync.)
//
// The planes of an fp32 operand are stacked along N: a tile of an activation, 128 x 64, is multiplied by [3 x R] rows of planes at
// once (R: the rank, padded to 16, 32 or 64; higher ranks go in groups of 64), so it is an operand once for a group and the planes' sums
// stand beside each other in tensor memory. Operands lie in shared memory in the 128-byte swizzle: rows of 128 bytes (64 elements), whose 16-byte chunk c lies at chunk
// c ^ (row % 8). down: the rows are the activation's and the sum runs along them (K-major); outer: the sum runs over the rows, the tile
// is read across them (MN-major), and t comes turned, [plane, rank][row].
//
// One thread of a ninth warp issues the products and one of a tenth brings the tiles (TMA, into the swizzle; the planes, already in its
// order, in bulk): a stage costs the one 0.35 us of issue and the other 0.2 us, whatever the rank; one thread for both, waits included, held
// every stage to 0.8 to 1.1 us. They wait for nobody else unless dropout masks the activation, which the 256 threads of the other warps
// do in place. The tensor cores cut their sums, so after every kFlush tiles of 64 the sums go to fp32 registers by rounded additions,
// which is the other warps' work. Activations that TMA cannot address (odd widths, other strides) are brought by these warps, element by
// element.
#pragma once

#include "rows.cuh"
#include "tcgen05.cuh"

namespace compams {
namespace {
namespace tensor {

constexpr int kTileBytes = 128 * 128;      // 128 rows of 64 elements, or 64 rows of 128
// Tiles between two additions to the registers. The largest error of dA, 2048 rows x 4096, rank 64, against its largest value: 4.3e-7 with
// 4, 8.8e-7 with 8, and 1.8e-6 for torch's fp32 product.
constexpr int kFlush = 8;

// What goes by the padded rank.
__host__ __device__ inline int padded_rank(int rank) { return rank <= 16 ? 16 : rank <= 32 ? 32 : 64; }
__host__ __device__ inline int groups_of(int rank) { return rank <= 64 ? 1 : (rank + 63) / 64; }
template <int R>
struct By {
    static constexpr int kN = 3 * R;                       // planes side by side
    static constexpr int kPlanesBytes = kN * 128;          // planes: rows of 64 elements
    static constexpr uint32_t kColumns = R == 64 ? 512 : R == 32 ? 256 : 128;  // of tensor memory: 2 kN used, a power of two taken
    // up: tiles of 128 rows for the three planes; they share a row's 128 bytes as far as they have room
    static constexpr int kUpTiles = R == 64 ? 3 : R == 32 ? 2 : 1, kUpBytes = kUpTiles * kTileBytes;
};
// Where plane p of an operand of up lies: the tile and the byte of the row.
template <int R>
__host__ __device__ constexpr uint32_t up_tile(uint32_t p) { return p * 2 * R / 128; }
template <int R>
__host__ __device__ constexpr uint32_t up_byte(uint32_t p) { return p * 2 * R % 128; }
// The stages of down (ACROSS = false) and outer: two tiles of the activation, which go to a sum each, and planes. outer: 64 rows of 256
// columns. down: 64 columns of 256 rows, or, up to rank 32, 128 columns of 128 rows (WIDE), whose two sums are of the same rows and are
// added in the end: twice as many CTAs for a few thousand rows (4096 x 4096, rank 16: 15.5 -> 13.7 us), for planes read twice as often.
template <int R, bool ACROSS>
struct Pipe {
    static constexpr bool kWide = !ACROSS && R <= 32;
    static constexpr int kRows = ACROSS ? 0 : kWide ? 128 : 256, kStep = kWide ? 128 : 64;  // down: rows of a CTA; columns (outer: rows) of a step
    static constexpr int kPlanesBytes = By<R>::kPlanesBytes * (kWide ? 2 : 1), kStageBytes = 2 * kTileBytes + kPlanesBytes;
    static constexpr int kStages = kStageBytes * 5 > 225 * 1024 ? 4 : 5;  // what 227 KB hold
    static constexpr int kShared = 1024 + kStages * kStageBytes;
    // The barriers: what is brought to a stage has landed; 256 threads have done their part on it; its products are done; the sums are
    // ready, and drained; where someone gave up: all products are done.
    static constexpr int kLanded = 0, kTouched = kStages, kEmpty = 2 * kStages, kReady = 3 * kStages, kDrained = 3 * kStages + 1,
                         kStopped = 3 * kStages + 2, kBars = 3 * kStages + 3;
};

// ---- images of the fp32 operands in global memory, in the order of shared memory --------------------------------------------

// All begin with the group of ranks. A factor for down: [64 columns, an even number of times][plane, rank][64 columns]; for up: [128 columns]
// [tile][column][plane, rank]: a column's 128 bytes hold a plane of 64 ranks, two of 32, all three of 16. Bytes of a group, and of a worker's.
__host__ __device__ inline int64_t down_group(int64_t h, int rank) { return (h + 127) / 128 * (2 * 3 * 128 * padded_rank(rank)); }
__host__ __device__ inline int64_t up_group(int64_t h, int rank) {
    const int r = padded_rank(rank);
    return (h + 127) / 128 * kTileBytes * (r == 64 ? By<64>::kUpTiles : r == 32 ? By<32>::kUpTiles : By<16>::kUpTiles);
}
__host__ __device__ inline int64_t down_image(int64_t h, int rank) { return groups_of(rank) * down_group(h, rank); }
__host__ __device__ inline int64_t up_image(int64_t h, int rank) { return groups_of(rank) * up_group(h, rank); }
// t for outer: [64 rows][plane, rank][row]; for up: [128 rows], as a factor's columns.
__host__ __device__ inline int64_t t_outer_group(int64_t rows, int rank) { return (rows + 63) / 64 * (3 * 128 * padded_rank(rank)); }
__host__ __device__ inline int64_t t_outer_image(int64_t rows, int rank) { return groups_of(rank) * t_outer_group(rows, rank); }
__host__ __device__ inline int64_t t_up_group(int64_t rows, int rank) { return up_group(rows, rank); }
__host__ __device__ inline int64_t t_up_image(int64_t rows, int rank) { return up_image(rows, rank); }

// Waits that give up, which no size or input should bring about. Whoever gave up marks the CTA's shared word and this one, which stays until
// it is asked for; no thread waits in vain twice. Before the tensor memory is given back the copies and products under way are
// waited for, with a limit of their own, and the CTA's results are NaN, so that what is computed from them shows it.
__device__ int32_t gave_up;
__device__ __forceinline__ void give_up(uint32_t* lost) {
    gave_up = 1;
    *lost = 1u;
}

// Eight planes' neighbours as a chunk of 16 bytes each.
__device__ __forceinline__ void planes8(const float (&v)[8], uint4 (&out)[3]) {
    uint32_t w[4][3];
#pragma unroll
    for (int q = 0; q < 4; ++q) split2<3>(v[2 * q], v[2 * q + 1], w[q]);
#pragma unroll
    for (int p = 0; p < 3; ++p) out[p] = make_uint4(w[0][p], w[1][p], w[2][p], w[3][p]);
}

// The planes of eight ranks of a row (a column of the factor) in an image for up.
template <int R>
__device__ __forceinline__ void store_up(char* tile, uint32_t row, uint32_t c, const uint4 (&w)[3]) {
#pragma unroll
    for (uint32_t p = 0; p < 3; ++p) *reinterpret_cast<uint4*>(tile + up_tile<R>(p) * kTileBytes + swizzled(row, up_byte<R>(p) / 16 + c)) = w[p];
}

// ---- prepare ---------------------------------------------------------------------------------------------------------------

struct PrepareArgs {
    Factor down, up;
    char *down_image, *up_image;  // may be null
    const float* t;
    char* t_image;  // t for outer; may be null
    int32_t down_h, up_h, rank;
    uint32_t rows, down_count, up_count, t_count;  // chunks of a worker's images, of one plane
    uint32_t down_blocks, up_blocks, t_blocks;     // of a group
    int32_t shared;
};
// A thread per chunk of 16 bytes. 2.4 us for the factors of 4096 x 4096 at rank 16, 7.5 for 4096 x 8192 at rank 64 with 16384 rows of t.
template <int R>
__global__ void __launch_bounds__(256) prepare_kernel(const __grid_constant__ PrepareArgs a) {
    uint32_t at = blockIdx.x * 256 + threadIdx.x;
    float v[8];
    uint4 w[3];
    if (at < a.t_count) {  // [64 rows][8 rows][rank]: neighbouring threads read neighbouring ranks
        const uint32_t lane = at % R, c = at / R % 8u, all = at / (8 * R), block = all % a.t_blocks, rank = all / a.t_blocks * R + lane;
#pragma unroll
        for (int k = 0; k < 8; ++k) {
            const uint32_t row = block * 64 + c * 8 + k;
            v[k] = row < a.rows && (int)rank < a.rank ? __ldg(a.t + ((int64_t)blockIdx.y * a.rows + row) * a.rank + rank) : 0.0f;
        }
        planes8(v, w);
        char* out = a.t_image + blockIdx.y * t_outer_image(a.rows, a.rank) + (int64_t)all * By<R>::kPlanesBytes;
#pragma unroll
        for (int p = 0; p < 3; ++p) *reinterpret_cast<uint4*>(out + swizzled(p * R + lane, c)) = w[p];
        return;
    }
    at -= a.t_count;
    if (a.shared && blockIdx.y) return;
    if (at < a.down_count) {
        // the faster index is the one along which the factor is packed
        const bool ranks_packed = a.down.sj == 1;
        const uint32_t lane = ranks_packed ? at % R : at / 8 % R, c = ranks_packed ? at / R % 8u : at % 8u, all = at / (8 * R);
        const uint32_t block = all % a.down_blocks, rank = all / a.down_blocks * R + lane;
        const float* f = a.down.p + (int64_t)blockIdx.y * a.down.ws;
#pragma unroll
        for (int k = 0; k < 8; ++k) {
            const int64_t col = (int64_t)block * 64 + c * 8 + k;
            v[k] = (int)rank < a.rank && col < a.down_h ? __ldg(f + rank * a.down.sj + col * a.down.sc) : 0.0f;
        }
        planes8(v, w);
        char* out = a.down_image + blockIdx.y * down_image(a.down_h, a.rank) + (int64_t)all * By<R>::kPlanesBytes;
#pragma unroll
        for (int p = 0; p < 3; ++p) *reinterpret_cast<uint4*>(out + swizzled(p * R + lane, c)) = w[p];
        return;
    }
    at -= a.down_count;
    if (at >= a.up_count) return;
    const bool ranks_packed = a.up.sj == 1;
    constexpr uint32_t C = R / 8;  // chunks of a plane's row
    const uint32_t col = ranks_packed ? at / C % 128u : at % 128u, c = ranks_packed ? at % C : at / 128 % C, all = at / (128 * C);
    const uint32_t block = all % a.up_blocks, group = all / a.up_blocks;
    const float* f = a.up.p + (int64_t)blockIdx.y * a.up.ws;
    const int64_t column = (int64_t)block * 128 + col;
#pragma unroll
    for (int k = 0; k < 8; ++k) {
        const int rank = (int)(group * R + c * 8) + k;
        v[k] = rank < a.rank && column < a.up_h ? __ldg(f + rank * a.up.sj + column * a.up.sc) : 0.0f;
    }
    planes8(v, w);
    store_up<R>(a.up_image + blockIdx.y * up_image(a.up_h, a.rank) + (int64_t)all * By<R>::kUpBytes, col, c, w);
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
    uint32_t tiles;        // down: of 256 rows (WIDE: 128), a worker's
    int32_t split;         // down: CTAs of a cluster, which share out the columns
    uint32_t chunks;       // outer: of a worker's rows
    uint32_t tries;        // of a wait
    float scale;
    Drop drop;
};

constexpr int kThreads = 320;
constexpr int kMostSplit = 4;  // CTAs of a cluster of down (with 8 no size was faster)

// Tensor memory and the barriers. The shared words, one that takes the address and one for who gives up, are the caller's.
template <typename P>
__device__ __forceinline__ void tensor_begin(uint64_t* bars, uint32_t* word, uint32_t columns, uint32_t& memory) {
    if (threadIdx.x < 32) memory_alloc(shared_address(word), columns);
    if (threadIdx.x == 0) {
        word[1] = 0u;
        for (int k = 0; k < P::kBars; ++k)
            barrier_init(shared_address(bars + k), (k >= P::kTouched && k < P::kEmpty) || k == P::kDrained ? 256u : 1u);
        fence_shared();
        asm volatile("fence.mbarrier_init.release.cluster;" ::: "memory");
    }
    fence_before();
    __syncthreads();
    fence_after();
    memory = *word;
}
// From its first 1024-byte boundary on.
__device__ __forceinline__ char* aligned(char* smem) { return smem + ((1024u - (shared_address(smem) & 1023u)) & 1023u); }
__device__ __forceinline__ void tensor_end(uint32_t memory, uint32_t columns) {
    fence_before();
    __syncthreads();
    fence_after();
    if (threadIdx.x < 32) memory_free(memory, columns);
}
// The same for down and outer: true if someone gave up. Then products and copies may still be under way, which nobody waited for: the
// ninth warp's thread waits for the former, the tenth's for the latter, of which it brought `turns` stages.
template <typename P>
__device__ __forceinline__ bool tensor_end(uint32_t memory, uint32_t columns, const uint32_t* lost, uint32_t bars, int turns) {
    fence_before();
    __syncthreads();
    const bool gone = *lost != 0u;
    if (gone) {
        if (threadIdx.x == 256) {
            products_done(bars + 8 * P::kStopped);
            barrier_wait(bars + 8 * P::kStopped, 0, kTries);
        }
        if (threadIdx.x == 288)
            for (int s = 0; s < min(turns, P::kStages); ++s)
                barrier_wait(bars + 8 * (P::kLanded + s), (uint32_t)((turns - s - 1) / P::kStages) & 1u, kTries);
        fence_before();
        __syncthreads();
    }
    fence_after();
    if (threadIdx.x < 32) memory_free(memory, columns);
    return gone;
}

// What the parts walk: steps first, first + stride, ... below last along the columns (down: rows from row0 on) or along the rows (outer,
// ACROSS: 256 columns from column0 on).
struct Walk {
    const char* image;  // of the factor or of t: the worker's, the group's
    uint32_t worker, row0;
    int column0, first, stride, last;
};

// The tenth warp's part; gives the number of stages that it brought. MAPPED: the activation is brought by TMA.
template <int R, bool MAPPED, bool ACROSS>
__device__ __forceinline__ int bring(const Args& a, const CUtensorMap* map, const Walk& k, char* smem, uint32_t bars, uint32_t* lost) {
    using P = Pipe<R, ACROSS>;
    const char* image = k.image;
    int stage = 0, turn = 0;
    uint32_t empty = 1;  // the phase to wait for: of a stage's first round none
    for (int step = k.first; step < k.last; step += k.stride, ++turn) {
        if (turn >= P::kStages && !barrier_wait(bars + 8 * (P::kEmpty + stage), empty, a.tries)) {
            give_up(lost);
            break;
        }
        const uint32_t bar = bars + 8 * (P::kLanded + stage), to = shared_address(smem + stage * P::kStageBytes);
        mbar_expect(bar, P::kPlanesBytes + (MAPPED ? 2 * kTileBytes : 0));
        if (MAPPED) {
            if (ACROSS) {
#pragma unroll
                for (int c = 0; c < 4; ++c) box_load(to + c * 8192, map, k.column0 + c * 64, step * 64, (int)k.worker, bar);
            } else {
#pragma unroll
                for (int m = 0; m < 2; ++m)
                    box_load(to + m * kTileBytes, map, step * P::kStep + (P::kWide ? m * 64 : 0), (int)k.row0 + (P::kWide ? 0 : m * 128),
                             (int)k.worker, bar);
            }
        }
        bulk_load(smem + stage * P::kStageBytes + 2 * kTileBytes, image + (int64_t)step * P::kPlanesBytes, P::kPlanesBytes, bar);
        if (++stage == P::kStages) {
            stage = 0;
            empty ^= 1u;
        }
    }
    return turn;
}

// The ninth warp's part.
template <int R, bool MAPPED, bool ACROSS>
__device__ __forceinline__ void issue(const Args& a, const Walk& k, char* smem, uint32_t memory, uint32_t bars, uint32_t* lost) {
    using P = Pipe<R, ACROSS>;
    const bool touched = !MAPPED || a.drop.on;
    const uint32_t tiles = shared_address(smem);
    const uint64_t left0 = operand(tiles, ACROSS ? 8192 : 16), right0 = operand(tiles + 2 * kTileBytes, 16);
    int stage = 0, since = 0;
    uint32_t here = 0, drained = 1;  // phases; nothing is to be drained at first
    for (int step = k.first, turn = 0; step < k.last; step += k.stride, ++turn) {
        bool ok = true;
        if (since == 0) {
            if (turn > 0) ok = barrier_wait(bars + 8 * P::kDrained, drained, a.tries);
            drained ^= 1u;
        }
        ok = ok && barrier_wait(bars + 8 * (P::kLanded + stage), here, a.tries) &&
             (!touched || barrier_wait(bars + 8 * (P::kTouched + stage), here, a.tries));
        if (!ok) {
            give_up(lost);
            break;
        }
        fence_after();
        // addresses count 16 bytes in the operands' lowest bits
        const uint64_t left = left0 + (uint32_t)(stage * (P::kStageBytes / 16)), right = right0 + (uint32_t)(stage * (P::kStageBytes / 16));
#pragma unroll
        for (int q = 0; q < 4; ++q)  // 16 of the 64
#pragma unroll
            for (int m = 0; m < 2; ++m)
                product(memory + m * By<R>::kN, left + (m * kTileBytes + q * (ACROSS ? 2048 : 32)) / 16,
                        right + (P::kWide ? m * By<R>::kPlanesBytes / 16 : 0) + q * 2, instruction(By<R>::kN, ACROSS, false), q > 0 || since > 0);
        products_done(bars + 8 * (P::kEmpty + stage));
        if (++since == kFlush || step + k.stride >= k.last) {
            since = 0;
            products_done(bars + 8 * P::kReady);
        }
        if (++stage == P::kStages) {
            stage = 0;
            here ^= 1u;
        }
    }
}
template <int R, bool MAPPED, bool ACROSS>
__device__ __forceinline__ int feed(const Args& a, const CUtensorMap* map, const Walk& k, char* smem, uint32_t memory, uint32_t bars,
                                     uint32_t* lost) {
    int turns = 0;
    if (threadIdx.x == 256) issue<R, MAPPED, ACROSS>(a, k, smem, memory, bars, lost);
    if (threadIdx.x == 288) turns = bring<R, MAPPED, ACROSS>(a, map, k, smem, bars, lost);
    __syncwarp();
    return turns;
}

// The first eight warps' part: sums[r] of a thread is rank r of row (outer: column) 32 (warp % 4) + lane of tile warp / 4. Where there is
// something to do on the tiles a thread has a column of eight chunks, every 32nd row's (or 8th row's).
template <int R, bool MAPPED, bool ACROSS>
__device__ __forceinline__ void sum_tiles(const Args& a, const Walk& k, char* smem, uint32_t memory, uint32_t bars, uint32_t* given_up,
                                          float (&sums)[R]) {
    using P = Pipe<R, ACROSS>;
    constexpr uint32_t kRows = ACROSS ? 8 : 32, kPlace = ACROSS ? 1024 : 4096;  // from one of a thread's chunks to the next
    const int warp = threadIdx.x >> 5;
    const uint32_t r0 = ACROSS ? threadIdx.x >> 5 : threadIdx.x >> 3, c0 = ACROSS ? threadIdx.x & 31u : threadIdx.x & 7u;
    char* at0 = smem + (ACROSS ? (c0 >> 3) * 8192u + swizzled(r0, c0 & 7u) : swizzled(r0, c0));
    const __nv_bfloat16* x = (const __nv_bfloat16*)a.x + (int64_t)k.worker * a.x_ws;
    const uint32_t call = drop_call(a.drop);
    const bool touch = !MAPPED || a.drop.on;
    bool lost = false;  // a wait gave up
    auto flush = [&]() {  // from tensor memory to the registers, the planes' together
        const uint32_t at = memory + ((uint32_t)(warp & 3) << 21) + (uint32_t)(warp >> 2) * By<R>::kN;
        constexpr int H = R == 64 ? 32 : R;  // columns at a time
#pragma unroll
        for (int from = 0; from < R; from += H) {
            float v[H], w[H];
            columns(at + 2 * R + from, v);
            columns(at + R + from, w);
            columns_wait(v);
            columns_wait(w);
#pragma unroll
            for (int e = 0; e < H; ++e) w[e] += v[e];
            columns(at + from, v);
            columns_wait(v);
#pragma unroll
            for (int e = 0; e < H; ++e) sums[from + e] += v[e] + w[e];
        }
    };
#pragma unroll
    for (int r = 0; r < R; ++r) sums[r] = 0.0f;
    int stage = 0, since = 0;
    uint32_t here = 0, empty = 0, ready = 0;  // phases
    for (int step = k.first, turn = 0; step < k.last; step += k.stride, ++turn) {
        if (touch) {
            char* at = at0 + stage * P::kStageBytes;
            const uint32_t row = (ACROSS ? (uint32_t)step * 64 : k.row0) + r0;
            const int64_t column0 = (ACROSS ? (int64_t)k.column0 : (int64_t)step * P::kStep) + c0 * 8;
            if (MAPPED) {
                lost = lost || !barrier_wait(bars + 8 * (P::kLanded + stage), here >> stage & 1u, a.tries);
            } else if (turn >= P::kStages) {
                lost = lost || !barrier_wait(bars + 8 * (P::kEmpty + stage), empty >> stage & 1u, a.tries);
                empty ^= 1u << stage;
            }
            here ^= 1u << stage;
#pragma unroll
            for (int e = 0; e < 8; ++e) {
                uint4* place = reinterpret_cast<uint4*>(at + e * kPlace);
                const uint32_t j = row + (P::kWide ? e & 3 : e) * kRows;
                const int64_t column = column0 + (P::kWide ? (e >> 2) * 64 : 0);
                Raw8<__nv_bfloat16> raw;
                if (MAPPED) {
                    raw.q = *place;
                } else {
                    const bool in = j < a.rows;
                    raw = raw_columns<__nv_bfloat16, false>(x + (in ? (int64_t)j * a.x_rs : 0), (int)min(column, (int64_t)a.h),
                                                            in ? a.h : 0);
                }
                if (a.drop.on) {
                    const uint4 u = drop_words(a.drop, (uint32_t)(column >> 3), j, a.drop.worker + k.worker, call);
                    uint32_t w[1][4];
                    raw_planes<__nv_bfloat16>(raw, a.drop, u, w);
                    raw.q = make_uint4(w[0][0], w[0][1], w[0][2], w[0][3]);
                }
                *place = raw.q;
            }
            fence_shared();
            barrier_arrive(bars + 8 * (P::kTouched + stage));
        }
        if (++since == kFlush || step + k.stride >= k.last) {
            since = 0;
            lost = lost || !barrier_wait(bars + 8 * P::kReady, ready, a.tries);
            ready ^= 1u;
            fence_after();
            flush();
            fence_before();
            barrier_arrive(bars + 8 * P::kDrained);
        }
        stage = stage + 1 == P::kStages ? 0 : stage + 1;
    }
    if (lost) give_up(given_up);
}

// A CTA takes 256 rows of a worker, or 128 (WIDE), and its share of the columns. Rank 64, 8 workers of 2048 rows: 8192 columns, 268 MB,
// 69 us (3.9 TB/s): 128 CTAs of 64 steps, 1.1 us a step, of which the products take 0.4; 56 KB come to a stage, 24 of them planes from the
// L2. 4096 columns with dropout, 134 MB, 69 us, bound by the generator. Rank 16, 4096 columns: 36 and 52 us.
template <int R, bool MAPPED>
__global__ void __launch_bounds__(kThreads, 1) down_kernel(const __grid_constant__ Args a, const __grid_constant__ CUtensorMap map) {
    extern __shared__ __align__(16) char dynamic[];
    using P = Pipe<R, false>;
    __shared__ uint64_t bars[P::kBars];
    __shared__ uint32_t word[2];
    dependency_wait();
    uint32_t memory;
    char* smem = aligned(dynamic);
    tensor_begin<P>(bars, word, By<R>::kColumns, memory);
    const uint32_t tile = blockIdx.x / a.split, i = tile / a.tiles, row0 = (tile - i * a.tiles) * P::kRows;
    const int part = (int)(blockIdx.x - tile * a.split), steps = (a.h + P::kStep - 1) / P::kStep;
    const bool main = threadIdx.x < 256;
    float sums[R];
    int turns = 0;
    const int group = (int)blockIdx.y;
    const Walk walk = {a.image + (int64_t)i * a.image_ws + group * down_group(a.h, a.rank), i, row0, 0, part, a.split, steps};
    if (main) sum_tiles<R, MAPPED, false>(a, walk, smem, memory, shared_address(bars), word + 1, sums);
    else turns = feed<R, MAPPED, false>(a, &map, walk, smem, memory, shared_address(bars), word + 1);
    const float worth = tensor_end<P>(memory, By<R>::kColumns, word + 1, shared_address(bars), turns) ? __int_as_float(0x7fffffff) : 1.0f;
    // this CTA's sums, then its share of the rows, joined over the cluster in order
    constexpr int L = R + 1;
    float *mine = reinterpret_cast<float*>(smem), *whole = mine + 256 * L;
    if (main)
#pragma unroll
        for (int r = 0; r < R; ++r) mine[threadIdx.x * L + r] = worth * sums[r];
    cooperative_groups::cluster_group cluster = cooperative_groups::this_cluster();
    cluster.sync();
    const float scale = a.scale * (a.drop.on ? a.drop.factor : 1.0f);
    const int share = P::kRows / a.split, from = part * share;  // split is a power of two: a share is 32 rows at least
    for (int e = threadIdx.x; e < share * R; e += kThreads) {
        const int r = e / R, j = e % R;
        float sum[kMostSplit], v = 0.0f;
#pragma unroll
        for (int s = 0; s < kMostSplit; ++s) {
            const float* at = s < a.split ? cluster.map_shared_rank(mine, s) + (from + r) * L + j : nullptr;
            sum[s] = at ? (P::kWide ? at[0] + at[128 * L] : at[0]) : 0.0f;
        }
#pragma unroll
        for (int s = 0; s < kMostSplit; ++s) v += sum[s];
        whole[r * L + j] = scale * v;
    }
    __syncthreads();
    const uint32_t first = row0 + from;  // a multiple of 16
    if (a.out)
        for (int e = threadIdx.x; e < share * R; e += kThreads) {
            const int r = e / R, j = e % R;
            if (first + r < a.rows && group * R + j < a.rank) a.out[((int64_t)i * a.rows + first + r) * a.rank + group * R + j] = whole[r * L + j];
        }
    for (int e = threadIdx.x; e < share * (R / 8); e += kThreads) {  // a row's eight ranks
        const int r = e / (R / 8), c = e % (R / 8);
        const uint32_t row = first + r;
        if (row >= (a.rows + 127) / 128 * 128) break;
        float v[8];
#pragma unroll
        for (int k = 0; k < 8; ++k) v[k] = whole[r * L + c * 8 + k];
        uint4 w[3];
        planes8(v, w);
        char* out = a.t_up + i * t_up_image(a.rows, a.rank) + group * t_up_group(a.rows, a.rank) + (int64_t)(row >> 7) * By<R>::kUpBytes;
        store_up<R>(out, row & 127u, c, w);
    }
    if (a.t_outer)
        for (int e = threadIdx.x; e < share / 8 * R; e += kThreads) {  // a rank's eight rows
            const int j = e % R, r = e / R * 8;
            const uint32_t row = first + r;
            if (row >= (a.rows + 63) / 64 * 64) break;
            float v[8];
#pragma unroll
            for (int k = 0; k < 8; ++k) v[k] = whole[(r + k) * L + j];
            uint4 w[3];
            planes8(v, w);
            char* out = a.t_outer + i * t_outer_image(a.rows, a.rank) + group * t_outer_group(a.rows, a.rank) +
                        (int64_t)(row >> 6) * By<R>::kPlanesBytes;
#pragma unroll
            for (int p = 0; p < 3; ++p) *reinterpret_cast<uint4*>(out + swizzled(p * R + j, (row >> 3) & 7u)) = w[p];
        }
    cluster.sync();  // the others may still be reading
}

// A CTA takes 256 columns and a chunk of a worker's rows. Rank 64, 8 workers of 2048 rows: 8192 columns, 268 MB, 57 us (4.7 TB/s), 256 CTAs
// of 32 steps in two waves, 0.9 us a step; 4096 with dropout, 134 MB, 57 us. Rank 16, 4096 columns: 22 us (6.2 TB/s), 49 with dropout.
template <int R, bool MAPPED>
__global__ void __launch_bounds__(kThreads, 1) outer_kernel(const __grid_constant__ Args a, const __grid_constant__ CUtensorMap map) {
    extern __shared__ __align__(16) char dynamic[];
    using P = Pipe<R, true>;
    __shared__ uint64_t bars[P::kBars];
    __shared__ uint32_t word[2];
    dependency_wait();
    uint32_t memory;
    char* smem = aligned(dynamic);
    tensor_begin<P>(bars, word, By<R>::kColumns, memory);
    const uint32_t i = blockIdx.y / a.chunks, chunk = blockIdx.y - i * a.chunks, blocks = (a.rows + 63) / 64;
    const int s0 = (int)((uint64_t)blocks * chunk / a.chunks), s1 = (int)((uint64_t)blocks * (chunk + 1) / a.chunks);
    float sums[R];
    int turns = 0;
    const int group = (int)blockIdx.z;
    const Walk walk = {a.image + (int64_t)i * a.image_ws + group * t_outer_group(a.rows, a.rank), i, 0, (int)blockIdx.x * 256, s0, 1, s1};
    if (threadIdx.x < 256) sum_tiles<R, MAPPED, true>(a, walk, smem, memory, shared_address(bars), word + 1, sums);
    else turns = feed<R, MAPPED, true>(a, &map, walk, smem, memory, shared_address(bars), word + 1);
    const bool gone = tensor_end<P>(memory, By<R>::kColumns, word + 1, shared_address(bars), turns);
    const int64_t c = (int64_t)blockIdx.x * 256 + threadIdx.x;
    if (threadIdx.x >= 256 || c >= a.h) return;
    const float scale = gone ? __int_as_float(0x7fffffff) : a.scale * (a.drop.on ? a.drop.factor : 1.0f);
    float* out = a.out + (int64_t)blockIdx.y * a.rank * a.h + c * a.sc + group * R * a.sj;
    const int ranks = a.rank - group * R;
    if (a.sj == 1 && (a.rank & 3) == 0 && (reinterpret_cast<uintptr_t>(a.out) & 15u) == 0) {
#pragma unroll
        for (int r = 0; r < R; r += 4)
            if (r < ranks)
                *reinterpret_cast<float4*>(out + r) = make_float4(scale * sums[r], scale * sums[r + 1], scale * sums[r + 2], scale * sums[r + 3]);
    } else {
#pragma unroll
        for (int r = 0; r < R; ++r)
            if (r < ranks) out[r * a.sj] = scale * sums[r];
    }
}

// ---- up --------------------------------------------------------------------------------------------------------------------

// A CTA takes CN columns, whose planes of the factor stay in shared memory, and goes through the 128-row tiles of a chunk: the planes of t
// and the base of the next tile are on their way while this one is done; products of 16 rank indices (the planes' indices together at
// most 2, the smallest first); the result into the base's place in shared memory and from there to memory by rows. Two CTAs to an SM: while
// one waits for its products the other's loads run. With 64 ranks there is room for one tile's planes of t: the next are asked for when the
// products are done, so they come while the results leave.
//
// GROUPS: of several groups of 64 ranks. A tile takes a round per group, whose products go onto the same sums, and the factor's planes come
// with t's for every round; one CTA of 128 columns to an SM, and one tile of the base, asked for when the tile before it has left. The
// small products (indices 1 and 2) have a sum of their own over all groups, so that the tensor cores' cuts of the sum are few.
//
// 8 workers of 2048 rows. Rank 16, 4096 columns: 47 us for 268 MB with the base (5.7 TB/s), 69 for dx with dropout, 134 MB: bound by
// memory, and by the generator. Rank 64, 8192 columns: 160 us for 537 MB (3.4 TB/s), 4096 columns for dx with dropout 97; rank 32, 4096
// columns 70 and 81: bound by shared memory, through which six products of planes and the planes of t pass for every tile (one CTA of 128
// columns to an SM reads less and waits more: rank 64 190 and 117, rank 32 78 and 104). Rank 128, 8192 columns 272 us, dx 164.
template <int R, bool GROUPS>
struct Up {
    static constexpr int kColumns = R == 16 || GROUPS ? 128 : 64;                    // CN
    static constexpr int kRow = 2 * kColumns;                                        // bytes of a row of the base's tile
    static constexpr int kFactorTile = kColumns * 128, kFactorBytes = By<R>::kUpTiles * kFactorTile, kFactors = GROUPS ? 2 : 1;
    static constexpr int kTs = R == 64 && !GROUPS ? 1 : 2, kBases = GROUPS ? 1 : 2;  // tiles of t and of the base
    static constexpr int kShared = kFactors * kFactorBytes + kTs * By<R>::kUpBytes + kBases * 128 * kRow + 256;
};

struct UpArgs {
    const void* base;  // may be null
    void* y;
    const char *image, *t_up;
    int64_t base_ws, base_rs, image_ws;
    uint32_t rows, chunks;
    int32_t h, rank;
    uint32_t tries;  // of a wait
    float scale;
    Drop drop;
};

template <int R, bool VEC, bool GROUPS>
__global__ void __launch_bounds__(256, GROUPS ? 1 : 2) up_kernel(const __grid_constant__ UpArgs a) {
    extern __shared__ __align__(1024) char smem[];  // (all of it: nothing static, so it starts on the boundary, and two CTAs fit)
    using B = By<R>;
    using U = Up<R, GROUPS>;
    constexpr int CN = U::kColumns, kRow = U::kRow;
    constexpr uint32_t kMemory = GROUPS ? 2 * CN : CN;
    using P = Pipe<R, true>;
    uint64_t* bars = reinterpret_cast<uint64_t*>(smem + U::kShared - 256);
    uint32_t* word = reinterpret_cast<uint32_t*>(bars + P::kBars);
    bool lost = false;  // a wait of this thread gave up, or one of the CTA's before the last barrier
    dependency_wait();
    uint32_t memory;
    tensor_begin<P>(bars, word, kMemory, memory);
    // a tile of the base: 128 rows, chunk c at c ^ (row % 8)
    char *planes = smem, *t0 = smem + U::kFactors * U::kFactorBytes, *tile0 = t0 + U::kTs * B::kUpBytes;
    const uint32_t i = blockIdx.y / a.chunks, chunk = blockIdx.y - i * a.chunks, blocks = (a.rows + 127) / 128;
    const uint32_t b0 = (uint32_t)((uint64_t)blocks * chunk / a.chunks), b1 = (uint32_t)((uint64_t)blocks * (chunk + 1) / a.chunks);
    const int c0 = (int)blockIdx.x * CN, warp = threadIdx.x >> 5, lane = threadIdx.x & 31;
    const uint32_t call = drop_call(a.drop), bar = shared_address(bars + P::kReady);
    const __nv_bfloat16* base = (const __nv_bfloat16*)a.base + (int64_t)i * a.base_ws;
    __nv_bfloat16* y = (__nv_bfloat16*)a.y + (int64_t)i * a.rows * a.h;
    const int groups = GROUPS ? groups_of(a.rank) : 1;
    const char* t_image = a.t_up + i * t_up_image(a.rows, a.rank);
    const char* factor = a.image + (int64_t)i * a.image_ws + (int64_t)(c0 / 128) * B::kUpBytes + c0 % 128 * 128;
    auto fetch_planes = [&](int group, char* to) {
        const char* from = factor + group * up_group(a.h, a.rank);
#pragma unroll
        for (int p = 0; p < B::kUpTiles; ++p)
#pragma unroll
            for (int k = 0; k < U::kFactorTile / 16 / 256; ++k)
                copy16(to + p * U::kFactorTile + (threadIdx.x + 256 * k) * 16, from + p * kTileBytes + (threadIdx.x + 256 * k) * 16);
    };
    // What a thread brings to a tile it takes away too. VEC: a column of chunks, every (256 / chunks of a row)-th row's; elsewhere a warp has
    // every eighth row and a lane every 32nd element.
    constexpr uint32_t kChunks = CN / 8, kRows = 256 / kChunks;
    const uint32_t r0 = threadIdx.x / kChunks, q0 = threadIdx.x % kChunks, at0 = r0 * kRow + ((q0 ^ (r0 & 7u)) << 4);
    const int column = c0 + (int)q0 * 8;
    auto element = [&](uint32_t row, uint32_t c) { return row * kRow + (((c >> 3) ^ (row & 7u)) << 4) + (c & 7u) * 2; };
    auto tile_of = [&](uint32_t b) { return tile0 + (U::kBases == 2 ? ((b - b0) & 1u) * (128 * kRow) : 0); };
    auto fetch_base = [&](uint32_t b) {
        if (!a.base || b >= b1) return;
        char* tile = tile_of(b);
        if constexpr (VEC) {
            const __nv_bfloat16* x = base + (int64_t)(b * 128 + r0) * a.base_rs + column;
#pragma unroll
            for (uint32_t k = 0; k < 128 / kRows; ++k) {
                const bool in = column < a.h && b * 128 + r0 + kRows * k < a.rows;
                copy16(tile + at0 + k * kRows * kRow, in ? (const void*)(x + k * kRows * a.base_rs) : a.base, in);
            }
        } else {
            for (uint32_t r = warp; r < 128; r += 8)
#pragma unroll
                for (int c = lane; c < CN; c += 32)
                    if (b * 128 + r < a.rows && c0 + c < a.h)
                        *reinterpret_cast<__nv_bfloat16*>(tile + element(r, c)) = __ldg(base + (int64_t)(b * 128 + r) * a.base_rs + c0 + c);
        }
    };
    auto fetch_t = [&](uint32_t b, int group, uint32_t turn) {
        if (b >= b1) return;
        char* t = t0 + (U::kTs == 2 ? (turn & 1u) * B::kUpBytes : 0);
        const char* from = t_image + group * t_up_group(a.rows, a.rank) + (int64_t)b * B::kUpBytes;
        if (GROUPS) fetch_planes(group, planes + (turn & 1u) * U::kFactorBytes);
#pragma unroll
        for (int k = 0; k < B::kUpBytes / 16 / 256; ++k) {
            const uint32_t e = threadIdx.x + 256 * k;
            if (R == 32 && k >= 4 && ((e ^ e >> 3) & 4u)) continue;  // the second tile's empty half
            copy16(t + e * 16, from + e * 16);
        }
    };
    if (!GROUPS) fetch_planes(0, planes);
    fetch_t(b0, 0, 0);
    fetch_base(b0);
    copies_commit();
    uint32_t turn = 0, formed = 0, b = b0;
    for (int group = 0; b < b1; ++turn) {
        const bool last = !GROUPS || group + 1 == groups;
        if constexpr (U::kTs == 2) {
            fetch_t(last ? b + 1 : b, last ? 0 : group + 1, turn + 1);
            if (!GROUPS) fetch_base(b + 1);
            copies_commit();
            copies_wait<1>();  // (GROUPS: the base was asked for in an earlier round than the tile's last)
        } else {
            copies_wait<0>();
        }
        fence_shared();
        fence_before();
        lost = __syncthreads_or(lost);
        char* tile = tile_of(b);
        if (!lost) formed = turn;
        if (threadIdx.x == 0 && !lost) {
            fence_after();
            const uint32_t left = shared_address(t0) + (U::kTs == 2 ? (turn & 1u) * B::kUpBytes : 0);
            const uint32_t right = shared_address(planes) + (GROUPS ? (turn & 1u) * U::kFactorBytes : 0);
#pragma unroll
            for (int both = 2; both >= 0; --both)  // the planes' indices together
#pragma unroll
                for (int p = 0; p <= both; ++p) {
                    const uint32_t l = left + up_tile<R>(p) * kTileBytes + up_byte<R>(p);
                    const uint32_t r = right + up_tile<R>(both - p) * U::kFactorTile + up_byte<R>(both - p);
                    const bool apart = GROUPS && both > 0, fresh = both == 2 ? p == 0 : GROUPS && both == 0;
#pragma unroll
                    for (int k = 0; k < R / 16; ++k)
                        product(memory + (apart ? CN : 0), operand(l + k * 32, 16), operand(r + k * 32, 16), instruction(CN, false, false),
                                !fresh || k > 0 || (GROUPS && group > 0));
                }
            products_done(bar);
        }
        if constexpr (U::kTs == 1) fetch_base(b + 1);
        // a lane's row: CN / 2 columns from CN / 2 (warp / 4) on
        const uint32_t r = (uint32_t)(warp & 3) * 32 + lane, row = b * 128 + r;
        lost = lost || !barrier_wait(bar, turn & 1u, a.tries);
        const float scale = lost ? __int_as_float(0x7fffffff) : a.scale;  // (a thread that did not give up has its sums)
        fence_after();
        if constexpr (U::kTs == 1) {
            fetch_t(b + 1, 0, turn + 1);
            copies_commit();
        }
        if (!last) {
            ++group;
            continue;
        }
#pragma unroll
        for (int part = 0; part < CN / 64; ++part) {
            const int first = (warp >> 2) * (CN / 2) + part * 32;
            float v[32];
            columns(memory + ((uint32_t)(warp & 3) << 21) + first, v);
            columns_wait(v);
            if constexpr (GROUPS) {
                float w[32];
                columns(memory + ((uint32_t)(warp & 3) << 21) + CN + first, w);
                columns_wait(w);
#pragma unroll
                for (int e = 0; e < 32; ++e) v[e] += w[e];
            }
#pragma unroll
            for (int k = 0; k < 4; ++k) {
                const uint32_t c = (uint32_t)(first >> 3) + k;
                uint4* at = reinterpret_cast<uint4*>(tile + r * kRow + ((c ^ (r & 7u)) << 4));
                float x[8] = {};
                if (a.base) raw_floats<__nv_bfloat16>({*at}, x);
#pragma unroll
                for (int e = 0; e < 8; ++e) x[e] = fmaf(scale, v[k * 8 + e], x[e]);
                if (a.drop.on) drop8(a.drop, drop_words(a.drop, (uint32_t)(c0 >> 3) + c, row, a.drop.worker + i, call), x);
                *at = make_uint4(pack(x[0], x[1], __nv_bfloat16()), pack(x[2], x[3], __nv_bfloat16()), pack(x[4], x[5], __nv_bfloat16()),
                                 pack(x[6], x[7], __nv_bfloat16()));
            }
        }
        fence_before();
        __syncthreads();
        if constexpr (VEC) {
            __nv_bfloat16* to = y + (int64_t)(b * 128 + r0) * a.h + column;
#pragma unroll
            for (uint32_t k = 0; k < 128 / kRows; ++k) {
                const uint4 u = *reinterpret_cast<const uint4*>(tile + at0 + k * kRows * kRow);
                if (column < a.h && b * 128 + r0 + kRows * k < a.rows) *reinterpret_cast<uint4*>(to + (int64_t)k * kRows * a.h) = u;
            }
        } else {
            for (uint32_t q = warp; q < 128; q += 8)
#pragma unroll
                for (int c = lane; c < CN; c += 32)
                    if (b * 128 + q < a.rows && c0 + c < a.h)
                        y[(int64_t)(b * 128 + q) * a.h + c0 + c] = *reinterpret_cast<const __nv_bfloat16*>(tile + element(q, c));
        }
        ++b;
        if (GROUPS) fetch_base(b);  // (its copies are counted with the next round's)
        group = 0;
    }
    copies_wait<0>();
    if (__syncthreads_or(lost)) {  // (or: the products of everyone's last wait are done)
        barrier_wait(bar, formed & 1u, kTries);  // the last products, which someone did not wait for
        gave_up = 1;
    }
    tensor_end(memory, kMemory);
}


}  // namespace tensor
}  // namespace
}  // namespace compams
