// The head's products on tcgen05.mma: one kernel in four forms, which differ in the order of their operands and in what becomes of a tile.
//
//   FORWARD   z = x W^T        x and W along the sum (K-major)      a row's maximum and sum of exponentials in the tile, the target's logit
//   PROBS     z = x W^T        again                                d = (softmax(z) - [target]) g, written as 16-bit planes
//   INPUT     dx = d W         d along the sum, W across it         added up over the pieces and parts of the vocabulary
//   WEIGHT    dW = d^T x       both across the sum                  written
//
// A pair of CTAs takes tiles of 256 x 256 (cta_group::2): each holds 128 rows of the left operand and 128 of the right in shared memory,
// half of what two CTAs of 128 x 256 would read from it and fetch from the L2, and has the sums of its 128 rows in its tensor memory,
// twice (2 x 256 columns): while eight warps take the sums of one stretch, the products of the next go to the other. The tensor cores cut
// their sums, so a stretch is at most 16 products of 64 (up to three pairs of planes) or 8 (more), which are 16, 8, 5 or 1 tiles along the sum,
// one at least, and joins the fp32 registers by rounded additions.
//
// Operands are bf16 or fp16. fp32 numbers are three bf16 planes, and fp16 ones beside fp32 two: the sum then runs over pairs of planes as
// well, listed in the arguments, small ones first.
//
// A tenth warp's thread brings tiles by TMA into the 128-byte swizzle, in both CTAs, to the first CTA's barriers; a ninth's, in the first
// CTA, issues the products. All waits are bounded. Who gives up marks the CTA, and a warp of results whose wait ran out leaves NaN from there on
// and says no more that it has drained anything: so no product goes to sums that another warp has still to take, the products come to an end,
// and with them every other warp's waits. What is finite then is as it would have been.
#pragma once

#include "rows.cuh"
#include "tcgen05.cuh"

namespace compams {
namespace {
namespace head {

using namespace tensor;

// Whoever's wait gave up marks the CTA's shared word and this one, which stays until it is asked for. No size or input should bring it about.
__device__ int32_t gave_up;
__device__ __forceinline__ void give_up(uint32_t* lost) {
    gave_up = 1;
    *lost = 1u;
}

enum Form : int { kForward, kProbs, kInput, kWeight };

constexpr int kTile = 256;          // rows and columns of a pair's tile
constexpr int kHalf = 128 * 128;    // bytes of a CTA's 128 x 64 of an operand's plane
constexpr int kHalves = 12;         // of them there is room for: six stages of one plane each, three of 1 + 3, two of 3 + 3
constexpr int kMostStages = 6;
constexpr int kStaging = 8 * 4096;  // for each of the eight warps two times 32 rows of 64 bytes
constexpr int kShared = 1024 + kHalves * kHalf + kStaging;
// Three groups of four warps at 168 registers; the two that keep sums take 224 and the third keeps 32: no more than the launch has.
constexpr int kThreads = 384;
constexpr int kSumRegisters = 224, kOtherRegisters = 32;
static_assert(256 * kSumRegisters + 128 * kOtherRegisters <= kThreads * 168, "registers of the launch");
// Products of 64 between two additions to the registers, at most (or those of one stage): what is drained of one half of the tensor memory,
// and at a tile's end written, has as long as the products that go to the other. Beside an fp32 weight, 8 workers of 256 bfloat16 rows: 1475 us
// with 8, 1400 with 16; with six pairs of planes nothing is faster and dx is 5.4e-7 off its length instead of 2.1e-7 (1.4e-6 with 32).
__host__ __device__ constexpr int flush_after(int pairs) { return pairs <= 3 ? 16 : 8; }
constexpr int kMostPairs = 6;
// The barriers: a stage has landed (of both CTAs, at the first); its products are done; the sums are ready, and drained (at the first).
constexpr int kFull = 0, kEmpty = kMostStages, kReady = 2 * kMostStages, kDrained = kReady + 2, kStopped = kDrained + 2, kBars = kStopped + 1;

// What a worker's rows of d are multiplied by: a number of its own, or its loss's gradient times `inverse`.
struct Scale {
    const float *own, *dloss, *inverse;
    int64_t stride;  // of dloss
    float factor;
};
__device__ __forceinline__ float scale_of(const Scale& s, int64_t worker) {
    return s.own ? s.own[worker] : s.factor * (s.dloss[worker * s.stride] * s.inverse[worker]);
}

struct Args {
    // the tiles, in this order: batch, part of the sum, row and column in groups of kRaster rows
    int32_t tiles_m, tiles_n, batches, parts;
    // tiles of 64 along the sum: of a segment, and of a part. WEIGHT of all workers together: a worker's rows are a segment; else there is
    // one. A stretch ends with its segment.
    int32_t segments, steps, part_steps;
    // operands: the third coordinate is plane * planes apart + batch * batch apart; where rows and the sum begin
    int32_t left_count, right_count;  // planes of a stage
    int32_t stages, stretch;          // stages there is room for; stages between two additions to the registers
    int32_t pairs;
    uint8_t left_plane[kMostPairs], right_plane[kMostPairs];
    int32_t left_planes, left_batch, left_row, left_sum;
    int32_t right_planes, right_batch, right_row, right_sum;
    int32_t f16;    // operands are fp16 (else bf16)
    uint32_t tries;  // of a wait
    int64_t rows;   // of a batch: rows of the result
    int32_t columns;  // of the result; FORWARD, PROBS: the vocabulary
    int32_t first;  // FORWARD, PROBS: the piece's first column
    // FORWARD, PROBS; rows are numbered through the batches
    const int64_t* target;
    float* target_logit;
    float2* stats;         // FORWARD: [half tile of the vocabulary][all rows]: maximum, sum of exp(z - maximum)
    int64_t all_rows;
    int64_t ignored;
    const float *lse, *row_gradient;  // PROBS: the latter is null where all rows' are 1, 0 for an ignored target
    int32_t probs_planes;
    // PROBS, INPUT, WEIGHT: the third map is of what is written, [plane or part][batch][row][column] from out_first's row on
    int32_t out_type, add;  // add: onto what is there (fp32, where the map serves)
    int32_t out_first;
    void* out;              // where the third map does not serve (rows off 16-byte boundaries); else null
    int64_t out_batch, out_row;  // elements
    Scale scale;            // of a worker
    int64_t worker_rows;
};

constexpr int kRaster = 16;  // (8192 rows, 4096 columns, 100000: 19.7 ms for both passes; 4: 21.1, 8: 20.0, 32: 21.0)

struct Place {
    int32_t batch, part, m, n;
};
__device__ __forceinline__ Place place_of(const Args& a, uint32_t t) {
    Place p;
    const uint32_t plane = (uint32_t)a.tiles_m * a.tiles_n, whole = t / plane, in = t - whole * plane;
    p.batch = (int32_t)(whole / a.parts);
    p.part = (int32_t)(whole - (uint32_t)p.batch * a.parts);
    const uint32_t band = kRaster * (uint32_t)a.tiles_n, group = in / band, left = in - group * band;
    const uint32_t high = min((uint32_t)kRaster, (uint32_t)a.tiles_m - group * kRaster);
    p.n = (int32_t)(left / high);
    p.m = (int32_t)(group * kRaster + (left - (uint32_t)p.n * high));
    return p;
}

// ---- instructions of a pair of CTAs ------------------------------------------------------------------------------------------

__device__ __forceinline__ void pair_alloc(uint32_t to) {  // a whole warp of each CTA
    asm volatile("tcgen05.alloc.cta_group::2.sync.aligned.shared::cta.b32 [%0], 512;" ::"r"(to) : "memory");
    asm volatile("tcgen05.relinquish_alloc_permit.cta_group::2.sync.aligned;" ::: "memory");
}
__device__ __forceinline__ void pair_free(uint32_t at) {
    asm volatile("tcgen05.dealloc.cta_group::2.sync.aligned.b32 %0, 512;" ::"r"(at) : "memory");
}
__device__ __forceinline__ uint32_t cta_rank() {
    uint32_t r;
    asm volatile("mov.u32 %0, %%cluster_ctarank;" : "=r"(r));
    return r;
}
// A shared address of this CTA as the first CTA's.
__device__ __forceinline__ uint32_t at_first(uint32_t address) {
    uint32_t r;
    asm volatile("mapa.shared::cluster.u32 %0, %1, 0;" : "=r"(r) : "r"(address));
    return r;
}
__device__ __forceinline__ void arrive_at(uint32_t cluster_bar) {
    // (what it orders is the reading of tensor memory, which a fence of its own stands in front of; a release for the cluster would wait
    // for the warp's global stores as well)
    asm volatile("mbarrier.arrive.shared::cluster.b64 _, [%0];" ::"r"(cluster_bar) : "memory");
}
__device__ __forceinline__ void pair_box(uint32_t to, const CUtensorMap* map, int x, int y, int z, uint32_t cluster_bar) {
    asm volatile(
        "cp.async.bulk.tensor.3d.cta_group::2.shared::cluster.global.tile.mbarrier::complete_tx::bytes [%0], [%1, {%2, %3, %4}], [%5];" ::"r"(to),
        "l"(map), "r"(x), "r"(y), "r"(z), "r"(cluster_bar)
        : "memory");
}
__device__ __forceinline__ void pair_product(uint32_t d, uint64_t a, uint64_t b, uint32_t what, bool onto) {
    asm volatile("{\n.reg .pred p;\nsetp.ne.u32 p, %4, 0;\ntcgen05.mma.cta_group::2.kind::f16 [%0], %1, %2, %3, p;\n}" ::"r"(d), "l"(a), "l"(b),
                 "r"(what), "r"((uint32_t)onto)
                 : "memory");
}
// Tells the barrier at this place in both CTAs when the products so far are done.
__device__ __forceinline__ void pair_done(uint32_t bar) {
    asm volatile("tcgen05.commit.cta_group::2.mbarrier::arrive::one.shared::cluster.multicast::cluster.b64 [%0], %1;" ::"r"(bar), "h"((uint16_t)3)
                 : "memory");
}
__device__ __forceinline__ void cluster_sync() {
    asm volatile("barrier.cluster.arrive.release.aligned;\nbarrier.cluster.wait.acquire.aligned;" ::: "memory");
}
// M = 256, N = 256.
__host__ __device__ constexpr uint32_t pair_instruction(bool bf16, bool left_across, bool right_across) {
    return 1u << 4 | (bf16 ? 1u << 7 | 1u << 10 : 0u) | (left_across ? 1u : 0u) << 15 | (right_across ? 1u : 0u) << 16 | (256u >> 3) << 17 |
           (256u >> 4) << 24;
}

template <int FORM> struct Order {
    static constexpr bool kLeftAcross = FORM == kWeight, kRightAcross = FORM == kInput || FORM == kWeight;
};

// One lane of a warp whose lanes are together.
__device__ __forceinline__ bool elected() {
    uint32_t is;
    asm volatile("{\n.reg .pred p;\nelect.sync _|p, 0xffffffff;\nselp.u32 %0, 1, 0, p;\n}" : "=r"(is));
    return is != 0u;
}

// A wait of a warp, which gives up as one.
__device__ __forceinline__ bool warp_wait(uint32_t bar, uint32_t parity, uint32_t tries) {
    return __all_sync(0xffffffffu, barrier_wait(bar, parity, tries));
}

// ---- the parts ---------------------------------------------------------------------------------------------------------------

__device__ __forceinline__ void steps_of(const Args& a, const Place& p, int& k0, int& k1) {
    k0 = p.part * a.part_steps;
    k1 = min(a.steps, k0 + a.part_steps);
}

// The tenth warp, in both CTAs. (It and the ninth stay together and elect a lane for what one thread does: so all that the instructions
// take is the same for the warp and is held in its uniform registers. With one thread on its own a stage's four products cost 700 cycles to
// issue, where the products take 512.)
template <int FORM>
__device__ __forceinline__ void bring(const Args& a, const CUtensorMap* left, const CUtensorMap* right, uint32_t tiles, char* smem, uint32_t bars,
                                      uint32_t rank, uint32_t* lost) {
    using O = Order<FORM>;
    const uint32_t bars0 = at_first(bars), mem = shared_address(smem);
    int stage = 0;
    uint32_t phase = 1;  // of a stage's first round there is nothing to wait for: the phase before it counts as ended
    for (uint32_t t = blockIdx.x / 2; t < tiles; t += gridDim.x / 2) {
        const Place p = place_of(a, t);
        int k0, k1;
        steps_of(a, p, k0, k1);
        const int m = a.left_row + p.m * kTile + (int)rank * 128, n = a.right_row + p.n * kTile + (int)rank * 128;
        for (int segment = 0, k = k0; segment < a.segments && k < k1; k + 1 < k1 ? ++k : (k = k0, ++segment)) {
            const int ls = a.left_sum + k * 64, rs = a.right_sum + k * 64;
            int lz = (p.batch + segment) * a.left_batch, rz = (p.batch + segment) * a.right_batch;
            if (!warp_wait(bars + 8 * (kEmpty + stage), phase, a.tries)) {
                give_up(lost);
                return;
            }
            const uint32_t bar = bars0 + 8 * (kFull + stage);
            uint32_t to = mem + stage * (a.left_count + a.right_count) * kHalf;
            if (elected()) {
                if (rank == 0) mbar_expect(bars + 8 * (kFull + stage), 2 * (a.left_count + a.right_count) * kHalf);
                for (int c = 0; c < a.left_count; ++c, lz += a.left_planes, to += kHalf) {
                    if (O::kLeftAcross) {
                        pair_box(to, left, m, ls, lz, bar);
                        pair_box(to + 8192, left, m + 64, ls, lz, bar);
                    } else {
                        pair_box(to, left, ls, m, lz, bar);
                    }
                }
                for (int c = 0; c < a.right_count; ++c, rz += a.right_planes, to += kHalf) {
                    if (O::kRightAcross) {
                        pair_box(to, right, n, rs, rz, bar);
                        pair_box(to + 8192, right, n + 64, rs, rz, bar);
                    } else {
                        pair_box(to, right, rs, n, rz, bar);
                    }
                }
            }
            __syncwarp();
            if (++stage == a.stages) {
                stage = 0;
                phase ^= 1u;
            }
        }
    }
}

// The ninth warp, in the first CTA.
template <int FORM>
__device__ __forceinline__ void issue(const Args& a, uint32_t tiles, char* smem, uint32_t memory, uint32_t bars, uint32_t* lost) {
    using O = Order<FORM>;
    const uint32_t mem = shared_address(smem), size = (a.left_count + a.right_count) * (kHalf / 16);
    const uint64_t left0 = operand(mem, O::kLeftAcross ? 8192 : 16), right0 = operand(mem + a.left_count * kHalf, O::kRightAcross ? 8192 : 16);
    constexpr uint32_t kLeft = (O::kLeftAcross ? 2048 : 32) / 16, kRight = (O::kRightAcross ? 2048 : 32) / 16;  // to the next 16 of the sum
    const uint32_t what = pair_instruction(!a.f16, O::kLeftAcross, O::kRightAcross);
    int stage = 0;
    uint32_t phase = 0, buffer = 0, drained = 3;  // a bit for each half of the tensor memory; nothing is to be drained at first
    for (uint32_t t = blockIdx.x / 2; t < tiles; t += gridDim.x / 2) {
        const Place p = place_of(a, t);
        int k0, k1;
        steps_of(a, p, k0, k1);
        const int all = k1 - k0;
        for (int segment = 0, done = 0; segment < a.segments && all > 0; done < all ? 0 : (done = 0, ++segment)) {
            const int end = min(done + a.stretch, all);
            if (!warp_wait(bars + 8 * (kDrained + buffer), drained >> buffer & 1u, a.tries)) {
                give_up(lost);
                return;
            }
            drained ^= 1u << buffer;
            fence_after();
            for (bool onto = false; done < end; ++done) {
                if (!warp_wait(bars + 8 * (kFull + stage), phase, a.tries)) {
                    give_up(lost);
                    return;
                }
                fence_after();
                if (elected()) {
                    for (int pair = 0; pair < a.pairs; ++pair) {
                        const uint64_t l = left0 + (uint32_t)(stage * size + a.left_plane[pair] * (kHalf / 16));
                        const uint64_t r = right0 + (uint32_t)(stage * size + a.right_plane[pair] * (kHalf / 16));
#pragma unroll
                        for (uint32_t q = 0; q < 4; ++q)
                            pair_product(memory + buffer * kTile, l + q * kLeft, r + q * kRight, what, onto || pair > 0 || q > 0);
                    }
                    pair_done(bars + 8 * (kEmpty + stage));
                }
                __syncwarp();
                onto = true;
                if (++stage == a.stages) {
                    stage = 0;
                    phase ^= 1u;
                }
            }
            if (elected()) pair_done(bars + 8 * (kReady + buffer));
            __syncwarp();
            buffer ^= 1u;
        }
    }
}

// 32 rows of 64 bytes of a warp's staging, chunk c of row r at c ^ (r / 2 % 4): the order of TMA's 64-byte swizzle.
__device__ __forceinline__ uint32_t staged(uint32_t row, uint32_t chunk) { return row * 64u + ((chunk ^ (row >> 1 & 3u)) << 4); }

// How the warps' results leave: 64 bytes of each of a warp's 32 rows at a time, from two places by turns.
struct Exit {
    char* places;
    const CUtensorMap* map;
    uint32_t turn;
    // The place to write to next; what was brought from it before is gone.
    __device__ __forceinline__ char* place() {
        if ((threadIdx.x & 31) == 0) asm volatile("cp.async.bulk.wait_group.read 1;" ::: "memory");
        __syncwarp();
        return places + turn * 2048;
    }
    __device__ __forceinline__ void leave(int column, int row, int z, bool add) {
        fence_shared();
        __syncwarp();
        if ((threadIdx.x & 31) == 0) {
            const uint32_t from = shared_address(places + turn * 2048);
            if (add)
                asm volatile("cp.reduce.async.bulk.tensor.3d.global.shared::cta.add.tile.bulk_group [%0, {%1, %2, %3}], [%4];" ::"l"(map),
                             "r"(column), "r"(row), "r"(z), "r"(from)
                             : "memory");
            else
                asm volatile("cp.async.bulk.tensor.3d.global.shared::cta.tile.bulk_group [%0, {%1, %2, %3}], [%4];" ::"l"(map), "r"(column), "r"(row),
                             "r"(z), "r"(from)
                             : "memory");
            asm volatile("cp.async.bulk.commit_group;" ::: "memory");
        }
        turn ^= 1u;
    }
    // Element by element, for rows that TMA cannot address: `count` of the columns and `rows` of the rows are there.
    template <typename T>
    __device__ __forceinline__ void leave_slowly(T* out, int64_t row, int rows, int count) {
        __syncwarp();
        constexpr int N = 64 / (int)sizeof(T);
        const char* from = places + turn * 2048;
        for (int e = threadIdx.x & 31; e < 32 * N; e += 32) {
            const int r = e / N, c = e % N;
            if (r < rows && c < count) {
                out[r * row + c] = *reinterpret_cast<const T*>(from + staged(r, c * sizeof(T) / 16) + c * sizeof(T) % 16);
            }
        }
        __syncwarp();
    }
    __device__ __forceinline__ void end() {
        if ((threadIdx.x & 31) == 0) asm volatile("cp.async.bulk.wait_group 0;" ::: "memory");
        __syncwarp();
    }
};

// Two values as one plane of the 16-bit type; what the plane leaves out stays in them.
__device__ __forceinline__ uint32_t plane_of(float& a, float& b, bool f16, bool last) {
    if (f16) return pack(a, b, __half());
    if (last) return pack(a, b, __nv_bfloat16());
    const uint32_t w = pack(a, b, __nv_bfloat16());
    a -= __uint_as_float(w << 16);
    b -= __uint_as_float(w & 0xffff0000u);
    return w;
}

constexpr float kLog2e = 1.4426950408889634f;
__device__ __forceinline__ float power2(float x) {  // within two units of the last place; 0 below 2^-126
    float y;
    asm("ex2.approx.ftz.f32 %0, %1;" : "=f"(y) : "f"(x));
    return y;
}
// fp16 holds d times this, so that probabilities down to 2^-38 are there; |d| <= 1. (The workers' scales have its inverse.)
constexpr float kF16Scale = 16384.0f;

// The first eight warps. A thread has row 32 (warp % 4) + lane of the CTA's 128 and 128 columns, from 128 (warp / 4) on.
template <int FORM>
__device__ __forceinline__ void finish(const Args& a, const CUtensorMap* map, uint32_t tiles, char* staging0, uint32_t memory, uint32_t bars, uint32_t rank, uint32_t* given_up) {
    const int warp = threadIdx.x >> 5, lane = threadIdx.x & 31, half = warp >> 2;
    const uint32_t at = memory + ((uint32_t)(warp & 3) << 21) + (uint32_t)half * 128;
    const uint32_t drained0 = at_first(bars + 8 * kDrained);
    Exit exit = {staging0 + warp * 4096, map, 0u};
    uint32_t buffer = 0, ready = 0;  // a bit for each half of the tensor memory
    bool lost = false;
    for (uint32_t t = blockIdx.x / 2; t < tiles; t += gridDim.x / 2) {
        const Place p = place_of(a, t);
        int k0, k1;
        steps_of(a, p, k0, k1);
        const int all = k1 - k0;
        float sum[128];
#pragma unroll
        for (int c = 0; c < 128; ++c) sum[c] = 0.0f;
        for (int segment = 0, done = 0; segment < a.segments && all > 0; done + a.stretch < all ? done += a.stretch : (done = 0, ++segment)) {
            const float worth = FORM == kWeight ? scale_of(a.scale, p.batch + segment) : 1.0f;
            lost = lost || !warp_wait(bars + 8 * (kReady + buffer), ready >> buffer & 1u, a.tries);
            ready ^= 1u << buffer;
            fence_after();
#pragma unroll
            for (int c = 0; c < 128; c += 32) {
                float v[32];
                columns(at + buffer * kTile + c, v);
                columns_wait(v);
#pragma unroll
                for (int e = 0; e < 32; ++e) sum[c + e] = FORM == kWeight ? fmaf(worth, v[e], sum[c + e]) : sum[c + e] + v[e];
            }
            fence_before();
            __syncwarp();
            if (lane == 0 && !lost) arrive_at(drained0 + 8 * buffer);
            buffer ^= 1u;
        }
        const int row0 = p.m * kTile + (int)rank * 128 + (warp & 3) * 32;  // of the warp, in the batch
        const int64_t row = row0 + lane;
        const int column0 = p.n * kTile + half * 128;  // in the piece, or of the result
        const bool there = row < a.rows;
        const float nan = __int_as_float(0x7fffffff);
        if constexpr (FORM == kForward || FORM == kProbs) {
            const int64_t number = (int64_t)p.batch * a.rows + row;
            const int left = a.columns - (a.first + column0);  // columns from here on
            const int64_t target = there ? a.target[number] : -1, wanted_at = target - a.first - column0;
            const int mine = target >= 0 && wanted_at >= 0 && wanted_at < min(left, 128) ? (int)wanted_at : -1;
            if constexpr (FORM == kForward) {
                float top = __int_as_float(0xff800000);
#pragma unroll
                for (int c = 0; c < 128; ++c) top = fmaxf(top, c < left ? sum[c] : top);
                const float base = top == __int_as_float(0xff800000) ? 0.0f : top;  // nothing but -inf here: a sum of 0
                float total = 0.0f, wanted = 0.0f;
#pragma unroll
                for (int c = 0; c < 128; ++c) {
                    total += c < left ? power2((sum[c] - base) * kLog2e) : 0.0f;
                    if (c == mine) wanted = sum[c];
                }
                if (there && left > 0) {
                    a.stats[((a.first + column0) >> 7) * a.all_rows + number] = lost ? make_float2(nan, nan) : make_float2(top, total);
                    if (mine >= 0) a.target_logit[number] = wanted;
                }
            } else {
                const float lse = there ? a.lse[number] : 0.0f;
                float g = 0.0f;
                if (there) g = a.row_gradient ? a.row_gradient[number] : target == a.ignored ? 0.0f : target >= 0 && target < a.columns ? 1.0f : nan;
                if (lost) g = nan;
                const float scale = a.f16 ? g * kF16Scale : g;
#pragma unroll
                for (int c = 0; c < 128; ++c) {
                    const float d = power2((sum[c] - lse) * kLog2e) - (c == mine ? 1.0f : 0.0f);
                    sum[c] = c < left && g != 0.0f ? d * scale : 0.0f;
                }
                if (row0 >= a.rows) continue;
                for (int plane = 0; plane < a.probs_planes; ++plane) {
                    const bool last = plane + 1 == a.probs_planes;
#pragma unroll
                    for (int part = 0; part < 4; ++part) {
                        char* place = exit.place();
#pragma unroll
                        for (int c = 0; c < 4; ++c) {
                            uint32_t w[4];
#pragma unroll
                            for (int q = 0; q < 4; ++q) {
                                const int e = part * 32 + c * 8 + q * 2;
                                w[q] = plane_of(sum[e], sum[e + 1], a.f16, last);
                            }
                            *reinterpret_cast<uint4*>(place + staged(lane, c)) = make_uint4(w[0], w[1], w[2], w[3]);
                        }
                        exit.leave(column0 + part * 32, row0, plane * a.batches + p.batch, false);
                    }
                }
            }
        } else {
            float scale = 1.0f;
            if (FORM == kInput && a.scale.factor != 0.0f) scale = there ? scale_of(a.scale, ((int64_t)p.batch * a.rows + row) / a.worker_rows) : 0.0f;
            if (lost) scale = nan;
            const int rows = (int)min((int64_t)32, a.rows - row0), left = a.columns - column0, z = p.part * a.batches + p.batch;
            const int64_t first = z * a.out_batch + (row0 + a.out_first) * a.out_row + column0;
            if (rows <= 0) continue;
            if (a.out_type == kTypeF32) {
#pragma unroll
                for (int part = 0; part < 8; ++part) {
                    if (part * 16 >= left) break;
                    char* place = exit.place();
#pragma unroll
                    for (int c = 0; c < 4; ++c) {
                        const float* v = &sum[part * 16 + c * 4];
                        *reinterpret_cast<float4*>(place + staged(lane, c)) = make_float4(scale * v[0], scale * v[1], scale * v[2], scale * v[3]);
                    }
                    if (!a.out) exit.leave(column0 + part * 16, row0 + a.out_first, z, a.add);
                    else exit.leave_slowly((float*)a.out + first + part * 16, a.out_row, rows, left - part * 16);
                }
            } else {
#pragma unroll
                for (int part = 0; part < 4; ++part) {
                    if (part * 32 >= left) break;
                    char* place = exit.place();
#pragma unroll
                    for (int c = 0; c < 4; ++c) {
                        uint32_t w[4];
#pragma unroll
                        for (int q = 0; q < 4; ++q) {
                            const float x = scale * sum[part * 32 + c * 8 + q * 2], y = scale * sum[part * 32 + c * 8 + q * 2 + 1];
                            w[q] = a.out_type == kTypeBF16 ? pack(x, y, __nv_bfloat16()) : pack(x, y, __half());
                        }
                        *reinterpret_cast<uint4*>(place + staged(lane, c)) = make_uint4(w[0], w[1], w[2], w[3]);
                    }
                    if (!a.out) exit.leave(column0 + part * 32, row0 + a.out_first, z, false);
                    else exit.leave_slowly((uint16_t*)a.out + first + part * 32, a.out_row, rows, left - part * 32);
                }
            }
        }
    }
    if (FORM != kForward) exit.end();
    if (lost) give_up(given_up);
}

template <int FORM>
__global__ void __launch_bounds__(kThreads, 1) head_kernel(const __grid_constant__ Args a, const __grid_constant__ CUtensorMap left,
                                                           const __grid_constant__ CUtensorMap right, const __grid_constant__ CUtensorMap out) {
    extern __shared__ __align__(16) char dynamic[];
    __shared__ uint64_t barriers[kBars];
    __shared__ uint32_t word[2];  // the tensor memory's address; whether someone gave up
    char* smem = dynamic + ((1024u - (shared_address(dynamic) & 1023u)) & 1023u);
    const uint32_t bars = shared_address(barriers), rank = cta_rank(), warp = __shfl_sync(0xffffffffu, threadIdx.x >> 5, 0);
    if (threadIdx.x < 32) pair_alloc(shared_address(word));
    if (threadIdx.x == 32) {
        word[1] = 0u;
        for (int k = 0; k < kBars; ++k) barrier_init(bars + 8 * k, k >= kDrained && k < kStopped ? 16u : 1u);
        asm volatile("fence.mbarrier_init.release.cluster;" ::: "memory");
        fence_shared();
    }
    fence_before();
    __syncthreads();
    cluster_sync();
    fence_after();
    const uint32_t memory = word[0];
    const uint32_t tiles = (uint32_t)a.tiles_m * a.tiles_n * a.batches * a.parts;
    dependency_wait();
    if (threadIdx.x < 256) {
        asm volatile("setmaxnreg.inc.sync.aligned.u32 %0;" ::"n"(kSumRegisters));
        finish<FORM>(a, &out, tiles, smem + kHalves * kHalf, memory, bars, rank, word + 1);
    } else {
        asm volatile("setmaxnreg.dec.sync.aligned.u32 %0;" ::"n"(kOtherRegisters));
        if (warp == 8 && rank == 0) issue<FORM>(a, tiles, smem, memory, bars, word + 1);
        else if (warp == 9) bring<FORM>(a, &left, &right, tiles, smem, bars, rank, word + 1);
    }
    __syncwarp();
    fence_before();
    __syncthreads();
    if (word[1]) {
        // products and copies may be under way that nobody waited for: the products are waited for, with a limit, and the copies are given
        // a millisecond, a hundred times what they take
        if (warp == 8 && rank == 0) {
            if (elected()) pair_done(bars + 8 * kStopped);
            __syncwarp();
            barrier_wait(bars + 8 * kStopped, 0, kTries);
        }
        if (threadIdx.x == 288)
            for (int k = 0; k < 1000; ++k) __nanosleep(1000);
        __syncwarp();
        __syncthreads();
    }
    cluster_sync();  // the other CTA's barriers and tensor memory are used until here
    fence_after();
    if (threadIdx.x < 32) pair_free(memory);
}

}  // namespace head
}  // namespace
}  // namespace compams
