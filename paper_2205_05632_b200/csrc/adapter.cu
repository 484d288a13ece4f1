// Low-rank adapters beside a projection, on [n, rows, .] activations, every worker (or request) with its own or all with one:
//
//   t_i = dropout(x_i) A_i^T                       [rows, rank]      "down"
//   y_i = base_i + scale t_i B_i^T                 [rows, out]       "up"
//   backward:  dt_i = scale dy_i B_i               down, from the other side
//              dA_i = dt_i^T dropout(x_i)          [rank, in]        "outer"
//              dB_i = scale dy_i^T t_i             [out, rank]       outer
//              dx_i = dropout(dt_i A_i)            up, onto nothing
//
// A, B, t and the gradients of A and B are fp32. An operand element (j, c), rank index j and column c, lies at j * sj + c * sc, so
// the three kernels serve both directions: A is (in, 1), B^T is (1, rank).
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
    float* out;     // down: t; outer: the partial sums [n, chunks, rank * h]
    Factor f;
    int64_t x_ws, x_rs;
    uint32_t rows, total;
    int32_t h, rank;
    uint32_t chunks;
    float scale;
    Drop drop;
};

constexpr int kRankBlock = 8;

// A warp per row and block of 8 rank indices.
template <typename T, bool VEC>
__global__ void __launch_bounds__(256) adapter_down_kernel(const __grid_constant__ AdapterArgs a) {
    dependency_wait();
    const int lane = threadIdx.x & 31, blocks = (a.rank + kRankBlock - 1) / kRankBlock;
    const uint64_t at = (uint64_t)blockIdx.x * 8 + (threadIdx.x >> 5);
    const uint32_t m = (uint32_t)(at / blocks);
    if (m >= a.total) return;
    const int j0 = (int)(at - (uint64_t)m * blocks) * kRankBlock;
    const uint32_t i = m / a.rows, j = m - i * a.rows, call = drop_call(a.drop);
    const T* x = (const T*)a.x + (int64_t)i * a.x_ws + (int64_t)j * a.x_rs;
    const float* f = a.f.p + (int64_t)i * a.f.ws;
    float acc[kRankBlock] = {};
    for (int c0 = 0; c0 < a.h; c0 += kSpan) {
        float v[8];
        span_load<T, VEC>(x, c0, a.h, lane, v);
        if (a.drop.on) span_drop<VEC>(a.drop, c0, j, a.drop.worker + i, call, lane, v);
#pragma unroll
        for (int k = 0; k < 8; ++k) {
            const int c = span_column<VEC>(c0, lane, k);
            if (c < a.h)
#pragma unroll
                for (int r = 0; r < kRankBlock; ++r)
                    if (j0 + r < a.rank) acc[r] = fmaf(v[k], __ldg(f + (j0 + r) * a.f.sj + c * a.f.sc), acc[r]);
        }
    }
#pragma unroll
    for (int r = 0; r < kRankBlock; ++r) {
#pragma unroll
        for (int o = 16; o > 0; o >>= 1) acc[r] += __shfl_xor_sync(0xffffffffu, acc[r], o);
        if (lane == 0 && j0 + r < a.rank) a.out[(int64_t)m * a.rank + j0 + r] = a.scale * acc[r];
    }
}

// A warp per span of a row.
template <typename T, bool VEC>
__global__ void __launch_bounds__(256) adapter_up_kernel(const __grid_constant__ AdapterArgs a) {
    dependency_wait();
    const int lane = threadIdx.x & 31, spans = (a.h + kSpan - 1) / kSpan;
    const uint64_t at = (uint64_t)blockIdx.x * 8 + (threadIdx.x >> 5);
    const uint32_t m = (uint32_t)(at / spans);
    if (m >= a.total) return;
    const int c0 = (int)(at - (uint64_t)m * spans) * kSpan;
    const uint32_t i = m / a.rows, j = m - i * a.rows;
    const float* f = a.f.p + (int64_t)i * a.f.ws;
    const float* t = a.t + (int64_t)m * a.rank;
    float acc[8] = {}, v[8] = {};
    for (int r = 0; r < a.rank; ++r) {
        const float tr = __ldcg(t + r);
#pragma unroll
        for (int k = 0; k < 8; ++k) {
            const int c = span_column<VEC>(c0, lane, k);
            if (c < a.h) acc[k] = fmaf(tr, __ldg(f + r * a.f.sj + c * a.f.sc), acc[k]);
        }
    }
    if (a.x) span_load<T, VEC>((const T*)a.x + (int64_t)i * a.x_ws + (int64_t)j * a.x_rs, c0, a.h, lane, v);
#pragma unroll
    for (int k = 0; k < 8; ++k) v[k] = fmaf(a.scale, acc[k], v[k]);
    if (a.drop.on) span_drop<VEC>(a.drop, c0, j, a.drop.worker + i, drop_call(a.drop), lane, v);
    span_store<T, VEC>((T*)a.y + (int64_t)m * a.h, c0, a.h, lane, v);
}

// A warp per span of the columns, block of 8 rank indices and chunk of a worker's rows.
template <typename T, bool VEC>
__global__ void __launch_bounds__(256) adapter_outer_kernel(const __grid_constant__ AdapterArgs a) {
    dependency_wait();
    const int lane = threadIdx.x & 31, spans = (a.h + kSpan - 1) / kSpan, blocks = (a.rank + kRankBlock - 1) / kRankBlock;
    uint64_t at = (uint64_t)blockIdx.x * 8 + (threadIdx.x >> 5);
    const uint32_t ic = (uint32_t)(at / ((uint64_t)spans * blocks));  // worker and chunk
    at -= (uint64_t)ic * spans * blocks;
    const uint32_t i = ic / a.chunks, chunk = ic - i * a.chunks;
    if ((uint64_t)i * a.rows >= a.total) return;
    const int c0 = (int)(at % spans) * kSpan, r0 = (int)(at / spans) * kRankBlock;
    const uint32_t j0 = (uint32_t)((uint64_t)a.rows * chunk / a.chunks), j1 = (uint32_t)((uint64_t)a.rows * (chunk + 1) / a.chunks);
    const uint32_t call = drop_call(a.drop);
    float acc[kRankBlock][8] = {};
    for (uint32_t j = j0; j < j1; ++j) {
        float v[8];
        span_load<T, VEC>((const T*)a.x + (int64_t)i * a.x_ws + (int64_t)j * a.x_rs, c0, a.h, lane, v);
        if (a.drop.on) span_drop<VEC>(a.drop, c0, j, a.drop.worker + i, call, lane, v);
        const float* t = a.t + ((int64_t)i * a.rows + j) * a.rank + r0;
#pragma unroll
        for (int r = 0; r < kRankBlock; ++r) {
            const float tr = r0 + r < a.rank ? __ldcg(t + r) : 0.0f;
#pragma unroll
            for (int k = 0; k < 8; ++k) acc[r][k] = fmaf(tr, v[k], acc[r][k]);
        }
    }
    float* out = a.out + (int64_t)ic * a.rank * a.h;
#pragma unroll
    for (int r = 0; r < kRankBlock; ++r)
#pragma unroll
        for (int k = 0; k < 8; ++k) {
            const int c = span_column<VEC>(c0, lane, k);
            if (c < a.h && r0 + r < a.rank) out[(r0 + r) * a.f.sj + c * a.f.sc] = a.scale * acc[r][k];
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

uint32_t outer_chunks(const AdapterShape& z, int64_t h) {
    const int64_t tiles = (h + kSpan - 1) / kSpan * ((z.rank + kRankBlock - 1) / kRankBlock) * z.n;
    int64_t c = (148 * 16 + tiles - 1) / tiles;
    const int64_t most = (z.rows + 31) / 32;
    if (c > most) c = most;
    return (uint32_t)(c < 1 ? 1 : c);
}
int64_t outer_floats(const AdapterShape& z, int64_t h) { return (int64_t)z.n * outer_chunks(z, h) * z.rank * h; }

template <typename F>
int by_type(int32_t type, F f) {
    return type == kTypeF32 ? f(float()) : type == kTypeBF16 ? f(__nv_bfloat16()) : f(__half());
}
int launched(cudaError_t e, const char* what) { return e == cudaSuccess ? COMPAMS_OK : cuda_fail(e, what); }
int warps(uint64_t count, uint32_t* ctas) {
    const uint64_t c = (count + 7) / 8;
    if (c > 0x7fffffffu) return COMPAMS_ERR_TOO_LARGE;
    *ctas = (uint32_t)c;
    return COMPAMS_OK;
}

int down(float* out, Rows x, const AdapterShape& z, int64_t h, Factor f, float scale, const Drop& d, cudaStream_t stream) {
    AdapterArgs a = {};
    a.x = x.p; a.x_ws = x.worker_stride; a.x_rs = x.row_stride; a.out = out; a.f = f; a.rows = (uint32_t)z.rows; a.total = z.total();
    a.h = (int32_t)h; a.rank = z.rank; a.scale = scale; a.drop = d;
    uint32_t ctas;
    const int rc = warps((uint64_t)a.total * ((z.rank + kRankBlock - 1) / kRankBlock), &ctas);
    if (rc != COMPAMS_OK) return rc;
    return by_type(x.type, [&](auto t) {
        using T = decltype(t);
        auto kernel = h % 8 == 0 && x.aligned() ? adapter_down_kernel<T, true> : adapter_down_kernel<T, false>;
        return launched(launch_plain(kernel, dim3(ctas), dim3(256), 0, stream, a), "adapter_down");
    });
}

int up(void* y, Rows base, const float* t, const AdapterShape& z, int64_t h, Factor f, float scale, const Drop& d, cudaStream_t stream) {
    AdapterArgs a = {};
    a.x = base.p; a.x_ws = base.worker_stride; a.x_rs = base.row_stride; a.y = y; a.t = t; a.f = f; a.rows = (uint32_t)z.rows;
    a.total = z.total(); a.h = (int32_t)h; a.rank = z.rank; a.scale = scale; a.drop = d;
    uint32_t ctas;
    const int rc = warps((uint64_t)a.total * ((h + kSpan - 1) / kSpan), &ctas);
    if (rc != COMPAMS_OK) return rc;
    return by_type(base.type, [&](auto tt) {
        using T = decltype(tt);
        const bool vec = h % 8 == 0 && (!base.p || base.aligned()) && packed(y, z.rows, h, base.type).aligned();
        auto kernel = vec ? adapter_up_kernel<T, true> : adapter_up_kernel<T, false>;
        return launched(launch_after(kernel, dim3(ctas), dim3(256), stream, a), "adapter_up");
    });
}

// out(j, c) at j * sj + c * sc of every worker's rank * h floats.
int outer(float* out, bool sum_workers, Rows x, const float* t, const AdapterShape& z, int64_t h, int64_t sj, int64_t sc, float scale,
          const Drop& d, float* partial, cudaStream_t stream) {
    AdapterArgs a = {};
    a.x = x.p; a.x_ws = x.worker_stride; a.x_rs = x.row_stride; a.t = t; a.f = {nullptr, 0, sj, sc}; a.rows = (uint32_t)z.rows;
    a.total = z.total(); a.h = (int32_t)h; a.rank = z.rank; a.scale = scale; a.drop = d; a.chunks = outer_chunks(z, h);
    const bool straight = a.chunks == 1 && (!sum_workers || z.n == 1);
    a.out = straight ? out : partial;
    uint32_t ctas;
    int rc = warps((uint64_t)z.n * a.chunks * ((h + kSpan - 1) / kSpan) * ((z.rank + kRankBlock - 1) / kRankBlock), &ctas);
    if (rc != COMPAMS_OK) return rc;
    rc = by_type(x.type, [&](auto tt) {
        using T = decltype(tt);
        auto kernel = h % 8 == 0 && x.aligned() ? adapter_outer_kernel<T, true> : adapter_outer_kernel<T, false>;
        return launched(launch_after(kernel, dim3(ctas), dim3(256), stream, a), "adapter_outer");
    });
    if (rc != COMPAMS_OK || straight) return rc;
    const int64_t len = z.rank * h;
    return launched(launch_after(adapter_join_kernel, dim3((uint32_t)((len + 255) / 256), sum_workers ? 1 : (uint32_t)z.n), dim3(256),
                                 stream, (const float*)partial, out, len, sum_workers ? z.n * a.chunks : a.chunks),
                    "adapter_join");
}

bool float_aligned(const void* p) { return (reinterpret_cast<uintptr_t>(p) & 3u) == 0; }
int64_t padded(int64_t floats) { return (floats + 63) / 64 * 64; }

}  // namespace
}  // namespace compams

using namespace compams;

extern "C" {

int compams_adapter_forward(void* y, float* t, const void* x, const void* base, int32_t type, int32_t n, int64_t rows, int64_t in,
                            int64_t out, int32_t rank, int64_t x_worker_stride, int64_t x_row_stride, int64_t base_worker_stride,
                            int64_t base_row_stride, const float* a, int64_t a_worker_stride, int64_t a_row_stride, const float* b,
                            int64_t b_worker_stride, int64_t b_row_stride, float scale, double p, uint64_t seed, uint32_t call,
                            const int64_t* call_device, uint32_t first_worker, void* cuda_stream) {
    const AdapterShape z{n, rows, in, out, rank};
    Drop d, none;
    if (!z.ok() || !type_known(type) || !make_drop(d, p, seed, call, call_device, first_worker) ||
        !make_drop(none, 0.0, 0, 0, nullptr, 0))
        return COMPAMS_ERR_INVALID_ARG;
    if (rows == 0) return COMPAMS_OK;
    const Rows xin{x, x_worker_stride, x_row_stride, type}, bin{base, base_worker_stride, base_row_stride, type};
    if (!x || !y || !t || !a || !b || !float_aligned(t) || !float_aligned(a) || !float_aligned(b) || !xin.element_aligned() ||
        !bin.element_aligned() || !packed(y, rows, out, type).element_aligned())
        return COMPAMS_ERR_INVALID_ARG;
    const cudaStream_t stream = (cudaStream_t)cuda_stream;
    const int rc = down(t, xin, z, in, {a, a_worker_stride, a_row_stride, 1}, 1.0f, d, stream);
    if (rc != COMPAMS_OK) return rc;
    return up(y, bin, t, z, out, {b, b_worker_stride, 1, b_row_stride}, scale, none, stream);
}

int compams_adapter_workspace_bytes(size_t* bytes, int32_t n, int64_t rows, int64_t in, int64_t out, int32_t rank) {
    const AdapterShape z{n, rows, in, out, rank};
    if (!bytes || !z.ok()) return COMPAMS_ERR_INVALID_ARG;
    const int64_t fa = outer_floats(z, in), fb = outer_floats(z, out);
    *bytes = (size_t)(padded((int64_t)z.total() * rank) + padded(fa > fb ? fa : fb)) * sizeof(float);
    return COMPAMS_OK;
}

int compams_adapter_backward(void* dx, float* da, float* db, int32_t sum_workers, const void* dy, const void* x, const float* t,
                             int32_t type, int32_t n, int64_t rows, int64_t in, int64_t out, int32_t rank, int64_t dy_worker_stride,
                             int64_t dy_row_stride, int64_t x_worker_stride, int64_t x_row_stride, const float* a,
                             int64_t a_worker_stride, int64_t a_row_stride, const float* b, int64_t b_worker_stride,
                             int64_t b_row_stride, float scale, double p, uint64_t seed, uint32_t call, const int64_t* call_device,
                             uint32_t first_worker, void* workspace, size_t workspace_bytes, void* cuda_stream) {
    const AdapterShape z{n, rows, in, out, rank};
    Drop d, none;
    size_t need = 0;
    if (!z.ok() || !type_known(type) || !make_drop(d, p, seed, call, call_device, first_worker) ||
        !make_drop(none, 0.0, 0, 0, nullptr, 0) || compams_adapter_workspace_bytes(&need, n, rows, in, out, rank) != COMPAMS_OK)
        return COMPAMS_ERR_INVALID_ARG;
    const cudaStream_t stream = (cudaStream_t)cuda_stream;
    if (rows == 0) {
        const size_t many = sum_workers ? 1 : n;
        cudaError_t e = da ? cudaMemsetAsync(da, 0, many * rank * in * sizeof(float), stream) : cudaSuccess;
        if (e == cudaSuccess && db) e = cudaMemsetAsync(db, 0, many * rank * out * sizeof(float), stream);
        return launched(e, "adapter_backward");
    }
    const Rows xin{x, x_worker_stride, x_row_stride, type}, gin{dy, dy_worker_stride, dy_row_stride, type};
    if (!dy || !a || !b || (da && !x) || (db && !t) || !workspace || workspace_bytes < need ||
        (reinterpret_cast<uintptr_t>(workspace) & 15u) || !float_aligned(t) || !float_aligned(a) || !float_aligned(b) ||
        !float_aligned(da) || !float_aligned(db) || !xin.element_aligned() || !gin.element_aligned() ||
        !packed(dx, rows, in, type).element_aligned())
        return COMPAMS_ERR_INVALID_ARG;
    float* dt = (float*)workspace;
    float* partial = dt + padded((int64_t)z.total() * rank);
    int rc = COMPAMS_OK;
    if (dx || da) rc = down(dt, gin, z, out, {b, b_worker_stride, 1, b_row_stride}, scale, none, stream);
    if (rc == COMPAMS_OK && db) rc = outer(db, sum_workers, gin, t, z, out, 1, rank, scale, none, partial, stream);
    if (rc == COMPAMS_OK && da) rc = outer(da, sum_workers, xin, dt, z, in, in, 1, 1.0f, d, partial, stream);
    if (rc == COMPAMS_OK && dx) rc = up(dx, {nullptr, 0, 0, type}, dt, z, in, {a, a_worker_stride, a_row_stride, 1}, 1.0f, d, stream);
    return rc;
}

}  // extern "C"
