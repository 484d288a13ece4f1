// The n workers' gradients, one tensor per parameter with a worker in each of its rows, gathered as the rows of G [n, d]; the global norm
// of each worker's gradient over all its tensors; and rows above a largest norm scaled down to it, on the way or where they lie:
//
//   norm_i = sqrt(sum over tensors and elements of g^2)        factor_i = min(1, max_norm / (norm_i + eps))        G_i = factor_i g_i
//
// Bound by memory: g is read for the norm, read again and written, 12 bytes an fp32 element, where a gradient that is above the L2 cannot
// do with less (8 bytes and 4 without clipping). The second reading goes through the tiles from the last to the first, so that what the
// first one left in the L2 is found there. Squares are added in fp32 by fours and in binary64 beyond, in a fixed order, so that the norms
// of a billion elements are good to the last bits and do not change from run to run; fours whose sum leaves the middle of fp32's range
// are squared in binary64 one by one.
//
// The tensors' addresses travel as the kernel's argument, up to kMost of them; a CTA finds its tensor by bisection in the constant bank.
#include <cuda_fp16.h>
#include <cuda_runtime.h>
#include <math.h>
#include <stdint.h>

#include <algorithm>

#include "context.h"
#include "rows.cuh"

namespace compams {
namespace {

constexpr int kMost = 320;           // tensors of one launch: 10 KB of arguments
constexpr int kPiece = 8192;         // elements of a CTA: 8 groups of 4 for each of 256 threads
constexpr int kMostPartials = 256;   // partial sums of a worker and launch: a CTA adds them up at once
constexpr int kNormCtas = 8;         // CTAs of the norm to an SM

struct List {
    const void* src[kMost];     // null: zeros
    int64_t stride[kMost];      // elements from worker to worker
    int64_t dst[kMost];         // first coordinate in the row
    int32_t piece0[kMost + 1];  // first piece of each tensor
    int32_t last[kMost];        // elements of its last piece
    int8_t type[kMost];
    int32_t count;
};
static_assert(sizeof(List) <= 16 * 1024, "kernel argument space");

// A CTA's piece of a worker's gradient.
struct Piece {
    const char* p;  // null: zeros
    int64_t dst;
    int type, len;
};
__device__ __forceinline__ Piece piece_of(const List& c, int piece, int64_t worker) {
    int lo = 0, hi = c.count - 1;
    while (lo < hi) {
        const int mid = (lo + hi + 1) >> 1;
        if (c.piece0[mid] <= piece) lo = mid;
        else hi = mid - 1;
    }
    const int64_t first = (int64_t)(piece - c.piece0[lo]) * kPiece;
    Piece r;
    r.type = c.type[lo];
    r.p = c.src[lo] ? (const char*)c.src[lo] + (worker * c.stride[lo] + first) * (r.type == kTypeF32 ? 4 : 2) : nullptr;
    r.dst = c.dst[lo] + first;
    r.len = piece + 1 == c.piece0[lo + 1] ? c.last[lo] : kPiece;
    return r;
}

__device__ __forceinline__ float widened(const char* p, int type, int at) {
    if (type == kTypeF32) return reinterpret_cast<const float*>(p)[at];
    const uint16_t bits = reinterpret_cast<const uint16_t*>(p)[at];
    return type == kTypeBF16 ? __uint_as_float((uint32_t)bits << 16) : __half2float(__ushort_as_half(bits));
}
// Four elements from `at` on, in the widest accesses that their address allows; cls: its elements past a boundary of four.
__device__ __forceinline__ float4 four(const char* p, int type, int at, int cls) {
    if (type == kTypeF32) return load4_stream(reinterpret_cast<const float*>(p) + at, cls);
    if (type == kTypeBF16) return load4_stream(reinterpret_cast<const bf16_bits*>(p) + at, cls);
    if (cls == 0) {
        const uint2 v = __ldg(reinterpret_cast<const uint2*>(reinterpret_cast<const uint16_t*>(p) + at));
        float4 r;
        unpack(v.x, r.x, r.y, __half());
        unpack(v.y, r.z, r.w, __half());
        return r;
    }
    return make_float4(widened(p, type, at), widened(p, type, at + 1), widened(p, type, at + 2), widened(p, type, at + 3));
}
__device__ __forceinline__ int boundary_class(const char* p, int type) {
    return (int)(reinterpret_cast<uintptr_t>(p) >> (type == kTypeF32 ? 2 : 1)) & 3;
}
__device__ __forceinline__ double squares(float4 v) {
    const float s = fmaf(v.x, v.x, fmaf(v.y, v.y, fmaf(v.z, v.z, v.w * v.w)));
    // below, a square may have lost bits; above, one may be infinite that is not, or is no number
    if (s > 1e-26f && s < 1e37f) return (double)s;
    if (v.x == 0.0f && v.y == 0.0f && v.z == 0.0f && v.w == 0.0f) return 0.0;
    const double x = v.x, y = v.y, z = v.z, w = v.w;
    return __fma_rn(x, x, __fma_rn(y, y, __fma_rn(z, z, w * w)));
}

// TYPE: of all the tensors, or kMixed. partials [worker][launches' partials]: blockIdx.x of this launch's.
constexpr int kMixed = -1;
// 16 workers of 11 million fp32 elements, 704 MB: 114 us (6.2 TB/s); 123 with registers for six CTAs to an SM, 134 for eight.
template <int TYPE>
__global__ void __launch_bounds__(256, 4) norm_kernel(const __grid_constant__ List c, double* __restrict__ partials, int32_t pitch, int32_t pieces) {
    __shared__ double scratch[8];
    const int64_t worker = blockIdx.y;
    double sum = 0.0;
    for (int piece = blockIdx.x; piece < pieces; piece += gridDim.x) {
        Piece s = piece_of(c, piece, worker);
        if (TYPE != kMixed) s.type = TYPE;
        if (!s.p) continue;
        const int past = boundary_class(s.p, s.type), lead = past ? 4 - past : 0;  // elements in front of a boundary
        if (s.len == kPiece) {
            float4 v[8];
#pragma unroll
            for (int u = 0; u < 8; ++u) {
                const int at = lead + (u * 256 + (int)threadIdx.x) * 4;
                v[u] = make_float4(0.f, 0.f, 0.f, 0.f);
                if (at + 3 < kPiece) v[u] = four(s.p, s.type, at, 0);
            }
#pragma unroll
            for (int u = 0; u < 8; ++u) sum += squares(v[u]);
        } else {
            for (int at = lead + (int)threadIdx.x * 4; at + 3 < s.len; at += 1024) sum += squares(four(s.p, s.type, at, 0));
        }
        // up to three in front and three behind
        const int whole = s.len > lead ? (s.len - lead) / 4 * 4 : 0, tail = lead + whole;
        if (threadIdx.x < 3 && (int)threadIdx.x < min(lead, s.len)) sum += squares(make_float4(widened(s.p, s.type, threadIdx.x), 0.f, 0.f, 0.f));
        if (threadIdx.x < 3 && tail + (int)threadIdx.x < s.len)
            sum += squares(make_float4(widened(s.p, s.type, tail + threadIdx.x), 0.f, 0.f, 0.f));
    }
    const double total = block_sum_double<8>(sum, scratch);
    if (threadIdx.x == 0) partials[worker * pitch + blockIdx.x] = total;
}

struct ClipArgs {
    const double* partials;  // null: no norms, no factors
    int32_t pitch;           // of a worker
    int32_t n, pieces;
    double max_norm, eps;
    float* norms;            // written by the CTA of a worker's first piece; may be null
    float* rows;             // [n][row_stride]; null: the tensors themselves
    int64_t row_stride;
};
// A CTA has a piece of a worker, the last first.
__device__ __forceinline__ int64_t worker_of(const ClipArgs& a) { return blockIdx.x % (uint32_t)a.n; }
__device__ __forceinline__ int piece_number(const ClipArgs& a) { return a.pieces - 1 - (int)(blockIdx.x / (uint32_t)a.n); }
// The worker's factor, for the whole CTA; behind dependency_wait().
__device__ __forceinline__ float factor_of(const ClipArgs& a, int64_t worker, int piece) {
    __shared__ double scratch[8];
    __shared__ float shared_factor;
    if (!a.partials) return 1.0f;
    double sum = 0.0;
    for (int p = threadIdx.x; p < a.pitch; p += 256) sum += a.partials[worker * a.pitch + p];
    const double norm = sqrt(block_sum_double<8>(sum, scratch));
    if (threadIdx.x == 0) {
        const double over = norm + a.eps;  // (no number makes the factor none; a gradient of zeros has 1 where max_norm and eps are 0, too)
        shared_factor = isinf(a.max_norm) || over <= a.max_norm ? 1.0f : (float)(a.max_norm / over);
        if (a.norms && piece == 0) a.norms[worker] = (float)norm;
    }
    __syncthreads();
    return shared_factor;
}

// In place: nothing to do for a factor of 1. 16 workers of 11 million elements, all clipped: fp32 315 us (4.5 TB/s; none clipped 69: the CTAs that
// look), bfloat16 253, fp16 252; the norm before it 120, 86 and 187 (fp16 by the kernel for mixed types).
__global__ void __launch_bounds__(256, 4) scale_kernel(const __grid_constant__ List c, const __grid_constant__ ClipArgs a) {
    const int64_t worker = worker_of(a);
    const int piece = piece_number(a);
    const Piece s = piece_of(c, piece, worker);
    dependency_wait();
    const float factor = factor_of(a, worker, piece);
    if (factor == 1.0f || !s.p) return;
    const int past = boundary_class(s.p, s.type), lead = past ? 4 - past : 0;
    auto scale_one = [&](int at) {
        const float x = factor * widened(s.p, s.type, at);
        if (s.type == kTypeF32) reinterpret_cast<float*>(const_cast<char*>(s.p))[at] = x;
        else if (s.type == kTypeBF16) reinterpret_cast<__nv_bfloat16*>(const_cast<char*>(s.p))[at] = __float2bfloat16_rn(x);
        else reinterpret_cast<__half*>(const_cast<char*>(s.p))[at] = __float2half_rn(x);
    };
#pragma unroll 4
    for (int at = lead + (int)threadIdx.x * 4; at + 3 < s.len; at += 1024) {
        char* p = const_cast<char*>(s.p);
        if (s.type == kTypeF32) {
            float4* to = reinterpret_cast<float4*>(reinterpret_cast<float*>(p) + at);
            const float4 v = *to;
            *to = make_float4(factor * v.x, factor * v.y, factor * v.z, factor * v.w);
        } else {
            uint2* to = reinterpret_cast<uint2*>(reinterpret_cast<uint16_t*>(p) + at);
            const uint2 v = *to;
            float x[4];
            if (s.type == kTypeBF16) {
                unpack(v.x, x[0], x[1], __nv_bfloat16());
                unpack(v.y, x[2], x[3], __nv_bfloat16());
                *to = make_uint2(pack(factor * x[0], factor * x[1], __nv_bfloat16()), pack(factor * x[2], factor * x[3], __nv_bfloat16()));
            } else {
                unpack(v.x, x[0], x[1], __half());
                unpack(v.y, x[2], x[3], __half());
                *to = make_uint2(pack(factor * x[0], factor * x[1], __half()), pack(factor * x[2], factor * x[3], __half()));
            }
        }
    }
    const int whole = s.len > lead ? (s.len - lead) / 4 * 4 : 0, tail = lead + whole;
    if (threadIdx.x < 3 && (int)threadIdx.x < min(lead, s.len)) scale_one(threadIdx.x);
    if (threadIdx.x < 3 && tail + (int)threadIdx.x < s.len) scale_one(tail + threadIdx.x);
}

// Gathered: as the rows of a.rows. The same 704 MB, read and written: 210 us (6.7 TB/s); with registers for two CTAs to an SM 316.
template <int TYPE>
__global__ void __launch_bounds__(256, 5) clip_kernel(const __grid_constant__ List c, const __grid_constant__ ClipArgs a) {
    const int64_t worker = worker_of(a);
    const int piece = piece_number(a);
    Piece s = piece_of(c, piece, worker);
    if (TYPE != kMixed) s.type = TYPE;
    dependency_wait();
    const float factor = factor_of(a, worker, piece);
    // groups of four that start on 16-byte boundaries of the row; the first and the last may be partial
    float* out = a.rows + worker * a.row_stride + s.dst;
    const int phase = align_class(out);
    const int cls = s.p ? (boundary_class(s.p, s.type) - phase) & 3 : 0;
    const bool clipped = factor != 1.0f;  // a row that is not is copied, whatever is in it
#pragma unroll
    for (int half = 0; half < 8; half += 4) {
        float4 x[4];
#pragma unroll
        for (int u = 0; u < 4; ++u) {
            const int r = ((half + u) * 256 + (int)threadIdx.x) * 4 - phase;
            x[u] = make_float4(0.f, 0.f, 0.f, 0.f);
            if (s.p && r >= 0 && r + 3 < s.len) x[u] = four(s.p, s.type, r, cls);
        }
#pragma unroll
        for (int u = 0; u < 4; ++u) {
            const int r = ((half + u) * 256 + (int)threadIdx.x) * 4 - phase;
            if (r >= 0 && r + 3 < s.len) {
                if (clipped) x[u] = make_float4(factor * x[u].x, factor * x[u].y, factor * x[u].z, factor * x[u].w);
                *reinterpret_cast<float4*>(out + r) = x[u];
            } else {
                for (int k = 0; k < 4; ++k)
                    if (r + k >= 0 && r + k < s.len) {
                        const float v = s.p ? widened(s.p, s.type, r + k) : 0.0f;
                        out[r + k] = clipped ? factor * v : v;
                    }
            }
        }
    }
    // a row that starts past a boundary leaves up to 3 elements of a full piece beyond the groups above
    const int tail = kPiece - phase + (int)threadIdx.x;
    if (tail < s.len) {
        const float v = s.p ? widened(s.p, s.type, tail) : 0.0f;
        out[tail] = clipped ? factor * v : v;
    }
}

// The one type of a list's tensors, or kMixed.
int type_of(const List& c) {
    for (int k = 1; k < c.count; ++k)
        if (c.type[k] != c.type[0]) return kMixed;
    return c.type[0];
}

// Launches of a call: lists of tensors, and where their partial sums stand.
template <typename F>
int by_lists(const void* const* tensors, const int64_t* strides, const int32_t* types, const int64_t* offsets, int32_t count, F f) {
    static thread_local List c;
    for (int32_t k0 = 0; k0 < count;) {
        int64_t pieces = 0;
        c.count = 0;
        for (; k0 < count && c.count < kMost; ++k0, ++c.count) {
            const int64_t len = offsets[k0 + 1] - offsets[k0], np = (len + kPiece - 1) / kPiece;
            if (pieces + np > 0x3fffffff) break;
            c.src[c.count] = tensors[k0];
            c.stride[c.count] = strides[k0];
            c.dst[c.count] = offsets[k0];
            c.piece0[c.count] = (int32_t)pieces;
            c.last[c.count] = (int32_t)(len - (np - 1) * kPiece);
            c.type[c.count] = (int8_t)types[k0];
            pieces += np;
        }
        c.piece0[c.count] = (int32_t)pieces;
        const int rc = f((const List&)c, (int32_t)pieces);
        if (rc != COMPAMS_OK) return rc;
    }
    return COMPAMS_OK;
}

}  // namespace
}  // namespace compams

using namespace compams;

extern "C" {

int compams_collect_workers_workspace_bytes(size_t* bytes, int32_t n, int32_t count) {
    if (!bytes || n < 1 || n > 65535 || count < 1) return COMPAMS_ERR_INVALID_ARG;
    *bytes = (size_t)n * (size_t)((count + kMost - 1) / kMost + 1) * kMostPartials * sizeof(double);
    return COMPAMS_OK;
}

int compams_collect_workers(float* rows, int64_t row_stride, float* norms, const void* const* tensors, const int64_t* strides,
                            const int32_t* types, const int64_t* offsets, int32_t count, int32_t n, double max_norm, double eps, void* workspace,
                            size_t workspace_bytes, void* cuda_stream) {
    if (!tensors || !strides || !types || !offsets || count < 1 || n < 1 || n > 65535 || offsets[0] < 0 || !(max_norm >= 0.0) || !(eps >= 0.0) ||
        (reinterpret_cast<uintptr_t>(rows) & 3u) || (reinterpret_cast<uintptr_t>(norms) & 3u) || (rows && row_stride < offsets[count] && n > 1))
        return COMPAMS_ERR_INVALID_ARG;
    const bool sums = norms || max_norm < (double)INFINITY;
    if (!rows && !sums) return COMPAMS_ERR_INVALID_ARG;
    int64_t pieces = 0;
    for (int32_t k = 0; k < count; ++k) {
        const int64_t len = offsets[k + 1] - offsets[k];
        if (len < 1 || len > ((int64_t)1 << 40) || !type_known(types[k]) || strides[k] < 0 || strides[k] > ((int64_t)1 << 46) ||
            (reinterpret_cast<uintptr_t>(tensors[k]) & (uintptr_t)(type_bytes(types[k]) - 1)) || (!rows && n > 1 && strides[k] < len && tensors[k]))
            return COMPAMS_ERR_INVALID_ARG;
        pieces += (len + kPiece - 1) / kPiece;
        if (pieces > 0x3fffffff) return COMPAMS_ERR_TOO_LARGE;
    }
    if (pieces * n > 0x7fffffff) return COMPAMS_ERR_TOO_LARGE;
    const cudaStream_t stream = (cudaStream_t)cuda_stream;
    const int32_t lists = (count + kMost - 1) / kMost;
    // a worker's partial sums: as many of each list as its pieces and the SMs call for
    const int32_t each = (int32_t)std::min<int64_t>(kMostPartials, std::max<int64_t>(1, ((int64_t)multiprocessors() * kNormCtas + n - 1) / n));
    const int32_t pitch = lists * each;
    if (sums && (!workspace || (reinterpret_cast<uintptr_t>(workspace) & 7u) || workspace_bytes < (size_t)n * pitch * sizeof(double)))
        return COMPAMS_ERR_INVALID_ARG;
    cudaError_t e = cudaSuccess;
    int32_t list = 0;
    int rc = COMPAMS_OK;
    if (sums)
        rc = by_lists(tensors, strides, types, offsets, count, [&](const List& c, int32_t in) {
            double* to = (double*)workspace + list++ * each;
            const int type = type_of(c);
            const auto kernel = type == kTypeF32 ? norm_kernel<kTypeF32> : type == kTypeBF16 ? norm_kernel<kTypeBF16> : norm_kernel<kMixed>;
            e = launch_plain(kernel, dim3((uint32_t)each, (uint32_t)n), dim3(256), 0, stream, c, to, pitch, in);
            return e == cudaSuccess ? COMPAMS_OK : cuda_fail(e, "gradient_norm");
        });
    if (rc != COMPAMS_OK) return rc;
    bool first = true;
    return by_lists(tensors, strides, types, offsets, count, [&](const List& c, int32_t in) {
        ClipArgs a = {};
        a.partials = sums ? (const double*)workspace : nullptr;
        a.pitch = pitch; a.n = n; a.pieces = in; a.max_norm = max_norm; a.eps = eps; a.norms = first ? norms : nullptr; a.rows = rows;
        a.row_stride = row_stride;
        const dim3 grid((uint32_t)in * (uint32_t)n);
        const int type = type_of(c);
        const auto kernel = !rows ? scale_kernel : type == kTypeF32 ? clip_kernel<kTypeF32> : type == kTypeBF16 ? clip_kernel<kTypeBF16> : clip_kernel<kMixed>;
        e = first && sums ? launch_after(kernel, grid, dim3(256), stream, c, a) : launch_plain(kernel, grid, dim3(256), 0, stream, c, a);
        first = false;
        return e == cudaSuccess ? COMPAMS_OK : cuda_fail(e, "gradient_clip");
    });
}

}  // extern "C"
