// What the operators on [n, rows, h] activations share: element types, spans of 256 columns, the dropout mask.
//
// The leading axis is the worker's, so element (i, j, c) is column c of row j of worker i; rows are packed (column stride 1), the
// other two strides are the caller's. A warp takes a span of 256 columns at a time, eight per lane. Where every row starts on a
// 16-byte boundary and h is a multiple of 8 (VEC) they are eight neighbours, read and written 16 bytes at a time; elsewhere they are
// every 32nd column, one element per access, so that a warp's accesses stay contiguous.
#pragma once

#include <cuda_bf16.h>
#include <cuda_fp16.h>
#include <cuda_runtime.h>
#include <stdint.h>

#include <atomic>

namespace compams {

constexpr int kSpan = 256;

// ---- element types ---------------------------------------------------------------------------------------------------------

__device__ __forceinline__ float to_float(float x) { return x; }
__device__ __forceinline__ float to_float(__nv_bfloat16 x) { return __bfloat162float(x); }
__device__ __forceinline__ float to_float(__half x) { return __half2float(x); }
template <typename T> __device__ __forceinline__ T from_float(float x);
template <> __device__ __forceinline__ float from_float<float>(float x) { return x; }
template <> __device__ __forceinline__ __nv_bfloat16 from_float<__nv_bfloat16>(float x) { return __float2bfloat16_rn(x); }
template <> __device__ __forceinline__ __half from_float<__half>(float x) { return __float2half_rn(x); }

__device__ __forceinline__ void unpack(uint32_t w, float& a, float& b, __nv_bfloat16) {
    a = __uint_as_float(w << 16);
    b = __uint_as_float(w & 0xffff0000u);
}
__device__ __forceinline__ void unpack(uint32_t w, float& a, float& b, __half) {
    const float2 f = __half22float2(*reinterpret_cast<const __half2*>(&w));
    a = f.x;
    b = f.y;
}
__device__ __forceinline__ uint32_t pack(float a, float b, __nv_bfloat16) {
    const __nv_bfloat162 v = __floats2bfloat162_rn(a, b);
    return *reinterpret_cast<const uint32_t*>(&v);
}
__device__ __forceinline__ uint32_t pack(float a, float b, __half) {
    const __half2 v = __floats2half2_rn(a, b);
    return *reinterpret_cast<const uint32_t*>(&v);
}

// Eight neighbours on a 16-byte boundary, as they lie in memory: 16 bytes of a 16-bit type, 32 of fp32.
template <typename T> struct Raw8 { uint4 q; };
template <> struct Raw8<float> { float4 a, b; };

template <typename T> __device__ __forceinline__ Raw8<T> raw_load(const T* p) { return {__ldg(reinterpret_cast<const uint4*>(p))}; }
template <> __device__ __forceinline__ Raw8<float> raw_load<float>(const float* p) {
    return {__ldg(reinterpret_cast<const float4*>(p)), __ldg(reinterpret_cast<const float4*>(p) + 1)};
}
template <typename T> __device__ __forceinline__ void raw_floats(const Raw8<T>& r, float (&v)[8]) {
    unpack(r.q.x, v[0], v[1], T());
    unpack(r.q.y, v[2], v[3], T());
    unpack(r.q.z, v[4], v[5], T());
    unpack(r.q.w, v[6], v[7], T());
}
template <> __device__ __forceinline__ void raw_floats<float>(const Raw8<float>& r, float (&v)[8]) {
    v[0] = r.a.x; v[1] = r.a.y; v[2] = r.a.z; v[3] = r.a.w;
    v[4] = r.b.x; v[5] = r.b.y; v[6] = r.b.z; v[7] = r.b.w;
}
template <typename T> __device__ __forceinline__ void store8(T* p, const float (&v)[8]) {
    uint4 q;
    q.x = pack(v[0], v[1], T());
    q.y = pack(v[2], v[3], T());
    q.z = pack(v[4], v[5], T());
    q.w = pack(v[6], v[7], T());
    *reinterpret_cast<uint4*>(p) = q;
}
template <> __device__ __forceinline__ void store8<float>(float* p, const float (&v)[8]) {
    reinterpret_cast<float4*>(p)[0] = make_float4(v[0], v[1], v[2], v[3]);
    reinterpret_cast<float4*>(p)[1] = make_float4(v[4], v[5], v[6], v[7]);
}

// ---- pairs -------------------------------------------------------------------------------------------------------------------

// Two fp32 numbers that one instruction adds or multiplies, each rounded as by itself: the kernels below are bound by what the SMs can
// issue where they are not by memory.
struct Pair {
    uint64_t u;
};
__device__ __forceinline__ Pair pair(float a, float b) {
    Pair r;
    asm("mov.b64 %0, {%1, %2};" : "=l"(r.u) : "f"(a), "f"(b));
    return r;
}
__device__ __forceinline__ Pair pair(float a) { return pair(a, a); }
__device__ __forceinline__ void halves(Pair x, float& a, float& b) { asm("mov.b64 {%0, %1}, %2;" : "=f"(a), "=f"(b) : "l"(x.u)); }
__device__ __forceinline__ float joint(Pair x) {
    float a, b;
    halves(x, a, b);
    return a + b;
}
__device__ __forceinline__ Pair add(Pair a, Pair b) {
    Pair r;
    asm("add.rn.f32x2 %0, %1, %2;" : "=l"(r.u) : "l"(a.u), "l"(b.u));
    return r;
}
__device__ __forceinline__ Pair mul(Pair a, Pair b) {
    Pair r;
    asm("mul.rn.f32x2 %0, %1, %2;" : "=l"(r.u) : "l"(a.u), "l"(b.u));
    return r;
}
__device__ __forceinline__ Pair fma(Pair a, Pair b, Pair c) {
    Pair r;
    asm("fma.rn.f32x2 %0, %1, %2, %3;" : "=l"(r.u) : "l"(a.u), "l"(b.u), "l"(c.u));
    return r;
}

// ---- asynchronous copies -----------------------------------------------------------------------------------------------------

// Asynchronous copies of 16 bytes into shared memory; zeros where `there` is false (an address in bounds all the same).
__device__ __forceinline__ void copy16(void* shared, const void* global, bool there = true) {
    asm volatile("cp.async.cg.shared.global [%0], [%1], 16, %2;" ::"r"((uint32_t)__cvta_generic_to_shared(shared)), "l"(global),
                 "r"(there ? 16 : 0)
                 : "memory");
}
__device__ __forceinline__ void copies_commit() { asm volatile("cp.async.commit_group;" ::: "memory"); }
template <int N>
__device__ __forceinline__ void copies_wait() { asm volatile("cp.async.wait_group %0;" ::"n"(N) : "memory"); }

// ---- spans -----------------------------------------------------------------------------------------------------------------

// The column of a lane's value k in the span that starts at column c0.
template <bool VEC> __device__ __forceinline__ int span_column(int c0, int lane, int k) {
    return VEC ? c0 + lane * 8 + k : c0 + k * 32 + lane;
}
// A lane's values of a span; `beyond` stands in the columns from h on.
template <typename T, bool VEC>
__device__ __forceinline__ void span_load(const T* __restrict__ row, int c0, int h, int lane, float (&v)[8], float beyond = 0.0f) {
    if (VEC) {
        if (c0 + lane * 8 < h) {
            raw_floats<T>(raw_load<T>(row + c0 + lane * 8), v);
        } else {
#pragma unroll
            for (int k = 0; k < 8; ++k) v[k] = beyond;
        }
    } else {
#pragma unroll
        for (int k = 0; k < 8; ++k) {
            const int c = c0 + k * 32 + lane;
            v[k] = c < h ? to_float(__ldg(row + c)) : beyond;
        }
    }
}
template <typename T, bool VEC>
__device__ __forceinline__ void span_store(T* __restrict__ row, int c0, int h, int lane, const float (&v)[8]) {
    if (VEC) {
        if (c0 + lane * 8 < h) store8<T>(row + c0 + lane * 8, v);
    } else {
#pragma unroll
        for (int k = 0; k < 8; ++k) {
            const int c = c0 + k * 32 + lane;
            if (c < h) row[c] = from_float<T>(v[k]);
        }
    }
}

// The same in pairs: a lane's values 2 p and 2 p + 1.
template <typename T> __device__ __forceinline__ void raw_pairs(const Raw8<T>& r, Pair (&v)[4]) {
    float x[8];
    raw_floats<T>(r, x);
#pragma unroll
    for (int p = 0; p < 4; ++p) v[p] = pair(x[2 * p], x[2 * p + 1]);
}
template <typename T> __device__ __forceinline__ Raw8<T> pack_pairs(const Pair (&v)[4]) {
    float x[8];
#pragma unroll
    for (int p = 0; p < 4; ++p) halves(v[p], x[2 * p], x[2 * p + 1]);
    return {make_uint4(pack(x[0], x[1], T()), pack(x[2], x[3], T()), pack(x[4], x[5], T()), pack(x[6], x[7], T()))};
}
template <> __device__ __forceinline__ Raw8<float> pack_pairs<float>(const Pair (&v)[4]) {
    Raw8<float> r;
    halves(v[0], r.a.x, r.a.y);
    halves(v[1], r.a.z, r.a.w);
    halves(v[2], r.b.x, r.b.y);
    halves(v[3], r.b.z, r.b.w);
    return r;
}
template <typename T> __device__ __forceinline__ void raw_store(T* p, const Raw8<T>& r) { *reinterpret_cast<uint4*>(p) = r.q; }
template <> __device__ __forceinline__ void raw_store<float>(float* p, const Raw8<float>& r) {
    reinterpret_cast<float4*>(p)[0] = r.a;
    reinterpret_cast<float4*>(p)[1] = r.b;
}
template <typename T, bool VEC>
__device__ __forceinline__ void span_load(const T* __restrict__ row, int c0, int h, int lane, Pair (&v)[4], float beyond = 0.0f) {
    float x[8];
    span_load<T, VEC>(row, c0, h, lane, x, beyond);
#pragma unroll
    for (int p = 0; p < 4; ++p) v[p] = pair(x[2 * p], x[2 * p + 1]);
}
// Rounds to T and stores; v becomes what was stored where KEEP.
template <typename T, bool VEC, bool KEEP = false>
__device__ __forceinline__ void span_store(T* __restrict__ row, int c0, int h, int lane, Pair (&v)[4]) {
    if constexpr (VEC) {
        const Raw8<T> r = pack_pairs<T>(v);
        if (c0 + lane * 8 < h) raw_store<T>(row + c0 + lane * 8, r);
        if (KEEP) raw_pairs<T>(r, v);
    } else {
#pragma unroll
        for (int p = 0; p < 4; ++p) {
            float x[2];
            halves(v[p], x[0], x[1]);
#pragma unroll
            for (int k = 0; k < 2; ++k) {
                const T t = from_float<T>(x[k]);
                const int c = c0 + (2 * p + k) * 32 + lane;
                if (c < h) row[c] = t;
                x[k] = to_float(t);
            }
            if (KEEP) v[p] = pair(x[0], x[1]);
        }
    }
}

// ---- dropout ---------------------------------------------------------------------------------------------------------------

// Element c of row j of worker i is kept where a 16-bit number u is at least t = round(65536 p), and then multiplied by
// 65536 / (65536 - t), so that the expectation is exact for the share that is really dropped. u is a half of a word of the
// Philox4x32-10 block (Salmon, Moraes, Dror, Shaw, SC 2011) at counter (c / 8, j, i, call) under the seed's two halves as key:
// word (c % 8) / 2, its low half where c is even. Any kernel finds any element's bit again from its place, so a mask is never
// stored. Sixteen bits per element make one block serve eight, the elements of one 16-byte access: about 10 instructions an element,
// against the 22 or so that a sweep which reads and writes 2 bytes an element has time for at the memory's rate.
struct Drop {
    uint32_t key[20];         // the ten rounds' keys
    uint32_t limit;           // t in the upper 16 bits, less 1; all ones: everything is dropped
    float factor;             // 65536 / (65536 - t)
    uint32_t call;            // added to *call_device
    uint32_t worker;          // the number of the first worker
    const int64_t* call_device;  // may be null
    int32_t on;               // 0: t is 0, nothing is dropped
};

__device__ __forceinline__ uint32_t drop_call(const Drop& d) {
    return d.call + (d.on && d.call_device ? (uint32_t)*d.call_device : 0u);
}

// The block of columns 8 group ... 8 group + 7.
__device__ __forceinline__ uint4 drop_words(const Drop& d, uint32_t group, uint32_t row, uint32_t worker, uint32_t call) {
    uint32_t c0 = group, c1 = row, c2 = worker, c3 = call;
#pragma unroll
    for (int r = 0; r < 10; ++r) {
        const uint64_t a = (uint64_t)0xD2511F53u * c0, b = (uint64_t)0xCD9E8D57u * c2;
        c0 = (uint32_t)(b >> 32) ^ c1 ^ d.key[2 * r];
        c1 = (uint32_t)b;
        c2 = (uint32_t)(a >> 32) ^ c3 ^ d.key[2 * r + 1];
        c3 = (uint32_t)a;
    }
    return make_uint4(c0, c1, c2, c3);
}
// Whether element k of the eight is kept: its half, in the upper 16 bits, is above the limit, whatever the lower 16 are.
__device__ __forceinline__ bool drop_keeps(const Drop& d, const uint4& u, int k) {
    const uint32_t w = k < 2 ? u.x : k < 4 ? u.y : k < 6 ? u.z : u.w;
    return (k & 1 ? w : w << 16) > d.limit;
}
__device__ __forceinline__ void drop8(const Drop& d, const uint4& u, float (&v)[8]) {
#pragma unroll
    for (int k = 0; k < 8; ++k) v[k] = drop_keeps(d, u, k) ? v[k] * d.factor : 0.0f;
}
__device__ __forceinline__ uint32_t drop_bits(const Drop& d, uint32_t group, uint32_t row, uint32_t worker, uint32_t call) {
    const uint4 u = drop_words(d, group, row, worker, call);
    uint32_t bits = 0;
#pragma unroll
    for (int k = 0; k < 8; ++k) bits |= drop_keeps(d, u, k) ? 1u << k : 0u;
    return bits;
}

// Dropout of a lane's values of a span; the whole warp takes part.
template <bool VEC>
__device__ __forceinline__ void span_drop(const Drop& d, int c0, uint32_t row, uint32_t worker, uint32_t call, int lane, float (&v)[8]) {
    if (VEC) {
        drop8(d, drop_words(d, (uint32_t)(c0 >> 3) + lane, row, worker, call), v);
    } else {
        const uint32_t bits = drop_bits(d, (uint32_t)(c0 >> 3) + lane, row, worker, call);
#pragma unroll
        for (int k = 0; k < 8; ++k)
            v[k] = (__shfl_sync(0xffffffffu, bits, k * 4 + (lane >> 3)) >> (lane & 7)) & 1u ? v[k] * d.factor : 0.0f;
    }
}

template <bool VEC>
__device__ __forceinline__ void span_drop(const Drop& d, int c0, uint32_t row, uint32_t worker, uint32_t call, int lane, Pair (&v)[4]) {
    const uint4 u = drop_words(d, (uint32_t)(c0 >> 3) + lane, row, worker, call);
    uint32_t bits = 0;
    if (!VEC)
#pragma unroll
        for (int k = 0; k < 8; ++k) bits |= drop_keeps(d, u, k) ? 1u << k : 0u;
#pragma unroll
    for (int p = 0; p < 4; ++p) {
        float x[2];
        halves(mul(v[p], pair(d.factor)), x[0], x[1]);
#pragma unroll
        for (int k = 0; k < 2; ++k) {
            const int e = 2 * p + k;
            const bool keep = VEC ? drop_keeps(d, u, e) : (__shfl_sync(0xffffffffu, bits, e * 4 + (lane >> 3)) >> (lane & 7)) & 1u;
            x[k] = keep ? x[k] : 0.0f;
        }
        v[p] = pair(x[0], x[1]);
    }
}

// Fills a Drop from the arguments of a call; false where they are out of range.
inline bool make_drop(Drop& d, double p, uint64_t seed, uint32_t call, const int64_t* call_device, uint32_t worker) {
    if (!(p >= 0.0 && p <= 1.0) || (reinterpret_cast<uintptr_t>(call_device) & 7u)) return false;
    const uint32_t t = (uint32_t)(65536.0 * p + 0.5);
    for (uint32_t r = 0; r < 10; ++r) {
        d.key[2 * r] = (uint32_t)seed + r * 0x9E3779B9u;
        d.key[2 * r + 1] = (uint32_t)(seed >> 32) + r * 0xBB67AE85u;
    }
    d.limit = t < 65536u ? (t << 16) - 1u : 0xffffffffu;
    d.factor = t < 65536u ? (float)(65536.0 / (65536.0 - t)) : 0.0f;
    d.call = call;
    d.worker = worker;
    d.call_device = call_device;
    d.on = t > 0;
    return true;
}

// ---- host ------------------------------------------------------------------------------------------------------------------

enum : int32_t { kTypeF32 = 0, kTypeBF16 = 1, kTypeF16 = 2 };

// SMs of the current device; asked once for every device.
inline int multiprocessors() {
    static std::atomic<int> known[64];
    int device = 0, sms = 148;
    if (cudaGetDevice(&device) == cudaSuccess) {
        const int here = device < 64 ? known[device].load(std::memory_order_relaxed) : 0;
        if (here) return here;
        if (cudaDeviceGetAttribute(&sms, cudaDevAttrMultiProcessorCount, device) == cudaSuccess && device < 64)
            known[device].store(sms, std::memory_order_relaxed);
    }
    cudaGetLastError();
    return sms;
}

inline int type_bytes(int32_t type) { return type == kTypeF32 ? 4 : 2; }
inline bool type_known(int32_t type) { return type >= kTypeF32 && type <= kTypeF16; }

// A [n, rows, h] operand as the entry points take it.
struct Rows {
    const void* p;
    int64_t worker_stride, row_stride;
    int32_t type;
    bool aligned() const {  // every row on a 16-byte boundary
        const int64_t e = type_bytes(type);
        return ((reinterpret_cast<uintptr_t>(p) | (uint64_t)(worker_stride * e) | (uint64_t)(row_stride * e)) & 15u) == 0;
    }
    bool strides_ok() const { return worker_stride >= 0 && row_stride >= 0; }
    bool element_aligned() const { return (reinterpret_cast<uintptr_t>(p) & (uintptr_t)(type_bytes(type) - 1)) == 0; }
};
inline Rows packed(const void* p, int64_t rows, int64_t h, int32_t type) { return {p, rows * h, h, type}; }

}  // namespace compams
