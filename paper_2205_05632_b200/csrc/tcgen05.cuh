// What the kernels on tcgen05.mma share: its instructions, barriers and operands, the planes of fp32 numbers, launches in clusters.
#pragma once

#include <cuda.h>  // CUtensorMap
#include <cuda_bf16.h>
#include <cuda_fp16.h>
#include <cuda_runtime.h>
#include <stdint.h>

#include <atomic>

#include "context.h"

namespace compams {
namespace {

// ---- planes ----------------------------------------------------------------------------------------------------------------

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

namespace tensor {

// ---- instructions ----------------------------------------------------------------------------------------------------------

__device__ __forceinline__ uint32_t swizzled(uint32_t row, uint32_t chunk) { return row * 128u + ((chunk ^ (row & 7u)) << 4); }

__device__ __forceinline__ uint32_t shared_address(const void* p) { return (uint32_t)__cvta_generic_to_shared(p); }

__device__ __forceinline__ void barrier_init(uint32_t bar, uint32_t count) {
    asm volatile("mbarrier.init.shared::cta.b64 [%0], %1;" ::"r"(bar), "r"(count) : "memory");
}
__device__ __forceinline__ void barrier_arrive(uint32_t bar) { asm volatile("mbarrier.arrive.shared::cta.b64 _, [%0];" ::"r"(bar) : "memory"); }
// Waits for the phase of this parity to end; gives up after a number of tries, each of which the hardware may hold for a while (0:
// at once, whatever is there).
constexpr uint32_t kTries = 1u << 14;
__device__ __forceinline__ bool barrier_wait(uint32_t bar, uint32_t parity, uint32_t most) {
    uint32_t there = 0, tries = 0;
    do {
        asm volatile("{\n.reg .pred p;\nmbarrier.try_wait.parity.shared::cta.b64 p, [%1], %2;\nselp.u32 %0, 1, 0, p;\n}"
                     : "=r"(there)
                     : "r"(bar), "r"(parity)
                     : "memory");
    } while (!there && ++tries < most);
    return there && most;
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
// A box of a 3-d map, which is in parameter space, to shared memory.
__device__ __forceinline__ void box_load(uint32_t to, const CUtensorMap* map, int column, int row, int worker, uint32_t bar) {
    asm volatile("cp.async.bulk.tensor.3d.shared::cluster.global.tile.mbarrier::complete_tx::bytes [%0], [%1, {%2, %3, %4}], [%5];" ::"r"(to),
                 "l"(map), "r"(column), "r"(row), "r"(worker), "r"(bar)
                 : "memory");
}
// Behind it the values are there.
template <int N>
__device__ __forceinline__ void columns_wait(float (&v)[N]) {
    asm volatile("tcgen05.wait::ld.sync.aligned;" ::: "memory");
#pragma unroll
    for (int k = 0; k < N; ++k) asm volatile("" : "+f"(v[k]));
}

// N columns of a lane's row, 16 at a time.
template <int N>
__device__ __forceinline__ void columns(uint32_t at, float (&v)[N]) {
#pragma unroll
    for (int k = 0; k < N; k += 16) {
        uint32_t r[16];
        asm volatile("tcgen05.ld.sync.aligned.32x32b.x16.b32 {%0,%1,%2,%3,%4,%5,%6,%7,%8,%9,%10,%11,%12,%13,%14,%15}, [%16];"
                     : "=r"(r[0]), "=r"(r[1]), "=r"(r[2]), "=r"(r[3]), "=r"(r[4]), "=r"(r[5]), "=r"(r[6]), "=r"(r[7]), "=r"(r[8]), "=r"(r[9]),
                       "=r"(r[10]), "=r"(r[11]), "=r"(r[12]), "=r"(r[13]), "=r"(r[14]), "=r"(r[15])
                     : "r"(at + k));
#pragma unroll
        for (int e = 0; e < 16; ++e) v[k + e] = __uint_as_float(r[e]);
    }
}

}  // namespace tensor

// ---- host ------------------------------------------------------------------------------------------------------------------

using Encode = decltype(&cuTensorMapEncodeTiled);
// The encoder of tensor maps is the driver's; it is asked for once. Null if there is none.
Encode map_encoder() {
    static const Encode encode = [] {
        void* f = nullptr;
        cudaDriverEntryPointQueryResult found;
        if (cudaGetDriverEntryPoint("cuTensorMapEncodeTiled", &f, cudaEnableDefault, &found) != cudaSuccess || found != cudaDriverEntryPointSuccess)
            f = nullptr;
        return (Encode)f;
    }();
    // It wants the device's context current in its thread, which the first launch sees to; this may come before one.
    static thread_local int bound = -1;
    int device = 0;
    if (cudaGetDevice(&device) == cudaSuccess && device != bound && cudaSetDevice(device) == cudaSuccess) bound = device;
    return encode;
}

int launched(cudaError_t e, const char* what) { return e == cudaSuccess ? COMPAMS_OK : cuda_fail(e, what); }

// Lets a kernel have more than 48 KB of shared memory: asked once for every kernel and device, so always for the most that it may want.
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

// Dynamic shared memory of a launch, and the most that the kernel's launches have, where that differs.
struct Shared {
    size_t bytes, most;
    Shared(size_t all) : bytes(all), most(all) {}
    Shared(size_t some, size_t at_most) : bytes(some), most(at_most) {}
};
// A launch behind another of the same call (or the first), with dynamic shared memory and a cluster along x.
template <typename... KArgs, typename... Args>
cudaError_t launch_sized(void (*kernel)(KArgs...), dim3 grid, int threads, int cluster, Shared shared, bool first, cudaStream_t stream,
                         Args... args) {
    if (shared.bytes > 40 * 1024) {  // (the 48 KB are for a kernel's static part as well)
        const cudaError_t e = allow_shared((const void*)kernel, shared.most);
        if (e != cudaSuccess) return e;
    }
    cudaLaunchConfig_t cfg = {};
    cfg.gridDim = grid;
    cfg.blockDim = dim3(threads);
    cfg.dynamicSmemBytes = shared.bytes;
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

}  // namespace
}  // namespace compams
