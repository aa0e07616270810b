// serve.cuh -- what the serving kernels share (prompt.cu, paged.cu,
// paged_attention.cu): the status word of their workspaces, element loads,
// the host's checks of pointers and strides.
#pragma once

#include <cuda_bf16.h>
#include <cuda_runtime.h>
#include <stdint.h>

#include "../../include/gracekv.h"

namespace gkv {
namespace serve {

// A workspace begins with 256 bytes whose first word collects these bits.
constexpr int kStTimeout = 1;      // a bounded device-side wait gave up
constexpr int kStRange = 2;        // a page number, length, offset or cu word was not followed
constexpr size_t kWsHead = 256;
constexpr int kMaxDevices = 64;
constexpr float kLog2e = 1.4426950408889634f;

inline bool al(const void *p, uintptr_t m) { return (reinterpret_cast<uintptr_t>(p) & (m - 1)) == 0; }

inline int elem_bytes(int dtype) { return dtype == GKV_BF16 ? 2 : 4; }

// A tensor of token rows and heads: its pointer and strides (elements).
inline bool rows_ok(const void *p, int64_t ts, int64_t hs, int dtype) {
    const int64_t q = 16 / elem_bytes(dtype);
    return p && al(p, 16) && ts >= 0 && hs >= 0 && ts % q == 0 && hs % q == 0 && ts < (1LL << 40) && hs < (1LL << 40);
}

// The same for a tensor that is written: no two of its n x heads rows of d share an element by one stride alone.
inline bool out_ok(const void *p, int64_t ts, int64_t hs, int dtype, int64_t n, int heads, int d) {
    return rows_ok(p, ts, hs, dtype) && (n < 2 || ts >= d) && (heads < 2 || hs >= d);
}

// The sequence holding row i: the last s with cu[s] <= i.  cu is [n + 1],
// n >= 1; any contents end the search inside [0, n).
__device__ __forceinline__ int seq_of(const int32_t *cu, int n, int64_t i) {
    int lo = 0, hi = n;
    while (hi - lo > 1) {
        const int mid = (lo + hi) >> 1;
        if (cu[mid] <= i) lo = mid; else hi = mid;
    }
    return lo;
}

inline gkv_status read_status(void *workspace, void *stream) {
    if (!workspace || !al(workspace, 256)) return GKV_EINVAL;
    cudaStream_t s = static_cast<cudaStream_t>(stream);
    int h = 0;
    if (cudaMemcpyAsync(&h, workspace, sizeof(int), cudaMemcpyDeviceToHost, s) != cudaSuccess) return GKV_ECUDA;
    if (cudaStreamSynchronize(s) != cudaSuccess) return GKV_ECUDA;
    if (h == 0) return GKV_OK;
    if (cudaMemsetAsync(workspace, 0, sizeof(int), s) != cudaSuccess) return GKV_ECUDA;
    return (h & kStRange) ? GKV_EINVAL : GKV_ETIMEOUT;
}

// Launches of one stream overlap at their ends: a kernel lets the next one
// start when all its own blocks run (next_may_start), and waits for the whole of
// the one before, and for what it wrote, before it reads anything that a
// kernel can have written (after_previous).  What comes before that wait --
// barriers, TMEM, descriptors -- runs under the previous kernel's end.  Such
// memory is read with plain loads (or through TMA), which stay behind the wait;
// the read-only path is for data that nothing writes during a kernel's life.
__device__ __forceinline__ void next_may_start() { asm volatile("griddepcontrol.launch_dependents;" ::: "memory"); }
__device__ __forceinline__ void after_previous() { asm volatile("griddepcontrol.wait;" ::: "memory"); }

template <typename... P, typename... A>
inline cudaError_t launch_overlapped(void (*kernel)(P...), dim3 grid, unsigned threads, size_t smem, cudaStream_t s, A &&...args) {
    cudaLaunchAttribute at;
    at.id = cudaLaunchAttributeProgrammaticStreamSerialization;
    at.val.programmaticStreamSerializationAllowed = 1;
    cudaLaunchConfig_t c{};
    c.gridDim = grid;
    c.blockDim = dim3(threads);
    c.dynamicSmemBytes = smem;
    c.stream = s;
    c.attrs = &at;
    c.numAttrs = 1;
    return cudaLaunchKernelEx(&c, kernel, static_cast<P>(args)...);
}

__device__ __forceinline__ float to_f(float x) { return x; }
__device__ __forceinline__ float to_f(__nv_bfloat16 x) { return __bfloat162float(x); }
__device__ __forceinline__ void put(float *p, float x) { *p = x; }
__device__ __forceinline__ void put(__nv_bfloat16 *p, float x) { *p = __float2bfloat16(x); }

// Four neighbouring elements, on their own 4 x size boundary.
__device__ __forceinline__ void put4(float *p, float4 x) { *reinterpret_cast<float4 *>(p) = x; }
__device__ __forceinline__ void put4(__nv_bfloat16 *p, float4 x) {
    uint2 u;
    asm("cvt.rn.bf16x2.f32 %0, %1, %2;" : "=r"(u.x) : "f"(x.y), "f"(x.x));
    asm("cvt.rn.bf16x2.f32 %0, %1, %2;" : "=r"(u.y) : "f"(x.w), "f"(x.z));
    *reinterpret_cast<uint2 *>(p) = u;
}

}  // namespace serve
}  // namespace gkv
