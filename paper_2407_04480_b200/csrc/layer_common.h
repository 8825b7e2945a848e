// What the translation units of libloco_layer_b200.so share.
#pragma once
#include <cuda_bf16.h>
#include <cuda_runtime.h>
#include <stdint.h>

#include <atomic>
#include <cmath>

#include "../../include/loco_layer.h"

namespace loco_layer {

extern std::atomic<uint64_t> g_launches;

inline bool aligned(const void *p, uintptr_t to) { return (reinterpret_cast<uintptr_t>(p) & (to - 1)) == 0; }

// Streaming multiprocessors of the current device; 0 on an error.  Looked up once per device.
int sm_count();

// Launches a kernel whose blocks may be set up while the last ones of the stream's launch before are at work: every kernel
// here calls wait_for_previous() before it touches global memory, which restores the stream's order, and then
// let_next_start().  A call in a row of short ones takes 2 to 4 us less that way.
template <typename... Params, typename... Args>
int launch_clusters(void (*fn)(Params...), dim3 grid, unsigned threads, size_t shared, void *stream, unsigned cluster, const Args &...args) {
    cudaLaunchConfig_t how{};
    how.gridDim = grid;
    how.blockDim = dim3(threads);
    how.dynamicSmemBytes = shared;
    how.stream = static_cast<cudaStream_t>(stream);
    cudaLaunchAttribute attrs[2]{};
    attrs[0].id = cudaLaunchAttributeProgrammaticStreamSerialization;
    attrs[0].val.programmaticStreamSerializationAllowed = 1;
    attrs[1].id = cudaLaunchAttributeClusterDimension;
    attrs[1].val.clusterDim.x = cluster;
    attrs[1].val.clusterDim.y = attrs[1].val.clusterDim.z = 1;
    how.attrs = attrs;
    how.numAttrs = cluster > 1 ? 2 : 1;
    if (cudaLaunchKernelEx(&how, fn, args...) != cudaSuccess) {
        cudaGetLastError();
        return LOCO_ERR_CUDA;
    }
    g_launches.fetch_add(1);
    return LOCO_OK;
}
template <typename... Params, typename... Args>
int launch_kernel(void (*fn)(Params...), dim3 grid, unsigned threads, size_t shared, void *stream, const Args &...args) {
    return launch_clusters(fn, grid, threads, shared, stream, 1, args...);
}

// Returns when the launch before is complete and its results are visible.
__device__ __forceinline__ void wait_for_previous() { asm volatile("griddepcontrol.wait;" ::: "memory"); }
// Once every block has said so, the next launch's blocks may start as places become free.  Said only after
// wait_for_previous(), so that nothing older than this launch is still under way when they do.
__device__ __forceinline__ void let_next_start() { asm volatile("griddepcontrol.launch_dependents;" ::: "memory"); }

template <typename T> __device__ __forceinline__ float to_f32(T x);
template <> __device__ __forceinline__ float to_f32<float>(float x) { return x; }
template <> __device__ __forceinline__ float to_f32<__nv_bfloat16>(__nv_bfloat16 x) { return __bfloat162float(x); }
template <typename T> __device__ __forceinline__ T from_f32(float x);
template <> __device__ __forceinline__ float from_f32<float>(float x) { return x; }
template <> __device__ __forceinline__ __nv_bfloat16 from_f32<__nv_bfloat16>(float x) { return __float2bfloat16_rn(x); }

// N consecutive elements as one access of N * sizeof(T) bytes (16, 8 or 4), or one by one where N is 1.
template <typename T, int N> struct alignas(N * sizeof(T)) Pack { T v[N]; };

}  // namespace loco_layer
