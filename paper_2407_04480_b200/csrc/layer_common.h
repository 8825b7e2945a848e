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

// Status of the launch just made.
inline int launched(int kernels = 1) {
    if (cudaGetLastError() != cudaSuccess) return LOCO_ERR_CUDA;
    g_launches.fetch_add(static_cast<uint64_t>(kernels));
    return LOCO_OK;
}

template <typename T> __device__ __forceinline__ float to_f32(T x);
template <> __device__ __forceinline__ float to_f32<float>(float x) { return x; }
template <> __device__ __forceinline__ float to_f32<__nv_bfloat16>(__nv_bfloat16 x) { return __bfloat162float(x); }
template <typename T> __device__ __forceinline__ T from_f32(float x);
template <> __device__ __forceinline__ float from_f32<float>(float x) { return x; }
template <> __device__ __forceinline__ __nv_bfloat16 from_f32<__nv_bfloat16>(float x) { return __float2bfloat16_rn(x); }

// N consecutive elements as one access of N * sizeof(T) bytes (16, 8 or 4), or one by one where N is 1.
template <typename T, int N> struct alignas(N * sizeof(T)) Pack { T v[N]; };

}  // namespace loco_layer
