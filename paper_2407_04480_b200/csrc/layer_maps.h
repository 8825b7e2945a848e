// Tensor maps of bfloat16 operands, encoded on the host.
#pragma once
#include <cuda.h>

#include "layer_common.h"

namespace loco_layer {

using EncodeFn = CUresult (*)(CUtensorMap *, CUtensorMapDataType, cuuint32_t, void *, const cuuint64_t *, const cuuint64_t *, const cuuint32_t *,
                              const cuuint32_t *, CUtensorMapInterleave, CUtensorMapSwizzle, CUtensorMapL2promotion, CUtensorMapFloatOOBfill);

inline EncodeFn encode_fn() {
    static std::atomic<EncodeFn> known{nullptr};
    EncodeFn f = known.load();
    if (!f) {
        void *p = nullptr;
        cudaDriverEntryPointQueryResult how;
        if (cudaGetDriverEntryPoint("cuTensorMapEncodeTiled", &p, cudaEnableDefault, &how) != cudaSuccess || how != cudaDriverEntryPointSuccess) {
            cudaGetLastError();
            return nullptr;
        }
        f = reinterpret_cast<EncodeFn>(p);
        known.store(f);
    }
    return f;
}

// Boxes of a tensor of `dims` (at most 4) dimensions, sizes in elements, strides of all but the first in bytes, with the 128-byte
// swizzle; what lies past the tensor reads as zero.
inline bool encode_map(CUtensorMap &map, int dims, void *at, const cuuint64_t *size, const cuuint64_t *strides, const cuuint32_t *box) {
    const EncodeFn encode = encode_fn();
    if (!encode) return false;
    const cuuint32_t step[4] = {1, 1, 1, 1};
    const auto made = [&] {
        return encode(&map, CU_TENSOR_MAP_DATA_TYPE_BFLOAT16, static_cast<cuuint32_t>(dims), at, size, strides, box, step, CU_TENSOR_MAP_INTERLEAVE_NONE,
                      CU_TENSOR_MAP_SWIZZLE_128B, CU_TENSOR_MAP_L2_PROMOTION_L2_256B, CU_TENSOR_MAP_FLOAT_OOB_FILL_NONE) == CUDA_SUCCESS;
    };
    if (made()) return true;
    // Unlike a launch the encoding binds no context to the calling thread, and needs one: a thread's first call binds it.
    int dev = 0;
    if (cudaGetDevice(&dev) == cudaSuccess && cudaSetDevice(dev) == cudaSuccess) return made();
    cudaGetLastError();
    return false;
}

}  // namespace loco_layer
