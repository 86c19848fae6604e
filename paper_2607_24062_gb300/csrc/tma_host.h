// Host side of the tensor-core kernels: tensor maps, and where their operands live.
#pragma once

#include <cuda.h>
#include <cudaTypedefs.h>

#include <initializer_list>

#include "acrl_host.h"

namespace acrl {

// A two-dimensional map of rows of `cols` elements of `bytes` bytes at a stride of ld elements.
inline bool encode_map(CUtensorMap* map, CUtensorMapDataType type, uint32_t bytes, const void* ptr, uint64_t rows,
                       uint64_t cols, uint64_t ld, uint32_t box_rows, uint32_t box_cols, CUtensorMapSwizzle swizzle) {
    void* fn = nullptr;
    cudaDriverEntryPointQueryResult q;
    if (cudaGetDriverEntryPointByVersion("cuTensorMapEncodeTiled", &fn, 12000, cudaEnableDefault, &q) != cudaSuccess ||
        q != cudaDriverEntryPointSuccess || fn == nullptr)
        return false;
    auto encode = reinterpret_cast<PFN_cuTensorMapEncodeTiled_v12000>(fn);
    const cuuint64_t dims[2] = {cols, rows};
    const cuuint64_t strides[1] = {ld * bytes};
    const cuuint32_t box[2] = {box_cols, box_rows};
    const cuuint32_t estr[2] = {1, 1};
    return encode(map, type, 2, const_cast<void*>(ptr), dims, strides, box, estr,
                  CU_TENSOR_MAP_INTERLEAVE_NONE, swizzle, CU_TENSOR_MAP_L2_PROMOTION_L2_256B,
                  CU_TENSOR_MAP_FLOAT_OOB_FILL_NONE) == CUDA_SUCCESS;
}

// True when every pointer is device memory of the current device: not managed
// memory, not host memory and not a peer GPU's memory.  The GEMM's tensor maps
// are encoded over these pointers, and its TMA copies must stay within this
// GPU's own memory.  A failed query counts as "no" and leaves no error behind
// for a later launch check.
inline bool operands_on_current_device(std::initializer_list<const void*> ptrs) {
    int dev = 0;
    if (cudaGetDevice(&dev) != cudaSuccess) {
        (void)cudaGetLastError();
        return false;
    }
    for (const void* p : ptrs) {
        cudaPointerAttributes a{};
        if (cudaPointerGetAttributes(&a, p) != cudaSuccess) {
            (void)cudaGetLastError();
            return false;
        }
        if (a.type != cudaMemoryTypeDevice || a.device != dev) return false;
    }
    return true;
}

}  // namespace acrl
