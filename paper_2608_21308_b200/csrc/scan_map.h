// Tensor maps of the gated linear recurrence: [B][L][D] values, tiles of a few tokens of 64 channels of one sequence.
#pragma once
#include <cuda.h>
#include <cuda_runtime.h>
#include <stdint.h>

#include "scan.h"

namespace e2ttt {

struct ScanMaps {
    CUtensorMap in[4], out[3];
};

inline bool scan_map(CUtensorMap* map, const void* base, const ScanShape& s, int tokens) {
    typedef CUresult (*Encode)(CUtensorMap*, CUtensorMapDataType, cuuint32_t, void*, const cuuint64_t*, const cuuint64_t*, const cuuint32_t*, const cuuint32_t*,
                               CUtensorMapInterleave, CUtensorMapSwizzle, CUtensorMapL2promotion, CUtensorMapFloatOOBfill);
    static const Encode encode = [] {
        void* p = nullptr;
        cudaDriverEntryPointQueryResult found;
        if (cudaGetDriverEntryPoint("cuTensorMapEncodeTiled", &p, cudaEnableDefault, &found) != cudaSuccess || found != cudaDriverEntryPointSuccess) {
            (void)cudaGetLastError();
            p = nullptr;
        }
        return reinterpret_cast<Encode>(p);
    }();
    if (!encode) return false;
    const cuuint64_t size = s.f32 ? 4 : 2, dims[3] = {(cuuint64_t)s.D, (cuuint64_t)s.L, (cuuint64_t)s.B}, strides[2] = {s.D * size, (cuuint64_t)s.L * s.D * size};
    const cuuint32_t box[3] = {(cuuint32_t)kScanCh, (cuuint32_t)tokens, 1}, each[3] = {1, 1, 1};
    return encode(map, s.f32 ? CU_TENSOR_MAP_DATA_TYPE_FLOAT32 : CU_TENSOR_MAP_DATA_TYPE_BFLOAT16, 3, const_cast<void*>(base), dims, strides, box, each,
                  CU_TENSOR_MAP_INTERLEAVE_NONE, CU_TENSOR_MAP_SWIZZLE_NONE, CU_TENSOR_MAP_L2_PROMOTION_L2_128B, CU_TENSOR_MAP_FLOAT_OOB_FILL_NONE) == CUDA_SUCCESS;
}

}  // namespace e2ttt
