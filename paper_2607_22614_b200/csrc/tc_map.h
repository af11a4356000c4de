// Tensor maps for the linear layers' operands (host side).
#pragma once
#include <cudaTypedefs.h>

#include "dr_internal.h"

namespace dr {

inline PFN_cuTensorMapEncodeTiled_v12000 map_encoder()
{
    static const PFN_cuTensorMapEncodeTiled_v12000 fn = [] {
        void* p = nullptr;
        cudaDriverEntryPointQueryResult r;
        if (cudaGetDriverEntryPointByVersion("cuTensorMapEncodeTiled", &p, 12000, cudaEnableDefault, &r) != cudaSuccess ||
            r != cudaDriverEntryPointSuccess) {
            cudaGetLastError();
            p = nullptr;
        }
        return (PFN_cuTensorMapEncodeTiled_v12000)p;
    }();
    return fn;
}

// A map over rows of `ld` elements, `cols` of them valid, boxes of 128 bytes x box_rows; `groups` > 0 adds a third dimension
// of `rows` rows each.
inline int encode_map(CUtensorMap* map, CUtensorMapDataType type, uint32_t es, const void* base, uint64_t cols, uint64_t rows,
                      uint64_t groups, uint64_t ld, uint32_t box_rows)
{
    const cuuint64_t dims[3] = {cols, rows, groups};
    const cuuint64_t strides[2] = {ld * es, rows * ld * es};
    const cuuint32_t box[3] = {128 / es, box_rows, 1}, step[3] = {1, 1, 1};
    PFN_cuTensorMapEncodeTiled_v12000 fn = map_encoder();
    const CUresult r = fn ? fn(map, type, groups ? 3 : 2, (void*)base, dims, strides, box, step, CU_TENSOR_MAP_INTERLEAVE_NONE,
                               CU_TENSOR_MAP_SWIZZLE_128B, CU_TENSOR_MAP_L2_PROMOTION_L2_256B, CU_TENSOR_MAP_FLOAT_OOB_FILL_NONE)
                          : CUDA_ERROR_NOT_SUPPORTED;
    if (r != CUDA_SUCCESS) {
        set_error("tensor map: driver error %d", (int)r);
        return DR_ERR_CUDA;
    }
    return DR_OK;
}
inline int encode_map(CUtensorMap* map, const void* base, bool fp8, uint64_t cols, uint64_t rows, uint64_t groups, uint64_t ld, uint32_t box_rows)
{
    return encode_map(map, fp8 ? CU_TENSOR_MAP_DATA_TYPE_UINT8 : CU_TENSOR_MAP_DATA_TYPE_BFLOAT16, fp8 ? 1 : 2, base, cols, rows,
                      groups, ld, box_rows);
}
inline int encode_map_f32(CUtensorMap* map, const void* base, uint64_t cols, uint64_t rows, uint64_t groups, uint64_t ld, uint32_t box_rows)
{
    return encode_map(map, CU_TENSOR_MAP_DATA_TYPE_FLOAT32, 4, base, cols, rows, groups, ld, box_rows);
}

// Codes of `rows` rows of `cols` bytes (64 or 128), one behind another: boxes of whole rows, swizzled over their own length.
inline int encode_codes_map(CUtensorMap* map, const void* base, uint32_t cols, uint64_t rows, uint32_t box_rows)
{
    const cuuint64_t dims[2] = {cols, rows}, stride = cols;
    const cuuint32_t box[2] = {cols, box_rows}, step[2] = {1, 1};
    PFN_cuTensorMapEncodeTiled_v12000 fn = map_encoder();
    const CUresult r = fn ? fn(map, CU_TENSOR_MAP_DATA_TYPE_UINT8, 2, (void*)base, dims, &stride, box, step, CU_TENSOR_MAP_INTERLEAVE_NONE,
                               cols == 128 ? CU_TENSOR_MAP_SWIZZLE_128B : CU_TENSOR_MAP_SWIZZLE_64B, CU_TENSOR_MAP_L2_PROMOTION_L2_256B,
                               CU_TENSOR_MAP_FLOAT_OOB_FILL_NONE)
                          : CUDA_ERROR_NOT_SUPPORTED;
    if (r != CUDA_SUCCESS) {
        set_error("tensor map: driver error %d", (int)r);
        return DR_ERR_CUDA;
    }
    return DR_OK;
}

}  // namespace dr
