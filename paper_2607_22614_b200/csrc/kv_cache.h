// The key and value cache in 8 bits: what the entry points and the kernels that write and read it share.
#pragma once
#include <cuda.h>
#include <cuda_runtime.h>

#include "dr_internal.h"
#include "overlap.cuh"

struct dr_kv_cache {
    dr_kv_cache_desc d{};
    int device = -1;
    int sms = 0;
    uint32_t block_log2 = 0;
    // codes as rows of head_dim bytes, boxes of min(block_tokens, 64) rows, swizzled so that 8 x 16 bytes of a column of rows fall on
    // different banks
    CUtensorMap k_map, v_map;
};

namespace dr {

constexpr uint32_t kMaxRequests = 1u << 24, kMaxWidth = 1u << 24, kMaxStepRows = 1u << 30;
constexpr uint32_t kBoxTokens = 64;  // of the tensor maps, at most

int check_cache(const dr_kv_cache* cache);

}  // namespace dr
