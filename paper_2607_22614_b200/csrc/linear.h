// Linear layers over a rollout arena's weights: what the entry points and the kernels share.
#pragma once
#include <cuda_runtime.h>

#include "dr_internal.h"
#include "overlap.cuh"

namespace dr {
constexpr uint32_t kMaxSplit = 8;  // CTAs of a cluster that share a contraction
}

struct dr_linear {
    dr_linear_desc d{};  // strides filled in
    int device = -1;
    int sms = 0;
    uint32_t fit[dr::kMaxSplit + 1] = {};  // clusters of each size that the device runs at the same time
    bool fp8 = false;
};

namespace dr {

// One call, checked.  What the three products read and write:
//   forward  a = x [rows, k], c = y [rows, n]     dgrad  a = dy [rows, n], c = dx [rows, k]
//   wgrad    a = dy [rows, n], b = x [rows, k], c = dw [n_groups * n, k]
enum LinearOp { kForward = 0, kDgrad = 1, kWgrad = 2 };
struct LinearCall {
    const dr_linear* lin;
    LinearOp op;
    const void* a;
    const void* b;  // wgrad: x; otherwise the layer's weight
    uint64_t lda, ldb;
    const float* a_scale;
    uint64_t ld_scale;
    uint32_t rows;
    const int32_t* offsets;  // NULL: one group of all rows
    void* c;
    uint64_t ldc;
    bool c_f32, accumulate;
    cudaStream_t stream;
};

int launch_linear_simt(const LinearCall& c);  // linear_simt.cu: every stride and alignment

// linear_tc.cu: tensor cores, for operands that tensor maps can read
constexpr uint32_t kMaxTcGroups = 512;      // groups whose tile counts fit a CTA's table
bool linear_tc_takes(const LinearCall& c);
int launch_linear_tc(const LinearCall& c);
int prepare_linear_tc();                    // once per device
int linear_wait_failures(uint64_t* out);    // bounded waits that ran out (expected: 0)
uint32_t wait_limit_us(uint64_t steps);     // how long a wait may take when a tile's contraction has so many steps
bool waits_starve();                        // test hook: the copies are left out

// linear_small.cu: forward with few rows a group, the same operands
int launch_linear_small(const LinearCall& c);
int prepare_linear_small(uint32_t (&fit)[kMaxSplit + 1]);
int linear_small_wait_failures(uint64_t* out);

// Rows [lo, hi) of group e, held inside [0, rows] and never descending, whatever the offsets hold.
__device__ __forceinline__ void group_rows(const int32_t* offsets, uint32_t e, uint32_t rows, uint32_t& lo, uint32_t& hi)
{
    if (!offsets) {
        lo = 0;
        hi = rows;
        return;
    }
    const int32_t a = offsets[e], b = offsets[e + 1];
    lo = a < 0 ? 0u : min((uint32_t)a, rows);
    hi = b < 0 ? 0u : min((uint32_t)b, rows);
    if (hi < lo) hi = lo;
}

// The group that owns tile `t` when every group's rows are cut into tiles of BM: called by a whole warp, which scans
// 32 groups a step.  Returns false past the last tile; otherwise the group, its rows and the tile's index inside it.
template <uint32_t BM>
__device__ __forceinline__ bool find_tile(const int32_t* offsets, uint32_t n_groups, uint32_t rows, uint32_t t, uint32_t& e,
                                          uint32_t& lo, uint32_t& hi, uint32_t& tile)
{
    const uint32_t lane = threadIdx.x & 31;
    uint32_t before = 0;  // tiles of the groups scanned so far
    for (uint32_t e0 = 0; e0 < n_groups; e0 += 32) {
        uint32_t l = 0, h = 0;
        if (e0 + lane < n_groups) group_rows(offsets, e0 + lane, rows, l, h);
        const uint32_t mine = (h - l + BM - 1) / BM;
        uint32_t sum = mine;
#pragma unroll
        for (int o = 1; o < 32; o <<= 1) {
            const uint32_t up = __shfl_up_sync(0xFFFFFFFFu, sum, o);
            if (lane >= (uint32_t)o) sum += up;
        }
        const uint32_t total = __shfl_sync(0xFFFFFFFFu, sum, 31);
        if (t < before + total) {
            const uint32_t owner = __ballot_sync(0xFFFFFFFFu, t < before + sum);
            const uint32_t src = __ffs(owner) - 1;
            e = e0 + src;
            lo = __shfl_sync(0xFFFFFFFFu, l, src);
            hi = __shfl_sync(0xFFFFFFFFu, h, src);
            tile = t - before - __shfl_sync(0xFFFFFFFFu, sum - mine, src);
            return true;
        }
        before += total;
    }
    return false;
}

}  // namespace dr
