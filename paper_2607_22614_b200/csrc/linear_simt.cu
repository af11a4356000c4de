// Linear layers by plain fp32 arithmetic: the form that takes every stride and alignment.
//
// One CTA of 256 threads per 64 x 64 tile of the output, four by four outputs a thread, the contraction in steps of 16 through
// shared memory with scalar loads.  fp8 operands are widened to their codes' values; the sums of a block of 128 of the contraction are
// scaled by the product of the two scales, as in the tensor-core kernels (code * scale may overflow where that product does
// not: a row that holds an infinity has the scale FLT_MAX).  The tensor-core
// kernels read their operands with tensor maps, which need bases and row pitches that are multiples of 16 bytes; what
// cannot be read that way comes here.  Bound: fp32 FMA issue (two shared loads of four per sixteen FMAs).
#include <cuda_bf16.h>

#include "linear.h"

namespace dr {
namespace {

constexpr uint32_t kT = 64, kL = 16;

struct SimtArgs {
    const void* a;
    const void* b;
    const float* a_scale;
    const float* b_scale;
    uint64_t lda, ldb, ld_as, ld_bs;
    const int32_t* offsets;
    void* c;
    uint64_t ldc;
    uint32_t rows, n_groups, n, k;  // n, k: the layer's out and in features
    uint32_t col_tiles;
    uint32_t c_f32, accumulate;
};

__device__ __forceinline__ float bf(const void* p, uint64_t i) { return __bfloat162float(((const __nv_bfloat16*)p)[i]); }
__device__ __forceinline__ float e4m3(const void* p, uint64_t i)
{
    uint32_t h2;
    asm("cvt.rn.f16x2.e4m3x2 %0, %1;" : "=r"(h2) : "h"((uint16_t)((const uint8_t*)p)[i]));
    float f;
    asm("cvt.f32.f16 %0, %1;" : "=f"(f) : "h"((uint16_t)(h2 & 0xFFFF)));
    return f;
}

template <int OP, bool FP8>
__global__ void __launch_bounds__(256) simt_kernel(const SimtArgs s)
{
    __shared__ float As[kL][kT + 4], Bs[kL][kT + 4];  // [contraction][row or column of the tile]
    __shared__ uint32_t s_tile[4];
    const uint32_t tid = threadIdx.x;
    uint32_t e, lo, hi, i0, j0, len;  // tile's first output row and column; length of the contraction
    if (OP == kWgrad) {
        const uint32_t row_tiles = (s.n + kT - 1) / kT;
        const uint32_t t = blockIdx.x / s.col_tiles;
        e = t / row_tiles;
        group_rows(s.offsets, e, s.rows, lo, hi);
        i0 = (t - e * row_tiles) * kT;
        len = hi - lo;
    } else {
        if (tid < 32) {
            uint32_t tile = 0;
            const bool found = find_tile<kT>(s.offsets, s.n_groups, s.rows, blockIdx.x / s.col_tiles, e, lo, hi, tile);
            if (tid == 0) {
                s_tile[0] = found ? e : 0xFFFFFFFFu;
                s_tile[1] = lo;
                s_tile[2] = hi;
                s_tile[3] = tile;
            }
        }
        __syncthreads();
        e = s_tile[0];
        if (e == 0xFFFFFFFFu) return;
        lo = s_tile[1];
        hi = s_tile[2];
        i0 = lo + s_tile[3] * kT;
        len = OP == kForward ? s.k : s.n;
    }
    j0 = (blockIdx.x % s.col_tiles) * kT;
    const uint32_t i_end = OP == kWgrad ? s.n : hi, j_end = OP == kForward ? s.n : s.k;
    const uint64_t w0 = (uint64_t)e * s.n;  // the group's first row in the stacked weight

    float acc[4][4] = {}, sum[4][4] = {};  // fp8: acc of one block of the contraction, sum of the scaled blocks
    const uint32_t ti = tid >> 4, tj = tid & 15;
    for (uint32_t l0 = 0; l0 < len; l0 += kL) {
#pragma unroll
        for (uint32_t q = 0; q < 4; ++q) {
            // neighbouring threads follow the operand's contiguous dimension
            const uint32_t x = tid + 256 * q;
            {
                const bool along = OP != kWgrad;  // A is contiguous along the contraction, except dy in wgrad
                const uint32_t i = along ? x / kL : x % kT, l = along ? x % kL : x / kT;
                float v = 0.0f;
                if (i0 + i < i_end && l0 + l < len) {
                    if (OP == kWgrad)
                        v = bf(s.a, (uint64_t)(lo + l0 + l) * s.lda + i0 + i);
                    else if (FP8)
                        v = e4m3(s.a, (uint64_t)(i0 + i) * s.lda + l0 + l);
                    else
                        v = bf(s.a, (uint64_t)(i0 + i) * s.lda + l0 + l);
                }
                As[l][i] = v;
            }
            {
                const bool along = OP == kForward;
                const uint32_t j = along ? x / kL : x % kT, l = along ? x % kL : x / kT;
                float v = 0.0f;
                if (j0 + j < j_end && l0 + l < len) {
                    if (OP == kWgrad)
                        v = bf(s.b, (uint64_t)(lo + l0 + l) * s.ldb + j0 + j);
                    else if (OP == kDgrad)
                        v = bf(s.b, (w0 + l0 + l) * s.ldb + j0 + j);
                    else if (FP8)
                        v = e4m3(s.b, (w0 + j0 + j) * s.ldb + l0 + l);
                    else
                        v = bf(s.b, (w0 + j0 + j) * s.ldb + l0 + l);
                }
                Bs[l][j] = v;
            }
        }
        __syncthreads();
#pragma unroll
        for (uint32_t l = 0; l < kL; ++l) {
            const float4 a = *(const float4*)&As[l][ti * 4], b = *(const float4*)&Bs[l][tj * 4];
            const float av[4] = {a.x, a.y, a.z, a.w}, bv[4] = {b.x, b.y, b.z, b.w};
#pragma unroll
            for (int p = 0; p < 4; ++p)
#pragma unroll
                for (int r = 0; r < 4; ++r) acc[p][r] = fmaf(av[p], bv[r], acc[p][r]);
        }
        __syncthreads();
        if (FP8 && ((l0 + kL) % 128 == 0 || l0 + kL >= len)) {
            const uint32_t b = l0 >> 7;
            float xs[4], ws[4];
#pragma unroll
            for (int p = 0; p < 4; ++p) {
                const uint32_t i = i0 + ti * 4 + p, j = j0 + tj * 4 + p;
                xs[p] = i < i_end ? s.a_scale[b * s.ld_as + i] : 0.0f;
                ws[p] = j < j_end ? s.b_scale[((w0 + j) >> 7) * s.ld_bs + b] : 0.0f;
            }
#pragma unroll
            for (int p = 0; p < 4; ++p)
#pragma unroll
                for (int r = 0; r < 4; ++r) {
                    sum[p][r] = fmaf(__fmul_rn(xs[p], ws[r]), acc[p][r], sum[p][r]);
                    acc[p][r] = 0.0f;
                }
        }
    }
    if (FP8) {
#pragma unroll
        for (int p = 0; p < 4; ++p)
#pragma unroll
            for (int r = 0; r < 4; ++r) acc[p][r] = sum[p][r];
    }
#pragma unroll
    for (int p = 0; p < 4; ++p) {
        const uint32_t i = i0 + ti * 4 + p;
        if (i >= i_end) continue;
        const uint64_t row = OP == kWgrad ? w0 + i : i;
#pragma unroll
        for (int r = 0; r < 4; ++r) {
            const uint32_t j = j0 + tj * 4 + r;
            if (j >= j_end) continue;
            if (s.c_f32) {
                float* dst = (float*)s.c + row * s.ldc + j;
                *dst = s.accumulate ? *dst + acc[p][r] : acc[p][r];
            } else {
                ((__nv_bfloat16*)s.c)[row * s.ldc + j] = __float2bfloat16_rn(acc[p][r]);
            }
        }
    }
}

}  // namespace

int launch_linear_simt(const LinearCall& c)
{
    const dr_linear_desc& d = c.lin->d;
    SimtArgs s{};
    s.a = c.a;
    s.b = c.b;
    s.lda = c.lda;
    s.ldb = c.ldb;
    s.a_scale = c.a_scale;
    s.ld_as = c.ld_scale;
    s.b_scale = d.scale_dev;
    s.ld_bs = d.scale_ld;
    s.offsets = c.offsets;
    s.c = c.c;
    s.ldc = c.ldc;
    s.rows = c.rows;
    s.n_groups = d.n_groups;
    s.n = (uint32_t)d.out_features;
    s.k = (uint32_t)d.in_features;
    s.c_f32 = c.c_f32;
    s.accumulate = c.accumulate;
    const uint64_t width = c.op == kForward ? d.out_features : d.in_features;
    s.col_tiles = (uint32_t)((width + kT - 1) / kT);
    // forward and dgrad: at most one partly filled row tile for each group
    const uint64_t row_tiles = c.op == kWgrad ? d.n_groups * ((d.out_features + kT - 1) / kT)
                                              : ((uint64_t)c.rows + kT - 1) / kT + (c.offsets ? d.n_groups : 0);
    const uint64_t blocks = row_tiles * s.col_tiles;
    if (blocks > 0x7FFFFFFFull) {
        set_error("too many output tiles for one launch");
        return DR_ERR_UNSUPPORTED;
    }
    if (c.op == kWgrad)
        simt_kernel<kWgrad, false><<<(unsigned)blocks, 256, 0, c.stream>>>(s);
    else if (c.op == kDgrad)
        simt_kernel<kDgrad, false><<<(unsigned)blocks, 256, 0, c.stream>>>(s);
    else if (c.lin->fp8)
        simt_kernel<kForward, true><<<(unsigned)blocks, 256, 0, c.stream>>>(s);
    else
        simt_kernel<kForward, false><<<(unsigned)blocks, 256, 0, c.stream>>>(s);
    cudaError_t err = cudaGetLastError();
    if (err != cudaSuccess) {
        set_error("linear kernel launch: %s", cudaGetErrorString(err));
        return DR_ERR_CUDA;
    }
    return DR_OK;
}

}  // namespace dr
