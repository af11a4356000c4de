// Activations -> fp8 e4m3 with one fp32 scale per row and 128 columns (sm_100a).
//
// For every row r and block b of 128 columns: amax = max |v|, scale = amax / 448, code = e4m3(v / scale); v is the
// activation itself, silu(gate) * up, or a gathered row.  The bound is HBM: each value is read once and its code
// written once (3 B per element from bf16, 5 B from fp32, 5 B through SwiGLU from bf16).
//
// Sixteen lanes own one block of one row, eight values each (one 128-bit load of bf16), so a block is one contiguous 256 B
// request and its maximum takes four shuffles; nothing is staged in shared memory but the scales.  A CTA covers
// 8 * RPW rows of 256 columns: a warp starts the loads of its RPW rows before it reduces any of them, and
// the scales of a column block, side by side in memory, leave as one contiguous store per CTA instead of one
// 4-byte store per row.  The exact division is quantise8's (products with the reciprocal wherever that gives the same code).
#include <cuda_bf16.h>
#include <cuda_runtime.h>

#include "dr_internal.h"
#include "fp8_codes.cuh"

namespace dr {
namespace {

constexpr int kWarps = 8;

struct RowsArgs {
    const void* x;
    const int64_t* index;
    uint8_t* codes;
    float* scales;
    uint64_t ldx, ld_codes, ld_scales, src_rows;
    uint32_t rows, cols, col_pairs;  // col_pairs = ceil(cols / 256)
};

// silu(g) * u in fp32.  With e = e^-|g| the sigmoid is 1 / (1 + e) or e / (1 + e): the divisor stays in [1, 2], where the
// approximate division is good to 2 ulp and nothing overflows, however large |g| is.
__device__ __forceinline__ float swiglu(float g, float u)
{
    const float e = expf(-fabsf(g));
    return __fdividef(g >= 0.0f ? g : g * e, 1.0f + e) * u;
}

// Eight values of a row from column c on: zeros past `cols`.
template <bool F32, bool VEC>
__device__ __forceinline__ void load8(const void* row, uint32_t c, uint32_t cols, float (&v)[8])
{
#pragma unroll
    for (int k = 0; k < 8; ++k) v[k] = 0.0f;
    if (c >= cols) return;
    if (VEC && F32) {
        ld128f((const float*)row + c, &v[0]);
        ld128f((const float*)row + c + 4, &v[4]);
    } else if (VEC) {
        uint32_t w[4];
        asm volatile("ld.global.nc.L1::no_allocate.v4.b32 {%0,%1,%2,%3}, [%4];"
                     : "=r"(w[0]), "=r"(w[1]), "=r"(w[2]), "=r"(w[3])
                     : "l"((const uint16_t*)row + c));
#pragma unroll
        for (int k = 0; k < 4; ++k) {
            v[2 * k] = __uint_as_float(w[k] << 16);
            v[2 * k + 1] = __uint_as_float(w[k] & 0xFFFF0000u);
        }
    } else {
#pragma unroll
        for (int k = 0; k < 8; ++k)
            if (c + k < cols)
                v[k] = F32 ? ((const float*)row)[c + k] : __uint_as_float((uint32_t)((const uint16_t*)row)[c + k] << 16);
    }
}

template <bool F32, bool SWIGLU, bool VEC, int RPW>
__global__ void __launch_bounds__(32 * kWarps) rows_kernel(const RowsArgs a)
{
    constexpr int kRows = kWarps * RPW;
    __shared__ float s_scale[2][kRows];
    const uint32_t lane = threadIdx.x & 31, warp = threadIdx.x >> 5, half = lane >> 4;
    const uint32_t tile = blockIdx.x / a.col_pairs, pair = blockIdx.x - tile * a.col_pairs;
    const uint64_t row0 = (uint64_t)tile * kRows;
    const uint32_t c = pair * 256 + lane * 8;
    float v[RPW][8], u[SWIGLU ? RPW : 1][8];
#pragma unroll
    for (int i = 0; i < RPW; ++i) {
        const uint64_t r = row0 + warp * RPW + i;
        int64_t src = -1;
        if (r < a.rows) src = a.index ? a.index[r] : (int64_t)r;
        const bool ok = src >= 0 && (uint64_t)src < a.src_rows;
        const char* row = (const char*)a.x + (ok ? (uint64_t)src : 0) * a.ldx * (F32 ? 4 : 2);
        load8<F32, VEC>(row, ok ? c : a.cols, a.cols, v[i]);
        if (SWIGLU) load8<F32, VEC>(row + (uint64_t)a.cols * (F32 ? 4 : 2), ok ? c : a.cols, a.cols, u[i]);
    }
#pragma unroll
    for (int i = 0; i < RPW; ++i) {
        const uint32_t lr = warp * RPW + i;
        const uint64_t r = row0 + lr;
        float m = 0.0f;
#pragma unroll
        for (int k = 0; k < 8; ++k) {
            if (SWIGLU) v[i][k] = swiglu(v[i][k], u[i][k]);
            m = fmaxf(m, fabsf(v[i][k]));  // fmaxf drops NaN operands
        }
#pragma unroll
        for (int o = 8; o; o >>= 1) m = fmaxf(m, __shfl_xor_sync(0xFFFFFFFFu, m, o));
        const float scale = scale_of(m), recip = __frcp_rn(scale);
        if ((lane & 15) == 0) s_scale[half][lr] = scale;
        if (r < a.rows && c < a.cols) {
            const uint2 q = quantise8(v[i], scale, recip, small_code_of(recip));
            uint8_t* dst = a.codes + r * a.ld_codes + c;
            if (VEC) {
                *(uint2*)dst = q;
            } else {
#pragma unroll
                for (int k = 0; k < 8; ++k)
                    if (c + k < a.cols) dst[k] = (uint8_t)((k < 4 ? q.x : q.y) >> (8 * (k & 3)));
            }
        }
    }
    __syncthreads();
    for (uint32_t t = threadIdx.x; t < 2 * kRows; t += 32 * kWarps) {
        const uint32_t b = t / kRows, lr = t - b * kRows;
        if (row0 + lr < a.rows && pair * 256 + b * 128 < a.cols)
            a.scales[(uint64_t)(pair * 2 + b) * a.ld_scales + row0 + lr] = s_scale[b][lr];
    }
}

template <bool F32, bool SWIGLU, bool VEC>
int launch(const RowsArgs& a, int rpw, uint64_t blocks, cudaStream_t stream)
{
    if (rpw == 4)
        rows_kernel<F32, SWIGLU, VEC, 4><<<(unsigned)blocks, 32 * kWarps, 0, stream>>>(a);
    else
        rows_kernel<F32, SWIGLU, VEC, 1><<<(unsigned)blocks, 32 * kWarps, 0, stream>>>(a);
    cudaError_t e = cudaGetLastError();
    if (e != cudaSuccess) {
        set_error("row quantisation launch: %s", cudaGetErrorString(e));
        return DR_ERR_CUDA;
    }
    return DR_OK;
}

}  // namespace
}  // namespace dr

using namespace dr;

extern "C" int dr_quant_rows(const void* x_dev, uint32_t x_dtype, uint64_t ldx, uint64_t src_rows,
                             const int64_t* row_index_dev, uint32_t form, uint64_t rows, uint64_t cols, void* codes_dev,
                             uint64_t ld_codes, float* scales_dev, uint64_t ld_scales, void* cuda_stream)
{
    if (x_dtype != DR_BF16 && x_dtype != DR_F32) {
        set_error("x must be DR_BF16 or DR_F32");
        return DR_ERR_UNSUPPORTED;
    }
    if (form != DR_ROWS_PLAIN && form != DR_ROWS_SWIGLU) {
        set_error("unknown form of rows");
        return DR_ERR_UNSUPPORTED;
    }
    if (rows > 0x7FFFFFFFull || cols > 0x3FFFFFFFull || src_rows > 0x7FFFFFFFull) {
        set_error("rows or columns out of range");
        return DR_ERR_UNSUPPORTED;
    }
    const uint64_t width = form == DR_ROWS_SWIGLU ? 2 * cols : cols;
    if (cols == 0 || ldx < width || ld_codes < cols || ld_scales < rows || (!row_index_dev && src_rows < rows)) {
        set_error("no columns, a leading dimension below its row, or fewer source rows than rows");
        return DR_ERR_INVALID;
    }
    if (rows == 0) return DR_OK;
    if ((!x_dev && src_rows) || !codes_dev || !scales_dev) {
        set_error("NULL buffer");
        return DR_ERR_INVALID;
    }
    const uint32_t es = x_dtype == DR_F32 ? 4 : 2;
    if ((uintptr_t)x_dev % es || (uintptr_t)scales_dev % 4 || (uintptr_t)row_index_dev % 8) {
        set_error("a pointer is not aligned to its element size");
        return DR_ERR_ALIGN;
    }
    RowsArgs a{};
    a.x = x_dev;
    a.index = row_index_dev;
    a.codes = (uint8_t*)codes_dev;
    a.scales = scales_dev;
    a.ldx = ldx;
    a.ld_codes = ld_codes;
    a.ld_scales = ld_scales;
    a.src_rows = src_rows;
    a.rows = (uint32_t)rows;
    a.cols = (uint32_t)cols;
    a.col_pairs = (uint32_t)((cols + 255) / 256);
    // four rows per warp once that still gives every SM several CTAs; few rows are spread over more warps
    const int rpw = (rows + 31) / 32 * a.col_pairs >= 148 * 4 ? 4 : 1;
    const uint64_t blocks = (rows + 8 * rpw - 1) / (8 * rpw) * a.col_pairs;
    if (blocks > 0x7FFFFFFFull) {
        set_error("too many rows and columns for one launch");
        return DR_ERR_UNSUPPORTED;
    }
    const bool vec = cols % 8 == 0 && (uintptr_t)x_dev % 16 == 0 && ldx * es % 16 == 0 && (uintptr_t)codes_dev % 8 == 0 &&
                     ld_codes % 8 == 0;
    cudaStream_t s = (cudaStream_t)cuda_stream;
    const bool f32 = x_dtype == DR_F32, sw = form == DR_ROWS_SWIGLU;
    if (vec) {
        if (f32) return sw ? launch<true, true, true>(a, rpw, blocks, s) : launch<true, false, true>(a, rpw, blocks, s);
        return sw ? launch<false, true, true>(a, rpw, blocks, s) : launch<false, false, true>(a, rpw, blocks, s);
    }
    if (f32) return sw ? launch<true, true, false>(a, rpw, blocks, s) : launch<true, false, false>(a, rpw, blocks, s);
    return sw ? launch<false, true, false>(a, rpw, blocks, s) : launch<false, false, false>(a, rpw, blocks, s);
}
