// Activations -> fp8 e4m3 with one fp32 scale per row and 128 columns (sm_100a).
//
// For every row r and block b of 128 columns: amax = max |v|, scale = amax / 448, code = e4m3(v / scale); v is the
// activation itself, silu(gate) * up, or a gathered row.  The bound is HBM: each value is read once and its code
// written once (3 B per element from bf16, 5 B from fp32, 5 B through SwiGLU from bf16).
//
// Eight lanes own one block of one row, sixteen values each (one 256-bit load of bf16), so a warp reads 512 columns of a row as one
// request, a block's maximum takes three shuffles, and what every lane has to do once a block (scale, reciprocal) is spread
// over sixteen values.  A CTA covers 8 * RPW rows of 512 columns: a warp starts the loads of its RPW rows before it reduces any
// of them, and the scales of a column block, side by side in memory, leave as one contiguous store per CTA instead
// of one 4-byte store per row.  The exact division is quantise8_corrected's.
// Measured, 8192 x 12288, calls in a graph: from bf16 54 us = 5.6 TB/s, from fp32 73 us = 6.9 TB/s, through SwiGLU from bf16 105 us =
// 4.8 TB/s: there the arithmetic (an exponential, a reciprocal and their corrections, two values an instruction where that
// exists) bounds.  32768 rows of 2048 gathered from 4096: 34 us, 101 MB of reads that L2 serves and 67 MB of codes.
#include <cuda_bf16.h>
#include <cuda_runtime.h>

#include "dr_internal.h"
#include "fp8_codes.cuh"
#include "overlap.cuh"

namespace dr {
namespace {

constexpr int kWarps = 8;
// rows per warp: 128 bytes of raw values a thread (8192 x 12288 through SwiGLU, when 2 rows took 117 us: 4 rows 131, 1 row 126)
template <bool F32, bool SWIGLU> constexpr int kManyRows = F32 || SWIGLU ? 2 : 4;

struct RowsArgs {
    const void* x;
    const int64_t* index;
    uint8_t* codes;
    float* scales;
    uint64_t ldx, ld_codes, ld_scales, src_rows;
    uint32_t rows, cols, col_tiles;  // col_tiles = ceil(cols / 512)
};

// -silu(g) * u of two values, in fp32.  With e = e^-|g| the sigmoid is h / (1 + e), h = 1 or e: the divisor stays in [1, 2], and nothing
// overflows, however large |g| is.  From s = h * fl(1 / (1 + e)), the remainder h - s (1 + e) comes out with one rounding
// as (h - s) - s e, where h - s is exact (s lies between h / 2 and h), and adding it back corrects s: what is left is the error
// of e, of one rounding of the sigmoid and of two products (0.83 units of 2^-24 rms over normal values; 1.02 with the uncorrected quotient, 0.87
// for g / (1 + exp(-g)) * u with a division rounded to nearest).  Signs are turned over by the reciprocal, so that quantise8_corrected's
// negated values cost nothing.
__device__ __forceinline__ void swiglu(float g0, float g1, float u0, float u1, float& v0, float& v1)
{
    const float e0 = expf(-fabsf(g0)), e1 = expf(-fabsf(g1));
    float r0, r1;
    asm("rcp.approx.ftz.f32 %0, %1;" : "=f"(r0) : "f"(-1.0f - e0));
    asm("rcp.approx.ftz.f32 %0, %1;" : "=f"(r1) : "f"(-1.0f - e1));
    const uint64_t h = two_of(g0 >= 0.0f ? 1.0f : e0, g1 >= 0.0f ? 1.0f : e1), r = two_of(r0, r1);
    uint64_t s = mul_two(h, r);
    s = fma_two(fma_two(s, two_of(e0, e1), add_two(h, s)), r, s);
    s = mul_two(mul_two(two_of(g0, g1), s), two_of(u0, u1));
    asm("mov.b64 {%0, %1}, %2;" : "=f"(v0), "=f"(v1) : "l"(s));
}

// m / 448 rounded to nearest, by one step of Markstein's correction: q = m * fl(1 / 448) is within an ulp, the remainder m - 448 q
// is exact in one fused multiply-add, and adding it back rounds once.  (An infinity has no remainder: the caller's clamp
// to FLT_MAX is applied to it directly.)
__device__ __forceinline__ float scale_of_row(float m)
{
    const float q = m * (1.0f / 448.0f);
    const float s = fmaf(fmaf(-448.0f, q, m), 1.0f / 448.0f, q);
    return m > 3.40282347e+38f ? 3.40282347e+38f : fmaxf(s, 1.17549435e-38f);
}

// Sixteen raw values of a row from column c on (zeros past `cols`): 8 registers of bf16 pairs or 16 of fp32.
// Coherent loads that stay behind after_previous(): the kernel is already running while the previous one writes its x, so x
// is not read-only for the kernel's lifetime, as non-coherent loads (.nc, __ldg) would need.
// VEC 2: 32-byte aligned and whole groups of sixteen columns; 1: 16-byte aligned and whole groups of eight; 0: any.
template <bool F32, int VEC>
__device__ __forceinline__ void load16(const void* row, uint32_t c, uint32_t cols, uint32_t (&w)[F32 ? 16 : 8])
{
    constexpr int n = F32 ? 16 : 8;
    if (VEC == 2) {
#pragma unroll
        for (int k = 0; k < n; ++k) w[k] = 0;
        if (c >= cols) return;
#pragma unroll
        for (int k = 0; k < n; k += 8)
            asm volatile("ld.global.L1::no_allocate.v8.b32 {%0,%1,%2,%3,%4,%5,%6,%7}, [%8];"
                         : "=r"(w[k]), "=r"(w[k + 1]), "=r"(w[k + 2]), "=r"(w[k + 3]), "=r"(w[k + 4]), "=r"(w[k + 5]),
                           "=r"(w[k + 6]), "=r"(w[k + 7])
                         : "l"((const char*)row + (uint64_t)c * (F32 ? 4 : 2) + 4 * k)
                         : "memory");
    } else if (VEC == 1) {
#pragma unroll
        for (int k = 0; k < n; k += 4) {
            w[k] = w[k + 1] = w[k + 2] = w[k + 3] = 0;
            if (c + k * (F32 ? 1 : 2) < cols)
                asm volatile("ld.global.L1::no_allocate.v4.b32 {%0,%1,%2,%3}, [%4];"
                             : "=r"(w[k]), "=r"(w[k + 1]), "=r"(w[k + 2]), "=r"(w[k + 3])
                             : "l"((const char*)row + (uint64_t)c * (F32 ? 4 : 2) + 4 * k)
                             : "memory");
        }
    } else {
#pragma unroll
        for (int k = 0; k < n; ++k) {
            w[k] = 0;
            if (F32) {
                if (c + k < cols) w[k] = ((const uint32_t*)row)[c + k];
            } else {
                if (c + 2 * k < cols) w[k] = ((const uint16_t*)row)[c + 2 * k];
                if (c + 2 * k + 1 < cols) w[k] |= (uint32_t)((const uint16_t*)row)[c + 2 * k + 1] << 16;
            }
        }
    }
}
template <bool F32>
__device__ __forceinline__ float value(const uint32_t (&w)[F32 ? 16 : 8], int k)
{
    if (F32) return __uint_as_float(w[F32 ? k : 0]);
    return __uint_as_float(k & 1 ? w[k / 2] & 0xFFFF0000u : w[k / 2] << 16);
}

template <bool F32, bool SWIGLU, int VEC, int RPW>
__global__ void __launch_bounds__(32 * kWarps, SWIGLU ? 4 : 3) rows_kernel(const RowsArgs a)
{
    constexpr int kRows = kWarps * RPW, kRaw = F32 ? 16 : 8;
    __shared__ float s_scale[4][kRows];
    const uint32_t lane = threadIdx.x & 31, warp = threadIdx.x >> 5;
    const uint32_t tile = blockIdx.x / a.col_tiles, part = blockIdx.x - tile * a.col_tiles;
    const uint64_t row0 = (uint64_t)tile * kRows;
    const uint32_t c = part * 512 + lane * 16;
    uint32_t x[RPW][kRaw], up[SWIGLU ? RPW : 1][kRaw];
    after_previous();
    int64_t from[RPW];  // all indices first: the rows' loads keep their order, and each would wait for its own index
#pragma unroll
    for (int i = 0; i < RPW; ++i) {
        const uint64_t r = row0 + warp * RPW + i;
        from[i] = r < a.rows ? a.index ? a.index[r] : (int64_t)r : -1;
    }
#pragma unroll
    for (int i = 0; i < RPW; ++i) {
        const int64_t src = from[i];
        const bool ok = src >= 0 && (uint64_t)src < a.src_rows;
        const char* row = (const char*)a.x + (ok ? (uint64_t)src : 0) * a.ldx * (F32 ? 4 : 2);
        load16<F32, VEC>(row, c, ok ? a.cols : 0, x[i]);
        if (SWIGLU) load16<F32, VEC>(row + (uint64_t)a.cols * (F32 ? 4 : 2), c, ok ? a.cols : 0, up[i]);
    }
#pragma unroll
    for (int i = 0; i < RPW; ++i) {
        const uint32_t lr = warp * RPW + i;
        const uint64_t r = row0 + lr;
        // v holds the negated values, as quantise8_corrected wants them: turned over two at a time where they come from bf16
        float v[16], m = 0.0f;
        if (!F32 && !SWIGLU) {
#pragma unroll
            for (int k = 0; k < kRaw; ++k) x[i][k] ^= 0x80008000u;
        }
#pragma unroll
        for (int k = 0; k < 16; k += 2) {
            if (SWIGLU) {
                swiglu(value<F32>(x[i], k), value<F32>(x[i], k + 1), value<F32>(up[i], k), value<F32>(up[i], k + 1), v[k], v[k + 1]);
            } else {
                v[k] = F32 ? -value<F32>(x[i], k) : value<F32>(x[i], k);
                v[k + 1] = F32 ? -value<F32>(x[i], k + 1) : value<F32>(x[i], k + 1);
            }
            m = fmaxf(m, fmaxf(fabsf(v[k]), fabsf(v[k + 1])));  // fmaxf drops NaN operands
        }
#pragma unroll
        for (int o = 4; o; o >>= 1) m = fmaxf(m, __shfl_xor_sync(0xFFFFFFFFu, m, o));
        const float scale = scale_of_row(m), recip = __frcp_rn(scale);
        if ((lane & 7) == 0) s_scale[lane >> 3][lr] = scale;
        if (r < a.rows && c < a.cols) {
            uint2 q[2];
#pragma unroll
            for (int h = 0; h < 2; ++h) q[h] = quantise8_corrected<!F32>(v + 8 * h, scale, recip);
            uint8_t* dst = a.codes + r * a.ld_codes + c;
            if (VEC == 2) {
                *(uint4*)dst = make_uint4(q[0].x, q[0].y, q[1].x, q[1].y);
            } else if (VEC == 1) {
                *(uint2*)dst = q[0];
                if (c + 8 < a.cols) *(uint2*)(dst + 8) = q[1];
            } else {
#pragma unroll
                for (int k = 0; k < 16; ++k)
                    if (c + k < a.cols) dst[k] = (uint8_t)((k & 4 ? q[k / 8].y : q[k / 8].x) >> (8 * (k & 3)));
            }
        }
    }
    __syncthreads();
    for (uint32_t t = threadIdx.x; t < 4 * kRows; t += 32 * kWarps) {
        const uint32_t b = t / kRows, lr = t - b * kRows;
        if (row0 + lr < a.rows && part * 512 + b * 128 < a.cols)
            a.scales[(uint64_t)(part * 4 + b) * a.ld_scales + row0 + lr] = s_scale[b][lr];
    }
}

template <bool F32, bool SWIGLU, int VEC>
int launch(const RowsArgs& a, int rpw, uint64_t blocks, cudaStream_t stream)
{
    cudaLaunchAttribute attr = overlap_attribute();
    cudaLaunchConfig_t cfg{};
    cfg.gridDim = dim3((unsigned)blocks);
    cfg.blockDim = dim3(32 * kWarps);
    cfg.stream = stream;
    cfg.attrs = &attr;
    cfg.numAttrs = 1;
    constexpr int many = kManyRows<F32, SWIGLU>;
    const cudaError_t e = cudaLaunchKernelEx(&cfg, rpw == many ? rows_kernel<F32, SWIGLU, VEC, many> : rows_kernel<F32, SWIGLU, VEC, 1>, a);
    if (e != cudaSuccess) {
        cudaGetLastError();
        set_error("row quantisation launch: %s", cudaGetErrorString(e));
        return DR_ERR_CUDA;
    }
    return DR_OK;
}
template <bool F32, bool SWIGLU>
int launch(const RowsArgs& a, int vec, cudaStream_t stream)
{
    // several rows per warp once that still gives every SM a few CTAs; few rows are spread over more warps
    constexpr int many = kManyRows<F32, SWIGLU>;
    const int rpw = ((uint64_t)a.rows + 8 * many - 1) / (8 * many) * a.col_tiles >= 148 * 4 ? many : 1;
    const uint64_t blocks = ((uint64_t)a.rows + 8 * rpw - 1) / (8 * rpw) * a.col_tiles;
    if (blocks > 0x7FFFFFFFull) {
        set_error("too many rows and columns for one launch");
        return DR_ERR_UNSUPPORTED;
    }
    if (vec == 2) return launch<F32, SWIGLU, 2>(a, rpw, blocks, stream);
    return vec == 1 ? launch<F32, SWIGLU, 1>(a, rpw, blocks, stream) : launch<F32, SWIGLU, 0>(a, rpw, blocks, stream);
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
    if (cols == 0 || !pitch_ok(src_rows, width, ldx) || !pitch_ok(rows, cols, ld_codes) || !pitch_ok((cols + 127) / 128, rows, ld_scales) ||
        (!row_index_dev && src_rows < rows)) {
        set_error("no columns, a leading dimension below its row or out of range, or fewer source rows than rows");
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
    a.col_tiles = (uint32_t)((cols + 511) / 512);
    const uint64_t in = (uintptr_t)x_dev | ldx * es, out = (uintptr_t)codes_dev | ld_codes;
    const int vec = cols % 16 == 0 && in % 32 == 0 && out % 16 == 0 ? 2 : cols % 8 == 0 && in % 16 == 0 && out % 8 == 0 ? 1 : 0;
    cudaStream_t s = (cudaStream_t)cuda_stream;
    const bool f32 = x_dtype == DR_F32, sw = form == DR_ROWS_SWIGLU;
    if (f32) return sw ? launch<true, true>(a, vec, s) : launch<true, false>(a, vec, s);
    return sw ? launch<false, true>(a, vec, s) : launch<false, false>(a, vec, s);
}
