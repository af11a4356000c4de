// Entry points of the linear layers: argument checks, the handle, choice of kernel.
#include "linear.h"

#include <atomic>
#include <cstring>
#include <mutex>
#include <new>

using namespace dr;

namespace {

constexpr uint64_t kMaxRows = 0x7FFFFFFFull;
constexpr uint64_t kMaxFeatures = 0x7FFFFFFFull - 511;  // the kernels count features in int, up to two tiles past the last

// A role may wait for a whole tile (bf16 accumulators are handed over at its end), and a contraction may have up to 2^25 steps: at 0.2 to
// 0.4 us each that is 10 s, so the limit grows with them.
constexpr uint32_t kWaitUs = 2000000, kStepWaitUs = 10;
std::atomic<uint32_t> g_wait_us{kWaitUs};
std::atomic<bool> g_starve{false};

int check_layer(const dr_linear* lin)
{
    if (!lin) {
        set_error("NULL layer");
        return DR_ERR_INVALID;
    }
    int dev = -1;
    if (cudaGetDevice(&dev) != cudaSuccess || dev != lin->device) {
        set_error("current device differs from the layer's device");
        return DR_ERR_STATE;
    }
    return DR_OK;
}

// Rows, offsets, and the two row-major operands every product has.
int check_rows(const dr_linear* lin, uint64_t rows, const int32_t* offsets, const void* p, uint64_t ldp, uint64_t p_cols,
               uint32_t p_es, const void* q, uint64_t ldq, uint64_t q_cols, uint32_t q_es)
{
    if (rows > kMaxRows) {
        set_error("more than 2^31 - 1 rows");
        return DR_ERR_UNSUPPORTED;
    }
    if (!offsets && lin->d.n_groups != 1) {
        set_error("a layer of %u groups needs offsets", lin->d.n_groups);
        return DR_ERR_INVALID;
    }
    if (rows && (!p || !q)) {
        set_error("NULL buffer");
        return DR_ERR_INVALID;
    }
    if (!pitch_ok(rows, p_cols, ldp) || !pitch_ok(rows, q_cols, ldq)) {
        set_error("leading dimension below the row's length or out of range");
        return DR_ERR_INVALID;
    }
    if ((uintptr_t)p % p_es || (uintptr_t)q % q_es || (uintptr_t)offsets % 4) {
        set_error("a pointer is not aligned to its element size");
        return DR_ERR_ALIGN;
    }
    return DR_OK;
}

// Once per device: shared memory for the kernels, and how many clusters of each size run at the same time.
constexpr int kDevices = 64;
std::mutex g_prepare;
bool g_prepared[kDevices];
uint32_t g_fit[kDevices][kMaxSplit + 1];

int prepare_device(int dev, uint32_t (&fit)[kMaxSplit + 1])
{
    std::lock_guard<std::mutex> hold(g_prepare);
    const bool known = dev >= 0 && dev < kDevices;
    if (!known || !g_prepared[dev]) {
        int rc = prepare_linear_tc();
        if (rc == DR_OK) rc = prepare_linear_small(fit);
        if (rc) return rc;
        if (!known) return DR_OK;
        memcpy(g_fit[dev], fit, sizeof fit);
        g_prepared[dev] = true;
    }
    memcpy(fit, g_fit[dev], sizeof fit);
    return DR_OK;
}

int check_out_dtype(uint32_t dtype)
{
    if (dtype != DR_BF16 && dtype != DR_F32) {
        set_error("output must be DR_BF16 or DR_F32");
        return DR_ERR_UNSUPPORTED;
    }
    return DR_OK;
}

int check_gradient(const dr_linear* lin)
{
    if (lin->fp8) {
        set_error("gradients need a bf16 layer");
        return DR_ERR_UNSUPPORTED;
    }
    return DR_OK;
}

// Up to this many rows a group (on average) the kernel that reads weights 128 features at a time wins over pairs of CTAs: in us,
// pairs second, fp8 1 x 6144 x 4096 8.4 / 17.0, 64 x 6144 x 4096 10.5 / 17.5; 128 groups of 1536 x 2048, 32 rows each 71 / 100, bf16 48 rows
// each 133 / 134.  Beyond 64 rows it reads the weights more than once: 128 x 24576 x 4096 fp8 41 / 35.  All of equal groups: the
// offsets are on the device, so a skewed batch goes by its average as well.
constexpr uint64_t kSmallRows = 64;

int launch(const LinearCall& c)
{
    // wgrad without rows only writes zeros, which needs no operand a tensor map could describe
    if (c.rows && linear_tc_takes(c)) {
        if (c.op == kForward && c.rows <= kSmallRows * c.lin->d.n_groups) return launch_linear_small(c);
        return launch_linear_tc(c);
    }
    return launch_linear_simt(c);
}

}  // namespace

namespace dr {
uint32_t wait_limit_us(uint64_t steps)
{
    const uint64_t us = g_wait_us.load(std::memory_order_relaxed) + steps * kStepWaitUs;
    return us < 0xFFFFFFFFull ? (uint32_t)us : 0xFFFFFFFFu;
}
bool waits_starve() { return g_starve.load(std::memory_order_relaxed); }
}  // namespace dr

extern "C" {

int dr_linear_create(const dr_linear_desc* desc, dr_linear** out)
{
    if (!out) {
        set_error("NULL out");
        return DR_ERR_INVALID;
    }
    *out = nullptr;
    if (!desc || desc->struct_size != sizeof(dr_linear_desc)) {
        set_error("NULL descriptor or struct_size mismatch");
        return DR_ERR_INVALID;
    }
    if (desc->dtype != DR_BF16 && desc->dtype != DR_FP8_E4M3_B128) {
        set_error("a layer's weight is DR_BF16 or DR_FP8_E4M3_B128");
        return DR_ERR_UNSUPPORTED;
    }
    dr_linear_desc d = *desc;
    const bool fp8 = d.dtype == DR_FP8_E4M3_B128;
    if (!d.n_groups || !d.out_features || !d.in_features) {
        set_error("zero layer dimension");
        return DR_ERR_INVALID;
    }
    if (d.out_features > kMaxFeatures || d.in_features > kMaxFeatures || d.n_groups > kMaxFeatures || d.out_features * d.n_groups > kMaxFeatures) {
        set_error("layer dimension above 2^31 - 512");
        return DR_ERR_UNSUPPORTED;
    }
    const uint64_t rows = d.out_features * d.n_groups, sr = (rows + 127) / 128, sc = (d.in_features + 127) / 128;
    if (!d.weight_ld) d.weight_ld = d.in_features;
    if (!d.scale_ld) d.scale_ld = sc;
    if (!d.weight_dev || (fp8 && !d.scale_dev) || (!fp8 && d.scale_dev)) {
        set_error("NULL weight, fp8 without scales or bf16 with them");
        return DR_ERR_INVALID;
    }
    if (!pitch_ok(rows, d.in_features, d.weight_ld) || (fp8 && !pitch_ok(sr, sc, d.scale_ld))) {
        set_error("leading dimension out of range");
        return DR_ERR_INVALID;
    }
    const uint32_t es = fp8 ? 1 : 2;
    if ((uintptr_t)d.weight_dev % es || (uintptr_t)d.scale_dev % 4) {
        set_error("a pointer is not aligned to its element size");
        return DR_ERR_ALIGN;
    }
    if (!rows_fit(rows, d.in_features, d.weight_ld, es, d.weight_bytes) || (fp8 && !rows_fit(sr, sc, d.scale_ld, 4, d.scale_bytes))) {
        set_error("weight or scales smaller than the layer");
        return DR_ERR_SIZE;
    }
    int dev = -1;
    int sms = 0;
    DR_CUDA(cudaGetDevice(&dev));
    DR_CUDA(cudaDeviceGetAttribute(&sms, cudaDevAttrMultiProcessorCount, dev));
    dr_linear* lin = new (std::nothrow) dr_linear();
    if (!lin) return DR_ERR_NOMEM;
    const int rc = prepare_device(dev, lin->fit);
    if (rc) {
        delete lin;
        return rc;
    }
    lin->d = d;
    lin->device = dev;
    lin->sms = sms;
    lin->fp8 = fp8;
    *out = lin;
    return DR_OK;
}

int dr_diag_linear_wait_failures(uint64_t* count)
{
    if (!count) {
        set_error("NULL argument");
        return DR_ERR_INVALID;
    }
    // calls may run on streams that the default stream, which the counters are read on, does not wait for
    DR_CUDA(cudaDeviceSynchronize());
    uint64_t small = 0;
    int rc = linear_wait_failures(count);
    if (rc == DR_OK) rc = linear_small_wait_failures(&small);
    *count += small;
    return rc;
}

int dr_diag_linear_waits(uint32_t limit_us, uint32_t starve)
{
    if (limit_us > kWaitUs || starve > 1) {
        set_error("a limit above the ordinary one, or starve not 0 / 1");
        return DR_ERR_INVALID;
    }
    g_wait_us = limit_us ? limit_us : kWaitUs;
    g_starve = starve != 0;
    return DR_OK;
}

int dr_linear_destroy(dr_linear* lin)
{
    delete lin;
    return DR_OK;
}

int dr_linear_forward(const dr_linear* lin, const void* x_dev, uint64_t ldx, const float* x_scale_dev, uint64_t ld_scale,
                      uint64_t rows, const int32_t* offsets_dev, void* y_dev, uint64_t ldy, uint32_t y_dtype,
                      void* cuda_stream)
{
    int rc = check_layer(lin);
    if (rc == DR_OK) rc = check_out_dtype(y_dtype);
    if (rc) return rc;
    const dr_linear_desc& d = lin->d;
    rc = check_rows(lin, rows, offsets_dev, x_dev, ldx, d.in_features, lin->fp8 ? 1 : 2, y_dev, ldy, d.out_features,
                    y_dtype == DR_F32 ? 4 : 2);
    if (rc) return rc;
    if (lin->fp8 ? rows && (!x_scale_dev || !pitch_ok((d.in_features + 127) / 128, rows, ld_scale)) : x_scale_dev != nullptr) {
        set_error("an fp8 layer needs x's scales (ld_scale >= rows), a bf16 layer takes none");
        return DR_ERR_INVALID;
    }
    if ((uintptr_t)x_scale_dev % 4) {
        set_error("a pointer is not aligned to its element size");
        return DR_ERR_ALIGN;
    }
    if (rows == 0) return DR_OK;
    LinearCall c{lin,  kForward, x_dev, d.weight_dev, ldx, d.weight_ld, x_scale_dev, ld_scale, (uint32_t)rows,
                 offsets_dev, y_dev, ldy, y_dtype == DR_F32, false, (cudaStream_t)cuda_stream};
    return launch(c);
}

int dr_linear_dgrad(const dr_linear* lin, const void* dy_dev, uint64_t lddy, uint64_t rows, const int32_t* offsets_dev,
                    void* dx_dev, uint64_t lddx, uint32_t dx_dtype, void* cuda_stream)
{
    int rc = check_layer(lin);
    if (rc == DR_OK) rc = check_gradient(lin);
    if (rc == DR_OK) rc = check_out_dtype(dx_dtype);
    if (rc) return rc;
    const dr_linear_desc& d = lin->d;
    rc = check_rows(lin, rows, offsets_dev, dy_dev, lddy, d.out_features, 2, dx_dev, lddx, d.in_features,
                    dx_dtype == DR_F32 ? 4 : 2);
    if (rc || rows == 0) return rc;
    LinearCall c{lin,  kDgrad, dy_dev, d.weight_dev, lddy, d.weight_ld, nullptr, 0, (uint32_t)rows,
                 offsets_dev, dx_dev, lddx, dx_dtype == DR_F32, false, (cudaStream_t)cuda_stream};
    return launch(c);
}

int dr_linear_wgrad(const dr_linear* lin, const void* x_dev, uint64_t ldx, const void* dy_dev, uint64_t lddy, uint64_t rows,
                    const int32_t* offsets_dev, float* dw_dev, uint64_t lddw, uint32_t accumulate, void* cuda_stream)
{
    int rc = check_layer(lin);
    if (rc == DR_OK) rc = check_gradient(lin);
    if (rc) return rc;
    const dr_linear_desc& d = lin->d;
    rc = check_rows(lin, rows, offsets_dev, x_dev, ldx, d.in_features, 2, dy_dev, lddy, d.out_features, 2);
    if (rc) return rc;
    if (!dw_dev || !pitch_ok(d.out_features * d.n_groups, d.in_features, lddw) || accumulate > 1) {
        set_error("NULL dw, leading dimension below the row's length or out of range, or accumulate not 0 / 1");
        return DR_ERR_INVALID;
    }
    if ((uintptr_t)dw_dev % 4) {
        set_error("a pointer is not aligned to its element size");
        return DR_ERR_ALIGN;
    }
    if (rows == 0 && accumulate) return DR_OK;
    LinearCall c{lin,  kWgrad, dy_dev, x_dev, lddy, ldx, nullptr, 0, (uint32_t)rows,
                 offsets_dev, dw_dev, lddw, true, accumulate != 0, (cudaStream_t)cuda_stream};
    return launch(c);
}

}  // extern "C"
