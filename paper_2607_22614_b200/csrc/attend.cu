// Entry points of the attention over the 8-bit cache: argument checks and the choice of kernel.
#include "attend.h"

#include <cmath>
#include <cstring>

#include "linear.h"

using namespace dr;

namespace {

int check_sizes(const dr_kv_cache* cache, uint64_t n_q_heads, uint64_t requests, uint64_t rows)
{
    const uint64_t kv = cache->d.kv_heads;
    if (!n_q_heads || n_q_heads % kv) {
        set_error("%llu query heads over %llu heads of the cache", (unsigned long long)n_q_heads, (unsigned long long)kv);
        return DR_ERR_INVALID;
    }
    if (n_q_heads / kv > 64 || requests > kMaxRequests || rows > kMaxStepRows || rows * (n_q_heads / kv) > 0x7FFFFFFFull) {
        set_error("query heads for a head of the cache, requests or rows out of range");
        return DR_ERR_UNSUPPORTED;
    }
    return DR_OK;
}

}  // namespace

extern "C" {

int dr_attend_work(const dr_kv_cache* cache, uint64_t n_q_heads, uint64_t requests, uint64_t rows, uint64_t* bytes)
{
    if (!cache || !bytes) {
        set_error("NULL argument");
        return DR_ERR_INVALID;
    }
    const int rc = check_sizes(cache, n_q_heads, requests, rows);
    if (rc == DR_OK) *bytes = attend_few_work(cache);
    return rc;
}

int dr_attend(const dr_kv_cache* cache, const void* q_dev, uint64_t ldq, uint64_t n_q_heads, uint64_t rows, const int32_t* offsets_dev,
              const int32_t* lengths_dev, uint64_t requests, const int32_t* table_dev, uint64_t ld_table, uint64_t width, float scale,
              uint64_t window, uint64_t sinks, void* out_dev, uint64_t ldo, void* work_dev, uint64_t work_bytes, void* cuda_stream)
{
    int rc = check_cache(cache);
    if (rc == DR_OK) rc = check_sizes(cache, n_q_heads, requests, rows);
    if (rc) return rc;
    const dr_kv_cache_desc& d = cache->d;
    if (width > kMaxWidth) {
        set_error("more than 2^24 blocks a request");
        return DR_ERR_UNSUPPORTED;
    }
    if (!offsets_dev && rows != requests) {
        set_error("without offsets there is one row for each request");
        return DR_ERR_INVALID;
    }
    if (rows == 0 || requests == 0) return DR_OK;
    const uint64_t cols = n_q_heads * d.head_dim;
    if (!q_dev || !out_dev || !lengths_dev || !table_dev || !width || !std::isfinite(scale)) {
        set_error("NULL buffer, a table without columns or a scale that is not finite");
        return DR_ERR_INVALID;
    }
    if (!pitch_ok(rows, cols, ldq) || !pitch_ok(rows, cols, ldo) || !pitch_ok(requests, width, ld_table)) {
        set_error("leading dimension below the row's length or out of range");
        return DR_ERR_INVALID;
    }
    if (((uintptr_t)q_dev | (uintptr_t)out_dev) % 2 || ((uintptr_t)offsets_dev | (uintptr_t)lengths_dev | (uintptr_t)table_dev) % 4 ||
        (uintptr_t)work_dev % 16) {
        set_error("a pointer is not aligned to its element size, or work off 16 bytes");
        return DR_ERR_ALIGN;
    }
    // contexts of eight tiles at most are not divided, which saves the launch that joins, and its memory (300 tokens: 8.3 us a call, divided 10.5)
    const bool whole = (width << cache->block_log2) <= 8 * kTileTokens;
    uint64_t need = 0;
    if (!whole) dr_attend_work(cache, n_q_heads, requests, rows, &need);
    if (need && (!work_dev || work_bytes < need)) {
        set_error("work holds %llu bytes, %llu are needed", (unsigned long long)(work_dev ? work_bytes : 0), (unsigned long long)need);
        return DR_ERR_SIZE;
    }
    AttendArgs a{};
    a.q = q_dev;
    a.out = out_dev;
    a.offsets = offsets_dev;
    a.lengths = lengths_dev;
    a.table = table_dev;
    a.k_scale = d.k_scale_dev;
    a.v_scale = d.v_scale_dev;
    a.ldq = ldq;
    a.ldo = ldo;
    a.ld_table = ld_table;
    a.requests = (uint32_t)requests;
    a.rows = (uint32_t)rows;
    a.width = (uint32_t)width;
    a.n_q = (uint32_t)n_q_heads;
    a.n_kv = d.kv_heads;
    a.group = a.n_q / a.n_kv;
    a.n_blocks = d.n_blocks;
    a.block_log2 = cache->block_log2;
    // a window that no token lies outside of is none: positions end at 2^31 - 2
    a.window = window < 0x7FFFFFFFull ? (uint32_t)window : 0;
    a.sinks = (uint32_t)(sinks < 0x7FFFFFFFull ? sinks : 0x7FFFFFFFull);
    a.scale = scale * 1.4426950408889634f;
    auto vec = [](const void* p, uint64_t ld) { const uint64_t bits = (uintptr_t)p | ld * 2; return bits % 16 == 0 ? 2u : bits % 8 == 0 ? 1u : 0u; };
    a.vec_q = vec(q_dev, ldq);
    a.vec_out = vec(out_dev, ldo);
    a.limit_us = wait_limit_us(0);
    a.starve = waits_starve();
    a.whole = whole;
    // each request's rows on the device decide which of the two takes it; without offsets every request has few
    if (offsets_dev) rc = launch_attend_many(cache, a, (cudaStream_t)cuda_stream);
    return rc ? rc : launch_attend_few(cache, a, work_dev, (cudaStream_t)cuda_stream);
}

int dr_call(uint32_t what, const uint64_t* w)
{
    if (!w || what > DR_CALL_ATTEND) {
        set_error("NULL words or an unknown entry point");
        return DR_ERR_INVALID;
    }
    if (what == DR_CALL_KV_EXTEND)
        return dr_kv_extend((const dr_kv_cache*)w[0], (const int32_t*)w[1], (const int32_t*)w[2], (int32_t*)w[3], w[4], (int32_t*)w[5], w[6], w[7],
                            (int32_t*)w[8], (const int32_t*)w[9], (int32_t*)w[10], w[11], (int32_t*)w[12], (int32_t*)w[13], (int32_t*)w[14], w[15], (void*)w[16]);
    if (what == DR_CALL_QK_FORWARD)
        return dr_qk_forward((const dr_qk*)w[0], (const void*)w[1], (uint32_t)w[2], w[3], (const int32_t*)w[4], w[5], (void*)w[6], w[7], (void*)w[8]);
    if (what == DR_CALL_QK_APPEND)
        return dr_qk_append((const dr_qk*)w[0], (const void*)w[1], (uint32_t)w[2], w[3], (const int32_t*)w[4], w[5], (const int32_t*)w[6], w[7],
                            (const dr_kv_cache*)w[8], (void*)w[9], w[10], (void*)w[11]);
    if (what == DR_CALL_QK_GRAD)
        return dr_qk_grad((const dr_qk*)w[0], (const void*)w[1], (uint32_t)w[2], w[3], (const int32_t*)w[4], (const void*)w[5], w[6], w[7], (void*)w[8], w[9],
                          (float*)w[10], (float*)w[11], (uint32_t)w[12], (void*)w[13], w[14], (void*)w[15]);
    double scale;
    memcpy(&scale, w + 11, sizeof scale);
    return dr_attend((const dr_kv_cache*)w[0], (const void*)w[1], w[2], w[3], w[4], (const int32_t*)w[5], (const int32_t*)w[6], w[7], (const int32_t*)w[8],
                     w[9], w[10], (float)scale, w[12], w[13], (void*)w[14], w[15], (void*)w[16], w[17], (void*)w[18]);
}

}  // extern "C"
