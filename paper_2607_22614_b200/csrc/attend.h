// Attention over the 8-bit cache: what the entry point and the kernels share.
#pragma once
#include "kv_cache.h"

namespace dr {

struct AttendArgs {
    const void* q;
    void* out;
    const int32_t* offsets;  // NULL: one row a request
    const int32_t* lengths;
    const int32_t* table;
    const float* k_scale;
    const float* v_scale;
    uint64_t ldq, ldo, ld_table;
    uint32_t requests, rows, width, n_q, n_kv, group, n_blocks, block_log2;
    uint32_t window, sinks;  // window 0: none
    float scale;             // of the logits, times log2(e)
    uint32_t vec_q, vec_out;  // rows of q and out start on 16 bytes: 2, on 8: 1, neither: 0
    uint32_t limit_us, starve;
    uint32_t whole;  // few rows: groups are not divided between CTAs
};

// A block's value scale goes into p: the kernels' running maximum is that of log2(p) + log2(scale), and the sum of p takes the scale out again by
// its reciprocal.  That is sound while the scales of a request differ by no more than an exponential's range: from 2^-40 to 2^40 what an
// exponential flushes to nothing, or keeps of a hidden token (2^-126), is below 2^-86 where the sum is above 2^-29.  From the first scale on that is
// not among those (the 2^-100 of a block without values, say) a row's sum has exponentials of its own, relative to a maximum of the logits alone.
constexpr float kLeastNear = 9.0949470e-13f, kMostNear = 1.0995116e12f;  // 2^-40, 2^40
constexpr float kLeastScale = 1.4e-45f;                                  // 2^-149, for the logarithm of 0
__device__ __forceinline__ float log2_scale(float scale) { return log2f(fmaxf(scale, kLeastScale)); }
// 0: the sum needs exponentials of its own.
__device__ __forceinline__ float reciprocal_near(float scale) { return scale >= kLeastNear && scale <= kMostNear ? 1.0f / scale : 0.0f; }

constexpr uint32_t kTileTokens = 64;  // of the cache that a step of the few-row kernel takes

// A request's rows and tokens, held inside the call's buffers whatever the arrays say.
struct Request {
    uint32_t row0, n, len;
};
__device__ __forceinline__ Request request_of(const AttendArgs& a, uint32_t r)
{
    Request q;
    if (a.offsets) {
        const int32_t lo = a.offsets[r], hi = a.offsets[r + 1];
        q.row0 = min((uint32_t)max(lo, 0), a.rows);
        q.n = max(min((uint32_t)max(hi, 0), a.rows), q.row0) - q.row0;
    } else {
        q.row0 = r;
        q.n = 1;
    }
    q.len = (uint32_t)min((uint64_t)(uint32_t)max(a.lengths[r], 0), min((uint64_t)a.width << a.block_log2, (uint64_t)0x7FFFFFFFu));
    return q;
}
// (Rows before a request's first token see nothing, whatever their position: -1 stands for all of them, from which any window can be taken.)
// The tiles of TILE tokens that rows at positions p_lo .. p_hi may see: [0, sinks) and [first, first + count - sinks).
struct Tiles {
    uint32_t sinks, first, count;
    __device__ __forceinline__ uint32_t at(uint32_t i) const { return i < sinks ? i : first + (i - sinks); }
};
template <uint32_t TILE>
__device__ __forceinline__ Tiles tiles_of(const AttendArgs& a, int p_lo, int p_hi)
{
    Tiles t{0, 0, p_hi >= 0 ? (uint32_t)p_hi / TILE + 1 : 0};
    if (a.window) {
        const uint32_t end = t.count;
        const int lo = max(0, max(p_lo, -1) - (int)a.window + 1);
        t.sinks = min((a.sinks + TILE - 1) / TILE, end);
        t.first = max(t.sinks, (uint32_t)lo / TILE);
        t.count = t.sinks + (end > t.first ? end - t.first : 0);
    }
    return t;
}

// Requests of up to this many rows (tokens times query heads of a cache head) go to the few-row kernel, which reads the cache once for
// each eight, sixteen or twenty-four of them; the others to the tensor cores, 256 rows a CTA.
constexpr uint32_t kFewRows = 64;

int launch_attend_many(const dr_kv_cache* cache, const AttendArgs& a, cudaStream_t stream);
int prepare_attend_many();
int attend_many_wait_failures(uint64_t* out);

int launch_attend_few(const dr_kv_cache* cache, const AttendArgs& a, void* work, cudaStream_t stream);
int prepare_attend_few();  // once per device
uint64_t attend_few_work(const dr_kv_cache* cache);
int attend_few_wait_failures(uint64_t* out);

}  // namespace dr
