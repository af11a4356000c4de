// The cache handle, and block tables and slot maps of one step (sm_100a).
//
// From lengths and arrivals of all requests: where each request's rows begin, which blocks come back, which new blocks it takes, and
// the runs of slots that its rows go to.  All of it is prefix sums over the requests (of rows, of blocks that come back, of
// blocks wanted, of runs), after which every output entry finds the request it belongs to by bisection of the sums in shared memory: a prompt
// of thousands of rows and thousands of requests of one row spread over the threads alike.
//
// A few KB in and out: the launch and two passes over memory bound it, so one CTA does a decode step, and a cluster of
// up to eight CTAs, each with the sums of all requests, shares the entries of a large one.  Between phases that read what another CTA
// may write (arrays that may be updated in place) stands the cluster's barrier.
// Measured, calls in a graph: 64 requests of one token, two of them ending, 6.4 us, 200 prompts of 10 600 rows 7.9 (the calls' host time: 7.3).
#include <new>

#include "attend.h"
#include "tc_map.h"

namespace dr {
namespace {

constexpr uint32_t kThreads = 512;  // requests of one chunk, too

struct ExtendArgs {
    const int32_t* added;
    const int32_t* lengths;
    int32_t* lengths_out;
    int32_t* table;
    int32_t* free_list;
    const int32_t* state;
    int32_t* state_out;
    int32_t* offsets;
    int32_t* positions;
    int4* runs;
    uint64_t ld_table;
    uint32_t requests, width, rows, n_runs, n_blocks, block_log2;
};

// Sums that stop at 2^31 - 1: order does not matter, and two of them do not wrap.
constexpr uint32_t kMost = 0x7FFFFFFFu;
__device__ __forceinline__ uint32_t sat(uint32_t a, uint32_t b) { return min(a + b, kMost); }

// Exclusive sums over the CTA's threads of two values, and their totals; `scratch` is free again on return.
__device__ __forceinline__ void scan2(uint32_t& a, uint32_t& b, uint32_t& all_a, uint32_t& all_b, uint2 (&scratch)[kThreads / 32])
{
    const uint32_t lane = threadIdx.x & 31, warp = threadIdx.x >> 5;
    uint32_t sa = a, sb = b;
#pragma unroll
    for (int o = 1; o < 32; o <<= 1) {
        const uint32_t ua = __shfl_up_sync(0xFFFFFFFFu, sa, o), ub = __shfl_up_sync(0xFFFFFFFFu, sb, o);
        if (lane >= (uint32_t)o) {
            sa = sat(sa, ua);
            sb = sat(sb, ub);
        }
    }
    const uint32_t ea = __shfl_up_sync(0xFFFFFFFFu, sa, 1), eb = __shfl_up_sync(0xFFFFFFFFu, sb, 1);
    if (lane == 31) scratch[warp] = make_uint2(sa, sb);
    __syncthreads();
    uint32_t before_a = 0, before_b = 0;
    all_a = all_b = 0;
#pragma unroll
    for (uint32_t w = 0; w < kThreads / 32; ++w) {
        const uint2 v = scratch[w];
        if (w < warp) {
            before_a = sat(before_a, v.x);
            before_b = sat(before_b, v.y);
        }
        all_a = sat(all_a, v.x);
        all_b = sat(all_b, v.y);
    }
    a = lane ? sat(before_a, ea) : before_a;
    b = lane ? sat(before_b, eb) : before_b;
    __syncthreads();
}

// The last i < n with begin[i] <= x, where begin ascends and begin[0] <= x: among equal ones the last, which owns the entry.
__device__ __forceinline__ uint32_t owner(const uint32_t* begin, uint32_t n, uint32_t x)
{
    uint32_t lo = 0, hi = n;
    while (hi - lo > 1) {
        const uint32_t mid = (lo + hi) / 2;
        if (begin[mid] <= x) lo = mid; else hi = mid;
    }
    return lo;
}

template <bool CLUSTER>
__device__ __forceinline__ void sync_all()
{
    if (CLUSTER) {
        __threadfence();
        asm volatile("barrier.cluster.arrive.release.aligned;\nbarrier.cluster.wait.acquire.aligned;" ::: "memory");
    } else {
        __syncthreads();
    }
}

// Lists the blocks that a chunk's ending requests hold behind the first `from` entries of the free list, and returns how many they are: `total` entries of the
// table, request r0 + o's from begin[o] on, of which those that stand for no block are skipped.  A warp has a stretch of them: it counts the
// blocks in it, adds the counts of the warps before it, which may be in other CTAs, and lists its own.  (A call, as most steps have none.)
template <bool CLUSTER>
__device__ __noinline__ uint32_t come_back(const ExtendArgs& a, uint32_t r0, uint32_t total, uint64_t from, uint32_t ctas, uint32_t cta, const uint32_t* begin,
                                              uint32_t (&counts)[kThreads / 32])
{
    constexpr uint32_t kOf = kThreads / 32;  // warps of a CTA
    const uint32_t lane = threadIdx.x & 31, me = cta * kOf + (threadIdx.x >> 5), warps = ctas * kOf;
    const uint32_t per = (uint32_t)(((uint64_t)total + 32 * warps - 1) / (32 * warps)) * 32, lo = min((uint64_t)me * per, (uint64_t)total),
                   hi = min((uint64_t)lo + per, (uint64_t)total);
    uint32_t o = 0, end = 0;  // of the request that a lane's last entry belongs to; the entries ascend, but for the second time round
    auto entry = [&](uint32_t i) {
        if (i >= hi) return -1;
        if (i >= end) {
            o = owner(begin, kThreads, i);
            end = o + 1 < kThreads ? begin[o + 1] : total;
        }
        return a.table[(uint64_t)(r0 + o) * a.ld_table + (i - begin[o])];
    };
    auto held = [&](int32_t id) { return __ballot_sync(0xFFFFFFFFu, (uint32_t)id < a.n_blocks); };
    int32_t id = entry(lo + lane);
    uint32_t n = __popc(held(id));
#pragma unroll 4
    for (uint32_t i = lo + 32; i < hi; i += 32) n += __popc(held(entry(i + lane)));
    if (lane == 0) counts[threadIdx.x >> 5] = n;
    sync_all<CLUSTER>();
    uint32_t before = 0, sum = 0;
    for (uint32_t w = lane; w < warps; w += 32) {
        uint32_t v;
        if (CLUSTER) {
            uint32_t at = (uint32_t)__cvta_generic_to_shared(&counts[w % kOf]);
            asm volatile("mapa.shared::cluster.u32 %0, %0, %1;" : "+r"(at) : "r"(w / kOf));
            asm volatile("ld.shared::cluster.u32 %0, [%1];" : "=r"(v) : "r"(at) : "memory");
        } else {
            v = counts[w];
        }
        sum += v;
        if (w < me) before += v;
    }
#pragma unroll
    for (int o = 16; o; o >>= 1) {
        before += __shfl_xor_sync(0xFFFFFFFFu, before, o);
        sum += __shfl_xor_sync(0xFFFFFFFFu, sum, o);
    }
    uint64_t to = from + before;
    end = 0;
    for (uint32_t i = lo; i < hi; i += 32) {
        if (i > lo) id = entry(i + lane);
        const uint32_t bits = held(id);
        const uint64_t at = to + __popc(bits & ((1u << lane) - 1));
        if ((uint32_t)id < a.n_blocks && at < a.n_blocks) a.free_list[at] = id;
        to += __popc(bits);
    }
    return sum;
}

template <bool CLUSTER>
__global__ void __launch_bounds__(kThreads) extend_kernel(const ExtendArgs a)
{
    __shared__ uint2 scratch[kThreads / 32];
    __shared__ uint32_t s_row[kThreads], s_take[kThreads], s_run[kThreads], s_len[kThreads], s_flag[kThreads], s_back[2][kThreads / 32];
    const uint32_t ctas = CLUSTER ? gridDim.x : 1, cta = CLUSTER ? blockIdx.x : 0;
    const uint32_t tid = threadIdx.x, me = cta * kThreads + tid, all = ctas * kThreads;
    const uint32_t block = 1u << a.block_log2, most = min((uint64_t)a.width << a.block_log2, (uint64_t)kMost);
    after_previous();
    const int32_t listed = a.state[0];
    const uint32_t count = min((uint32_t)max(listed, 0), a.n_blocks);
    auto load = [&](uint32_t r, uint32_t& len, int32_t& add) {
        len = 0;
        add = 0;
        if (r < a.requests) {
            len = min((uint32_t)max(a.lengths[r], 0), most);
            add = a.added[r];
        }
    };
    auto blocks_of = [&](uint32_t tokens) { return (tokens + block - 1) >> a.block_log2; };

    // what comes back
    uint32_t back = 0, turn = 0;
    for (uint32_t r0 = 0; r0 < a.requests; r0 += kThreads) {
        uint32_t len;
        int32_t add;
        load(r0 + tid, len, add);
        uint32_t mine = add < 0 ? blocks_of(len) : 0, none = 0, total, unused;
        scan2(mine, none, total, unused, scratch);
        if (total == 0) continue;
        s_take[tid] = mine;
        __syncthreads();
        back = sat(back, come_back<CLUSTER>(a, r0, total, (uint64_t)count + back, ctas, cta, s_take, s_back[turn]));
        turn ^= 1;  // (a CTA may be a chunk ahead of one that still reads its counts)
        __syncthreads();
    }
    const uint32_t available = min(sat(count, back), a.n_blocks);
    if (back) sync_all<CLUSTER>();

    uint32_t rows = 0, taken = 0, given = 0, runs = 0, refused = 0;
    for (uint32_t r0 = 0; r0 < a.requests; r0 += kThreads) {
        const uint32_t r = r0 + tid;
        uint32_t len;
        int32_t add;
        load(r, len, add);
        const uint32_t n = max(add, 0), has = blocks_of(len);
        uint32_t row = min(n, a.rows), row_total, want_total;
        // the first scan needs to know which requests fit the rows, which is a matter of the sums before them
        uint32_t dummy = 0, unused;
        scan2(row, dummy, row_total, unused, scratch);
        row = min(sat(rows, row), a.rows);
        const uint64_t end = (uint64_t)len + n;
        const bool fits = end <= most && (uint64_t)row + n <= a.rows;
        const uint32_t after = fits ? blocks_of((uint32_t)end) : has;
        uint32_t want = n && fits ? after - has : 0, take = want;
        scan2(take, dummy, want_total, unused, scratch);
        take = sat(taken, take);
        const bool served = n && fits && (want == 0 || sat(take, want) <= available);
        uint32_t run = served ? ((len + n - 1) >> a.block_log2) - (len >> a.block_log2) + 1 : 0, run_total;
        uint32_t got = served ? want : 0, got_total;
        scan2(run, got, run_total, got_total, scratch);
        run = sat(runs, run);
        refused += __syncthreads_count(n && !served);
        s_row[tid] = row;
        s_take[tid] = take;
        s_run[tid] = run;
        s_len[tid] = len;
        s_flag[tid] = served;
        if (CLUSTER) sync_all<true>(); else __syncthreads();  // every CTA has read the chunk's lengths
        const uint32_t next_row = min(sat(rows, row_total), a.rows), next_run = sat(runs, run_total);
        if (cta == 0 && r < a.requests) {
            a.offsets[r] = (int32_t)row;
            a.lengths_out[r] = add < 0 ? 0 : (int32_t)(served ? len + n : len);
        }
        for (uint32_t i = rows + me; i < next_row; i += all) {
            const uint32_t o = owner(s_row, kThreads, i);
            a.positions[i] = s_flag[o] ? (int32_t)(s_len[o] + (i - s_row[o])) : -1;
        }
        // new blocks: the i-th one taken is the i-th from the end of the list (all requests before a served one that want any are served)
        for (uint32_t i = given + me; i < given + got_total; i += all) {
            const uint32_t o = owner(s_take, kThreads, i);
            a.table[(uint64_t)(r0 + o) * a.ld_table + blocks_of(s_len[o]) + (i - s_take[o])] = a.free_list[available - 1 - i];
        }
        for (uint32_t i = runs + me; i < min(next_run, a.n_runs); i += all) {
            const uint32_t o = owner(s_run, kThreads, i);
            const uint32_t len_o = s_len[o], k = i - s_run[o], col = (len_o >> a.block_log2) + k, has_o = blocks_of(len_o);
            const uint32_t row_end = o + 1 < kThreads ? s_row[o + 1] : next_row, lead = len_o & (block - 1);
            const uint32_t first = k ? (k << a.block_log2) - lead : 0, start = k ? 0 : lead;
            const uint32_t n_o = row_end - s_row[o];
            const int32_t id = col < has_o ? a.table[(uint64_t)(r0 + o) * a.ld_table + col] : a.free_list[available - 1 - (s_take[o] + col - has_o)];
            a.runs[i] = make_int4(id, (int)start, (int)(s_row[o] + first), (int)min(block - start, n_o - first));
        }
        rows = next_row;
        taken = sat(taken, want_total);
        given += got_total;
        runs = next_run;
        __syncthreads();
    }
    for (uint32_t i = rows + me; i < a.rows; i += all) a.positions[i] = -1;
    for (uint32_t i = runs + me; i < a.n_runs; i += all) a.runs[i] = make_int4(-1, 0, 0, 0);
    if (CLUSTER) sync_all<true>();  // every CTA has read the state
    if (me == 0) {
        a.offsets[a.requests] = (int32_t)rows;
        a.state_out[0] = (int32_t)(available - given);
        a.state_out[1] = (int32_t)refused;
    }
}

}  // namespace

int check_cache(const dr_kv_cache* cache)
{
    if (!cache) {
        set_error("NULL cache");
        return DR_ERR_INVALID;
    }
    int dev = -1;
    if (cudaGetDevice(&dev) != cudaSuccess || dev != cache->device) {
        set_error("current device differs from the cache's device");
        return DR_ERR_STATE;
    }
    return DR_OK;
}

}  // namespace dr

using namespace dr;

extern "C" {

int dr_kv_cache_create(const dr_kv_cache_desc* desc, dr_kv_cache** out)
{
    if (!out) {
        set_error("NULL out");
        return DR_ERR_INVALID;
    }
    *out = nullptr;
    if (!desc || desc->struct_size != sizeof(dr_kv_cache_desc)) {
        set_error("NULL descriptor or struct_size mismatch");
        return DR_ERR_INVALID;
    }
    const dr_kv_cache_desc& d = *desc;
    if (!d.n_blocks || !d.kv_heads || !d.k_dev || !d.v_dev || !d.k_scale_dev || !d.v_scale_dev) {
        set_error("zero cache dimension or NULL buffer");
        return DR_ERR_INVALID;
    }
    if (d.block_tokens != 16 && d.block_tokens != 32 && d.block_tokens != 64 && d.block_tokens != 128) {
        set_error("blocks hold 16, 32, 64 or 128 tokens");
        return DR_ERR_UNSUPPORTED;
    }
    if (d.head_dim != 64 && d.head_dim != 128) {
        set_error("heads have 64 or 128 dimensions");
        return DR_ERR_UNSUPPORTED;
    }
    if ((unsigned __int128)d.n_blocks * d.kv_heads * d.block_tokens > 0x7FFFFFFFull) {
        set_error("more than 2^31 - 1 rows of codes");
        return DR_ERR_UNSUPPORTED;
    }
    if (((uintptr_t)d.k_dev | (uintptr_t)d.v_dev) % 16 || ((uintptr_t)d.k_scale_dev | (uintptr_t)d.v_scale_dev) % 4) {
        set_error("codes off 16 bytes or scales off 4");
        return DR_ERR_ALIGN;
    }
    dr_kv_cache* c = new (std::nothrow) dr_kv_cache();
    if (!c) return DR_ERR_NOMEM;
    c->d = d;
    while ((1u << c->block_log2) < d.block_tokens) ++c->block_log2;
    int rc = [&]() -> int {
        DR_CUDA(cudaGetDevice(&c->device));
        DR_CUDA(cudaDeviceGetAttribute(&c->sms, cudaDevAttrMultiProcessorCount, c->device));
        return DR_OK;
    }();
    const uint64_t rows = (uint64_t)d.n_blocks * d.kv_heads * d.block_tokens;
    const uint32_t box = d.block_tokens < kBoxTokens ? d.block_tokens : kBoxTokens;
    if (rc == DR_OK) rc = prepare_attend_few();
    if (rc == DR_OK) rc = prepare_attend_many();
    if (rc == DR_OK) rc = encode_codes_map(&c->k_map, d.k_dev, d.head_dim, rows, box);
    if (rc == DR_OK) rc = encode_codes_map(&c->v_map, d.v_dev, d.head_dim, rows, box);
    if (rc) {
        delete c;
        return rc;
    }
    *out = c;
    return DR_OK;
}

int dr_kv_cache_destroy(dr_kv_cache* cache)
{
    delete cache;
    return DR_OK;
}

int dr_kv_extend(const dr_kv_cache* cache, const int32_t* added, const int32_t* lengths, int32_t* lengths_out, uint64_t requests,
                 int32_t* table, uint64_t ld_table, uint64_t width, int32_t* free_list, const int32_t* state, int32_t* state_out,
                 uint64_t rows, int32_t* offsets, int32_t* positions, int32_t* runs, uint64_t n_runs, void* cuda_stream)
{
    int rc = check_cache(cache);
    if (rc) return rc;
    if (requests > kMaxRequests || rows > kMaxStepRows || width > kMaxWidth || n_runs > kMaxStepRows) {
        set_error("requests, rows, runs or blocks of a request out of range");
        return DR_ERR_UNSUPPORTED;
    }
    if (!state || !state_out || !free_list || !offsets || (requests && (!added || !lengths || !lengths_out || !table || !width)) ||
        (rows && !positions) || (n_runs && !runs)) {
        set_error("NULL buffer or a table without columns");
        return DR_ERR_INVALID;
    }
    if (requests && !pitch_ok(requests, width, ld_table)) {
        set_error("leading dimension below the row's length or out of range");
        return DR_ERR_INVALID;
    }
    const uint64_t by_block = (rows >> cache->block_log2) + 2 * requests, need = rows < by_block ? rows : by_block;
    if (n_runs < need) {
        set_error("runs has room for %llu entries, the step may need %llu", (unsigned long long)n_runs, (unsigned long long)need);
        return DR_ERR_SIZE;
    }
    if (((uintptr_t)added | (uintptr_t)lengths | (uintptr_t)lengths_out | (uintptr_t)table | (uintptr_t)free_list | (uintptr_t)state |
         (uintptr_t)state_out | (uintptr_t)offsets | (uintptr_t)positions) % 4 || (uintptr_t)runs % 16) {
        set_error("a pointer off 4 bytes, or runs off 16");
        return DR_ERR_ALIGN;
    }
    ExtendArgs a{added, lengths, lengths_out, table, free_list, state, state_out, offsets, positions, (int4*)runs, ld_table,
                 (uint32_t)requests, (uint32_t)width, (uint32_t)rows, (uint32_t)n_runs, cache->d.n_blocks, cache->block_log2};
    // one CTA up to four entries a thread, then as many as that takes, up to a cluster of eight
    const uint64_t entries = rows + n_runs;
    unsigned ctas = 1;
    while (ctas < 8 && entries > 4ull * kThreads * ctas) ctas *= 2;
    cudaLaunchAttribute attr[2] = {overlap_attribute(), {}};
    attr[1].id = cudaLaunchAttributeClusterDimension;
    attr[1].val.clusterDim.x = ctas;
    attr[1].val.clusterDim.y = attr[1].val.clusterDim.z = 1;
    cudaLaunchConfig_t cfg{};
    cfg.gridDim = dim3(ctas);
    cfg.blockDim = dim3(kThreads);
    cfg.stream = (cudaStream_t)cuda_stream;
    cfg.attrs = attr;
    cfg.numAttrs = ctas > 1 ? 2 : 1;
    const cudaError_t e = cudaLaunchKernelEx(&cfg, ctas > 1 ? extend_kernel<true> : extend_kernel<false>, a);
    if (e != cudaSuccess) {
        cudaGetLastError();
        set_error("table launch: %s", cudaGetErrorString(e));
        return DR_ERR_CUDA;
    }
    return DR_OK;
}

}  // extern "C"
