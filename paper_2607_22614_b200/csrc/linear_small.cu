// Forward products of few rows (decoding): the weights are read once at the memory's rate, everything else hides behind that.
//
// D[n, r] = sum_k W[n, k] x[r, k] with 128 features on the M side of a CTA's product and a group's rows, at most 64 at a time in
// steps of 16, on its N side.  Bound: HBM, the weights' bytes; a stage holds two steps of the contraction, 32 KB of weights and 4 KB for
// each 16 rows, and three stages keep 96 KB of weights in flight on every SM.  What else costs time is the issuing of a step (waits,
// products, commits), hence the two steps a stage.  There is no time to lose in filling the machine either: with
// fewer feature blocks than SMs, a cluster of up to eight CTAs splits the contraction, and its CTAs add their fp32 sums through
// distributed shared memory, always in the order of their ranks.
//
// Roles: warp 0 copies the operands, 1 issues the products, 2 copies the scales (fp8), 3 finds the tiles,
// 4-11 read the accumulators.  fp8 takes a new
// accumulator (eight of 64 columns in turn) for every block of 128 of the contraction, scales it and adds it to fp32 sums in
// registers, as the kernel for many rows does.
#include "linear.h"
#include "tc_map.h"
#include "tc_ptx.cuh"

namespace dr {
namespace {

using namespace tc;

__device__ unsigned long long g_wait_failures;

constexpr uint32_t kTurn = 2;  // steps of the contraction that a stage holds and that are handed over at a time
constexpr uint32_t kRowsTile = 64, kStages = 3, kWeightBytes = 16384, kRowBytes = kRowsTile * 128;
constexpr uint32_t kStageBytes = kTurn * (kWeightBytes + kRowBytes);  // weights of each step, then rows of each step
constexpr uint32_t kReaders = 8, kThreads = 128 + 32 * kReaders, kBuffers = 512 / kRowsTile;
constexpr uint32_t kTurns = kBuffers / kTurn;
constexpr uint32_t kScratchPitch = 80;
constexpr uint32_t kTurnPitch = 36;  // floats

struct Tile {
    uint32_t e, row0, row_end, feature, nt;  // feature: row of the stacked weight; nt: N of the product
    uint32_t step0, steps;                   // this CTA's part of the contraction
};

struct Shared {
    alignas(1024) uint8_t stage[kStages][kStageBytes];
    alignas(16) float turn[kReaders][16][kTurnPitch];              // a warp's features of 16 rows, on their way to the cluster
    alignas(16) float sums[kRowsTile + kMaxSplit][128];     // [CTA][its rows that end here][features]
    alignas(16) uint8_t scratch[kReaders][8 * kScratchPitch];
    alignas(16) float scale[kBuffers][kRowsTile + 4];  // the rows' scales of a block, then the weight's
    uint64_t full[kStages], empty[kStages];
    uint64_t acc_full[kTurns], acc_empty[kTurns], scale_full[kTurns], scale_empty[kTurns];
    uint64_t sums_full, sums_empty;
    TileRing<Tile> tiles;
    uint32_t tmem;
    Limit limit;
    uint32_t tiles_before[kMaxTcGroups + 1];  // row tiles of the groups before
};

struct Args {
    const int32_t* offsets;
    const float* a_scale;
    const float* b_scale;
    void* c;
    uint64_t ld_as, ld_bs, ldc;
    uint32_t rows, n_groups, n, k;
    uint32_t feature_blocks;
    uint32_t split;  // CTAs of a cluster
    uint32_t c_f32, vector;
    uint32_t limit_us, starve;
};

template <bool FP8>
struct Walk {
    static constexpr uint32_t kStep = FP8 ? 128 : 64;
    uint32_t e = 0;
    __device__ __forceinline__ bool get(const Args& a, const Shared& s, uint32_t t, Tile& o)
    {
        while (e < a.n_groups && t >= s.tiles_before[e + 1] * a.feature_blocks) ++e;
        if (e >= a.n_groups) return false;
        uint32_t lo, hi;
        group_rows(a.offsets, e, a.rows, lo, hi);
        const uint32_t tiles = s.tiles_before[e + 1] - s.tiles_before[e], i = t - s.tiles_before[e] * a.feature_blocks;
        const uint32_t f = i / tiles, m = i - f * tiles;  // the tiles of one feature block follow each other: its weights stay in L2
        const uint32_t first = e * a.n;
        o.e = e;
        o.nt = ((hi - lo + tiles - 1) / tiles + 15) / 16 * 16;
        o.row0 = lo + m * o.nt;
        o.row_end = min(hi, o.row0 + o.nt);
        o.feature = (FP8 ? first / 128 * 128 : first) + f * 128;
        if (o.feature >= first + a.n || o.row0 >= o.row_end) o.nt = 0;
        const uint32_t all = (a.k + kStep - 1) / kStep, part = a.split > 1 ? cta_rank() : 0;
        o.step0 = part * all / a.split;
        o.steps = (part + 1) * all / a.split - o.step0;
        return true;
    }
};

// Eight rows (columns of the accumulator) of the warp's 32 features, as the kernel for many rows stores them.
__device__ __forceinline__ void store_rows(const Args& a, uint32_t scratch, uint32_t row, uint32_t row_end, int f, const float (&v)[4][2])
{
    const uint32_t lane = threadIdx.x & 31;
    if (a.vector) {
        __syncwarp();
        store_transposed(scratch + (lane & 7) * kScratchPitch + (lane >> 3) * 16, pack_bf16(v[0][0], v[0][1]),
                         pack_bf16(v[1][0], v[1][1]), pack_bf16(v[2][0], v[2][1]), pack_bf16(v[3][0], v[3][1]));
        __syncwarp();
        const uint32_t r = row + (lane >> 2);
        const int ff = f + (int)(lane & 3) * 8;
        uint32_t w[4];
        asm volatile("ld.shared.v4.b32 {%0,%1,%2,%3}, [%4];"
                     : "=r"(w[0]), "=r"(w[1]), "=r"(w[2]), "=r"(w[3])
                     : "r"(scratch + (lane >> 2) * kScratchPitch + (lane & 3) * 16));
        if (r < row_end && ff >= 0 && ff < (int)a.n) *(uint4*)((uint16_t*)a.c + (uint64_t)r * a.ldc + ff) = make_uint4(w[0], w[1], w[2], w[3]);
        return;
    }
#pragma unroll
    for (int g = 0; g < 4; ++g)
#pragma unroll
        for (int i = 0; i < 2; ++i) {
            const uint32_t r = row + 2 * (lane & 3) + i;
            const int ff = f + (int)(lane >> 2) + 8 * g;
            if (r >= row_end || ff < 0 || ff >= (int)a.n) continue;
            if (a.c_f32)
                ((float*)a.c)[(uint64_t)r * a.ldc + ff] = v[g][i];
            else
                ((uint16_t*)a.c)[(uint64_t)r * a.ldc + ff] = (uint16_t)pack_bf16(v[g][i], 0.0f);
        }
}

// Finds the cluster's tiles for the other warps.
template <bool FP8>
__device__ __forceinline__ void schedule(const Args& a, Shared& s)
{
    Walk<FP8> walk;
    Turn<kTilesAhead> turn;
    Tile t;
    const uint32_t stride = gridDim.x / a.split;
    for (uint32_t i = blockIdx.x / a.split; walk.get(a, s, i, t); i += stride)
        if (t.nt && !s.tiles.put(t, turn, &s.limit, &g_wait_failures)) return;
    t.nt = kNoTile;
    s.tiles.put(t, turn, &s.limit, &g_wait_failures);
}

template <bool FP8>
__device__ __forceinline__ void produce(const Args& a, Shared& s, const CUtensorMap* map_w, const CUtensorMap* map_x)
{
    constexpr uint32_t kStep = Walk<FP8>::kStep;
    const uint32_t stages = smem_u32(s.stage), full = smem_u32(s.full), empty = smem_u32(s.empty);
    Turn<kStages> ring;
    uint32_t used = 0;  // stages in use, up to all of them
    Turn<kTilesAhead> turn;
    Tile t;
    bool ok = true;
    while (ok && s.tiles.get(t, turn, &s.limit, &g_wait_failures)) {
        for (uint32_t l = 0; l < t.steps; l += kTurn) {
            const uint32_t at = stages + ring.slot * kStageBytes, bar = full + 8 * ring.slot, steps = min(kTurn, t.steps - l);
            ok = warp_wait(empty + 8 * ring.slot, ring.round ^ 1, &s.limit, &g_wait_failures);
            if (!ok) break;
            if (!a.starve && elect()) {
                bar_expect(bar, steps * (kWeightBytes + t.nt * 128));
                for (uint32_t q = 0; q < steps; ++q) load_2d<false>(at + q * kWeightBytes, map_w, bar, (t.step0 + l + q) * kStep, t.feature);
                for (uint32_t q = 0; q < steps; ++q)
                    for (uint32_t r = 0; r < t.nt; r += 16)
                        load_2d<false>(at + kTurn * kWeightBytes + q * kRowBytes + r * 128, map_x, bar, (t.step0 + l + q) * kStep, t.row0 + r);
            }
            ring.next();
            used = min(used + 1, kStages);
        }
    }
    drain(ring, used, empty, &s.limit, &g_wait_failures);
}

template <bool FP8>
__device__ __forceinline__ void multiply(const Args& a, Shared& s)
{
    const uint32_t full = smem_u32(s.full), empty = smem_u32(s.empty);
    const uint32_t acc_full = smem_u32(s.acc_full), acc_empty = smem_u32(s.acc_empty), tmem = s.tmem;
    const uint64_t first_a = operand(smem_u32(s.stage), 0), first_b = operand(smem_u32(s.stage) + kTurn * kWeightBytes, 0);
    Turn<kStages> ring;
    Turn<kTurns> acc;
    Turn<kTilesAhead> turn;
    Tile t;
    while (s.tiles.get(t, turn, &s.limit, &g_wait_failures)) {
        const uint32_t shape = shape_of(FP8, false, false, 128, t.nt);
        for (uint32_t l = 0; l < t.steps; l += kTurn) {
            if (FP8 || l == 0)
                if (!warp_wait(acc_empty + 8 * acc.slot, acc.round ^ 1, &s.limit, &g_wait_failures)) return;
            if (!warp_wait(full + 8 * ring.slot, ring.round, &s.limit, &g_wait_failures)) return;
            fence_after();
            const uint64_t da = first_a + ring.slot * (kStageBytes >> 4), db = first_b + ring.slot * (kStageBytes >> 4);
            const uint32_t d = tmem + acc.slot * kTurn * kRowsTile;
            const bool last = FP8 || l + kTurn >= t.steps, both = l + 1 < t.steps;
            if (elect()) {
#pragma unroll
                for (uint32_t q = 0; q < 4; ++q) mma<1, FP8>(d, da + 2 * q, db + 2 * q, shape, FP8 ? q != 0 : (l | q) != 0);
                if (both) {
#pragma unroll
                    for (uint32_t q = 0; q < 4; ++q)
                        mma<1, FP8>(d + (FP8 ? kRowsTile : 0), da + (kWeightBytes >> 4) + 2 * q, db + (kRowBytes >> 4) + 2 * q, shape,
                                    FP8 ? q != 0 : 1);
                }
                if (last) commit<1>(acc_full + 8 * acc.slot);
                commit<1>(empty + 8 * ring.slot);
            }
            __syncwarp();
            ring.next();
            if (last) acc.next();
        }
    }
}

__device__ __forceinline__ void copy_scales(const Args& a, Shared& s)
{
    const uint32_t lane = threadIdx.x & 31, full = smem_u32(s.scale_full), empty = smem_u32(s.scale_empty);
    const uint32_t scale_rows = (a.n_groups * a.n + 127) / 128;
    Turn<kTurns> acc;
    Turn<kTilesAhead> turn;
    Tile t;
    while (s.tiles.get(t, turn, &s.limit, &g_wait_failures)) {
        const float* xs = a.a_scale + t.row0;
        const float* ws = a.b_scale + (uint64_t)min(t.feature / 128, scale_rows - 1) * a.ld_bs;
        const uint32_t left = t.row_end - t.row0;
        for (uint32_t l = 0; l < t.steps; l += kTurn) {
            if (!__all_sync(0xFFFFFFFFu, bar_wait(empty + 8 * acc.slot, acc.round ^ 1, &s.limit, &g_wait_failures))) return;
#pragma unroll
            for (uint32_t q = 0; q < kTurn; ++q) {
                if (l + q >= t.steps) break;
                const uint32_t to = smem_u32(s.scale[acc.slot * kTurn + q]);
                const float* from = xs + (t.step0 + l + q) * a.ld_as;
#pragma unroll
                for (uint32_t j = lane; j < kRowsTile; j += 32) copy_4(to + 4 * j, from + (j < left ? j : 0), j < left);
                if (lane == 0) copy_4(to + 4 * kRowsTile, ws + t.step0 + l + q, true);
            }
            copies_arrive(full + 8 * acc.slot);
            acc.next();
        }
    }
}

template <bool FP8>
__device__ __forceinline__ void write_out(const Args& a, Shared& s)
{
    const uint32_t lane = threadIdx.x & 31, warp = (threadIdx.x >> 5) - 4;
    const uint32_t acc_full = smem_u32(s.acc_full), acc_empty = smem_u32(s.acc_empty);
    const uint32_t scale_full = smem_u32(s.scale_full), scale_empty = smem_u32(s.scale_empty);
    const uint32_t quarter = warp & 3, side = warp >> 2;  // 32 features, and 32 of the rows
    const uint32_t scratch = smem_u32(s.scratch[warp]), tmem = s.tmem + (quarter * 32 << 16) + side * 32;
    Turn<kTurns> acc;
    uint32_t handed = 0;
    // r / split for the rows of a tile: exact for r < 64 and split <= 8
    const uint32_t magic = (65536 + a.split - 1) / a.split;
    Turn<kTilesAhead> turn;
    Tile t;
    while (s.tiles.get(t, turn, &s.limit, &g_wait_failures)) {
        const bool idle = side * 32 >= t.nt;  // (such a warp only keeps the barriers going)
        float sum[2][16];
        if (FP8) {
#pragma unroll
            for (int h = 0; h < 2; ++h)
#pragma unroll
                for (int r = 0; r < 16; ++r) sum[h][r] = 0.0f;
        }
        for (uint32_t l = 0; l < t.steps; l += FP8 ? kTurn : t.steps) {
            bool ok = !FP8 || bar_wait(scale_full + 8 * acc.slot, acc.round, &s.limit, &g_wait_failures);
            ok = ok && bar_wait(acc_full + 8 * acc.slot, acc.round, &s.limit, &g_wait_failures);
            if (!__all_sync(0xFFFFFFFFu, ok)) return;
            fence_after();
            const uint32_t from = tmem + acc.slot * kTurn * kRowsTile;
            if (idle) {
            } else if (FP8) {
#pragma unroll
                for (uint32_t q = 0; q < kTurn; ++q) {
                    if (l + q >= t.steps) break;
                    const float* sc = s.scale[acc.slot * kTurn + q];
                    const float w = sc[kRowsTile];
                    const uint64_t ww = pair_of(w, w);
                    sc += side * 32 + 2 * (lane & 3);
                    float p[2][16];
                    tmem_load(from + q * kRowsTile, p[0], p[1]);
#pragma unroll
                    for (int j = 0; j < 4; ++j) {
                        const uint64_t two = mul2(*(const uint64_t*)(sc + j * 8), ww);
#pragma unroll
                        for (int h = 0; h < 2; ++h) {
                            fma2(sum[h][4 * j], sum[h][4 * j + 1], p[h][4 * j], p[h][4 * j + 1], two);
                            fma2(sum[h][4 * j + 2], sum[h][4 * j + 3], p[h][4 * j + 2], p[h][4 * j + 3], two);
                        }
                    }
                }
            } else {
                tmem_load(from, sum[0], sum[1]);
            }
            fence_before();
            __syncwarp();
            if (lane == 0) {
                bar_arrive(acc_empty + 8 * acc.slot);
                if (FP8) bar_arrive(scale_empty + 8 * acc.slot);
            }
            acc.next();
        }
        const int f = (int)(t.feature + quarter * 32 - t.e * a.n);  // in a row of c
        if (a.split == 1) {
#pragma unroll
            for (int j = 0; j < 4; ++j) {
                const uint32_t c = side * 32 + j * 8;
                if (c >= t.nt) break;
                const float v[4][2] = {{sum[0][4 * j], sum[0][4 * j + 1]}, {sum[0][4 * j + 2], sum[0][4 * j + 3]},
                                       {sum[1][4 * j], sum[1][4 * j + 1]}, {sum[1][4 * j + 2], sum[1][4 * j + 3]}};
                store_rows(a, scratch, t.row0 + c, t.row_end, f, v);
            }
            continue;
        }
        // Every row of the tile ends in one CTA of the cluster (row r in CTA r mod split): the others send it their sums with
        // stores that count on its barrier, so that no CTA waits on a fence, and it adds them in the order of the ranks.
        const uint32_t rank = cta_rank(), rows = t.row_end - t.row0;
        const uint32_t most = (kRowsTile - 1) * magic / 65536 + 1, owned = rows > rank ? (rows - 1 - rank) * magic / 65536 + 1 : 0;
        if (!__all_sync(0xFFFFFFFFu, bar_wait<true>(smem_u32(&s.sums_empty), (handed & 1) ^ 1, &s.limit, &g_wait_failures))) return;
        if (warp == 0 && lane == 0) bar_expect(smem_u32(&s.sums_full), owned * a.split * 512);
#pragma unroll
        for (int c = 0; c < 2; ++c) {  // sixteen rows at a time
            if (side * 32 + c * 16 >= t.nt) break;
            __syncwarp();
#pragma unroll
            for (int j = 0; j < 2; ++j)
#pragma unroll
                for (int g = 0; g < 4; ++g)
#pragma unroll
                    for (int q = 0; q < 2; ++q)
                        s.turn[warp][j * 8 + 2 * (lane & 3) + q][(lane >> 2) + 8 * g] =
                            sum[g >> 1][4 * (c * 2 + j) + 2 * (g & 1) + q];
            __syncwarp();
#pragma unroll
            for (uint32_t i = 0; i < 4; ++i) {
                const uint32_t r = side * 32 + c * 16 + i * 4 + (lane >> 3);
                if (r >= rows) continue;
                const float4 v = *(const float4*)&s.turn[warp][r & 15][(lane & 7) * 4];
                const uint32_t nth = r * magic / 65536, to = r - nth * a.split;
                store_counted(in_cta(smem_u32(&s.sums[rank * most + nth][quarter * 32 + (lane & 7) * 4]), to), v,
                              in_cta(smem_u32(&s.sums_full), to));
            }
        }
        if (!__all_sync(0xFFFFFFFFu, bar_wait<true>(smem_u32(&s.sums_full), handed & 1, &s.limit, &g_wait_failures))) return;
        for (uint32_t o = warp; o < owned; o += kReaders) {
            float v[4] = {0.0f, 0.0f, 0.0f, 0.0f};
            for (uint32_t q = 0; q < a.split; ++q) {
                const float4 p = *(const float4*)&s.sums[q * most + o][lane * 4];
                v[0] += p.x;
                v[1] += p.y;
                v[2] += p.z;
                v[3] += p.w;
            }
            const int ff = (int)(t.feature + lane * 4 - t.e * a.n);
            const uint64_t at = (uint64_t)(t.row0 + rank + o * a.split) * a.ldc;
            if (a.vector && ff >= 0 && ff < (int)a.n) {  // the rows of c are a multiple of eight features here
                *(uint2*)((uint16_t*)a.c + at + ff) = make_uint2(pack_bf16(v[0], v[1]), pack_bf16(v[2], v[3]));
            } else if (!a.vector) {
#pragma unroll
                for (int j = 0; j < 4; ++j) {
                    if (ff + j < 0 || ff + j >= (int)a.n) continue;
                    if (a.c_f32)
                        ((float*)a.c)[at + ff + j] = v[j];
                    else
                        ((uint16_t*)a.c)[at + ff + j] = (uint16_t)pack_bf16(v[j], 0.0f);
                }
            }
        }
        __syncwarp();
        if (lane < a.split) bar_arrive_cluster(in_cta(smem_u32(&s.sums_empty), lane), true);
        ++handed;
    }
}

template <bool FP8>
__global__ void __launch_bounds__(kThreads, 1)
    small_kernel(const __grid_constant__ CUtensorMap map_w, const __grid_constant__ CUtensorMap map_x, const Args a)
{
    extern __shared__ __align__(1024) uint8_t raw[];
    Shared& s = *(Shared*)raw;
    if (smem_u32(raw) & 1023) {  // the swizzled stages need the alignment asked for; nothing has been started yet
        if (threadIdx.x == 0) atomicAdd(&g_wait_failures, 1ull);
        return;
    }
    const uint32_t warp = threadIdx.x >> 5, lane = threadIdx.x & 31;
    if (threadIdx.x == 0) {
        prefetch_map(&map_w);
        prefetch_map(&map_x);
        for (uint32_t i = 0; i < kStages; ++i) {
            bar_init(smem_u32(&s.full[i]), 1);
            bar_init(smem_u32(&s.empty[i]), 1);
        }
        for (uint32_t i = 0; i < kTurns; ++i) {
            bar_init(smem_u32(&s.acc_full[i]), 1);
            bar_init(smem_u32(&s.acc_empty[i]), kReaders);
            bar_init(smem_u32(&s.scale_full[i]), 32);
            bar_init(smem_u32(&s.scale_empty[i]), kReaders);
        }
        bar_init(smem_u32(&s.sums_full), 1);
        bar_init(smem_u32(&s.sums_empty), kReaders * a.split);
        s.tiles.init(2 + FP8 + kReaders);  // readers: the copies, the products, the scales, the accumulators
        s.limit.stop = 0;
        s.limit.us = a.limit_us;
        bar_init_fence();
    }
    if (warp == 1) tmem_alloc<1>(smem_u32(&s.tmem), 512);
    after_previous();
    for (uint32_t e = threadIdx.x; e < a.n_groups; e += kThreads) {
        uint32_t lo, hi;
        group_rows(a.offsets, e, a.rows, lo, hi);
        s.tiles_before[e + 1] = (hi - lo + kRowsTile - 1) / kRowsTile;
    }
    fence_before();
    __syncthreads();
    if (warp == 2) {  // running sum of the groups' row tiles
        uint32_t before = 0;
        if (lane == 0) s.tiles_before[0] = 0;
        for (uint32_t e0 = 0; e0 < a.n_groups; e0 += 32) {
            uint32_t sum = e0 + lane < a.n_groups ? s.tiles_before[e0 + lane + 1] : 0;
#pragma unroll
            for (int o = 1; o < 32; o <<= 1) {
                const uint32_t up = __shfl_up_sync(0xFFFFFFFFu, sum, o);
                if (lane >= (uint32_t)o) sum += up;
            }
            if (e0 + lane < a.n_groups) s.tiles_before[e0 + lane + 1] = before + sum;
            before += __shfl_sync(0xFFFFFFFFu, sum, 31);
        }
    }
    __syncthreads();
    if (a.split > 1) cluster_sync();
    fence_after();

    if (warp == 0) {
        produce<FP8>(a, s, &map_w, &map_x);
    } else if (warp == 1) {
        multiply<FP8>(a, s);
    } else if (warp == 2) {
        if (FP8) copy_scales(a, s);
    } else if (warp == 3) {
        schedule<FP8>(a, s);
    } else {
        write_out<FP8>(a, s);
    }
    __syncwarp();
    let_copies_end(&s.limit);
    fence_before();
    __syncthreads();
    if (a.split > 1) cluster_sync();  // other CTAs may still be reading this one's sums
    let_copies_end(&s.limit);
    fence_after();
    if (warp == 1) tmem_free<1>(s.tmem, 512);
}

constexpr size_t kSharedBytes = sizeof(Shared);

// CTAs that share a tile's contraction: `fit[s]` clusters of s CTAs run at the same time, so that `tiles` take
// ceil(tiles / fit[s]) rounds.  A round is 1 / s of the contraction and the end of a tile, which costs about two steps' time, or
// five to eight with an exchange of 16 to 64 rows (measured, 64 rows: a step of 128 takes 0.3 us, the exchange 2.5 us).
uint32_t choose_split(uint64_t tiles, const uint32_t (&fit)[kMaxSplit + 1], uint32_t steps, uint32_t rows)
{
    uint32_t best = 1;
    uint64_t least = ~0ull;
    for (uint32_t s = 1; s <= kMaxSplit && (s == 1 || s * 2 <= steps); ++s) {
        if (fit[s] == 0) continue;
        const uint64_t time = ((tiles + fit[s] - 1) / fit[s]) * ((steps + s - 1) / s + (s == 1 ? 2 : 4 + (rows + 15) / 16));
        if (time < least) {
            best = s;
            least = time;
        }
    }
    return best;
}

cudaLaunchConfig_t config(cudaLaunchAttribute (&attr)[2], uint64_t clusters, uint32_t split, cudaStream_t stream)
{
    attr[0].id = cudaLaunchAttributeClusterDimension;
    attr[0].val.clusterDim.x = split;
    attr[0].val.clusterDim.y = attr[0].val.clusterDim.z = 1;
    attr[1] = overlap_attribute();
    cudaLaunchConfig_t cfg{};
    cfg.gridDim = dim3((unsigned)(clusters * split));
    cfg.blockDim = dim3(kThreads);
    cfg.dynamicSmemBytes = kSharedBytes;
    cfg.stream = stream;
    cfg.attrs = attr;
    cfg.numAttrs = 2;
    return cfg;
}

template <bool FP8>
int launch(const LinearCall& c, const CUtensorMap& mw, const CUtensorMap& mx, const Args& a, uint64_t tiles)
{
    const uint64_t clusters = c.lin->fit[a.split];
    cudaLaunchAttribute attr[2];
    const cudaLaunchConfig_t cfg = config(attr, tiles < clusters ? tiles : clusters, a.split, c.stream);
    const cudaError_t err = cudaLaunchKernelEx(&cfg, small_kernel<FP8>, mw, mx, a);
    if (err != cudaSuccess) {
        cudaGetLastError();
        set_error("linear kernel launch: %s", cudaGetErrorString(err));
        return DR_ERR_CUDA;
    }
    return DR_OK;
}

}  // namespace

int prepare_linear_small(uint32_t (&fit)[kMaxSplit + 1])
{
    DR_CUDA(cudaFuncSetAttribute(small_kernel<true>, cudaFuncAttributeMaxDynamicSharedMemorySize, (int)kSharedBytes));
    DR_CUDA(cudaFuncSetAttribute(small_kernel<false>, cudaFuncAttributeMaxDynamicSharedMemorySize, (int)kSharedBytes));
    for (uint32_t s = 1; s <= kMaxSplit; ++s) {
        cudaLaunchAttribute attr[2];
        const cudaLaunchConfig_t cfg = config(attr, 64, s, nullptr);
        int n = 0;
        DR_CUDA(cudaOccupancyMaxActiveClusters(&n, small_kernel<true>, &cfg));
        fit[s] = n > 0 ? (uint32_t)n : 0;
    }
    if (fit[1] == 0) {
        set_error("the linear kernel does not fit this device");
        return DR_ERR_CUDA;
    }
    return DR_OK;
}

int launch_linear_small(const LinearCall& c)
{
    const dr_linear_desc& d = c.lin->d;
    const bool fp8 = c.lin->fp8;
    Args a{};
    a.offsets = c.offsets;
    a.a_scale = c.a_scale;
    a.b_scale = d.scale_dev;
    a.c = c.c;
    a.ld_as = c.ld_scale;
    a.ld_bs = d.scale_ld;
    a.ldc = c.ldc;
    a.rows = c.rows;
    a.n_groups = d.n_groups;
    a.n = (uint32_t)d.out_features;
    a.k = (uint32_t)d.in_features;
    a.c_f32 = c.c_f32;
    a.limit_us = wait_limit_us((a.k + 63ull) / 64);
    a.starve = waits_starve();
    a.vector = !c.c_f32 && a.n % 8 == 0 && c.ldc % 8 == 0 && (uintptr_t)c.c % 16 == 0;
    a.feature_blocks = (a.n + (fp8 && a.n % 128 ? 127 : 0) + 127) / 128;
    // at most one row tile more than full ones for each group that has rows
    const uint64_t spare = c.offsets ? (c.rows < d.n_groups ? c.rows : d.n_groups) : 0;
    const uint64_t tiles = (c.offsets ? c.rows / kRowsTile + spare : (c.rows + kRowsTile - 1) / kRowsTile) * a.feature_blocks;
    if (tiles > 0x7FFFFFFFull) {
        set_error("too many output tiles for one launch");
        return DR_ERR_UNSUPPORTED;
    }
    const uint32_t step = fp8 ? 128 : 64;
    a.split = choose_split(tiles, c.lin->fit, (a.k + step - 1) / step, c.rows < kRowsTile ? c.rows : kRowsTile);
    CUtensorMap mw, mx;
    int rc = encode_map(&mw, c.b, fp8, a.k, (uint64_t)a.n * a.n_groups, 0, c.ldb, 128);
    if (rc == DR_OK) rc = encode_map(&mx, c.a, fp8, a.k, c.rows, 0, c.lda, 16);
    if (rc) return rc;
    return fp8 ? launch<true>(c, mw, mx, a, tiles) : launch<false>(c, mw, mx, a, tiles);
}

int linear_small_wait_failures(uint64_t* out)
{
    unsigned long long n = 0;
    DR_CUDA(cudaMemcpyFromSymbol(&n, g_wait_failures, sizeof n));
    *out = n;
    return DR_OK;
}

}  // namespace dr
