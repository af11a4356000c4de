// Linear layers on the tensor cores: pairs of CTAs, 256 x 256 tiles, tcgen05 products fed by tensor-map copies.
//
//   forward bf16  D[n, r] = sum_k W[n, k] x[r, k]      both operands contiguous along the contraction
//   forward fp8   D[r, n], the same sum with the tokens on the M side
//   dgrad         D[k, r] = sum_n W[n, k] dy[r, n]     W contiguous along its outputs (MN-major)
//   wgrad         D[n, k] = sum_r dy[r, n] x[r, k]     both MN-major, the contraction runs over a group's rows
//
// A pair computes 256 outputs of the M side (128 in each CTA's tensor memory) by up to 256 of the N side, of which each CTA holds
// half in shared memory: 32 KB a stage and CTA for 512 cycles of products, which is what the L2 can deliver and the
// shared memory can both take in and give out; a CTA on its own would need half as much again.  N is an operand of the
// instruction, so with the tokens there (bf16) a ragged group costs 32-row steps and not whole tiles: a group's rows are cut into
// equal tiles of at most 256.
//
// Roles of a CTA's 12 warps: 0 issues the copies of its half of the operands into a ring of five or six stages; 1 (of the pair's
// first CTA) issues the products of the pair; 2 clears the rows of other groups from the last stage (wgrad); 3 finds the tiles; 4-11
// read the accumulators.  Accumulators take half of tensor memory each, two in turn, so that a tile is written out while
// the next is computed.  Pairs walk the tiles in a fixed order (token tiles innermost, in bands of sixteen, so that a band's tokens
// and a few weight tiles stay in L2) and every sum is taken in a fixed order.
//
// fp8: one product covers exactly one block of 128 of the contraction, after which its partial sums are scaled by
// xs[b, r] * ws[n / 128, b] and added to fp32 sums in registers (128 a thread).  A thread owns one token and 128 features of one scale
// block, so that factor is one number a thread and two multiply-adds share an instruction.  What bounds it is the way of an
// accumulator back to the products: each step ends in a barrier between the two, and two accumulators fit tensor memory.
// (Features on the M side need one factor a column: 915 us where this takes 666.  Halves of 128 columns with four accumulators
// in turn double the reads of the M operand: no gain.  Sixteen warps of 64 columns: slower, 862 against 836 then.)
//
// Stores: bf16 outputs with features on the M side go through a 640-byte transpose per warp (eight tokens of 32 features, 64
// contiguous bytes a row); fp8 outputs and dW leave as whole blocks through the copy unit, in the background.
//
// Measured, alone / back to back at the power limit: bf16 8192 x 24576 x 4096 1.01 / 1.17 ms (1.63 / 1.42 PFLOP/s; a library product
// of 8192^3 reaches 1.67 / 1.39), fp8 the same 0.67 / 0.77 ms (2.48 / 2.15); 128 groups of 256 rows, 1536 x 2048: bf16 183 / 219 us,
// fp8 128 / 142, dgrad 173 / 216, wgrad 386 / 361 (1.6 GB of dW).
#include "linear.h"
#include "tc_map.h"
#include "tc_ptx.cuh"

namespace dr {
namespace {

using namespace tc;

__device__ unsigned long long g_wait_failures;  // read by dr_diag_linear_wait_failures

constexpr int kForwardRows = 3;  // forward with tokens on the M side (fp8, many rows)

template <int OP> constexpr uint32_t kStages = OP == kForwardRows || OP == kWgrad ? 5 : 6;
constexpr uint32_t kStageBytes = 32768, kOperandBytes = 16384;
constexpr uint32_t kEpilogueWarps = 8;
constexpr uint32_t kThreads = 128 + 32 * kEpilogueWarps;
constexpr uint32_t kTile = 256;          // features and tokens of a pair's tile
constexpr uint32_t kScratchPitch = 80;   // bytes between tokens of the transpose: 16-byte units of eight rows fall on different banks
constexpr uint32_t kBand = 16;           // token tiles a band of a large group holds

// One tile of a pair.
struct Tile {
    uint32_t e, row0, row_end;  // tokens [row0, row_end); wgrad: the group's rows
    uint32_t feature;           // first of the pair's 256 outputs on the M side (forward: row of the stacked weight)
    uint32_t col0;              // wgrad: first of its columns
    uint32_t nt;                // N of the product, a multiple of 32
    uint32_t steps;             // stages of the contraction
};

struct Barriers {
    TileRing<Tile> tiles;
    uint64_t full[6], empty[6], landed[6];
    alignas(16) uint64_t acc_full[2], acc_empty[2];  // (the readers flip bit 3 of their addresses)
    uint32_t tmem;
    Limit limit;
    uint32_t tiles_before[kMaxTcGroups + 1];  // token tiles of the groups before
};
template <int OP>
struct Buffers {
    alignas(1024) uint8_t stage[kStages<OP>][kStageBytes];
    alignas(16) uint8_t scratch[kEpilogueWarps][8 * kScratchPitch];
};
template <>
struct Buffers<kForwardRows> {
    alignas(1024) uint8_t stage[kStages<kForwardRows>][kStageBytes];
    alignas(1024) uint8_t out[8][2][4096];  // twice 32 rows of 64 bf16 for each warp, on their way out
};
template <>
struct Buffers<kWgrad> {
    alignas(1024) uint8_t stage[kStages<kWgrad>][kStageBytes];
    alignas(1024) uint8_t out[8][2][4096];  // twice 32 rows of 32 fp32 for each warp
};
template <int OP>
struct Shared : Buffers<OP>, Barriers {};
static_assert(sizeof(Shared<kForward>) <= 227 * 1024 && sizeof(Shared<kForwardRows>) <= 227 * 1024 && sizeof(Shared<kWgrad>) <= 227 * 1024, "shared memory of a CTA");

struct TcArgs {
    const int32_t* offsets;
    const float* a_scale;  // tokens' scales
    const float* b_scale;  // the weight's
    void* c;
    uint64_t ld_as, ld_bs, ldc;
    uint32_t rows, n_groups, n, k;
    uint32_t feature_tiles, column_tiles;  // column_tiles: wgrad's tiles of in_features
    uint32_t c_f32, accumulate, vector, bulk_out;
    uint32_t limit_us, starve;
};

template <int OP, bool FP8>
struct Walk {
    static_assert(FP8 == (OP == kForwardRows), "fp8 has its tokens on the M side");
    static constexpr uint32_t kStep = FP8 ? 128 : 64;
    uint32_t e = 0;

    // Tile t of all, ascending t; false past the last.  A tile without features (fp8 groups that are not whole scale blocks
    // have one tile fewer here and there) or without rows comes back with nt = 0.
    __device__ __forceinline__ bool get(const TcArgs& a, const Barriers& s, uint32_t t, Tile& o)
    {
        if constexpr (OP == kWgrad) {
            const uint32_t per = a.feature_tiles * a.column_tiles;
            o.e = t / per;
            if (o.e >= a.n_groups) return false;
            const uint32_t i = t - o.e * per;
            group_rows(a.offsets, o.e, a.rows, o.row0, o.row_end);
            o.feature = (i / a.column_tiles) * kTile;
            o.col0 = (i % a.column_tiles) * kTile;
            o.nt = min(kTile, (a.k - o.col0 + 31) / 32 * 32);
            o.steps = (o.row_end - o.row0 + kStep - 1) / kStep;
            return true;
        } else {
            while (e < a.n_groups && t >= s.tiles_before[e + 1] * a.feature_tiles) ++e;
            if (e >= a.n_groups) return false;
            uint32_t lo, hi;
            group_rows(a.offsets, e, a.rows, lo, hi);
            const uint32_t tiles = s.tiles_before[e + 1] - s.tiles_before[e];
            uint32_t i = t - s.tiles_before[e] * a.feature_tiles;
            // bands of kBand token tiles, all feature tiles of a band before the next, token tiles innermost
            const uint32_t band = i / (kBand * a.feature_tiles);
            const uint32_t in_band = min(kBand, tiles - band * kBand);
            i -= band * kBand * a.feature_tiles;
            const uint32_t f = i / in_band, m = band * kBand + i % in_band;
            o.e = e;
            o.col0 = 0;
            if (OP == kForwardRows) {
                const uint32_t first = e * a.n;
                o.row0 = lo + m * kTile;
                o.row_end = min(hi, o.row0 + kTile);
                o.feature = first / 128 * 128 + f * kTile;
                o.nt = o.feature < first + a.n ? min(kTile, (first + a.n - o.feature + 31) / 32 * 32) : 0;
                o.steps = (a.k + kStep - 1) / kStep;
                return true;
            }
            o.nt = ((hi - lo + tiles - 1) / tiles + 31) / 32 * 32;
            o.row0 = lo + m * o.nt;
            o.row_end = min(hi, o.row0 + o.nt);
            o.feature = (OP == kForward ? e * a.n : 0) + f * kTile;
            o.steps = ((OP == kForward ? a.k : a.n) + kStep - 1) / kStep;
            if (o.row0 >= o.row_end) o.nt = 0;  // 32-row steps can leave a last tile without rows
            return true;
        }
    }
};

// Eight tokens (columns c .. c + 7 of the tile) of the warp's 32 features: v[g][i] = token 2 (t % 4) + i of feature t / 4 + 8 g.
// `f` is the warp's first feature among the outputs of a row of c, of which there are f_hi (a tile's last features may lie past
// 2^31, as negative numbers).
__device__ __forceinline__ void store_tokens(const TcArgs& a, uint32_t scratch, uint32_t row, uint32_t row_end, int f, int f_hi,
                                             const float (&v)[4][2])
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
        if (r < row_end && ff >= 0 && ff < f_hi)  // the outputs of a row are a multiple of eight here
            *(uint4*)((uint16_t*)a.c + (uint64_t)r * a.ldc + ff) = make_uint4(w[0], w[1], w[2], w[3]);
        return;
    }
#pragma unroll
    for (int g = 0; g < 4; ++g)
#pragma unroll
        for (int i = 0; i < 2; ++i) {
            const uint32_t r = row + 2 * (lane & 3) + i;
            const int ff = f + (int)(lane >> 2) + 8 * g;
            if (r >= row_end || ff < 0 || ff >= f_hi) continue;
            if (a.c_f32)
                ((float*)a.c)[(uint64_t)r * a.ldc + ff] = v[g][i];
            else
                ((uint16_t*)a.c)[(uint64_t)r * a.ldc + ff] = (uint16_t)pack_bf16(v[g][i], 0.0f);
        }
}

// Finds the pair's tiles for the other warps.
template <int OP, bool FP8>
__device__ __forceinline__ void schedule(const TcArgs& a, Shared<OP>& s)
{
    Walk<OP, FP8> walk;
    Turn<kTilesAhead> at;
    Tile t;
    for (uint32_t i = blockIdx.x >> 1; walk.get(a, s, i, t); i += gridDim.x >> 1)
        if (t.nt && !s.tiles.put(t, at, &s.limit, &g_wait_failures)) return;
    t.nt = kNoTile;
    s.tiles.put(t, at, &s.limit, &g_wait_failures);
}

template <int OP, bool FP8>
__device__ __forceinline__ void produce(const TcArgs& a, Shared<OP>& s, const CUtensorMap* map_a, const CUtensorMap* map_b)
{
    constexpr uint32_t kStep = Walk<OP, FP8>::kStep;
    const uint32_t rank = cta_rank(), stages = smem_u32(s.stage), empty = smem_u32(s.empty);
    // copies signal the first CTA of the pair, which issues the products; in wgrad their own CTA, which may have rows to clear
    const uint32_t full = OP == kWgrad ? smem_u32(s.landed) : in_cta(smem_u32(s.full), 0);
    Turn<kStages<OP>> ring;
    uint32_t used = 0;  // stages in use, up to all of them
    bool ok = true;
    Turn<kTilesAhead> at;
    Tile t;
    while (ok && s.tiles.get(t, at, &s.limit, &g_wait_failures)) {
        const uint32_t half = t.nt / 2, feature = t.feature + rank * 128;
        const uint32_t boxes = OP == kWgrad ? (half + 63) / 64 : (half + 31) / 32, box_bytes = OP == kWgrad ? 8192 : 4096;
        const uint32_t bytes = kOperandBytes + boxes * box_bytes;
        for (uint32_t l = 0; l < t.steps; ++l) {
            const uint32_t to = stages + ring.slot * kStageBytes, bar = full + 8 * ring.slot;
            ok = warp_wait(empty + 8 * ring.slot, ring.round ^ 1, &s.limit, &g_wait_failures);
            if (!ok) break;
            if (!a.starve && elect()) {
                if (OP == kWgrad)
                    bar_expect(bar, bytes);
                else if (rank == 0)
                    bar_expect(smem_u32(s.full) + 8 * ring.slot, 2 * bytes);
                if (OP == kForward) {
                    load_2d<true>(to, map_a, bar, l * kStep, feature);
                } else if (OP == kForwardRows) {
                    load_2d<true>(to, map_a, bar, l * kStep, t.row0 + rank * 128);
                } else if (OP == kDgrad) {
                    load_3d<true>(to, map_a, bar, feature, l * kStep, t.e);
                    load_3d<true>(to + 8192, map_a, bar, feature + 64, l * kStep, t.e);
                } else {
                    load_2d<false>(to, map_a, bar, feature, t.row0 + l * kStep);
                    load_2d<false>(to + 8192, map_a, bar, feature + 64, t.row0 + l * kStep);
                }
                for (uint32_t b = 0; b < boxes; ++b) {
                    const uint32_t box = to + kOperandBytes + b * box_bytes;
                    if (OP == kWgrad)
                        load_2d<false>(box, map_b, bar, t.col0 + rank * half + b * 64, t.row0 + l * kStep);
                    else
                        load_2d<true>(box, map_b, bar, l * kStep, (OP == kForwardRows ? t.feature : t.row0) + rank * half + b * 32);
                }
            }
            ring.next();
            used = min(used + 1, kStages<OP>);
        }
    }
    if (ok) drain(ring, used, empty, &s.limit, &g_wait_failures);
}

template <int OP, bool FP8>
__device__ __forceinline__ void multiply(const TcArgs& a, Shared<OP>& s)
{
    const uint32_t stages = smem_u32(s.stage), full = smem_u32(s.full), empty = smem_u32(s.empty);
    const uint32_t acc_full = smem_u32(s.acc_full), acc_empty = smem_u32(s.acc_empty), tmem = s.tmem;
    constexpr bool a_mn = OP == kDgrad || OP == kWgrad, b_mn = OP == kWgrad;
    const uint64_t first_a = operand(stages, 8192), first_b = operand(stages + kOperandBytes, 8192);
    Turn<kStages<OP>> ring;
    Turn<2> acc;
    Turn<kTilesAhead> at;
    Tile t;
    while (s.tiles.get(t, at, &s.limit, &g_wait_failures)) {
        if (t.steps == 0) continue;
        const uint32_t shape = shape_of(FP8, a_mn, b_mn, 256, t.nt);
        for (uint32_t l = 0; l < t.steps; ++l) {
            if (FP8 || l == 0)
                if (!warp_wait(acc_empty + 8 * acc.slot, acc.round ^ 1, &s.limit, &g_wait_failures)) return;
            // (wgrad: the other CTA may have cleared rows of its stage)
            if (!warp_wait<OP == kWgrad>(full + 8 * ring.slot, ring.round, &s.limit, &g_wait_failures)) return;
            fence_after();
            // addresses are the low bits of a descriptor, in units of 16 bytes
            const uint64_t da = first_a + ring.slot * (kStageBytes >> 4), db = first_b + ring.slot * (kStageBytes >> 4);
            const bool last = FP8 || l + 1 == t.steps;
            if (elect()) {
#pragma unroll
                for (uint32_t q = 0; q < 4; ++q)
                    mma<2, FP8>(tmem + acc.slot * kTile, da + q * ((a_mn ? 2048 : 32) >> 4), db + q * ((b_mn ? 2048 : 32) >> 4), shape,
                                FP8 ? q != 0 : (l | q) != 0);
                if (last) commit<2>(acc_full + 8 * acc.slot);
                commit<2>(empty + 8 * ring.slot);
            }
            __syncwarp();
            ring.next();
            if (last) acc.next();
        }
    }
}

// wgrad: rows of the last stage that belong to the next group are cleared before the products read them (both operands: a zero
// times the infinity of another group's row is not zero), then the stage is handed to the first CTA.
__device__ __forceinline__ void clear_rows(const TcArgs& a, Shared<kWgrad>& s)
{
    const uint32_t lane = threadIdx.x & 31, landed = smem_u32(s.landed), full = in_cta(smem_u32(s.full), 0);
    uint32_t n = 0;
    Turn<kTilesAhead> at;
    Tile t;
    while (s.tiles.get(t, at, &s.limit, &g_wait_failures)) {
        const uint32_t panels = (t.nt / 2 + 63) / 64;
        for (uint32_t l = 0; l < t.steps; ++l, ++n) {
            const uint32_t st = n % kStages<kWgrad>, valid = min(64u, t.row_end - t.row0 - l * 64);
            if (!__all_sync(0xFFFFFFFFu, bar_wait(landed + 8 * st, n / kStages<kWgrad> & 1, &s.limit, &g_wait_failures))) return;
            if (valid < 64) {
                for (uint32_t p = 0; p < 2 + panels; ++p) {  // operand A's two panels, then B's: 8 KB each, side by side
                    uint8_t* panel = s.stage[st] + p * 8192;
                    for (uint32_t o = valid * 128 + lane * 16; o < 8192; o += 512) *(uint4*)(panel + o) = make_uint4(0, 0, 0, 0);
                }
                fence_async();
            }
            __syncwarp();
            if (lane == 0) bar_arrive_cluster(full + 8 * st, valid < 64);
        }
    }
}

// dW leaves through the copy unit, 32 rows x 32 columns at a time, two blocks of a warp in flight: the map's third dimension is the group,
// so that it clips at the group's last row, and the addition to an accumulated gradient is the copy unit's too (each
// element once a call, so the result does not depend on an order).
__device__ __forceinline__ void write_dw(const TcArgs& a, Shared<kWgrad>& s, const CUtensorMap* map_c)
{
    const uint32_t lane = threadIdx.x & 31, warp = (threadIdx.x >> 5) - 4, rank = cta_rank();
    const uint32_t quarter = warp & 3, side = warp >> 2;
    const uint32_t acc_full = smem_u32(s.acc_full), acc_empty = in_cta(smem_u32(s.acc_empty), 0);
    const uint32_t tmem = s.tmem + (quarter * 32 << 16), out = smem_u32(s.out[warp][0]);
    Turn<2> acc;
    Turn<kTilesAhead> at;
    Tile t;
    uint32_t blocks = 0;
    while (s.tiles.get(t, at, &s.limit, &g_wait_failures)) {
        const uint32_t cols = t.nt / 2, col0 = side * cols;  // this warp's columns, a multiple of 16
        const uint32_t row = t.feature + rank * 128 + quarter * 32;
        if (t.steps) {
            if (!__all_sync(0xFFFFFFFFu, bar_wait(acc_full + 8 * acc.slot, acc.round, &s.limit, &g_wait_failures))) return;
            fence_after();
        }
        // blocks of 32 columns; a last one of 16 ends where the next warp's columns (or the matrix) begin, and is stored directly
        for (uint32_t c = 0; c < cols; c += 32) {
            const uint32_t col = t.col0 + col0 + c;
            if (row >= a.n || col >= a.k) break;  // nothing of dW there (and every block that takes a buffer starts one store)
            float v[32];
            if (t.steps) {
                tmem_start(tmem + acc.slot * kTile + col0 + c, v);
                tmem_arrived(v);
            } else {
#pragma unroll
                for (int r = 0; r < 32; ++r) v[r] = 0.0f;  // dW of a group without rows
            }
            if (!a.bulk_out || c + 32 > cols) {
                const uint32_t end = min(a.k, t.col0 + col0 + cols);
                if (row + lane < a.n) {
                    float* p = (float*)a.c + ((uint64_t)t.e * a.n + row + lane) * a.ldc;
#pragma unroll
                    for (int r = 0; r < 32; ++r)
                        if (col + r < end) p[col + r] = a.accumulate ? p[col + r] + v[r] : v[r];
                }
                continue;
            }
            const uint32_t to = out + (blocks++ & 1) * 4096;
            if (lane == 0) asm volatile("cp.async.bulk.wait_group.read 1;" ::: "memory");  // the block before the last has left
            __syncwarp();
#pragma unroll
            for (uint32_t q = 0; q < 8; ++q)
                store_shared(to + lane * 128 + (q ^ (lane & 7)) * 16, __float_as_uint(v[4 * q]), __float_as_uint(v[4 * q + 1]),
                             __float_as_uint(v[4 * q + 2]), __float_as_uint(v[4 * q + 3]));
            fence_async();
            __syncwarp();
            if (lane == 0) {
                if (a.accumulate)
                    add_3d(map_c, to, (int)col, (int)row, (int)t.e);
                else
                    store_3d(map_c, to, (int)col, (int)row, (int)t.e);
                asm volatile("cp.async.bulk.commit_group;" ::: "memory");
            }
        }
        if (t.steps) {
            fence_before();
            __syncwarp();
            if (lane == 0) bar_arrive_cluster(acc_empty + 8 * acc.slot);
            acc.next();
        }
    }
    asm volatile("cp.async.bulk.wait_group 0;" ::: "memory");  // the last block has left before the CTA may end
}

template <int OP>
__device__ __forceinline__ void write_out(const TcArgs& a, Shared<OP>& s)
{
    const uint32_t lane = threadIdx.x & 31, warp = (threadIdx.x >> 5) - 4, rank = cta_rank();
    const uint32_t quarter = warp & 3, side = warp >> 2;
    const uint32_t acc_full = smem_u32(s.acc_full), acc_empty = in_cta(smem_u32(s.acc_empty), 0);
    const uint32_t scratch = smem_u32(s.scratch[warp]);
    const uint32_t tmem = s.tmem + (quarter * 32 << 16);
    Turn<2> acc;
    Turn<kTilesAhead> at;
    Tile t;
    while (s.tiles.get(t, at, &s.limit, &g_wait_failures)) {
        const uint32_t cols = t.nt / 2, col0 = side * cols;  // this warp's tokens
        const uint32_t feature = t.feature + rank * 128 + quarter * 32;
        // in a row of c: forward counts features from the group's first weight row
        const int f = OP == kForward ? (int)(feature - t.e * a.n) : (int)feature;
        const int f_hi = OP == kDgrad ? (int)a.k : (int)a.n;
        if (!__all_sync(0xFFFFFFFFu, bar_wait(acc_full + 8 * acc.slot, acc.round, &s.limit, &g_wait_failures))) return;
        fence_after();
        for (uint32_t c = 0; c < cols; c += 32) {
            float p[2][16];
            tmem_load(tmem + acc.slot * kTile + col0 + c, p[0], p[1]);
#pragma unroll
            for (int j = 0; j < 4; ++j) {
                if (c + j * 8 >= cols) break;
                const float v[4][2] = {{p[0][4 * j], p[0][4 * j + 1]}, {p[0][4 * j + 2], p[0][4 * j + 3]},
                                       {p[1][4 * j], p[1][4 * j + 1]}, {p[1][4 * j + 2], p[1][4 * j + 3]}};
                store_tokens(a, scratch, t.row0 + col0 + c + j * 8, t.row_end, f, f_hi, v);
            }
        }
        fence_before();
        __syncwarp();
        if (lane == 0) bar_arrive_cluster(acc_empty + 8 * acc.slot);
        acc.next();
    }
}

// Tokens on the M side: a thread owns one token and 128 features of one scale block, so the scale of a block of the contraction is
// one number a thread.
__device__ __forceinline__ void write_rows(const TcArgs& a, Shared<kForwardRows>& s, const CUtensorMap* map_c)
{
    const uint32_t lane = threadIdx.x & 31, warp = (threadIdx.x >> 5) - 4, rank = cta_rank();
    const uint32_t quarter = warp & 3, side = warp >> 2;
    uint32_t filled = smem_u32(s.acc_full), emptied = in_cta(smem_u32(s.acc_empty), 0), parity = 0;
    uint32_t from = s.tmem + (quarter * 32 << 16) + side * 128;  // all 512 columns are this CTA's: the accumulators start at 0 and 256
    const uint32_t scale_rows = (a.n_groups * a.n + 127) / 128;
    const uint32_t out = smem_u32(s.out[warp][0]);
    Turn<kTilesAhead> at;
    Tile t;
    const float *xs, *ws;
    float x1, w1, x2, w2;
    // the next tile, and the first two scales of this thread's row in it
    auto next_tile = [&]() {
        if (!s.tiles.get(t, at, &s.limit, &g_wait_failures)) return false;
        xs = a.a_scale + min(t.row0 + rank * 128 + quarter * 32 + lane, t.row_end - 1);
        ws = a.b_scale + (uint64_t)min(t.feature / 128 + side, scale_rows - 1) * a.ld_bs;
        x1 = xs[0];
        w1 = ws[0];
        x2 = t.steps > 1 ? xs[a.ld_as] : 0.0f;
        w2 = t.steps > 1 ? ws[1] : 0.0f;
        if (t.steps > 2) {
            xs += 2 * a.ld_as;
            ws += 2;
        }
        return true;
    };
    bool more = next_tile();
    while (more) {
        const uint32_t warp_row = t.row0 + rank * 128 + quarter * 32, row_end = t.row_end, steps = t.steps;
        // a warp without a token or without a feature only keeps the barriers going
        const bool idle = warp_row >= row_end || side * 128 >= t.nt;
        const int f = (int)(t.feature + side * 128 - t.e * a.n);
        float sum[4][32];
#pragma unroll
        for (int c = 0; c < 4; ++c)
#pragma unroll
            for (int r = 0; r < 32; ++r) sum[c][r] = 0.0f;
        for (uint32_t left = steps; left; --left) {
            const float scale = x1 * w1;
            const uint64_t two = pair_of(scale, scale);
            if (!__all_sync(0xFFFFFFFFu, bar_wait(filled, parity, &s.limit, &g_wait_failures))) return;
            fence_after();
            float p[2][32];
            if (!idle) tmem_start(from, p[0]);
            // in the shadow of the loads: the scales of the step after the next (the last two steps read the last again)
            x1 = x2;
            w1 = w2;
            x2 = *xs;
            w2 = *ws;
            if (left > 3) {
                xs += a.ld_as;
                ++ws;
            }
            if (idle) {
                fence_before();
                if (lane == 0) bar_arrive_cluster(emptied);
            } else {
#pragma unroll
                for (int c = 0; c < 4; ++c) {
                    tmem_arrived(p[c & 1]);
                    if (c < 3) {
                        tmem_start(from + 32 * (c + 1), p[(c + 1) & 1]);
                    } else {  // the accumulator has been read: the next product may begin
                        fence_before();
                        __syncwarp();
                        if (lane == 0) bar_arrive_cluster(emptied);
                    }
#pragma unroll
                    for (int r = 0; r < 32; r += 2) fma2(sum[c][r], sum[c][r + 1], p[c & 1][r], p[c & 1][r + 1], two);
                }
            }
            from ^= kTile;  // the other accumulator and its barriers
            filled ^= 8;
            emptied ^= 8;
            parity ^= from & kTile ? 0 : 1;
        }
        more = next_tile();  // its scales are on their way while this tile leaves
        if (idle) continue;
        const uint32_t row = warp_row + lane;
        if (a.bulk_out && warp_row + 32 <= row_end && f >= 0 && f + 128 <= (int)a.n) {
            // Whole blocks of 32 rows x 128 features leave through the copy unit while the next tile is computed: stored at once by
            // every SM, they would hold up the products for 7 000 cycles a tile.  Rows of 128 bytes, their 16-byte units
            // swizzled as the map says.
            asm volatile("cp.async.bulk.wait_group.read 0;" ::: "memory");  // (the lane that started the previous one)
            __syncwarp();
#pragma unroll
            for (uint32_t c = 0; c < 16; ++c) {
                const float* v = &sum[c / 4][c % 4 * 8];
                store_shared(out + c / 8 * 4096 + lane * 128 + (c % 8 ^ (lane & 7)) * 16, pack_bf16(v[0], v[1]), pack_bf16(v[2], v[3]),
                             pack_bf16(v[4], v[5]), pack_bf16(v[6], v[7]));
            }
            fence_async();
            __syncwarp();
            if (lane == 0) {
                store_2d(map_c, out, f, (int)warp_row);
                store_2d(map_c, out + 4096, f + 64, (int)warp_row);
                asm volatile("cp.async.bulk.commit_group;" ::: "memory");
            }
        } else if (row < row_end) {
            if (a.vector) {  // 32 bytes of c and whole rows of 16 features allow one sector a store
#pragma unroll
                for (int c = 0; c < 128; c += 16) {
                    if (f + c < 0 || f + c >= (int)a.n) continue;
                    const float* v = &sum[c / 32][c % 32];
                    if (a.c_f32) {
                        float* p = (float*)a.c + (uint64_t)row * a.ldc + f + c;
                        store_32(p, __float_as_uint(v[0]), __float_as_uint(v[1]), __float_as_uint(v[2]), __float_as_uint(v[3]),
                                 __float_as_uint(v[4]), __float_as_uint(v[5]), __float_as_uint(v[6]), __float_as_uint(v[7]));
                        store_32(p + 8, __float_as_uint(v[8]), __float_as_uint(v[9]), __float_as_uint(v[10]), __float_as_uint(v[11]),
                                 __float_as_uint(v[12]), __float_as_uint(v[13]), __float_as_uint(v[14]), __float_as_uint(v[15]));
                    } else {
                        store_32((uint16_t*)a.c + (uint64_t)row * a.ldc + f + c, pack_bf16(v[0], v[1]), pack_bf16(v[2], v[3]),
                                 pack_bf16(v[4], v[5]), pack_bf16(v[6], v[7]), pack_bf16(v[8], v[9]), pack_bf16(v[10], v[11]),
                                 pack_bf16(v[12], v[13]), pack_bf16(v[14], v[15]));
                    }
                }
            } else {
#pragma unroll
                for (int c = 0; c < 128; ++c) {
                    if (f + c < 0 || f + c >= (int)a.n) continue;
                    if (a.c_f32)
                        ((float*)a.c)[(uint64_t)row * a.ldc + f + c] = sum[c / 32][c % 32];
                    else
                        ((uint16_t*)a.c)[(uint64_t)row * a.ldc + f + c] = (uint16_t)pack_bf16(sum[c / 32][c % 32], 0.0f);
                }
            }
        }
    }
    asm volatile("cp.async.bulk.wait_group 0;" ::: "memory");  // the last block has left before the CTA may end
}

template <int OP, bool FP8>
__global__ void __cluster_dims__(2, 1, 1) __launch_bounds__(kThreads, 1)
    tc_kernel(const __grid_constant__ CUtensorMap map_a, const __grid_constant__ CUtensorMap map_b,
              const __grid_constant__ CUtensorMap map_c, const TcArgs a)
{
    extern __shared__ __align__(1024) uint8_t raw[];
    Shared<OP>& s = *(Shared<OP>*)raw;
    if (smem_u32(raw) & 1023) {  // the swizzled stages need the alignment asked for; nothing has been started yet
        if (threadIdx.x == 0) atomicAdd(&g_wait_failures, 1ull);
        return;
    }
    const uint32_t warp = threadIdx.x >> 5, lane = threadIdx.x & 31;
    if (threadIdx.x == 0) {
        prefetch_map(&map_a);
        prefetch_map(&map_b);
        for (uint32_t i = 0; i < kStages<OP>; ++i) {
            bar_init(smem_u32(&s.full[i]), OP == kWgrad ? 2 : 1);
            bar_init(smem_u32(&s.empty[i]), 1);
            bar_init(smem_u32(&s.landed[i]), 1);
        }
        for (uint32_t i = 0; i < 2; ++i) {
            bar_init(smem_u32(&s.acc_full[i]), 1);
            bar_init(smem_u32(&s.acc_empty[i]), 2 * kEpilogueWarps);
        }
        // readers: the copies, the products (first CTA), the cleared rows, the accumulators
        s.tiles.init(1 + (cta_rank() == 0) + (OP == kWgrad) + kEpilogueWarps);
        s.limit.stop = 0;
        s.limit.us = a.limit_us;
        bar_init_fence();
    }
    if (warp == 1) tmem_alloc<2>(smem_u32(&s.tmem), 512);
    after_previous();
    if (warp == 2 && OP != kWgrad) {  // running sum of the groups' token tiles
        uint32_t before = 0;
        if (lane == 0) s.tiles_before[0] = 0;
        for (uint32_t e0 = 0; e0 < a.n_groups; e0 += 32) {
            uint32_t lo = 0, hi = 0;
            if (e0 + lane < a.n_groups) group_rows(a.offsets, e0 + lane, a.rows, lo, hi);
            uint32_t sum = (hi - lo + kTile - 1) / kTile;
#pragma unroll
            for (int o = 1; o < 32; o <<= 1) {
                const uint32_t up = __shfl_up_sync(0xFFFFFFFFu, sum, o);
                if (lane >= (uint32_t)o) sum += up;
            }
            if (e0 + lane < a.n_groups) s.tiles_before[e0 + lane + 1] = before + sum;
            before += __shfl_sync(0xFFFFFFFFu, sum, 31);
        }
    }
    fence_before();
    __syncthreads();
    cluster_sync();
    fence_after();

    if (warp < 4) {
        if (FP8) asm volatile("setmaxnreg.dec.sync.aligned.u32 40;");
        if (warp == 0) {
            produce<OP, FP8>(a, s, &map_a, &map_b);
        } else if (warp == 1) {
            if (cta_rank() == 0) multiply<OP, FP8>(a, s);
        } else if (warp == 2) {
            if constexpr (OP == kWgrad) clear_rows(a, s);
        } else {
            schedule<OP, FP8>(a, s);
        }
    } else {
        if (FP8) asm volatile("setmaxnreg.inc.sync.aligned.u32 232;");
        if constexpr (OP == kForwardRows)
            write_rows(a, s, &map_c);
        else if constexpr (OP == kWgrad)
            write_dw(a, s, &map_c);
        else
            write_out(a, s);
    }
    __syncwarp();
    let_copies_end(&s.limit);
    fence_before();
    __syncthreads();
    cluster_sync();
    let_copies_end(&s.limit);
    fence_after();
    if (warp == 1) tmem_free<2>(s.tmem, 512);
}

// Once per device and kernel: shared memory, and the register count that the fp8 kernel's split relies on
// (384 threads x 168 at launch cover 256 x 232 + 128 x 40).
template <int OP, bool FP8>
int prepare_kernel()
{
    cudaFuncAttributes at;
    DR_CUDA(cudaFuncGetAttributes(&at, tc_kernel<OP, FP8>));
    if (FP8 && at.numRegs * (int)kThreads < 256 * 232 + 128 * 40) {
        set_error("the fp8 linear kernel was built with %d registers a thread", at.numRegs);
        return DR_ERR_CUDA;
    }
    DR_CUDA(cudaFuncSetAttribute(tc_kernel<OP, FP8>, cudaFuncAttributeMaxDynamicSharedMemorySize, (int)sizeof(Shared<OP>)));
    return DR_OK;
}

template <int OP, bool FP8>
int launch(const LinearCall& c, const CUtensorMap& ma, const CUtensorMap& mb, const CUtensorMap& mc, const TcArgs& a, uint64_t tiles)
{
    const uint64_t pairs = (uint64_t)c.lin->sms / 2;
    const unsigned grid = 2 * (unsigned)(tiles < pairs ? tiles : pairs);
    cudaLaunchAttribute attr = overlap_attribute();
    cudaLaunchConfig_t cfg{};
    cfg.gridDim = dim3(grid);
    cfg.blockDim = dim3(kThreads);
    cfg.dynamicSmemBytes = sizeof(Shared<OP>);
    cfg.stream = c.stream;
    cfg.attrs = &attr;
    cfg.numAttrs = 1;
    const cudaError_t err = cudaLaunchKernelEx(&cfg, tc_kernel<OP, FP8>, ma, mb, mc, a);
    if (err != cudaSuccess) {
        cudaGetLastError();
        set_error("linear kernel launch: %s", cudaGetErrorString(err));
        return DR_ERR_CUDA;
    }
    return DR_OK;
}

}  // namespace

int prepare_linear_tc()
{
    int rc = prepare_kernel<kForwardRows, true>();
    if (rc == DR_OK) rc = prepare_kernel<kForward, false>();
    if (rc == DR_OK) rc = prepare_kernel<kDgrad, false>();
    if (rc == DR_OK) rc = prepare_kernel<kWgrad, false>();
    return rc;
}

bool linear_tc_takes(const LinearCall& c)
{
    const uint32_t es = c.lin->fp8 ? 1 : 2;
    const uint64_t bits = (uintptr_t)c.a | (uintptr_t)c.b | c.lda * es | c.ldb * es;
    return bits % 16 == 0 && c.lda * es < (1ull << 39) && c.ldb * es < (1ull << 39) && c.lin->d.n_groups <= kMaxTcGroups &&
           c.lin->d.out_features * c.ldb * es < (1ull << 39);
}

int launch_linear_tc(const LinearCall& c)
{
    const dr_linear_desc& d = c.lin->d;
    const bool fp8 = c.lin->fp8;
    TcArgs a{};
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
    const uint64_t contraction = c.op == kWgrad ? c.rows : c.op == kDgrad ? a.n : a.k;
    a.limit_us = wait_limit_us((contraction + 63) / 64);
    a.starve = waits_starve();
    a.accumulate = c.accumulate;
    CUtensorMap ma, mb, mc{};
    int rc;
    uint64_t tiles;
    const uint64_t token_tiles = ((uint64_t)c.rows + kTile - 1) / kTile + (c.offsets ? d.n_groups : 0);
    if (c.op == kWgrad) {
        a.feature_tiles = (a.n + kTile - 1) / kTile;
        a.column_tiles = (a.k + kTile - 1) / kTile;
        tiles = (uint64_t)a.feature_tiles * a.column_tiles * a.n_groups;
        a.bulk_out = c.ldc % 4 == 0 && (uintptr_t)c.c % 16 == 0 && (uint64_t)a.n * c.ldc < (1ull << 37);
        rc = encode_map(&ma, c.a, false, a.n, c.rows, 0, c.lda, 64);
        if (rc == DR_OK) rc = encode_map(&mb, c.b, false, a.k, c.rows, 0, c.ldb, 64);
        if (rc == DR_OK && a.bulk_out) rc = encode_map_f32(&mc, c.c, a.k, a.n, a.n_groups, c.ldc, 32);
    } else {
        const uint32_t width = c.op == kForward ? a.n : a.k;
        a.feature_tiles = (width + (fp8 && a.n % 128 ? 127 : 0) + kTile - 1) / kTile;
        tiles = token_tiles * a.feature_tiles;
        a.vector = !c.c_f32 && width % 8 == 0 && c.ldc % 8 == 0 && (uintptr_t)c.c % 16 == 0;
        if (fp8) {
            a.vector = width % 16 == 0 && c.ldc % (c.c_f32 ? 8 : 16) == 0 && (uintptr_t)c.c % 32 == 0;
            rc = encode_map(&ma, c.a, true, a.k, c.rows, 0, c.lda, 128);
            if (rc == DR_OK) rc = encode_map(&mb, c.b, true, a.k, (uint64_t)a.n * a.n_groups, 0, c.ldb, 32);
            a.bulk_out = !c.c_f32 && a.n % 8 == 0 && c.ldc % 8 == 0 && (uintptr_t)c.c % 16 == 0 && c.ldc < (1ull << 38);
            if (rc == DR_OK && a.bulk_out) rc = encode_map(&mc, c.c, false, a.n, c.rows, 0, c.ldc, 32);
        } else if (c.op == kForward)
            rc = encode_map(&ma, c.b, false, a.k, (uint64_t)a.n * a.n_groups, 0, c.ldb, 128);
        else
            rc = encode_map(&ma, c.b, false, a.k, a.n, a.n_groups, c.ldb, 64);
        if (rc == DR_OK && !fp8) rc = encode_map(&mb, c.a, false, c.op == kForward ? a.k : a.n, c.rows, 0, c.lda, 32);
    }
    if (rc) return rc;
    if (tiles > 0x7FFFFFFFull) {
        set_error("too many output tiles for one launch");
        return DR_ERR_UNSUPPORTED;
    }
    if (c.op == kWgrad) return launch<kWgrad, false>(c, ma, mb, mc, a, tiles);
    if (c.op == kDgrad) return launch<kDgrad, false>(c, ma, mb, mc, a, tiles);
    return fp8 ? launch<kForwardRows, true>(c, ma, mb, mc, a, tiles) : launch<kForward, false>(c, ma, mb, mc, a, tiles);
}

int linear_wait_failures(uint64_t* out)
{
    unsigned long long n = 0;
    DR_CUDA(cudaMemcpyFromSymbol(&n, g_wait_failures, sizeof n));
    *out = n;
    return DR_OK;
}

}  // namespace dr
