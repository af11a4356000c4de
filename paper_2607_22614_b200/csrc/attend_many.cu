// Attention over the 8-bit cache for many rows of a request: prompts, on the tensor cores (sm_100a).
//
// A CTA takes 256 rows of one request and cache head (the query heads that share the head, times 256 / group tokens), as two halves of 128,
// and walks the tokens that they may see, 64 at a time.  For each half and 64 tokens
//   S = Q K^T      tcgen05, fp8: the keys' codes as the cache holds them, brought in by tensor maps and never converted; a query row,
//                  scaled by a power of two, is the sum of two rows of codes (bf16 has eight significant bits, e4m3 four), both
//                  products into the same fp32 accumulator.  Exact but for bits below 2^-17 of the row's maximum.
//   P = exp2(...)  a thread a row, the row's 64 logits in registers: no shuffles, one pass with the running maximum and sum
//   O += P V       tcgen05, fp16: P goes back to tensor memory, over S, and is the product's first operand from there; the values'
//                  codes become fp16, exactly, in four warps of their own
// Tensor memory holds two S of 64 columns for each half, so the next S is computed while the exponentials of this one are.  (One S of 128 columns, which
// has to wait for the P over it to be read: a tile took 4600 cycles, 2100 of them exponentials and 1600 waiting for S.)  Exponentials (16 a
// cycle), products and the shared memory's reads for them would each take some 2100 to 2600 cycles for 128 tokens: what bounds it is how well
// they overlap.
//
// As in the few-row kernel the running maximum is that of log2(p) + log2(value scale) (attend.h); O is multiplied anew only when it grows by more than
// 2^4, so that p scale in fp16 is at most 2^15 and normal down to 2^-25 of the largest.
//
// Warps: 0-3 and 4-7 the exponentials of the two halves, 8-11 the values' codes, 12 the copies, 14 and 15 the products of the halves.
// CTAs are started in the order of their number: the longest request first, and a request's last rows, which see the most tokens, first.
// Measured: a tile 2.11 us, a CTA's start and end some 6; a prompt of 8192 tokens, 32 query over 8 cache heads of 128: 571 us = 960 TFLOP/s (a
// library product of 8192^3: 1694; with half of the blocks without values 949 us); 3501 and 4500 tokens, these behind 4501 others: 619 to 655 us
// in a graph, 690 a pass among other inputs (966 to 913 and 867).
#include "attend.h"
#include "linear.h"
#include "tc_ptx.cuh"

namespace dr {
namespace {

using namespace tc;

__device__ unsigned long long g_wait_failures;  // read by dr_diag_linear_wait_failures

constexpr uint32_t kThreads = 512, kHalf = 128, kRowsCta = 2 * kHalf;
constexpr uint32_t kTile = 128, kStep = 64;  // tokens of a copy, and of a product
constexpr uint32_t kKeyStages = 3, kCodeStages = 2, kValueStages = 2, kMetas = 4;
constexpr uint32_t kRanked = 128;  // requests up to which the longest are begun first
constexpr uint32_t kGroups = kTile / 16, kStepGroups = kStep / 16;  // of sixteen tokens, which share a block
constexpr int kByFma = 3;  // pairs of each eight whose exponentials multiply-adds take (a tile: 2.23 us with none, 2.11 with 2 or 3, 2.16 with 4)
constexpr float kTop = 11.0f, kLag = 4.0f;

struct Meta {
    float k_scale[kGroups], v_log[kGroups], v_inv[kGroups];
    uint32_t held;   // a bit for each group
    uint32_t apart;  // and one where the value scale is not near
    uint32_t token;  // first of the tile
};

template <int D>
struct Shared {
    alignas(1024) uint8_t q[2][2][kHalf * D];  // [half][codes, codes of the rest]
    alignas(1024) uint8_t k[kKeyStages][kTile * D];
    alignas(1024) uint8_t codes[kCodeStages][kTile * D];
    alignas(1024) uint8_t v[kValueStages][kTile * D * 2];
    Meta meta[kMetas];
    uint64_t k_full[kKeyStages], k_empty[kKeyStages], c_full[kCodeStages], c_empty[kCodeStages], v_full[kValueStages], v_empty[kValueStages];
    uint64_t q_full[2], s_full[2][2], p_full[2][2], o_done[2], o_last[2];  // of each half; S and P of even and odd steps
    uint32_t tmem;
    Limit limit;
    uint32_t sums[kThreads / 32];
    uint32_t request, item;
    float apart_r[kRowsCta], apart_l[kRowsCta];  // the rows' sums of p that have exponentials of their own, relative to 2^r
    uint32_t lengths[kRanked], tiles[kRanked], ranked[kRanked];
};
static_assert(sizeof(Shared<128>) <= 227 * 1024, "shared memory of a CTA");

// What a CTA works on.
struct Item {
    Request q;
    uint32_t r, head, rows0, rows;  // rows0: first of its rows among the request's n * group
    Tiles tiles;
};

__device__ __forceinline__ uint32_t tiles_of_rows(const AttendArgs& a, uint32_t r)
{
    if (r >= a.requests) return 0;
    const uint32_t rows = request_of(a, r).n * a.group;
    return rows > kFewRows ? (rows + kRowsCta - 1) / kRowsCta : 0;
}

__device__ __forceinline__ void mma_ts(uint32_t d, uint32_t a, uint64_t b, uint32_t shape, uint32_t add)
{
    asm volatile("{\n.reg .pred p;\nsetp.ne.u32 p, %4, 0;\ntcgen05.mma.cta_group::1.kind::f16 [%0], [%1], %2, %3, p;\n}"
                 ::"r"(d), "r"(a), "l"(b), "r"(shape), "r"(add) : "memory");
}
// 16 columns of the thread's own lane times f, and back.
__device__ __forceinline__ void tmem_scale(uint32_t addr, float f)
{
    float v[16];
    asm volatile("tcgen05.ld.sync.aligned.32x32b.x16.b32 {%0,%1,%2,%3,%4,%5,%6,%7,%8,%9,%10,%11,%12,%13,%14,%15}, [%16];\n"
                 "tcgen05.wait::ld.sync.aligned;"
                 : "=f"(v[0]), "=f"(v[1]), "=f"(v[2]), "=f"(v[3]), "=f"(v[4]), "=f"(v[5]), "=f"(v[6]), "=f"(v[7]), "=f"(v[8]), "=f"(v[9]), "=f"(v[10]), "=f"(v[11]), "=f"(v[12]), "=f"(v[13]), "=f"(v[14]), "=f"(v[15])
                 : "r"(addr)
                 : "memory");
#pragma unroll
    for (int k = 0; k < 16; ++k) v[k] *= f;
    asm volatile("tcgen05.st.sync.aligned.32x32b.x16.b32 [%0], {%1,%2,%3,%4,%5,%6,%7,%8,%9,%10,%11,%12,%13,%14,%15,%16};"
                 ::"r"(addr), "f"(v[0]), "f"(v[1]), "f"(v[2]), "f"(v[3]), "f"(v[4]), "f"(v[5]), "f"(v[6]), "f"(v[7]), "f"(v[8]), "f"(v[9]), "f"(v[10]), "f"(v[11]), "f"(v[12]), "f"(v[13]), "f"(v[14]), "f"(v[15])
                 : "memory");
}
// 16 columns of the thread's own lane; complete after tmem_stored().
__device__ __forceinline__ void tmem_store(uint32_t addr, const uint32_t (&v)[16])
{
    asm volatile("tcgen05.st.sync.aligned.32x32b.x16.b32 [%0], {%1,%2,%3,%4,%5,%6,%7,%8,%9,%10,%11,%12,%13,%14,%15,%16};"
                 ::"r"(addr), "r"(v[0]), "r"(v[1]), "r"(v[2]), "r"(v[3]), "r"(v[4]), "r"(v[5]), "r"(v[6]), "r"(v[7]), "r"(v[8]), "r"(v[9]), "r"(v[10]), "r"(v[11]), "r"(v[12]), "r"(v[13]), "r"(v[14]), "r"(v[15])
                 : "memory");
}
__device__ __forceinline__ void tmem_stored() { asm volatile("tcgen05.wait::st.sync.aligned;" ::: "memory"); }
__device__ __forceinline__ float exp2_of(float x)
{
    float y;
    asm("ex2.approx.ftz.f32 %0, %1;" : "=f"(y) : "f"(x));
    return y;
}
__device__ __forceinline__ uint32_t half2_of(float lo, float hi)
{
    uint32_t d;
    asm("cvt.rn.f16x2.f32 %0, %1, %2;" : "=r"(d) : "f"(hi), "f"(lo));
    return d;
}
__device__ __forceinline__ uint32_t e4m3x2_of(float lo, float hi)
{
    uint16_t d;
    asm("cvt.rn.satfinite.e4m3x2.f32 %0, %1, %2;" : "=h"(d) : "f"(hi), "f"(lo));
    return d;
}
__device__ __forceinline__ void e4m3x4_to_half(uint32_t codes, uint32_t& lo, uint32_t& hi)
{
    asm("{\n.reg .b16 a, b;\nmov.b32 {a, b}, %2;\ncvt.rn.f16x2.e4m3x2 %0, a;\ncvt.rn.f16x2.e4m3x2 %1, b;\n}" : "=r"(lo), "=r"(hi) : "r"(codes));
}
// The larger one; NaN where one of them is.
__device__ __forceinline__ float max_nan(float a, float b)
{
    float d;
    asm("max.NaN.f32 %0, %1, %2;" : "=f"(d) : "f"(a), "f"(b));
    return d;
}
__device__ __forceinline__ uint64_t fma_pair(uint64_t a, uint64_t b, uint64_t c)
{
    uint64_t d;
    asm("fma.rn.f32x2 %0, %1, %2, %3;" : "=l"(d) : "l"(a), "l"(b), "l"(c));
    return d;
}
__device__ __forceinline__ uint64_t add_pair(uint64_t a, uint64_t b)
{
    uint64_t d;
    asm("add.rn.f32x2 %0, %1, %2;" : "=l"(d) : "l"(a), "l"(b));
    return d;
}
// 2^x for a pair by multiply-adds, where the exponential unit (16 a cycle) is busy: x = n + f with n a whole number, which the addition of
// 1.5 * 2^23 leaves in the low bits, |f| <= 1/2, and 2^f by a polynomial of degree 4 whose largest relative error is the least possible
// (2.6e-6, found by weighted least squares), n added to its exponent.  Below 2^-126: 2^-126.  Not for NaN.
__device__ __forceinline__ uint64_t exp2_pair(float x0, float x1)
{
    const uint64_t big = 0x4B4000004B400000ull, minus_big = 0xCB400000CB400000ull, minus_one = 0xBF800000BF800000ull;
    const uint64_t x = tc::pair_of(fmaxf(x0, -126.0f), fmaxf(x1, -126.0f)), t = add_pair(x, big);
    const uint64_t f = fma_pair(add_pair(t, minus_big), minus_one, x);
    uint64_t y = fma_pair(f, tc::pair_of(0.009570102f, 0.009570102f), tc::pair_of(0.05591786f, 0.05591786f));
    y = fma_pair(y, f, tc::pair_of(0.24024744f, 0.24024744f));
    y = fma_pair(y, f, tc::pair_of(0.6931218f, 0.6931218f));
    y = fma_pair(y, f, tc::pair_of(0.9999993f, 0.9999993f));
    uint32_t y0, y1, t0, t1;
    asm("mov.b64 {%0, %1}, %2;" : "=r"(y0), "=r"(y1) : "l"(y));
    asm("mov.b64 {%0, %1}, %2;" : "=r"(t0), "=r"(t1) : "l"(t));
    return tc::pair_of(__uint_as_float(y0 + (t0 << 23)), __uint_as_float(y1 + (t1 << 23)));
}
__device__ __forceinline__ void split(uint64_t v, float& lo, float& hi) { asm("mov.b64 {%0, %1}, %2;" : "=f"(lo), "=f"(hi) : "l"(v)); }
// Rows of D codes, swizzled over their own length as the tensor maps do: where chunk `c` of sixteen bytes of a row lies.
template <int D>
__device__ __forceinline__ uint32_t swizzled(uint32_t row, uint32_t c)
{
    return row * D + ((D == 128 ? c ^ (row & 7) : c ^ (row >> 1 & 3)) << 4);
}
// Descriptor of codes whose rows of 64 or 128 bytes run along the contraction.
template <int D>
__device__ __forceinline__ uint64_t codes_operand(uint32_t addr)
{
    return (uint64_t)((addr & 0x3FFFF) >> 4) | 1ull << 16 | (uint64_t)(8 * D >> 4) << 32 | 1ull << 46 | (D == 128 ? 2ull : 4ull) << 61;
}

// Finds blocks and scales four tiles at a time (a lane for each sixteen tokens) and starts the copies of keys and values.
template <int D>
__device__ __forceinline__ void produce(const AttendArgs& a, Shared<D>& s, const Item& it, const CUtensorMap* k_map, const CUtensorMap* v_map)
{
    const uint32_t lane = threadIdx.x & 31, box = min(1u << a.block_log2, kBoxTokens);
    const uint32_t k_full = smem_u32(s.k_full), k_empty = smem_u32(s.k_empty), c_full = smem_u32(s.c_full), c_empty = smem_u32(s.c_empty);
    Turn<kKeyStages> keys;
    Turn<kCodeStages> codes;
    uint32_t used = 0;
    bool ok = true;
    for (uint32_t i0 = 0; ok && i0 < it.tiles.count; i0 += 4) {
        const uint32_t i = i0 + lane / 8, token = it.tiles.at(i) * kTile + (lane & 7) * 16;
        uint32_t id = 0xFFFFFFFFu;
        float ks = 0.0f, vs = 1.0f;
        if (i < it.tiles.count && token < it.q.len) id = (uint32_t)a.table[(uint64_t)it.r * a.ld_table + (token >> a.block_log2)];
        const bool held = id < a.n_blocks;
        if (held) {
            ks = a.k_scale[(uint64_t)id * a.n_kv + it.head];
            vs = a.v_scale[(uint64_t)id * a.n_kv + it.head];
        }
        const uint32_t all = __ballot_sync(0xFFFFFFFFu, held), apart = __ballot_sync(0xFFFFFFFFu, reciprocal_near(vs) == 0.0f),
                       pieces = __ballot_sync(0xFFFFFFFFu, held && (lane & 7) * 16 % box == 0);
        const int row = (int)((id * a.n_kv + it.head << a.block_log2) + (token & (1u << a.block_log2) - 1));
        for (uint32_t b = 0; b < 4 && i0 + b < it.tiles.count; ++b) {
            const uint32_t mine = pieces >> (8 * b) & 255, bytes = (uint32_t)__popc(mine) * box * D;
            ok = warp_wait(k_empty + 8 * keys.slot, keys.round ^ 1, &s.limit, &g_wait_failures);
            if (!ok) break;
            // the copy first: it needs no scales, which may still be on their way
            const bool copy = !a.starve && lane / 8 == b && (mine >> (lane & 7) & 1);
            if (copy) load_2d<false>(smem_u32(s.k[keys.slot]) + (lane & 7) * 16 * D, k_map, k_full + 8 * keys.slot, 0, row);
            // (the softmax of the tile that the slot was for has read it: its products came before those that freed the key stage)
            Meta& m = s.meta[(i0 + b) % kMetas];
            if (lane / 8 == b) {
                m.k_scale[lane & 7] = ks;
                m.v_log[lane & 7] = log2_scale(vs);
                m.v_inv[lane & 7] = reciprocal_near(vs);
                if ((lane & 7) == 0) {
                    m.held = all >> (8 * b) & 255;
                    m.apart = apart >> (8 * b) & 255;
                    m.token = token;
                }
            }
            __syncwarp();
            // (the stage cannot be full before this arrival, whatever has landed)
            if (!a.starve && lane == 0) bar_expect(k_full + 8 * keys.slot, bytes);
            __syncwarp();
            keys.next();
            used = min(used + 1, kKeyStages);
            ok = warp_wait(c_empty + 8 * codes.slot, codes.round ^ 1, &s.limit, &g_wait_failures);
            if (!ok) break;
            if (!a.starve) {
                if (lane == 0) bar_expect(c_full + 8 * codes.slot, bytes);
                __syncwarp();
                if (copy) load_2d<false>(smem_u32(s.codes[codes.slot]) + (lane & 7) * 16 * D, v_map, c_full + 8 * codes.slot, 0, row);
            }
            __syncwarp();
            codes.next();
        }
    }
    if (ok) drain(keys, used, k_empty, &s.limit, &g_wait_failures);
}

// The products of one half: S of the next step, then this one's part of O.
template <int D>
__device__ __forceinline__ void multiply(const AttendArgs& a, Shared<D>& s, const Item& it, uint32_t half)
{
    const uint32_t k_full = smem_u32(s.k_full), k_empty = smem_u32(s.k_empty), v_full = smem_u32(s.v_full), v_empty = smem_u32(s.v_empty);
    const uint32_t s_full = smem_u32(s.s_full[half]), p_full = smem_u32(s.p_full[half]), o_done = smem_u32(&s.o_done[half]);
    const uint32_t shape_s = shape_of(true, false, false, kHalf, kStep), shape_o = shape_of(true, false, true, kHalf, D);  // (format 0: e4m3, fp16)
    const uint64_t q0 = codes_operand<D>(smem_u32(s.q[half])), k0 = codes_operand<D>(smem_u32(s.k)), v0 = operand(smem_u32(s.v), kTile * 128);
    const uint32_t s_at = s.tmem + half * 2 * kStep, o_at = s.tmem + 4 * kStep + half * D;
    const uint32_t steps = it.tiles.count * (kTile / kStep);
    Turn<kKeyStages> keys;
    Turn<kValueStages> values;
    // S of step i lies over the P of step i - 2, which its product must have read
    auto logits = [&](uint32_t i) {
        if (!(i & 1) && !warp_wait(k_full + 8 * keys.slot, keys.round, &s.limit, &g_wait_failures)) return false;
        if (i > 1 && !warp_wait(o_done, i & 1, &s.limit, &g_wait_failures)) return false;
        fence_after();
        const uint64_t dk = k0 + keys.slot * (kTile * D >> 4) + (i & 1) * (kStep * D >> 4);
        if (elect()) {
#pragma unroll
            for (uint32_t rest = 0; rest < 2; ++rest)
#pragma unroll
                for (uint32_t c = 0; c < D / 32; ++c)
                    mma<1, true>(s_at + (i & 1) * kStep, q0 + rest * (kHalf * D >> 4) + c * 2, dk + c * 2, shape_s, rest | c);
            commit<1>(s_full + 8 * (i & 1));
            if (i & 1) commit<1>(k_empty + 8 * keys.slot);
        }
        __syncwarp();
        if (i & 1) keys.next();
        return true;
    };
    if (!warp_wait(smem_u32(&s.q_full[half]), 0, &s.limit, &g_wait_failures) || !logits(0)) return;
    for (uint32_t i = 0; i < steps; ++i) {
        if (i + 1 < steps && !logits(i + 1)) return;
        if (!(i & 1) && !warp_wait(v_full + 8 * values.slot, values.round, &s.limit, &g_wait_failures)) return;
        if (!warp_wait(p_full + 8 * (i & 1), i >> 1 & 1, &s.limit, &g_wait_failures)) return;
        fence_after();
        const uint64_t dv = v0 + values.slot * (kTile * D * 2 >> 4) + (i & 1) * (kStep * 128 >> 4);
        if (elect()) {
#pragma unroll
            for (uint32_t c = 0; c < kStep / 16; ++c)
                mma_ts(o_at, s_at + (i & 1) * kStep + c * 8, dv + c * (2048 >> 4), shape_o, i | c);
            commit<1>(o_done);
            if (i + 1 == steps) commit<1>(smem_u32(&s.o_last[half]));
            if (i & 1) commit<1>(v_empty + 8 * values.slot);
        }
        __syncwarp();
        if (i & 1) values.next();
    }
}

// The values' codes to fp16, a thread a token: rows of 64 dimensions, swizzled, 128 tokens behind one another; the next 64 dimensions behind
// them.  Tokens that are not held become zeros, whatever the bytes are.
template <int D>
__device__ __forceinline__ void convert(const AttendArgs& a, Shared<D>& s, const Item& it)
{
    const uint32_t t = threadIdx.x & 127, lane = threadIdx.x & 31;
    const uint32_t c_full = smem_u32(s.c_full), c_empty = smem_u32(s.c_empty), v_full = smem_u32(s.v_full), v_empty = smem_u32(s.v_empty);
    Turn<kCodeStages> codes;
    Turn<kValueStages> values;
    uint32_t used = 0;
    for (uint32_t i = 0; i < it.tiles.count; ++i) {
        if (!warp_wait(c_full + 8 * codes.slot, codes.round, &s.limit, &g_wait_failures)) return;
        if (!warp_wait(v_empty + 8 * values.slot, values.round ^ 1, &s.limit, &g_wait_failures)) return;
        const Meta& m = s.meta[i % kMetas];
        const bool live = (m.held >> (t / 16) & 1) && m.token + t < it.q.len;
        const uint8_t* from = s.codes[codes.slot];
        const uint32_t to = smem_u32(s.v[values.slot]) + t * 128;
#pragma unroll
        for (uint32_t c = 0; c < D / 16; ++c) {
            uint4 w = *(const uint4*)(from + swizzled<D>(t, c));
            if (!live) w = make_uint4(0, 0, 0, 0);
            uint32_t h[8];
            e4m3x4_to_half(w.x, h[0], h[1]);
            e4m3x4_to_half(w.y, h[2], h[3]);
            e4m3x4_to_half(w.z, h[4], h[5]);
            e4m3x4_to_half(w.w, h[6], h[7]);
            const uint32_t panel = to + c / 4 * (kTile * 128);
            store_shared(panel + ((c % 4 * 2 ^ (t & 7)) << 4), h[0], h[1], h[2], h[3]);
            store_shared(panel + (((c % 4 * 2 + 1) ^ (t & 7)) << 4), h[4], h[5], h[6], h[7]);
        }
        fence_async();
        __syncwarp();
        if (lane == 0) {
            bar_arrive(c_empty + 8 * codes.slot);
            bar_arrive(v_full + 8 * values.slot);
        }
        codes.next();
        values.next();
        used = min(used + 1, kValueStages);
    }
    drain(values, used, v_empty, &s.limit, &g_wait_failures);
}

// The lowest n of sixteen bits; none for n <= 0.
__device__ __forceinline__ uint32_t low_bits(int n) { return (1u << min(max(n, 0), 16)) - 1; }
// One step's part of a row's sum of p with exponentials of its own: r is the largest logit so far, l the sum relative to 2^r.  (The logits are read
// from tensor memory anew, sixteen at a time, before the step needs its registers: with the 64 that it has loaded a prompt that
// never comes here takes 6 % longer.)
__device__ __forceinline__ void sum_apart(const AttendArgs& a, const Meta& meta, uint32_t at, int odd, float back, int p, float& r, float& l)
{
    float now = r, all = l;
#pragma unroll 1
    for (int g = 0; g < (int)kStepGroups; ++g) {
        float v[16];
        asm volatile("tcgen05.ld.sync.aligned.32x32b.x16.b32 {%0,%1,%2,%3,%4,%5,%6,%7,%8,%9,%10,%11,%12,%13,%14,%15}, [%16];\n"
                     "tcgen05.wait::ld.sync.aligned;"
                     : "=f"(v[0]), "=f"(v[1]), "=f"(v[2]), "=f"(v[3]), "=f"(v[4]), "=f"(v[5]), "=f"(v[6]), "=f"(v[7]), "=f"(v[8]), "=f"(v[9]), "=f"(v[10]), "=f"(v[11]), "=f"(v[12]), "=f"(v[13]), "=f"(v[14]), "=f"(v[15])
                     : "r"(at + 16 * g)
                     : "memory");
        const int of = odd * (int)kStepGroups + g, t0 = (int)meta.token + 16 * of;
        const float f = fmaxf(back * meta.k_scale[of], 1.2e-38f);
        const int far = p - (int)a.window;  // (from 1 - 2^31 on)
        uint32_t seen = meta.held >> of & 1 ? low_bits(p - t0 + 1) : 0;
        if (a.window && far >= t0) seen &= ~low_bits(far - t0 + 1) | low_bits((int)a.sinks - t0);
        float top[2] = {-INFINITY, -INFINITY}, sum[2] = {0.0f, 0.0f};
#pragma unroll
        for (int k = 0; k < 16; ++k) {
            if (!(seen >> k & 1)) v[k] = -INFINITY;
            top[k & 1] = fmaxf(top[k & 1], v[k]);
        }
        const float was = now;
        now = fmaxf(now, fmaxf(top[0], top[1]) * f);
        const float base = kTop - (now == -INFINITY ? 0.0f : now);
#pragma unroll
        for (int k = 0; k < 16; ++k) sum[k & 1] += exp2_of(fmaf(v[k], f, base));
        all = fmaf(all, now == -INFINITY ? 1.0f : exp2_of(was - now), sum[0] + sum[1]);
    }
    l = all;
    r = now;
}

// A half's rows, a thread a row.
template <int D>
__device__ __forceinline__ void softmax(const AttendArgs& a, Shared<D>& s, const Item& it, uint32_t half)
{
    const uint32_t lane = threadIdx.x & 31, i_row = threadIdx.x & 127, x = it.rows0 + half * kHalf + i_row;
    const uint32_t last = it.q.n * a.group - 1, y = min(x, last), j = y / a.group;
    const bool real = x <= last;
    const int p = max((int)it.q.len - (int)it.q.n + (int)j, -1);
    const uint64_t index = it.q.row0 + j;
    const uint32_t head = it.head * a.group + y % a.group;
    // the row as the sum of two rows of codes
    float back;
    {
        const char* q = (const char*)a.q + (index * a.ldq + (uint64_t)head * D) * 2;
        uint32_t w[D / 2], most = 0;
#pragma unroll
        for (int c = 0; c < D / 2; c += 4) {
            if (a.vec_q == 2) {
                asm volatile("ld.global.v4.b32 {%0,%1,%2,%3}, [%4];" : "=r"(w[c]), "=r"(w[c + 1]), "=r"(w[c + 2]), "=r"(w[c + 3]) : "l"(q + 4 * c) : "memory");
            } else {
#pragma unroll
                for (int k = c; k < c + 4; ++k)
                    w[k] = ((const volatile uint16_t*)q)[2 * k] | (uint32_t)((const volatile uint16_t*)q)[2 * k + 1] << 16;
            }
        }
#pragma unroll
        for (int c = 0; c < D / 2; ++c) most = max(most, max(w[c] & 0x7FFFu, w[c] >> 16 & 0x7FFFu));
        // times 2^up the maximum lies in (224, 448]; a row that is not finite becomes NaN codes, below
        const int e = (int)(most >> 7);
        const int up = e == 255 || most == 0 ? 0 : 8 - (e - 127) - ((most & 127) > 96);  // 448 = 1.75 * 2^8
        const float x1 = __uint_as_float((uint32_t)(127 + up / 2) << 23), x2 = __uint_as_float((uint32_t)(127 + up - up / 2) << 23);
        const float sign = a.scale < 0.0f ? -1.0f : 1.0f;
        back = fabsf(a.scale) * __uint_as_float((uint32_t)(127 - up / 2) << 23) * __uint_as_float((uint32_t)(127 - (up - up / 2)) << 23);
#pragma unroll
        for (int c = 0; c < D / 16; ++c) {
            uint32_t hi[4], rest[4];
#pragma unroll
            for (int k = 0; k < 8; k += 2) {
                uint32_t h2[2], r2[2];
#pragma unroll
                for (int u = 0; u < 2; ++u) {
                    const uint32_t v = w[8 * c + k + u];
                    float f0 = __uint_as_float(v << 16) * x1 * x2 * sign, f1 = __uint_as_float(v & 0xFFFF0000u) * x1 * x2 * sign;
                    if (e == 255) f0 = f1 = __uint_as_float(0x7FC00000u);
                    if (!real) f0 = f1 = 0.0f;
                    h2[u] = e4m3x2_of(f0, f1);
                    uint32_t wide;
                    asm("cvt.rn.f16x2.e4m3x2 %0, %1;" : "=r"(wide) : "h"((uint16_t)h2[u]));
                    float g0, g1;
                    asm("{\n.reg .b16 a, b;\nmov.b32 {a, b}, %2;\ncvt.f32.f16 %0, a;\ncvt.f32.f16 %1, b;\n}" : "=f"(g0), "=f"(g1) : "r"(wide));
                    r2[u] = e4m3x2_of(f0 - g0, f1 - g1);
                }
                hi[k / 2] = h2[0] | h2[1] << 16;
                rest[k / 2] = r2[0] | r2[1] << 16;
            }
            const uint32_t o = swizzled<D>(i_row, c);
            store_shared(smem_u32(s.q[half][0]) + o, hi[0], hi[1], hi[2], hi[3]);
            store_shared(smem_u32(s.q[half][1]) + o, rest[0], rest[1], rest[2], rest[3]);
        }
    }
    fence_async();
    __syncwarp();
    if (lane == 0) bar_arrive(smem_u32(&s.q_full[half]));
    const uint32_t quarter = (threadIdx.x >> 5 & 3) * 32 << 16;
    const uint32_t s_at = s.tmem + quarter + half * 2 * kStep, o_at = s.tmem + quarter + 4 * kStep + half * D;
    const uint32_t s_full = smem_u32(s.s_full[half]), p_full = smem_u32(s.p_full[half]), o_done = smem_u32(&s.o_done[half]);
    const int p_lo = __shfl_sync(0xFFFFFFFFu, p, 0), p_hi = __shfl_sync(0xFFFFFFFFu, p, 31);  // rows ascend
    const uint32_t steps = it.tiles.count * (kTile / kStep);
    float m = -INFINITY, l = 0.0f;
    bool apart = false;  // the row's sum is in s.apart_l
    for (uint32_t i = 0; i < steps; ++i) {
        const uint32_t odd = i & 1, at = s_at + odd * kStep;
        if (!__all_sync(0xFFFFFFFFu, bar_wait(s_full + 8 * odd, i >> 1 & 1, &s.limit, &g_wait_failures))) return;
        fence_after();
        const Meta& meta = s.meta[(i >> 1) % kMetas];
        if (apart || (!odd && meta.apart)) {
            float& r_row = s.apart_r[half * kHalf + i_row];
            float& l_row = s.apart_l[half * kHalf + i_row];
            if (!apart) {
                r_row = m;
                l_row = l;
            }
            apart = true;
            sum_apart(a, meta, at, (int)odd, back, p, r_row, l_row);
        }
        float v[2][32];
        tmem_start(at, v[0]);
        tmem_start(at + 32, v[1]);
        const int t0 = (int)(meta.token + odd * kStep), g0 = (int)(odd * kStepGroups);
        const uint32_t held = meta.held >> g0 & ((1u << kStepGroups) - 1);
        const bool all = held == (1u << kStepGroups) - 1 && t0 + (int)kStep - 1 <= p_lo &&
                         (!a.window || t0 > p_hi - (int)a.window || t0 + (int)kStep - 1 < (int)a.sinks);
        tmem_arrived(v[0]);
        tmem_arrived(v[1]);
        if (!all) {
#pragma unroll
            for (int k = 0; k < (int)kStep; ++k) {
                const int t = t0 + k;
                if (!(held >> (k / 16) & 1) || t > p || (a.window && t <= p - (int)a.window && t >= (int)a.sinks)) v[k / 32][k % 32] = -INFINITY;
            }
        }
        float top = -INFINITY, f[kStepGroups];
#pragma unroll
        for (int g = 0; g < (int)kStepGroups; ++g) {
            const float* const u = &v[g / 2][g % 2 * 16];
            float most = u[0], other = u[1];  // (two chains)
#pragma unroll
            for (int k = 2; k < 16; k += 2) {
                most = max_nan(most, u[k]);
                other = max_nan(other, u[k + 1]);
            }
            most = max_nan(most, other);
            f[g] = fmaxf(back * meta.k_scale[g0 + g], 1.2e-38f);  // (never zero: a hidden logit stays hidden)
            top = max_nan(top, fmaf(most, f[g], meta.v_log[g0 + g]));
        }
        if (top != top) l = top;  // a NaN among the logits: the row's sum, and its result, are NaN
        if (__any_sync(0xFFFFFFFFu, i == 0 || top > m + kLag || (m == -INFINITY && top > m))) {
            const float now = fmaxf(m, top), shrink = now == -INFINITY ? 1.0f : exp2_of(m - now);
            m = now;
            l *= shrink;
            if (i) {  // once every product so far has ended
                if (!__all_sync(0xFFFFFFFFu, bar_wait(o_done, (i - 1) & 1, &s.limit, &g_wait_failures))) return;
                fence_after();
#pragma unroll 1
                for (int c = 0; c < D / 16; ++c) tmem_scale(o_at + 16 * c, shrink);
            }
        }
        const float base = kTop - (m == -INFINITY ? 0.0f : m);
#pragma unroll
        for (int c = 0; c < 2; ++c) {
            uint32_t w[16];
#pragma unroll
            for (int g = 2 * c; g < 2 * c + 2; ++g) {
                const float from = meta.v_log[g0 + g] + base;
                const uint64_t f2 = pair_of(f[g], f[g]), from2 = pair_of(from, from);
                uint64_t sum = 0;
#pragma unroll
                for (int k = 0; k < 16; k += 2) {
                    float x0, x1;
                    split(fma_pair(pair_of(v[c][g % 2 * 16 + k], v[c][g % 2 * 16 + k + 1]), f2, from2), x0, x1);
                    uint64_t y;
                    if (k % 16 < 16 - 2 * kByFma) {
                        y = pair_of(exp2_of(x0), exp2_of(x1));
                    } else {
                        y = exp2_pair(x0, x1);
                    }
                    split(y, x0, x1);
                    sum = add_pair(sum, y);
                    w[(g - 2 * c) * 8 + k / 2] = half2_of(x0, x1);
                }
                float lo, hi;
                split(sum, lo, hi);
                l = fmaf(lo + hi, meta.v_inv[g0 + g], l);
            }
            tmem_store(at + 16 * c, w);
        }
        tmem_stored();
        fence_before();
        __syncwarp();
        if (lane == 0) bar_arrive(p_full + 8 * odd);
    }
    // (a barrier of its own: o_done may be one or two phases on, which its parity does not tell apart)
    if (!__all_sync(0xFFFFFFFFu, bar_wait(smem_u32(&s.o_last[half]), 0, &s.limit, &g_wait_failures))) return;
    fence_after();
    float lift = 1.0f;
    if (apart) {  // (in two steps, whose product need not be a float)
        l = s.apart_l[half * kHalf + i_row];
        lift = m == -INFINITY ? 1.0f : exp2_of((m - s.apart_r[half * kHalf + i_row]) * 0.5f);
#pragma unroll 1
        for (int c = 0; c < D / 16; ++c) tmem_scale(o_at + 16 * c, lift);
        tmem_stored();
    }
    const float norm = l == 0.0f || (m == -INFINITY && l == l) ? 0.0f : 1.0f / l * lift;  // (a row that has seen nothing: zeros)
    uint16_t* out = (uint16_t*)a.out + index * a.ldo + (uint64_t)head * D;
#pragma unroll
    for (int c = 0; c < D / 32; ++c) {
        float o[32];
        tmem_start(o_at + 32 * c, o);
        tmem_arrived(o);
        if (real) {
#pragma unroll
            for (int k = 0; k < 32; k += 8) {
                uint32_t w[4];
#pragma unroll
                for (int u = 0; u < 4; ++u) w[u] = pack_bf16(o[k + 2 * u] * norm, o[k + 2 * u + 1] * norm);
                if (a.vec_out == 2) {
                    *(uint4*)(out + 32 * c + k) = make_uint4(w[0], w[1], w[2], w[3]);
                } else {
#pragma unroll
                    for (int u = 0; u < 8; ++u) out[32 * c + k + u] = (uint16_t)(w[u / 2] >> (u & 1 ? 16 : 0));
                }
            }
        }
        __syncwarp();
    }
}

template <int D>
__global__ void __launch_bounds__(kThreads, 1)
    many_kernel(const __grid_constant__ CUtensorMap k_map, const __grid_constant__ CUtensorMap v_map, const __grid_constant__ AttendArgs a)
{
    extern __shared__ __align__(1024) uint8_t raw[];
    Shared<D>& s = *(Shared<D>*)raw;
    if (smem_u32(raw) & 1023) {  // the swizzled tiles need the alignment asked for; nothing has been started yet
        if (threadIdx.x == 0) atomicAdd(&g_wait_failures, 1ull);
        return;
    }
    const uint32_t warp = threadIdx.x >> 5, lane = threadIdx.x & 31;
    after_previous();
    // the request, rows and head of this CTA
    {
        const uint32_t want = blockIdx.x / a.n_kv;
        uint32_t base = 0;
        bool found = false;
        const bool ranked = a.requests <= kRanked;
        if (ranked) {  // by their tokens, so that the last CTAs to start are short ones
            const uint32_t r = threadIdx.x, len = r < a.requests ? request_of(a, r).len : 0;
            if (r < a.requests) s.lengths[r] = len;
            __syncthreads();
            if (r < a.requests) {
                uint32_t rank = 0;
                for (uint32_t i = 0; i < a.requests; ++i) rank += s.lengths[i] > len || (s.lengths[i] == len && i < r);
                s.ranked[rank] = r;
                s.tiles[rank] = tiles_of_rows(a, r);
            }
            __syncthreads();
        }
        for (uint32_t r0 = 0; r0 < a.requests && base <= want; r0 += kThreads) {
            const uint32_t mine = !ranked ? tiles_of_rows(a, r0 + threadIdx.x) : threadIdx.x < a.requests ? s.tiles[threadIdx.x] : 0;
            uint32_t sum = mine;
#pragma unroll
            for (int o = 1; o < 32; o <<= 1) {
                const uint32_t up = __shfl_up_sync(0xFFFFFFFFu, sum, o);
                if (lane >= (uint32_t)o) sum += up;
            }
            __syncthreads();
            if (lane == 31) s.sums[warp] = sum;
            __syncthreads();
            uint32_t before = base, total = 0;
#pragma unroll
            for (uint32_t w = 0; w < kThreads / 32; ++w) {
                if (w < warp) before += s.sums[w];
                total += s.sums[w];
            }
            before += sum - mine;
            if (before <= want && want < before + mine) {
                s.request = ranked ? s.ranked[threadIdx.x] : r0 + threadIdx.x;
                s.item = mine - 1 - (want - before);  // a request's last rows first
            }
            base += total;
            found = base > want;
        }
        if (!found) return;  // (by all threads, before anything was set up)
    }
    if (threadIdx.x == 0) {
        prefetch_map(&k_map);
        prefetch_map(&v_map);
    }
    __syncthreads();
    Item it;
    it.r = s.request;
    it.q = request_of(a, it.r);
    it.head = blockIdx.x % a.n_kv;
    it.rows0 = s.item * kRowsCta;
    it.rows = min(kRowsCta, it.q.n * a.group - it.rows0);
    const int before = (int)it.q.len - (int)it.q.n;
    it.tiles = tiles_of<kTile>(a, before + (int)(it.rows0 / a.group), before + (int)((it.rows0 + it.rows - 1) / a.group));
    if (it.tiles.count == 0) it.tiles = Tiles{0, 0, 1};  // rows that see nothing still have to be written
    const uint32_t halves = it.rows > kHalf ? 2 : 1;
    if (threadIdx.x == 0) {
        for (uint32_t i = 0; i < kKeyStages; ++i) {
            bar_init(smem_u32(&s.k_full[i]), 1);
            bar_init(smem_u32(&s.k_empty[i]), halves);
        }
        for (uint32_t i = 0; i < kCodeStages; ++i) {
            bar_init(smem_u32(&s.c_full[i]), 1);
            bar_init(smem_u32(&s.c_empty[i]), 4);
        }
        for (uint32_t i = 0; i < kValueStages; ++i) {
            bar_init(smem_u32(&s.v_full[i]), 4);
            bar_init(smem_u32(&s.v_empty[i]), halves);
        }
        for (uint32_t h = 0; h < 2; ++h) {
            bar_init(smem_u32(&s.q_full[h]), 4);
            for (uint32_t i = 0; i < 2; ++i) {
                bar_init(smem_u32(&s.s_full[h][i]), 1);
                bar_init(smem_u32(&s.p_full[h][i]), 4);
            }
            bar_init(smem_u32(&s.o_done[h]), 1);
            bar_init(smem_u32(&s.o_last[h]), 1);
        }
        s.limit.stop = 0;
        s.limit.us = a.limit_us;
        bar_init_fence();
    }
    if (warp == 13) tmem_alloc<1>(smem_u32(&s.tmem), 512);
    fence_before();
    __syncthreads();
    fence_after();

    if (warp < 8) {
        asm volatile("setmaxnreg.inc.sync.aligned.u32 192;");
        if (warp < 4 * halves) softmax<D>(a, s, it, warp >> 2);
    } else if (warp < 12) {
        asm volatile("setmaxnreg.dec.sync.aligned.u32 64;");
        convert<D>(a, s, it);
    } else {
        asm volatile("setmaxnreg.dec.sync.aligned.u32 64;");
        if (warp == 12) produce<D>(a, s, it, &k_map, &v_map);
        if (warp >= 14 && warp < 14 + halves) multiply<D>(a, s, it, warp - 14);
    }
    __syncwarp();
    let_copies_end(&s.limit);
    fence_before();
    __syncthreads();
    fence_after();
    if (warp == 13) tmem_free<1>(s.tmem, 512);
}

template <int D>
int prepare_many()
{
    cudaFuncAttributes at;
    DR_CUDA(cudaFuncGetAttributes(&at, many_kernel<D>));
    // the split of the registers draws on what the CTA was launched with
    if (at.numRegs * (int)kThreads < 256 * 192 + 128 * 64 + 128 * 64) {
        set_error("the attention kernel was built with %d registers a thread", at.numRegs);
        return DR_ERR_CUDA;
    }
    DR_CUDA(cudaFuncSetAttribute(many_kernel<D>, cudaFuncAttributeMaxDynamicSharedMemorySize, (int)sizeof(Shared<D>)));
    return DR_OK;
}

template <int D>
int launch_many(const dr_kv_cache* cache, const AttendArgs& a, uint64_t ctas, cudaStream_t stream)
{
    cudaLaunchAttribute attr = overlap_attribute();
    cudaLaunchConfig_t cfg{};
    cfg.gridDim = dim3((unsigned)ctas);
    cfg.blockDim = dim3(kThreads);
    cfg.dynamicSmemBytes = sizeof(Shared<D>);
    cfg.stream = stream;
    cfg.attrs = &attr;
    cfg.numAttrs = 1;
    const cudaError_t e = cudaLaunchKernelEx(&cfg, many_kernel<D>, cache->k_map, cache->v_map, a);
    if (e != cudaSuccess) {
        cudaGetLastError();
        set_error("attention launch: %s", cudaGetErrorString(e));
        return DR_ERR_CUDA;
    }
    return DR_OK;
}

}  // namespace

int prepare_attend_many()
{
    const int rc = prepare_many<64>();
    return rc ? rc : prepare_many<128>();
}

int launch_attend_many(const dr_kv_cache* cache, const AttendArgs& a, cudaStream_t stream)
{
    // no more tiles than this have rows: a full one for every 256 of all rows, and a last one for each request that has any
    const uint64_t by_rows = (uint64_t)a.rows * a.group, most = by_rows / (kFewRows + 1);
    const uint64_t tiles = by_rows / kRowsCta + (a.requests < most ? a.requests : most);
    if (tiles * a.n_kv > 0x7FFFFFFFull) {
        set_error("too many rows for one launch");
        return DR_ERR_UNSUPPORTED;
    }
    if (tiles == 0) return DR_OK;
    return cache->d.head_dim == 64 ? launch_many<64>(cache, a, tiles * a.n_kv, stream) : launch_many<128>(cache, a, tiles * a.n_kv, stream);
}

int attend_many_wait_failures(uint64_t* out)
{
    unsigned long long n = 0;
    DR_CUDA(cudaMemcpyFromSymbol(&n, g_wait_failures, sizeof n));
    *out = n;
    return DR_OK;
}

}  // namespace dr
