// Attention over the 8-bit cache for few rows of a request: one token, or some drafted ones (sm_100a).
//
// out = sum_t p_t v_t with p = softmax(scale q . k_t): every code of the visible tokens is read once from HBM for up to 24
// rows (the query heads that share a head of the cache, times the request's rows), so the memory bounds it and all else has to stay out of
// its way.
//
// Work is counted in tiles of 64 tokens of one request, cache head and group of rows, one behind another, and every CTA takes the
// same share of them, wherever a request ends: three CTAs on each SM for groups of eight rows and two for larger ones, whatever the
// lengths.  A CTA that ends inside a group leaves its part (running maximum, sum, unnormalised output) in the work buffer, and a second launch adds the parts in order.
//
// A CTA's fifth warp looks blocks up and brings tiles in through tensor maps, some stages ahead; the other four take sixteen
// tokens of a tile each: codes leave shared memory through ldmatrix (keys as they lie, values transposed two dimensions at a time),
// become fp16 exactly, and meet the rows in m16n8k16 products with fp32 sums.  The tokens (keys) and dimensions (values) are on the M side
// and the rows on the N side, eight at a time, so that four query heads fill half a product and not a quarter; the logits, tokens by
// rows, become the second product's operand by transposing 8 x 8 blocks between the lanes.  A warp keeps its own running maximum,
// sum and output and the four are joined at the end of a group.  The tensor cores of tcgen05 would have nothing to win: the bytes are the same.
//
// Roundings: a query row is scaled by a power of two to 2^14 before it becomes fp16 (no bits of bf16 are lost above 2^-28 of the row's
// maximum).  A block's value scale goes into p: the running maximum is that of log2(p) + log2(scale), raised only when it grows by more
// than 2^4, and p scale enters the second product in fp16, eleven bits, at most 2^15, so that it stays normal down to 2^-25 of the
// largest; the sum of p takes the scale out again (attend.h says how far that goes).
// Measured, calls in a graph: 64 sequences of 700 to 32768 tokens, 32 query over 8 cache heads of 128 (1.1 GB) 184 us = 6.0 TB/s; one of 131000
// tokens over 4 cache heads 35 us = 3.8 TB/s (start, and 111 parts a group to join); 16 sequences with five rows each, 20 rows a cache head, 65 us =
// 1.8 TB/s: there the products, in eight warps an SM, bound it.  32 sequences that see 1000 tokens each: 13.7 us, start and join.
// 64 sequences of 8192 tokens, half of the blocks without values: 231 us, 172 with values.
#include "attend.h"
#include "linear.h"
#include "tc_ptx.cuh"

namespace dr {
namespace {

using namespace tc;

__device__ unsigned long long g_wait_failures;  // read by dr_diag_linear_wait_failures

constexpr uint32_t kConsumers = 4, kThreads = 32 * (kConsumers + 1);
template <int SETS> constexpr uint32_t kRows = 8 * SETS;
// CTAs on an SM and their stages, the rest of whose shared memory goes to the warps' outputs: three hide the products' latency better than
// two (64 sequences 194 us against 211), for which more rows leave no registers
template <int SETS> constexpr uint32_t kCtasPerSm = SETS == 1 ? 3 : 2;
template <int SETS> constexpr uint32_t kStages = SETS == 1 ? 3 : 6 - SETS;
constexpr float kTop = 11.0f, kLag = 4.0f;     // log2 of p at the running maximum in fp16, and how far a p may be above it

// What the consumers have to know of a stage.
enum : uint32_t { kFirst = 1, kLast = 2, kEnd = 4 };
enum : uint32_t { kWhole = 0, kTail = 1, kHead = 2 };  // what the CTA has of the group: all, its end (begun by another CTA), its beginning
struct Meta {
    uint32_t flags, have;
    uint32_t row0, n, len, head, rows0;  // rows0: first of the group's rows among the request's n * group
    uint32_t token;                      // first of the tile
    float k_scale[4], v_log[4], v_inv[4];  // of each sixteen tokens: the keys' scale, log2 of the values' and reciprocal_near of it
    uint32_t ok[4];                        // whether they are held
};
// A part of a group that other CTAs have parts of, too: output and sum of p relative to 2^m; a sum below zero is one that has had exponentials of
// its own, negated, relative to 2^r.
template <int D, int SETS>
struct Part {
    float m[kRows<SETS>], r[kRows<SETS>], l[kRows<SETS>], o[kRows<SETS>][D];
};
// What the second launch joins: parts of CTAs first .. first + count - 1.
struct Join {
    uint32_t count, row0, n, head, rows0, pad[3];
};

template <int D, int SETS>
struct Shared {
    alignas(1024) uint8_t k[kStages<SETS>][kTileTokens * D];
    alignas(1024) uint8_t v[kStages<SETS>][kTileTokens * D];
    float o[kConsumers][kRows<SETS>][D + 4];
    float m[kConsumers][kRows<SETS>], r[kConsumers][kRows<SETS>], l[kConsumers][kRows<SETS>];  // (as in Part)
    uint2 q[SETS < 3 ? 1 : SETS][D / 16][32];  // the rows' fragments, where registers do not hold them
    float back[kRows<SETS>];
    int p[kRows<SETS>];
    Meta meta[kStages<SETS>];
    uint64_t full[kStages<SETS>], empty[kStages<SETS>], met;
    Limit limit;
    uint64_t sums[kThreads / 32];
    uint64_t offset;
    uint32_t request;
};
template <int SETS> constexpr bool kFits = kCtasPerSm<SETS> * (sizeof(Shared<128, SETS>) + 1024) <= 228 * 1024;
static_assert(kFits<1> && kFits<2> && kFits<3>, "shared memory of an SM");

template <int SETS>
__device__ __forceinline__ uint32_t groups_of(const AttendArgs& a, uint32_t n)
{
    return (uint32_t)(((uint64_t)n * a.group + kRows<SETS> - 1) / kRows<SETS>);
}
__device__ __forceinline__ Tiles tiles_of_request(const AttendArgs& a, const Request& q)
{
    Tiles t = tiles_of<kTileTokens>(a, (int)q.len - (int)q.n, (int)q.len - 1);
    if (t.count == 0) t = Tiles{0, 0, 1};  // rows that see nothing still have to be written
    return t;
}
template <int SETS>
__device__ __forceinline__ uint64_t cost_of(const AttendArgs& a, uint32_t r)
{
    if (r >= a.requests) return 0;
    const Request q = request_of(a, r);
    if (q.n * a.group > kFewRows) return 0;
    return (uint64_t)a.n_kv * groups_of<SETS>(a, q.n) * (a.whole ? 1 : tiles_of_request(a, q).count);
}

// Exclusive sum over the CTA's threads and the total.
template <class S>
__device__ __forceinline__ uint64_t scan(S& s, uint64_t v, uint64_t& total)
{
    const uint32_t lane = threadIdx.x & 31, warp = threadIdx.x >> 5;
    uint64_t sum = v;
#pragma unroll
    for (int o = 1; o < 32; o <<= 1) {
        const uint64_t up = __shfl_up_sync(0xFFFFFFFFu, sum, o);
        if (lane >= (uint32_t)o) sum += up;
    }
    __syncthreads();
    if (lane == 31) s.sums[warp] = sum;
    __syncthreads();
    uint64_t before = 0;
    total = 0;
#pragma unroll
    for (uint32_t w = 0; w < kThreads / 32; ++w) {
        if (w < warp) before += s.sums[w];
        total += s.sums[w];
    }
    return before + sum - v;
}

template <int D>
__device__ __forceinline__ uint32_t swizzled(uint32_t row, uint32_t chunk)
{
    return row * D + ((D == 128 ? chunk ^ (row & 7) : chunk ^ (row >> 1 & 3)) << 4);
}
__device__ __forceinline__ void ldmatrix(uint32_t addr, uint32_t (&r)[4])
{
    asm volatile("ldmatrix.sync.aligned.m8n8.x4.shared.b16 {%0,%1,%2,%3}, [%4];" : "=r"(r[0]), "=r"(r[1]), "=r"(r[2]), "=r"(r[3]) : "r"(addr) : "memory");
}
__device__ __forceinline__ void ldmatrix_t(uint32_t addr, uint32_t (&r)[4])
{
    asm volatile("ldmatrix.sync.aligned.m8n8.x4.trans.shared.b16 {%0,%1,%2,%3}, [%4];" : "=r"(r[0]), "=r"(r[1]), "=r"(r[2]), "=r"(r[3]) : "r"(addr) : "memory");
}
// Four codes -> two pairs of fp16.
__device__ __forceinline__ void wide(uint32_t codes, uint32_t& lo, uint32_t& hi)
{
    asm("{\n.reg .b16 a, b;\nmov.b32 {a, b}, %2;\ncvt.rn.f16x2.e4m3x2 %0, a;\ncvt.rn.f16x2.e4m3x2 %1, b;\n}" : "=r"(lo), "=r"(hi) : "r"(codes));
}
__device__ __forceinline__ uint32_t half2_of(float lo, float hi)
{
    uint32_t d;
    asm("cvt.rn.f16x2.f32 %0, %1, %2;" : "=r"(d) : "f"(hi), "f"(lo));
    return d;
}
__device__ __forceinline__ void mma(float (&c)[4], const uint32_t (&a)[4], uint32_t b0, uint32_t b1)
{
    asm("mma.sync.aligned.m16n8k16.row.col.f32.f16.f16.f32 {%0,%1,%2,%3}, {%4,%5,%6,%7}, {%8,%9}, {%0,%1,%2,%3};"
                 : "+f"(c[0]), "+f"(c[1]), "+f"(c[2]), "+f"(c[3])
                 : "r"(a[0]), "r"(a[1]), "r"(a[2]), "r"(a[3]), "r"(b0), "r"(b1));
}
__device__ __forceinline__ float exp2_of(float x)
{
    float y;
    asm("ex2.approx.ftz.f32 %0, %1;" : "=f"(y) : "f"(x));
    return y;
}
// The square root of what an output relative to 2^m is multiplied with over a sum relative to 2^r: twice it reaches where one float does not.
__device__ __forceinline__ float half_lift(float m, float r) { return exp2_of((m - r) * 0.5f); }
// An 8 x 8 block of 16-bit values, transposed between the lanes.
__device__ __forceinline__ uint32_t transposed(uint32_t v)
{
    uint32_t d;
    asm("movmatrix.sync.aligned.m8n8.trans.b16 %0, %1;" : "=r"(d) : "r"(v));
    return d;
}
// The four consuming warps meet; false where one of them has given up.
template <class S>
__device__ __forceinline__ bool meet(S& s, uint32_t& round)
{
    __syncwarp();
    if ((threadIdx.x & 31) == 0) bar_arrive(smem_u32(&s.met));
    const bool ok = __all_sync(0xFFFFFFFFu, bar_wait(smem_u32(&s.met), round, &s.limit, &g_wait_failures));
    round ^= 1;
    return ok;
}

// Walks the CTA's tiles: finds blocks and scales eight tiles at a time (a lane for each sixteen tokens) and starts the copies.
template <int D, int SETS>
__device__ __forceinline__ void produce(const AttendArgs& a, Shared<D, SETS>& s, const CUtensorMap* k_map, const CUtensorMap* v_map, uint64_t begin,
                                        uint64_t end)
{
    const uint32_t lane = threadIdx.x & 31, box = min(1u << a.block_log2, kBoxTokens);
    const uint32_t full = smem_u32(s.full), empty = smem_u32(s.empty);
    Turn<kStages<SETS>> ring;
    uint32_t r = s.request;
    uint64_t at = begin, offset = s.offset;  // of the range in the request
    while (at < end) {
        const Request q = request_of(a, r);
        const uint32_t groups = groups_of<SETS>(a, q.n);
        const Tiles tiles = tiles_of_request(a, q);
        const uint64_t cost = cost_of<SETS>(a, r);
        while (at < end && offset < cost) {
            const uint32_t per = a.whole ? 1 : tiles.count;
            const uint64_t segment = offset / per;
            const uint32_t tile0 = (uint32_t)(offset - segment * per);
            const uint32_t head = (uint32_t)(segment / groups), rows0 = (uint32_t)(segment % groups) * kRows<SETS>;
            const uint32_t count = a.whole ? tiles.count : (uint32_t)min((uint64_t)(tiles.count - tile0), end - at);
            const uint32_t have = tile0 ? kTail : count < tiles.count ? kHead : kWhole;
            for (uint32_t t0 = 0; t0 < count; t0 += 8) {
                const uint32_t i = tile0 + t0 + lane / 4, token = tiles.at(i) * kTileTokens + (lane & 3) * 16;
                uint32_t id = 0xFFFFFFFFu;
                float ks = 0.0f, vs = 1.0f;
                if (t0 + lane / 4 < count && token < q.len) id = (uint32_t)a.table[(uint64_t)r * a.ld_table + (token >> a.block_log2)];
                const bool ok = id < a.n_blocks;
                if (ok) {
                    ks = a.k_scale[(uint64_t)id * a.n_kv + head];
                    vs = a.v_scale[(uint64_t)id * a.n_kv + head];
                }
                const uint32_t pieces = __ballot_sync(0xFFFFFFFFu, ok && (lane & 3) * 16 % box == 0);
                const int row = (int)((id * a.n_kv + head << a.block_log2) + (token & (1u << a.block_log2) - 1));
                for (uint32_t b = 0; b < 8 && t0 + b < count; ++b) {
                    if (!warp_wait(empty + 8 * ring.slot, ring.round ^ 1, &s.limit, &g_wait_failures)) return;
                    // the copies first: they need no scales, which may still be on their way
                    const uint32_t mine = pieces >> (4 * b) & 15, bar = full + 8 * ring.slot;
                    if (!a.starve && lane / 4 == b && (mine >> (lane & 3) & 1)) {
                        const uint32_t to = (lane & 3) * 16 * D;
                        load_2d<false>(smem_u32(s.k[ring.slot]) + to, k_map, bar, 0, row);
                        load_2d<false>(smem_u32(s.v[ring.slot]) + to, v_map, bar, 0, row);
                    }
                    Meta& m = s.meta[ring.slot];
                    if (lane / 4 == b) {
                        m.k_scale[lane & 3] = ks;
                        m.v_log[lane & 3] = log2_scale(vs);
                        m.v_inv[lane & 3] = reciprocal_near(vs);
                        m.ok[lane & 3] = ok;
                        if ((lane & 3) == 0) {
                            m.flags = (t0 + b == 0 ? kFirst : 0) | (t0 + b + 1 == count ? kLast : 0);
                            m.have = have;
                            m.row0 = q.row0;
                            m.n = q.n;
                            m.len = q.len;
                            m.head = head;
                            m.rows0 = rows0;
                            m.token = token;
                        }
                    }
                    __syncwarp();
                    // (the stage cannot be full before this arrival, whatever has landed)
                    if (!a.starve && lane == 0) bar_expect(bar, (uint32_t)__popc(mine) * box * D * 2);
                    __syncwarp();
                    ring.next();
                }
            }
            at += a.whole ? 1 : count;
            offset += a.whole ? 1 : count;
        }
        ++r;
        offset = 0;
    }
    if (!warp_wait(empty + 8 * ring.slot, ring.round ^ 1, &s.limit, &g_wait_failures)) return;
    if (lane == 0) {
        s.meta[ring.slot].flags = kEnd;
        bar_arrive(full + 8 * ring.slot);
    }
}

// Row i of a group: its position, and where it is in q and out.
struct Row {
    int p;
    bool real;
    uint64_t index;  // of the row
    uint32_t head;
};
__device__ __forceinline__ Row row_of(const AttendArgs& a, const Meta& m, uint32_t i)
{
    Row r;
    const uint32_t x = m.rows0 + i;
    r.real = x < m.n * a.group;
    const uint32_t y = min(x, m.n * a.group - 1), j = y / a.group;
    r.p = max((int)m.len - (int)m.n + (int)j, -1);
    r.index = m.row0 + j;
    r.head = m.head * a.group + y % a.group;
    return r;
}

// A row's fragments in fp16, scaled by the power of two that brings its maximum to [2^14, 2^15); returns what undoes it, with the
// logits' scale.  Lanes 4 g .. 4 g + 3 hold row g of the set.
template <int D>
__device__ __forceinline__ float load_row(const AttendArgs& a, const Row& row, uint32_t (&f)[D / 16][2])
{
    const uint32_t tig = threadIdx.x & 3;
    const char* p = (const char*)a.q + (row.index * a.ldq + (uint64_t)row.head * D + 4 * tig) * 2;
    uint32_t w[D / 16][2], most = 0;
#pragma unroll
    for (int c = 0; c < D / 16; ++c) {
        if (a.vec_q) {
            asm volatile("ld.global.v2.b32 {%0,%1}, [%2];" : "=r"(w[c][0]), "=r"(w[c][1]) : "l"(p + 32 * c) : "memory");
        } else {
#pragma unroll
            for (int k = 0; k < 2; ++k)
                w[c][k] = ((const volatile uint16_t*)p)[16 * c + 2 * k] | (uint32_t)((const volatile uint16_t*)p)[16 * c + 2 * k + 1] << 16;
        }
    }
#pragma unroll
    for (int c = 0; c < D / 16; ++c)
#pragma unroll
        for (int k = 0; k < 2; ++k) most = max(most, max(w[c][k] & 0x7FFFu, w[c][k] >> 16 & 0x7FFFu));
#pragma unroll
    for (int o = 1; o < 4; o <<= 1) most = max(most, __shfl_xor_sync(0xFFFFFFFFu, most, o));
    // exponent of the maximum; rows of zeros and subnormals are left as they are, rows that are not finite become NaN
    const int e = (int)(most >> 7);
    const int up = e > 0 && e < 255 ? 14 - (e - 127) : 0;  // -113 .. 140
    const float x1 = __uint_as_float((uint32_t)(127 + up / 2) << 23), x2 = __uint_as_float((uint32_t)(127 + up - up / 2) << 23);
#pragma unroll
    for (int c = 0; c < D / 16; ++c)
#pragma unroll
        for (int k = 0; k < 2; ++k) {
            const float lo = __uint_as_float(w[c][k] << 16) * x1 * x2, hi = __uint_as_float(w[c][k] & 0xFFFF0000u) * x1 * x2;
            f[c][k] = !row.real ? 0 : e == 255 ? 0x7FFF7FFFu : half2_of(lo, hi);
        }
    return a.scale * __uint_as_float((uint32_t)(127 - up / 2) << 23) * __uint_as_float((uint32_t)(127 - (up - up / 2)) << 23);
}

__device__ __forceinline__ void write4(const AttendArgs& a, const Row& row, uint64_t col, float x, float y, float z, float w)
{
    uint16_t* to = (uint16_t*)a.out + row.index * a.ldo + col;
    const uint32_t lo = pack_bf16(x, y), hi = pack_bf16(z, w);
    if (a.vec_out) {
        *(uint2*)to = make_uint2(lo, hi);
    } else {
        to[0] = (uint16_t)lo;
        to[1] = (uint16_t)(lo >> 16);
        to[2] = (uint16_t)hi;
        to[3] = (uint16_t)(hi >> 16);
    }
}

// Joins the four warps' outputs: eight threads a row, every eighth piece of four dimensions each.
template <int D, int SETS>
__device__ __forceinline__ void write_group(const AttendArgs& a, Shared<D, SETS>& s, const Meta& m, Part<D, SETS>* parts)
{
    const uint32_t piece = threadIdx.x & 7;
    for (uint32_t i = threadIdx.x >> 3; i < kRows<SETS>; i += kConsumers * 4) {
        const Row row = row_of(a, m, i);
        if (!row.real) return;
        float most = -INFINITY;
#pragma unroll
        for (uint32_t w = 0; w < kConsumers; ++w) most = fmaxf(most, s.m[w][i]);
        const float safe = most == -INFINITY ? 0.0f : most;
        float weight[kConsumers], l = 0.0f;
#pragma unroll
        for (uint32_t w = 0; w < kConsumers; ++w) {
            weight[w] = exp2_of(s.m[w][i] - safe);
            l = fmaf(s.l[w][i], weight[w], l);
        }
        Part<D, SETS>& part = parts[blockIdx.x * 2 + (m.have == kHead)];
        float lift = 1.0f, sign = 1.0f;
        if (fminf(fminf(s.l[0][i], s.l[1][i]), fminf(s.l[2][i], s.l[3][i])) < 0.0f) {
            float most_r = -INFINITY, r[kConsumers];
#pragma unroll
            for (uint32_t w = 0; w < kConsumers; ++w) {
                r[w] = s.l[w][i] < 0.0f ? s.r[w][i] : s.m[w][i];
                most_r = fmaxf(most_r, r[w]);
            }
            l = 0.0f;
#pragma unroll
            for (uint32_t w = 0; w < kConsumers; ++w) l = fmaf(fabsf(s.l[w][i]), exp2_of(r[w] - most_r), l);
            if (m.have == kWhole) {
                lift = half_lift(most, most_r);
#pragma unroll
                for (uint32_t w = 0; w < kConsumers; ++w) weight[w] *= lift;
            } else {
                part.r[i] = most_r;
                sign = -1.0f;
            }
        }
        const float norm = l == 0.0f ? 0.0f : lift / l;
        if (m.have != kWhole && piece == 0) {
            part.m[i] = most;
            part.l[i] = sign * l;
        }
#pragma unroll
        for (uint32_t d = piece * 4; d < D; d += 32) {
            float4 o = make_float4(0.0f, 0.0f, 0.0f, 0.0f);
#pragma unroll
            for (uint32_t w = 0; w < kConsumers; ++w) {
                const float4 v = *(const float4*)&s.o[w][i][d];
                o.x = fmaf(v.x, weight[w], o.x);
                o.y = fmaf(v.y, weight[w], o.y);
                o.z = fmaf(v.z, weight[w], o.z);
                o.w = fmaf(v.w, weight[w], o.w);
            }
            if (m.have != kWhole)
                *(float4*)&part.o[i][d] = o;
            else
                write4(a, row, (uint64_t)row.head * D + d, o.x * norm, o.y * norm, o.z * norm, o.w * norm);
        }
    }
}

// A row's sixteen logits (log2 of p, plus v_log) into its sum of p with exponentials of its own, held negated relative to 2^r; the first time behind eight
// sums so far, relative to 2^x[24].
__device__ __noinline__ void sum_apart(const float* x, float v_log, bool apart, float& r, float& l)
{
    float sum = 0.0f, was = 0.0f;
    const float from = apart ? r : x[24];
    float now = from;
#pragma unroll
    for (int k = 0; k < 16; ++k) now = fmaxf(now, x[k] - v_log);
    const float base = kTop - (now == -INFINITY ? 0.0f : now);
#pragma unroll
    for (int k = 0; k < 16; ++k) sum += exp2_of(x[k] - v_log + base);
#pragma unroll
    for (int k = 16; k < 24; ++k) was += x[k];
    l = -fmaf(apart ? -l : was, now == -INFINITY ? 1.0f : exp2_of(from - now), sum);
    r = now;
}

template <int D, int SETS>
__device__ __forceinline__ void consume(const AttendArgs& a, Shared<D, SETS>& s, Part<D, SETS>* parts)
{
    constexpr int kChunks = D / 16;
    const uint32_t lane = threadIdx.x & 31, warp = threadIdx.x >> 5, g = lane >> 2, tig = lane & 3;
    const uint32_t full = smem_u32(s.full), empty = smem_u32(s.empty);
    // ldmatrix: lanes 0-7 and 8-15 give the rows of tokens 0-7 and 8-15 of a chunk of sixteen bytes, lanes 16-31 of the next
    const uint32_t my_row = warp * 16 + (lane & 15), my_chunk = lane >> 4;
    uint32_t addr[kChunks / 2];
#pragma unroll
    for (int c = 0; c < kChunks / 2; ++c) addr[c] = swizzled<D>(my_row, 2 * c + my_chunk);
    // rows 2 tig and 2 tig + 1 of each set: [.][row][.]; o: dimensions 16 c + 2 g + {0, 1} at e = row + 2 dimension
    constexpr bool kHeld = SETS < 3;  // the rows' fragments in registers: with three sets 400 bytes a thread would be spilled
    uint32_t qf[kHeld ? SETS : 1][kChunks][2];
    float o[SETS][kChunks][4], m[SETS][2], l[SETS][2];
    bool apart = false;  // the sums have exponentials of their own: the rows' are in s.l, negated, relative to 2^s.r
    Turn<kStages<SETS>> ring;
    uint32_t met = 0;
    // a group's rows (everybody has read those of the group before: the warps met at its end)
    auto load_rows = [&](const Meta& g_) {
#pragma unroll
        for (int n = 0; n < SETS; ++n) {
            const Row row = row_of(a, g_, 8 * n + g);
            const float undo = load_row<D>(a, row, qf[kHeld ? n : 0]);
            if (warp == 0 && tig == 0) {
                s.back[8 * n + g] = undo;
                s.p[8 * n + g] = row.p;
            }
            if (!kHeld && warp == n) {
#pragma unroll
                for (int c = 0; c < kChunks; ++c) s.q[kHeld ? 0 : n][c][lane] = make_uint2(qf[0][c][0], qf[0][c][1]);
            }
        }
        return meet(s, met);
    };
    // the first group's while its tiles are on their way
    {
        const Request q = request_of(a, s.request);
        const uint32_t groups = groups_of<SETS>(a, q.n);
        const uint64_t segment = s.offset / (a.whole ? 1 : tiles_of_request(a, q).count);
        Meta first;
        first.row0 = q.row0;
        first.n = q.n;
        first.len = q.len;
        first.head = (uint32_t)(segment / groups);
        first.rows0 = (uint32_t)(segment % groups) * kRows<SETS>;
        if (!load_rows(first)) return;
    }
    bool loaded = true;
    for (;;) {
        if (!__all_sync(0xFFFFFFFFu, bar_wait(full + 8 * ring.slot, ring.round, &s.limit, &g_wait_failures))) return;
        const Meta& meta = s.meta[ring.slot];
        const uint32_t flags = meta.flags;
        if (flags & kEnd) return;
        if (flags & kFirst) {
            if (!loaded && !load_rows(meta)) return;
            loaded = false;
            apart = false;
#pragma unroll
            for (int n = 0; n < SETS; ++n) {
#pragma unroll
                for (int h = 0; h < 2; ++h) {
                    m[n][h] = -INFINITY;
                    l[n][h] = 0.0f;
                }
#pragma unroll
                for (int c = 0; c < kChunks; ++c)
#pragma unroll
                    for (int e = 0; e < 4; ++e) o[n][c][e] = 0.0f;
            }
        }
        const int t0 = (int)(meta.token + warp * 16);
        if (meta.ok[warp] && t0 < (int)meta.len) {
            const uint32_t k_at = smem_u32(s.k[ring.slot]), v_at = smem_u32(s.v[ring.slot]);
            float x[SETS][4], odd[SETS][4];  // two chains of products
#pragma unroll
            for (int n = 0; n < SETS; ++n)
#pragma unroll
                for (int e = 0; e < 4; ++e) x[n][e] = odd[n][e] = 0.0f;
            // all of the keys' loads, and where there are registers the values', are on their way before the first product
            uint32_t kr[kChunks / 2][4], vr[kChunks / 2][4];
#pragma unroll
            for (int c = 0; c < kChunks / 2; ++c) ldmatrix(k_at + addr[c], kr[c]);
            if (kHeld) {
#pragma unroll
                for (int c = 0; c < kChunks / 2; ++c) ldmatrix_t(v_at + addr[c], vr[c]);
            }
#pragma unroll
            for (int c = 0; c < kChunks / 2; ++c) {
                uint32_t f[2][4];
#pragma unroll
                for (int i = 0; i < 4; ++i) wide(kr[c][i], f[i >> 1][i & 1], f[i >> 1][2 + (i & 1)]);
#pragma unroll
                for (int n = 0; n < SETS; ++n) {
                    if (kHeld) {
                        mma(x[n], f[0], qf[kHeld ? n : 0][2 * c][0], qf[kHeld ? n : 0][2 * c][1]);
                        mma(odd[n], f[1], qf[kHeld ? n : 0][2 * c + 1][0], qf[kHeld ? n : 0][2 * c + 1][1]);
                    } else {
                        const uint2 q0 = s.q[kHeld ? 0 : n][2 * c][lane], q1 = s.q[kHeld ? 0 : n][2 * c + 1][lane];
                        mma(x[n], f[0], q0.x, q0.y);
                        mma(odd[n], f[1], q1.x, q1.y);
                    }
                }
            }
            if (!kHeld) {
#pragma unroll
                for (int c = 0; c < kChunks / 2; ++c) ldmatrix_t(v_at + addr[c], vr[c]);
            }
            const float ks = meta.k_scale[warp], v_log = meta.v_log[warp];
            const float v_inv = meta.v_inv[warp];
            // (sums that have exponentials of their own are made where a maximum grows: a branch for them here costs 300 tokens 0.3 us a call)
            bool grows = apart || v_inv == 0.0f;
            // whether every row sees all sixteen tokens: rows ascend in position, and the last one's is at most len - 1
            const int p_lo = (int)meta.len - (int)meta.n + (int)(meta.rows0 / a.group);
            const bool all = t0 + 15 <= p_lo && (!a.window || t0 > (int)meta.len - 1 - (int)a.window || t0 + 15 < (int)a.sinks);
            uint32_t keep[2] = {0xFFFFFFFFu, 0xFFFFFFFFu};  // of the codes of values: those behind the last token may be anything
#pragma unroll
            for (int n = 0; n < SETS; ++n)
#pragma unroll
                for (int h = 0; h < 2; ++h) {
                    const float f = s.back[8 * n + 2 * tig + h] * ks;
                    x[n][h] = fmaf(x[n][h] + odd[n][h], f, v_log);
                    x[n][h + 2] = fmaf(x[n][h + 2] + odd[n][h + 2], f, v_log);
                }
            if (!all) {
#pragma unroll
                for (int n = 0; n < SETS; ++n)
#pragma unroll
                    for (int e = 0; e < 4; ++e) {
                        const int t = t0 + (int)g + 8 * (e >> 1), at = s.p[8 * n + 2 * tig + (e & 1)];
                        if (t > at || (a.window && t <= at - (int)a.window && t >= (int)a.sinks)) x[n][e] = -INFINITY;
                    }
#pragma unroll
                for (int e = 0; e < 4; ++e)
                    if (t0 + 2 * (int)tig + (e & 1) + 8 * (e >> 1) >= (int)meta.len) keep[e >> 1] &= e & 1 ? 0x0000FFFFu : 0xFFFF0000u;
            }
#pragma unroll
            for (int n = 0; n < SETS; ++n)
#pragma unroll
                for (int e = 0; e < 4; ++e) grows |= x[n][e] > m[n][e & 1] + kLag;
            if (__any_sync(0xFFFFFFFFu, grows)) {
                if (apart || v_inv == 0.0f) {
                    // the logits, and the sums so far, go through the warp's part of s.o, so that little code stands here
#pragma unroll
                    for (int n = 0; n < SETS; ++n)
#pragma unroll
                        for (int e = 0; e < 4; ++e) {
                            float* const row = s.o[warp][8 * n + 2 * tig + (e & 1)];
                            row[g + (e & 2) * 4] = x[n][e];
                            if (e < 2) {
                                row[16 + g] = l[n][e];
                                row[24] = m[n][e];
                            }
                        }
                    __syncwarp();
                    if (lane < kRows<SETS>) sum_apart(s.o[warp][lane], v_log, apart, s.r[warp][lane], s.l[warp][lane]);
                    apart = true;
                    __syncwarp();
                }
#pragma unroll
                for (int n = 0; n < SETS; ++n) {
                    float f[2];
#pragma unroll
                    for (int h = 0; h < 2; ++h) {
                        float now = fmaxf(m[n][h], fmaxf(x[n][h], x[n][h + 2]));
#pragma unroll
                        for (int b = 4; b < 32; b <<= 1) now = fmaxf(now, __shfl_xor_sync(0xFFFFFFFFu, now, b));
                        f[h] = now == -INFINITY ? 1.0f : exp2_of(m[n][h] - now);
                        l[n][h] *= f[h];
                        m[n][h] = now;
                    }
#pragma unroll
                    for (int c = 0; c < kChunks; ++c)
#pragma unroll
                        for (int e = 0; e < 4; ++e) o[n][c][e] *= f[e & 1];
                }
            }
            uint32_t pf[SETS][2];
#pragma unroll
            for (int n = 0; n < SETS; ++n) {
                float y[4];
#pragma unroll
                for (int e = 0; e < 4; ++e) y[e] = exp2_of(x[n][e] - ((m[n][e & 1] == -INFINITY ? 0.0f : m[n][e & 1]) - kTop));
#pragma unroll
                for (int h = 0; h < 2; ++h) l[n][h] = fmaf(y[h] + y[h + 2], v_inv, l[n][h]);
                pf[n][0] = transposed(half2_of(y[0], y[1]));
                pf[n][1] = transposed(half2_of(y[2], y[3]));
            }
#pragma unroll
            for (int c = 0; c < kChunks / 2; ++c) {
                uint32_t f[2][4];
#pragma unroll
                for (int i = 0; i < 4; ++i) wide(__byte_perm(vr[c][i] & keep[i & 1], 0, 0x3120), f[i >> 1][2 * (i & 1)], f[i >> 1][2 * (i & 1) + 1]);
#pragma unroll
                for (int n = 0; n < SETS; ++n) {
                    mma(o[n][2 * c], f[0], pf[n][0], pf[n][1]);
                    mma(o[n][2 * c + 1], f[1], pf[n][0], pf[n][1]);
                }
            }
        }
        if (flags & kLast) {
#pragma unroll
            for (int n = 0; n < SETS; ++n)
#pragma unroll
                for (int h = 0; h < 2; ++h) {
                    const uint32_t row = 8 * n + 2 * tig + h;
#pragma unroll
                    for (int b = 4; b < 32; b <<= 1) l[n][h] += __shfl_xor_sync(0xFFFFFFFFu, l[n][h], b);
                    if (g == 0) {
                        s.m[warp][row] = m[n][h];
                        if (!apart) s.l[warp][row] = l[n][h];
                    }
#pragma unroll
                    for (int c = 0; c < kChunks; ++c) *(float2*)&s.o[warp][row][16 * c + 2 * g] = make_float2(o[n][c][h], o[n][c][h + 2]);
                }
            if (!meet(s, met)) return;
            write_group<D, SETS>(a, s, meta, parts);
            if (!meet(s, met)) return;
        }
        __syncwarp();
        if (lane == 0) bar_arrive(empty + 8 * ring.slot);
        ring.next();
    }
}

template <int D, int SETS>
__global__ void __launch_bounds__(kThreads, kCtasPerSm<SETS>)
    few_kernel(const __grid_constant__ CUtensorMap k_map, const __grid_constant__ CUtensorMap v_map, const __grid_constant__ AttendArgs a,
               Part<D, SETS>* parts, Join* joins)
{
    extern __shared__ __align__(1024) uint8_t raw[];
    Shared<D, SETS>& s = *(Shared<D, SETS>*)raw;
    if (smem_u32(raw) & 1023) {  // the swizzled tiles need the alignment asked for; nothing has been started yet
        after_previous();
        if (threadIdx.x == 0) {
            atomicAdd(&g_wait_failures, 1ull);
            if (!a.whole) joins[blockIdx.x] = Join{};  // (the second launch reads it)
        }
        return;
    }
    const uint32_t warp = threadIdx.x >> 5;
    if (threadIdx.x == 0) {
        prefetch_map(&k_map);
        prefetch_map(&v_map);
        for (uint32_t i = 0; i < kStages<SETS>; ++i) {
            bar_init(smem_u32(&s.full[i]), 1);
            bar_init(smem_u32(&s.empty[i]), kConsumers);
        }
        bar_init(smem_u32(&s.met), kConsumers);
        s.limit.stop = 0;
        s.limit.us = a.limit_us;
        bar_init_fence();
    }
    after_previous();
    // all tiles of the call, the CTA's share of them, and the request that it begins in
    const uint64_t own = cost_of<SETS>(a, threadIdx.x);
    uint64_t all, total = 0;
    const uint64_t first = scan(s, own, all);
    total = all;
    if (a.requests > kThreads) {
        uint64_t mine = 0, rest;
        for (uint32_t r = kThreads + threadIdx.x; r < a.requests; r += kThreads) mine += cost_of<SETS>(a, r);
        scan(s, mine, rest);
        total += rest;
    }
    const uint64_t ctas = min((uint64_t)gridDim.x, total), cta = blockIdx.x;
    const uint64_t begin = cta < ctas ? total * cta / ctas : total, end = cta < ctas ? total * (cta + 1) / ctas : total;
    if (begin < end) {
        uint64_t c = own, before = first, base = all;  // base: of all up to and with the chunk at hand
        for (uint32_t r0 = 0;;) {
            if (before <= begin && begin < before + c) {
                s.request = r0 + threadIdx.x;
                s.offset = begin - before;
            }
            if (base > begin) break;
            r0 += kThreads;
            c = cost_of<SETS>(a, r0 + threadIdx.x);
            before = base + scan(s, c, all);
            base += all;
        }
    }
    __syncthreads();
    if (threadIdx.x == 0) {
        // a group that an earlier CTA has begun: the CTA behind the one that began it has it joined
        Join j{};
        if (begin < end && s.offset && !a.whole) {
            const Request q = request_of(a, s.request);
            const uint32_t groups = groups_of<SETS>(a, q.n), tiles = tiles_of_request(a, q).count;
            const uint64_t segment = s.offset / tiles, inside = s.offset - segment * tiles, first = begin - inside, last = first + tiles;
            if (inside && total * (cta - 1) / ctas <= first) {
                j.count = (uint32_t)min((last * ctas + total - 1) / total, ctas) - (uint32_t)cta + 1;
                j.row0 = q.row0;
                j.n = q.n;
                j.head = (uint32_t)(segment / groups);
                j.rows0 = (uint32_t)(segment % groups) * kRows<SETS>;
            }
        }
        if (!a.whole) joins[cta] = j;
    }
    if (begin < end) {
        if (warp == kConsumers)
            produce<D, SETS>(a, s, &k_map, &v_map, begin, end);
        else
            consume<D, SETS>(a, s, parts);
    }
    __syncwarp();
    let_copies_end(&s.limit);
}

// The parts of a group that several CTAs have, added in an order of their own: eight rows a CTA and a warp for each where a group has few
// parts, two rows and eight warps for each where it has many (111 parts one after another took 30 us); eight parts' loads are on their
// way together.
template <int WARPS> constexpr uint32_t kJoinRows = WARPS == 1 ? 8 : 2;
template <int D, int SETS, int WARPS>
__global__ void __launch_bounds__(32 * kJoinRows<WARPS> * WARPS, 1024 / (32 * kJoinRows<WARPS> * WARPS)) join_kernel(const __grid_constant__ AttendArgs a, const Part<D, SETS>* parts, const Join* joins)
{
    constexpr int kOwn = D / 32;  // dimensions a lane has, side by side
    __shared__ float s_m[kJoinRows<WARPS>][WARPS], s_l[kJoinRows<WARPS>][WARPS], s_o[kJoinRows<WARPS>][WARPS][D];
    after_previous();
    const uint32_t lane = threadIdx.x & 31, warp = threadIdx.x >> 5, r = warp / WARPS, w = warp % WARPS, cta = blockIdx.x;
    const uint32_t i = blockIdx.y * kJoinRows<WARPS> + r;
    const uint32_t count = *(const volatile uint32_t*)&joins[cta].count;
    if (count == 0) return;
    Meta m;
    m.row0 = *(const volatile uint32_t*)&joins[cta].row0;
    m.n = *(const volatile uint32_t*)&joins[cta].n;
    m.head = *(const volatile uint32_t*)&joins[cta].head;
    m.rows0 = *(const volatile uint32_t*)&joins[cta].rows0;
    m.len = 0;
    const Row row = row_of(a, m, i);
    // part 0 is the group's beginning in CTA cta - 1, the others the ends that the CTAs behind it met first
    auto part = [&](uint32_t k) -> const Part<D, SETS>& { return parts[(cta - 1 + k) * 2 + (k == 0)]; };
    float most = -INFINITY, l = 0.0f, least = 0.0f, o[kOwn] = {};  // least: below zero where a part has a sum relative to 2^r
    if (row.real) {
        for (uint32_t k0 = w; k0 < count; k0 += 8 * WARPS) {
            float pm[8], pl[8], po[8][kOwn];
#pragma unroll
            for (int u = 0; u < 8; ++u) {
                const uint32_t k = k0 + u * WARPS;
                pm[u] = -INFINITY;
                pl[u] = 0.0f;
                for (int d = 0; d < kOwn; ++d) po[u][d] = 0.0f;
                if (k >= count) continue;
                const Part<D, SETS>& q = part(k);
                pm[u] = *(const volatile float*)&q.m[i];
                pl[u] = *(const volatile float*)&q.l[i];
                const char* at = (const char*)&q.o[i][lane * kOwn];
                if (D == 128)
                    asm volatile("ld.global.v4.f32 {%0,%1,%2,%3}, [%4];" : "=f"(po[u][0]), "=f"(po[u][1]), "=f"(po[u][D == 128 ? 2 : 0]), "=f"(po[u][D == 128 ? 3 : 0]) : "l"(at) : "memory");
                else
                    asm volatile("ld.global.v2.f32 {%0,%1}, [%2];" : "=f"(po[u][0]), "=f"(po[u][1]) : "l"(at) : "memory");
            }
            float now = most;
#pragma unroll
            for (int u = 0; u < 8; ++u) {
                now = fmaxf(now, pm[u]);
                least = fminf(least, pl[u]);
            }
            const float safe = now == -INFINITY ? 0.0f : now, old = exp2_of(most - safe);
            l *= old;
#pragma unroll
            for (int d = 0; d < kOwn; ++d) o[d] *= old;
#pragma unroll
            for (int u = 0; u < 8; ++u) {
                const float e = exp2_of(pm[u] - safe);
                l = fmaf(pl[u], e, l);
#pragma unroll
                for (int d = 0; d < kOwn; ++d) o[d] = fmaf(po[u][d], e, o[d]);
            }
            most = now;
        }
        if (lane == 0) {
            s_m[r][w] = most;
            s_l[r][w] = least < 0.0f ? least : l;
        }
#pragma unroll
        for (int d = 0; d < kOwn; ++d) s_o[r][w][lane * kOwn + d] = o[d];
    }
    __syncthreads();
    if (w || !row.real) return;
    most = -INFINITY;
#pragma unroll
    for (uint32_t k = 0; k < WARPS; ++k) most = fmaxf(most, s_m[r][k]);
    const float safe = most == -INFINITY ? 0.0f : most;
    l = 0.0f;
#pragma unroll
    for (int d = 0; d < kOwn; ++d) o[d] = 0.0f;
#pragma unroll
    for (uint32_t k = 0; k < WARPS; ++k) {
        const float e = exp2_of(s_m[r][k] - safe);
        l = fmaf(s_l[r][k], e, l);
        least = fminf(least, s_l[r][k]);
#pragma unroll
        for (int d = 0; d < kOwn; ++d) o[d] = fmaf(s_o[r][k][lane * kOwn + d], e, o[d]);
    }
    float norm = l == 0.0f ? 0.0f : 1.0f / l;
    if (least < 0.0f) {  // the sum anew, a lane a part (l is of no account)
        float most_r = -INFINITY;
        l = 0.0f;
        for (uint32_t k0 = 0; k0 < count; k0 += 32) {
            float pr = -INFINITY, pl = 0.0f;
            if (k0 + lane < count) {
                const Part<D, SETS>& q = part(k0 + lane);
                pl = *(const volatile float*)&q.l[i];
                pr = pl < 0.0f ? *(const volatile float*)&q.r[i] : *(const volatile float*)&q.m[i];
            }
            const float now = fmaxf(most_r, pr), safe_r = now == -INFINITY ? 0.0f : now;
            l = fmaf(fabsf(pl), exp2_of(pr - safe_r), l * exp2_of(most_r - safe_r));
            most_r = now;
        }
        float all_r = most_r;
#pragma unroll
        for (int b = 16; b; b >>= 1) all_r = fmaxf(all_r, __shfl_xor_sync(0xFFFFFFFFu, all_r, b));
        l *= exp2_of(most_r - all_r);  // (a part with a sum has a finite r)
#pragma unroll
        for (int b = 16; b; b >>= 1) l += __shfl_xor_sync(0xFFFFFFFFu, l, b);
        const float lift = half_lift(most, all_r);
        norm = lift / l;
#pragma unroll
        for (int d = 0; d < kOwn; ++d) o[d] *= lift;
    }
    uint16_t* out = (uint16_t*)a.out + row.index * a.ldo + (uint64_t)row.head * D + lane * kOwn;
#pragma unroll
    for (int d = 0; d < kOwn; ++d) out[d] = (uint16_t)pack_bf16(o[d] * norm, 0.0f);
}

template <int SETS>
uint64_t ctas_of(const dr_kv_cache* cache) { return kCtasPerSm<SETS> * (uint64_t)cache->sms; }

template <int D, int SETS>
int launch_few(const dr_kv_cache* cache, const AttendArgs& a, void* work, cudaStream_t stream)
{
    const uint32_t ctas = (uint32_t)ctas_of<SETS>(cache);
    Part<D, SETS>* parts = (Part<D, SETS>*)work;
    Join* joins = (Join*)(parts + 2 * (uint64_t)ctas);
    cudaLaunchAttribute attr = overlap_attribute();
    cudaLaunchConfig_t cfg{};
    cfg.gridDim = dim3(ctas);
    cfg.blockDim = dim3(kThreads);
    cfg.dynamicSmemBytes = sizeof(Shared<D, SETS>);
    cfg.stream = stream;
    cfg.attrs = &attr;
    cfg.numAttrs = 1;
    cudaError_t e = cudaLaunchKernelEx(&cfg, few_kernel<D, SETS>, cache->k_map, cache->v_map, a, parts, joins);
    if (e == cudaSuccess && !a.whole) {
        // a dozen parts a group on average divide the two
        const uint64_t rows = ((uint64_t)a.rows * a.group + a.requests - 1) / a.requests, groups = (uint64_t)a.requests * a.n_kv * ((rows + kRows<SETS> - 1) / kRows<SETS>);
        const bool few = groups * 12 >= ctas;
        cfg.gridDim = dim3(ctas, kRows<SETS> / (few ? kJoinRows<1> : kJoinRows<8>));
        cfg.blockDim = dim3(few ? 32 * kJoinRows<1> : 32 * 8 * kJoinRows<8>);
        cfg.dynamicSmemBytes = 0;
        e = cudaLaunchKernelEx(&cfg, few ? join_kernel<D, SETS, 1> : join_kernel<D, SETS, 8>, a, (const Part<D, SETS>*)parts, (const Join*)joins);
    }
    if (e != cudaSuccess) {
        cudaGetLastError();
        set_error("attention launch: %s", cudaGetErrorString(e));
        return DR_ERR_CUDA;
    }
    return DR_OK;
}

template <int D>
int launch_few(const dr_kv_cache* cache, const AttendArgs& a, void* work, cudaStream_t stream)
{
    // sets of eight rows for what a request has on average: more rows than a group holds read the cache again (out of L2), empty sets
    // cost products
    const uint64_t rows = ((uint64_t)a.rows * a.group + a.requests - 1) / a.requests;
    if (rows <= 8) return launch_few<D, 1>(cache, a, work, stream);
    return rows <= 16 ? launch_few<D, 2>(cache, a, work, stream) : launch_few<D, 3>(cache, a, work, stream);
}

template <int D, int SETS>
int prepare_few()
{
    DR_CUDA(cudaFuncSetAttribute(few_kernel<D, SETS>, cudaFuncAttributeMaxDynamicSharedMemorySize, (int)sizeof(Shared<D, SETS>)));
    return DR_OK;
}

}  // namespace

int prepare_attend_few()
{
    int rc = prepare_few<64, 1>();
    if (rc == DR_OK) rc = prepare_few<64, 2>();
    if (rc == DR_OK) rc = prepare_few<64, 3>();
    if (rc == DR_OK) rc = prepare_few<128, 1>();
    if (rc == DR_OK) rc = prepare_few<128, 2>();
    if (rc == DR_OK) rc = prepare_few<128, 3>();
    return rc;
}

template <int D>
uint64_t few_work(const dr_kv_cache* cache)
{
    const uint64_t one = ctas_of<1>(cache) * (2 * sizeof(Part<D, 1>) + sizeof(Join)), two = ctas_of<2>(cache) * (2 * sizeof(Part<D, 2>) + sizeof(Join)),
                   three = ctas_of<3>(cache) * (2 * sizeof(Part<D, 3>) + sizeof(Join));
    return one > two ? (one > three ? one : three) : two > three ? two : three;
}
uint64_t attend_few_work(const dr_kv_cache* cache) { return cache->d.head_dim == 64 ? few_work<64>(cache) : few_work<128>(cache); }

int launch_attend_few(const dr_kv_cache* cache, const AttendArgs& a, void* work, cudaStream_t stream)
{
    return cache->d.head_dim == 64 ? launch_few<64>(cache, a, work, stream) : launch_few<128>(cache, a, work, stream);
}

int attend_few_wait_failures(uint64_t* out)
{
    unsigned long long n = 0;
    DR_CUDA(cudaMemcpyFromSymbol(&n, g_wait_failures, sizeof n));
    *out = n;
    return DR_OK;
}

}  // namespace dr
