// Attention over the 8-bit cache for few rows of a request: one token, or some drafted ones (sm_100a).
//
// out = sum_t p_t v_t with p = softmax(scale q . k_t): every code of the visible tokens is read once from HBM for up to sixteen
// rows (the query heads that share a head of the cache, times the request's rows), so the memory bounds it and all else has to stay out of
// its way.
//
// Work is counted in tiles of 64 tokens of one request, cache head and group of sixteen rows, one behind another, and every CTA takes the
// same share of them, wherever a request ends: two CTAs on each SM, whatever the lengths.  A CTA that ends inside a group
// leaves its part (running maximum, sum, unnormalised output) in the work buffer, and a second launch adds the parts in order.
//
// A CTA's fifth warp looks blocks up and brings tiles in through tensor maps, four stages ahead; the other four take sixteen
// tokens of a tile each: codes leave shared memory through ldmatrix (keys as they lie, values transposed two dimensions at a time),
// become fp16 exactly, and meet the rows in m16n8k16 products with fp32 sums.  A warp keeps its own running maximum, sum and output
// and the four are joined at the end of a group.  The tensor cores of tcgen05 would have nothing to win: 16 of their 128 rows
// would be used, and the bytes are the same.
//
// Roundings: a query row is scaled by a power of two to 2^14 before it becomes fp16 (no bits of bf16 are lost above 2^-28 of the row's
// maximum).  A block's value scale goes into p: the running maximum is that of log2(p) + log2(scale), and p scale enters the second
// product in fp16, eleven bits, at most 2^15, so that it stays normal down to 2^-29 of the largest; the sum of p takes the scale out again.
// Measured: PLACEHOLDER
#include "attend.h"
#include "linear.h"
#include "tc_ptx.cuh"

namespace dr {
namespace {

using namespace tc;

__device__ unsigned long long g_wait_failures;  // read by dr_diag_linear_wait_failures

constexpr uint32_t kStages = 4, kConsumers = 4, kThreads = 32 * (kConsumers + 1), kCtasPerSm = 2;
constexpr uint32_t kRows = 16;  // of a group
constexpr float kTop = 15.0f;   // log2 of the largest p in fp16
constexpr float kLeastScale = 7.8886091e-31f;  // 2^-100

// What the consumers have to know of a stage.
enum : uint32_t { kFirst = 1, kLast = 2, kEnd = 4 };
enum : uint32_t { kWhole = 0, kTail = 1, kHead = 2 };  // what the CTA has of the group: all, its end (begun by another CTA), its beginning
struct Meta {
    uint32_t flags, have;
    uint32_t row0, n, len, head, rows0;  // rows0: first of the group's rows among the request's n * group
    uint32_t token;                      // first of the tile
    float k_scale[4], v_log[4], v_inv[4];  // of each sixteen tokens: the keys' scale, log2 of the values' and its reciprocal
    uint32_t ok[4];                        // whether they are held
};
// A part of a group that other CTAs have parts of, too: output and sum of p relative to 2^m.
template <int D>
struct Part {
    float m[kRows], l[kRows], o[kRows][D];
};
// What the second launch joins: parts of CTAs first .. first + count - 1.
struct Join {
    uint32_t count, row0, n, head, rows0, pad[3];
};

template <int D>
struct Shared {
    alignas(1024) uint8_t k[kStages][kTileTokens * D];
    alignas(1024) uint8_t v[kStages][kTileTokens * D];
    float o[kConsumers][kRows][D + 16];
    float m[kConsumers][kRows], l[kConsumers][kRows];
    Meta meta[kStages];
    uint64_t full[kStages], empty[kStages];
    Limit limit;
    uint64_t sums[kThreads / 32];
    uint64_t total, offset;
    uint32_t request;
};

__device__ __forceinline__ uint32_t groups_of(const AttendArgs& a, uint32_t n) { return (uint32_t)(((uint64_t)n * a.group + kRows - 1) / kRows); }
__device__ __forceinline__ Tiles tiles_of_request(const AttendArgs& a, const Request& q)
{
    Tiles t = tiles_of<kTileTokens>(a, (int)q.len - (int)q.n, (int)q.len - 1);
    if (t.count == 0) t = Tiles{0, 0, 1};  // rows that see nothing still have to be written
    return t;
}
__device__ __forceinline__ uint64_t cost_of(const AttendArgs& a, uint32_t r)
{
    if (r >= a.requests) return 0;
    const Request q = request_of(a, r);
    if (q.n * a.group > kFewRows) return 0;
    return (uint64_t)a.n_kv * groups_of(a, q.n) * tiles_of_request(a, q).count;
}

// Exclusive sum over the CTA's threads and the total.
template <int D>
__device__ __forceinline__ uint64_t scan(Shared<D>& s, uint64_t v, uint64_t& total)
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
    asm volatile("mma.sync.aligned.m16n8k16.row.col.f32.f16.f16.f32 {%0,%1,%2,%3}, {%4,%5,%6,%7}, {%8,%9}, {%0,%1,%2,%3};"
                 : "+f"(c[0]), "+f"(c[1]), "+f"(c[2]), "+f"(c[3])
                 : "r"(a[0]), "r"(a[1]), "r"(a[2]), "r"(a[3]), "r"(b0), "r"(b1));
}
__device__ __forceinline__ float exp2_of(float x)
{
    float y;
    asm("ex2.approx.ftz.f32 %0, %1;" : "=f"(y) : "f"(x));
    return y;
}
__device__ __forceinline__ void sync_consumers() { asm volatile("bar.sync 1, 128;" ::: "memory"); }

// Walks the CTA's tiles: finds blocks and scales eight tiles at a time (a lane for each sixteen tokens) and starts the copies.
template <int D>
__device__ __forceinline__ void produce(const AttendArgs& a, Shared<D>& s, const CUtensorMap* k_map, const CUtensorMap* v_map, uint64_t begin,
                                        uint64_t end)
{
    const uint32_t lane = threadIdx.x & 31, box = min(1u << a.block_log2, kBoxTokens);
    const uint32_t full = smem_u32(s.full), empty = smem_u32(s.empty);
    Turn<kStages> ring;
    uint32_t r = s.request;
    uint64_t at = begin, offset = s.offset;  // of the range in the request
    while (at < end) {
        const Request q = request_of(a, r);
        const uint32_t groups = groups_of(a, q.n);
        const Tiles tiles = tiles_of_request(a, q);
        const uint64_t cost = cost_of(a, r);
        while (at < end && offset < cost) {
            const uint64_t segment = offset / tiles.count;
            const uint32_t tile0 = (uint32_t)(offset - segment * tiles.count);
            const uint32_t head = (uint32_t)(segment / groups), rows0 = (uint32_t)(segment % groups) * kRows;
            const uint32_t count = (uint32_t)min((uint64_t)(tiles.count - tile0), end - at);
            const uint32_t have = tile0 ? kTail : count < tiles.count ? kHead : kWhole;
            for (uint32_t t0 = 0; t0 < count; t0 += 8) {
                const uint32_t i = tile0 + t0 + lane / 4, token = tiles.at(i) * kTileTokens + (lane & 3) * 16;
                uint32_t id = 0xFFFFFFFFu;
                float ks = 0.0f, vs = 1.0f;
                if (t0 + lane / 4 < count && token < q.len) id = (uint32_t)a.table[(uint64_t)r * a.ld_table + (token >> a.block_log2)];
                const bool ok = id < a.n_blocks;
                if (ok) {
                    ks = a.k_scale[(uint64_t)id * a.n_kv + head];
                    vs = fmaxf(a.v_scale[(uint64_t)id * a.n_kv + head], kLeastScale);
                }
                const float v_log = log2f(vs), v_inv = 1.0f / vs;
                const uint32_t pieces = __ballot_sync(0xFFFFFFFFu, ok && (lane & 3) * 16 % box == 0);
                const int row = (int)((id * a.n_kv + head << a.block_log2) + (token & (1u << a.block_log2) - 1));
                for (uint32_t b = 0; b < 8 && t0 + b < count; ++b) {
                    if (!warp_wait(empty + 8 * ring.slot, ring.round ^ 1, &s.limit, &g_wait_failures)) return;
                    Meta& m = s.meta[ring.slot];
                    if (lane / 4 == b) {
                        m.k_scale[lane & 3] = ks;
                        m.v_log[lane & 3] = v_log;
                        m.v_inv[lane & 3] = v_inv;
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
                    const uint32_t mine = pieces >> (4 * b) & 15, bar = full + 8 * ring.slot;
                    if (!a.starve) {
                        if (lane == 0) bar_expect(bar, (uint32_t)__popc(mine) * box * D * 2);
                        __syncwarp();
                        if (lane / 4 == b && (mine >> (lane & 3) & 1)) {
                            const uint32_t to = (lane & 3) * 16 * D;
                            load_2d<false>(smem_u32(s.k[ring.slot]) + to, k_map, bar, 0, row);
                            load_2d<false>(smem_u32(s.v[ring.slot]) + to, v_map, bar, 0, row);
                        }
                    }
                    __syncwarp();
                    ring.next();
                }
            }
            at += count;
            offset += count;
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
    r.p = (int)m.len - (int)m.n + (int)j;
    r.index = m.row0 + j;
    r.head = m.head * a.group + y % a.group;
    return r;
}

// The rows' fragments in fp16, each row scaled by the power of two that brings its maximum to [2^14, 2^15); back: what undoes it, with the
// logits' scale.
template <int D>
__device__ __forceinline__ void load_rows(const AttendArgs& a, const Row (&row)[2], uint32_t (&f)[D / 16][4], float (&back)[2])
{
    const uint32_t tig = threadIdx.x & 3;
#pragma unroll
    for (int h = 0; h < 2; ++h) {
        const char* p = (const char*)a.q + (row[h].index * a.ldq + (uint64_t)row[h].head * D + 4 * tig) * 2;
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
#pragma unroll
            for (int k = 0; k < 2; ++k) most = max(most, max(w[c][k] & 0x7FFFu, w[c][k] >> 16 & 0x7FFFu));
        }
#pragma unroll
        for (int o = 1; o < 4; o <<= 1) most = max(most, __shfl_xor_sync(0xFFFFFFFFu, most, o));
        // exponent of the maximum; rows of zeros and subnormals are left as they are, rows that are not finite become NaN
        const int e = (int)(most >> 7);
        const int up = e > 0 && e < 255 ? 14 - (e - 127) : 0;  // -113 .. 140
        const float x1 = __uint_as_float((uint32_t)(127 + up / 2) << 23), x2 = __uint_as_float((uint32_t)(127 + up - up / 2) << 23);
        back[h] = a.scale * __uint_as_float((uint32_t)(127 - up / 2) << 23) * __uint_as_float((uint32_t)(127 - (up - up / 2)) << 23);
#pragma unroll
        for (int c = 0; c < D / 16; ++c)
#pragma unroll
            for (int k = 0; k < 2; ++k) {
                const float lo = __uint_as_float(w[c][k] << 16) * x1 * x2, hi = __uint_as_float(w[c][k] & 0xFFFF0000u) * x1 * x2;
                f[c][2 * k + h] = !row[h].real ? 0 : e == 255 ? 0x7FFF7FFFu : half2_of(lo, hi);
            }
    }
}

template <int D>
__device__ __forceinline__ void write_group(const AttendArgs& a, Shared<D>& s, const Meta& m, Part<D>* parts)
{
    // thread: one row, every eighth piece of four dimensions
    const uint32_t i = threadIdx.x >> 3, piece = threadIdx.x & 7;
    const Row row = row_of(a, m, i);
    if (!row.real) return;
    float most = -INFINITY;
#pragma unroll
    for (uint32_t w = 0; w < kConsumers; ++w) most = fmaxf(most, s.m[w][i]);
    const float safe = most == -INFINITY ? 0.0f : most;
    float weight[kConsumers], l = 0.0f;
#pragma unroll
    for (uint32_t w = 0; w < kConsumers; ++w) {
        const float e = exp2_of(s.m[w][i] - safe);
        l = fmaf(s.l[w][i], e, l);
        weight[w] = e;
    }
    const float norm = m.have != kWhole ? 1.0f : l == 0.0f ? 0.0f : 1.0f / l;
    Part<D>& part = parts[blockIdx.x * 2 + (m.have == kHead)];
    if (m.have != kWhole && piece == 0) {
        part.m[i] = most;
        part.l[i] = l;
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
        if (m.have != kWhole) {
            *(float4*)&part.o[i][d] = o;
        } else {
            uint16_t* to = (uint16_t*)a.out + row.index * a.ldo + (uint64_t)row.head * D + d;
            const uint32_t lo = pack_bf16(o.x * norm, o.y * norm), hi = pack_bf16(o.z * norm, o.w * norm);
            if (a.vec_out) {
                *(uint2*)to = make_uint2(lo, hi);
            } else {
                to[0] = (uint16_t)lo;
                to[1] = (uint16_t)(lo >> 16);
                to[2] = (uint16_t)hi;
                to[3] = (uint16_t)(hi >> 16);
            }
        }
    }
}

template <int D>
__device__ __forceinline__ void consume(const AttendArgs& a, Shared<D>& s, Part<D>* parts)
{
    constexpr int kChunks = D / 16;
    const uint32_t lane = threadIdx.x & 31, warp = threadIdx.x >> 5, g = lane >> 2, tig = lane & 3;
    const uint32_t full = smem_u32(s.full), empty = smem_u32(s.empty);
    // ldmatrix: lanes 0-7 and 8-15 give the rows of tokens 0-7 and 8-15 of a chunk of sixteen bytes, lanes 16-31 of the next
    const uint32_t my_row = warp * 16 + (lane & 15), my_chunk = lane >> 4;
    uint32_t addr[kChunks / 2];
#pragma unroll
    for (int c = 0; c < kChunks / 2; ++c) addr[c] = swizzled<D>(my_row, 2 * c + my_chunk);
    uint32_t qf[kChunks][4];
    float o[kChunks][2][4], m[2] = {}, l[2] = {}, back[2] = {};
    int p[2] = {};
    Turn<kStages> ring;
    for (;;) {
        if (!__all_sync(0xFFFFFFFFu, bar_wait(full + 8 * ring.slot, ring.round, &s.limit, &g_wait_failures))) return;
        const Meta& meta = s.meta[ring.slot];
        const uint32_t flags = meta.flags;
        if (flags & kEnd) return;
        if (flags & kFirst) {
            const Row row[2] = {row_of(a, meta, g), row_of(a, meta, g + 8)};
            load_rows<D>(a, row, qf, back);
#pragma unroll
            for (int h = 0; h < 2; ++h) {
                p[h] = row[h].p;
                m[h] = -INFINITY;
                l[h] = 0.0f;
            }
#pragma unroll
            for (int c = 0; c < kChunks; ++c)
#pragma unroll
                for (int e = 0; e < 4; ++e) o[c][0][e] = o[c][1][e] = 0.0f;
        }
        const int t0 = (int)(meta.token + warp * 16);
        if (meta.ok[warp] && t0 < (int)meta.len) {
            const uint32_t k_at = smem_u32(s.k[ring.slot]), v_at = smem_u32(s.v[ring.slot]);
            float acc[2][2][4] = {};  // [token half][even or odd chunk]: four chains of products
#pragma unroll
            for (int c = 0; c < kChunks / 2; ++c) {
                uint32_t r[4];
                ldmatrix(k_at + addr[c], r);
#pragma unroll
                for (int i = 0; i < 4; ++i) {
                    uint32_t b0, b1;
                    wide(r[i], b0, b1);
                    mma(acc[i & 1][i >> 1], qf[2 * c + (i >> 1)], b0, b1);
                }
            }
            const float ks = meta.k_scale[warp], v_log = meta.v_log[warp];
            float x[2][4];  // [row g, g + 8][tokens 2 tig, 2 tig + 1, 8 + 2 tig, 9 + 2 tig]
#pragma unroll
            for (int i = 0; i < 2; ++i)
#pragma unroll
                for (int e = 0; e < 4; ++e) x[e >> 1][2 * i + (e & 1)] = fmaf(acc[i][0][e] + acc[i][1][e], back[e >> 1] * ks, v_log);
            // whether every row sees all sixteen tokens: rows ascend in position, and the last one's is at most len - 1
            const int p_lo = (int)meta.len - (int)meta.n + (int)(meta.rows0 / a.group);
            const bool all = t0 + 15 <= p_lo && (!a.window || t0 > (int)meta.len - 1 - (int)a.window || t0 + 15 < (int)a.sinks);
            uint32_t keep[2] = {0xFFFFFFFFu, 0xFFFFFFFFu};  // of the codes of values: those behind the last token may be anything
            if (!all) {
#pragma unroll
                for (int e = 0; e < 4; ++e) {
                    const int t = t0 + 2 * (int)tig + (e & 1) + 8 * (e >> 1);
#pragma unroll
                    for (int h = 0; h < 2; ++h)
                        if (t > p[h] || (a.window && t <= p[h] - (int)a.window && t >= (int)a.sinks)) x[h][e] = -INFINITY;
                    if (t >= (int)meta.len) keep[e >> 1] &= e & 1 ? 0x0000FFFFu : 0xFFFF0000u;
                }
            }
            float most[2];
#pragma unroll
            for (int h = 0; h < 2; ++h) {
                most[h] = fmaxf(fmaxf(x[h][0], x[h][1]), fmaxf(x[h][2], x[h][3]));
                most[h] = fmaxf(most[h], __shfl_xor_sync(0xFFFFFFFFu, most[h], 1));
                most[h] = fmaxf(most[h], __shfl_xor_sync(0xFFFFFFFFu, most[h], 2));
            }
            if (__any_sync(0xFFFFFFFFu, most[0] > m[0] || most[1] > m[1])) {
                float f[2];
#pragma unroll
                for (int h = 0; h < 2; ++h) {
                    const float now = fmaxf(m[h], most[h]);
                    f[h] = now == -INFINITY ? 1.0f : exp2_of(m[h] - now);
                    l[h] *= f[h];
                    m[h] = now;
                }
#pragma unroll
                for (int c = 0; c < kChunks; ++c)
#pragma unroll
                    for (int e = 0; e < 4; ++e) {
                        o[c][0][e] *= f[e >> 1];
                        o[c][1][e] *= f[e >> 1];
                    }
            }
            const float v_inv = meta.v_inv[warp];
            uint32_t pf[4];
#pragma unroll
            for (int h = 0; h < 2; ++h) {
                const float safe = (m[h] == -INFINITY ? 0.0f : m[h]) - kTop;
                float y[4];
#pragma unroll
                for (int e = 0; e < 4; ++e) y[e] = exp2_of(x[h][e] - safe);
                l[h] = fmaf((y[0] + y[1]) + (y[2] + y[3]), v_inv, l[h]);
                pf[h] = half2_of(y[0], y[1]);
                pf[2 + h] = half2_of(y[2], y[3]);
            }
#pragma unroll
            for (int c = 0; c < kChunks / 2; ++c) {
                uint32_t r[4], b[4][2];
                ldmatrix_t(v_at + addr[c], r);
#pragma unroll
                for (int i = 0; i < 4; ++i) wide(__byte_perm(r[i] & keep[i & 1], 0, 0x3120), b[i][0], b[i][1]);
#pragma unroll
                for (int i = 0; i < 2; ++i) {
                    mma(o[2 * c + i][0], pf, b[2 * i][0], b[2 * i + 1][0]);
                    mma(o[2 * c + i][1], pf, b[2 * i][1], b[2 * i + 1][1]);
                }
            }
        }
        if (flags & kLast) {
#pragma unroll
            for (int h = 0; h < 2; ++h) {
                l[h] += __shfl_xor_sync(0xFFFFFFFFu, l[h], 1);
                l[h] += __shfl_xor_sync(0xFFFFFFFFu, l[h], 2);
                if (tig == 0) {
                    s.m[warp][g + 8 * h] = m[h];
                    s.l[warp][g + 8 * h] = l[h];
                }
#pragma unroll
                for (int c = 0; c < kChunks; ++c)
                    *(float4*)&s.o[warp][g + 8 * h][16 * c + 4 * tig] = make_float4(o[c][0][2 * h], o[c][1][2 * h], o[c][0][2 * h + 1], o[c][1][2 * h + 1]);
            }
            sync_consumers();
            write_group<D>(a, s, meta, parts);
            sync_consumers();
        }
        __syncwarp();
        if (lane == 0) bar_arrive(empty + 8 * ring.slot);
        ring.next();
    }
}

template <int D>
__global__ void __launch_bounds__(kThreads, kCtasPerSm)
    few_kernel(const __grid_constant__ CUtensorMap k_map, const __grid_constant__ CUtensorMap v_map, const __grid_constant__ AttendArgs a,
               Part<D>* parts, Join* joins)
{
    extern __shared__ __align__(1024) uint8_t raw[];
    Shared<D>& s = *(Shared<D>*)raw;
    if (smem_u32(raw) & 1023) {  // the swizzled tiles need the alignment asked for; nothing has been started yet
        if (threadIdx.x == 0) atomicAdd(&g_wait_failures, 1ull);
        return;
    }
    const uint32_t warp = threadIdx.x >> 5;
    if (threadIdx.x == 0) {
        prefetch_map(&k_map);
        prefetch_map(&v_map);
        for (uint32_t i = 0; i < kStages; ++i) {
            bar_init(smem_u32(&s.full[i]), 1);
            bar_init(smem_u32(&s.empty[i]), kConsumers);
        }
        s.limit.stop = 0;
        s.limit.us = a.limit_us;
        bar_init_fence();
    }
    after_previous();
    // all tiles of the call, the CTA's share of them, and the request that it begins in
    uint64_t mine = 0, total, unused;
    for (uint32_t r = threadIdx.x; r < a.requests; r += kThreads) mine += cost_of(a, r);
    scan(s, mine, total);
    const uint64_t ctas = min((uint64_t)gridDim.x, total), cta = blockIdx.x;
    const uint64_t begin = cta < ctas ? total * cta / ctas : total, end = cta < ctas ? total * (cta + 1) / ctas : total;
    if (begin < end) {
        uint64_t base = 0;
        for (uint32_t r0 = 0; base <= begin; r0 += kThreads) {
            const uint64_t c = cost_of(a, r0 + threadIdx.x), before = base + scan(s, c, unused);
            if (before <= begin && begin < before + c) {
                s.request = r0 + threadIdx.x;
                s.offset = begin - before;
            }
            base += unused;
        }
    }
    __syncthreads();
    if (threadIdx.x == 0) {
        // a group that an earlier CTA has begun: the CTA behind the one that began it has it joined
        Join j{};
        if (begin < end && s.offset) {
            const Request q = request_of(a, s.request);
            const uint32_t groups = groups_of(a, q.n), tiles = tiles_of_request(a, q).count;
            const uint64_t segment = s.offset / tiles, inside = s.offset - segment * tiles, first = begin - inside, last = first + tiles;
            if (inside && total * (cta - 1) / ctas <= first) {
                j.count = (uint32_t)min((last * ctas + total - 1) / total, ctas) - (uint32_t)cta + 1;
                j.row0 = q.row0;
                j.n = q.n;
                j.head = (uint32_t)(segment / groups);
                j.rows0 = (uint32_t)(segment % groups) * kRows;
            }
        }
        joins[cta] = j;
    }
    if (begin < end) {
        if (warp == kConsumers)
            produce<D>(a, s, &k_map, &v_map, begin, end);
        else
            consume<D>(a, s, parts);
    }
    __syncwarp();
    let_copies_end(&s.limit);
}

// The parts of a group that several CTAs have, added in their order: a warp takes a row.
template <int D>
__global__ void __launch_bounds__(32 * kRows) join_kernel(const __grid_constant__ AttendArgs a, const Part<D>* parts, const Join* joins)
{
    after_previous();
    const uint32_t lane = threadIdx.x & 31, i = threadIdx.x >> 5, cta = blockIdx.x;
    const uint32_t count = *(const volatile uint32_t*)&joins[cta].count;
    if (count == 0) return;
    Meta m;
    m.row0 = *(const volatile uint32_t*)&joins[cta].row0;
    m.n = *(const volatile uint32_t*)&joins[cta].n;
    m.head = *(const volatile uint32_t*)&joins[cta].head;
    m.rows0 = *(const volatile uint32_t*)&joins[cta].rows0;
    m.len = 0;
    const Row row = row_of(a, m, i);
    if (!row.real) return;
    // part 0 is the group's beginning in CTA cta - 1, the others the ends that the CTAs behind it met first
    auto part = [&](uint32_t k) -> const Part<D>& { return parts[(cta - 1 + k) * 2 + (k == 0)]; };
    float most = -INFINITY;
    for (uint32_t k = lane; k < count; k += 32) most = fmaxf(most, *(const volatile float*)&part(k).m[i]);
#pragma unroll
    for (int o = 16; o; o >>= 1) most = fmaxf(most, __shfl_xor_sync(0xFFFFFFFFu, most, o));
    const float safe = most == -INFINITY ? 0.0f : most;
    float l = 0.0f, o[D / 32] = {};
#pragma unroll 4
    for (uint32_t k = 0; k < count; ++k) {
        const Part<D>& q = part(k);
        const float e = exp2_of(*(const volatile float*)&q.m[i] - safe);
        l = fmaf(*(const volatile float*)&q.l[i], e, l);
#pragma unroll
        for (int d = 0; d < D / 32; ++d) o[d] = fmaf(*(const volatile float*)&q.o[i][lane + 32 * d], e, o[d]);
    }
    const float norm = l == 0.0f ? 0.0f : 1.0f / l;
#pragma unroll
    for (int d = 0; d < D / 32; ++d)
        ((uint16_t*)a.out)[row.index * a.ldo + (uint64_t)row.head * D + lane + 32 * d] = (uint16_t)pack_bf16(o[d] * norm, 0.0f);
}

uint32_t ctas_of(const dr_kv_cache* cache) { return kCtasPerSm * (uint32_t)cache->sms; }

template <int D>
int launch_few(const dr_kv_cache* cache, const AttendArgs& a, void* work, cudaStream_t stream)
{
    const uint32_t ctas = ctas_of(cache);
    Part<D>* parts = (Part<D>*)work;
    Join* joins = (Join*)(parts + 2 * (uint64_t)ctas);
    cudaLaunchAttribute attr = overlap_attribute();
    cudaLaunchConfig_t cfg{};
    cfg.gridDim = dim3(ctas);
    cfg.blockDim = dim3(kThreads);
    cfg.dynamicSmemBytes = sizeof(Shared<D>);
    cfg.stream = stream;
    cfg.attrs = &attr;
    cfg.numAttrs = 1;
    cudaError_t e = cudaLaunchKernelEx(&cfg, few_kernel<D>, cache->k_map, cache->v_map, a, parts, joins);
    if (e == cudaSuccess) {
        cfg.blockDim = dim3(32 * kRows);
        cfg.dynamicSmemBytes = 0;
        e = cudaLaunchKernelEx(&cfg, join_kernel<D>, a, (const Part<D>*)parts, (const Join*)joins);
    }
    if (e != cudaSuccess) {
        cudaGetLastError();
        set_error("attention launch: %s", cudaGetErrorString(e));
        return DR_ERR_CUDA;
    }
    return DR_OK;
}

}  // namespace

int prepare_attend_few()
{
    DR_CUDA(cudaFuncSetAttribute(few_kernel<64>, cudaFuncAttributeMaxDynamicSharedMemorySize, (int)sizeof(Shared<64>)));
    DR_CUDA(cudaFuncSetAttribute(few_kernel<128>, cudaFuncAttributeMaxDynamicSharedMemorySize, (int)sizeof(Shared<128>)));
    return DR_OK;
}

uint64_t attend_few_work(const dr_kv_cache* cache)
{
    const uint64_t ctas = ctas_of(cache);
    return ctas * (2 * (cache->d.head_dim == 64 ? sizeof(Part<64>) : sizeof(Part<128>)) + sizeof(Join));
}

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
