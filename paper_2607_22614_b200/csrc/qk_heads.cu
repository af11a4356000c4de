// Norms of query and key heads with the position rotation, forward, into the 8-bit cache, and back (sm_100a).
//
// A head of 64 or 128 values is spread over 4 or 8 lanes, sixteen values each: eight of its first half and the eight of its second half that
// the rotation pairs them with, so the rotation stays inside a lane, a sum over a head takes two or three shuffles, and every access is
// 16 bytes a lane.  A warp takes eight or four heads of one token at a time; the angles belong to the token, so a warp that goes on to the
// token's next heads keeps their sines.  Every value is read once and written once: HBM bounds it.
//
// Angles: base^(-2 i / d) / 2 pi is held as a fraction of a turn in 64 bits, so that position * fraction, taken modulo 2^64, is the
// angle modulo a turn, exact to 2^-64 * position.  No reduction, no table over positions, and the far end of a long context is as
// exact as its start.  Arithmetic is two values an instruction where that exists.
//
// Into the cache: a CTA owns one run (the new tokens of one block) for one head, keys and values both, so that the block's two
// scales are reductions inside the CTA and nobody else touches the block.  Scales are powers of two: the code of v is e4m3(v 2^-e), one
// rounding from fp32, and a scale that grows shifts the codes the block holds already.
//
// Back: with r = 1 / sqrt(mean x^2 + eps), n = x r, g = the rotation back of dy, h = g w:  dx = r (h - n mean(h n)),
// dw = sum of g n over all rows and heads.  A warp keeps the sums of dw for its lanes' sixteen values over all the tokens it takes, a CTA adds its
// warps' in a fixed order, and a second launch adds the CTAs'.
// Measured, calls in a graph, 32 query and 8 key heads of 128, bf16: 8192 rows forward 33.6 us = 5.0 TB/s, back 55.5 = 4.5, into the cache 48.9
// = 3.8 (a run's CTA makes its angles for each head anew, and its 64 registers hold one token a group of lanes); one row into the cache 3.7.
#include <cmath>
#include <new>

#include "fp8_codes.cuh"
#include "kv_cache.h"

struct dr_qk {
    dr_qk_desc d{};
    int device = -1;
    int sms = 0;
    uint64_t turns[64] = {};  // base^(-2 i / d) / 2 pi, in units of 2^-64 of a turn
};

namespace dr {
namespace {

constexpr int kWarps = 8, kThreads = 32 * kWarps;  // of a CTA from x to y, and back
constexpr int kAppendThreads = 512;                // of a CTA into the cache: a run of 64 tokens of a head of 128

struct HeadsArgs {
    const void* x;
    void* y;
    const void* dy;
    const int32_t* positions;
    const void* q_norm;
    const void* k_norm;
    float* work;
    uint64_t ldx, ldy, lddy;
    uint32_t rows, n_q, n_kv;
    uint32_t heads;      // heads that are normed and rotated from x to y
    uint32_t parts;      // warps a token's heads are dealt to
    uint32_t norm_f32, vec, vec_y;
    float eps;
    // into the cache
    uint32_t cache_ctas;
    const int4* runs;
    uint8_t* k;
    uint8_t* v;
    float* k_scale;
    float* v_scale;
    uint32_t n_blocks, block_tokens;
    uint64_t turns[64];
};

template <bool F32> constexpr uint64_t kSize = F32 ? 4 : 2;

// Sixteen values of a head as they lie in memory: eight from p on, eight from half a head further.  Coherent loads that stay behind
// after_previous(), and in their order: a load written before the work on the values before it is on its way meanwhile.
template <bool F32>
struct Raw {
    uint32_t w[F32 ? 16 : 8];
    __device__ __forceinline__ uint64_t pair(int half, int k) const
    {
        if (F32) return two_of(__uint_as_float(w[F32 ? 8 * half + 2 * k : 0]), __uint_as_float(w[F32 ? 8 * half + 2 * k + 1 : 0]));
        const uint32_t v = w[4 * half + k];
        return two_of(__uint_as_float(v << 16), __uint_as_float(v & 0xFFFF0000u));
    }
    __device__ __forceinline__ void get(uint64_t (&lo)[4], uint64_t (&hi)[4]) const
    {
#pragma unroll
        for (int k = 0; k < 4; ++k) {
            lo[k] = pair(0, k);
            hi[k] = pair(1, k);
        }
    }
};
template <int D, bool F32>
__device__ __forceinline__ void load16(const char* p, bool vec, Raw<F32>& r)
{
    constexpr int n = F32 ? 8 : 4;
#pragma unroll
    for (int h = 0; h < 2; ++h) {
        const char* at = p + h * (D / 2) * kSize<F32>;
        if (vec) {
#pragma unroll
            for (int k = h * n; k < h * n + n; k += 4, at += 16)
                asm volatile("ld.global.v4.b32 {%0,%1,%2,%3}, [%4];" : "=r"(r.w[k]), "=r"(r.w[k + 1]), "=r"(r.w[k + 2]), "=r"(r.w[k + 3]) : "l"(at) : "memory");
        } else {
#pragma unroll
            for (int k = 0; k < n; ++k)
                r.w[h * n + k] = F32 ? ((const volatile uint32_t*)at)[k]
                                     : ((const volatile uint16_t*)at)[2 * k] | (uint32_t)((const volatile uint16_t*)at)[2 * k + 1] << 16;
        }
    }
}
__device__ __forceinline__ uint32_t bf16x2(float lo, float hi)
{
    uint32_t d;
    asm("cvt.rn.bf16x2.f32 %0, %1, %2;" : "=r"(d) : "f"(hi), "f"(lo));
    return d;
}
template <bool F32>
__device__ __forceinline__ void store8(char* p, bool vec, const uint64_t (&two)[4])
{
    float v[8];
#pragma unroll
    for (int k = 0; k < 4; ++k) asm("mov.b64 {%0, %1}, %2;" : "=f"(v[2 * k]), "=f"(v[2 * k + 1]) : "l"(two[k]));
    if (F32) {
        if (vec) {
            ((float4*)p)[0] = make_float4(v[0], v[1], v[2], v[3]);
            ((float4*)p)[1] = make_float4(v[4], v[5], v[6], v[7]);
        } else {
#pragma unroll
            for (int k = 0; k < 8; ++k) ((float*)p)[k] = v[k];
        }
    } else {
        uint32_t w[4];
#pragma unroll
        for (int k = 0; k < 4; ++k) w[k] = bf16x2(v[2 * k], v[2 * k + 1]);
        if (vec) {
            *(uint4*)p = make_uint4(w[0], w[1], w[2], w[3]);
        } else {
#pragma unroll
            for (int k = 0; k < 8; ++k) ((uint16_t*)p)[k] = (uint16_t)(w[k / 2] >> (k & 1 ? 16 : 0));
        }
    }
}

__device__ __forceinline__ uint64_t same_two(float v) { return two_of(v, v); }
__device__ __forceinline__ void parts_of(uint64_t v, float& lo, float& hi) { asm("mov.b64 {%0, %1}, %2;" : "=f"(lo), "=f"(hi) : "l"(v)); }
__device__ __forceinline__ uint64_t two_of_bf16(uint32_t w) { return two_of(__uint_as_float(w << 16), __uint_as_float(w & 0xFFFF0000u)); }

// What a CTA keeps of the handle: the turns, and the norms in their own type (their reads take as much of the shared memory's
// time as the rows' do of the L1's: half as much in bf16).
template <int D>
struct HeadsShared {
    uint64_t turns[D / 2];
    alignas(16) uint32_t norm[2][D];
};
template <int D>
__device__ __forceinline__ void fill_turns(HeadsShared<D>& s, const HeadsArgs& a)
{
    if (threadIdx.x < D / 2) s.turns[threadIdx.x] = a.turns[threadIdx.x];
}
template <int D>
__device__ __forceinline__ void fill_norms(HeadsShared<D>& s, const HeadsArgs& a)
{
    if (a.q_norm && threadIdx.x < 2 * D) {
        const void* w = threadIdx.x < D ? a.q_norm : a.k_norm;
        const uint32_t key = threadIdx.x / D, i = threadIdx.x & (D - 1);
        if (a.norm_f32)
            s.norm[key][i] = ((const volatile uint32_t*)w)[i];
        else
            ((uint16_t*)s.norm[key])[i] = ((const volatile uint16_t*)w)[i];
    }
}
template <int D>
__device__ __forceinline__ void load_norm(const HeadsShared<D>& s, const HeadsArgs& a, uint32_t key, uint32_t i0, uint64_t (&w)[8])
{
    if (a.norm_f32) {
#pragma unroll
        for (int k = 0; k < 8; k += 2) {
            const uint4 f = *(const uint4*)&s.norm[key][k / 4 * (D / 2) + i0 + k % 4 * 2];
            w[k] = two_of(__uint_as_float(f.x), __uint_as_float(f.y));
            w[k + 1] = two_of(__uint_as_float(f.z), __uint_as_float(f.w));
        }
    } else {
#pragma unroll
        for (int h = 0; h < 2; ++h) {
            const uint4 f = *(const uint4*)((const uint16_t*)s.norm[key] + h * (D / 2) + i0);
            w[4 * h] = two_of_bf16(f.x);
            w[4 * h + 1] = two_of_bf16(f.y);
            w[4 * h + 2] = two_of_bf16(f.z);
            w[4 * h + 3] = two_of_bf16(f.w);
        }
    }
}

// Cosines and sines of the lane's eight angles at a position, in pairs.  A turn is 2^32: the nearest quarter turn comes off, sine and cosine
// of the rest, within an eighth of a turn, are their Taylor series (the first terms left out are 2e-9 and 3e-8), and the
// quarter turns swap and negate them.
template <int D>
__device__ __forceinline__ void angles(const HeadsShared<D>& s, uint32_t i0, int32_t position, uint64_t (&c)[4], uint64_t (&sn)[4])
{
#pragma unroll
    for (int k = 0; k < 4; ++k) {
        uint32_t quarter[2];
        float z[2];
#pragma unroll
        for (int h = 0; h < 2; ++h) {
            const uint32_t turn = (uint32_t)((uint64_t)position * s.turns[i0 + 2 * k + h] >> 32);
            quarter[h] = turn + 0x20000000u;
            z[h] = (float)(int32_t)(turn - (quarter[h] & 0xC0000000u)) * 1.4629180792671596e-9f;  // 2 pi / 2^32
        }
        const uint64_t x = two_of(z[0], z[1]), x2 = mul_two(x, x);
        uint64_t a = fma_two(x2, same_two(1.0f / 362880), same_two(-1.0f / 5040)), b = fma_two(x2, same_two(1.0f / 40320), same_two(-1.0f / 720));
        a = fma_two(a, x2, same_two(1.0f / 120));
        b = fma_two(b, x2, same_two(1.0f / 24));
        a = fma_two(a, x2, same_two(-1.0f / 6));
        b = fma_two(b, x2, same_two(-0.5f));
        a = fma_two(mul_two(x, x2), a, x);
        b = fma_two(b, x2, same_two(1.0f));
        float sine[2], cosine[2];
        parts_of(a, sine[0], sine[1]);
        parts_of(b, cosine[0], cosine[1]);
#pragma unroll
        for (int h = 0; h < 2; ++h) {
            const bool swap = quarter[h] & 0x40000000u;
            const float u = swap ? cosine[h] : sine[h], v = swap ? sine[h] : cosine[h];
            sine[h] = __uint_as_float(__float_as_uint(u) ^ (quarter[h] & 0x80000000u));
            cosine[h] = __uint_as_float(__float_as_uint(v) ^ ((quarter[h] + 0x40000000u) & 0x80000000u));
        }
        c[k] = two_of(cosine[0], cosine[1]);
        sn[k] = two_of(sine[0], sine[1]);
    }
}
template <int D>
__device__ __forceinline__ float head_sum(float v)
{
#pragma unroll
    for (int o = 1; o < D / 16; o <<= 1) v += __shfl_xor_sync(0xFFFFFFFFu, v, o);
    return v;
}
// x -> normed and rotated, in place: pairs of the lane's eight of the first half, then of the second
template <int D>
__device__ __forceinline__ void norm_rotate(const HeadsShared<D>& s, const HeadsArgs& a, uint32_t key, uint32_t i0, const uint64_t (&c)[4],
                                            const uint64_t (&sn)[4], uint64_t (&lo)[4], uint64_t (&hi)[4])
{
    if (a.q_norm) {
        uint64_t sum = mul_two(lo[0], lo[0]), other = mul_two(hi[0], hi[0]);
#pragma unroll
        for (int k = 1; k < 4; ++k) {
            sum = fma_two(lo[k], lo[k], sum);
            other = fma_two(hi[k], hi[k], other);
        }
        float x, y;
        parts_of(add_two(sum, other), x, y);
        const float r = rsqrtf(head_sum<D>(x + y) * (1.0f / D) + a.eps);
        uint64_t w[8];
        load_norm<D>(s, a, key, i0, w);
        const uint64_t r2 = same_two(r);
#pragma unroll
        for (int k = 0; k < 4; ++k) {
            lo[k] = mul_two(lo[k], mul_two(w[k], r2));
            hi[k] = mul_two(hi[k], mul_two(w[4 + k], r2));
        }
    }
#pragma unroll
    for (int k = 0; k < 4; ++k) {
        const uint64_t l = lo[k], h = hi[k];
        lo[k] = fma_two(l, c[k], mul_two(h, sn[k] ^ 0x8000000080000000ull));
        hi[k] = fma_two(h, c[k], mul_two(l, sn[k]));
    }
}

// Heads [0, a.heads) of the CTA's tokens.  `ready` fills the CTA's shared memory and waits for all of it: the first rows are on their way before.
template <int D, bool F32, class Ready>
__device__ __forceinline__ void rotate_heads(const HeadsArgs& a, const HeadsShared<D>& s, uint32_t cta, Ready ready)
{
    constexpr uint32_t kLanes = D / 16, kHeads = 32 / kLanes;  // of a head; heads of a warp
    const uint32_t lane = threadIdx.x & 31, i0 = (lane % kLanes) * 8, sub = lane / kLanes;
    const uint64_t w = (uint64_t)cta * (blockDim.x / 32) + (threadIdx.x >> 5);
    const uint32_t row = (uint32_t)(w / a.parts), part = (uint32_t)(w % a.parts);
    const uint32_t groups = (a.heads + kHeads - 1) / kHeads, per = (groups + a.parts - 1) / a.parts;
    const uint32_t first = part * per, end = row < a.rows ? min(groups, first + per) : 0;
    const char* x = (const char*)a.x + (uint64_t)row * a.ldx * kSize<F32>;
    char* y = (char*)a.y + (uint64_t)row * a.ldy * kSize<F32>;
    auto at = [&](uint32_t g) { return ((uint64_t)min(g * kHeads + sub, a.heads - 1) * D + i0) * kSize<F32>; };
    Raw<F32> next;  // (loads two groups ahead, with three CTAs an SM for their registers, gain nothing)
    int32_t position = -1;
    if (first < end) {
        position = ((const volatile int32_t*)a.positions)[row];
        load16<D, F32>(x + at(first), a.vec, next);
    }
    ready();
    if (position < 0) return;
    uint64_t c[4], sn[4];
    angles<D>(s, i0, position, c, sn);
    for (uint32_t g = first; g < end; ++g) {
        uint64_t lo[4], hi[4];
        next.get(lo, hi);
        if (g + 1 < end) load16<D, F32>(x + at(g + 1), a.vec, next);
        const uint32_t head = g * kHeads + sub;
        norm_rotate<D>(s, a, head >= a.n_q, i0, c, sn, lo, hi);
        if (head < a.heads) {
            store8<F32>(y + at(g), a.vec_y, lo);
            store8<F32>(y + at(g) + D / 2 * kSize<F32>, a.vec_y, hi);
        }
    }
}

// The exponent e of the smallest scale 2^e >= 2^-100 with m <= 448 * 2^e (448 = 1.75 * 2^8); m is finite.
__device__ __forceinline__ float scale_above(float m)
{
    const uint32_t bits = __float_as_uint(m);
    const int e = (int)(bits >> 23) - 127 - 8 + ((bits & 0x7FFFFFu) > 0x600000u);
    return __uint_as_float((uint32_t)(max(e, -100) + 127) << 23);
}
__device__ __forceinline__ uint64_t finite_or_zero(uint64_t two)
{
    float v[2];
    parts_of(two, v[0], v[1]);
#pragma unroll
    for (int h = 0; h < 2; ++h)
        if ((__float_as_uint(v[h]) & 0x7F800000u) == 0x7F800000u) v[h] = 0.0f;
    return two_of(v[0], v[1]);
}
__device__ __forceinline__ float most_of(uint64_t two)
{
    float lo, hi;
    parts_of(two, lo, hi);
    return fmaxf(fabsf(lo), fabsf(hi));
}
__device__ __forceinline__ uint2 codes_of(const uint64_t (&two)[4], float inv)
{
    float v[8];
    const uint64_t by = two_of(inv, inv);
#pragma unroll
    for (int k = 0; k < 4; ++k) parts_of(mul_two(two[k], by), v[2 * k], v[2 * k + 1]);
    return pack8(v);
}

// Codes of the block's first `bytes` bytes, held at a scale `ratio` times the new one.
__device__ __forceinline__ void shift_codes(uint8_t* codes, uint32_t bytes, float ratio)
{
    for (uint32_t o = threadIdx.x * 8; o < bytes; o += kAppendThreads * 8) {
        uint32_t w[2];
        asm volatile("ld.global.v2.b32 {%0,%1}, [%2];" : "=r"(w[0]), "=r"(w[1]) : "l"(codes + o) : "memory");
        float f[8];
#pragma unroll
        for (int k = 0; k < 4; ++k) {
            const uint16_t two = (uint16_t)(w[k / 2] >> (k & 1 ? 16 : 0));
            uint32_t h;
            asm("cvt.rn.f16x2.e4m3x2 %0, %1;" : "=r"(h) : "h"(two));
            float lo, hi;
            asm("{\n.reg .b16 a, b;\nmov.b32 {a, b}, %2;\ncvt.f32.f16 %0, a;\ncvt.f32.f16 %1, b;\n}" : "=f"(lo), "=f"(hi) : "r"(h));
            f[2 * k] = lo * ratio;
            f[2 * k + 1] = hi * ratio;
        }
        *(uint2*)(codes + o) = pack8(f);
    }
}

// One run of one head: keys normed and rotated, values as they are, both to codes.  TURNS: tokens a group of lanes takes; its one token's values
// stay in registers until the scales are known, of several they are made twice (with two in registers the kernel takes twice as many).
template <int D, bool F32, int TURNS, class Ready>
__device__ __forceinline__ void append_run(const HeadsArgs& a, const HeadsShared<D>& s, uint32_t cta, Ready ready)
{
    constexpr uint32_t kLanes = D / 16, kGroups = kAppendThreads / kLanes;
    __shared__ uint32_t s_most[2];  // bits of the largest magnitudes
    const uint32_t head = cta % a.n_kv;
    int4 run;
    asm volatile("ld.global.v4.b32 {%0,%1,%2,%3}, [%4];" : "=r"(run.x), "=r"(run.y), "=r"(run.z), "=r"(run.w) : "l"(a.runs + cta / a.n_kv) : "memory");
    if (threadIdx.x < 2) s_most[threadIdx.x] = 0;
    const uint32_t block = (uint32_t)run.x, start = (uint32_t)run.y, row0 = (uint32_t)run.z, count = (uint32_t)run.w;
    if (count == 0 || block >= a.n_blocks || start >= a.block_tokens || count > a.block_tokens - start || row0 >= a.rows || count > a.rows - row0)
        return;
    const uint32_t lane = threadIdx.x & 31, i0 = (threadIdx.x % kLanes) * 8, group = threadIdx.x / kLanes;
    const uint64_t tile = (uint64_t)block * a.n_kv + head;
    float k_was = 0.0f, v_was = 0.0f;
    if (start) {
        k_was = *(const volatile float*)(a.k_scale + tile);
        v_was = *(const volatile float*)(a.v_scale + tile);
    }
    // (all lanes take part in the head's sums; those without a token take the run's last one)
    auto row_of = [&](int t) { return row0 + min(group + t * kGroups, count - 1); };
    Raw<F32> rk, rv;
    int32_t position;
    auto load = [&](int t) {
        const uint32_t row = row_of(t);
        const char* x = (const char*)a.x + ((uint64_t)row * a.ldx + (uint64_t)(a.n_q + head) * D + i0) * kSize<F32>;
        position = ((const volatile int32_t*)a.positions)[row];
        load16<D, F32>(x, a.vec, rk);
        load16<D, F32>(x + (uint64_t)a.n_kv * D * kSize<F32>, a.vec, rv);
    };
    uint64_t k_lo[4], k_hi[4], v_lo[4], v_hi[4];
    bool poisoned;
    auto token = [&] {
        uint64_t c[4], sn[4];
        angles<D>(s, i0, position, c, sn);
        rk.get(k_lo, k_hi);
        rv.get(v_lo, v_hi);
        norm_rotate<D>(s, a, 1, i0, c, sn, k_lo, k_hi);
        // zero times a value is zero, unless the value is not finite
        uint64_t odd = 0;
#pragma unroll
        for (int k = 0; k < 4; ++k) {
            odd = fma_two(k_lo[k], 0, odd);
            odd = fma_two(k_hi[k], 0, odd);
            odd = fma_two(v_lo[k], 0, odd);
            odd = fma_two(v_hi[k], 0, odd);
        }
        float p, q;
        parts_of(odd, p, q);
        const uint32_t bad = __ballot_sync(0xFFFFFFFFu, p != 0.0f || q != 0.0f);
        poisoned = bad >> (lane / kLanes * kLanes) & ((1u << kLanes) - 1);
        if (poisoned) {
#pragma unroll
            for (int k = 0; k < 4; ++k) {
                k_lo[k] = finite_or_zero(k_lo[k]);
                k_hi[k] = finite_or_zero(k_hi[k]);
                v_lo[k] = finite_or_zero(v_lo[k]);
                v_hi[k] = finite_or_zero(v_hi[k]);
            }
        }
    };
    load(0);
    ready();
    float k_most = 0.0f, v_most = 0.0f;
#pragma unroll 1
    for (int t = 0; t < TURNS; ++t) {
        if (t) load(t);
        token();
#pragma unroll
        for (int k = 0; k < 4; ++k) {
            k_most = fmaxf(k_most, fmaxf(most_of(k_lo[k]), most_of(k_hi[k])));
            v_most = fmaxf(v_most, fmaxf(most_of(v_lo[k]), most_of(v_hi[k])));
        }
    }
#pragma unroll
    for (int o = 16; o; o >>= 1) {
        k_most = fmaxf(k_most, __shfl_xor_sync(0xFFFFFFFFu, k_most, o));
        v_most = fmaxf(v_most, __shfl_xor_sync(0xFFFFFFFFu, v_most, o));
    }
    if (lane < 2) atomicMax(&s_most[lane], __float_as_uint(lane ? v_most : k_most));
    __syncthreads();
    const float k_scale = fmaxf(scale_above(__uint_as_float(s_most[0])), k_was), v_scale = fmaxf(scale_above(__uint_as_float(s_most[1])), v_was);
    const float k_inv = __frcp_rn(k_scale), v_inv = __frcp_rn(v_scale);
    if (threadIdx.x == 0) {  // (read by all before the barrier)
        a.k_scale[tile] = k_scale;
        a.v_scale[tile] = v_scale;
    }
    uint8_t* const k = a.k + tile * a.block_tokens * D;
    uint8_t* const v = a.v + tile * a.block_tokens * D;
    if (start && k_was != k_scale) shift_codes(k, start * D, k_was * k_inv);
    if (start && v_was != v_scale) shift_codes(v, start * D, v_was * v_inv);
#pragma unroll 1
    for (int t = 0; t < TURNS; ++t) {
        if (TURNS > 1) {
            load(t);
            token();
        }
        const uint32_t j = group + t * kGroups;
        if (j < count) {
            const uint32_t o = (start + j) * D + i0;
            uint2 first = codes_of(k_lo, k_inv);
            if (poisoned && i0 == 0) first.x = (first.x & ~0xFFu) | 0x7Fu;
            *(uint2*)(k + o) = first;
            *(uint2*)(k + o + D / 2) = codes_of(k_hi, k_inv);
            *(uint2*)(v + o) = codes_of(v_lo, v_inv);
            *(uint2*)(v + o + D / 2) = codes_of(v_hi, v_inv);
        }
    }
}

// TURNS 0: x to y alone.  Otherwise the first CTAs take the runs, the others x to y.
template <int D, bool F32, int TURNS>
__global__ void __launch_bounds__(TURNS ? kAppendThreads : kThreads, TURNS ? 2 : 4) heads_kernel(const __grid_constant__ HeadsArgs a)
{
    __shared__ HeadsShared<D> s;
    fill_turns<D>(s, a);
    after_previous();
    auto ready = [&] {
        fill_norms<D>(s, a);
        __syncthreads();
    };
    if (TURNS && blockIdx.x < a.cache_ctas) {  // (the two kinds of CTA in turn: 51 us where this takes 49)
        if constexpr (TURNS > 0) append_run<D, F32, TURNS>(a, s, blockIdx.x, ready);
    } else {
        rotate_heads<D, F32>(a, s, blockIdx.x - a.cache_ctas, ready);
    }
}

// Back through rotation and norm.  Warps stride over tokens, or parts of their heads: groups of query heads, then of key heads.
template <int D, bool F32>
__global__ void __launch_bounds__(kThreads, 2) grad_kernel(const __grid_constant__ HeadsArgs a)
{
    constexpr uint32_t kLanes = D / 16, kHeads = 32 / kLanes;
    __shared__ HeadsShared<D> s;
    __shared__ float s_sum[kWarps][2][D];
    fill_turns<D>(s, a);
    after_previous();
    fill_norms<D>(s, a);
    __syncthreads();
    const uint32_t lane = threadIdx.x & 31, warp = threadIdx.x >> 5, i0 = (lane % kLanes) * 8;
    uint64_t dw[2][8];
#pragma unroll
    for (int k = 0; k < 8; ++k) dw[0][k] = dw[1][k] = 0;
    const uint32_t q_groups = (a.n_q + kHeads - 1) / kHeads, groups = q_groups + (a.n_kv + kHeads - 1) / kHeads;
    for (uint64_t u = (uint64_t)blockIdx.x * kWarps + warp; u < (uint64_t)a.rows * a.parts; u += (uint64_t)gridDim.x * kWarps) {
        const uint64_t row = u / a.parts;
        const uint32_t part = (uint32_t)(u - row * a.parts), begin = groups * part / a.parts, end = groups * (part + 1) / a.parts;
        const int32_t position = ((const volatile int32_t*)a.positions)[row];
        if (position < 0) continue;
        const char* x = (const char*)a.x + row * a.ldx * kSize<F32>;
        const char* dy = (const char*)a.dy + row * a.lddy * kSize<F32>;
        char* dx = (char*)a.y + row * a.ldy * kSize<F32>;
        // groups of query heads, then of key heads: the lane's head of group g, and where its values are
        auto head_of = [&](uint32_t g) { return (g < q_groups ? g : g - q_groups) * kHeads + lane / kLanes; };
        auto at_of = [&](uint32_t g) {
            const uint32_t h = g < q_groups ? min(head_of(g), a.n_q - 1) : a.n_q + min(head_of(g), a.n_kv - 1);
            return ((uint64_t)h * D + i0) * kSize<F32>;
        };
        Raw<F32> next_dy, next_x;
        if (begin < end) {
            load16<D, F32>(dy + at_of(begin), a.vec, next_dy);
            if (a.q_norm) load16<D, F32>(x + at_of(begin), a.vec, next_x);
        }
        uint64_t c[4], sn[4];
        angles<D>(s, i0, position, c, sn);
        for (uint32_t gr = begin; gr < end; ++gr) {
            const bool key = gr >= q_groups, mine = head_of(gr) < (key ? a.n_kv : a.n_q);
            const uint64_t at = at_of(gr);
            uint64_t v[2][4], g[2][4];
            next_dy.get(g[0], g[1]);
            if (a.q_norm) next_x.get(v[0], v[1]);
            if (gr + 1 < end) {
                load16<D, F32>(dy + at_of(gr + 1), a.vec, next_dy);
                if (a.q_norm) load16<D, F32>(x + at_of(gr + 1), a.vec, next_x);
            }
#pragma unroll
            for (int k = 0; k < 4; ++k) {
                const uint64_t l = g[0][k], up = g[1][k];
                g[0][k] = fma_two(l, c[k], mul_two(up, sn[k]));
                g[1][k] = fma_two(up, c[k], mul_two(l, sn[k] ^ 0x8000000080000000ull));
            }
            if (a.q_norm) {
                uint64_t sum2 = 0, dot2 = 0, w[8];
                load_norm<D>(s, a, key, i0, w);
#pragma unroll
                for (int i = 0; i < 8; ++i) {
                    const uint64_t f = v[i / 4][i % 4];
                    sum2 = fma_two(f, f, sum2);
                    w[i] = mul_two(g[i / 4][i % 4], w[i]);
                    dot2 = fma_two(w[i], f, dot2);
                }
                float lo, hi;
                parts_of(sum2, lo, hi);
                const float sum = head_sum<D>(lo + hi);
                parts_of(dot2, lo, hi);
                const float dot = head_sum<D>(lo + hi);
                const float r = rsqrtf(sum * (1.0f / D) + a.eps);
                const uint64_t r2 = same_two(r), back = same_two(-dot * (1.0f / D) * r * r), mine2 = same_two(mine ? r : 0.0f);
                if (key) {
#pragma unroll
                    for (int i = 0; i < 8; ++i) dw[1][i] = fma_two(g[i / 4][i % 4], mul_two(v[i / 4][i % 4], mine2), dw[1][i]);
                } else {
#pragma unroll
                    for (int i = 0; i < 8; ++i) dw[0][i] = fma_two(g[i / 4][i % 4], mul_two(v[i / 4][i % 4], mine2), dw[0][i]);
                }
#pragma unroll
                for (int i = 0; i < 8; ++i) g[i / 4][i % 4] = mul_two(r2, fma_two(v[i / 4][i % 4], back, w[i]));
            }
            if (mine) {
                store8<F32>(dx + at, a.vec_y, g[0]);
                store8<F32>(dx + at + D / 2 * kSize<F32>, a.vec_y, g[1]);
            }
        }
    }
    if (!a.q_norm) return;
#pragma unroll
    for (int i = 0; i < 32; ++i) {
        float v, other;
        parts_of(dw[i / 16][i % 16 / 2], i & 1 ? other : v, i & 1 ? v : other);
#pragma unroll
        for (int o = kLanes; o < 32; o <<= 1) v += __shfl_xor_sync(0xFFFFFFFFu, v, o);
        if (lane < kLanes) s_sum[warp][i / 16][(i % 16 / 8) * (D / 2) + i0 + i % 8] = v;
    }
    __syncthreads();
    if (threadIdx.x < 2 * D) {
        float v = 0.0f;
#pragma unroll
        for (int w = 0; w < kWarps; ++w) v += ((const float*)s_sum[w])[threadIdx.x];
        a.work[(uint64_t)blockIdx.x * 2 * D + threadIdx.x] = v;
    }
}

// The CTAs' sums of dw, added in their order: 32 columns a CTA, 32 threads a column.
__global__ void __launch_bounds__(1024) norm_sum_kernel(const float* work, uint32_t n, uint32_t d, float* dq, float* dk, uint32_t accumulate)
{
    __shared__ float s[32][33];
    const uint32_t lane = threadIdx.x & 31, part = threadIdx.x >> 5, col = blockIdx.x * 32 + lane;
    after_previous();
    float v = 0.0f;
    for (uint32_t i = part; i < n; i += 32) v += *(const volatile float*)(work + (uint64_t)i * 2 * d + col);
    s[part][lane] = v;
    __syncthreads();
    v = s[lane][part];
#pragma unroll
    for (int o = 16; o; o >>= 1) v += __shfl_xor_sync(0xFFFFFFFFu, v, o);
    if (lane == 0) {
        const uint32_t c = blockIdx.x * 32 + part;
        float* to = c < d ? dq + c : dk + (c - d);
        *to = accumulate ? *to + v : v;
    }
}

template <class K, class... A>
int launch(const char* what, K kernel, uint64_t ctas, int threads, cudaStream_t stream, const A&... args)
{
    if (ctas > 0x7FFFFFFFull) {
        set_error("too many rows for one launch");
        return DR_ERR_UNSUPPORTED;
    }
    cudaLaunchAttribute attr = overlap_attribute();
    cudaLaunchConfig_t cfg{};
    cfg.gridDim = dim3((unsigned)ctas);
    cfg.blockDim = dim3(threads);
    cfg.stream = stream;
    cfg.attrs = &attr;
    cfg.numAttrs = 1;
    const cudaError_t e = cudaLaunchKernelEx(&cfg, kernel, args...);
    if (e != cudaSuccess) {
        cudaGetLastError();
        set_error("%s launch: %s", what, cudaGetErrorString(e));
        return DR_ERR_CUDA;
    }
    return DR_OK;
}

template <int D, int TURNS>
int launch_heads(bool f32, const HeadsArgs& a, uint64_t ctas, cudaStream_t s)
{
    constexpr int threads = TURNS ? kAppendThreads : kThreads;
    return f32 ? launch("heads", heads_kernel<D, true, TURNS>, ctas, threads, s, a) : launch("heads", heads_kernel<D, false, TURNS>, ctas, threads, s, a);
}

int check_qk(const dr_qk* qk)
{
    if (!qk) {
        set_error("NULL heads");
        return DR_ERR_INVALID;
    }
    int dev = -1;
    if (cudaGetDevice(&dev) != cudaSuccess || dev != qk->device) {
        set_error("current device differs from the heads' device");
        return DR_ERR_STATE;
    }
    return DR_OK;
}

// x, positions and one more matrix of rows.
int check_rows(uint32_t dtype, uint64_t rows, const void* x, uint64_t ldx, uint64_t x_cols, const int32_t* positions, const void* y,
               uint64_t ldy, uint64_t y_cols)
{
    if (dtype != DR_BF16 && dtype != DR_F32) {
        set_error("rows must be DR_BF16 or DR_F32");
        return DR_ERR_UNSUPPORTED;
    }
    if (rows > 0x7FFFFFFFull) {
        set_error("more than 2^31 - 1 rows");
        return DR_ERR_UNSUPPORTED;
    }
    if (rows && (!x || !y || !positions)) {
        set_error("NULL buffer");
        return DR_ERR_INVALID;
    }
    if (!pitch_ok(rows, x_cols, ldx) || !pitch_ok(rows, y_cols, ldy)) {
        set_error("leading dimension below the row's length or out of range");
        return DR_ERR_INVALID;
    }
    const uint32_t es = dtype == DR_F32 ? 4 : 2;
    if (((uintptr_t)x | (uintptr_t)y) % es || (uintptr_t)positions % 4) {
        set_error("a pointer is not aligned to its element size");
        return DR_ERR_ALIGN;
    }
    return DR_OK;
}

HeadsArgs heads_args(const dr_qk* qk, const void* x, uint32_t dtype, uint64_t ldx, const int32_t* positions, uint64_t rows, void* y, uint64_t ldy)
{
    HeadsArgs a{};
    const uint32_t es = dtype == DR_F32 ? 4 : 2;
    a.x = x;
    a.y = y;
    a.positions = positions;
    a.q_norm = qk->d.q_norm_dev;
    a.k_norm = qk->d.k_norm_dev;
    a.norm_f32 = qk->d.norm_dtype == DR_F32;
    a.ldx = ldx;
    a.ldy = ldy;
    a.rows = (uint32_t)rows;
    a.n_q = qk->d.n_q_heads;
    a.n_kv = qk->d.n_kv_heads;
    a.eps = qk->d.eps;
    a.vec = ((uintptr_t)x | ldx * es) % 16 == 0;
    a.vec_y = ((uintptr_t)y | ldy * es) % 16 == 0;
    for (int i = 0; i < 64; ++i) a.turns[i] = qk->turns[i];
    return a;
}

constexpr uint32_t kWarpsWanted = 40;  // for each SM, of which 32 run at a time (8192 tokens of 40 heads: 34 us; three times as many 35, six times 44)

// How many warps a token's head groups are dealt to: one while the tokens alone fill the machine some times over, so that it works out the
// angles once; with few tokens every group has a warp of its own.
void deal(HeadsArgs& a, int sms, uint32_t dim)
{
    const uint32_t per_warp = 512 / dim, groups = (a.heads + per_warp - 1) / per_warp;
    a.parts = 1;
    while (a.parts < groups && (uint64_t)a.rows * a.parts < (uint64_t)sms * kWarpsWanted) a.parts *= 2;
    if (a.parts > groups) a.parts = groups;
}

constexpr uint32_t kGradCtas = 2;  // for each SM
constexpr uint32_t kGradParts = 2;  // 8192 tokens of 40 heads: 55.7 us; undivided 57.7, in three 59.9

}  // namespace
}  // namespace dr

using namespace dr;

extern "C" {

int dr_qk_create(const dr_qk_desc* desc, dr_qk** out)
{
    if (!out) {
        set_error("NULL out");
        return DR_ERR_INVALID;
    }
    *out = nullptr;
    if (!desc || desc->struct_size != sizeof(dr_qk_desc)) {
        set_error("NULL descriptor or struct_size mismatch");
        return DR_ERR_INVALID;
    }
    const dr_qk_desc& d = *desc;
    if (!d.n_q_heads || !d.n_kv_heads || !d.q_norm_dev != !d.k_norm_dev) {
        set_error("no heads, or one norm without the other");
        return DR_ERR_INVALID;
    }
    if (!std::isfinite(d.eps) || d.eps < 0.0f || !std::isfinite(d.base) || d.base < 1.0) {
        set_error("eps must be finite and not negative, base finite and at least 1");
        return DR_ERR_INVALID;
    }
    if (d.head_dim != 64 && d.head_dim != 128) {
        set_error("heads have 64 or 128 dimensions");
        return DR_ERR_UNSUPPORTED;
    }
    if (d.n_q_heads > 65536 || d.n_kv_heads > 65536 || (d.q_norm_dev && d.norm_dtype != DR_BF16 && d.norm_dtype != DR_F32)) {
        set_error("norms must be DR_BF16 or DR_F32, heads at most 2^16");
        return DR_ERR_UNSUPPORTED;
    }
    if (((uintptr_t)d.q_norm_dev | (uintptr_t)d.k_norm_dev) % (d.norm_dtype == DR_F32 ? 4 : 2)) {
        set_error("a norm is not aligned to its element size");
        return DR_ERR_ALIGN;
    }
    dr_qk* qk = new (std::nothrow) dr_qk();
    if (!qk) return DR_ERR_NOMEM;
    qk->d = d;
    const long double two_pi = 6.283185307179586476925286766559L;
    for (uint32_t i = 0; i < d.head_dim / 2; ++i) {
        const long double f = powl((long double)d.base, -2.0L * i / d.head_dim) / two_pi;  // below 1 / 6
        qk->turns[i] = (uint64_t)roundl(ldexpl(f, 64));
    }
    const int rc = [&]() -> int {
        DR_CUDA(cudaGetDevice(&qk->device));
        DR_CUDA(cudaDeviceGetAttribute(&qk->sms, cudaDevAttrMultiProcessorCount, qk->device));
        return DR_OK;
    }();
    if (rc) {
        delete qk;
        return rc;
    }
    *out = qk;
    return DR_OK;
}

int dr_qk_destroy(dr_qk* qk)
{
    delete qk;
    return DR_OK;
}

int dr_qk_forward(const dr_qk* qk, const void* x_dev, uint32_t dtype, uint64_t ldx, const int32_t* positions_dev, uint64_t rows,
                  void* y_dev, uint64_t ldy, void* cuda_stream)
{
    int rc = check_qk(qk);
    if (rc) return rc;
    const uint64_t cols = (uint64_t)(qk->d.n_q_heads + qk->d.n_kv_heads) * qk->d.head_dim;
    rc = check_rows(dtype, rows, x_dev, ldx, cols, positions_dev, y_dev, ldy, cols);
    if (rc || rows == 0) return rc;
    HeadsArgs a = heads_args(qk, x_dev, dtype, ldx, positions_dev, rows, y_dev, ldy);
    a.heads = a.n_q + a.n_kv;
    deal(a, qk->sms, qk->d.head_dim);
    const uint64_t ctas = (rows * a.parts + kWarps - 1) / kWarps;
    cudaStream_t s = (cudaStream_t)cuda_stream;
    return qk->d.head_dim == 64 ? launch_heads<64, 0>(dtype == DR_F32, a, ctas, s) : launch_heads<128, 0>(dtype == DR_F32, a, ctas, s);
}

int dr_qk_append(const dr_qk* qk, const void* x_dev, uint32_t dtype, uint64_t ldx, const int32_t* positions_dev, uint64_t rows,
                 const int32_t* runs_dev, uint64_t n_runs, const dr_kv_cache* cache, void* y_dev, uint64_t ldy, void* cuda_stream)
{
    int rc = check_qk(qk);
    if (rc == DR_OK) rc = check_cache(cache);
    if (rc) return rc;
    const dr_qk_desc& d = qk->d;
    if (cache->d.kv_heads != d.n_kv_heads || cache->d.head_dim != d.head_dim) {
        set_error("the cache has %u heads of %u dimensions, the rows have %u of %u", cache->d.kv_heads, cache->d.head_dim, d.n_kv_heads, d.head_dim);
        return DR_ERR_INVALID;
    }
    rc = check_rows(dtype, rows, x_dev, ldx, (uint64_t)(d.n_q_heads + 2 * d.n_kv_heads) * d.head_dim, positions_dev, y_dev, ldy,
                    (uint64_t)d.n_q_heads * d.head_dim);
    if (rc) return rc;
    if (n_runs > 0x7FFFFFFFull) {
        set_error("more than 2^31 - 1 runs");
        return DR_ERR_UNSUPPORTED;
    }
    if (n_runs && !runs_dev) {
        set_error("NULL buffer");
        return DR_ERR_INVALID;
    }
    if ((uintptr_t)runs_dev % 16) {
        set_error("runs off 16 bytes");
        return DR_ERR_ALIGN;
    }
    if (rows == 0) return DR_OK;
    HeadsArgs a = heads_args(qk, x_dev, dtype, ldx, positions_dev, rows, y_dev, ldy);
    a.heads = a.n_q;
    deal(a, qk->sms, d.head_dim);
    a.runs = (const int4*)runs_dev;
    a.k = (uint8_t*)cache->d.k_dev;
    a.v = (uint8_t*)cache->d.v_dev;
    a.k_scale = cache->d.k_scale_dev;
    a.v_scale = cache->d.v_scale_dev;
    a.n_blocks = cache->d.n_blocks;
    a.block_tokens = cache->d.block_tokens;
    const uint64_t cache_ctas = n_runs * d.n_kv_heads, ctas = cache_ctas + (rows * a.parts + kAppendThreads / 32 - 1) / (kAppendThreads / 32);
    if (ctas > 0x7FFFFFFFull) {
        set_error("too many rows and runs for one launch");
        return DR_ERR_UNSUPPORTED;
    }
    a.cache_ctas = (uint32_t)cache_ctas;
    cudaStream_t s = (cudaStream_t)cuda_stream;
    if (d.head_dim == 64) return launch_heads<64, 1>(dtype == DR_F32, a, ctas, s);  // (a block of 128 tokens is one turn)
    return a.block_tokens <= 64 ? launch_heads<128, 1>(dtype == DR_F32, a, ctas, s) : launch_heads<128, 2>(dtype == DR_F32, a, ctas, s);
}

int dr_qk_grad_work(const dr_qk* qk, uint64_t* bytes)
{
    if (!qk || !bytes) {
        set_error("NULL argument");
        return DR_ERR_INVALID;
    }
    *bytes = qk->d.q_norm_dev ? (uint64_t)kGradCtas * qk->sms * 2 * qk->d.head_dim * 4 : 0;
    return DR_OK;
}

int dr_qk_grad(const dr_qk* qk, const void* x_dev, uint32_t dtype, uint64_t ldx, const int32_t* positions_dev, const void* dy_dev,
               uint64_t lddy, uint64_t rows, void* dx_dev, uint64_t lddx, float* dq_norm_dev, float* dk_norm_dev, uint32_t accumulate,
               void* work_dev, uint64_t work_bytes, void* cuda_stream)
{
    int rc = check_qk(qk);
    if (rc) return rc;
    const bool norms = qk->d.q_norm_dev != nullptr;
    const uint64_t cols = (uint64_t)(qk->d.n_q_heads + qk->d.n_kv_heads) * qk->d.head_dim;
    rc = check_rows(dtype, rows, norms ? x_dev : dy_dev, norms ? ldx : lddy, cols, positions_dev, dx_dev, lddx, cols);
    if (rc == DR_OK) rc = check_rows(dtype, rows, dy_dev, lddy, cols, positions_dev, dx_dev, lddx, cols);
    if (rc) return rc;
    if (accumulate > 1 || (norms && (!dq_norm_dev || !dk_norm_dev))) {
        set_error("NULL gradient of a norm, or accumulate not 0 / 1");
        return DR_ERR_INVALID;
    }
    uint64_t need = 0;
    dr_qk_grad_work(qk, &need);
    if (norms && (!work_dev || work_bytes < need)) {
        set_error("work holds %llu bytes, %llu are needed", (unsigned long long)(work_dev ? work_bytes : 0), (unsigned long long)need);
        return DR_ERR_SIZE;
    }
    if (((uintptr_t)dq_norm_dev | (uintptr_t)dk_norm_dev) % 4 || (norms && (uintptr_t)work_dev % 16)) {
        set_error("a gradient off 4 bytes or work off 16");
        return DR_ERR_ALIGN;
    }
    if (rows == 0 && (!norms || accumulate)) return DR_OK;
    HeadsArgs a = heads_args(qk, x_dev, dtype, ldx, positions_dev, rows, dx_dev, lddx);
    const uint32_t es = dtype == DR_F32 ? 4 : 2;
    a.dy = dy_dev;
    a.lddy = lddy;
    a.vec = ((norms ? (uintptr_t)x_dev | ldx * es : 0) | (uintptr_t)dy_dev | lddy * es) % 16 == 0;
    a.work = (float*)work_dev;
    // parts of a token's heads, so that the warps' shares differ by little
    const uint64_t most = (uint64_t)kGradCtas * qk->sms;
    const uint32_t per_warp = 512 / qk->d.head_dim, groups = (a.n_q + per_warp - 1) / per_warp + (a.n_kv + per_warp - 1) / per_warp;
    a.parts = groups < kGradParts ? groups : kGradParts;
    const uint64_t wanted = (rows * a.parts + kWarps - 1) / kWarps, ctas = wanted < most ? wanted : most;
    cudaStream_t s = (cudaStream_t)cuda_stream;
    if (ctas) {
        if (qk->d.head_dim == 64)
            rc = dtype == DR_F32 ? launch("heads", grad_kernel<64, true>, ctas, kThreads, s, a) : launch("heads", grad_kernel<64, false>, ctas, kThreads, s, a);
        else
            rc = dtype == DR_F32 ? launch("heads", grad_kernel<128, true>, ctas, kThreads, s, a) : launch("heads", grad_kernel<128, false>, ctas, kThreads, s, a);
        if (rc) return rc;
    }
    if (!norms) return DR_OK;
    return launch("norm sums", norm_sum_kernel, 2 * qk->d.head_dim / 32, 1024, s, (const float*)work_dev, (uint32_t)ctas, qk->d.head_dim,
                  dq_norm_dev, dk_norm_dev, accumulate);
}

}  // extern "C"
