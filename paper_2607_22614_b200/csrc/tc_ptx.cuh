// The sm_100a instructions the tensor-core kernels are written with: mbarriers with bounded waits, tensor-map copies,
// tcgen05 products and their accumulators in tensor memory.
#pragma once
#include <cuda.h>
#include <cstdint>

namespace dr {
namespace tc {

__device__ __forceinline__ uint32_t smem_u32(const void* p) { return (uint32_t)__cvta_generic_to_shared(p); }
__device__ __forceinline__ uint32_t cta_rank()
{
    uint32_t r;
    asm volatile("mov.u32 %0, %%cluster_ctarank;" : "=r"(r));
    return r;
}
__device__ __forceinline__ uint64_t now_ns()
{
    uint64_t t;
    asm volatile("mov.u64 %0, %%globaltimer;" : "=l"(t));
    return t;
}
// The address of a shared variable of this CTA in the CTA `rank` of the cluster.
__device__ __forceinline__ uint32_t in_cta(uint32_t addr, uint32_t rank)
{
    uint32_t r;
    asm volatile("mapa.shared::cluster.u32 %0, %1, %2;" : "=r"(r) : "r"(addr), "r"(rank));
    return r;
}
__device__ __forceinline__ void cluster_sync()
{
    asm volatile("barrier.cluster.arrive.aligned;\nbarrier.cluster.wait.aligned;" ::: "memory");
}

// ---- mbarriers -----------------------------------------------------------------------------------------------------
__device__ __forceinline__ void bar_init(uint32_t bar, uint32_t count)
{
    asm volatile("mbarrier.init.shared::cta.b64 [%0], %1;" ::"r"(bar), "r"(count) : "memory");
}
__device__ __forceinline__ void bar_init_fence() { asm volatile("fence.mbarrier_init.release.cluster;" ::: "memory"); }
__device__ __forceinline__ void bar_expect(uint32_t bar, uint32_t bytes)
{
    asm volatile("mbarrier.arrive.expect_tx.shared::cta.b64 _, [%0], %1;" ::"r"(bar), "r"(bytes) : "memory");
}
__device__ __forceinline__ void bar_arrive(uint32_t bar)
{
    asm volatile("mbarrier.arrive.shared::cta.b64 _, [%0];" ::"r"(bar) : "memory");
}
// `bar` may lie in another CTA of the cluster (an address of in_cta).  What the arrival hands over is tensor memory that has
// been read (ordered by fence_before) or stages that only the copy unit wrote, so no release at cluster scope, which would
// stall the warp on a memory barrier, is needed; where the warp itself has written or read ordinary shared memory that the other
// CTA will read or write, `release` asks for it, and the wait for that barrier acquires at cluster scope.
__device__ __forceinline__ void bar_arrive_cluster(uint32_t bar, bool release = false)
{
    if (release)
        asm volatile("mbarrier.arrive.release.cluster.shared::cluster.b64 _, [%0];" ::"r"(bar) : "memory");
    else
        asm volatile("mbarrier.arrive.shared::cluster.b64 _, [%0];" ::"r"(bar) : "memory");
}
// CLUSTER: what other CTAs of the cluster released with their arrivals (or sent with store_counted) is acquired.
template <bool CLUSTER = false>
__device__ __forceinline__ bool bar_try(uint32_t bar, uint32_t parity)
{
    uint32_t ok;
    if (CLUSTER)
        asm volatile("{\n.reg .pred p;\nmbarrier.try_wait.parity.acquire.cluster.shared::cta.b64 p, [%1], %2;\nselp.u32 %0, 1, 0, p;\n}"
                     : "=r"(ok)
                     : "r"(bar), "r"(parity)
                     : "memory");
    else
        asm volatile("{\n.reg .pred p;\nmbarrier.try_wait.parity.shared::cta.b64 p, [%1], %2;\nselp.u32 %0, 1, 0, p;\n}"
                     : "=r"(ok)
                     : "r"(bar), "r"(parity)
                     : "memory");
    return ok;
}

// How long the CTA's waits may take, and whether one of them has run out.
struct Limit {
    uint32_t stop, us;
};
// Waits for the phase of this parity to complete, at most limit->us.  A wait that runs out (which nothing in these kernels should
// make happen) raises the CTA's `stop` flag and counts in *failures; every role then leaves its loop at its next wait.
template <bool CLUSTER = false>
__device__ __forceinline__ bool bar_wait(uint32_t bar, uint32_t parity, volatile Limit* limit, unsigned long long* failures)
{
    uint64_t since = 0;
    for (uint32_t n = 1; !bar_try<CLUSTER>(bar, parity); ++n) {
        if (n & 63) continue;
        if (limit->stop) return false;
        const uint64_t t = now_ns();
        if (since == 0) since = t;
        if (t - since > limit->us * 1000ull) {
            limit->stop = 1;
            atomicAdd(failures, 1ull);
            return false;
        }
    }
    return true;
}

// The same by a whole warp, with one answer for all lanes.  The roles that issue copies and products run their loops with all lanes
// and let one elected lane issue: the compiler then keeps addresses and descriptors in uniform registers, where these
// instructions want them (with a single lane in the loop every operand is moved there first: 70 cycles a product, measured).
template <bool CLUSTER>
static __device__ __noinline__ bool warp_wait_long(uint32_t bar, uint32_t parity, volatile Limit* limit, unsigned long long* failures)
{
    return __all_sync(0xFFFFFFFFu, bar_wait<CLUSTER>(bar, parity, limit, failures));
}
template <bool CLUSTER = false>
__device__ __forceinline__ bool warp_wait(uint32_t bar, uint32_t parity, volatile Limit* limit, unsigned long long* failures)
{
    if (__all_sync(0xFFFFFFFFu, bar_try<CLUSTER>(bar, parity))) return true;
    return warp_wait_long<CLUSTER>(bar, parity, limit, failures);
}
__device__ __forceinline__ bool elect()
{
    uint32_t p;
    asm volatile("{\n.reg .pred p;\nelect.sync _|p, 0xFFFFFFFF;\nselp.u32 %0, 1, 0, p;\n}" : "=r"(p));
    return p;
}
// For a CTA that has given up: its copies and products in flight end meanwhile.  Before the cluster's last barrier, so that the others
// outlive what this CTA has sent them, and behind it, so that this CTA outlives what they have sent.
__device__ __forceinline__ void let_copies_end(const volatile Limit* limit)
{
    if (!limit->stop) return;
    const uint64_t since = now_ns();
    while (now_ns() - since < 10000000ull) __nanosleep(1000);
}
// A place in a ring of N slots and the parity of its round.
template <uint32_t N>
struct Turn {
    uint32_t slot = 0, round = 0;
    __device__ __forceinline__ void next()
    {
        if (++slot == N) {
            slot = 0;
            round ^= 1;
        }
    }
};

// Waits until the last `used` slots before the ring's place have been given back: their copies have landed and the commits that
// freed them have arrived, so that the CTA may end.
template <uint32_t N>
__device__ __forceinline__ void drain(Turn<N> ring, uint32_t used, uint32_t empty, volatile Limit* limit, unsigned long long* failures)
{
    for (; used; --used) {
        if (ring.slot-- == 0) {
            ring.slot = N - 1;
            ring.round ^= 1;
        }
        if (!warp_wait(empty + 8 * ring.slot, ring.round, limit, failures)) return;
    }
}

// Tiles that one warp of a CTA finds (the divisions and the walk over ragged groups take some 900 cycles) and the others read, up
// to four ahead.  A tile with nt = kNoTile ends the loop.
constexpr uint32_t kTilesAhead = 4, kNoTile = 0xFFFFFFFFu;
template <class T>
struct TileRing {
    T tile[kTilesAhead];
    uint64_t full[kTilesAhead], empty[kTilesAhead];
    __device__ __forceinline__ void init(uint32_t readers)  // warps that read every tile
    {
        for (uint32_t i = 0; i < kTilesAhead; ++i) {
            bar_init(smem_u32(&full[i]), 1);
            bar_init(smem_u32(&empty[i]), readers);
        }
    }
    // by a whole warp
    __device__ __forceinline__ bool put(const T& t, Turn<kTilesAhead>& at, volatile Limit* limit, unsigned long long* failures)
    {
        if (!__all_sync(0xFFFFFFFFu, bar_wait(smem_u32(&empty[at.slot]), at.round ^ 1, limit, failures))) return false;
        if ((threadIdx.x & 31) == 0) {
            tile[at.slot] = t;
            bar_arrive(smem_u32(&full[at.slot]));
        }
        __syncwarp();
        at.next();
        return true;
    }
    __device__ __forceinline__ bool get(T& t, Turn<kTilesAhead>& at, volatile Limit* limit, unsigned long long* failures)
    {
        if (!__all_sync(0xFFFFFFFFu, bar_wait(smem_u32(&full[at.slot]), at.round, limit, failures))) return false;
        t = tile[at.slot];
        __syncwarp();
        if ((threadIdx.x & 31) == 0) bar_arrive(smem_u32(&empty[at.slot]));
        at.next();
        return t.nt != kNoTile;
    }
};

// 16 bytes to the shared memory of a CTA of the cluster, counted on a barrier of that CTA: whoever waits for the barrier sees them.
__device__ __forceinline__ void store_counted(uint32_t dst, const float4& v, uint32_t bar)
{
    asm volatile("st.async.shared::cluster.mbarrier::complete_tx::bytes.v4.b32 [%0], {%1, %2, %3, %4}, [%5];" ::"r"(dst),
                 "r"(__float_as_uint(v.x)), "r"(__float_as_uint(v.y)), "r"(__float_as_uint(v.z)), "r"(__float_as_uint(v.w)), "r"(bar)
                 : "memory");
}

// ---- tensor-map copies ---------------------------------------------------------------------------------------------
// Completion is counted in bytes on `bar`, which for the PAIR form may lie in either CTA of the pair.
template <bool PAIR>
__device__ __forceinline__ void load_2d(uint32_t dst, const CUtensorMap* map, uint32_t bar, int x, int y)
{
    if (PAIR)
        asm volatile("cp.async.bulk.tensor.2d.cta_group::2.shared::cluster.global.mbarrier::complete_tx::bytes [%0], [%1, {%3, %4}], [%2];"
                     ::"r"(dst), "l"(map), "r"(bar), "r"(x), "r"(y) : "memory");
    else
        asm volatile("cp.async.bulk.tensor.2d.shared::cluster.global.mbarrier::complete_tx::bytes [%0], [%1, {%3, %4}], [%2];"
                     ::"r"(dst), "l"(map), "r"(bar), "r"(x), "r"(y) : "memory");
}
template <bool PAIR>
__device__ __forceinline__ void load_3d(uint32_t dst, const CUtensorMap* map, uint32_t bar, int x, int y, int z)
{
    if (PAIR)
        asm volatile("cp.async.bulk.tensor.3d.cta_group::2.shared::cluster.global.mbarrier::complete_tx::bytes [%0], [%1, {%3, %4, %5}], [%2];"
                     ::"r"(dst), "l"(map), "r"(bar), "r"(x), "r"(y), "r"(z) : "memory");
    else
        asm volatile("cp.async.bulk.tensor.3d.shared::cluster.global.mbarrier::complete_tx::bytes [%0], [%1, {%3, %4, %5}], [%2];"
                     ::"r"(dst), "l"(map), "r"(bar), "r"(x), "r"(y), "r"(z) : "memory");
}
// The way back: a box of shared memory to the tensor of the map (coordinates inside it).
__device__ __forceinline__ void store_2d(const CUtensorMap* map, uint32_t src, int x, int y)
{
    asm volatile("cp.async.bulk.tensor.2d.global.shared::cta.bulk_group [%0, {%2, %3}], [%1];" ::"l"(map), "r"(src), "r"(x), "r"(y)
                 : "memory");
}
__device__ __forceinline__ void store_3d(const CUtensorMap* map, uint32_t src, int x, int y, int z)
{
    asm volatile("cp.async.bulk.tensor.3d.global.shared::cta.bulk_group [%0, {%2, %3, %4}], [%1];" ::"l"(map), "r"(src), "r"(x),
                 "r"(y), "r"(z)
                 : "memory");
}
__device__ __forceinline__ void add_3d(const CUtensorMap* map, uint32_t src, int x, int y, int z)
{
    asm volatile("cp.reduce.async.bulk.tensor.3d.global.shared::cta.add.tile.bulk_group [%0, {%2, %3, %4}], [%1];" ::"l"(map),
                 "r"(src), "r"(x), "r"(y), "r"(z)
                 : "memory");
}
__device__ __forceinline__ void prefetch_map(const CUtensorMap* map)
{
    asm volatile("prefetch.tensormap [%0];" ::"l"(map) : "memory");
}
// Generic writes to shared memory become visible to the tensor cores and the copy unit.
__device__ __forceinline__ void fence_async() { asm volatile("fence.proxy.async.shared::cta;" ::: "memory"); }

// One 4-byte copy to shared memory, a zero when !valid; copies_arrive makes the thread's copies so far arrive on `bar`.
__device__ __forceinline__ void copy_4(uint32_t dst, const void* src, bool valid)
{
    asm volatile("cp.async.ca.shared.global [%0], [%1], 4, %2;" ::"r"(dst), "l"(src), "r"(valid ? 4 : 0) : "memory");
}
__device__ __forceinline__ void copies_arrive(uint32_t bar)
{
    asm volatile("cp.async.mbarrier.arrive.noinc.shared::cta.b64 [%0];" ::"r"(bar) : "memory");
}

// ---- tensor memory and products --------------------------------------------------------------------------------------
template <int CTAS>
__device__ __forceinline__ void tmem_alloc(uint32_t dst, uint32_t columns)
{
    if (CTAS == 2)
        asm volatile("tcgen05.alloc.cta_group::2.sync.aligned.shared::cta.b32 [%0], %1;" ::"r"(dst), "r"(columns) : "memory");
    else
        asm volatile("tcgen05.alloc.cta_group::1.sync.aligned.shared::cta.b32 [%0], %1;" ::"r"(dst), "r"(columns) : "memory");
}
template <int CTAS>
__device__ __forceinline__ void tmem_free(uint32_t addr, uint32_t columns)
{
    if (CTAS == 2) {
        asm volatile("tcgen05.relinquish_alloc_permit.cta_group::2.sync.aligned;");
        asm volatile("tcgen05.dealloc.cta_group::2.sync.aligned.b32 %0, %1;" ::"r"(addr), "r"(columns) : "memory");
    } else {
        asm volatile("tcgen05.relinquish_alloc_permit.cta_group::1.sync.aligned;");
        asm volatile("tcgen05.dealloc.cta_group::1.sync.aligned.b32 %0, %1;" ::"r"(addr), "r"(columns) : "memory");
    }
}
__device__ __forceinline__ void fence_before() { asm volatile("tcgen05.fence::before_thread_sync;" ::: "memory"); }
__device__ __forceinline__ void fence_after() { asm volatile("tcgen05.fence::after_thread_sync;" ::: "memory"); }

// Descriptor of an operand whose rows of 128 bytes are swizzled in groups of eight rows.  K-major: a row holds 128 bytes
// of the contraction, eight-row groups follow each other every 1024 bytes.  MN-major: a row holds 64 bf16 of the output
// dimension at one position of the contraction, eight positions every 1024 bytes, the next 64 outputs `panel` bytes on.
__device__ __forceinline__ uint64_t operand(uint32_t addr, uint32_t panel)
{
    return (uint64_t)((addr & 0x3FFFF) >> 4) | (uint64_t)(panel >> 4) << 16 | (uint64_t)(1024 >> 4) << 32 | 1ull << 46 | 2ull << 61;
}
// Shape and types of a product: fp32 accumulators, bf16 (fp8 = false) or e4m3 operands, M and N outputs.
__device__ __forceinline__ uint32_t shape_of(bool fp8, bool a_mn, bool b_mn, uint32_t m, uint32_t n)
{
    return 1u << 4 | (fp8 ? 0u : 1u << 7 | 1u << 10) | (uint32_t)a_mn << 15 | (uint32_t)b_mn << 16 | (n >> 3) << 17 | (m >> 4) << 24;
}
template <int CTAS, bool FP8>
__device__ __forceinline__ void mma(uint32_t d, uint64_t a, uint64_t b, uint32_t shape, uint32_t add)
{
    if (CTAS == 2 && FP8)
        asm volatile("{\n.reg .pred p;\nsetp.ne.u32 p, %4, 0;\ntcgen05.mma.cta_group::2.kind::f8f6f4 [%0], %1, %2, %3, p;\n}"
                     ::"r"(d), "l"(a), "l"(b), "r"(shape), "r"(add) : "memory");
    else if (CTAS == 2)
        asm volatile("{\n.reg .pred p;\nsetp.ne.u32 p, %4, 0;\ntcgen05.mma.cta_group::2.kind::f16 [%0], %1, %2, %3, p;\n}"
                     ::"r"(d), "l"(a), "l"(b), "r"(shape), "r"(add) : "memory");
    else if (FP8)
        asm volatile("{\n.reg .pred p;\nsetp.ne.u32 p, %4, 0;\ntcgen05.mma.cta_group::1.kind::f8f6f4 [%0], %1, %2, %3, p;\n}"
                     ::"r"(d), "l"(a), "l"(b), "r"(shape), "r"(add) : "memory");
    else
        asm volatile("{\n.reg .pred p;\nsetp.ne.u32 p, %4, 0;\ntcgen05.mma.cta_group::1.kind::f16 [%0], %1, %2, %3, p;\n}"
                     ::"r"(d), "l"(a), "l"(b), "r"(shape), "r"(add) : "memory");
}
// Arrives on `bar` (in both CTAs of a pair) once every product issued so far has been computed.
template <int CTAS>
__device__ __forceinline__ void commit(uint32_t bar)
{
    if (CTAS == 2)
        asm volatile("tcgen05.commit.cta_group::2.mbarrier::arrive::one.shared::cluster.multicast::cluster.b64 [%0], %1;"
                     ::"r"(bar), "h"((uint16_t)3) : "memory");
    else
        asm volatile("tcgen05.commit.cta_group::1.mbarrier::arrive::one.shared::cluster.b64 [%0];" ::"r"(bar) : "memory");
}
// 32 lanes x 32 columns of the warp's quarter of tensor memory, complete on return (the wait is part of the statement, so
// that no use of the registers can move above it).  With t the lane of the warp: a[4 j + 0, 1] = columns 8 j + 2 (t % 4) + {0, 1}
// of lane t / 4, a[4 j + 2, 3] the same of lane t / 4 + 8; b: of lanes t / 4 + 16 and t / 4 + 24.
__device__ __forceinline__ void tmem_load(uint32_t addr, float (&a)[16], float (&b)[16])
{
    asm volatile("tcgen05.ld.sync.aligned.16x256b.x4.b32 {%0,%1,%2,%3,%4,%5,%6,%7,%8,%9,%10,%11,%12,%13,%14,%15}, [%32];\n"
                 "tcgen05.ld.sync.aligned.16x256b.x4.b32 {%16,%17,%18,%19,%20,%21,%22,%23,%24,%25,%26,%27,%28,%29,%30,%31}, [%33];\n"
                 "tcgen05.wait::ld.sync.aligned;"
                 : "=f"(a[0]), "=f"(a[1]), "=f"(a[2]), "=f"(a[3]), "=f"(a[4]), "=f"(a[5]), "=f"(a[6]), "=f"(a[7]), "=f"(a[8]), "=f"(a[9]), "=f"(a[10]), "=f"(a[11]), "=f"(a[12]), "=f"(a[13]), "=f"(a[14]), "=f"(a[15]),
                   "=f"(b[0]), "=f"(b[1]), "=f"(b[2]), "=f"(b[3]), "=f"(b[4]), "=f"(b[5]), "=f"(b[6]), "=f"(b[7]), "=f"(b[8]), "=f"(b[9]), "=f"(b[10]), "=f"(b[11]), "=f"(b[12]), "=f"(b[13]), "=f"(b[14]), "=f"(b[15])
                 : "r"(addr), "r"(addr + (16u << 16))
                 : "memory");
}
// 32 columns of the thread's own lane.  The load is only started: tmem_arrived(v) makes the registers usable.
__device__ __forceinline__ void tmem_start(uint32_t addr, float (&v)[32])
{
    asm volatile("tcgen05.ld.sync.aligned.32x32b.x32.b32 {%0,%1,%2,%3,%4,%5,%6,%7,%8,%9,%10,%11,%12,%13,%14,%15,%16,%17,%18,%19,%20,%21,%22,%23,%24,%25,%26,%27,%28,%29,%30,%31}, [%32];"
                 : "=f"(v[0]), "=f"(v[1]), "=f"(v[2]), "=f"(v[3]), "=f"(v[4]), "=f"(v[5]), "=f"(v[6]), "=f"(v[7]), "=f"(v[8]), "=f"(v[9]), "=f"(v[10]), "=f"(v[11]), "=f"(v[12]), "=f"(v[13]), "=f"(v[14]), "=f"(v[15]), "=f"(v[16]), "=f"(v[17]), "=f"(v[18]), "=f"(v[19]), "=f"(v[20]), "=f"(v[21]), "=f"(v[22]), "=f"(v[23]), "=f"(v[24]), "=f"(v[25]), "=f"(v[26]), "=f"(v[27]), "=f"(v[28]), "=f"(v[29]), "=f"(v[30]), "=f"(v[31])
                 : "r"(addr)
                 : "memory");
}
__device__ __forceinline__ void tmem_arrived(float (&v)[32])
{
    asm volatile("tcgen05.wait::ld.sync.aligned;"
                 : "+f"(v[0]), "+f"(v[1]), "+f"(v[2]), "+f"(v[3]), "+f"(v[4]), "+f"(v[5]), "+f"(v[6]), "+f"(v[7]), "+f"(v[8]), "+f"(v[9]), "+f"(v[10]), "+f"(v[11]), "+f"(v[12]), "+f"(v[13]), "+f"(v[14]), "+f"(v[15]), "+f"(v[16]), "+f"(v[17]), "+f"(v[18]), "+f"(v[19]), "+f"(v[20]), "+f"(v[21]), "+f"(v[22]), "+f"(v[23]), "+f"(v[24]), "+f"(v[25]), "+f"(v[26]), "+f"(v[27]), "+f"(v[28]), "+f"(v[29]), "+f"(v[30]), "+f"(v[31])
                 :
                 : "memory");
}

// ---- arithmetic and stores -------------------------------------------------------------------------------------------
__device__ __forceinline__ uint64_t pair_of(float lo, float hi)
{
    uint64_t d;
    asm("mov.b64 %0, {%1, %2};" : "=l"(d) : "f"(lo), "f"(hi));
    return d;
}
__device__ __forceinline__ uint64_t mul2(uint64_t a, uint64_t b)
{
    uint64_t d;
    asm("mul.rn.f32x2 %0, %1, %2;" : "=l"(d) : "l"(a), "l"(b));
    return d;
}
// (a0, a1) += (p0, p1) * (s0, s1), two fp32 multiply-adds in one instruction; volatile, so that it keeps its place between the
// loads of the accumulators
__device__ __forceinline__ void fma2(float& a0, float& a1, float p0, float p1, uint64_t s)
{
    uint64_t a, p;
    asm("mov.b64 %0, {%1, %2};" : "=l"(a) : "f"(a0), "f"(a1));
    asm("mov.b64 %0, {%1, %2};" : "=l"(p) : "f"(p0), "f"(p1));
    asm volatile("fma.rn.f32x2 %0, %1, %2, %0;" : "+l"(a) : "l"(p), "l"(s));
    asm("mov.b64 {%0, %1}, %2;" : "=f"(a0), "=f"(a1) : "l"(a));
}
__device__ __forceinline__ uint32_t pack_bf16(float lo, float hi)
{
    uint32_t d;
    asm("cvt.rn.bf16x2.f32 %0, %1, %2;" : "=r"(d) : "f"(hi), "f"(lo));
    return d;
}
// Four 8 x 8 blocks of 16-bit values, transposed: the thread's packed pair of columns goes to two rows of shared memory.
__device__ __forceinline__ void store_transposed(uint32_t addr, uint32_t a, uint32_t b, uint32_t c, uint32_t d)
{
    asm volatile("stmatrix.sync.aligned.m8n8.x4.trans.shared.b16 [%0], {%1, %2, %3, %4};" ::"r"(addr), "r"(a), "r"(b), "r"(c), "r"(d)
                 : "memory");
}

__device__ __forceinline__ void store_32(void* p, uint32_t a, uint32_t b, uint32_t c, uint32_t d, uint32_t e, uint32_t f, uint32_t g,
                                         uint32_t h)
{
    asm volatile("st.global.v8.b32 [%0], {%1,%2,%3,%4,%5,%6,%7,%8};" ::"l"(p), "r"(a), "r"(b), "r"(c), "r"(d), "r"(e), "r"(f),
                 "r"(g), "r"(h)
                 : "memory");
}

__device__ __forceinline__ void store_shared(uint32_t addr, uint32_t a, uint32_t b, uint32_t c, uint32_t d)
{
    asm volatile("st.shared.v4.b32 [%0], {%1,%2,%3,%4};" ::"r"(addr), "r"(a), "r"(b), "r"(c), "r"(d) : "memory");
}

}  // namespace tc
}  // namespace dr
