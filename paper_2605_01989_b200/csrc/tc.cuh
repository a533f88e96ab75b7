// Building blocks of the tensor-core kernels (sm_100a): mbarriers with bounded waits, TMA tile loads, tcgen05 products
// with accumulators in tensor memory, and the shared-memory layout that all of them agree on.
//
// Layout.  A tile of R rows (tokens) by up to 64 16-bit columns is R * 128 bytes, row r at r * 128, its 16-byte chunk c at
// place c ^ (r % 8) of the row (the 128-byte swizzle that TMA writes and tcgen05 reads); wider tiles are several such
// blocks one after the other.  The same bytes serve as an operand whose summed dimension runs along the row (K-major) or
// over the rows (MN-major), which is how one copy of q, k, v, dout or ds enters two products, once transposed.
#pragma once

#include <cuda.h>

#include "types.cuh"

namespace dblp {

constexpr uint32_t kBlockBytes = 128 * 128;         // 128 rows x 64 columns of 16 bits

__device__ __forceinline__ uint32_t smem_addr(const void* p) { return (uint32_t)__cvta_generic_to_shared(p); }

__device__ __forceinline__ void bar_init(uint64_t* b, uint32_t count)
{
    asm volatile("mbarrier.init.shared::cta.b64 [%0], %1;" ::"r"(smem_addr(b)), "r"(count) : "memory");
}
__device__ __forceinline__ void bar_arrive(uint64_t* b)
{
    asm volatile("mbarrier.arrive.shared::cta.b64 _, [%0];" ::"r"(smem_addr(b)) : "memory");
}
// One arrival for a warp: arrivals on one barrier are served one after the other, 512 of them cost thousands of cycles.
__device__ __forceinline__ void warp_arrive(uint64_t* b)
{
    __syncwarp();
    if ((threadIdx.x & 31) == 0) bar_arrive(b);
}
__device__ __forceinline__ void bar_expect(uint64_t* b, uint32_t bytes)
{
    asm volatile("mbarrier.arrive.expect_tx.shared::cta.b64 _, [%0], %1;" ::"r"(smem_addr(b)), "r"(bytes) : "memory");
}
// (A time hint for the sleep, 200 ns to 1 ms, and test_wait were tried: 2 to 9 % slower in all kernels.)
__device__ __forceinline__ bool bar_try(uint64_t* b, uint32_t parity)
{
    uint32_t ok;
    asm volatile("{\n.reg .pred p;\nmbarrier.try_wait.parity.shared::cta.b64 p, [%1], %2;\nselp.u32 %0, 1, 0, p;\n}"
                 : "=r"(ok)
                 : "r"(smem_addr(b)), "r"(parity)
                 : "memory");
    return ok != 0;
}

// The same without waiting at all: try_wait may sleep for microseconds before it says no.
__device__ __forceinline__ bool bar_test(uint64_t* b, uint32_t parity)
{
    uint32_t ok;
    asm volatile("{\n.reg .pred p;\nmbarrier.test_wait.parity.shared::cta.b64 p, [%1], %2;\nselp.u32 %0, 1, 0, p;\n}"
                 : "=r"(ok)
                 : "r"(smem_addr(b)), "r"(parity)
                 : "memory");
    return ok != 0;
}

// Every wait is bounded: after about two seconds the waiting thread raises the block's flag, which ends all other waits of
// the block at once; the block then skips its work, lets its copies land, frees its tensor memory and returns.  The results
// of such a launch are incomplete, and the device's count of timeouts (dblp_wait_timeouts) says so.
constexpr long long kWaitCycles = 1ll << 32;

struct Guard {
    volatile uint32_t* dead;            // shared memory, one per block, starts at 0
    unsigned long long* timeouts;       // device memory, one per device
};

__device__ __forceinline__ bool bar_wait_slow(uint64_t* b, uint32_t parity, Guard g)
{
    const long long t0 = clock64();
    for (;;) {
        if (bar_try(b, parity)) return true;
        if (*g.dead) return false;
        if (clock64() - t0 > kWaitCycles) {
            if (atomicExch((uint32_t*)g.dead, 1u) == 0) atomicAdd(g.timeouts, 1ull);
            return false;
        }
    }
}
__device__ __forceinline__ bool bar_wait(uint64_t* b, uint32_t parity, const Guard& g)
{
    if (bar_try(b, parity)) return true;
    return bar_wait_slow(b, parity, g);
}
// The same for a warp that runs together: one answer for all its lanes.
__device__ __forceinline__ bool warp_wait(uint64_t* b, uint32_t parity, const Guard& g)
{
    return __all_sync(0xFFFFFFFFu, bar_wait(b, parity, g));
}
// For copies and products that were issued and must be done before the block ends, and for nothing else: it tells nobody when
// it gives up.  Bounded by itself, whatever the flag says.
__device__ __forceinline__ void bar_drain(uint64_t* b, uint32_t parity)
{
    const long long t0 = clock64();
    while (!bar_try(b, parity) && clock64() - t0 < kWaitCycles) {}
}

// A value that is the same in all lanes, in a form from which the compiler sees that: loops and branches on it, and the
// operands of the products inside them, then stay in uniform registers.
__device__ __forceinline__ uint32_t uniform(uint32_t x) { return __shfl_sync(0xFFFFFFFFu, x, 0); }

// ---- TMA -------------------------------------------------------------------------------------------------------------
__device__ __forceinline__ void tma_tile(void* dst, const CUtensorMap* map, uint64_t* bar, int c0, int c1, int c2, int c3)
{
    asm volatile("cp.async.bulk.tensor.4d.shared::cluster.global.tile.mbarrier::complete_tx::bytes [%0], [%1, {%2, %3, %4, %5}], [%6];"
                 ::"r"(smem_addr(dst)), "l"(map), "r"(c0), "r"(c1), "r"(c2), "r"(c3), "r"(smem_addr(bar))
                 : "memory");
}
// bytes: a multiple of 16, both addresses 16-byte aligned
__device__ __forceinline__ void bulk_load(void* dst, const void* src, uint32_t bytes, uint64_t* bar)
{
    asm volatile("cp.async.bulk.shared::cluster.global.mbarrier::complete_tx::bytes [%0], [%1], %2, [%3];"
                 ::"r"(smem_addr(dst)), "l"(src), "r"(bytes), "r"(smem_addr(bar))
                 : "memory");
}
// shared -> global, plain or added in fp32 by the memory system; grouped per issuing thread
__device__ __forceinline__ void bulk_store(void* dst, const void* src, uint32_t bytes)
{
    asm volatile("cp.async.bulk.global.shared::cta.bulk_group [%0], [%1], %2;" ::"l"(dst), "r"(smem_addr(src)), "r"(bytes) : "memory");
}
__device__ __forceinline__ void bulk_add_f32(void* dst, const void* src, uint32_t bytes)
{
    asm volatile("cp.reduce.async.bulk.global.shared::cta.bulk_group.add.f32 [%0], [%1], %2;" ::"l"(dst), "r"(smem_addr(src)), "r"(bytes) : "memory");
}
__device__ __forceinline__ void tma_store3(const CUtensorMap* map, const void* src, int c0, int c1, int c2)
{
    asm volatile("cp.async.bulk.tensor.3d.global.shared::cta.tile.bulk_group [%0, {%1, %2, %3}], [%4];" ::"l"(map), "r"(c0), "r"(c1), "r"(c2),
                 "r"(smem_addr(src))
                 : "memory");
}
__device__ __forceinline__ void bulk_commit() { asm volatile("cp.async.bulk.commit_group;" ::: "memory"); }
// at most N groups of this thread still read shared memory / are not yet written
template <int N> __device__ __forceinline__ void bulk_wait_read() { asm volatile("cp.async.bulk.wait_group.read %0;" ::"n"(N) : "memory"); }
template <int N> __device__ __forceinline__ void bulk_wait() { asm volatile("cp.async.bulk.wait_group %0;" ::"n"(N) : "memory"); }
__device__ __forceinline__ void fence_async_smem() { asm volatile("fence.proxy.async.shared::cta;" ::: "memory"); }
__device__ __forceinline__ void fence_bar_init() { asm volatile("fence.mbarrier_init.release.cluster;" ::: "memory"); }

// ---- tensor memory ---------------------------------------------------------------------------------------------------
// Everything here is .sync.aligned: all 32 lanes execute the same instruction together, anything else is undefined.  After code
// that only some lanes went through (a copy issued by lane 0, a store under a lane's bound) a __syncwarp() or a warp_wait comes
// first.
template <int COLS> __device__ __forceinline__ void tmem_alloc(uint32_t* slot)
{
    asm volatile("tcgen05.alloc.cta_group::1.sync.aligned.shared::cta.b32 [%0], %1;" ::"r"(smem_addr(slot)), "n"(COLS) : "memory");
    asm volatile("tcgen05.relinquish_alloc_permit.cta_group::1.sync.aligned;" ::: "memory");
}
template <int COLS> __device__ __forceinline__ void tmem_free(uint32_t addr)
{
    asm volatile("tcgen05.dealloc.cta_group::1.sync.aligned.b32 %0, %1;" ::"r"(addr), "n"(COLS) : "memory");
}
__device__ __forceinline__ void tc_fence_before() { asm volatile("tcgen05.fence::before_thread_sync;" ::: "memory"); }
__device__ __forceinline__ void tc_fence_after() { asm volatile("tcgen05.fence::after_thread_sync;" ::: "memory"); }
// Registers that tcgen05.ld fills may be read only after the wait: the empty statements make every later use of x depend on
// it, so that no arithmetic moves up past it.
template <int N> __device__ __forceinline__ void tmem_loaded(uint32_t* x)
{
#pragma unroll
    for (int i = 0; i < N; ++i) asm volatile("" : "+r"(x[i]));
}
__device__ __forceinline__ void tmem_wait_ld() { asm volatile("tcgen05.wait::ld.sync.aligned;" ::: "memory"); }
template <int N> __device__ __forceinline__ void tmem_wait_ld(uint32_t* x)
{
    tmem_wait_ld();
    tmem_loaded<N>(x);
}
__device__ __forceinline__ void tmem_wait_st() { asm volatile("tcgen05.wait::st.sync.aligned;" ::: "memory"); }

// 32 columns of the calling warp's 32 lanes (one row per thread).
__device__ __forceinline__ void tmem_ld32(uint32_t addr, uint32_t* r)
{
    asm volatile(
        "tcgen05.ld.sync.aligned.32x32b.x32.b32 {%0,%1,%2,%3,%4,%5,%6,%7,%8,%9,%10,%11,%12,%13,%14,%15,%16,%17,%18,%19,%20,%21,%22,"
        "%23,%24,%25,%26,%27,%28,%29,%30,%31}, [%32];"
        : "=r"(r[0]), "=r"(r[1]), "=r"(r[2]), "=r"(r[3]), "=r"(r[4]), "=r"(r[5]), "=r"(r[6]), "=r"(r[7]), "=r"(r[8]), "=r"(r[9]),
          "=r"(r[10]), "=r"(r[11]), "=r"(r[12]), "=r"(r[13]), "=r"(r[14]), "=r"(r[15]), "=r"(r[16]), "=r"(r[17]), "=r"(r[18]),
          "=r"(r[19]), "=r"(r[20]), "=r"(r[21]), "=r"(r[22]), "=r"(r[23]), "=r"(r[24]), "=r"(r[25]), "=r"(r[26]), "=r"(r[27]),
          "=r"(r[28]), "=r"(r[29]), "=r"(r[30]), "=r"(r[31])
        : "r"(addr));
}
__device__ __forceinline__ void tmem_ld16(uint32_t addr, uint32_t* r)
{
    asm volatile("tcgen05.ld.sync.aligned.32x32b.x16.b32 {%0,%1,%2,%3,%4,%5,%6,%7,%8,%9,%10,%11,%12,%13,%14,%15}, [%16];"
                 : "=r"(r[0]), "=r"(r[1]), "=r"(r[2]), "=r"(r[3]), "=r"(r[4]), "=r"(r[5]), "=r"(r[6]), "=r"(r[7]), "=r"(r[8]),
                   "=r"(r[9]), "=r"(r[10]), "=r"(r[11]), "=r"(r[12]), "=r"(r[13]), "=r"(r[14]), "=r"(r[15])
                 : "r"(addr));
}
__device__ __forceinline__ void tmem_st16(uint32_t addr, const uint32_t* r)
{
    asm volatile("tcgen05.st.sync.aligned.32x32b.x16.b32 [%0], {%1,%2,%3,%4,%5,%6,%7,%8,%9,%10,%11,%12,%13,%14,%15,%16};" ::"r"(addr),
                 "r"(r[0]), "r"(r[1]), "r"(r[2]), "r"(r[3]), "r"(r[4]), "r"(r[5]), "r"(r[6]), "r"(r[7]), "r"(r[8]), "r"(r[9]),
                 "r"(r[10]), "r"(r[11]), "r"(r[12]), "r"(r[13]), "r"(r[14]), "r"(r[15])
                 : "memory");
}

__device__ __forceinline__ void tmem_st8(uint32_t addr, const uint32_t* r)
{
    asm volatile("tcgen05.st.sync.aligned.32x32b.x8.b32 [%0], {%1,%2,%3,%4,%5,%6,%7,%8};" ::"r"(addr), "r"(r[0]), "r"(r[1]), "r"(r[2]),
                 "r"(r[3]), "r"(r[4]), "r"(r[5]), "r"(r[6]), "r"(r[7])
                 : "memory");
}

// ---- products --------------------------------------------------------------------------------------------------------
// Operand descriptors for the layout above.  K-major: groups of 8 rows are 1024 bytes apart; a step of 16 along the summed
// dimension is 32 bytes within the row.  MN-major: the summed dimension runs over the rows, 8 of them 1024 bytes apart,
// and blocks of 64 columns `block` bytes apart; a step of 16 along the summed dimension is 2048 bytes.
__device__ __forceinline__ uint64_t desc_base() { return 1ull << 46 | 2ull << 61 | (uint64_t)(1024 >> 4) << 32; }
__device__ __forceinline__ uint64_t desc_k(uint32_t addr) { return desc_base() | 1ull << 16 | (uint64_t)((addr & 0x3FFFFu) >> 4); }
__device__ __forceinline__ uint64_t desc_mn(uint32_t addr, uint32_t block)
{
    return desc_base() | (uint64_t)(block >> 4) << 16 | (uint64_t)((addr & 0x3FFFFu) >> 4);
}

// kind::f16 instruction descriptor: fp32 accumulator, both operands of one 16-bit type.
template <typename T> __host__ __device__ constexpr uint32_t mma_desc(int m, int n, bool a_mn, bool b_mn)
{
    return 1u << 4 | (std::is_same<T, __nv_bfloat16>::value ? (1u << 7 | 1u << 10) : 0u) | (a_mn ? 1u << 15 : 0u) |
           (b_mn ? 1u << 16 : 0u) | (uint32_t)(n >> 3) << 17 | (uint32_t)(m >> 4) << 24;
}
// Products are issued by one lane of a warp that runs together, elected in the same statement (the same lane every time, so a
// commit covers the products before it).  Operands, loops and branches around them have to be visibly uniform (`uniform`):
// with a branch on the lane number each product cost about 95 cycles to issue.
__device__ __forceinline__ void mma_ss(uint32_t d, uint64_t a, uint64_t b, uint32_t idesc, uint32_t acc)
{
    asm volatile("{\n.reg .pred p, q;\nsetp.ne.b32 p, %4, 0;\nelect.sync _|q, 0xFFFFFFFF;\n"
                 "@q tcgen05.mma.cta_group::1.kind::f16 [%0], %1, %2, %3, p;\n}" ::"r"(d), "l"(a), "l"(b), "r"(idesc), "r"(acc)
                 : "memory");
}
__device__ __forceinline__ void mma_ts(uint32_t d, uint32_t a, uint64_t b, uint32_t idesc, uint32_t acc)
{
    asm volatile("{\n.reg .pred p, q;\nsetp.ne.b32 p, %4, 0;\nelect.sync _|q, 0xFFFFFFFF;\n"
                 "@q tcgen05.mma.cta_group::1.kind::f16 [%0], [%1], %2, %3, p;\n}" ::"r"(d), "r"(a), "l"(b), "r"(idesc), "r"(acc)
                 : "memory");
}
// The barrier completes a phase when every product issued before by this warp is done.
__device__ __forceinline__ void mma_commit(uint64_t* bar)
{
    asm volatile("{\n.reg .pred q;\nelect.sync _|q, 0xFFFFFFFF;\n"
                 "@q tcgen05.commit.cta_group::1.mbarrier::arrive::one.shared::cluster.b64 [%0];\n}" ::"r"(smem_addr(bar))
                 : "memory");
}

// ---- arithmetic on pairs ---------------------------------------------------------------------------------------------
__device__ __forceinline__ float2 pair(uint32_t a, uint32_t b) { return make_float2(__uint_as_float(a), __uint_as_float(b)); }
__device__ __forceinline__ float2 fma2(float2 a, float2 b, float2 c)
{
    uint64_t r;
    asm("fma.rn.f32x2 %0, %1, %2, %3;"
        : "=l"(r)
        : "l"(*reinterpret_cast<uint64_t*>(&a)), "l"(*reinterpret_cast<uint64_t*>(&b)), "l"(*reinterpret_cast<uint64_t*>(&c)));
    return *reinterpret_cast<float2*>(&r);
}
__device__ __forceinline__ float2 add2(float2 a, float2 b)
{
    uint64_t r;
    asm("add.rn.f32x2 %0, %1, %2;" : "=l"(r) : "l"(*reinterpret_cast<uint64_t*>(&a)), "l"(*reinterpret_cast<uint64_t*>(&b)));
    return *reinterpret_cast<float2*>(&r);
}
__device__ __forceinline__ float2 mul2(float2 a, float2 b)
{
    uint64_t r;
    asm("mul.rn.f32x2 %0, %1, %2;" : "=l"(r) : "l"(*reinterpret_cast<uint64_t*>(&a)), "l"(*reinterpret_cast<uint64_t*>(&b)));
    return *reinterpret_cast<float2*>(&r);
}
__device__ __forceinline__ float max3(float a, float b, float c)
{
    float r;
    asm("max.f32 %0, %1, %2, %3;" : "=f"(r) : "f"(a), "f"(b), "f"(c));
    return r;
}
__device__ __forceinline__ float exp2_fast(float x)
{
    float r;
    asm("ex2.approx.ftz.f32 %0, %1;" : "=f"(r) : "f"(x));
    return r;
}

__device__ __forceinline__ float max_nan(float a, float b)      // NaN if either is
{
    float r;
    asm("max.NaN.f32 %0, %1, %2;" : "=f"(r) : "f"(a), "f"(b));
    return r;
}

// 2^x of two values on the FMA and integer units, for x < 128: x = n + f with n the nearest integer, 2^f by a polynomial of
// degree 4 fitted here to the least largest relative error on [-1/2, 1/2] (2.7e-6, evaluated in fp32), times 2^n made of its bits;
// n = -127 makes the bits of 0, so what falls below the exponent's range, -infinity too, gives 0.  NaN stays NaN and +infinity
// becomes NaN: both pass through f.  The special function unit gives 16 results a cycle and SM; a part of them computed this way
// shortens a softmax.
__device__ __forceinline__ float2 exp2_pair(float2 x)
{
    constexpr float kShift = 12582912.0f;                       // 1.5 * 2^23: adding it rounds to an integer in the low bits
    x.x = max_nan(x.x, -127.0f);
    x.y = max_nan(x.y, -127.0f);
    const float2 t = add2(x, make_float2(kShift, kShift)), n = add2(t, make_float2(-kShift, -kShift));
    const float2 f = fma2(n, make_float2(-1.0f, -1.0f), x);
    float2 p = fma2(f, make_float2(0.009570102207362652f, 0.009570102207362652f), make_float2(0.05591785907745361f, 0.05591785907745361f));
    p = fma2(p, f, make_float2(0.240247443318367f, 0.240247443318367f));
    p = fma2(p, f, make_float2(0.6931217908859253f, 0.6931217908859253f));
    p = fma2(p, f, make_float2(0.9999992847442627f, 0.9999992847442627f));
    return mul2(p, make_float2(__int_as_float((__float_as_int(t.x) << 23) + 0x3F800000), __int_as_float((__float_as_int(t.y) << 23) + 0x3F800000)));
}

// ---- pairs of blocks ---------------------------------------------------------------------------------------------------
// Two blocks of a cluster on neighbouring multiprocessors compute one product of 256 rows: each holds its own 128 rows of A and of
// the accumulator and half of B's columns; the first one issues the products, which read both blocks' shared memory at the
// same offsets.  Loads of both blocks are counted on the first one's barrier.
__device__ __forceinline__ uint32_t cluster_rank()
{
    uint32_t r;
    asm volatile("mov.u32 %0, %%cluster_ctarank;" : "=r"(r));
    return r;
}
__device__ __forceinline__ void cluster_sync()
{
    asm volatile("barrier.cluster.arrive.release.aligned;\nbarrier.cluster.wait.acquire.aligned;" ::: "memory");
}
// The address, in the cluster's window, of the same place in block `rank`.
__device__ __forceinline__ uint32_t in_block(const void* p, uint32_t rank)
{
    uint32_t r;
    asm volatile("mapa.shared::cluster.u32 %0, %1, %2;" : "=r"(r) : "r"(smem_addr(p)), "r"(rank));
    return r;
}
__device__ __forceinline__ void warp_arrive_in(uint32_t cluster_bar)
{
    __syncwarp();
    if ((threadIdx.x & 31) == 0) asm volatile("mbarrier.arrive.release.cluster.shared::cluster.b64 _, [%0];" ::"r"(cluster_bar) : "memory");
}
// A tile load by one lane of a warp that runs together, elected in the same statement, with addresses that are visibly uniform (as
// for products: by a branch on the lane number a load took 150 cycles to issue).  bar: in the cluster's window; a pair's loads
// may count on the barrier of either block.
template <int CG> __device__ __forceinline__ void warp_tma3(uint32_t dst, const CUtensorMap* map, uint32_t bar, int c0, int c1, int c2)
{
    if (CG == 2)
        asm volatile("{\n.reg .pred q;\nelect.sync _|q, 0xFFFFFFFF;\n"
                     "@q cp.async.bulk.tensor.3d.shared::cluster.global.tile.mbarrier::complete_tx::bytes.cta_group::2 [%0], [%1, {%2, %3, %4}], [%5];\n}"
                     ::"r"(dst), "l"(map), "r"(c0), "r"(c1), "r"(c2), "r"(bar)
                     : "memory");
    else
        asm volatile("{\n.reg .pred q;\nelect.sync _|q, 0xFFFFFFFF;\n"
                     "@q cp.async.bulk.tensor.3d.shared::cluster.global.tile.mbarrier::complete_tx::bytes [%0], [%1, {%2, %3, %4}], [%5];\n}"
                     ::"r"(dst), "l"(map), "r"(c0), "r"(c1), "r"(c2), "r"(bar)
                     : "memory");
}
__device__ __forceinline__ void prefetch_map(const CUtensorMap* map) { asm volatile("prefetch.tensormap [%0];" ::"l"(map) : "memory"); }
__device__ __forceinline__ void warp_expect(uint32_t bar, uint32_t bytes)
{
    asm volatile("{\n.reg .pred q;\nelect.sync _|q, 0xFFFFFFFF;\n@q mbarrier.arrive.expect_tx.shared::cta.b64 _, [%0], %1;\n}" ::"r"(bar), "r"(bytes)
                 : "memory");
}
// cols: a power of two from 32 to 512; by one warp of each block
template <int CG> __device__ __forceinline__ void tmem_alloc_cols(uint32_t* slot, uint32_t cols)
{
    if (CG == 2) {
        asm volatile("tcgen05.alloc.cta_group::2.sync.aligned.shared::cta.b32 [%0], %1;" ::"r"(smem_addr(slot)), "r"(cols) : "memory");
        asm volatile("tcgen05.relinquish_alloc_permit.cta_group::2.sync.aligned;" ::: "memory");
    } else {
        asm volatile("tcgen05.alloc.cta_group::1.sync.aligned.shared::cta.b32 [%0], %1;" ::"r"(smem_addr(slot)), "r"(cols) : "memory");
        asm volatile("tcgen05.relinquish_alloc_permit.cta_group::1.sync.aligned;" ::: "memory");
    }
}
template <int CG> __device__ __forceinline__ void tmem_free_cols(uint32_t addr, uint32_t cols)
{
    if (CG == 2) asm volatile("tcgen05.dealloc.cta_group::2.sync.aligned.b32 %0, %1;" ::"r"(addr), "r"(cols) : "memory");
    else asm volatile("tcgen05.dealloc.cta_group::1.sync.aligned.b32 %0, %1;" ::"r"(addr), "r"(cols) : "memory");
}
// Four products along the summed dimension, 16 each, descriptors `a_step` and `b_step` apart, and their commit to `bar` (of both
// blocks of a pair): one statement, one election (apart, an election each, they cost 330 cycles a stage to issue).
template <int CG>
__device__ __forceinline__ void mma4_commit(uint32_t d, uint64_t a, uint64_t b, uint32_t a_step, uint32_t b_step, uint32_t idesc, uint32_t acc, uint64_t* bar)
{
#define DBLP_MMA4(CGS, COMMIT)                                                                                                   \
    asm volatile("{\n.reg .pred p, q, t;\n.reg .b64 a, b, x, y;\n.reg .b16 m;\nmov.b16 m, 3;\ncvt.u64.u32 x, %3;\ncvt.u64.u32 y, %4;\n" \
                 "setp.ne.b32 p, %6, 0;\nsetp.eq.b32 t, %6, %6;\nelect.sync _|q, 0xFFFFFFFF;\n"                                   \
                 "@q tcgen05.mma.cta_group::" CGS ".kind::f16 [%0], %1, %2, %5, p;\nadd.u64 a, %1, x;\nadd.u64 b, %2, y;\n"      \
                 "@q tcgen05.mma.cta_group::" CGS ".kind::f16 [%0], a, b, %5, t;\nadd.u64 a, a, x;\nadd.u64 b, b, y;\n"          \
                 "@q tcgen05.mma.cta_group::" CGS ".kind::f16 [%0], a, b, %5, t;\nadd.u64 a, a, x;\nadd.u64 b, b, y;\n"          \
                 "@q tcgen05.mma.cta_group::" CGS ".kind::f16 [%0], a, b, %5, t;\n"                                               \
                 "@q tcgen05.commit.cta_group::" CGS ".mbarrier::arrive::one.shared::cluster" COMMIT ";\n}" ::"r"(d),            \
                 "l"(a), "l"(b), "r"(a_step), "r"(b_step), "r"(idesc), "r"(acc), "r"(smem_addr(bar))                               \
                 : "memory")
    if (CG == 2) DBLP_MMA4("2", ".multicast::cluster.b64 [%7], m");
    else DBLP_MMA4("1", ".b64 [%7]");
#undef DBLP_MMA4
}
// As mma_commit; a pair's arrives on the barriers of both blocks.
template <int CG> __device__ __forceinline__ void commit_cg(uint64_t* bar)
{
    if (CG == 2)
        asm volatile("{\n.reg .pred q;\n.reg .b16 m;\nmov.b16 m, 3;\nelect.sync _|q, 0xFFFFFFFF;\n"
                     "@q tcgen05.commit.cta_group::2.mbarrier::arrive::one.shared::cluster.multicast::cluster.b64 [%0], m;\n}" ::"r"(smem_addr(bar))
                     : "memory");
    else
        mma_commit(bar);
}
// On the issuing block's barrier alone.
template <int CG> __device__ __forceinline__ void mma_commit_idle(uint64_t* bar)
{
    if (CG == 2)
        asm volatile("{\n.reg .pred q;\nelect.sync _|q, 0xFFFFFFFF;\n"
                     "@q tcgen05.commit.cta_group::2.mbarrier::arrive::one.shared::cluster.b64 [%0];\n}" ::"r"(in_block(bar, 0))
                     : "memory");
    else
        mma_commit(bar);
}

// ---- host side ---------------------------------------------------------------------------------------------------------
// Lets kernel K use `bytes` of shared memory on the current device; asked of the runtime once per kernel and device.
template <auto K> inline cudaError_t allow_shared(int bytes)
{
    static std::atomic<unsigned long long> done{0};
    int dev = 0;
    cudaError_t e = cudaGetDevice(&dev);
    if (e != cudaSuccess) return e;
    if (dev < 64 && (done.load(std::memory_order_acquire) >> dev & 1)) return cudaSuccess;
    e = cudaFuncSetAttribute(K, cudaFuncAttributeMaxDynamicSharedMemorySize, bytes);
    if (e == cudaSuccess && dev < 64) done.fetch_or(1ull << dev, std::memory_order_acq_rel);
    return e;
}

unsigned long long* timeout_counter();     // of the current device; null after a CUDA error

// The driver's encoder of tensor maps, looked up through the runtime (the library does not link the driver); null if missing.
using EncodeTiled = CUresult (*)(CUtensorMap*, CUtensorMapDataType, cuuint32_t, void*, const cuuint64_t*, const cuuint64_t*,
                                 const cuuint32_t*, const cuuint32_t*, CUtensorMapInterleave, CUtensorMapSwizzle,
                                 CUtensorMapL2promotion, CUtensorMapFloatOOBfill);
EncodeTiled map_encoder();

}  // namespace dblp
