// The instructions of the attention kernels: mbarriers with bounded waits, tensor copies (TMA), and fifth-generation
// tensor core products (tcgen05) with their memory (TMEM).
#pragma once
#include <cuda.h>
#include <cuda_fp16.h>
#include <stdint.h>

namespace bload {
namespace tc {

__device__ __forceinline__ uint32_t smem_of(const void* p) { return (uint32_t)__cvta_generic_to_shared(p); }

// ---- mbarriers ----------------------------------------------------------------------------------------------------
__device__ __forceinline__ void bar_init(uint32_t bar, uint32_t count)
{
    asm volatile("mbarrier.init.shared::cta.b64 [%0], %1;" ::"r"(bar), "r"(count) : "memory");
}
__device__ __forceinline__ void bar_init_done()
{
    asm volatile("fence.mbarrier_init.release.cluster;" ::: "memory");
}
__device__ __forceinline__ void bar_inval(uint32_t bar)  // its place may be used again
{
    asm volatile("mbarrier.inval.shared::cta.b64 [%0];" ::"r"(bar) : "memory");
}
__device__ __forceinline__ void bar_expect(uint32_t bar, uint32_t bytes)
{
    asm volatile("mbarrier.arrive.expect_tx.shared::cta.b64 _, [%0], %1;" ::"r"(bar), "r"(bytes) : "memory");
}
__device__ __forceinline__ void bar_arrive(uint32_t bar)
{
    asm volatile("mbarrier.arrive.shared::cta.b64 _, [%0];" ::"r"(bar) : "memory");
}
// Waits until the phase with this parity has completed.  Everything these kernels wait for is a copy, a product or a
// stretch of arithmetic of the same CTA, microseconds away; four seconds are never reached unless the hardware fails, and
// then the caller gives up.
__device__ __forceinline__ uint64_t nanoseconds()
{
    uint64_t t;
    asm volatile("mov.u64 %0, %globaltimer;" : "=l"(t));
    return t;
}
__device__ __forceinline__ bool bar_wait(uint32_t bar, uint32_t parity)
{
    uint64_t since = 0;
    for (uint32_t i = 0; i < (1u << 30); ++i) {
        uint32_t done;
        asm volatile(
            "{\n\t.reg .pred p;\n\tmbarrier.try_wait.parity.shared::cta.b64 p, [%1], %2;\n\tselp.u32 %0, 1, 0, p;\n\t}"
            : "=r"(done)
            : "r"(bar), "r"(parity)
            : "memory");
        if (done) return true;
        if ((i & 1023) == 1023) {
            const uint64_t now = nanoseconds();
            if (since == 0) since = now;
            if (now - since > 4000000000ull) break;
        }
    }
    return false;
}

// ---- tensor copies ------------------------------------------------------------------------------------------------
__device__ __forceinline__ void tensor_load(uint32_t dst, const CUtensorMap* map, int x, int row, int head, int block, uint32_t bar)
{
    asm volatile(
        "cp.async.bulk.tensor.4d.shared::cta.global.tile.mbarrier::complete_tx::bytes [%0], [%1, {%2, %3, %4, %5}], [%6];"
        ::"r"(dst), "l"(map), "r"(x), "r"(row), "r"(head), "r"(block), "r"(bar)
        : "memory");
}
__device__ __forceinline__ void tensor_store(const CUtensorMap* map, int x, int row, int head, int block, uint32_t src)
{
    asm volatile("cp.async.bulk.tensor.4d.global.shared::cta.tile.bulk_group [%0, {%1, %2, %3, %4}], [%5];" ::"l"(map), "r"(x),
                 "r"(row), "r"(head), "r"(block), "r"(src)
                 : "memory");
}
__device__ __forceinline__ void stores_read()  // the sources of this thread's stores may be reused, or the CTA may end
{
    asm volatile("cp.async.bulk.commit_group;\n\tcp.async.bulk.wait_group.read 0;" ::: "memory");
}
// Writes of this thread to shared memory become visible to copies and tensor cores.
__device__ __forceinline__ void writes_to_async() { asm volatile("fence.proxy.async.shared::cta;" ::: "memory"); }

// ---- tensor memory ------------------------------------------------------------------------------------------------
template <int COLUMNS>
__device__ __forceinline__ void tmem_alloc(uint32_t where)  // a whole warp; the address is written to shared memory
{
    asm volatile("tcgen05.alloc.cta_group::1.sync.aligned.shared::cta.b32 [%0], %1;" ::"r"(where), "n"(COLUMNS) : "memory");
    asm volatile("tcgen05.relinquish_alloc_permit.cta_group::1.sync.aligned;");
}
template <int COLUMNS>
__device__ __forceinline__ void tmem_free(uint32_t tmem)
{
    asm volatile("tcgen05.dealloc.cta_group::1.sync.aligned.b32 %0, %1;" ::"r"(tmem), "n"(COLUMNS));
}
__device__ __forceinline__ void fence_before() { asm volatile("tcgen05.fence::before_thread_sync;" ::: "memory"); }
__device__ __forceinline__ void fence_after() { asm volatile("tcgen05.fence::after_thread_sync;" ::: "memory"); }

// 32 columns of the warp's 32 lanes: lane l of the warp gets row l, one column per register
__device__ __forceinline__ void tmem_load(uint32_t (&r)[32], uint32_t at)
{
    asm volatile(
        "tcgen05.ld.sync.aligned.32x32b.x32.b32 {%0, %1, %2, %3, %4, %5, %6, %7, %8, %9, %10, %11, %12, %13, %14, %15, %16, "
        "%17, %18, %19, %20, %21, %22, %23, %24, %25, %26, %27, %28, %29, %30, %31}, [%32];"
        : "=r"(r[0]), "=r"(r[1]), "=r"(r[2]), "=r"(r[3]), "=r"(r[4]), "=r"(r[5]), "=r"(r[6]), "=r"(r[7]), "=r"(r[8]), "=r"(r[9]),
          "=r"(r[10]), "=r"(r[11]), "=r"(r[12]), "=r"(r[13]), "=r"(r[14]), "=r"(r[15]), "=r"(r[16]), "=r"(r[17]), "=r"(r[18]),
          "=r"(r[19]), "=r"(r[20]), "=r"(r[21]), "=r"(r[22]), "=r"(r[23]), "=r"(r[24]), "=r"(r[25]), "=r"(r[26]), "=r"(r[27]),
          "=r"(r[28]), "=r"(r[29]), "=r"(r[30]), "=r"(r[31])
        : "r"(at));
}
__device__ __forceinline__ uint32_t tmem_load1(uint32_t at)  // one column
{
    uint32_t r;
    asm volatile("tcgen05.ld.sync.aligned.32x32b.x1.b32 {%0}, [%1];" : "=r"(r) : "r"(at));
    return r;
}
__device__ __forceinline__ void tmem_load(uint32_t (&r)[16], uint32_t at)
{
    asm volatile(
        "tcgen05.ld.sync.aligned.32x32b.x16.b32 {%0, %1, %2, %3, %4, %5, %6, %7, %8, %9, %10, %11, %12, %13, %14, %15}, [%16];"
        : "=r"(r[0]), "=r"(r[1]), "=r"(r[2]), "=r"(r[3]), "=r"(r[4]), "=r"(r[5]), "=r"(r[6]), "=r"(r[7]), "=r"(r[8]), "=r"(r[9]),
          "=r"(r[10]), "=r"(r[11]), "=r"(r[12]), "=r"(r[13]), "=r"(r[14]), "=r"(r[15])
        : "r"(at));
}
__device__ __forceinline__ void tmem_store(uint32_t at, const uint32_t (&r)[32])
{
    asm volatile(
        "tcgen05.st.sync.aligned.32x32b.x32.b32 [%0], {%1, %2, %3, %4, %5, %6, %7, %8, %9, %10, %11, %12, %13, %14, %15, %16, "
        "%17, %18, %19, %20, %21, %22, %23, %24, %25, %26, %27, %28, %29, %30, %31, %32};"
        ::"r"(at), "r"(r[0]), "r"(r[1]), "r"(r[2]), "r"(r[3]), "r"(r[4]), "r"(r[5]), "r"(r[6]), "r"(r[7]), "r"(r[8]), "r"(r[9]),
          "r"(r[10]), "r"(r[11]), "r"(r[12]), "r"(r[13]), "r"(r[14]), "r"(r[15]), "r"(r[16]), "r"(r[17]), "r"(r[18]), "r"(r[19]),
          "r"(r[20]), "r"(r[21]), "r"(r[22]), "r"(r[23]), "r"(r[24]), "r"(r[25]), "r"(r[26]), "r"(r[27]), "r"(r[28]), "r"(r[29]),
          "r"(r[30]), "r"(r[31])
        : "memory");
}
__device__ __forceinline__ void tmem_store16(uint32_t at, const uint32_t (&r)[16])
{
    asm volatile(
        "tcgen05.st.sync.aligned.32x32b.x16.b32 [%0], {%1, %2, %3, %4, %5, %6, %7, %8, %9, %10, %11, %12, %13, %14, %15, %16};"
        ::"r"(at), "r"(r[0]), "r"(r[1]), "r"(r[2]), "r"(r[3]), "r"(r[4]), "r"(r[5]), "r"(r[6]), "r"(r[7]), "r"(r[8]), "r"(r[9]),
          "r"(r[10]), "r"(r[11]), "r"(r[12]), "r"(r[13]), "r"(r[14]), "r"(r[15])
        : "memory");
}
__device__ __forceinline__ void tmem_loaded() { asm volatile("tcgen05.wait::ld.sync.aligned;" ::: "memory"); }
// (ties the registers to this place: no use of them moves in front of tmem_loaded)
__device__ __forceinline__ void settle(uint32_t (&r)[32])
{
    asm volatile("" : "+r"(r[0]), "+r"(r[1]), "+r"(r[2]), "+r"(r[3]), "+r"(r[4]), "+r"(r[5]), "+r"(r[6]), "+r"(r[7]),
                 "+r"(r[8]), "+r"(r[9]), "+r"(r[10]), "+r"(r[11]), "+r"(r[12]), "+r"(r[13]), "+r"(r[14]), "+r"(r[15]), "+r"(r[16]),
                 "+r"(r[17]), "+r"(r[18]), "+r"(r[19]), "+r"(r[20]), "+r"(r[21]), "+r"(r[22]), "+r"(r[23]), "+r"(r[24]), "+r"(r[25]),
                 "+r"(r[26]), "+r"(r[27]), "+r"(r[28]), "+r"(r[29]), "+r"(r[30]), "+r"(r[31]));
}
__device__ __forceinline__ void settle(uint32_t& r) { asm volatile("" : "+r"(r)); }
__device__ __forceinline__ void settle(uint32_t (&r)[16])
{
    asm volatile("" : "+r"(r[0]), "+r"(r[1]), "+r"(r[2]), "+r"(r[3]), "+r"(r[4]), "+r"(r[5]), "+r"(r[6]), "+r"(r[7]),
                 "+r"(r[8]), "+r"(r[9]), "+r"(r[10]), "+r"(r[11]), "+r"(r[12]), "+r"(r[13]), "+r"(r[14]), "+r"(r[15]));
}
__device__ __forceinline__ void tmem_stored() { asm volatile("tcgen05.wait::st.sync.aligned;" ::: "memory"); }

// ---- products -----------------------------------------------------------------------------------------------------
// Tiles in shared memory are rows of 64 elements of 16 bits (128 bytes), 128-byte swizzle, as a tensor copy writes them; a
// head of 128 elements is two such tiles, one behind the other.
//
// Operand whose rows run along the product's sum (K-major): groups of 8 rows are 1,024 bytes apart.
__device__ __forceinline__ uint64_t rows_desc(uint32_t at)
{
    return (uint64_t)((at & 0x3ffff) >> 4) | ((uint64_t)1 << 16) | ((uint64_t)(1024 >> 4) << 32) | ((uint64_t)1 << 46) | ((uint64_t)2 << 61);
}
// Operand whose rows are the sum (the same tile, read across): 64 elements along a row, the next 64 in the tile `next` bytes
// behind, groups of 8 rows 1,024 bytes apart.
__device__ __forceinline__ uint64_t across_desc(uint32_t at, uint32_t next)
{
    return (uint64_t)((at & 0x3ffff) >> 4) | ((uint64_t)(next >> 4) << 16) | ((uint64_t)(1024 >> 4) << 32) | ((uint64_t)1 << 46) |
           ((uint64_t)2 << 61);
}
// 16-bit operands of one type, sums in 32 bits, M = 128
template <bool BF16, int N, bool ACROSS>
__host__ __device__ constexpr uint32_t product_shape()
{
    return (1u << 4) | ((BF16 ? 1u : 0u) << 7) | ((BF16 ? 1u : 0u) << 10) | ((ACROSS ? 1u : 0u) << 16) | ((uint32_t)(N >> 3) << 17) |
           ((128u >> 4) << 24);
}
// Products are issued by one thread, but written for a whole converged warp with `leader` set in one lane: descriptors are then
// uniform values, and a product takes some 20 cycles to issue instead of the 57 it takes from a branch of a single lane (eight
// of 128 x 64 x 16 then took longer to issue than to run).
__device__ __forceinline__ uint32_t elect()
{
    uint32_t leader;
    asm volatile("{\n\t.reg .pred p;\n\telect.sync _|p, 0xffffffff;\n\tselp.u32 %0, 1, 0, p;\n\t}" : "=r"(leader));
    return leader;
}
__device__ __forceinline__ void product(uint32_t leader, uint32_t d, uint64_t a, uint64_t b, uint32_t shape, bool add)
{
    asm volatile(
        "{\n\t.reg .pred p, q;\n\tsetp.ne.u32 p, %4, 0;\n\tsetp.ne.u32 q, %5, 0;\n\t"
        "@q tcgen05.mma.cta_group::1.kind::f16 [%0], %1, %2, %3, p;\n\t}" ::"r"(d),
        "l"(a), "l"(b), "r"(shape), "r"((uint32_t)add), "r"(leader)
        : "memory");
}
__device__ __forceinline__ void product_tmem(uint32_t leader, uint32_t d, uint32_t a, uint64_t b, uint32_t shape, bool add)
{
    asm volatile(
        "{\n\t.reg .pred p, q;\n\tsetp.ne.u32 p, %4, 0;\n\tsetp.ne.u32 q, %5, 0;\n\t"
        "@q tcgen05.mma.cta_group::1.kind::f16 [%0], [%1], %2, %3, p;\n\t}" ::"r"(d),
        "r"(a), "l"(b), "r"(shape), "r"((uint32_t)add), "r"(leader)
        : "memory");
}
// arrives on the barrier when every product that the leader issued so far has ended
__device__ __forceinline__ void products_arrive(uint32_t leader, uint32_t bar)
{
    asm volatile("{\n\t.reg .pred q;\n\tsetp.ne.u32 q, %1, 0;\n\t"
                 "@q tcgen05.commit.cta_group::1.mbarrier::arrive::one.shared::cluster.b64 [%0];\n\t}" ::"r"(bar), "r"(leader)
                 : "memory");
}

// D[128, N] (+)= A[128, DP] B[N, DP]^T, both tiles in shared memory
template <bool BF16, int N, int DP>
__device__ __forceinline__ void product_rows(uint32_t leader, uint32_t d, uint32_t a, uint32_t b)
{
#pragma unroll
    for (int k = 0; k < DP / 16; ++k)
        product(leader, d, rows_desc(a + (k / 4) * (128 * 128) + (k % 4) * 32), rows_desc(b + (k / 4) * (N * 128) + (k % 4) * 32),
                product_shape<BF16, N, false>(), k > 0);
}
// D[128, DP] (+)= A[128, K] B[K, DP]: B's K rows in shared memory; A in tensor memory, two elements per column, PIECE elements
// at the start of every PIECE columns (each piece over the scores it was made from)
template <bool BF16, int K, int DP, int PIECE>
__device__ __forceinline__ void product_across(uint32_t leader, uint32_t d, uint32_t a, uint32_t b, bool add)
{
    constexpr int kSteps = PIECE / 16;
#pragma unroll
    for (int k = 0; k < K / 16; ++k)
        product_tmem(leader, d, a + (k / kSteps) * PIECE + (k % kSteps) * 8, across_desc(b + k * (16 * 128), K * 128),
                     product_shape<BF16, DP, true>(), add || k > 0);
}

// ---- arithmetic ---------------------------------------------------------------------------------------------------
__device__ __forceinline__ float exp2_fast(float x)  // 2 units in the last place; 0 below 2^-126
{
    float y;
    asm("ex2.approx.ftz.f32 %0, %1;" : "=f"(y) : "f"(x));
    return y;
}
__device__ __forceinline__ float inverse_fast(float x)
{
    float y;
    asm("rcp.approx.ftz.f32 %0, %1;" : "=f"(y) : "f"(x));
    return y;
}
__device__ __forceinline__ float largest(float a, float b, float c)  // of the magnitudes
{
    float r;
    asm("max.abs.f32 %0, %1, %2, %3;" : "=f"(r) : "f"(a), "f"(b), "f"(c));
    return r;
}
// of the magnitudes of two pairs in fp16, each
__device__ __forceinline__ uint32_t largest_halves(uint32_t a, uint32_t b)
{
    const __half2 m = __hmax2(__habs2(*reinterpret_cast<const __half2*>(&a)), __habs2(*reinterpret_cast<const __half2*>(&b)));
    return *reinterpret_cast<const uint32_t*>(&m);
}
__device__ __forceinline__ float largest_of_halves(const uint4& x)  // the largest magnitude of eight in fp16
{
    const uint32_t m = largest_halves(largest_halves(x.x, x.y), largest_halves(x.z, x.w));
    const float2 f = __half22float2(*reinterpret_cast<const __half2*>(&m));
    return fmaxf(f.x, f.y);
}
// lo in the lower half
template <bool BF16>
__device__ __forceinline__ uint32_t pack(float lo, float hi)
{
    uint32_t r;
    if (BF16)
        asm("cvt.rn.bf16x2.f32 %0, %1, %2;" : "=r"(r) : "f"(hi), "f"(lo));
    else
        asm("cvt.rn.f16x2.f32 %0, %1, %2;" : "=r"(r) : "f"(hi), "f"(lo));
    return r;
}
// acc + 0 * (both elements of x): stays 0 while everything is finite, NaN after an infinity or NaN
template <bool BF16>
__device__ __forceinline__ uint32_t probe(uint32_t acc, uint32_t x)
{
    uint32_t r;
    if (BF16)
        asm("fma.rn.bf16x2 %0, %1, %2, %3;" : "=r"(r) : "r"(x), "r"(0u), "r"(acc));
    else
        asm("fma.rn.f16x2 %0, %1, %2, %3;" : "=r"(r) : "r"(x), "r"(0u), "r"(acc));
    return r;
}

}  // namespace tc
}  // namespace bload
