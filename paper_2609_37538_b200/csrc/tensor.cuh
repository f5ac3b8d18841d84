// Blackwell's matrix unit, its memory (TMEM) and the barriers that order them, as inline PTX for sm_100a.
#pragma once
#include <stdint.h>

namespace avsg {

__device__ __forceinline__ uint32_t shared_address(const void* p) { return (uint32_t)__cvta_generic_to_shared(p); }

// ---- barriers in shared memory ---------------------------------------------------------------------------------------
__device__ __forceinline__ void barrier_init(uint32_t bar, uint32_t arrivals)
{
    asm volatile("mbarrier.init.shared::cta.b64 [%0], %1;" :: "r"(bar), "r"(arrivals) : "memory");
}
__device__ __forceinline__ void barrier_arrive(uint32_t bar)
{
    asm volatile("mbarrier.arrive.shared::cta.b64 _, [%0];" :: "r"(bar) : "memory");
}
// With a pause in it while the phase lasts: many warps looking all the time take shared memory's bandwidth from the matrix unit (sixteen of
// them doubled the time of its products).
__device__ __forceinline__ bool barrier_wait(uint32_t bar, uint32_t parity)
{
    uint32_t done;
    asm volatile("{\n\t.reg .pred p;\n\tmbarrier.try_wait.parity.shared::cta.b64 p, [%1], %2;\n\tselp.u32 %0, 1, 0, p;\n\t}"
                 : "=r"(done) : "r"(bar), "r"(parity) : "memory");
    return done;
}
__device__ __forceinline__ bool barrier_done(uint32_t bar, uint32_t parity)
{
    uint32_t done;
    asm volatile("{\n\t.reg .pred p;\n\tmbarrier.test_wait.parity.shared::cta.b64 p, [%1], %2;\n\tselp.u32 %0, 1, 0, p;\n\t}"
                 : "=r"(done) : "r"(bar), "r"(parity) : "memory");
    return done;
}
// One lane of a converged warp.
__device__ __forceinline__ bool one_lane()
{
    uint32_t p;
    asm volatile("{\n\t.reg .pred p;\n\telect.sync _|p, 0xffffffff;\n\tselp.u32 %0, 1, 0, p;\n\t}" : "=r"(p));
    return p;
}
// What is written to shared memory by ordinary stores is seen by the matrix unit behind this and a barrier.
__device__ __forceinline__ void fence_for_matrix_unit() { asm volatile("fence.proxy.async.shared::cta;" ::: "memory"); }

// ---- TMEM --------------------------------------------------------------------------------------------------------------
// (a warp allocates and frees; its address goes to shared memory)
__device__ __forceinline__ void tmem_alloc(uint32_t to, uint32_t columns)
{
    asm volatile("tcgen05.alloc.cta_group::1.sync.aligned.shared::cta.b32 [%0], %1;" :: "r"(to), "r"(columns) : "memory");
    asm volatile("tcgen05.relinquish_alloc_permit.cta_group::1.sync.aligned;" ::: "memory");
}
__device__ __forceinline__ void tmem_free(uint32_t at, uint32_t columns)
{
    asm volatile("tcgen05.dealloc.cta_group::1.sync.aligned.b32 %0, %1;" :: "r"(at), "r"(columns) : "memory");
}
__device__ __forceinline__ void tmem_before_sync() { asm volatile("tcgen05.fence::before_thread_sync;" ::: "memory"); }
__device__ __forceinline__ void tmem_after_sync() { asm volatile("tcgen05.fence::after_thread_sync;" ::: "memory"); }
__device__ __forceinline__ void tmem_loaded() { asm volatile("tcgen05.wait::ld.sync.aligned;" ::: "memory"); }
__device__ __forceinline__ void tmem_stored() { asm volatile("tcgen05.wait::st.sync.aligned;" ::: "memory"); }

// 16 lanes x 32 columns (or 16) of 32 bits, spread over the warp: x[4 g + i] is row lane / 4 + 8 (i / 2), column 8 g + 2 (lane % 4) + i % 2.
__device__ __forceinline__ void tmem_load_scores(uint32_t at, float (&x)[8])
{
    uint32_t* r = reinterpret_cast<uint32_t*>(x);
    asm volatile("tcgen05.ld.sync.aligned.16x256b.x2.b32 {%0, %1, %2, %3, %4, %5, %6, %7}, [%8];"
                 : "=r"(r[0]), "=r"(r[1]), "=r"(r[2]), "=r"(r[3]), "=r"(r[4]), "=r"(r[5]), "=r"(r[6]), "=r"(r[7]) : "r"(at));
}
__device__ __forceinline__ void tmem_load_scores(uint32_t at, float (&x)[16])
{
    uint32_t* r = reinterpret_cast<uint32_t*>(x);
    asm volatile("tcgen05.ld.sync.aligned.16x256b.x4.b32 {%0, %1, %2, %3, %4, %5, %6, %7, %8, %9, %10, %11, %12, %13, %14, %15}, [%16];"
                 : "=r"(r[0]), "=r"(r[1]), "=r"(r[2]), "=r"(r[3]), "=r"(r[4]), "=r"(r[5]), "=r"(r[6]), "=r"(r[7]), "=r"(r[8]), "=r"(r[9]),
                   "=r"(r[10]), "=r"(r[11]), "=r"(r[12]), "=r"(r[13]), "=r"(r[14]), "=r"(r[15])
                 : "r"(at));
}
// 32 lanes x 16 columns: thread i has lane i.
__device__ __forceinline__ void tmem_load_32x16(uint32_t at, float (&x)[16])
{
    uint32_t* r = reinterpret_cast<uint32_t*>(x);
    asm volatile("tcgen05.ld.sync.aligned.32x32b.x16.b32 {%0, %1, %2, %3, %4, %5, %6, %7, %8, %9, %10, %11, %12, %13, %14, %15}, [%16];"
                 : "=r"(r[0]), "=r"(r[1]), "=r"(r[2]), "=r"(r[3]), "=r"(r[4]), "=r"(r[5]), "=r"(r[6]), "=r"(r[7]), "=r"(r[8]), "=r"(r[9]),
                   "=r"(r[10]), "=r"(r[11]), "=r"(r[12]), "=r"(r[13]), "=r"(r[14]), "=r"(r[15])
                 : "r"(at));
}
__device__ __forceinline__ void tmem_store_32x16(uint32_t at, const float (&x)[16])
{
    const uint32_t* r = reinterpret_cast<const uint32_t*>(x);
    asm volatile("tcgen05.st.sync.aligned.32x32b.x16.b32 [%0], {%1, %2, %3, %4, %5, %6, %7, %8, %9, %10, %11, %12, %13, %14, %15, %16};"
                 :: "r"(at), "r"(r[0]), "r"(r[1]), "r"(r[2]), "r"(r[3]), "r"(r[4]), "r"(r[5]), "r"(r[6]), "r"(r[7]), "r"(r[8]), "r"(r[9]),
                    "r"(r[10]), "r"(r[11]), "r"(r[12]), "r"(r[13]), "r"(r[14]), "r"(r[15]) : "memory");
}

// ---- products ------------------------------------------------------------------------------------------------------------
// Operands lie in shared memory in pieces of 8 lines of 128 bytes, 1024-byte aligned, whose 16-byte units are swizzled: unit u of line
// i is at u ^ (i & 7).  Lines run along the sum, one for each row of the operand; or along rows, 64 (16-bit ones) of them, the next 64
// being `next` bytes further on, one for each step of the sum.  The next 8 lines are 1024 bytes further on.
// An operand is its low word, to which (bytes / 16) may be added, and OPERAND_HIGH.
__device__ __forceinline__ uint32_t operand(uint32_t at, uint32_t next) { return (at & 0x3FFFFu) >> 4 | (next >> 4) << 16; }
constexpr uint32_t OPERAND_HIGH = 1024u >> 4 | 1u << 14 | 2u << 29;
// Both operands' type; sums are in 32 bits.
enum class Product { FP16, BF16, E4M3 };
__host__ __device__ constexpr uint32_t product_shape(Product type, uint32_t m, uint32_t n, bool a_along_rows)
{
    return 1u << 4 | (type == Product::BF16 ? 1u << 7 | 1u << 10 : 0u) | (a_along_rows ? 1u : 0u) << 15 | (n >> 3) << 17 | (m >> 4) << 24;
}
// 16 steps of the sum (32 for e4m3): 32 bytes of lines along it, or so many lines.  Sums at TMEM address `to`, added to what is there
// if add.  One thread issues; see products_done().
template <Product TYPE>
__device__ __forceinline__ void multiply(uint32_t to, uint32_t a, uint32_t b, uint32_t shape, bool add)
{
    if constexpr (TYPE == Product::E4M3)
        asm volatile("{\n\t.reg .pred p;\n\t.reg .b64 a, b;\n\tsetp.ne.b32 p, %4, 0;\n\tmov.b64 a, {%1, %5};\n\tmov.b64 b, {%2, %5};\n\t"
                     "tcgen05.mma.cta_group::1.kind::f8f6f4 [%0], a, b, %3, p;\n\t}"
                     :: "r"(to), "r"(a), "r"(b), "r"(shape), "r"((uint32_t)add), "r"(OPERAND_HIGH) : "memory");
    else
        asm volatile("{\n\t.reg .pred p;\n\t.reg .b64 a, b;\n\tsetp.ne.b32 p, %4, 0;\n\tmov.b64 a, {%1, %5};\n\tmov.b64 b, {%2, %5};\n\t"
                     "tcgen05.mma.cta_group::1.kind::f16 [%0], a, b, %3, p;\n\t}"
                     :: "r"(to), "r"(a), "r"(b), "r"(shape), "r"((uint32_t)add), "r"(OPERAND_HIGH) : "memory");
}
// The barrier gets an arrival when all products issued by this thread so far are through.
__device__ __forceinline__ void products_done(uint32_t bar)
{
    asm volatile("tcgen05.commit.cta_group::1.mbarrier::arrive::one.shared::cluster.b64 [%0];" :: "r"(bar) : "memory");
}

// ---- copies of 16 bytes that wait in no register ---------------------------------------------------------------------------
__device__ __forceinline__ void copy16(uint32_t to, const void* from, bool zero)
{
    asm volatile("cp.async.cg.shared.global [%0], [%1], 16, %2;" :: "r"(to), "l"(from), "r"(zero ? 0u : 16u) : "memory");
}
__device__ __forceinline__ void copies_close() { asm volatile("cp.async.commit_group;" ::: "memory"); }
template <int OPEN>
__device__ __forceinline__ void copies_wait() { asm volatile("cp.async.wait_group %0;" :: "n"(OPEN) : "memory"); }

// ---- clusters --------------------------------------------------------------------------------------------------------------
__device__ __forceinline__ void cluster_sync()
{
    asm volatile("barrier.cluster.arrive.release.aligned;\n\tbarrier.cluster.wait.acquire.aligned;" ::: "memory");
}
__device__ __forceinline__ uint32_t in_block(uint32_t at, uint32_t rank)       // the same place in another block's shared memory
{
    uint32_t r;
    asm("mapa.shared::cluster.u32 %0, %1, %2;" : "=r"(r) : "r"(at), "r"(rank));
    return r;
}
__device__ __forceinline__ float4 load_float4(uint32_t at)
{
    float4 v;
    asm volatile("ld.shared::cluster.v4.f32 {%0, %1, %2, %3}, [%4];" : "=f"(v.x), "=f"(v.y), "=f"(v.z), "=f"(v.w) : "r"(at));
    return v;
}

}  // namespace avsg
