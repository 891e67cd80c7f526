// Inline PTX for the fifth-generation tensor cores: barriers in shared memory, asynchronous copies of tiles, tensor memory and the
// block-scaled product of 4-bit floats.
#pragma once
#include <cuda_runtime.h>
#include <stdint.h>

namespace conef {
namespace tc {

__device__ __forceinline__ uint32_t saddr(const void *p) { return (uint32_t)__cvta_generic_to_shared(p); }

// Copies and products are issued by the one lane that this says, of a warp whose control flow is the same for all lanes as far as the
// compiler can see (conditions by votes, counters from parameters): under a test of the lane's number, or with a loop that ends on what a lane
// found, every operand took a move to the uniform registers that the instructions read, and a product of 128 cycles took 265 to issue.
__device__ __forceinline__ bool elect()
{
    uint32_t e;
    asm volatile("{\n\t.reg .pred q;\n\telect.sync _|q, 0xffffffff;\n\tselp.u32 %0, 1, 0, q;\n\t}" : "=r"(e));
    return e != 0;
}

// ------------------------------------------------------------------ barriers
__device__ __forceinline__ void bar_init(uint64_t *bar, uint32_t count) { asm volatile("mbarrier.init.shared.b64 [%0], %1;" ::"r"(saddr(bar)), "r"(count) : "memory"); }
__device__ __forceinline__ void bar_arrive(uint64_t *bar) { asm volatile("mbarrier.arrive.shared.b64 _, [%0];" ::"r"(saddr(bar)) : "memory"); }
__device__ __forceinline__ void bar_expect(uint64_t *bar, uint32_t bytes)
{
    asm volatile("mbarrier.arrive.expect_tx.shared.b64 _, [%0], %1;" ::"r"(saddr(bar)), "r"(bytes) : "memory");
}
__device__ __forceinline__ bool bar_try(uint64_t *bar, uint32_t parity)
{
    uint32_t ok;
    asm volatile("{\n\t.reg .pred q;\n\tmbarrier.try_wait.parity.shared.b64 q, [%1], %2;\n\tselp.u32 %0, 1, 0, q;\n\t}" : "=r"(ok) : "r"(saddr(bar)), "r"(parity) : "memory");
    return ok != 0;
}
__device__ __forceinline__ uint64_t nanoseconds()
{
    uint64_t t;
    asm volatile("mov.u64 %0, %globaltimer;" : "=l"(t));
    return t;
}
// Waits are bounded.  `dead` says that one of a CTA's has run out, or one of the other CTA's of a pair: all that are not over then end.
struct Waits {
    volatile int *dead;
    uint32_t others;                // the other CTA's `dead` (a cluster address), or 0
    unsigned long long *ran_out;    // counts the CTAs in which a wait has run out
};
__device__ __forceinline__ void give_up(const Waits &w)
{
    if (atomicExch((int *)w.dead, 1) == 0)
        atomicAdd(w.ran_out, 1ull);
    if (w.others)
        asm volatile("st.shared::cluster.u32 [%0], %1;" ::"r"(w.others), "r"(1) : "memory");
}
// A warp waits for a phase, for `limit` nanoseconds or a little more; the answer is no where that runs out, or once another wait has.
__device__ __forceinline__ bool bar_wait(uint64_t *bar, uint32_t parity, const Waits &w, uint64_t limit)
{
    bool there = bar_try(bar, parity);
    if (!there) {
        const uint64_t t0 = nanoseconds();
        for (int i = 1; !there && !*w.dead; ++i) {
            there = bar_try(bar, parity);
            if (!there && i % 64 == 0 && nanoseconds() - t0 > limit)
                give_up(w);
        }
    }
    return __all_sync(0xffffffffu, there);
}
// ... for copies or products in flight that nobody will use, two seconds at most after t0, whatever *dead says
__device__ __forceinline__ void bar_drain(uint64_t *bar, uint32_t parity, uint64_t t0)
{
    while (!bar_try(bar, parity) && nanoseconds() - t0 <= 2000000000ull) {
    }
}

// ------------------------------------------------------------------ pairs of CTAs (a cluster of two; the even rank leads)
__device__ __forceinline__ void cluster_sync()
{
    asm volatile("barrier.cluster.arrive.release.aligned;" ::: "memory");
    asm volatile("barrier.cluster.wait.acquire.aligned;" ::: "memory");
}
// a variable in shared memory of either CTA, and that of the leader
__device__ __forceinline__ uint32_t address_in(const void *p, uint32_t rank)
{
    uint32_t r;
    asm volatile("mapa.shared::cluster.u32 %0, %1, %2;" : "=r"(r) : "r"(saddr(p)), "r"(rank));
    return r;
}
__device__ __forceinline__ uint32_t leaders(const void *p) { return address_in(p, 0); }
__device__ __forceinline__ uint32_t load_at(uint32_t at)
{
    uint32_t v;
    asm volatile("ld.shared::cluster.u32 %0, [%1];" : "=r"(v) : "r"(at) : "memory");
    return v;
}
__device__ __forceinline__ void bar_arrive_at(uint32_t bar) { asm volatile("mbarrier.arrive.release.cluster.shared::cluster.b64 _, [%0];" ::"r"(bar) : "memory"); }

// ------------------------------------------------------------------ asynchronous copies into shared memory
__device__ __forceinline__ void tile_load(uint32_t dst, const void *map, uint32_t x, uint32_t y, uint64_t *bar)
{
    asm volatile("cp.async.bulk.tensor.2d.shared::cta.global.tile.mbarrier::complete_tx::bytes [%0], [%1, {%2, %3}], [%4];" ::"r"(dst), "l"(map), "r"(x), "r"(y),
                 "r"(saddr(bar))
                 : "memory");
}
__device__ __forceinline__ void bulk_load(uint32_t dst, const void *src, uint32_t bytes, uint64_t *bar)
{
    asm volatile("cp.async.bulk.shared::cta.global.mbarrier::complete_tx::bytes [%0], [%1], %2, [%3];" ::"r"(dst), "l"(src), "r"(bytes), "r"(saddr(bar)) : "memory");
}
// ... of a CTA of a pair, into its own memory; the leader's barrier is told
__device__ __forceinline__ void tile_load_pair(uint32_t dst, const void *map, uint32_t x, uint32_t y, uint32_t bar)
{
    asm volatile("cp.async.bulk.tensor.2d.cta_group::2.shared::cluster.global.tile.mbarrier::complete_tx::bytes [%0], [%1, {%2, %3}], [%4];" ::"r"(dst), "l"(map), "r"(x),
                 "r"(y), "r"(bar)
                 : "memory");
}

// ... and out of it: one thread stores a tile that the warp wrote (store_fence by each writer, then a barrier), and waits until the memory
// may be written again, or until all its stores have ended
__device__ __forceinline__ void store_fence() { asm volatile("fence.proxy.async.shared::cta;" ::: "memory"); }
__device__ __forceinline__ void tile_store(const void *map, uint32_t src, uint32_t x, uint32_t y)
{
    asm volatile("cp.async.bulk.tensor.2d.global.shared::cta.tile.bulk_group [%0, {%2, %3}], [%1];" ::"l"(map), "r"(src), "r"(x), "r"(y) : "memory");
    asm volatile("cp.async.bulk.commit_group;" ::: "memory");
}
__device__ __forceinline__ void store_wait_read() { asm volatile("cp.async.bulk.wait_group.read 0;" ::: "memory"); }
__device__ __forceinline__ void store_wait() { asm volatile("cp.async.bulk.wait_group 0;" ::: "memory"); }

// ------------------------------------------------------------------ tensor memory (PAIR: by both CTAs)
template <bool PAIR>
__device__ __forceinline__ void tmem_alloc(uint32_t *where, uint32_t columns)   // a whole warp
{
    if constexpr (PAIR) {
        asm volatile("tcgen05.alloc.cta_group::2.sync.aligned.shared::cta.b32 [%0], %1;" ::"r"(saddr(where)), "r"(columns) : "memory");
        asm volatile("tcgen05.relinquish_alloc_permit.cta_group::2.sync.aligned;" ::: "memory");
    } else {
        asm volatile("tcgen05.alloc.cta_group::1.sync.aligned.shared::cta.b32 [%0], %1;" ::"r"(saddr(where)), "r"(columns) : "memory");
        asm volatile("tcgen05.relinquish_alloc_permit.cta_group::1.sync.aligned;" ::: "memory");
    }
}
template <bool PAIR>
__device__ __forceinline__ void tmem_free(uint32_t at, uint32_t columns)   // the same warp
{
    if constexpr (PAIR)
        asm volatile("tcgen05.dealloc.cta_group::2.sync.aligned.b32 %0, %1;" ::"r"(at), "r"(columns) : "memory");
    else
        asm volatile("tcgen05.dealloc.cta_group::1.sync.aligned.b32 %0, %1;" ::"r"(at), "r"(columns) : "memory");
}
__device__ __forceinline__ void fence_before() { asm volatile("tcgen05.fence::before_thread_sync;" ::: "memory"); }
__device__ __forceinline__ void fence_after() { asm volatile("tcgen05.fence::after_thread_sync;" ::: "memory"); }
// 32 columns of the warp's 32 lanes
__device__ __forceinline__ void tmem_load32(uint32_t at, uint32_t (&v)[32])
{
    asm volatile("tcgen05.ld.sync.aligned.32x32b.x32.b32 {%0, %1, %2, %3, %4, %5, %6, %7, %8, %9, %10, %11, %12, %13, %14, %15, %16, %17, %18, %19, %20, %21, "
                 "%22, %23, %24, %25, %26, %27, %28, %29, %30, %31}, [%32];"
                 : "=r"(v[0]), "=r"(v[1]), "=r"(v[2]), "=r"(v[3]), "=r"(v[4]), "=r"(v[5]), "=r"(v[6]), "=r"(v[7]), "=r"(v[8]), "=r"(v[9]), "=r"(v[10]),
                   "=r"(v[11]), "=r"(v[12]), "=r"(v[13]), "=r"(v[14]), "=r"(v[15]), "=r"(v[16]), "=r"(v[17]), "=r"(v[18]), "=r"(v[19]), "=r"(v[20]),
                   "=r"(v[21]), "=r"(v[22]), "=r"(v[23]), "=r"(v[24]), "=r"(v[25]), "=r"(v[26]), "=r"(v[27]), "=r"(v[28]), "=r"(v[29]), "=r"(v[30]),
                   "=r"(v[31])
                 : "r"(at));
}
__device__ __forceinline__ void tmem_load_wait() { asm volatile("tcgen05.wait::ld.sync.aligned;" ::: "memory"); }

// ------------------------------------------------------------------ products
// Low word of the descriptor of an operand in shared memory (its address in 16 bytes), and the high words: rows of 128 bytes along k, eight
// to a 1024-byte group, 16-byte pieces exchanged within a group as the tile copy with the 128-byte pattern leaves them;
// 32 rows of 16 bytes, one behind the other (a tile of scales)
__device__ __forceinline__ uint32_t desc_low(const void *p) { return ((saddr(p) & 0x3FFFFu) >> 4) | (1u << 16); }
constexpr uint32_t kDescRows128 = 64u | (1u << 14) | (2u << 29), kDescScales = 8u | (1u << 14);
// 512 bytes into four columns, the 32 rows to the lanes of each of the four warps; PAIR: by each CTA from its own shared memory
template <bool PAIR>
__device__ __forceinline__ void scales_copy(uint32_t at, uint32_t low)
{
    const uint64_t desc = (uint64_t)kDescScales << 32 | low;
    if constexpr (PAIR)
        asm volatile("tcgen05.cp.cta_group::2.32x128b.warpx4 [%0], %1;" ::"r"(at), "l"(desc) : "memory");
    else
        asm volatile("tcgen05.cp.cta_group::1.32x128b.warpx4 [%0], %1;" ::"r"(at), "l"(desc) : "memory");
}

// 4-bit floats with power-of-two scales, 128 rows of A (PAIR: of each CTA), n of B (a multiple of 16 up to 256; PAIR: half of them with each
// CTA, the scales of all with both), both along k
template <bool PAIR>
__device__ __forceinline__ uint32_t mx4_instruction(uint32_t n) { return (1u << 7) | (1u << 10) | ((n >> 3) << 17) | (1u << 23) | ((PAIR ? 16u : 8u) << 24); }
// 64 elements along k; HALF: which two of the four scales in a column's word are theirs (number 0 or 2, of B and of A)
template <bool PAIR, int HALF>
__device__ __forceinline__ void mx4_product(uint32_t d, uint32_t a, uint32_t b, uint32_t instruction, uint32_t sa, uint32_t sb, uint32_t add)
{
    const uint64_t da = (uint64_t)kDescRows128 << 32 | a, db = (uint64_t)kDescRows128 << 32 | b;
    instruction |= (uint32_t)(HALF << 5) | ((uint32_t)HALF << 30);
    if constexpr (PAIR)
        asm volatile("{\n\t.reg .pred q;\n\tsetp.ne.u32 q, %6, 0;\n\ttcgen05.mma.cta_group::2.kind::mxf4.block_scale.scale_vec::2X [%0], %1, %2, %3, [%4], [%5], q;\n\t}" ::"r"(d),
                     "l"(da), "l"(db), "r"(instruction), "r"(sa), "r"(sb), "r"(add)
                     : "memory");
    else
        asm volatile("{\n\t.reg .pred q;\n\tsetp.ne.u32 q, %6, 0;\n\ttcgen05.mma.cta_group::1.kind::mxf4.block_scale.scale_vec::2X [%0], %1, %2, %3, [%4], [%5], q;\n\t}" ::"r"(d),
                     "l"(da), "l"(db), "r"(instruction), "r"(sa), "r"(sb), "r"(add)
                     : "memory");
}
// the barrier (PAIR: that of each CTA) is told when all that this lane has issued is done
template <bool PAIR>
__device__ __forceinline__ void commit(uint64_t *bar)
{
    if constexpr (PAIR)
        asm volatile("tcgen05.commit.cta_group::2.mbarrier::arrive::one.shared::cluster.multicast::cluster.b64 [%0], %1;" ::"r"(saddr(bar)), "h"((uint16_t)3) : "memory");
    else
        asm volatile("tcgen05.commit.cta_group::1.mbarrier::arrive::one.shared::cluster.b64 [%0];" ::"r"(saddr(bar)) : "memory");
}

}  // namespace tc
}  // namespace conef
