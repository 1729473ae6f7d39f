// nfad_tcgen.cuh -- the few hardware operations that the matrix products are built from: transaction barriers with bounded
// waits, tensor copies from global to shared memory, and fifth-generation tensor-core products with their accumulators in
// tensor memory.
#pragma once

#include <cuda.h>
#include <cuda_runtime.h>
#include <stdint.h>

namespace nfad {
namespace tc {

#define NFAD_TC __device__ __forceinline__

NFAD_TC uint32_t shared_address(const void* p) { return uint32_t(__cvta_generic_to_shared(p)); }

// ---------------------------------------------------------------- barriers in shared memory

NFAD_TC void barrier_init(uint32_t bar, uint32_t count) { asm volatile("mbarrier.init.shared::cta.b64 [%0], %1;" ::"r"(bar), "r"(count) : "memory"); }
NFAD_TC void barrier_init_done() { asm volatile("fence.mbarrier_init.release.cluster;" ::: "memory"); }
NFAD_TC void barrier_arrive(uint32_t bar) { asm volatile("mbarrier.arrive.shared::cta.b64 _, [%0];" ::"r"(bar) : "memory"); }
// the first CTA of the pair's own copy of a shared-memory address
NFAD_TC uint32_t first_of_pair(uint32_t address)
{
    uint32_t r;
    asm("mapa.shared::cluster.u32 %0, %1, 0;" : "=r"(r) : "r"(address));
    return r;
}
NFAD_TC uint32_t rank_in_pair()
{
    uint32_t r;
    asm("mov.u32 %0, %%cluster_ctarank;" : "=r"(r));
    return r;
}
NFAD_TC void pair_sync()
{
    asm volatile("barrier.cluster.arrive.release.aligned;\n barrier.cluster.wait.acquire.aligned;" ::: "memory");
}
// On a barrier of the first CTA (an address from first_of_pair).  No cluster-wide release: what these arrivals stand for are
// asynchronous copies (the transaction count orders them) and tensor-memory reads (fenced on their own); a release at
// cluster scope in every step halved the rate of the products.
NFAD_TC void barrier_arrive_first(uint32_t bar) { asm volatile("mbarrier.arrive.shared::cluster.b64 _, [%0];" ::"r"(bar) : "memory"); }
NFAD_TC void barrier_expect_first(uint32_t bar, uint32_t bytes)
{
    asm volatile("mbarrier.arrive.expect_tx.shared::cluster.b64 _, [%0], %1;" ::"r"(bar), "r"(bytes) : "memory");
}
// orders plain writes of one CTA of the pair before an arrival that the other waits for
NFAD_TC void pair_fence() { asm volatile("fence.acq_rel.cluster;" ::: "memory"); }
NFAD_TC void barrier_expect(uint32_t bar, uint32_t bytes)
{
    asm volatile("mbarrier.arrive.expect_tx.shared::cta.b64 _, [%0], %1;" ::"r"(bar), "r"(bytes) : "memory");
}
// a thread that finds the phase unfinished sleeps until it is, or for about this many nanoseconds
constexpr uint32_t kSuspend = 20000;
NFAD_TC bool barrier_try(uint32_t bar, uint32_t parity)
{
    uint32_t ok;
    asm volatile("{\n .reg .pred p;\n mbarrier.try_wait.parity.shared::cta.b64 p, [%1], %2, %3;\n selp.u32 %0, 1, 0, p;\n}"
                 : "=r"(ok) : "r"(bar), "r"(parity), "r"(kSuspend) : "memory");
    return ok != 0;
}

// A wait that ends: when the barrier's phase completes (true), when another role of the CTA has given up, or after about ten
// seconds of SM cycles (false; nothing that a correct launch waits for takes a hundredth of that).
constexpr long long kWaitCycles = 20000000000ll;
constexpr long long kWaitDrain = 2000000000ll;      // what a CTA that gave up leaves its own work in flight
NFAD_TC bool barrier_wait(uint32_t bar, uint32_t parity, volatile uint32_t* gave_up)
{
    if (barrier_try(bar, parity)) return true;
    const long long t0 = clock64();
    while (!barrier_try(bar, parity)) {
        if (*gave_up) return false;
        if (clock64() - t0 > kWaitCycles) {
            *gave_up = 1;
            return false;
        }
    }
    return true;
}

// plain shared-memory writes become visible to the asynchronous copies and products that follow
NFAD_TC void writes_to_async() { asm volatile("fence.proxy.async.shared::cta;" ::: "memory"); }

// ---------------------------------------------------------------- tensor copies

NFAD_TC void prefetch_map(const CUtensorMap* m) { asm volatile("prefetch.tensormap [%0];" ::"l"(m) : "memory"); }

// kPair: `bar` may be a barrier of the first CTA of the pair
template <bool kPair> NFAD_TC void load_box(uint32_t dst, const CUtensorMap* m, uint32_t bar, int c0, int c1)
{
    if (kPair)
        asm volatile("cp.async.bulk.tensor.2d.cta_group::2.shared::cluster.global.tile.mbarrier::complete_tx::bytes [%0], [%1, {%3, %4}], [%2];"
                     ::"r"(dst), "l"(m), "r"(bar), "r"(c0), "r"(c1) : "memory");
    else
        asm volatile("cp.async.bulk.tensor.2d.shared::cta.global.tile.mbarrier::complete_tx::bytes [%0], [%1, {%3, %4}], [%2];"
                     ::"r"(dst), "l"(m), "r"(bar), "r"(c0), "r"(c1) : "memory");
}
template <bool kPair> NFAD_TC void load_box(uint32_t dst, const CUtensorMap* m, uint32_t bar, int c0, int c1, int c2)
{
    if (kPair)
        asm volatile("cp.async.bulk.tensor.3d.cta_group::2.shared::cluster.global.tile.mbarrier::complete_tx::bytes [%0], [%1, {%3, %4, %5}], [%2];"
                     ::"r"(dst), "l"(m), "r"(bar), "r"(c0), "r"(c1), "r"(c2) : "memory");
    else
        asm volatile("cp.async.bulk.tensor.3d.shared::cta.global.tile.mbarrier::complete_tx::bytes [%0], [%1, {%3, %4, %5}], [%2];"
                     ::"r"(dst), "l"(m), "r"(bar), "r"(c0), "r"(c1), "r"(c2) : "memory");
}

// `bytes` (a multiple of 16) between 16-byte boundaries, no tensor map
NFAD_TC void load_run(uint32_t dst, const void* src, uint32_t bytes, uint32_t bar)
{
    asm volatile("cp.async.bulk.shared::cta.global.mbarrier::complete_tx::bytes [%0], [%1], %2, [%3];" ::"r"(dst), "l"(src), "r"(bytes), "r"(bar) : "memory");
}

// ---------------------------------------------------------------- tensor memory and products

// kPair: the pair allocates and frees together (one warp of each CTA)
template <bool kPair> NFAD_TC void tmem_alloc(uint32_t slot, uint32_t columns)
{
    if (kPair) {
        asm volatile("tcgen05.alloc.cta_group::2.sync.aligned.shared::cta.b32 [%0], %1;" ::"r"(slot), "r"(columns) : "memory");
        asm volatile("tcgen05.relinquish_alloc_permit.cta_group::2.sync.aligned;" ::: "memory");
    } else {
        asm volatile("tcgen05.alloc.cta_group::1.sync.aligned.shared::cta.b32 [%0], %1;" ::"r"(slot), "r"(columns) : "memory");
        asm volatile("tcgen05.relinquish_alloc_permit.cta_group::1.sync.aligned;" ::: "memory");
    }
}
template <bool kPair> NFAD_TC void tmem_free(uint32_t at, uint32_t columns)
{
    if (kPair) asm volatile("tcgen05.dealloc.cta_group::2.sync.aligned.b32 %0, %1;" ::"r"(at), "r"(columns) : "memory");
    else asm volatile("tcgen05.dealloc.cta_group::1.sync.aligned.b32 %0, %1;" ::"r"(at), "r"(columns) : "memory");
}
NFAD_TC void fence_before_sync() { asm volatile("tcgen05.fence::before_thread_sync;" ::: "memory"); }
NFAD_TC void fence_after_sync() { asm volatile("tcgen05.fence::after_thread_sync;" ::: "memory"); }

// 32 accumulator columns of this warp's 32 lanes: v[i] is column i of the lane's row
NFAD_TC void tmem_load32(uint32_t at, uint32_t (&v)[32])
{
    asm volatile(
        "tcgen05.ld.sync.aligned.32x32b.x32.b32 {%0, %1, %2, %3, %4, %5, %6, %7, %8, %9, %10, %11, %12, %13, %14, %15, %16, %17, %18, "
        "%19, %20, %21, %22, %23, %24, %25, %26, %27, %28, %29, %30, %31}, [%32];"
        : "=r"(v[0]), "=r"(v[1]), "=r"(v[2]), "=r"(v[3]), "=r"(v[4]), "=r"(v[5]), "=r"(v[6]), "=r"(v[7]), "=r"(v[8]), "=r"(v[9]),
          "=r"(v[10]), "=r"(v[11]), "=r"(v[12]), "=r"(v[13]), "=r"(v[14]), "=r"(v[15]), "=r"(v[16]), "=r"(v[17]), "=r"(v[18]), "=r"(v[19]),
          "=r"(v[20]), "=r"(v[21]), "=r"(v[22]), "=r"(v[23]), "=r"(v[24]), "=r"(v[25]), "=r"(v[26]), "=r"(v[27]), "=r"(v[28]), "=r"(v[29]),
          "=r"(v[30]), "=r"(v[31])
        : "r"(at));
}
NFAD_TC void tmem_load_wait() { asm volatile("tcgen05.wait::ld.sync.aligned;" ::: "memory"); }

// Shared-memory operand with 128-byte swizzle.  Reduction-major: rows of 128 bytes along the reduction, eight rows to a
// 1024-byte group, `stride` between groups.  Row-major along the other dimension: 128-byte runs of it, eight reduction
// steps to a group, `stride` between groups, `lead` between the runs.
NFAD_TC uint64_t operand(uint32_t address, uint32_t lead, uint32_t stride)
{
    return uint64_t((address >> 4) & 0x3fff) | (uint64_t((lead >> 4) & 0x3fff) << 16) | (uint64_t((stride >> 4) & 0x3fff) << 32) |
           (1ull << 46) | (2ull << 61);
}

enum Number { kNumberF16 = 0, kNumberBF16 = 1, kNumberS8 = 2 };

// The instruction's description: accumulator type, operand types, which operands run along their own dimension in shared
// memory instead of along the reduction, and the tile's shape.
NFAD_TC uint32_t instruction(int number, bool a_turned, bool b_turned, uint32_t m, uint32_t n)
{
    const uint32_t acc = number == kNumberS8 ? 2 : 1, in = number == kNumberF16 ? 0 : 1;
    return (acc << 4) | (in << 7) | (in << 10) | (uint32_t(a_turned) << 15) | (uint32_t(b_turned) << 16) | ((n >> 3) << 17) | ((m >> 4) << 24);
}

// kPair: one product of both CTAs, 128 rows of the result in each one's tensor memory; A's rows and B's columns are split
// between their shared memories.  Issued by the first CTA.
template <bool kBytes, bool kPair> NFAD_TC void product(uint32_t acc, uint64_t a, uint64_t b, uint32_t what, bool add)
{
#define NFAD_PRODUCT(group, kind)                                                                                                    \
    asm volatile("{\n .reg .pred p;\n setp.ne.u32 p, %4, 0;\n tcgen05.mma.cta_group::" group ".kind::" kind " [%0], %1, %2, %3, p;\n}" \
                 ::"r"(acc), "l"(a), "l"(b), "r"(what), "r"(uint32_t(add)) : "memory")
    if (kBytes && kPair) NFAD_PRODUCT("2", "i8");
    else if (kBytes) NFAD_PRODUCT("1", "i8");
    else if (kPair) NFAD_PRODUCT("2", "f16");
    else NFAD_PRODUCT("1", "f16");
#undef NFAD_PRODUCT
}

// the barrier (kPair: that of each CTA of the pair) gets one arrival when every product issued so far by this thread is done
template <bool kPair> NFAD_TC void products_to(uint32_t bar)
{
    if (kPair)
        asm volatile("tcgen05.commit.cta_group::2.mbarrier::arrive::one.shared::cluster.multicast::cluster.b64 [%0], %1;" ::"r"(bar), "h"((unsigned short)3) : "memory");
    else
        asm volatile("tcgen05.commit.cta_group::1.mbarrier::arrive::one.shared::cluster.b64 [%0];" ::"r"(bar) : "memory");
}

}  // namespace tc
}  // namespace nfad
