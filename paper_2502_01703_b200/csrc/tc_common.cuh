// sm_100a building blocks used by the tensor-core kernels: mbarriers with bounded waits, TMA tile
// loads, tensor-memory (TMEM) allocation and access, tcgen05.mma issue and commit, descriptors.
#pragma once

#include <cuda.h>

#include "qless_common.cuh"

namespace qless {
namespace tc {

// Codes stored in the device timeout word (which wait gave up).
enum : uint32_t { TO_PRODUCER = 1u, TO_MMA = 2u, TO_GENERATOR = 4u, TO_EPILOGUE = 8u, TO_UNPACK = 16u };

// A wait gives up after about two seconds. A poll takes 0.1 to 4 us (the hardware may park the thread for a while; 2 us alone on an own
// barrier, 4 us with cluster scope), so their number alone bounds little: 2^26 polls were two to four minutes. The clock counts from the
// 256th poll on and only together with a least number of polls, so that a context that was switched out does not give up when it comes back.
constexpr uint32_t kWaitMs = 2000, kWaitLeastPolls = 1u << 18, kWaitLimit = 1u << 26;

__device__ __forceinline__ uint32_t smem_u32(const void* p) { return (uint32_t)__cvta_generic_to_shared(p); }

// ---- mbarrier ----------------------------------------------------------------------------------
__device__ __forceinline__ uint32_t wall_ms()           // in units of 2^20 ns
{
    uint64_t t;
    asm volatile("mov.u64 %0, %%globaltimer;" : "=l"(t));
    return (uint32_t)(t >> 20);
}
// Looked at every 256th poll: is the wait to end without success (another role has given up, or the time is up)?
__device__ __forceinline__ bool wait_over(uint32_t it, uint32_t& begin, volatile uint32_t* abort_flag)
{
    if (*abort_flag) return true;
    if (it == 255u) begin = wall_ms();
    if (it < kWaitLeastPolls || wall_ms() - begin < kWaitMs) return false;
    return true;
}
__device__ __forceinline__ void mbar_init(uint32_t bar, uint32_t count)
{
    asm volatile("mbarrier.init.shared::cta.b64 [%0], %1;" ::"r"(bar), "r"(count) : "memory");
}
__device__ __forceinline__ void fence_barrier_init()
{
    asm volatile("fence.mbarrier_init.release.cluster;" ::: "memory");
}
__device__ __forceinline__ void mbar_arrive(uint32_t bar)
{
    asm volatile("mbarrier.arrive.shared::cta.b64 _, [%0];" ::"r"(bar) : "memory");
}
__device__ __forceinline__ void mbar_arrive_expect_tx(uint32_t bar, uint32_t bytes)
{
    asm volatile("mbarrier.arrive.expect_tx.shared::cta.b64 _, [%0], %1;" ::"r"(bar), "r"(bytes) : "memory");
}
__device__ __forceinline__ bool mbar_try_wait(uint32_t bar, uint32_t parity)
{
    uint32_t ok;
    asm volatile(
        "{\n\t.reg .pred p;\n\t"
        "mbarrier.try_wait.parity.shared::cta.b64 p, [%1], %2;\n\t"
        "selp.u32 %0, 1, 0, p;\n\t}"
        : "=r"(ok)
        : "r"(bar), "r"(parity)
        : "memory");
    return ok != 0;
}
// try_wait that lets the hardware park the thread for up to hint_ns while the phase is open (it wakes when the phase
// closes): for waits of roles that share their scheduler with warps that have work to do.
__device__ __forceinline__ bool mbar_try_wait_parked(uint32_t bar, uint32_t parity, uint32_t hint_ns)
{
    uint32_t ok;
    asm volatile(
        "{\n\t.reg .pred p;\n\t"
        "mbarrier.try_wait.parity.shared::cta.b64 p, [%1], %2, %3;\n\t"
        "selp.u32 %0, 1, 0, p;\n\t}"
        : "=r"(ok)
        : "r"(bar), "r"(parity), "r"(hint_ns)
        : "memory");
    return ok != 0;
}
// Bounded wait built on it (same contract as mbar_wait).
__device__ __forceinline__ bool mbar_wait_parked(uint32_t bar, uint32_t parity, volatile uint32_t* abort_flag,
                                                 unsigned int* timeout_word, uint32_t code, uint32_t hint_ns = 2000u)
{
    uint32_t begin = 0u;
    for (uint32_t it = 0; it < (1u << 22); ++it) {
        if (mbar_try_wait_parked(bar, parity, hint_ns)) return true;
        if ((it & 15u) == 15u && wait_over(it, begin, abort_flag)) break;
    }
    if (*abort_flag) return false;
    *abort_flag = 1u;
    atomicOr(timeout_word, code);
    return false;
}
// One look at the barrier, never suspending the thread (try_wait may park it for a while when the phase is
// still open): for opportunistic checks on a path that has other work to do.
__device__ __forceinline__ bool mbar_test_wait(uint32_t bar, uint32_t parity)
{
    uint32_t ok;
    asm volatile(
        "{\n\t.reg .pred p;\n\t"
        "mbarrier.test_wait.parity.shared::cta.b64 p, [%1], %2;\n\t"
        "selp.u32 %0, 1, 0, p;\n\t}"
        : "=r"(ok)
        : "r"(bar), "r"(parity)
        : "memory");
    return ok != 0;
}
// Bounded wait. Returns false if the wait gave up or another role already aborted; the first thread to
// give up records `code` in the device timeout word and raises the CTA-wide abort flag.
__device__ __forceinline__ bool mbar_wait(uint32_t bar, uint32_t parity, volatile uint32_t* abort_flag,
                                          unsigned int* timeout_word, uint32_t code, uint32_t limit = kWaitLimit)
{
    uint32_t begin = 0u;
    for (uint32_t it = 0; it < limit; ++it) {
        if (mbar_try_wait(bar, parity)) return true;
        if ((it & 255u) == 255u && wait_over(it, begin, abort_flag)) break;
    }
    if (*abort_flag) return false;
    *abort_flag = 1u;
    atomicOr(timeout_word, code);
    return false;
}

// Bounded wait of the abort path: a role that is leaving after a failed wait uses it to let work it has already
// started (tensor-core instructions issued, copies armed) finish before tensor memory is freed and the CTA exits.
// It records nothing: the timeout word already says which wait gave up.
constexpr uint32_t kDrainLimit = 1u << 18;
__device__ __forceinline__ bool mbar_wait_quiet(uint32_t bar, uint32_t parity, uint32_t limit = kDrainLimit)
{
    for (uint32_t it = 0; it < limit; ++it)
        if (mbar_try_wait(bar, parity)) return true;
    return false;
}

// True in one lane of a fully active warp. A role that issues copies or tensor-core instructions runs with its whole warp and issues
// under this: the operands then live in uniform registers (eight products with a wait and a commit take 770 clocks of the issuing
// warp this way and 1310 when a single thread runs the role).
__device__ __forceinline__ bool elect_one()
{
    uint32_t p;
    asm volatile("{\n\t.reg .pred p;\n\telect.sync _|p, 0xFFFFFFFF;\n\tselp.u32 %0, 1, 0, p;\n\t}" : "=r"(p));
    return p != 0;
}

// Lane 0's value in every lane: tells the compiler that it is one value for the warp, so that branches on it and what is computed from it (operands
// of copies and tensor-core instructions above all) stay in uniform registers.
__device__ __forceinline__ int warp_uniform(int x) { return __shfl_sync(0xFFFFFFFFu, x, 0); }

// ---- CTA pairs (cta_group::2) --------------------------------------------------------------------
// A commit of the pair's leader (mma_commit_pair) arrives on a barrier in both CTAs' shared memory. Neither CTA may leave before the last of
// these arrivals has landed in it, for its shared memory may be another block's by then, and the cluster barrier at the end orders the
// pair's threads, not the arrivals of commits. So the role that waits for the slots of a ring waits, behind its last use of it, for all of them
// to be free once more (ring_drained), and at the end both CTAs wait for the leader's last commit (pair_drained; the roles have ended, so this is
// short; bounded: after a failed wait the leader's commits still come).
__device__ __forceinline__ uint32_t cluster_ctarank()
{
    uint32_t r;
    asm volatile("mov.u32 %0, %%cluster_ctarank;" : "=r"(r));
    return r;
}
__device__ __forceinline__ void cluster_sync_all()      // every thread of every CTA in the cluster
{
    asm volatile("barrier.cluster.arrive.release.aligned;" ::: "memory");
    asm volatile("barrier.cluster.wait.acquire.aligned;" ::: "memory");
}
// shared::cluster address of the same shared-memory location in CTA `rank` of the cluster
__device__ __forceinline__ uint32_t map_to_cta(uint32_t smem_addr, uint32_t rank)
{
    uint32_t r;
    asm volatile("mapa.shared::cluster.u32 %0, %1, %2;" : "=r"(r) : "r"(smem_addr), "r"(rank));
    return r;
}
// arrive on a barrier that may live in the peer CTA (address from map_to_cta)
__device__ __forceinline__ void mbar_arrive_cluster(uint32_t cluster_addr)
{
    asm volatile("mbarrier.arrive.release.cluster.shared::cluster.b64 _, [%0];" ::"r"(cluster_addr) : "memory");
}
// Arrival that only has to order tensor-memory accesses (already ordered by tcgen05.wait / tcgen05.fence),
// on the leader's barrier: a plain CTA-scope arrive in the leader, a relaxed cluster-scope one in the peer.
// (A release at cluster scope costs about 1500 clocks; these arrivals sit on the critical path of a stage.)
__device__ __forceinline__ void mbar_arrive_leader_tmem(uint32_t own_bar, uint32_t rank)
{
    if (rank == 0) {
        asm volatile("mbarrier.arrive.shared::cta.b64 _, [%0];" ::"r"(own_bar) : "memory");
    } else {
        uint32_t r;
        asm volatile("mapa.shared::cluster.u32 %0, %1, 0;" : "=r"(r) : "r"(own_bar));
        asm volatile("mbarrier.arrive.relaxed.cluster.shared::cluster.b64 _, [%0], 1;" ::"r"(r) : "memory");
    }
}
__device__ __forceinline__ bool mbar_try_wait_cluster(uint32_t bar, uint32_t parity)
{
    uint32_t ok;
    asm volatile(
        "{\n\t.reg .pred p;\n\t"
        "mbarrier.try_wait.parity.acquire.cluster.shared::cta.b64 p, [%1], %2;\n\t"
        "selp.u32 %0, 1, 0, p;\n\t}"
        : "=r"(ok)
        : "r"(bar), "r"(parity)
        : "memory");
    return ok != 0;
}
// Bounded wait on an own barrier whose arrivals may come from the peer CTA.
// backoff_ns > 0: sleep between polls, so that a warp in a long wait leaves the issue slots to the warps
// that share its scheduler.
__device__ __forceinline__ bool mbar_wait_cluster(uint32_t bar, uint32_t parity, volatile uint32_t* abort_flag,
                                                  unsigned int* timeout_word, uint32_t code, uint32_t backoff_ns = 0)
{
    uint32_t begin = 0u;
    for (uint32_t it = 0; it < kWaitLimit; ++it) {
        if (mbar_try_wait_cluster(bar, parity)) return true;
        if (backoff_ns) __nanosleep(backoff_ns);
        if ((it & 255u) == 255u && wait_over(it, begin, abort_flag)) break;
    }
    if (*abort_flag) return false;
    *abort_flag = 1u;
    atomicOr(timeout_word, code);
    return false;
}
template <typename Ring>
__device__ __forceinline__ bool ring_drained(uint64_t* empty, Ring ring, uint32_t slots, volatile uint32_t* abort_flag, unsigned int* timeout_word,
                                             uint32_t code)
{
    for (uint32_t j = 0; j < slots; ++j, ring.next(slots))
        if (!mbar_wait_cluster(smem_u32(&empty[ring.slot]), ring.parity ^ 1u, abort_flag, timeout_word, code)) return false;
    return true;
}
__device__ __forceinline__ void pair_drained(uint64_t* drain) { mbar_wait_quiet(smem_u32(drain), 0u); }
// TMA tile load whose completion is signalled on a barrier that may belong to the peer CTA of the pair.
__device__ __forceinline__ void tma_load_2d_pair(uint32_t smem_dst, const CUtensorMap* tmap, uint32_t bar_cluster_addr,
                                                 int32_t c0, int32_t c1)
{
    asm volatile(
        "cp.async.bulk.tensor.2d.shared::cluster.global.tile.mbarrier::complete_tx::bytes.cta_group::2 [%0], [%1, {%3, %4}], [%2];"
        ::"r"(smem_dst), "l"(tmap), "r"(bar_cluster_addr), "r"(c0), "r"(c1)
        : "memory");
}
__device__ __forceinline__ void tma_load_3d_pair(uint32_t smem_dst, const CUtensorMap* tmap, uint32_t bar_cluster_addr,
                                                 int32_t c0, int32_t c1, int32_t c2)
{
    asm volatile(
        "cp.async.bulk.tensor.3d.shared::cluster.global.tile.mbarrier::complete_tx::bytes.cta_group::2 [%0], [%1, {%3, %4, %5}], [%2];"
        ::"r"(smem_dst), "l"(tmap), "r"(bar_cluster_addr), "r"(c0), "r"(c1), "r"(c2)
        : "memory");
}
__device__ __forceinline__ void tmem_alloc_pair(uint32_t smem_result, uint32_t ncols)   // one warp in EACH CTA of the pair
{
    asm volatile("tcgen05.alloc.cta_group::2.sync.aligned.shared::cta.b32 [%0], %1;" ::"r"(smem_result), "r"(ncols) : "memory");
}
__device__ __forceinline__ void tmem_relinquish_pair()
{
    asm volatile("tcgen05.relinquish_alloc_permit.cta_group::2.sync.aligned;" ::: "memory");
}
__device__ __forceinline__ void tmem_dealloc_pair(uint32_t taddr, uint32_t ncols)
{
    asm volatile("tcgen05.dealloc.cta_group::2.sync.aligned.b32 %0, %1;" ::"r"(taddr), "r"(ncols) : "memory");
}
// Pair MMA (issued by one thread of the leader CTA): M = 256 split over the two CTAs' TMEM lanes, each CTA
// supplies its 128 rows of A (TMEM) and its N/2 rows of B (shared memory, same offset in both CTAs).
__device__ __forceinline__ void mma_f16_ts_pair(uint32_t d_tmem, uint32_t a_tmem, uint64_t b_desc, uint32_t idesc, uint32_t accumulate)
{
    asm volatile(
        "{\n\t.reg .pred p;\n\t"
        "setp.ne.b32 p, %4, 0;\n\t"
        "tcgen05.mma.cta_group::2.kind::f16 [%0], [%1], %2, %3, p;\n\t}"
        ::"r"(d_tmem), "r"(a_tmem), "l"(b_desc), "r"(idesc), "r"(accumulate)
        : "memory");
}
__device__ __forceinline__ void mma_i8_ss_pair(uint32_t d_tmem, uint64_t a_desc, uint64_t b_desc, uint32_t idesc, uint32_t accumulate)
{
    asm volatile(
        "{\n\t.reg .pred p;\n\t"
        "setp.ne.b32 p, %4, 0;\n\t"
        "tcgen05.mma.cta_group::2.kind::i8 [%0], %1, %2, %3, p;\n\t}"
        ::"r"(d_tmem), "l"(a_desc), "l"(b_desc), "r"(idesc), "r"(accumulate)
        : "memory");
}
// Pair MMA, bf16 (or f16) operands from shared memory, fp32 accumulation.
__device__ __forceinline__ void mma_f16_ss_pair(uint32_t d_tmem, uint64_t a_desc, uint64_t b_desc, uint32_t idesc, uint32_t accumulate)
{
    asm volatile(
        "{\n\t.reg .pred p;\n\t"
        "setp.ne.b32 p, %4, 0;\n\t"
        "tcgen05.mma.cta_group::2.kind::f16 [%0], %1, %2, %3, p;\n\t}"
        ::"r"(d_tmem), "l"(a_desc), "l"(b_desc), "r"(idesc), "r"(accumulate)
        : "memory");
}
// Pair MMA with the int8 A operand in tensor memory (lane = row, four codes per 32-bit column).
__device__ __forceinline__ void mma_i8_ts_pair(uint32_t d_tmem, uint32_t a_tmem, uint64_t b_desc, uint32_t idesc, uint32_t accumulate)
{
    asm volatile(
        "{\n\t.reg .pred p;\n\t"
        "setp.ne.b32 p, %4, 0;\n\t"
        "tcgen05.mma.cta_group::2.kind::i8 [%0], [%1], %2, %3, p;\n\t}"
        ::"r"(d_tmem), "r"(a_tmem), "l"(b_desc), "r"(idesc), "r"(accumulate)
        : "memory");
}
// Pair MMA on e2m1 operands (kind::mxf4, block-scaled, 64 codes per instruction, fp32 accumulation), both operands from
// shared memory. The scale factors (one UE8M0 byte per 32 codes of a row) are all 2^0: every byte of the tensor-memory
// columns at sf_tmem is 0x7F, so the layout in which the instruction reads them does not matter.
__device__ __forceinline__ void mma_mxf4_ss_pair(uint32_t d_tmem, uint64_t a_desc, uint64_t b_desc, uint32_t idesc, uint32_t sf_tmem,
                                                 uint32_t accumulate)
{
    asm volatile(
        "{\n\t.reg .pred p;\n\t"
        "setp.ne.b32 p, %4, 0;\n\t"
        "tcgen05.mma.cta_group::2.kind::mxf4.block_scale.scale_vec::2X [%0], %1, %2, %3, [%5], [%5], p;\n\t}"
        ::"r"(d_tmem), "l"(a_desc), "l"(b_desc), "r"(idesc), "r"(accumulate), "r"(sf_tmem)
        : "memory");
}
// Instruction descriptor of kind::mxf4: A and B format e2m1 (1) at bits [7,10) and [10,13), K-major, N/8 at [17,23),
// scale format UE8M0 (1) at bit 23, M/16 at [24,29), scale-factor byte offsets 0.
__host__ __device__ constexpr uint32_t make_idesc_mxf4(uint32_t M, uint32_t N)
{
    return (1u << 7) | (1u << 10) | ((N >> 3) << 17) | (1u << 23) | ((M >> 4) << 24);
}

// The same with A in tensor memory (lane = row, eight codes per 32-bit column, code j of them in bits [4j, 4j + 4)).
__device__ __forceinline__ void mma_mxf4_ts_pair(uint32_t d_tmem, uint32_t a_tmem, uint64_t b_desc, uint32_t idesc, uint32_t sf_tmem,
                                                 uint32_t accumulate)
{
    asm volatile(
        "{\n\t.reg .pred p;\n\t"
        "setp.ne.b32 p, %4, 0;\n\t"
        "tcgen05.mma.cta_group::2.kind::mxf4.block_scale.scale_vec::2X [%0], [%1], %2, %3, [%5], [%5], p;\n\t}"
        ::"r"(d_tmem), "r"(a_tmem), "l"(b_desc), "r"(idesc), "r"(accumulate), "r"(sf_tmem)
        : "memory");
}
// Arrive, once every MMA issued so far has completed, on the barrier at this offset in BOTH CTAs of the pair.
__device__ __forceinline__ void mma_commit_pair(uint32_t bar)
{
    const uint16_t mask = 3;
    asm volatile("tcgen05.commit.cta_group::2.mbarrier::arrive::one.shared::cluster.multicast::cluster.b64 [%0], %1;"
                 ::"r"(bar), "h"(mask) : "memory");
}

// ---- TMA ---------------------------------------------------------------------------------------
__device__ __forceinline__ void tma_load_2d(uint32_t smem_dst, const CUtensorMap* tmap, uint32_t bar, int32_t c0,
                                            int32_t c1)
{
    asm volatile(
        "cp.async.bulk.tensor.2d.shared::cluster.global.tile.mbarrier::complete_tx::bytes [%0], [%1, {%3, %4}], [%2];"
        ::"r"(smem_dst), "l"(tmap), "r"(bar), "r"(c0), "r"(c1)
        : "memory");
}
__device__ __forceinline__ void tma_load_3d(uint32_t smem_dst, const CUtensorMap* tmap, uint32_t bar, int32_t c0,
                                            int32_t c1, int32_t c2)
{
    asm volatile(
        "cp.async.bulk.tensor.3d.shared::cluster.global.tile.mbarrier::complete_tx::bytes [%0], [%1, {%3, %4, %5}], [%2];"
        ::"r"(smem_dst), "l"(tmap), "r"(bar), "r"(c0), "r"(c1), "r"(c2)
        : "memory");
}
// `bytes` consecutive bytes (a multiple of 16, both addresses 16-byte aligned) without a tensor map.
__device__ __forceinline__ void bulk_load(uint32_t smem_dst, const void* src, uint32_t bytes, uint32_t bar)
{
    asm volatile("cp.async.bulk.shared::cluster.global.mbarrier::complete_tx::bytes [%0], [%1], %2, [%3];"
                 ::"r"(smem_dst), "l"(src), "r"(bytes), "r"(bar) : "memory");
}
__device__ __forceinline__ void prefetch_l2(const void* p) { asm volatile("prefetch.global.L2 [%0];" ::"l"(p)); }
// The box of a tile into L2.
__device__ __forceinline__ void tma_prefetch_2d(const CUtensorMap* tmap, int32_t c0, int32_t c1)
{
    asm volatile("cp.async.bulk.prefetch.tensor.2d.L2.global.tile [%0, {%1, %2}];" ::"l"(tmap), "r"(c0), "r"(c1) : "memory");
}
__device__ __forceinline__ void tma_prefetch_3d(const CUtensorMap* tmap, int32_t c0, int32_t c1, int32_t c2)
{
    asm volatile("cp.async.bulk.prefetch.tensor.3d.L2.global.tile [%0, {%1, %2, %3}];" ::"l"(tmap), "r"(c0), "r"(c1), "r"(c2) : "memory");
}
__device__ __forceinline__ void prefetch_tmap(const CUtensorMap* tmap)
{
    asm volatile("prefetch.tensormap [%0];" ::"l"(tmap) : "memory");
}
__device__ __forceinline__ void fence_proxy_async_smem()
{
    asm volatile("fence.proxy.async.shared::cta;" ::: "memory");
}

// ---- TMEM --------------------------------------------------------------------------------------
__device__ __forceinline__ void tmem_alloc(uint32_t smem_result, uint32_t ncols)   // whole warp
{
    asm volatile("tcgen05.alloc.cta_group::1.sync.aligned.shared::cta.b32 [%0], %1;" ::"r"(smem_result), "r"(ncols) : "memory");
}
__device__ __forceinline__ void tmem_relinquish()   // whole warp
{
    asm volatile("tcgen05.relinquish_alloc_permit.cta_group::1.sync.aligned;" ::: "memory");
}
__device__ __forceinline__ void tmem_dealloc(uint32_t taddr, uint32_t ncols)   // whole warp
{
    asm volatile("tcgen05.dealloc.cta_group::1.sync.aligned.b32 %0, %1;" ::"r"(taddr), "r"(ncols) : "memory");
}
__device__ __forceinline__ void tc_fence_before() { asm volatile("tcgen05.fence::before_thread_sync;" ::: "memory"); }
__device__ __forceinline__ void tc_fence_after() { asm volatile("tcgen05.fence::after_thread_sync;" ::: "memory"); }
__device__ __forceinline__ void tmem_wait_ld() { asm volatile("tcgen05.wait::ld.sync.aligned;" ::: "memory"); }
__device__ __forceinline__ void tmem_wait_st() { asm volatile("tcgen05.wait::st.sync.aligned;" ::: "memory"); }

// 32 lanes x 16 consecutive 32-bit columns, one lane per thread (whole warp).
__device__ __forceinline__ void tmem_st_x16(uint32_t taddr, const uint32_t (&v)[16])
{
    asm volatile(
        "tcgen05.st.sync.aligned.32x32b.x16.b32 [%0], {%1, %2, %3, %4, %5, %6, %7, %8, %9, %10, %11, %12, %13, %14, %15, %16};"
        ::"r"(taddr), "r"(v[0]), "r"(v[1]), "r"(v[2]), "r"(v[3]), "r"(v[4]), "r"(v[5]), "r"(v[6]), "r"(v[7]), "r"(v[8]),
        "r"(v[9]), "r"(v[10]), "r"(v[11]), "r"(v[12]), "r"(v[13]), "r"(v[14]), "r"(v[15])
        : "memory");
}
// 32 lanes x 8 consecutive 32-bit columns (whole warp).
__device__ __forceinline__ void tmem_st_x8(uint32_t taddr, const uint32_t (&v)[8])
{
    asm volatile("tcgen05.st.sync.aligned.32x32b.x8.b32 [%0], {%1, %2, %3, %4, %5, %6, %7, %8};"
                 ::"r"(taddr), "r"(v[0]), "r"(v[1]), "r"(v[2]), "r"(v[3]), "r"(v[4]), "r"(v[5]), "r"(v[6]), "r"(v[7]) : "memory");
}
// 32 lanes x 32 consecutive 32-bit columns (whole warp).
__device__ __forceinline__ void tmem_ld_x32(uint32_t taddr, uint32_t (&v)[32])
{
    asm volatile(
        "tcgen05.ld.sync.aligned.32x32b.x32.b32 {%0, %1, %2, %3, %4, %5, %6, %7, %8, %9, %10, %11, %12, %13, %14, %15, "
        "%16, %17, %18, %19, %20, %21, %22, %23, %24, %25, %26, %27, %28, %29, %30, %31}, [%32];"
        : "=r"(v[0]), "=r"(v[1]), "=r"(v[2]), "=r"(v[3]), "=r"(v[4]), "=r"(v[5]), "=r"(v[6]), "=r"(v[7]), "=r"(v[8]),
          "=r"(v[9]), "=r"(v[10]), "=r"(v[11]), "=r"(v[12]), "=r"(v[13]), "=r"(v[14]), "=r"(v[15]), "=r"(v[16]),
          "=r"(v[17]), "=r"(v[18]), "=r"(v[19]), "=r"(v[20]), "=r"(v[21]), "=r"(v[22]), "=r"(v[23]), "=r"(v[24]),
          "=r"(v[25]), "=r"(v[26]), "=r"(v[27]), "=r"(v[28]), "=r"(v[29]), "=r"(v[30]), "=r"(v[31])
        : "r"(taddr)
        : "memory");
}

// 32 lanes x 16 consecutive 32-bit columns (whole warp).
__device__ __forceinline__ void tmem_ld_x16(uint32_t taddr, uint32_t (&v)[16])
{
    asm volatile(
        "tcgen05.ld.sync.aligned.32x32b.x16.b32 {%0, %1, %2, %3, %4, %5, %6, %7, %8, %9, %10, %11, %12, %13, %14, %15}, [%16];"
        : "=r"(v[0]), "=r"(v[1]), "=r"(v[2]), "=r"(v[3]), "=r"(v[4]), "=r"(v[5]), "=r"(v[6]), "=r"(v[7]), "=r"(v[8]),
          "=r"(v[9]), "=r"(v[10]), "=r"(v[11]), "=r"(v[12]), "=r"(v[13]), "=r"(v[14]), "=r"(v[15])
        : "r"(taddr)
        : "memory");
}

// ---- MMA ---------------------------------------------------------------------------------------
// Instruction descriptor of tcgen05.mma kind::f16 / kind::i8: D format bits [4,6) (1 = F32, 2 = S32),
// A format bits [7,10), B format bits [10,13) (f16 kinds: 0 = F16, 1 = BF16; i8: 0 = U8, 1 = S8),
// A/B major bits 15/16 (0 = K-major), N/8 bits [17,23), M/16 bits [24,29).
__host__ __device__ constexpr uint32_t make_idesc(uint32_t d_fmt, uint32_t a_fmt, uint32_t b_fmt, uint32_t M, uint32_t N)
{
    return (d_fmt << 4) | (a_fmt << 7) | (b_fmt << 10) | ((N >> 3) << 17) | ((M >> 4) << 24);
}
// Shared-memory matrix descriptor of a K-major operand stored as rows of 128 bytes with the 128-byte
// swizzle (what a TMA load with SWIZZLE_128B writes): start address / 16 in bits [0,14), leading byte
// offset (unused for this layout) bits [16,30), stride between 8-row groups (1024 B) / 16 in bits
// [32,46), descriptor version 1 at bit 46, layout type 2 (128-byte swizzle) in bits [61,64).
__device__ __forceinline__ uint64_t make_smem_desc_sw128(uint32_t smem_addr)
{
    return (uint64_t)((smem_addr & 0x3FFFFu) >> 4) | ((uint64_t)1 << 16) | ((uint64_t)(1024 >> 4) << 32) |
           ((uint64_t)1 << 46) | ((uint64_t)2 << 61);
}
// Instruction-descriptor bits that mark an operand as M-major (A) or N-major (B): its smem rows run along M or N.
constexpr uint32_t IDESC_A_MN = 1u << 15, IDESC_B_MN = 1u << 16;
// Descriptor of an M- or N-major 16-bit operand: blocks of 64 consecutive M (or N) values, each block rows of 128 bytes, one
// row per k, 128-byte swizzled (a TMA box 64 wide and as many rows high as the k block). `block_bytes` (leading byte offset)
// is the distance between neighbouring 64-wide blocks; groups of eight k rows are 1024 bytes apart, so 16 k values further
// on is 2048 bytes further on.
__device__ __forceinline__ uint64_t make_smem_desc_mn_sw128(uint32_t smem_addr, uint32_t block_bytes)
{
    return (uint64_t)((smem_addr & 0x3FFFFu) >> 4) | ((uint64_t)(block_bytes >> 4) << 16) | ((uint64_t)(1024 >> 4) << 32) |
           ((uint64_t)1 << 46) | ((uint64_t)2 << 61);
}
// D[tmem] (+)= A[tmem] * B[smem]^T, bf16 operands (one thread issues).
__device__ __forceinline__ void mma_f16_ts(uint32_t d_tmem, uint32_t a_tmem, uint64_t b_desc, uint32_t idesc, uint32_t accumulate)
{
    asm volatile(
        "{\n\t.reg .pred p;\n\t"
        "setp.ne.b32 p, %4, 0;\n\t"
        "tcgen05.mma.cta_group::1.kind::f16 [%0], [%1], %2, %3, p;\n\t}"
        ::"r"(d_tmem), "r"(a_tmem), "l"(b_desc), "r"(idesc), "r"(accumulate)
        : "memory");
}
// D[tmem] (+)= A[smem] * B[smem]^T, bf16 operands, fp32 accumulation.
__device__ __forceinline__ void mma_f16_ss(uint32_t d_tmem, uint64_t a_desc, uint64_t b_desc, uint32_t idesc, uint32_t accumulate)
{
    asm volatile(
        "{\n\t.reg .pred p;\n\t"
        "setp.ne.b32 p, %4, 0;\n\t"
        "tcgen05.mma.cta_group::1.kind::f16 [%0], %1, %2, %3, p;\n\t}"
        ::"r"(d_tmem), "l"(a_desc), "l"(b_desc), "r"(idesc), "r"(accumulate)
        : "memory");
}
// D[tmem] (+)= A[smem] * B[smem]^T, signed 8-bit operands, int32 accumulation.
__device__ __forceinline__ void mma_i8_ss(uint32_t d_tmem, uint64_t a_desc, uint64_t b_desc, uint32_t idesc, uint32_t accumulate)
{
    asm volatile(
        "{\n\t.reg .pred p;\n\t"
        "setp.ne.b32 p, %4, 0;\n\t"
        "tcgen05.mma.cta_group::1.kind::i8 [%0], %1, %2, %3, p;\n\t}"
        ::"r"(d_tmem), "l"(a_desc), "l"(b_desc), "r"(idesc), "r"(accumulate)
        : "memory");
}
// Arrive on an mbarrier once every MMA issued so far by this thread has completed.
__device__ __forceinline__ void mma_commit(uint32_t bar)
{
    asm volatile("tcgen05.commit.cta_group::1.mbarrier::arrive::one.shared::cluster.b64 [%0];" ::"r"(bar) : "memory");
}

// Four neighbouring lanes hold four 16-byte pieces each of a row of their own; afterwards lane i of the four holds piece i of each of the
// four rows: a store instruction then covers 64 consecutive bytes of eight rows instead of 16 of thirty-two.
__device__ __forceinline__ void transpose4(uint4 (&v)[4], int lane)
{
    auto swap = [](uint4 a, int m) {
        a.x = __shfl_xor_sync(0xFFFFFFFFu, a.x, m); a.y = __shfl_xor_sync(0xFFFFFFFFu, a.y, m);
        a.z = __shfl_xor_sync(0xFFFFFFFFu, a.z, m); a.w = __shfl_xor_sync(0xFFFFFFFFu, a.w, m);
        return a;
    };
#pragma unroll
    for (int m = 1; m <= 2; m <<= 1) {
        const bool up = (lane & m) != 0;
#pragma unroll
        for (int k = 0; k < 4; ++k) {
            if (k & m) continue;
            const uint4 got = swap(up ? v[k] : v[k + m], m);
            if (up) v[k] = got;
            else v[k + m] = got;
        }
    }
}

}  // namespace tc

// Host: 2-D row-major tensor map (inner dimension contiguous) with a 128-byte-swizzled box.
// elem_bytes in {1, 2}; box_inner * elem_bytes must be 128.
qless_status make_tmap_2d_sw128(CUtensorMap* out, const void* base, int elem_bytes, uint64_t inner, uint64_t outer,
                                uint64_t row_stride_bytes, uint32_t box_inner, uint32_t box_outer);

// Host: a matrix of `blocks` side-by-side column blocks of 128 bytes, seen as [block][row][128 bytes] (block_stride bytes apart,
// rows row_stride bytes apart), so that one copy brings box_blocks blocks of box_rows rows each, 128-byte-swizzled.
qless_status make_tmap_blocks_sw128(CUtensorMap* out, const void* base, int elem_bytes, uint64_t blocks, uint64_t rows, uint64_t row_stride,
                                    uint64_t block_stride, uint32_t box_rows, uint32_t box_blocks);

// Host: bf16 [tokens][heads][head_dim] (token_stride bytes between tokens), boxes of 64 columns x box_heads x box_tokens, 128-byte-swizzled: rows
// of 128 bytes, the heads of a token one behind the other; columns behind head_dim and tokens behind the last read as zeros.
qless_status make_tmap_heads_sw128(CUtensorMap* out, const void* base, uint64_t head_dim, uint64_t heads, uint64_t tokens, uint64_t token_stride,
                                   uint32_t box_heads, uint32_t box_tokens);

// Host: 3-D byte tensor map [outer2][outer1][inner bytes] (uint8 elements). swizzle128 = true needs a 128-byte
// wide box; otherwise the box lands in shared memory as plain rows of box_inner bytes (a multiple of 16).
qless_status make_tmap_3d_u8(CUtensorMap* out, const void* base, uint64_t inner_bytes, uint64_t outer1, uint64_t outer2,
                             uint64_t stride1_bytes, uint64_t stride2_bytes, uint32_t box_inner, uint32_t box_outer1,
                             bool swizzle128);

}  // namespace qless
