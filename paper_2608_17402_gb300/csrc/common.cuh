// common.cuh -- device helpers shared by the MoE-ViE layer kernels (sm_103a).
//
// Device errors never trap: a kernel that finds a bad index, or whose pipeline
// wait runs past its time limit, records the first such event in the status
// block at the start of the caller's workspace and returns.
#pragma once

#include <cuda.h>
#include <cuda_bf16.h>
#include <cuda_runtime.h>
#include <stdint.h>

#include "moevie.h"

namespace mv {

// ------------------------------------------------------------------ status

// Lives at byte 0 of every workspace (256 bytes, zeroed by moevie_workspace_init).
struct DevStatus {
    int code;        // first device error (MOEVIE_ERR_*), 0 when none
    int site;        // which check (Site)
    int a, b;        // two values describing it
    int fb_count;    // router: tokens re-decided with exact logits in the last call
    int bar_count;   // grid barrier of a cooperative launch: arrivals so far (0 between barriers)
    int bar_gen;     //   and the barrier's generation (bumped by the last arrival)
    int pad0;
    unsigned long long few_arrivals;   // grid barriers of the few-token kernel: CTAs arrived so far
    unsigned bal_ticket;   // CTAs of the balance loss that are done (0 between calls)
    int pad[53];
};
static_assert(sizeof(DevStatus) == 256, "status block is 256 bytes");

enum Site : int {
    SITE_GEMM_WAIT_FULL = 1,
    SITE_GEMM_WAIT_EMPTY = 2,
    SITE_GEMM_WAIT_TFULL = 3,
    SITE_GEMM_WAIT_TEMPTY = 4,
    SITE_GEMM_DRAIN = 5,
    SITE_GEMM_A_ROW = 6,
    SITE_GEMM_TILES = 7,
    SITE_GEMM_OUT_ROW = 8,
    SITE_PERMUTE_ID = 10,
    SITE_ROUTE_FALLBACK = 20,
    SITE_BIAS_COUNTS = 21,
    SITE_TIMEOUT_PROBE = 30,
    SITE_PERMUTE_BARRIER = 31,
    SITE_NS_WAIT_EMPTY = 40,
    SITE_NS_WAIT_FULL = 41,
    SITE_NS_WAIT_TFULL = 42,
    SITE_NS_WAIT_TEMPTY = 43,
    SITE_NS_DRAIN = 44,
    SITE_NS_WAIT_INPUT = 45,
    SITE_NS_WAIT_BUFFER = 46,
    SITE_NS_WAIT_SLOT = 47,
    SITE_FEW_WAIT_EMPTY = 50,
    SITE_FEW_WAIT_FULL = 51,
    SITE_FEW_WAIT_TFULL = 52,
    SITE_FEW_WAIT_TEMPTY = 53,
    SITE_FEW_WAIT_UP = 54,
    SITE_FEW_BARRIER = 55,
    SITE_FEW_DRAIN = 56,
    SITE_FEW_WAIT_Y = 57,
    SITE_FEW_WAIT_TURN = 58,
    SITE_RUNS = 60,
    SITE_BALANCE_ID = 61,
};

__device__ __forceinline__ void report(DevStatus* st, int code, int site, int a, int b) {
    if (atomicCAS(&st->code, 0, code) == 0) {
        st->site = site;
        st->a = a;
        st->b = b;
    }
}

// Grid-wide barrier of a cooperative launch (all nblocks CTAs co-resident) with a time
// limit: the last CTA to arrive resets the count and bumps the generation; the others
// wait for the bump for at most limit_ns.  Returns false (after recording
// MOEVIE_ERR_TIMEOUT at `site`) when the wait ran out; the caller then stops.  The count
// starts at 0 (a zeroed status block) and returns to 0 after every barrier.
__device__ __forceinline__ bool grid_barrier(DevStatus* st, unsigned nblocks, uint64_t limit_ns, int site) {
    __shared__ int s_ok;
    __syncthreads();
    if (threadIdx.x == 0) {
        volatile int* genp = &st->bar_gen;
        const int gen = *genp;
        __threadfence();   // this CTA's writes before its arrival
        int ok = 1;
        if (atomicAdd(&st->bar_count, 1) == (int)nblocks - 1) {
            st->bar_count = 0;
            __threadfence();
            atomicAdd(&st->bar_gen, 1);
        } else {
            uint64_t t0;
            asm volatile("mov.u64 %0, %%globaltimer;" : "=l"(t0));
            for (uint32_t i = 1; *genp == gen; ++i) {
                if ((i & 63u) == 0u) {
                    uint64_t t1;
                    asm volatile("mov.u64 %0, %%globaltimer;" : "=l"(t1));
                    if (t1 - t0 > limit_ns) {
                        ok = 0;
                        report(st, MOEVIE_ERR_TIMEOUT, site, (int)blockIdx.x, gen);
                        break;
                    }
                }
            }
        }
        __threadfence();   // the other CTAs' writes after the barrier
        s_ok = ok;
    }
    __syncthreads();
    return s_ok != 0;
}

// The run that row t lies in, of runs [seg[g], seg[g + 1]): the last g < G with seg[g] <= t, 0 where
// there is none.  By a whole warp, which looks at 32 of them at a time.
__device__ __forceinline__ int64_t warp_run_of(const int32_t* seg, int64_t G, int64_t t) {
    int64_t lo = 0, n = G;   // it is one of the n from lo on
    while (n > 1) {
        const int64_t step = (n + 31) / 32, at = lo + (threadIdx.x & 31) * step;
        const unsigned below = __ballot_sync(0xffffffffu, at < lo + n && seg[at] <= t);
        const int hit = below ? 31 - __clz(below) : 0;   // (the lanes below it, too, where seg ascends)
        n = min(step, lo + n - (lo + hit * step));
        lo += hit * step;
    }
    return lo;
}

// Programmatic dependent launch: a kernel launched with programmatic stream
// serialization may start while its predecessor finishes; it waits here (at the
// top, before touching anything the predecessor writes) until that predecessor has
// completed and its memory is visible.  A no-op for ordinary launches.
__device__ __forceinline__ void pdl_wait() { asm volatile("griddepcontrol.wait;" ::: "memory"); }

// ---------------------------------------------------------------- basics

__device__ __forceinline__ uint64_t globaltimer_ns() {
    uint64_t t;
    asm volatile("mov.u64 %0, %%globaltimer;" : "=l"(t));
    return t;
}

__device__ __forceinline__ uint32_t smem_u32(const void* p) {
    return static_cast<uint32_t>(__cvta_generic_to_shared(p));
}

// True in one lane of a converged warp.  A role that a single thread plays branches on this
// rather than on a lane number: the compiler then knows that the branch has one active thread
// and issues tcgen05.mma and TMA instructions from uniform registers directly, instead of
// looping over possibly active lanes (measured: 25 instead of 61 cycles per TMA instruction).
__device__ __forceinline__ bool elect_one() {
    uint32_t ok;
    asm volatile("{\n\t.reg .pred p;\n\telect.sync _|p, 0xffffffff;\n\tselp.u32 %0, 1, 0, p;\n\t}" : "=r"(ok));
    return ok != 0;
}

// --------------------------------------------------------------- mbarrier

__device__ __forceinline__ void mbar_init(uint32_t bar, uint32_t count) {
    asm volatile("mbarrier.init.shared::cta.b64 [%0], %1;" ::"r"(bar), "r"(count) : "memory");
}
__device__ __forceinline__ void mbar_fence_init() {
    asm volatile("fence.mbarrier_init.release.cluster;" ::: "memory");
}
__device__ __forceinline__ void mbar_arrive(uint32_t bar) {
    asm volatile("mbarrier.arrive.shared::cta.b64 _, [%0];" ::"r"(bar) : "memory");
}
__device__ __forceinline__ void mbar_arrive_expect_tx(uint32_t bar, uint32_t bytes) {
    asm volatile("mbarrier.arrive.expect_tx.shared::cta.b64 _, [%0], %1;" ::"r"(bar), "r"(bytes)
                 : "memory");
}
__device__ __forceinline__ bool mbar_try_wait(uint32_t bar, uint32_t parity) {
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

// Wait for the phase of `parity` to complete.  Gives up (returns false) once
// `limit_ns` of device time has passed, or as soon as *abort_flag is set by
// another role of the same CTA.  Every pipeline wait in this library goes here.
__device__ __forceinline__ bool mbar_wait(uint32_t bar, uint32_t parity, uint64_t limit_ns,
                                          const volatile int* abort_flag) {
    if (mbar_try_wait(bar, parity)) return true;
    const uint64_t t0 = globaltimer_ns();
    for (uint32_t i = 1;; ++i) {
        if (mbar_try_wait(bar, parity)) return true;
        if ((i & 127u) == 0u) {
            if (abort_flag && *abort_flag) return false;
            if (globaltimer_ns() - t0 > limit_ns) return false;
        }
    }
}

// A CTA whose pipeline gave up may still have copies under way into its shared memory, on barriers
// whose other arrivals never come, so no barrier says when they have landed.  They take
// microseconds: before such a CTA (or its pair) ends, a millisecond passes.  Called by one whole
// warp, after a barrier behind the last copy and before what it ends the CTA (or the pair) with.
static __device__ __noinline__ void wait_for_copies() {
    const uint64_t t0 = globaltimer_ns();
    for (int i = 0; i < 100000 && globaltimer_ns() - t0 < 1000000ull; ++i) __nanosleep(1000);
    __syncwarp();
}
__device__ __forceinline__ void settle_copies(const volatile int* abort_flag) {
    if (*abort_flag) wait_for_copies();
}

// ------------------------------------------- publishing data between CTAs

__device__ __forceinline__ void fence_proxy_async_all() { asm volatile("fence.proxy.async;" ::: "memory"); }
__device__ __forceinline__ int ld_acquire(const int32_t* p) {
    int v;
    asm volatile("ld.acquire.gpu.global.b32 %0, [%1];" : "=r"(v) : "l"(p) : "memory");
    return v;
}
// Counter updates that publish what this thread wrote or has seen written through a barrier,
// and (acq_rel) order its later reads after the other contributors' writes.
__device__ __forceinline__ void add_release(int32_t* p, int v) {
    asm volatile("red.add.release.gpu.global.s32 [%0], %1;" ::"l"(p), "r"(v) : "memory");
}
__device__ __forceinline__ int add_acq_rel(int32_t* p, int v) {
    int old;
    asm volatile("atom.add.acq_rel.gpu.global.s32 %0, [%1], %2;" : "=r"(old) : "l"(p), "r"(v) : "memory");
    return old;
}

// ------------------------------------------------------------- cp.async

// 16-byte global->shared copy; src_bytes < 16 zero-fills the rest (0: all zeros,
// nothing read).
__device__ __forceinline__ void cp_async16(uint32_t dst, const void* src, uint32_t src_bytes) {
    asm volatile("cp.async.cg.shared.global [%0], [%1], 16, %2;" ::"r"(dst), "l"(src),
                 "r"(src_bytes)
                 : "memory");
}
// L2 cache policies (createpolicy): keep lines (evict_last) or let them go first.
__device__ __forceinline__ uint64_t l2_policy_evict_last() {
    uint64_t pol;
    asm volatile("createpolicy.fractional.L2::evict_last.b64 %0, 1.0;" : "=l"(pol));
    return pol;
}
__device__ __forceinline__ uint64_t l2_policy_evict_first() {
    uint64_t pol;
    asm volatile("createpolicy.fractional.L2::evict_first.b64 %0, 1.0;" : "=l"(pol));
    return pol;
}
// cp_async16 with an L2 cache policy for the global read.
__device__ __forceinline__ void cp_async16_hint(uint32_t dst, const void* src, uint32_t src_bytes,
                                                uint64_t pol) {
    asm volatile("cp.async.cg.shared.global.L2::cache_hint [%0], [%1], 16, %2, %3;" ::"r"(dst),
                 "l"(src), "r"(src_bytes), "l"(pol)
                 : "memory");
}
// 16-byte global store with an L2 cache policy.
__device__ __forceinline__ void st_global_v4_hint(void* p, const uint4& v, uint64_t pol) {
    asm volatile("st.global.L2::cache_hint.v4.b32 [%0], {%1, %2, %3, %4}, %5;" ::"l"(p), "r"(v.x),
                 "r"(v.y), "r"(v.z), "r"(v.w), "l"(pol)
                 : "memory");
}
__device__ __forceinline__ void cp_async_commit() {
    asm volatile("cp.async.commit_group;" ::: "memory");
}
template <int N>
__device__ __forceinline__ void cp_async_wait() {
    asm volatile("cp.async.wait_group %0;" ::"n"(N) : "memory");
}
// Orders this thread's generic-proxy shared-memory writes before later
// async-proxy reads (tcgen05.mma operands, TMA stores).
// Arrive on `bar` once all cp.async copies issued so far by this thread have landed
// (the barrier's expected count includes this arrival).
__device__ __forceinline__ void cp_async_arrive_noinc(uint32_t bar) {
    asm volatile("cp.async.mbarrier.arrive.noinc.shared::cta.b64 [%0];" ::"r"(bar) : "memory");
}
__device__ __forceinline__ void cp_async_wait_all() {
    asm volatile("cp.async.wait_all;" ::: "memory");
}
__device__ __forceinline__ void fence_proxy_async_smem() {
    asm volatile("fence.proxy.async.shared::cta;" ::: "memory");
}

// ------------------------------------------------------------------- TMA

__device__ __forceinline__ void tma_load_3d(uint32_t dst, const CUtensorMap* tm, uint32_t bar,
                                            int c0, int c1, int c2) {
    asm volatile(
        "cp.async.bulk.tensor.3d.shared::cluster.global.tile.mbarrier::complete_tx::bytes"
        " [%0], [%1, {%2, %3, %4}], [%5];" ::"r"(dst),
        "l"(tm), "r"(c0), "r"(c1), "r"(c2), "r"(bar)
        : "memory");
}
// with an L2 cache policy for the global read
__device__ __forceinline__ void tma_load_3d_hint(uint32_t dst, const CUtensorMap* tm, uint32_t bar,
                                                 int c0, int c1, int c2, uint64_t pol) {
    asm volatile(
        "cp.async.bulk.tensor.3d.shared::cluster.global.tile.mbarrier::complete_tx::bytes.L2::cache_hint"
        " [%0], [%1, {%2, %3, %4}], [%5], %6;" ::"r"(dst),
        "l"(tm), "r"(c0), "r"(c1), "r"(c2), "r"(bar), "l"(pol)
        : "memory");
}
__device__ __forceinline__ void tma_load_2d(uint32_t dst, const CUtensorMap* tm, uint32_t bar,
                                            int c0, int c1) {
    asm volatile(
        "cp.async.bulk.tensor.2d.shared::cluster.global.tile.mbarrier::complete_tx::bytes"
        " [%0], [%1, {%2, %3}], [%4];" ::"r"(dst),
        "l"(tm), "r"(c0), "r"(c1), "r"(bar)
        : "memory");
}
// Four rows r0..r3 of a 2-D tensor (box {cols, 1}) into four consecutive box rows
// at dst.  The 128-byte swizzle follows the shared-memory address, so four rows
// written at dst = tile + 128 * r land exactly as rows r..r+3 of a swizzled tile.
__device__ __forceinline__ void tma_gather4(uint32_t dst, const CUtensorMap* tm, uint32_t bar,
                                            int col, int r0, int r1, int r2, int r3) {
    asm volatile(
        "cp.async.bulk.tensor.2d.shared::cluster.global.tile::gather4.mbarrier::complete_tx::bytes"
        " [%0], [%1, {%2, %3, %4, %5, %6}], [%7];" ::"r"(dst),
        "l"(tm), "r"(col), "r"(r0), "r"(r1), "r"(r2), "r"(r3), "r"(bar)
        : "memory");
}
__device__ __forceinline__ void tma_prefetch_desc(const CUtensorMap* tm) {
    asm volatile("prefetch.tensormap [%0];" ::"l"(tm) : "memory");
}

// --------------------------------------------------------------- tcgen05

__device__ __forceinline__ void tmem_alloc(uint32_t slot, uint32_t ncols) {
    asm volatile("tcgen05.alloc.cta_group::1.sync.aligned.shared::cta.b32 [%0], %1;" ::"r"(slot),
                 "r"(ncols)
                 : "memory");
}
__device__ __forceinline__ void tmem_relinquish() {
    asm volatile("tcgen05.relinquish_alloc_permit.cta_group::1.sync.aligned;" ::: "memory");
}
__device__ __forceinline__ void tmem_dealloc(uint32_t taddr, uint32_t ncols) {
    asm volatile("tcgen05.dealloc.cta_group::1.sync.aligned.b32 %0, %1;" ::"r"(taddr), "r"(ncols)
                 : "memory");
}
__device__ __forceinline__ void tc_fence_before() {
    asm volatile("tcgen05.fence::before_thread_sync;" ::: "memory");
}
__device__ __forceinline__ void tc_fence_after() {
    asm volatile("tcgen05.fence::after_thread_sync;" ::: "memory");
}
// D[tmem] (+)= A[smem] . B[smem], bf16 inputs, fp32 accumulate (kind::f16).
__device__ __forceinline__ void tc_mma_bf16(uint32_t d_tmem, uint64_t adesc, uint64_t bdesc,
                                            uint32_t idesc, uint32_t accumulate) {
    asm volatile(
        "{\n\t.reg .pred p;\n\t"
        "setp.ne.b32 p, %4, 0;\n\t"
        "tcgen05.mma.cta_group::1.kind::f16 [%0], %1, %2, %3, p;\n\t}" ::"r"(d_tmem),
        "l"(adesc), "l"(bdesc), "r"(idesc), "r"(accumulate)
        : "memory");
}
// Arrive once on `bar` when every tcgen05 operation issued so far by this thread
// has completed.
__device__ __forceinline__ void tc_commit(uint32_t bar) {
    asm volatile(
        "tcgen05.commit.cta_group::1.mbarrier::arrive::one.shared::cluster.b64 [%0];" ::"r"(bar)
        : "memory");
}
// 32 lanes x 32 consecutive 32-bit columns: thread i of the warp gets lane
// (base lane + i), columns [col, col + 32).
__device__ __forceinline__ void tmem_ld_32x32b_x32(uint32_t taddr, uint32_t (&r)[32]) {
    asm volatile(
        "tcgen05.ld.sync.aligned.32x32b.x32.b32 "
        "{%0,%1,%2,%3,%4,%5,%6,%7,%8,%9,%10,%11,%12,%13,%14,%15,"
        "%16,%17,%18,%19,%20,%21,%22,%23,%24,%25,%26,%27,%28,%29,%30,%31}, [%32];"
        : "=r"(r[0]), "=r"(r[1]), "=r"(r[2]), "=r"(r[3]), "=r"(r[4]), "=r"(r[5]), "=r"(r[6]),
          "=r"(r[7]), "=r"(r[8]), "=r"(r[9]), "=r"(r[10]), "=r"(r[11]), "=r"(r[12]),
          "=r"(r[13]), "=r"(r[14]), "=r"(r[15]), "=r"(r[16]), "=r"(r[17]), "=r"(r[18]),
          "=r"(r[19]), "=r"(r[20]), "=r"(r[21]), "=r"(r[22]), "=r"(r[23]), "=r"(r[24]),
          "=r"(r[25]), "=r"(r[26]), "=r"(r[27]), "=r"(r[28]), "=r"(r[29]), "=r"(r[30]),
          "=r"(r[31])
        : "r"(taddr)
        : "memory");
}
// 32 lanes x 16 consecutive 32-bit columns (thread i: lane base + i, columns col..col+15).
__device__ __forceinline__ void tmem_ld_32x32b_x16(uint32_t taddr, uint32_t (&r)[16]) {
    asm volatile(
        "tcgen05.ld.sync.aligned.32x32b.x16.b32 "
        "{%0,%1,%2,%3,%4,%5,%6,%7,%8,%9,%10,%11,%12,%13,%14,%15}, [%16];"
        : "=r"(r[0]), "=r"(r[1]), "=r"(r[2]), "=r"(r[3]), "=r"(r[4]), "=r"(r[5]), "=r"(r[6]),
          "=r"(r[7]), "=r"(r[8]), "=r"(r[9]), "=r"(r[10]), "=r"(r[11]), "=r"(r[12]),
          "=r"(r[13]), "=r"(r[14]), "=r"(r[15])
        : "r"(taddr)
        : "memory");
}
// 16 lanes x 4 repetitions of 256 bits (8 32-bit columns): for repetition j,
// thread i gets r[4j], r[4j+1] = lane (base + i / 4), columns col + 8j + 2 (i % 4)
// and +1, and r[4j+2], r[4j+3] = lane (base + 8 + i / 4), the same columns.  Four
// consecutive threads hold 8 consecutive columns (32 bytes) of one lane.
__device__ __forceinline__ void tmem_ld_16x256b_x4(uint32_t taddr, uint32_t (&r)[16]) {
    asm volatile(
        "tcgen05.ld.sync.aligned.16x256b.x4.b32 "
        "{%0,%1,%2,%3,%4,%5,%6,%7,%8,%9,%10,%11,%12,%13,%14,%15}, [%16];"
        : "=r"(r[0]), "=r"(r[1]), "=r"(r[2]), "=r"(r[3]), "=r"(r[4]), "=r"(r[5]), "=r"(r[6]),
          "=r"(r[7]), "=r"(r[8]), "=r"(r[9]), "=r"(r[10]), "=r"(r[11]), "=r"(r[12]),
          "=r"(r[13]), "=r"(r[14]), "=r"(r[15])
        : "r"(taddr)
        : "memory");
}
__device__ __forceinline__ void tmem_wait_ld() {
    asm volatile("tcgen05.wait::ld.sync.aligned;" ::: "memory");
}

// Shared-memory matrix descriptor (tcgen05), 128-byte swizzle.
//   bits  0-13 start address >> 4      bits 16-29 leading byte offset >> 4
//   bits 32-45 stride byte offset >> 4 bits 46-47 descriptor version (1)
//   bits 49-51 base offset (0: atoms 1024-byte aligned)   bits 61-63 layout (2 = SW128)
__device__ __forceinline__ uint64_t smem_desc_sw128(uint32_t saddr, uint32_t lbo, uint32_t sbo) {
    uint64_t d = 0;
    d |= static_cast<uint64_t>((saddr & 0x3FFFFu) >> 4);
    d |= static_cast<uint64_t>((lbo >> 4) & 0x3FFFu) << 16;
    d |= static_cast<uint64_t>((sbo >> 4) & 0x3FFFu) << 32;
    d |= static_cast<uint64_t>(1) << 46;
    d |= static_cast<uint64_t>(2) << 61;
    return d;
}

// Instruction descriptor of kind::f16 with bf16 A/B and fp32 D.
//   bits 4-5 D format (1 = f32)   bits 7-9 A format (1 = bf16)  bits 10-12 B format (1 = bf16)
//   bit 15 A major (0 = K)        bit 16 B major (1 = MN)       bits 17-22 N >> 3
//   bits 24-28 M >> 4
__host__ __device__ constexpr uint32_t idesc_bf16_f32(int M, int N, bool a_mn_major,
                                                     bool b_mn_major) {
    return (1u << 4) | (1u << 7) | (1u << 10) | (static_cast<uint32_t>(a_mn_major) << 15) |
           (static_cast<uint32_t>(b_mn_major) << 16) | ((static_cast<uint32_t>(N) >> 3) << 17) |
           ((static_cast<uint32_t>(M) >> 4) << 24);
}

// ------------------------------------------------------------ pair helpers

__device__ __forceinline__ uint32_t cluster_rank() {
    uint32_t r;
    asm volatile("mov.u32 %0, %%cluster_ctarank;" : "=r"(r));
    return r;
}
// Address of the same shared-memory object in CTA `rank` of the cluster.
__device__ __forceinline__ uint32_t peer_addr(uint32_t addr, uint32_t rank) {
    uint32_t r;
    asm volatile("mapa.shared::cluster.u32 %0, %1, %2;" : "=r"(r) : "r"(addr), "r"(rank));
    return r;
}
__device__ __forceinline__ void cluster_sync() {
    asm volatile("barrier.cluster.arrive.release.aligned;\n\tbarrier.cluster.wait.acquire.aligned;" ::
                     : "memory");
}
// 16-byte async-proxy copy from this CTA's shared memory to `dst_cluster` (shared
// memory of a CTA of the cluster) that completes 16 transaction bytes on the
// barrier `bar_cluster` of that CTA.
__device__ __forceinline__ void bulk_signal_remote(uint32_t dst_cluster, uint32_t src,
                                                   uint32_t bar_cluster) {
    asm volatile(
        "cp.async.bulk.shared::cluster.shared::cta.mbarrier::complete_tx::bytes [%0], [%1], 16, [%2];" ::
            "r"(dst_cluster), "r"(src), "r"(bar_cluster)
        : "memory");
}
// Arrival on a barrier of another CTA of the cluster, with the default (CTA-scope)
// release: used where the arriving thread has nothing to publish but completed
// tcgen05.ld reads (ordered by tcgen05 fences around the barrier), so no
// cluster-wide release of its earlier stores is needed.
__device__ __forceinline__ void mbar_arrive_remote(uint32_t bar_cluster) {
    asm volatile("mbarrier.arrive.shared::cluster.b64 _, [%0];" ::"r"(bar_cluster) : "memory");
}
// TMA loads into this CTA's shared memory that complete on a barrier of either CTA
// of the pair.
__device__ __forceinline__ void tma_load_3d_pair(uint32_t dst, const CUtensorMap* tm,
                                                 uint32_t bar_cluster, int c0, int c1, int c2) {
    asm volatile(
        "cp.async.bulk.tensor.3d.cta_group::2.shared::cluster.global.tile.mbarrier::complete_tx::bytes"
        " [%0], [%1, {%2, %3, %4}], [%5];" ::"r"(dst),
        "l"(tm), "r"(c0), "r"(c1), "r"(c2), "r"(bar_cluster)
        : "memory");
}
__device__ __forceinline__ void tma_load_2d_pair(uint32_t dst, const CUtensorMap* tm,
                                                 uint32_t bar_cluster, int c0, int c1) {
    asm volatile(
        "cp.async.bulk.tensor.2d.cta_group::2.shared::cluster.global.tile.mbarrier::complete_tx::bytes"
        " [%0], [%1, {%2, %3}], [%4];" ::"r"(dst),
        "l"(tm), "r"(c0), "r"(c1), "r"(bar_cluster)
        : "memory");
}
__device__ __forceinline__ void tmem_alloc_pair(uint32_t slot, uint32_t ncols) {
    asm volatile("tcgen05.alloc.cta_group::2.sync.aligned.shared::cta.b32 [%0], %1;" ::"r"(slot),
                 "r"(ncols)
                 : "memory");
}
__device__ __forceinline__ void tmem_relinquish_pair() {
    asm volatile("tcgen05.relinquish_alloc_permit.cta_group::2.sync.aligned;" ::: "memory");
}
__device__ __forceinline__ void tmem_dealloc_pair(uint32_t taddr, uint32_t ncols) {
    asm volatile("tcgen05.dealloc.cta_group::2.sync.aligned.b32 %0, %1;" ::"r"(taddr), "r"(ncols)
                 : "memory");
}
__device__ __forceinline__ void tc_mma_bf16_pair(uint32_t d_tmem, uint64_t adesc, uint64_t bdesc,
                                                 uint32_t idesc, uint32_t accumulate) {
    asm volatile(
        "{\n\t.reg .pred p;\n\t"
        "setp.ne.b32 p, %4, 0;\n\t"
        "tcgen05.mma.cta_group::2.kind::f16 [%0], %1, %2, %3, p;\n\t}" ::"r"(d_tmem),
        "l"(adesc), "l"(bdesc), "r"(idesc), "r"(accumulate)
        : "memory");
}
// Arrive once on the barrier at shared offset `bar` of both CTAs when all prior
// tcgen05 operations of this thread have completed.
__device__ __forceinline__ void tc_commit_pair(uint32_t bar) {
    asm volatile(
        "tcgen05.commit.cta_group::2.mbarrier::arrive::one.shared::cluster.multicast::cluster.b64"
        " [%0], %1;" ::"r"(bar),
        "h"((uint16_t)3)
        : "memory");
}

// -------------------------------------------------------------- bf16 pack

__device__ __forceinline__ uint32_t pack_bf16x2(float lo, float hi) {
    __nv_bfloat162 v = __floats2bfloat162_rn(lo, hi);
    return *reinterpret_cast<uint32_t*>(&v);
}
// Packed pairs of fp32 values (one 64-bit register pair) and the sm_100-family
// two-wide fp32 arithmetic on them: one instruction does the work of two.
__device__ __forceinline__ uint64_t f2_pack(float a, float b) {
    uint64_t r;
    asm("mov.b64 %0, {%1, %2};" : "=l"(r) : "f"(a), "f"(b));
    return r;
}
__device__ __forceinline__ void f2_unpack(uint64_t r, float& a, float& b) {
    asm("mov.b64 {%0, %1}, %2;" : "=f"(a), "=f"(b) : "l"(r));
}
__device__ __forceinline__ uint64_t f2_mul(uint64_t a, uint64_t b) {
    uint64_t d;
    asm("mul.rn.f32x2 %0, %1, %2;" : "=l"(d) : "l"(a), "l"(b));
    return d;
}
__device__ __forceinline__ uint64_t f2_fma(uint64_t a, uint64_t b, uint64_t c) {
    uint64_t d;
    asm("fma.rn.f32x2 %0, %1, %2, %3;" : "=l"(d) : "l"(a), "l"(b), "l"(c));
    return d;
}
__device__ __forceinline__ float rcp_approx(float x) {
    float r;
    asm("rcp.approx.ftz.f32 %0, %1;" : "=f"(r) : "f"(x));
    return r;
}

// GELU(u) = u/2 (1 + erf(u / sqrt 2)) = max(u, 0) - |u|/2 erfc(|u| / sqrt 2), the
// second form free of the cancellation of 1 + erf for u < 0.  erfc from Abramowitz &
// Stegun 7.1.28: erfc(z) = (1 + a1 z + a2 z^2 + ... + a6 z^6)^-16 for z >= 0, with
// |error| <= 3e-7 (one reciprocal and no exponential; the sixteenth power by four
// squarings, which overflow to +inf, and so to erfc = 0, only where erfc is far
// below fp32 resolution).  Evaluated in fp32 the GELU error stays below 1e-6 in
// absolute value; the hidden activation is then rounded to bf16 (2^-9 relative).
// Two values at a time with the packed fp32x2 instructions.
__device__ __forceinline__ void erfc_as2(float a0, float a1, float& q0, float& q1) {   // a0, a1 >= 0
    const uint64_t z = f2_mul(f2_pack(a0, a1), f2_pack(0.70710678118654752f, 0.70710678118654752f));
    uint64_t P = f2_fma(z, f2_pack(0.0000430638f, 0.0000430638f), f2_pack(0.0002765672f, 0.0002765672f));
    P = f2_fma(P, z, f2_pack(0.0001520143f, 0.0001520143f));
    P = f2_fma(P, z, f2_pack(0.0092705272f, 0.0092705272f));
    P = f2_fma(P, z, f2_pack(0.0422820123f, 0.0422820123f));
    P = f2_fma(P, z, f2_pack(0.0705230784f, 0.0705230784f));
    P = f2_fma(P, z, f2_pack(1.0f, 1.0f));
    P = f2_mul(P, P);
    P = f2_mul(P, P);
    P = f2_mul(P, P);
    P = f2_mul(P, P);
    float p0, p1;
    f2_unpack(P, p0, p1);
    q0 = rcp_approx(p0);
    q1 = rcp_approx(p1);
}

__device__ __forceinline__ void gelu_erf2(float& u0, float& u1) {
    float q0, q1;
    erfc_as2(fabsf(u0), fabsf(u1), q0, q1);
    const uint64_t r = f2_fma(f2_mul(f2_pack(fabsf(u0), fabsf(u1)), f2_pack(-0.5f, -0.5f)), f2_pack(q0, q1),
                              f2_pack(fmaxf(u0, 0.0f), fmaxf(u1, 0.0f)));
    f2_unpack(r, u0, u1);
}

__device__ __forceinline__ void unpack_bf16x8(const uint4& u, float (&v)[8]) {
    const __nv_bfloat162* p = reinterpret_cast<const __nv_bfloat162*>(&u);
#pragma unroll
    for (int i = 0; i < 4; ++i) {
        float2 f = __bfloat1622float2(p[i]);
        v[2 * i] = f.x;
        v[2 * i + 1] = f.y;
    }
}

}  // namespace mv
