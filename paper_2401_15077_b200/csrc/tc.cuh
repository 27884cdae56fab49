// Tensor-core, tensor-memory, TMA and mbarrier instructions of sm_100a as inline functions, for kernels whose CTAs work in
// pairs (chunk.cu, window.cu), and the host functions that encode their tensor maps.
#pragma once
#include <cuda.h>
#include <cuda_bf16.h>
#include <stdint.h>

namespace eagle {
namespace tc {

__device__ __forceinline__ uint32_t smem_u32(const void* p) { return static_cast<uint32_t>(__cvta_generic_to_shared(p)); }

// ------------------------------------------------------------------------------------------------ mbarriers, bounded waits
__device__ __forceinline__ void mbar_init(uint32_t bar, uint32_t count) {
  asm volatile("mbarrier.init.shared::cta.b64 [%0], %1;" ::"r"(bar), "r"(count) : "memory");
}
__device__ __forceinline__ void mbar_arrive(uint32_t bar) {
  asm volatile("mbarrier.arrive.shared::cta.b64 _, [%0];" ::"r"(bar) : "memory");
}
// The address of the other CTA's (or one's own) shared memory, for arrivals across the pair.
__device__ __forceinline__ uint32_t map_to_rank(uint32_t addr, uint32_t rank) {
  uint32_t r;
  asm volatile("mapa.shared::cluster.u32 %0, %1, %2;" : "=r"(r) : "r"(addr), "r"(rank));
  return r;
}
// An arrival at either CTA's barrier.  Copies and tensor memory are ordered by their own completion and fences, so the plain
// form will do; the form with cluster scope is for ordinary stores to shared memory (it waits for all of the thread's memory
// operations: 1300 cycles, more than a step of the attention kernel).
__device__ __forceinline__ void mbar_arrive_pair(uint32_t bar) {
  asm volatile("mbarrier.arrive.shared::cluster.b64 _, [%0];" ::"r"(bar) : "memory");
}
__device__ __forceinline__ void mbar_arrive_release_pair(uint32_t bar) {
  asm volatile("mbarrier.arrive.release.cluster.shared::cluster.b64 _, [%0];" ::"r"(bar) : "memory");
}
__device__ __forceinline__ uint32_t cluster_rank() {
  uint32_t r;
  asm volatile("mov.u32 %0, %%cluster_ctarank;" : "=r"(r));
  return r;
}
__device__ __forceinline__ void cluster_sync() {
  asm volatile("barrier.cluster.arrive.release.aligned;\n\tbarrier.cluster.wait.acquire.aligned;" ::: "memory");
}
__device__ __forceinline__ void mbar_expect_tx(uint32_t bar, uint32_t bytes) {
  asm volatile("mbarrier.arrive.expect_tx.shared::cta.b64 _, [%0], %1;" ::"r"(bar), "r"(bytes) : "memory");
}
__device__ __forceinline__ bool mbar_try_wait(uint32_t bar, uint32_t parity) {
  uint32_t ok;
  asm volatile(
      "{\n\t.reg .pred p;\n\tmbarrier.try_wait.parity.shared::cta.b64 p, [%1], %2;\n\tselp.u32 %0, 1, 0, p;\n\t}"
      : "=r"(ok) : "r"(bar), "r"(parity) : "memory");
  return ok != 0;
}
__device__ __forceinline__ unsigned long long global_timer() {
  unsigned long long t;
  asm volatile("mov.u64 %0, %%globaltimer;" : "=l"(t));
  return t;
}
// Every wait gives up after the limit that the host set (it sits in shared memory right behind the abort flag), raises
// the flag and returns false; so does every other wait of the CTA from then on.
static __device__ __noinline__ bool mbar_wait_slow(uint32_t bar, uint32_t parity, volatile int* abort_flag) {
  const unsigned long long t0 = global_timer(), limit = *reinterpret_cast<volatile unsigned long long*>(abort_flag + 1);
  for (uint32_t spins = 1;; ++spins) {
    if (mbar_try_wait(bar, parity)) return true;
    if ((spins & 63u) == 0) {
      if (*abort_flag) return false;
      if (global_timer() - t0 > limit) {
        *abort_flag = 1;
        return false;
      }
    }
  }
}
__device__ __forceinline__ bool mbar_wait(uint32_t bar, uint32_t parity, volatile int* abort_flag) {
  if (mbar_try_wait(bar, parity)) return true;     // (a suspended wait: polling would take issue slots from the warps that work)
  return mbar_wait_slow(bar, parity, abort_flag);
}
// After an abort: copies and MMAs that the CTA has issued may still be at work on its shared and tensor memory.  They take
// microseconds; this waits a hundred before it may leave.
static __device__ __noinline__ void let_work_land() {
  const unsigned long long t0 = global_timer();
  while (global_timer() - t0 < 100000ull) __nanosleep(1000);
}
// A wait for arrivals with release at cluster scope, whose senders' stores to their own shared memory are to be seen by what follows.
__device__ __forceinline__ bool mbar_try_wait_cluster(uint32_t bar, uint32_t parity) {
  uint32_t ok;
  asm volatile(
      "{\n\t.reg .pred p;\n\tmbarrier.try_wait.parity.acquire.cluster.shared::cta.b64 p, [%1], %2;\n\tselp.u32 %0, 1, 0, p;\n\t}"
      : "=r"(ok) : "r"(bar), "r"(parity) : "memory");
  return ok != 0;
}
__device__ __forceinline__ bool mbar_wait_cluster(uint32_t bar, uint32_t parity, volatile int* abort_flag) {
  if (mbar_try_wait_cluster(bar, parity)) return true;
  return mbar_wait_slow(bar, parity, abort_flag) && mbar_try_wait_cluster(bar, parity);      // (the phase is over: the second try succeeds at once)
}
// mbar_wait with a verdict that is uniform over the warp (the callers go on to warp-collective instructions).
__device__ __forceinline__ bool mbar_wait_warp(uint32_t bar, uint32_t parity, volatile int* abort_flag) {
  return __all_sync(0xffffffffu, mbar_wait(bar, parity, abort_flag));
}

// ------------------------------------------------------------------------------------------------ words with numbers
// A float with a number, written and read in one piece.
__device__ __forceinline__ unsigned long long tagged(uint32_t number, float x) { return static_cast<unsigned long long>(number) << 32 | __float_as_uint(x); }
__device__ __forceinline__ float value_of(unsigned long long t) { return __uint_as_float(static_cast<uint32_t>(t)); }
__device__ __forceinline__ bool has_tag(unsigned long long t, uint32_t want) { return static_cast<uint32_t>(t >> 32) == want; }
// Bounded wait for the word with number `want` in shared memory; one with another number when the CTA was aborted or the time
// limit passed.
static __device__ __noinline__ unsigned long long tag_wait_slow(volatile unsigned long long* slot, uint32_t want, volatile int* abort_flag) {
  const unsigned long long t0 = global_timer(), limit = *reinterpret_cast<volatile unsigned long long*>(abort_flag + 1);
  for (uint32_t spins = 1;; ++spins) {
    const unsigned long long t = *slot;
    if (has_tag(t, want)) return t;
    if ((spins & 63u) == 0) {
      if (*abort_flag) return tagged(~want, 0.f);
      if (global_timer() - t0 > limit) {
        *abort_flag = 1;
        return tagged(~want, 0.f);
      }
    }
    __nanosleep(20);
  }
}
__device__ __forceinline__ unsigned long long tag_wait(volatile unsigned long long* slot, uint32_t want, volatile int* abort_flag) {
  const unsigned long long t = *slot;
  if (has_tag(t, want)) return t;
  return tag_wait_slow(slot, want, abort_flag);
}

// Counts steps through a ring of N slots: the slot of the next step, and the parity of its use.
template <int N>
struct Ring {
  uint32_t slot = 0, par = 0;
  __device__ __forceinline__ void step() {
    if (++slot == N) { slot = 0; par ^= 1u; }
  }
};

// ------------------------------------------------------------------------------------------------ fences, commits, copies
__device__ __forceinline__ void fence_proxy_async() { asm volatile("fence.proxy.async.shared::cta;" ::: "memory"); }
__device__ __forceinline__ void fence_before() { asm volatile("tcgen05.fence::before_thread_sync;" ::: "memory"); }
__device__ __forceinline__ void fence_after() { asm volatile("tcgen05.fence::after_thread_sync;" ::: "memory"); }
__device__ __forceinline__ void wait_ld() { asm volatile("tcgen05.wait::ld.sync.aligned;" ::: "memory"); }
__device__ __forceinline__ void wait_st() { asm volatile("tcgen05.wait::st.sync.aligned;" ::: "memory"); }
// Arrives on the barrier of both CTAs of the pair when every MMA that this thread has issued so far has finished.
__device__ __forceinline__ void commit_pair(uint32_t bar) {
  asm volatile("tcgen05.commit.cta_group::2.mbarrier::arrive::one.shared::cluster.multicast::cluster.b64 [%0], %1;"
               ::"r"(bar), "h"(static_cast<uint16_t>(3)) : "memory");
}
__device__ __forceinline__ void tma_load_3d(uint32_t dst, const CUtensorMap* map, int x, int y, int z, uint32_t bar) {
  asm volatile(
      "cp.async.bulk.tensor.3d.shared::cluster.global.mbarrier::complete_tx::bytes [%0], [%1, {%2, %3, %4}], [%5];"
      ::"r"(dst), "l"(reinterpret_cast<uint64_t>(map)), "r"(x), "r"(y), "r"(z), "r"(bar) : "memory");
}
// The same, with a barrier that may lie in the other CTA of the pair.
__device__ __forceinline__ void tma_load_3d_pair(uint32_t dst, const CUtensorMap* map, int x, int y, int z, uint32_t bar) {
  asm volatile(
      "cp.async.bulk.tensor.3d.cta_group::2.shared::cluster.global.mbarrier::complete_tx::bytes [%0], [%1, {%2, %3, %4}], [%5];"
      ::"r"(dst), "l"(reinterpret_cast<uint64_t>(map)), "r"(x), "r"(y), "r"(z), "r"(bar) : "memory");
}
__device__ __forceinline__ void prefetch_map(const CUtensorMap* map) {
  asm volatile("prefetch.tensormap [%0];" ::"l"(reinterpret_cast<uint64_t>(map)) : "memory");
}
// One 32-byte store (the address must be 32-byte aligned).
__device__ __forceinline__ void st_global_v8(void* dst, const uint32_t* v) {
  asm volatile("st.global.v8.b32 [%0], {%1, %2, %3, %4, %5, %6, %7, %8};" ::"l"(dst), "r"(v[0]), "r"(v[1]), "r"(v[2]), "r"(v[3]),
               "r"(v[4]), "r"(v[5]), "r"(v[6]), "r"(v[7]) : "memory");
}

// Programmatic launches: the next kernel of the stream may start its prologue from here on / waits until the kernel before it
// has finished and its stores are visible.
__device__ __forceinline__ void launch_dependents() { asm volatile("griddepcontrol.launch_dependents;" ::: "memory"); }
__device__ __forceinline__ void wait_for_prerequisites() { asm volatile("griddepcontrol.wait;" ::: "memory"); }

// ------------------------------------------------------------------------------------------------ tensor memory
__device__ __forceinline__ void ld32(uint32_t addr, uint32_t* r) {
  asm volatile(
      "tcgen05.ld.sync.aligned.32x32b.x32.b32 "
      "{%0,%1,%2,%3,%4,%5,%6,%7,%8,%9,%10,%11,%12,%13,%14,%15,%16,%17,%18,%19,%20,%21,%22,%23,%24,%25,%26,%27,%28,%29,%30,%31}, [%32];"
      : "=r"(r[0]), "=r"(r[1]), "=r"(r[2]), "=r"(r[3]), "=r"(r[4]), "=r"(r[5]), "=r"(r[6]), "=r"(r[7]), "=r"(r[8]), "=r"(r[9]),
        "=r"(r[10]), "=r"(r[11]), "=r"(r[12]), "=r"(r[13]), "=r"(r[14]), "=r"(r[15]), "=r"(r[16]), "=r"(r[17]), "=r"(r[18]),
        "=r"(r[19]), "=r"(r[20]), "=r"(r[21]), "=r"(r[22]), "=r"(r[23]), "=r"(r[24]), "=r"(r[25]), "=r"(r[26]), "=r"(r[27]),
        "=r"(r[28]), "=r"(r[29]), "=r"(r[30]), "=r"(r[31])
      : "r"(addr) : "memory");
}
__device__ __forceinline__ void ld16(uint32_t addr, uint32_t* r) {
  asm volatile(
      "tcgen05.ld.sync.aligned.32x32b.x16.b32 {%0,%1,%2,%3,%4,%5,%6,%7,%8,%9,%10,%11,%12,%13,%14,%15}, [%16];"
      : "=r"(r[0]), "=r"(r[1]), "=r"(r[2]), "=r"(r[3]), "=r"(r[4]), "=r"(r[5]), "=r"(r[6]), "=r"(r[7]), "=r"(r[8]), "=r"(r[9]),
        "=r"(r[10]), "=r"(r[11]), "=r"(r[12]), "=r"(r[13]), "=r"(r[14]), "=r"(r[15])
      : "r"(addr) : "memory");
}
__device__ __forceinline__ void st8(uint32_t addr, const uint32_t* r) {
  asm volatile(
      "tcgen05.st.sync.aligned.32x32b.x8.b32 [%0], {%1,%2,%3,%4,%5,%6,%7,%8};"
      ::"r"(addr), "r"(r[0]), "r"(r[1]), "r"(r[2]), "r"(r[3]), "r"(r[4]), "r"(r[5]), "r"(r[6]), "r"(r[7])
      : "memory");
}
__device__ __forceinline__ void st32(uint32_t addr, const uint32_t* r) {
  asm volatile(
      "tcgen05.st.sync.aligned.32x32b.x32.b32 [%0], "
      "{%1,%2,%3,%4,%5,%6,%7,%8,%9,%10,%11,%12,%13,%14,%15,%16,%17,%18,%19,%20,%21,%22,%23,%24,%25,%26,%27,%28,%29,%30,%31,%32};"
      ::"r"(addr), "r"(r[0]), "r"(r[1]), "r"(r[2]), "r"(r[3]), "r"(r[4]), "r"(r[5]), "r"(r[6]), "r"(r[7]), "r"(r[8]), "r"(r[9]),
        "r"(r[10]), "r"(r[11]), "r"(r[12]), "r"(r[13]), "r"(r[14]), "r"(r[15]), "r"(r[16]), "r"(r[17]), "r"(r[18]), "r"(r[19]),
        "r"(r[20]), "r"(r[21]), "r"(r[22]), "r"(r[23]), "r"(r[24]), "r"(r[25]), "r"(r[26]), "r"(r[27]), "r"(r[28]), "r"(r[29]),
        "r"(r[30]), "r"(r[31])
      : "memory");
}
__device__ __forceinline__ void st16(uint32_t addr, const uint32_t* r) {
  asm volatile(
      "tcgen05.st.sync.aligned.32x32b.x16.b32 [%0], {%1,%2,%3,%4,%5,%6,%7,%8,%9,%10,%11,%12,%13,%14,%15,%16};"
      ::"r"(addr), "r"(r[0]), "r"(r[1]), "r"(r[2]), "r"(r[3]), "r"(r[4]), "r"(r[5]), "r"(r[6]), "r"(r[7]), "r"(r[8]), "r"(r[9]),
        "r"(r[10]), "r"(r[11]), "r"(r[12]), "r"(r[13]), "r"(r[14]), "r"(r[15])
      : "memory");
}

// ------------------------------------------------------------------------------------------------ MMAs
// kind::f16 instruction descriptor: bf16 x bf16 -> fp32, A K-major, B K-major or MN-major.
__host__ __device__ constexpr uint32_t instr_desc(int M, int N, bool b_mn_major) {
  return (1u << 4) | (1u << 7) | (1u << 10) | (b_mn_major ? (1u << 16) : 0u) | (static_cast<uint32_t>(N >> 3) << 17) |
         (static_cast<uint32_t>(M >> 4) << 24);
}
// The same for fp16 x fp16 -> fp32.
__host__ __device__ constexpr uint32_t instr_desc_half(int M, int N, bool b_mn_major) {
  return (1u << 4) | (b_mn_major ? (1u << 16) : 0u) | (static_cast<uint32_t>(N >> 3) << 17) | (static_cast<uint32_t>(M >> 4) << 24);
}
// Shared-memory descriptor of a swizzled tile.  Low word: start address and leading-dimension offset, so stepping along the
// contraction is a 32-bit add; high word: stride of 8-row groups, version, swizzle (128-byte rows, or 64-byte rows).
constexpr uint32_t kDescHi128 = (1024u >> 4) | (1u << 14) | (2u << 29);
constexpr uint32_t kDescHi64 = (512u >> 4) | (1u << 14) | (4u << 29);
__device__ __forceinline__ uint32_t desc_lo(uint32_t addr) { return ((addr >> 4) & 0x3fffu) | (1u << 16); }

// The MMAs of a pair of CTAs (M = 256: 128 rows of each CTA; each holds half of B's N extent), one asm block per tile, so that
// little but the MMAs stands in the issuing thread's way.
// S[256 x 128] = Q[256 x D] K[128 x D]^T: Q 128 rows and K 64 rows per CTA, 128-byte rows, 64 columns to a slab (16 KB and 8 KB).
template <int D>
__device__ __forceinline__ void issue_qk_pair(uint32_t d_tmem, uint32_t q_lo, uint32_t k_lo, uint32_t idesc) {
  if constexpr (D == 128) {
    asm volatile(
      "{\n\t.reg .pred p;\n\t.reg .b64 da, db;\n\t.reg .b32 ta, tb;\n\t"
      "add.u32 ta, %1, 0;\n\tadd.u32 tb, %2, 0;\n\tmov.b64 da, {ta, %4};\n\tmov.b64 db, {tb, %4};\n\t"
      "setp.ne.b32 p, 0, 0;\n\ttcgen05.mma.cta_group::2.kind::f16 [%0], da, db, %3, p;\n\t"
      "add.u32 ta, %1, 2;\n\tadd.u32 tb, %2, 2;\n\tmov.b64 da, {ta, %4};\n\tmov.b64 db, {tb, %4};\n\t"
      "setp.ne.b32 p, 1, 0;\n\ttcgen05.mma.cta_group::2.kind::f16 [%0], da, db, %3, p;\n\t"
      "add.u32 ta, %1, 4;\n\tadd.u32 tb, %2, 4;\n\tmov.b64 da, {ta, %4};\n\tmov.b64 db, {tb, %4};\n\t"
      "setp.ne.b32 p, 1, 0;\n\ttcgen05.mma.cta_group::2.kind::f16 [%0], da, db, %3, p;\n\t"
      "add.u32 ta, %1, 6;\n\tadd.u32 tb, %2, 6;\n\tmov.b64 da, {ta, %4};\n\tmov.b64 db, {tb, %4};\n\t"
      "setp.ne.b32 p, 1, 0;\n\ttcgen05.mma.cta_group::2.kind::f16 [%0], da, db, %3, p;\n\t"
      "add.u32 ta, %1, 1024;\n\tadd.u32 tb, %2, 512;\n\tmov.b64 da, {ta, %4};\n\tmov.b64 db, {tb, %4};\n\t"
      "setp.ne.b32 p, 1, 0;\n\ttcgen05.mma.cta_group::2.kind::f16 [%0], da, db, %3, p;\n\t"
      "add.u32 ta, %1, 1026;\n\tadd.u32 tb, %2, 514;\n\tmov.b64 da, {ta, %4};\n\tmov.b64 db, {tb, %4};\n\t"
      "setp.ne.b32 p, 1, 0;\n\ttcgen05.mma.cta_group::2.kind::f16 [%0], da, db, %3, p;\n\t"
      "add.u32 ta, %1, 1028;\n\tadd.u32 tb, %2, 516;\n\tmov.b64 da, {ta, %4};\n\tmov.b64 db, {tb, %4};\n\t"
      "setp.ne.b32 p, 1, 0;\n\ttcgen05.mma.cta_group::2.kind::f16 [%0], da, db, %3, p;\n\t"
      "add.u32 ta, %1, 1030;\n\tadd.u32 tb, %2, 518;\n\tmov.b64 da, {ta, %4};\n\tmov.b64 db, {tb, %4};\n\t"
      "setp.ne.b32 p, 1, 0;\n\ttcgen05.mma.cta_group::2.kind::f16 [%0], da, db, %3, p;\n\t"
      "}"
      ::"r"(d_tmem), "r"(q_lo), "r"(k_lo), "r"(idesc), "r"(kDescHi128) : "memory");
  } else {
    asm volatile(
      "{\n\t.reg .pred p;\n\t.reg .b64 da, db;\n\t.reg .b32 ta, tb;\n\t"
      "add.u32 ta, %1, 0;\n\tadd.u32 tb, %2, 0;\n\tmov.b64 da, {ta, %4};\n\tmov.b64 db, {tb, %4};\n\t"
      "setp.ne.b32 p, 0, 0;\n\ttcgen05.mma.cta_group::2.kind::f16 [%0], da, db, %3, p;\n\t"
      "add.u32 ta, %1, 2;\n\tadd.u32 tb, %2, 2;\n\tmov.b64 da, {ta, %4};\n\tmov.b64 db, {tb, %4};\n\t"
      "setp.ne.b32 p, 1, 0;\n\ttcgen05.mma.cta_group::2.kind::f16 [%0], da, db, %3, p;\n\t"
      "add.u32 ta, %1, 4;\n\tadd.u32 tb, %2, 4;\n\tmov.b64 da, {ta, %4};\n\tmov.b64 db, {tb, %4};\n\t"
      "setp.ne.b32 p, 1, 0;\n\ttcgen05.mma.cta_group::2.kind::f16 [%0], da, db, %3, p;\n\t"
      "add.u32 ta, %1, 6;\n\tadd.u32 tb, %2, 6;\n\tmov.b64 da, {ta, %4};\n\tmov.b64 db, {tb, %4};\n\t"
      "setp.ne.b32 p, 1, 0;\n\ttcgen05.mma.cta_group::2.kind::f16 [%0], da, db, %3, p;\n\t"
      "}"
      ::"r"(d_tmem), "r"(q_lo), "r"(k_lo), "r"(idesc), "r"(kDescHi128) : "memory");
  }
}
// O[256 x D] (+)= P[256 x 128] V[128 x D]: P from tensor memory (8 columns per MMA), V 128 keys x D / 2 columns per CTA (rows of
// 128 or 64 bytes, 16 keys per MMA).
template <int D>
__device__ __forceinline__ void issue_pv_pair(uint32_t o_tmem, uint32_t p_tmem, uint32_t v_lo, uint32_t idesc, uint32_t acc0) {
  if constexpr (D == 128) {
    asm volatile(
      "{\n\t.reg .pred p;\n\t.reg .b64 db;\n\t.reg .b32 ta, tb;\n\t"
      "add.u32 ta, %1, 0;\n\tadd.u32 tb, %2, 0;\n\tmov.b64 db, {tb, %4};\n\t"
      "setp.ne.b32 p, %5, 0;\n\ttcgen05.mma.cta_group::2.kind::f16 [%0], [ta], db, %3, p;\n\t"
      "add.u32 ta, %1, 8;\n\tadd.u32 tb, %2, 128;\n\tmov.b64 db, {tb, %4};\n\t"
      "setp.ne.b32 p, 1, 0;\n\ttcgen05.mma.cta_group::2.kind::f16 [%0], [ta], db, %3, p;\n\t"
      "add.u32 ta, %1, 16;\n\tadd.u32 tb, %2, 256;\n\tmov.b64 db, {tb, %4};\n\t"
      "setp.ne.b32 p, 1, 0;\n\ttcgen05.mma.cta_group::2.kind::f16 [%0], [ta], db, %3, p;\n\t"
      "add.u32 ta, %1, 24;\n\tadd.u32 tb, %2, 384;\n\tmov.b64 db, {tb, %4};\n\t"
      "setp.ne.b32 p, 1, 0;\n\ttcgen05.mma.cta_group::2.kind::f16 [%0], [ta], db, %3, p;\n\t"
      "add.u32 ta, %1, 32;\n\tadd.u32 tb, %2, 512;\n\tmov.b64 db, {tb, %4};\n\t"
      "setp.ne.b32 p, 1, 0;\n\ttcgen05.mma.cta_group::2.kind::f16 [%0], [ta], db, %3, p;\n\t"
      "add.u32 ta, %1, 40;\n\tadd.u32 tb, %2, 640;\n\tmov.b64 db, {tb, %4};\n\t"
      "setp.ne.b32 p, 1, 0;\n\ttcgen05.mma.cta_group::2.kind::f16 [%0], [ta], db, %3, p;\n\t"
      "add.u32 ta, %1, 48;\n\tadd.u32 tb, %2, 768;\n\tmov.b64 db, {tb, %4};\n\t"
      "setp.ne.b32 p, 1, 0;\n\ttcgen05.mma.cta_group::2.kind::f16 [%0], [ta], db, %3, p;\n\t"
      "add.u32 ta, %1, 56;\n\tadd.u32 tb, %2, 896;\n\tmov.b64 db, {tb, %4};\n\t"
      "setp.ne.b32 p, 1, 0;\n\ttcgen05.mma.cta_group::2.kind::f16 [%0], [ta], db, %3, p;\n\t"
      "}"
      ::"r"(o_tmem), "r"(p_tmem), "r"(v_lo), "r"(idesc), "r"(kDescHi128), "r"(acc0) : "memory");
  } else {
    asm volatile(
      "{\n\t.reg .pred p;\n\t.reg .b64 db;\n\t.reg .b32 ta, tb;\n\t"
      "add.u32 ta, %1, 0;\n\tadd.u32 tb, %2, 0;\n\tmov.b64 db, {tb, %4};\n\t"
      "setp.ne.b32 p, %5, 0;\n\ttcgen05.mma.cta_group::2.kind::f16 [%0], [ta], db, %3, p;\n\t"
      "add.u32 ta, %1, 8;\n\tadd.u32 tb, %2, 64;\n\tmov.b64 db, {tb, %4};\n\t"
      "setp.ne.b32 p, 1, 0;\n\ttcgen05.mma.cta_group::2.kind::f16 [%0], [ta], db, %3, p;\n\t"
      "add.u32 ta, %1, 16;\n\tadd.u32 tb, %2, 128;\n\tmov.b64 db, {tb, %4};\n\t"
      "setp.ne.b32 p, 1, 0;\n\ttcgen05.mma.cta_group::2.kind::f16 [%0], [ta], db, %3, p;\n\t"
      "add.u32 ta, %1, 24;\n\tadd.u32 tb, %2, 192;\n\tmov.b64 db, {tb, %4};\n\t"
      "setp.ne.b32 p, 1, 0;\n\ttcgen05.mma.cta_group::2.kind::f16 [%0], [ta], db, %3, p;\n\t"
      "add.u32 ta, %1, 32;\n\tadd.u32 tb, %2, 256;\n\tmov.b64 db, {tb, %4};\n\t"
      "setp.ne.b32 p, 1, 0;\n\ttcgen05.mma.cta_group::2.kind::f16 [%0], [ta], db, %3, p;\n\t"
      "add.u32 ta, %1, 40;\n\tadd.u32 tb, %2, 320;\n\tmov.b64 db, {tb, %4};\n\t"
      "setp.ne.b32 p, 1, 0;\n\ttcgen05.mma.cta_group::2.kind::f16 [%0], [ta], db, %3, p;\n\t"
      "add.u32 ta, %1, 48;\n\tadd.u32 tb, %2, 384;\n\tmov.b64 db, {tb, %4};\n\t"
      "setp.ne.b32 p, 1, 0;\n\ttcgen05.mma.cta_group::2.kind::f16 [%0], [ta], db, %3, p;\n\t"
      "add.u32 ta, %1, 56;\n\tadd.u32 tb, %2, 448;\n\tmov.b64 db, {tb, %4};\n\t"
      "setp.ne.b32 p, 1, 0;\n\ttcgen05.mma.cta_group::2.kind::f16 [%0], [ta], db, %3, p;\n\t"
      "}"
      ::"r"(o_tmem), "r"(p_tmem), "r"(v_lo), "r"(idesc), "r"(kDescHi64), "r"(acc0) : "memory");
  }
}

// ------------------------------------------------------------------------------------------------ arithmetic
__device__ __forceinline__ float fast_exp2(float x) {
  float y;
  asm("ex2.approx.ftz.f32 %0, %1;" : "=f"(y) : "f"(x));
  return y;
}
// Packed pairs of floats and the two-wide FP32 instructions: one issue slot does the work of two.
__device__ __forceinline__ uint64_t pack2(float lo, float hi) {
  uint64_t r;
  asm("mov.b64 %0, {%1, %2};" : "=l"(r) : "f"(lo), "f"(hi));
  return r;
}
__device__ __forceinline__ void unpack2(uint64_t v, float& lo, float& hi) { asm("mov.b64 {%0, %1}, %2;" : "=f"(lo), "=f"(hi) : "l"(v)); }
__device__ __forceinline__ uint64_t fma2(uint64_t a, uint64_t b, uint64_t c) {
  uint64_t d;
  asm("fma.rn.f32x2 %0, %1, %2, %3;" : "=l"(d) : "l"(a), "l"(b), "l"(c));
  return d;
}
__device__ __forceinline__ uint64_t add2(uint64_t a, uint64_t b) {
  uint64_t d;
  asm("add.rn.f32x2 %0, %1, %2;" : "=l"(d) : "l"(a), "l"(b));
  return d;
}
__device__ __forceinline__ float max3(float a, float b, float c) {
  float d;
  asm("max.f32 %0, %1, %2, %3;" : "=f"(d) : "f"(a), "f"(b), "f"(c));
  return d;
}
// The same, but NaN when one of them is.
__device__ __forceinline__ float max3_nan(float a, float b, float c) {
  float d;
  asm("max.NaN.f32 %0, %1, %2, %3;" : "=f"(d) : "f"(a), "f"(b), "f"(c));
  return d;
}
// 2^x of a pair on the FMA and integer pipes (x <= ~8): x = n + f with n whole and f in [-1/2, 1/2] (adding and taking off
// 1.5 * 2^23 rounds to a whole number), a cubic for 2^f fitted over that interval (relative error 1e-4, well below the bf16
// rounding of what it is used for), n added to the exponent field.  At -127 and below, -inf among them, the sum is exactly 0 (f = 0,
// 2^f = 1, and n takes its whole exponent away); between -127 and -126 it is some number from 0 to 2^-126.  A NaN comes out as 0:
// the caller looks for those.
__device__ __forceinline__ void poly_exp2_pair(uint64_t x2, float& p0, float& p1) {
  float a, b;
  unpack2(x2, a, b);
  const uint64_t xc = pack2(fmaxf(a, -127.f), fmaxf(b, -127.f));
  const uint64_t t2 = add2(xc, pack2(12582912.f, 12582912.f));
  const uint64_t u2 = add2(t2, pack2(-12582912.f, -12582912.f));
  const uint64_t f2 = fma2(u2, pack2(-1.f, -1.f), xc);
  uint64_t r2 = fma2(pack2(0.05500841f, 0.05500841f), f2, pack2(0.24220926f, 0.24220926f));
  r2 = fma2(r2, f2, pack2(0.69328277f, 0.69328277f));
  r2 = fma2(r2, f2, pack2(1.0f, 1.0f));
  float ta, tb, ra, rb;
  unpack2(t2, ta, tb);
  unpack2(r2, ra, rb);
  p0 = __uint_as_float(__float_as_uint(ta) * 0x800000u + __float_as_uint(ra));   // the constant's own bits shift out
  p1 = __uint_as_float(__float_as_uint(tb) * 0x800000u + __float_as_uint(rb));
}
__device__ __forceinline__ uint32_t pack_bf16(float lo, float hi) {
  __nv_bfloat162 v = __floats2bfloat162_rn(lo, hi);
  return *reinterpret_cast<uint32_t*>(&v);
}

// ------------------------------------------------------------------------------------------------ tensor maps (host)
typedef CUresult (*EncodeTiledFn)(CUtensorMap*, CUtensorMapDataType, cuuint32_t, void*, const cuuint64_t*, const cuuint64_t*,
                                  const cuuint32_t*, const cuuint32_t*, CUtensorMapInterleave, CUtensorMapSwizzle,
                                  CUtensorMapL2promotion, CUtensorMapFloatOOBfill);
inline EncodeTiledFn encode_fn() {
  static EncodeTiledFn fn = [] {
    void* f = nullptr;
    cudaDriverEntryPointQueryResult q;
    if (cudaGetDriverEntryPoint("cuTensorMapEncodeTiled", &f, cudaEnableDefault, &q) != cudaSuccess || q != cudaDriverEntryPointSuccess)
      f = nullptr;
    return reinterpret_cast<EncodeTiledFn>(f);
  }();
  return fn;
}
// A dense bf16 tensor [n2, n1, D] read in boxes of b2 x b1 rows by `cols` columns (64: 128-byte swizzle, 32: 64-byte swizzle).
inline bool map_bf16_3d(CUtensorMap* map, const void* base, int D, long long n1, long long n2, int cols, int b1, int b2) {
  EncodeTiledFn fn = encode_fn();
  if (!fn) return false;
  const cuuint64_t dims[3] = {static_cast<cuuint64_t>(D), static_cast<cuuint64_t>(n1), static_cast<cuuint64_t>(n2)};
  const cuuint64_t strides[2] = {static_cast<cuuint64_t>(D) * 2, static_cast<cuuint64_t>(n1) * D * 2};
  const cuuint32_t box[3] = {static_cast<cuuint32_t>(cols), static_cast<cuuint32_t>(b1), static_cast<cuuint32_t>(b2)};
  const cuuint32_t estr[3] = {1, 1, 1};
  return fn(map, CU_TENSOR_MAP_DATA_TYPE_BFLOAT16, 3, const_cast<void*>(base), dims, strides, box, estr, CU_TENSOR_MAP_INTERLEAVE_NONE,
            cols == 64 ? CU_TENSOR_MAP_SWIZZLE_128B : CU_TENSOR_MAP_SWIZZLE_64B, CU_TENSOR_MAP_L2_PROMOTION_L2_256B,
            CU_TENSOR_MAP_FLOAT_OOB_FILL_NONE) == CUDA_SUCCESS;
}

// Configuration of a programmatic launch: the kernel may start before the one in front of it in the stream has finished.
struct BehindLaunch {
  cudaLaunchConfig_t config = {};
  cudaLaunchAttribute attr;
  BehindLaunch(int blocks, int threads, size_t smem, cudaStream_t stream) {
    attr.id = cudaLaunchAttributeProgrammaticStreamSerialization;
    attr.val.programmaticStreamSerializationAllowed = 1;
    config.gridDim = dim3(blocks);
    config.blockDim = dim3(threads);
    config.dynamicSmemBytes = smem;
    config.stream = stream;
    config.attrs = &attr;
    config.numAttrs = 1;
  }
  BehindLaunch(const BehindLaunch&) = delete;
};

}  // namespace tc
}  // namespace eagle
