// Building blocks of the tensor-core kernels: mbarriers with bounded waits, TMA tile loads, tcgen05
// matrix instructions with their accumulators in tensor memory, and programmatic launch order.
#pragma once

#include <cuda.h>
#include <cuda_runtime.h>
#include <stdint.h>

namespace rtopk {
namespace mat {

__device__ __forceinline__ uint32_t smem_addr(const void* p) { return (uint32_t)__cvta_generic_to_shared(p); }

__device__ __forceinline__ uint64_t now_ns() {
  uint64_t t;
  asm volatile("mov.u64 %0, %globaltimer;" : "=l"(t));
  return t;
}

// True in one thread of the converged warp, always the same one.  The warps that feed and issue products run their loops whole and let
// one thread through here, so that addresses and descriptors stay in uniform registers, where these instructions take them
// from; a loop that one thread runs alone moves each of them there first.
__device__ __forceinline__ bool elect_one() {
  uint32_t is;
  asm volatile("{\n\t.reg .pred p;\n\telect.sync _|p, 0xFFFFFFFF;\n\tselp.u32 %0, 1, 0, p;\n\t}" : "=r"(is));
  return is != 0;
}

// ----------------------------------------------------------------------------- mbarriers
__device__ __forceinline__ void bar_init(uint32_t bar, uint32_t count) {
  asm volatile("mbarrier.init.shared::cta.b64 [%0], %1;" ::"r"(bar), "r"(count) : "memory");
}
__device__ __forceinline__ void bar_init_fence() { asm volatile("fence.mbarrier_init.release.cluster;" ::: "memory"); }
__device__ __forceinline__ void bar_expect(uint32_t bar, uint32_t bytes) {
  asm volatile("mbarrier.arrive.expect_tx.shared::cta.b64 _, [%0], %1;" ::"r"(bar), "r"(bytes) : "memory");
}
// Stands in for the bytes of a copy that was expected and never issued.
__device__ __forceinline__ void bar_complete(uint32_t bar, uint32_t bytes) {
  asm volatile("mbarrier.complete_tx.relaxed.cta.shared::cta.b64 [%0], %1;" ::"r"(bar), "r"(bytes) : "memory");
}
__device__ __forceinline__ void bar_arrive(uint32_t bar) {
  asm volatile("mbarrier.arrive.shared::cta.b64 _, [%0];" ::"r"(bar) : "memory");
}
// On the barrier at the same place of the pair's first block.
__device__ __forceinline__ uint32_t first_of_pair(uint32_t bar) {
  uint32_t r;
  asm volatile("mapa.shared::cluster.u32 %0, %1, 0;" : "=r"(r) : "r"(bar));
  return r;
}
// The same place in the shared memory of a block of the cluster.
__device__ __forceinline__ uint32_t at_rank(uint32_t addr, uint32_t rank) {
  uint32_t r;
  asm volatile("mapa.shared::cluster.u32 %0, %1, %2;" : "=r"(r) : "r"(addr), "r"(rank));
  return r;
}
__device__ __forceinline__ float4 cluster_load4(uint32_t addr) {
  float4 v;
  asm volatile("ld.shared::cluster.v4.f32 {%0, %1, %2, %3}, [%4];" : "=f"(v.x), "=f"(v.y), "=f"(v.z), "=f"(v.w) : "r"(addr) : "memory");
  return v;
}
__device__ __forceinline__ uint32_t cluster_load(uint32_t addr) {
  uint32_t v;
  asm volatile("ld.shared::cluster.u32 %0, [%1];" : "=r"(v) : "r"(addr) : "memory");
  return v;
}
__device__ __forceinline__ void cluster_store(uint32_t addr, float v) { asm volatile("st.shared::cluster.f32 [%0], %1;" ::"r"(addr), "f"(v) : "memory"); }
__device__ __forceinline__ void cluster_store(uint32_t addr, double v) { asm volatile("st.shared::cluster.f64 [%0], %1;" ::"r"(addr), "d"(v) : "memory"); }
__device__ __forceinline__ void cluster_store(uint32_t addr, uint32_t v) { asm volatile("st.shared::cluster.u32 [%0], %1;" ::"r"(addr), "r"(v) : "memory"); }
__device__ __forceinline__ void cluster_store(uint32_t addr, uint2 v) {
  asm volatile("st.shared::cluster.v2.u32 [%0], {%1, %2};" ::"r"(addr), "r"(v.x), "r"(v.y) : "memory");
}
__device__ __forceinline__ void bar_arrive_cluster(uint32_t bar) {
  asm volatile("mbarrier.arrive.release.cluster.shared::cluster.b64 _, [%0];" ::"r"(bar) : "memory");
}
__device__ __forceinline__ uint32_t rank_in_cluster() {
  uint32_t r;
  asm volatile("mov.u32 %0, %cluster_ctarank;" : "=r"(r));
  return r;
}
__device__ __forceinline__ void cluster_sync() {
  __syncwarp();
  asm volatile("barrier.cluster.arrive.release.aligned;\n\tbarrier.cluster.wait.acquire.aligned;" ::: "memory");
}
__device__ __forceinline__ bool bar_try(uint32_t bar, uint32_t parity) {
  uint32_t done;
  asm volatile(
      "{\n\t.reg .pred p;\n\t"
      "mbarrier.try_wait.parity.shared::cta.b64 p, [%1], %2;\n\t"
      "selp.u32 %0, 1, 0, p;\n\t}"
      : "=r"(done)
      : "r"(bar), "r"(parity)
      : "memory");
  return done != 0;
}

// Every wait of these kernels is bounded: after kWaitNs a role raises the block's give-up word and the context's error
// word, and every other role of the block leaves at its next look at that word.
constexpr uint64_t kWaitNs = 2000000000ull;
enum : uint32_t { MAT_ERR_WAIT = 1u };

struct GiveUp {
  volatile uint32_t* word;   // in shared memory, one per block
  uint32_t* error;           // in the context
};

// What a wait that has run out does; for tests, at a wait that has not.
__device__ __forceinline__ bool give_up(const GiveUp& g) {
  *g.word = 1u;
  atomicOr(g.error, MAT_ERR_WAIT);
  return false;
}
__device__ __forceinline__ bool bar_wait(uint32_t bar, uint32_t parity, const GiveUp& g) {
  if (bar_try(bar, parity)) return true;
  const uint64_t t0 = now_ns();
  for (uint32_t n = 1;; ++n) {
    if (bar_try(bar, parity)) return true;
    if ((n & 63u) == 0) {
      if (*g.word) return false;
      if (now_ns() - t0 > kWaitNs) return give_up(g);
    }
  }
}
// For a block that gives up: waits for its own copies or products in flight, again with a limit, which counts from t0.
__device__ __forceinline__ void bar_drain(uint32_t bar, uint32_t parity, uint64_t t0) {
  while (!bar_try(bar, parity) && now_ns() - t0 < kWaitNs) {}
}

// ----------------------------------------------------------------------------- TMA
// The barrier may be the pair's first block's.
template <bool kPair>
__device__ __forceinline__ void tma_load(uint32_t dst, const CUtensorMap* map, int x, int y, int z, uint32_t bar) {
  if (kPair)
    asm volatile(
        "cp.async.bulk.tensor.3d.cta_group::2.shared::cluster.global.tile.mbarrier::complete_tx::bytes [%0], [%1, {%2, %3, %4}], [%5];" ::"r"(dst),
        "l"(map), "r"(x), "r"(y), "r"(z), "r"(bar)
        : "memory");
  else
    asm volatile(
        "cp.async.bulk.tensor.3d.shared::cluster.global.tile.mbarrier::complete_tx::bytes [%0], [%1, {%2, %3, %4}], [%5];" ::"r"(dst),
        "l"(map), "r"(x), "r"(y), "r"(z), "r"(bar)
        : "memory");
}
__device__ __forceinline__ void tma_prefetch(const CUtensorMap* map) {
  asm volatile("prefetch.tensormap [%0];" ::"l"(map) : "memory");
}

// ----------------------------------------------------------------------------- tcgen05
template <bool kPair>
__device__ __forceinline__ void tmem_alloc(uint32_t dst, uint32_t cols) {
  if (kPair) {
    asm volatile("tcgen05.alloc.cta_group::2.sync.aligned.shared::cta.b32 [%0], %1;" ::"r"(dst), "r"(cols) : "memory");
    asm volatile("tcgen05.relinquish_alloc_permit.cta_group::2.sync.aligned;" ::: "memory");
  } else {
    asm volatile("tcgen05.alloc.cta_group::1.sync.aligned.shared::cta.b32 [%0], %1;" ::"r"(dst), "r"(cols) : "memory");
    asm volatile("tcgen05.relinquish_alloc_permit.cta_group::1.sync.aligned;" ::: "memory");
  }
}
template <bool kPair>
__device__ __forceinline__ void tmem_free(uint32_t addr, uint32_t cols) {
  if (kPair) asm volatile("tcgen05.dealloc.cta_group::2.sync.aligned.b32 %0, %1;" ::"r"(addr), "r"(cols) : "memory");
  else asm volatile("tcgen05.dealloc.cta_group::1.sync.aligned.b32 %0, %1;" ::"r"(addr), "r"(cols) : "memory");
}
__device__ __forceinline__ void tc_fence_before() { asm volatile("tcgen05.fence::before_thread_sync;" ::: "memory"); }
__device__ __forceinline__ void tc_fence_after() { asm volatile("tcgen05.fence::after_thread_sync;" ::: "memory"); }

#define TC_MMA(group, kind)                                                                     \
  asm volatile("{\n\t.reg .pred p;\n\tsetp.ne.u32 p, %4, 0;\n\t"                                 \
               "tcgen05.mma.cta_group::" group ".kind::" kind " [%0], %1, %2, %3, p;\n\t}" ::"r"(d), \
               "l"(a), "l"(b), "r"(idesc), "r"(accumulate)                                      \
               : "memory")
template <bool kPair, bool kInt8>
__device__ __forceinline__ void tc_mma(uint32_t d, uint64_t a, uint64_t b, uint32_t idesc, uint32_t accumulate) {
  if (kPair && kInt8) TC_MMA("2", "i8");
  else if (kPair) TC_MMA("2", "f16");
  else if (kInt8) TC_MMA("1", "i8");
  else TC_MMA("1", "f16");
}
#undef TC_MMA
// 4-bit floating-point codes (64 of the contraction index) with a power of two for every 32 of them and row: the scales lie in
// tensor memory, byte pairs of a column's words, row r of 32 in lane r, the next 32 rows in the next column.
#define TC_MMA_MICRO(group)                                                                                             \
  asm volatile("{\n\t.reg .pred p;\n\tsetp.ne.u32 p, %4, 0;\n\t"                                                          \
               "tcgen05.mma.cta_group::" group ".kind::mxf4.block_scale.scale_vec::2X [%0], %1, %2, %3, [%5], [%6], p;\n\t}" ::"r"(d), \
               "l"(a), "l"(b), "r"(idesc), "r"(accumulate), "r"(scale_a), "r"(scale_b)                                  \
               : "memory")
template <bool kPair>
__device__ __forceinline__ void tc_mma_micro(uint32_t d, uint64_t a, uint64_t b, uint32_t idesc, uint32_t scale_a, uint32_t scale_b, uint32_t accumulate) {
  if (kPair) TC_MMA_MICRO("2");
  else TC_MMA_MICRO("1");
}
#undef TC_MMA_MICRO
// 512 bytes, 16 for each of 32 rows, into four columns of tensor memory, the same for each quarter of the lanes; in a pair each block's
// own bytes into its own columns.  Products issued after it by the same thread see them.
template <bool kPair>
__device__ __forceinline__ void tc_copy_scales(uint32_t dst, uint64_t src) {
  if (kPair) asm volatile("tcgen05.cp.cta_group::2.32x128b.warpx4 [%0], %1;" ::"r"(dst), "l"(src) : "memory");
  else asm volatile("tcgen05.cp.cta_group::1.32x128b.warpx4 [%0], %1;" ::"r"(dst), "l"(src) : "memory");
}
// The barrier (in a pair: both blocks') completes when all products issued before by this thread are done.
template <bool kPair>
__device__ __forceinline__ void tc_commit(uint32_t bar) {
  if (kPair)
    asm volatile("tcgen05.commit.cta_group::2.mbarrier::arrive::one.shared::cluster.multicast::cluster.b64 [%0], %1;" ::"r"(bar), "h"((uint16_t)3) : "memory");
  else
    asm volatile("tcgen05.commit.cta_group::1.mbarrier::arrive::one.shared::cluster.b64 [%0];" ::"r"(bar) : "memory");
}
// 32 columns of this warp's 32 lanes: register c holds column c of the thread's lane.  The load writes its registers
// after it was issued; the wait is part of the statement, so that no use can be moved before it.
__device__ __forceinline__ void tmem_load32(uint32_t addr, uint32_t (&r)[32]) {
  asm volatile(
      "tcgen05.ld.sync.aligned.32x32b.x32.b32 "
      "{%0, %1, %2, %3, %4, %5, %6, %7, %8, %9, %10, %11, %12, %13, %14, %15, "
      "%16, %17, %18, %19, %20, %21, %22, %23, %24, %25, %26, %27, %28, %29, %30, %31}, [%32];\n\t"
      "tcgen05.wait::ld.sync.aligned;"
      : "=r"(r[0]), "=r"(r[1]), "=r"(r[2]), "=r"(r[3]), "=r"(r[4]), "=r"(r[5]), "=r"(r[6]), "=r"(r[7]), "=r"(r[8]), "=r"(r[9]),
        "=r"(r[10]), "=r"(r[11]), "=r"(r[12]), "=r"(r[13]), "=r"(r[14]), "=r"(r[15]), "=r"(r[16]), "=r"(r[17]), "=r"(r[18]),
        "=r"(r[19]), "=r"(r[20]), "=r"(r[21]), "=r"(r[22]), "=r"(r[23]), "=r"(r[24]), "=r"(r[25]), "=r"(r[26]), "=r"(r[27]),
        "=r"(r[28]), "=r"(r[29]), "=r"(r[30]), "=r"(r[31])
      : "r"(addr)
      : "memory");
}

__device__ __forceinline__ void tmem_load16(uint32_t addr, uint32_t (&r)[16]) {
  asm volatile(
      "tcgen05.ld.sync.aligned.32x32b.x16.b32 "
      "{%0, %1, %2, %3, %4, %5, %6, %7, %8, %9, %10, %11, %12, %13, %14, %15}, [%16];\n\t"
      "tcgen05.wait::ld.sync.aligned;"
      : "=r"(r[0]), "=r"(r[1]), "=r"(r[2]), "=r"(r[3]), "=r"(r[4]), "=r"(r[5]), "=r"(r[6]), "=r"(r[7]), "=r"(r[8]), "=r"(r[9]),
        "=r"(r[10]), "=r"(r[11]), "=r"(r[12]), "=r"(r[13]), "=r"(r[14]), "=r"(r[15])
      : "r"(addr)
      : "memory");
}
// Ordinary stores to shared memory, seen by the tensor core and TMA after the next barrier.
__device__ __forceinline__ void smem_publish() { asm volatile("fence.proxy.async.shared::cta;" ::: "memory"); }
__device__ __forceinline__ void cluster_publish() { asm volatile("fence.proxy.async;" ::: "memory"); }

// Shared-memory matrix descriptor, 128-byte swizzle.  K-major tiles: rows of 128 bytes, groups of 8 rows 1024 bytes
// apart (the leading offset is not used).  MN-major tiles: slabs of 64 16-bit elements along the row index,
// `slab_bytes` apart, in which 8 steps of the contraction index take 1024 bytes.
__device__ __forceinline__ uint64_t smem_desc(uint32_t addr, uint32_t slab_bytes) {
  return (uint64_t)((addr & 0x3FFFFu) >> 4) | ((uint64_t)((slab_bytes & 0x3FFFFu) >> 4) << 16) | ((uint64_t)(1024u >> 4) << 32) |
         (1ull << 46) | (2ull << 61);
}
// Instruction descriptor: f16 x f16 -> f32 or s8 x s8 -> s32, m x n.
__host__ __device__ constexpr uint32_t instr_desc(bool int8, bool a_mn_major, uint32_t m, uint32_t n, bool b_mn_major = false) {
  return (int8 ? (2u << 4) | (1u << 7) | (1u << 10) : (1u << 4)) | (a_mn_major ? 1u << 15 : 0u) | (b_mn_major ? 1u << 16 : 0u) | ((n >> 3) << 17) | ((m >> 4) << 24);
}

// Of the scales' bytes: no swizzle, groups of eight 16-byte rows 128 bytes apart.
__device__ __forceinline__ uint64_t scale_desc(uint32_t addr) { return (uint64_t)((addr & 0x3FFFFu) >> 4) | ((uint64_t)(128u >> 4) << 32) | (1ull << 46); }
// 4-bit codes with a scale in 8 exponent bits for every 32; `pair`: which two of a word's four scales.
__host__ __device__ constexpr uint32_t micro_desc(uint32_t m, uint32_t n, uint32_t pair) {
  return (2 * pair << 4) | (1u << 7) | (1u << 10) | ((n >> 3) << 17) | (1u << 23) | ((m >> 4) << 24) | (2 * pair << 29);
}

// ----------------------------------------------------------------------------- launch order
// Every kernel here is launched with the programmatic attribute: it may start while its predecessor in the stream still runs,
// as soon as all of that one's blocks have called launch_next() or ended.  Nothing of the predecessor's output may be read, and
// nothing it reads may be written, before launch_wait(), which returns when the predecessor is complete.  Every kernel calls
// launch_next() after its own launch_wait(), so all that came before the predecessor is complete from the start.
__device__ __forceinline__ void launch_wait() { asm volatile("griddepcontrol.wait;" ::: "memory"); }
__device__ __forceinline__ void launch_next() { asm volatile("griddepcontrol.launch_dependents;" ::: "memory"); }

}  // namespace mat
}  // namespace rtopk
