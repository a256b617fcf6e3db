// What the kernels of this library share below their mathematics: status bits, bounded barrier waits, asynchronous copies.
#pragma once
#include <cuda_runtime.h>
#include <stdint.h>

namespace wkv {

constexpr uint32_t kSpinLimit = 1u << 22;             // polls of a bounded wait (mbarrier: some 20 s, see below; or a lane's arrival counter)

enum StatusBits : uint32_t { kStatusWaitTimeout = 1u, kStatusBadLink = 2u, kStatusBadTable = 4u };

// ------------------------------------------------------------------------------------------------
// small PTX wrappers
// ------------------------------------------------------------------------------------------------
__device__ __forceinline__ uint32_t smem_u32(const void* p) { return (uint32_t)__cvta_generic_to_shared(p); }

__device__ __forceinline__ void mbar_init(uint64_t* bar, uint32_t count) {
  asm volatile("mbarrier.init.shared::cta.b64 [%0], %1;" ::"r"(smem_u32(bar)), "r"(count) : "memory");
}
__device__ __forceinline__ void mbar_expect_tx(uint64_t* bar, uint32_t bytes) {
  asm volatile("mbarrier.arrive.expect_tx.shared::cta.b64 _, [%0], %1;" ::"r"(smem_u32(bar)), "r"(bytes) : "memory");
}
__device__ __forceinline__ void mbar_arrive(uint64_t* bar) {
  asm volatile("mbarrier.arrive.shared::cta.b64 _, [%0];" ::"r"(smem_u32(bar)) : "memory");
}
__device__ __forceinline__ bool mbar_try_wait(uint64_t* bar, uint32_t parity) {
  uint32_t ok;
  asm volatile(
      "{\n\t.reg .pred p;\n\t"
      "mbarrier.try_wait.parity.shared::cta.b64 p, [%1], %2;\n\t"
      "selp.u32 %0, 1, 0, p;\n\t}"
      : "=r"(ok)
      : "r"(smem_u32(bar)), "r"(parity)
      : "memory");
  return ok != 0;
}
// Bounded wait: gives up after `limit` polls, records it in the status word and returns false.
__device__ __forceinline__ bool mbar_wait(uint64_t* bar, uint32_t parity, uint32_t* status, uint32_t limit = kSpinLimit) {
  for (uint32_t it = 0; it < limit; ++it) {
    if (mbar_try_wait(bar, parity)) return true;
    if (it > 64) __nanosleep(64);
  }
  atomicOr(status, kStatusWaitTimeout);
  return false;
}
// Waits of warps that work for one another.  A wait that returns false has used up its limit and recorded it in the status word, and
// means "leave": who gets it neither touches what it waited for nor arrives anywhere any more, so the others' waits run out in turn
// and the CTA ends within a few limits.  Who has copies or matrix instructions in flight waits for those (drain_wait) before that.
// The polls do not sleep and are one instruction when the barrier is ready (a fifth of mbar_wait's cycles, whose loop the compiler
// guards for divergence); anything but straight code behind them, such as a second loop or a look at a flag of the CTA, cost the
// prompt kernel 4 to 6 %.  A poll in vain was measured to take 5 us (the instruction suspends the thread).
constexpr uint32_t kWaitPolls = 1u << 17;             // 0.7 s
constexpr uint32_t kDrainPolls = 1u << 15;
struct WaitLimit {
  uint32_t* status;
  uint32_t polls;
};
__device__ __forceinline__ bool mbar_poll(uint64_t* bar, uint32_t parity, uint32_t polls) {
  uint32_t left;
  asm volatile(
      "{\n\t.reg .pred done, more;\n\t.reg .u32 n;\n\tmov.u32 n, %3;\n"
      "POLL:\n\tmbarrier.try_wait.parity.shared::cta.b64 done, [%1], %2;\n\t@done bra OUT;\n\t"
      "sub.u32 n, n, 1;\n\tsetp.ne.u32 more, n, 0;\n\t@more bra POLL;\n"
      "OUT:\n\tmov.u32 %0, n;\n\t}"
      : "=r"(left)
      : "r"(smem_u32(bar)), "r"(parity), "r"(polls)
      : "memory");
  return left != 0;
}
// By one thread ...
[[nodiscard]] __device__ __forceinline__ bool thread_wait(uint64_t* bar, uint32_t parity, const WaitLimit& w) {
  if (mbar_poll(bar, parity, w.polls)) return true;
  atomicOr(w.status, kStatusWaitTimeout);
  return false;
}
// ... and by a converged warp, which gets one answer.
[[nodiscard]] __device__ __forceinline__ bool warp_wait(uint64_t* bar, uint32_t parity, const WaitLimit& w) {
  if (__all_sync(~0u, mbar_poll(bar, parity, w.polls))) return true;
  atomicOr(w.status, kStatusWaitTimeout);
  return false;
}
__device__ __forceinline__ bool drain_wait(uint64_t* bar, uint32_t parity, uint32_t* status) {
  return thread_wait(bar, parity, WaitLimit{status, kDrainPolls});
}
// A consumer warp hands a ring stage back to the producer.  The fence puts every lane's reads of the stage ahead of
// lane 0's arrival whatever instruction did the reading: with fragment loads (ldmatrix) in place of plain loads, the
// reads of a tile's last channels were observed behind the arrival, picking up the tile that the producer put there next.
__device__ __forceinline__ void release_stage(uint64_t* empty_bar) {
  __threadfence_block();
  __syncwarp();
  if ((threadIdx.x & 31) == 0) mbar_arrive(empty_bar);
}
// Bulk asynchronous copy global -> this CTA's shared memory, completion counted in bytes on an mbarrier.
// dst, src 16-byte aligned, bytes a multiple of 16.
__device__ __forceinline__ void bulk_g2s(void* dst, const void* src, uint32_t bytes, uint64_t* bar) {
  asm volatile("cp.async.bulk.shared::cluster.global.mbarrier::complete_tx::bytes [%0], [%1], %2, [%3];" ::"r"(
                   smem_u32(dst)),
               "l"(src), "r"(bytes), "r"(smem_u32(bar))
               : "memory");
}
__device__ __forceinline__ void bulk_g2s_hint(void* dst, const void* src, uint32_t bytes, uint64_t* bar, uint64_t policy) {
  asm volatile("cp.async.bulk.shared::cluster.global.mbarrier::complete_tx::bytes.L2::cache_hint [%0], [%1], %2, [%3], %4;" ::"r"(
                   smem_u32(dst)),
               "l"(src), "r"(bytes), "r"(smem_u32(bar)), "l"(policy)
               : "memory");
}
// Tiled tensor-map copy global -> this CTA's shared memory: the box of `tmap` whose first element is (x, y) = (element
// in the row, row).  x * element size must be a multiple of 16 bytes; dst 128-byte aligned (1024 for swizzled boxes).
__device__ __forceinline__ void tensor_g2s_2d(void* dst, const void* tmap, int x, int y, uint64_t* bar) {
  asm volatile("cp.async.bulk.tensor.2d.shared::cluster.global.tile.mbarrier::complete_tx::bytes [%0], [%1, {%2, %3}], [%4];" ::"r"(
                   smem_u32(dst)),
               "l"(tmap), "r"(x), "r"(y), "r"(smem_u32(bar))
               : "memory");
}
// The same copy with an L2 eviction-priority policy (from l2_policy_evict_first) for data that is streamed.
__device__ __forceinline__ void tensor_g2s_2d_hint(void* dst, const void* tmap, int x, int y, uint64_t* bar, uint64_t policy) {
  asm volatile(
      "cp.async.bulk.tensor.2d.shared::cluster.global.tile.mbarrier::complete_tx::bytes.L2::cache_hint [%0], [%1, {%2, %3}], [%4], %5;" ::"r"(
          smem_u32(dst)),
      "l"(tmap), "r"(x), "r"(y), "r"(smem_u32(bar)), "l"(policy)
      : "memory");
}
__device__ __forceinline__ uint64_t l2_policy_evict_first() {
  uint64_t p;
  asm volatile("createpolicy.fractional.L2::evict_first.b64 %0, 1.0;" : "=l"(p));
  return p;
}
// Hint: bring [src, src + bytes) into L2.  src 16-byte aligned, bytes a multiple of 16.
__device__ __forceinline__ void l2_prefetch(const void* src, uint32_t bytes) {
  asm volatile("cp.async.bulk.prefetch.L2.global [%0], %1;" ::"l"(src), "r"(bytes) : "memory");
}
// Programmatic dependent launch.  griddep_wait: block until the kernel this one was launched behind has completed and
// its writes are visible (returns at once when the launch carried no such dependency).  griddep_launch: allow the
// next kernel in the stream to begin once every CTA of this grid has called it or exited.
__device__ __forceinline__ void griddep_wait() { asm volatile("griddepcontrol.wait;" ::: "memory"); }
__device__ __forceinline__ void griddep_launch() { asm volatile("griddepcontrol.launch_dependents;" ::: "memory"); }

}  // namespace wkv
