// Barriers in shared memory and copies of blocks by TMA, for the kernels of kv_attend.
//
// Every wait is bounded: one that gives up sets KV_DEV_WAIT_EXPIRED and a flag that ends the CTA's other waits.
#pragma once
#include <cuda.h>

#include "kv_attend.cuh"

namespace kvt {

constexpr long long kWaitLimit = 4'000'000'000ll;   // cycles of the SM: about two seconds

__device__ __forceinline__ void bar_init(uint32_t bar, uint32_t count) {
  asm volatile("mbarrier.init.shared::cta.b64 [%0], %1;" ::"r"(bar), "r"(count) : "memory");
}
__device__ __forceinline__ void bar_expect(uint32_t bar, uint32_t bytes) {
  asm volatile("mbarrier.arrive.expect_tx.shared::cta.b64 _, [%0], %1;" ::"r"(bar), "r"(bytes) : "memory");
}
__device__ __forceinline__ void bar_arrive(uint32_t bar) {
  asm volatile("mbarrier.arrive.shared::cta.b64 _, [%0];" ::"r"(bar) : "memory");
}
__device__ __forceinline__ bool bar_try(uint32_t bar, uint32_t parity) {
  uint32_t done;
  asm volatile(
      "{\n\t.reg .pred p;\n\t"
      "mbarrier.try_wait.parity.shared::cta.b64 p, [%1], %2, %3;\n\t"
      "selp.u32 %0, 1, 0, p;\n\t}"
      : "=r"(done)
      : "r"(bar), "r"(parity), "r"(20000u)   // nanoseconds that the thread may sleep
      : "memory");
  return done != 0;
}
// The same without any sleep.
__device__ __forceinline__ bool bar_test(uint32_t bar, uint32_t parity) {
  uint32_t done;
  asm volatile(
      "{\n\t.reg .pred p;\n\t"
      "mbarrier.test_wait.parity.shared::cta.b64 p, [%1], %2;\n\t"
      "selp.u32 %0, 1, 0, p;\n\t}"
      : "=r"(done)
      : "r"(bar), "r"(parity)
      : "memory");
  return done != 0;
}
// False: this wait, or another of the CTA, has given up.
__device__ __forceinline__ bool bar_wait(uint32_t bar, uint32_t parity, volatile uint32_t* gave_up, uint32_t* status) {
  if (bar_try(bar, parity)) return true;
  const long long from = clock64();
  do {
    if (bar_try(bar, parity)) return true;
    if (*gave_up) return false;
  } while (clock64() - from < kWaitLimit);
  *gave_up = 1u;
  atomicOr(status, KV_DEV_WAIT_EXPIRED);
  return false;
}
// What the thread has written to shared memory comes before what copies and products do with it.
__device__ __forceinline__ void proxy_fence() { asm volatile("fence.proxy.async.shared::cta;" ::: "memory"); }
// A box from row y and panel (64 elements) x on; kv: the chunk of keys, or the one of values.
__device__ __forceinline__ void tma_box(uint32_t dst, const CUtensorMap* map, int32_t x, int32_t y, int32_t kv, uint32_t bar) {
  asm volatile(
      "cp.async.bulk.tensor.4d.shared::cluster.global.mbarrier::complete_tx::bytes [%0], [%1, {%2, %3, %4, %5}], [%6];" ::"r"(dst),
      "l"(map), "r"(0), "r"(y), "r"(x), "r"(kv), "r"(bar)
      : "memory");
}

// Tensor map of a partition's slab as [K, V][panel][row][64 elements], rows of dk elements; a box is box_rows rows of
// box_panels panels of box_kv chunks, panel by panel, each a row of 128 bytes with the 128-byte swizzle.  Boxes are as large as
// blocks and layouts let them be (one for a unit of 16 tokens instead of four: 64 chats 74 -> 71 us).
// False: the driver refuses the map.
bool block_map(const TableView& tv, uint32_t dk, uint32_t box_rows, uint32_t box_panels, uint32_t box_kv, CUtensorMap* map);
bool has_block_map();

}  // namespace kvt
