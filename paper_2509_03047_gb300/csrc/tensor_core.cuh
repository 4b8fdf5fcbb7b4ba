// tensor_core.cuh -- what a kernel on a pair of CTAs needs of the fifth-generation
// tensor cores: barriers in shared memory with bounded waits, bulk copies, the
// pair's products in tensor memory.
//
// A pair is a cluster of two CTAs on neighbouring SMs.  The first one's thread
// issues products of 256 rows for both: each CTA's shared memory holds 128 rows of
// the first factor and half of the second one's, its tensor memory 128 rows of the
// result.
#pragma once

#include <cuda.h>
#include <cuda_runtime.h>

#include <cstdint>

namespace frk {

__device__ __forceinline__ uint32_t shared_address(const void* p) { return static_cast<uint32_t>(__cvta_generic_to_shared(p)); }
// The same place in the pair's first CTA.
__device__ __forceinline__ uint32_t in_first(uint32_t address) { return address & 0xFEFFFFFFu; }

__device__ __forceinline__ uint32_t rank_in_pair() {
  uint32_t r;
  asm volatile("mov.u32 %0, %%cluster_ctarank;" : "=r"(r));
  return r;
}
// One lane of the warp, all of which call.  (A warp that goes together and lets one lane issue keeps addresses in uniform registers, which these
// instructions take them from.)
__device__ __forceinline__ bool one_lane() {
  uint32_t mine;
  asm volatile("{\n\t.reg .pred q;\n\telect.sync _|q, 0xFFFFFFFF;\n\tselp.u32 %0, 1, 0, q;\n\t}" : "=r"(mine));
  return mine != 0;
}
__device__ __forceinline__ void pair_sync() {
  asm volatile("barrier.cluster.arrive.release.aligned;\n\tbarrier.cluster.wait.acquire.aligned;" ::: "memory");
}

// ---- barriers in shared memory

__device__ __forceinline__ void barrier_init(uint32_t bar, uint32_t count) {
  asm volatile("mbarrier.init.shared::cta.b64 [%0], %1;" ::"r"(bar), "r"(count) : "memory");
}
__device__ __forceinline__ void barrier_init_done() { asm volatile("fence.mbarrier_init.release.cluster;" ::: "memory"); }
__device__ __forceinline__ void expect_bytes(uint32_t bar, uint32_t bytes) {
  asm volatile("mbarrier.arrive.expect_tx.shared::cta.b64 _, [%0], %1;" ::"r"(bar), "r"(bytes) : "memory");
}
// (Released to this CTA alone: what it tells the other one is that loads from tensor memory have ended, no writes.  A wider release waits for
// every write on its way, 3,000 clocks.)
__device__ __forceinline__ void arrive_in_first(uint32_t bar) {
  asm volatile("{\n\t.reg .b32 a;\n\tmapa.shared::cluster.u32 a, %0, 0;\n\tmbarrier.arrive.shared::cluster.b64 _, [a];\n\t}" ::"r"(bar) : "memory");
}
__device__ __forceinline__ bool try_wait(uint32_t bar, uint32_t parity) {
  uint32_t done;
  asm volatile(
      "{\n\t.reg .pred q;\n\tmbarrier.try_wait.parity.shared::cta.b64 q, [%1], %2;\n\tselp.u32 %0, 1, 0, q;\n\t}"
      : "=r"(done)
      : "r"(bar), "r"(parity)
      : "memory");
  return done != 0;
}
// Until the barrier's phase of this parity is over: false after `limit` clocks, or if somebody else in the CTA has given up.
__device__ __forceinline__ bool wait_phase(uint32_t bar, uint32_t parity, int64_t limit, volatile uint32_t* gave_up) {
  if (try_wait(bar, parity)) return true;
  const long long start = clock64();
  while (!try_wait(bar, parity)) {
    if (*gave_up || clock64() - start > limit) {
      *gave_up = 1;
      return false;
    }
  }
  return true;
}
// Until a counter in memory has reached `count`; with it the writes before its additions are visible (to copies after before_reading_copies).
__device__ __forceinline__ bool wait_count(const uint32_t* counter, uint32_t count, int64_t limit, volatile uint32_t* gave_up) {
  const long long start = clock64();
  for (;;) {
    uint32_t now;
    asm volatile("ld.acquire.gpu.global.u32 %0, [%1];" : "=r"(now) : "l"(counter) : "memory");
    if (now >= count) break;
    if (*gave_up || clock64() - start > limit) {
      *gave_up = 1;
      return false;
    }
  }
  return true;
}
__device__ __forceinline__ void before_reading_copies() { asm volatile("fence.proxy.async;" ::: "memory"); }
// After this thread's writes, and those of the warp's others before its last barrier.
__device__ __forceinline__ void add_to_count(uint32_t* counter) {
  asm volatile("red.release.gpu.global.add.u32 [%0], 1;" ::"l"(counter) : "memory");
}
// The part of a role that has given up: its copies in flight land meanwhile.
__device__ __forceinline__ void let_copies_land() {
  for (int i = 0; i < 20; ++i) __nanosleep(1000000);
}

// ---- copies

// A box of a map of blocks in halves of 64 rows of 128 bytes; the bytes count at the pair's first CTA.
__device__ __forceinline__ void load_blocks(uint32_t to, const CUtensorMap* map, int32_t half, int32_t block, uint32_t bar) {
  asm volatile("cp.async.bulk.tensor.4d.cta_group::2.shared::cluster.global.mbarrier::complete_tx::bytes [%0], [%1, {%2, %2, %3, %4}], [%5];" ::"r"(to),
               "l"(map), "r"(0), "r"(half), "r"(block), "r"(in_first(bar))
               : "memory");
}
__device__ __forceinline__ void store_bytes(void* to, uint32_t from, uint32_t bytes) {
  asm volatile("cp.async.bulk.global.shared::cta.bulk_group [%0], [%1], %2;" ::"l"(to), "r"(from), "r"(bytes) : "memory");
}
__device__ __forceinline__ void end_stores() { asm volatile("cp.async.bulk.commit_group;" ::: "memory"); }
__device__ __forceinline__ void wait_stores_read() { asm volatile("cp.async.bulk.wait_group.read 0;" ::: "memory"); }
__device__ __forceinline__ void wait_stores() { asm volatile("cp.async.bulk.wait_group 0;" ::: "memory"); }
// This thread's writes to shared memory before copies that read it.
__device__ __forceinline__ void before_copies() { asm volatile("fence.proxy.async.shared::cta;" ::: "memory"); }

// ---- tensor memory

__device__ __forceinline__ void tensor_alloc(uint32_t where, uint32_t columns) {
  asm volatile("tcgen05.alloc.cta_group::2.sync.aligned.shared::cta.b32 [%0], %1;" ::"r"(where), "r"(columns) : "memory");
}
__device__ __forceinline__ void tensor_free(uint32_t at, uint32_t columns) {
  asm volatile("tcgen05.relinquish_alloc_permit.cta_group::2.sync.aligned;\n\ttcgen05.dealloc.cta_group::2.sync.aligned.b32 %0, %1;" ::"r"(at),
               "r"(columns)
               : "memory");
}
__device__ __forceinline__ void tensor_fence_before() { asm volatile("tcgen05.fence::before_thread_sync;" ::: "memory"); }
__device__ __forceinline__ void tensor_fence_after() { asm volatile("tcgen05.fence::after_thread_sync;" ::: "memory"); }

// 32 columns of the thread's row.
__device__ __forceinline__ void tensor_load(uint32_t at, float* x) {
  uint32_t* v = reinterpret_cast<uint32_t*>(x);
  asm volatile(
      "tcgen05.ld.sync.aligned.32x32b.x32.b32 {%0, %1, %2, %3, %4, %5, %6, %7, %8, %9, %10, %11, %12, %13, %14, %15, %16, %17, %18, %19, %20, %21, "
      "%22, %23, %24, %25, %26, %27, %28, %29, %30, %31}, [%32];"
      : "=r"(v[0]), "=r"(v[1]), "=r"(v[2]), "=r"(v[3]), "=r"(v[4]), "=r"(v[5]), "=r"(v[6]), "=r"(v[7]), "=r"(v[8]), "=r"(v[9]), "=r"(v[10]), "=r"(v[11]),
        "=r"(v[12]), "=r"(v[13]), "=r"(v[14]), "=r"(v[15]), "=r"(v[16]), "=r"(v[17]), "=r"(v[18]), "=r"(v[19]), "=r"(v[20]), "=r"(v[21]), "=r"(v[22]),
        "=r"(v[23]), "=r"(v[24]), "=r"(v[25]), "=r"(v[26]), "=r"(v[27]), "=r"(v[28]), "=r"(v[29]), "=r"(v[30]), "=r"(v[31])
      : "r"(at));
}
__device__ __forceinline__ void tensor_load_wait() { asm volatile("tcgen05.wait::ld.sync.aligned;" ::: "memory"); }

// A factor in shared memory: rows of 128 bytes (64 fp16 numbers), their 16-byte chunks permuted by the row's index modulo 8.
//   by rows     the contraction runs along the rows: 16 numbers of it are 32 bytes; groups of eight rows follow one another
//   by columns  the contraction runs over the rows: 16 of them are 2 KiB; 64 columns, then `next` bytes on the next 64
__device__ __forceinline__ uint64_t factor(uint32_t at, bool by_columns, uint32_t next) {
  const uint64_t lead = by_columns ? next >> 4 : 1, groups = 1024 >> 4;
  return (at >> 4 & 0x3FFF) | lead << 16 | groups << 32 | 1ull << 46 | 2ull << 61;
}
// fp16 times fp16 to fp32, 256 rows in the pair.
__device__ __forceinline__ uint32_t product_kind(bool a_by_columns, bool b_by_columns, uint32_t columns) {
  return 1u << 4 | static_cast<uint32_t>(a_by_columns) << 15 | static_cast<uint32_t>(b_by_columns) << 16 | (columns >> 3) << 17 | (256u >> 4) << 24;
}
__device__ __forceinline__ void multiply(uint32_t d, uint64_t a, uint64_t b, uint32_t kind, bool add) {
  asm volatile("{\n\t.reg .pred q;\n\tsetp.ne.u32 q, %4, 0;\n\ttcgen05.mma.cta_group::2.kind::f16 [%0], %1, %2, %3, q;\n\t}" ::"r"(d), "l"(a), "l"(b),
               "r"(kind), "r"(static_cast<uint32_t>(add))
               : "memory");
}
// The barrier, in both CTAs, is arrived at once all products before have ended.
__device__ __forceinline__ void arrive_after_products(uint32_t bar) {
  asm volatile("tcgen05.commit.cta_group::2.mbarrier::arrive::one.shared::cluster.multicast::cluster.b64 [%0], %1;" ::"r"(bar),
               "h"(static_cast<uint16_t>(3))
               : "memory");
}

}  // namespace frk
