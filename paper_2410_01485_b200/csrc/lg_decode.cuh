// Warp-level building blocks of the two decode kernels (bf16 ring, paged 8-bit cache).
#pragma once
#include "lg_common.cuh"

namespace lg {

constexpr int kDecWarps = 8;          // warps per CTA, each with its own pipeline of tiles
constexpr int kDecThreads = kDecWarps * 32;
constexpr int kDecHeads = 8;          // query heads per CTA (mma N)

// A decode workspace: the header, the arrival counters of the units that several CTAs share (zero between calls), the records.  All three lie
// where no call's sizes move them, so that one workspace serves calls of any size in turn: behind counters as many as a call's units, the
// records of a small batch would lie where a larger one counts.  Of the units that begin in a CTA only its last goes on into the next, so the
// shared ones are told apart by their first CTA, of which there are no more than the grid has; where the units are that few, by
// their own number.
constexpr int kDecMaxCtas = 320;      // upper bound of the grids (two CTAs per SM)
constexpr size_t kDecCountOffset = sizeof(WsHeader), kDecRecordOffset = kDecCountOffset + kDecMaxCtas * sizeof(unsigned int);
static_assert(kDecRecordOffset % 256 == 0, "records are read 16 bytes at a time");
__device__ __forceinline__ unsigned int* unit_counter(unsigned int* counters, int units, int unit, int first_cta) {
  return counters + (units <= kDecMaxCtas ? unit : first_cta);
}

__device__ __forceinline__ void prefetch_l2(const void* gptr, uint32_t bytes) {   // 16-byte aligned, a multiple of 16 bytes
  asm volatile("cp.async.bulk.prefetch.L2.global [%0], %1;" ::"l"(gptr), "r"(bytes) : "memory");
}
__device__ __forceinline__ unsigned ticket_add(unsigned int* p) {
  unsigned old;
  asm volatile("atom.add.acq_rel.gpu.global.u32 %0, [%1], 1;" : "=r"(old) : "l"(p) : "memory");
  return old;
}
__device__ __forceinline__ void ldsm_x4(uint32_t addr, uint32_t& r0, uint32_t& r1, uint32_t& r2, uint32_t& r3) {
  asm volatile("ldmatrix.sync.aligned.m8n8.x4.shared.b16 {%0, %1, %2, %3}, [%4];"
               : "=r"(r0), "=r"(r1), "=r"(r2), "=r"(r3)
               : "r"(addr));
}
__device__ __forceinline__ void ldsm_x4_t(uint32_t addr, uint32_t& r0, uint32_t& r1, uint32_t& r2, uint32_t& r3) {
  asm volatile("ldmatrix.sync.aligned.m8n8.x4.trans.shared.b16 {%0, %1, %2, %3}, [%4];"
               : "=r"(r0), "=r"(r1), "=r"(r2), "=r"(r3)
               : "r"(addr));
}
__device__ __forceinline__ uint32_t movmatrix_t(uint32_t x) {
  uint32_t y;
  asm volatile("movmatrix.sync.aligned.m8n8.trans.b16 %0, %1;" : "=r"(y) : "r"(x));
  return y;
}

}  // namespace lg
