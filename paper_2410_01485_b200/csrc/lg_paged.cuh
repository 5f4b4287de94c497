// Device side of the paged cache that the append, the attention and the chunk's copy share.
#pragma once
#include <cuda_fp16.h>

#include "lg_common.cuh"
#include "lg_paged.h"

namespace lg {

// ---- e4m3 -------------------------------------------------------------------------------
__device__ __forceinline__ uint32_t e4m3x2_to_f16x2(uint32_t two) {   // low 16 bits: two codes
  uint32_t r;
  asm("{\n\t.reg .b16 x, y;\n\tmov.b32 {x, y}, %1;\n\tcvt.rn.f16x2.e4m3x2 %0, x;\n\t}" : "=r"(r) : "r"(two));
  return r;
}
__device__ __forceinline__ uint32_t e4m3x2_hi_to_f16x2(uint32_t four) {   // high 16 bits
  uint32_t r;
  asm("{\n\t.reg .b16 x, y;\n\tmov.b32 {x, y}, %1;\n\tcvt.rn.f16x2.e4m3x2 %0, y;\n\t}" : "=r"(r) : "r"(four));
  return r;
}
__device__ __forceinline__ float2 f16x2_to_f32x2(uint32_t h) {
  return __half22float2(*reinterpret_cast<const __half2*>(&h));
}

// The page of a table entry, or -1 where the entry names no page of the pool.
__device__ __forceinline__ int checked_page(int page, int num_pages) { return page >= 0 && page < num_pages ? page : -1; }

// ---- rows of the cache in bf16 ---------------------------------------------------------------
// 16 codes times the page's scale (exact for a power-of-two scale: 4 significant bits) as two 16-byte pieces.
__device__ __forceinline__ void dequant16(uint4 c, float s, uint4& lo, uint4& hi) {
  auto two = [s](uint32_t h) { const float2 f = f16x2_to_f32x2(h); return pack_bf16(f.x * s, f.y * s); };
  lo = make_uint4(two(e4m3x2_to_f16x2(c.x)), two(e4m3x2_hi_to_f16x2(c.x)), two(e4m3x2_to_f16x2(c.y)), two(e4m3x2_hi_to_f16x2(c.y)));
  hi = make_uint4(two(e4m3x2_to_f16x2(c.z)), two(e4m3x2_hi_to_f16x2(c.z)), two(e4m3x2_to_f16x2(c.w)), two(e4m3x2_hi_to_f16x2(c.w)));
}

constexpr int kGatherThreads = 256;

constexpr int kLineariseSeqs = 128;   // sequences of one launch
struct PagedLinearise {
  const void* pool[2];       // K, V
  const float* scale[2];
  const void* chunk[2];      // [B, Hkv, T, D] bf16
  void* lin[2];              // [B, Hkv, kept + T, D] bf16
  const int32_t* table;
  unsigned int* error_word;
  int B, Hkv, D, T, kept, sink, window, page_shift, num_pages, stride;
  ChunkSeq seq[kLineariseSeqs];
};
// One thread: 16 elements of K and of V, piece i of kv head h of sequence b.  Rows of the gap, rows whose page is absent and rows that no token
// of the chunk sees are zeros: the weight of zero that they get does not silence a NaN.  Blocks of 64 that lie in the gap whole are on
// no list and are not written.
__device__ __forceinline__ void paged_linearise(const PagedLinearise& a, int64_t i, int h, int b) {
  const int row_shift = a.D == 128 ? 3 : 2, per_row = 1 << row_shift, L = a.kept + a.T;
  const int64_t v = i >> row_shift;
  const int c = static_cast<int>(i) & (per_row - 1);
  if (v >= L) return;
  const int64_t bh = static_cast<int64_t>(b) * a.Hkv + h;
  uint4 lo[2], hi[2];
  if (v < a.kept) {
    const ChunkSeq& s = a.seq[b];
    const ChunkView view = chunk_view(a.kept, a.sink, s);
    int slot = static_cast<int>(v);
    if (!chunk_block_held(view, a.sink, slot >> 6)) return;
    bool held = slot < view.sink_end;
    if (slot >= a.sink) {
      const int first = max(view.first, a.sink);
      held = slot >= first && slot >= s.seen;
      slot = s.ring0 + (held ? slot - first : 0);
      if (slot >= a.window) slot -= a.window;
      slot += a.sink;
    }
    const int page = held ? checked_page(a.table[static_cast<int64_t>(b) * a.stride + (slot >> a.page_shift)], a.num_pages) : -1;
    const int64_t unit = (page < 0 ? 0 : page) * static_cast<int64_t>(a.Hkv) + h;
    const int64_t at = ((unit << a.page_shift) + (slot & ((1 << a.page_shift) - 1))) * per_row + c;
#pragma unroll
    for (int x = 0; x < 2; ++x) {
      lo[x] = hi[x] = make_uint4(0, 0, 0, 0);
      if (page >= 0) dequant16(*(reinterpret_cast<const uint4*>(a.pool[x]) + at), a.scale[x][unit], lo[x], hi[x]);
    }
  } else {
    const int64_t from = ((bh * a.T + (v - a.kept)) * per_row + c) * 2;
#pragma unroll
    for (int x = 0; x < 2; ++x) {
      lo[x] = *(reinterpret_cast<const uint4*>(a.chunk[x]) + from);
      hi[x] = *(reinterpret_cast<const uint4*>(a.chunk[x]) + from + 1);
    }
  }
  const int64_t to = ((bh * L + v) * per_row + c) * 2;
#pragma unroll
  for (int x = 0; x < 2; ++x) {
    reinterpret_cast<uint4*>(a.lin[x])[to] = lo[x];
    reinterpret_cast<uint4*>(a.lin[x])[to + 1] = hi[x];
  }
}
// Whether some entry that the kept tokens lie behind names no page; all threads of a block look.
__device__ __forceinline__ bool paged_entry_missing(const PagedLinearise& a, int threads) {
  const int round = (1 << a.page_shift) - 1, pages = (a.kept + round) >> a.page_shift;   // (at most: a full ring, or its first slots)
  bool missing = false;
  for (int64_t i = threadIdx.x; i < static_cast<int64_t>(a.B) * pages; i += threads) {
    const int64_t b = i / pages;
    const int page = static_cast<int>(i - b * pages);
    if (page < (a.seq[b].held + round) >> a.page_shift) missing |= checked_page(a.table[b * a.stride + page], a.num_pages) < 0;
  }
  return __syncthreads_or(missing) != 0;
}

}  // namespace lg
