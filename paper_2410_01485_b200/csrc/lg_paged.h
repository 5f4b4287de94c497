// Index arithmetic of the paged cache, shared by the host and the kernels.  The slots of a sequence are those of the
// rolling-buffer ring (paper Section 3.2): token j lives in slot j < sink ? j : sink + (j - sink) % window, and the
// sink + window slots are cut into pages of page_tokens each.
#pragma once
#include <cuda_runtime.h>
#include <stdint.h>

namespace lg {

// Smallest exponent of a page's scale: its inverse and the scale itself stay normal fp32 numbers (the largest one, for the
// largest bf16, is 2^120).  Values that would need a smaller one are below 2^-111 and become small codes or zeros.
constexpr int kPageMinExp = -120;
constexpr int kPageMaxTokens = 128;

__host__ __device__ __forceinline__ int slot_of(int64_t pos, int sink, int window) {
  return static_cast<int>(pos < sink ? pos : sink + (pos - sink) % window);
}

// Where the newest token of a ring lies: its ring offset, and how often the ring had been filled before its lap (64-bit divisions
// take 200 cycles: one for all slots of a sequence).  Only meaningful for n > sink.
struct RingHead {
  int64_t laps;
  int offset;
};
__host__ __device__ __forceinline__ RingHead ring_head(int64_t n, int sink, int window) {
  const int64_t d = n - 1 - sink;
  if (d < window) return RingHead{0, static_cast<int>(d < 0 ? 0 : d)};
  const int64_t laps = static_cast<uint64_t>(d) <= 0xffffffffull ? static_cast<uint32_t>(d) / static_cast<uint32_t>(window) : d / window;
  return RingHead{laps, static_cast<int>(d - laps * window)};
}

// position of the token that `slot` holds once n tokens have been appended, -1: none yet (head: ring_head of n)
__host__ __device__ __forceinline__ int64_t held_position(int64_t slot, int64_t n, const RingHead& head, int sink, int window) {
  if (slot >= n || slot >= static_cast<int64_t>(sink) + window) return -1;
  return slot < sink ? slot : slot + (slot - sink <= head.offset ? head.laps : head.laps - 1) * window;
}

// pages that the cache of a sequence of n tokens takes (n < 0 counts as 0)
__host__ __device__ __forceinline__ int pages_of(int64_t n, int sink, int window, int page_shift) {
  const int64_t cap = static_cast<int64_t>(sink) + window, held = n < 0 ? 0 : n < cap ? n : cap;
  return static_cast<int>((held + (1 << page_shift) - 1) >> page_shift);
}

// The pages that a call writes which takes a sequence from n0 to n1 tokens: the slots of the new tokens are up to three
// runs (in the sink; in the ring from its start, if the call wraps around; in the ring up to its end), listed here by
// ascending page, no page twice.
struct TouchedPages {
  int first[3], count[3];
  __host__ __device__ __forceinline__ int total() const { return count[0] + count[1] + count[2]; }
  __host__ __device__ __forceinline__ int page(int i) const {   // 0 <= i < total()
    if (i < count[0]) return first[0] + i;
    if (i < count[0] + count[1]) return first[1] + i - count[0];
    return first[2] + i - count[0] - count[1];
  }
};
__host__ __device__ __forceinline__ TouchedPages touched_pages(int64_t n0, int64_t n1, const RingHead& head /* of n1 */, int sink, int window,
                                                               int page_shift) {
  int from[3] = {0, 0, 0}, to[3] = {0, 0, 0};                  // slot runs [from, to)
  if (n0 < sink) { from[0] = static_cast<int>(n0); to[0] = n1 < sink ? static_cast<int>(n1) : sink; }
  const int64_t start = n0 > sink ? n0 : sink;                 // first new token of the ring
  if (n1 > start) {
    const int m = n1 - start < window ? static_cast<int>(n1 - start) : window;   // those of them that survive the call
    const int r0 = head.offset + 1 - m;                        // ring offset of the oldest of them, below 0: from the lap before
    if (r0 >= 0) {
      from[2] = sink + r0; to[2] = sink + head.offset + 1;
    } else {
      from[2] = sink + r0 + window; to[2] = sink + window;
      from[1] = sink; to[1] = sink + head.offset + 1;
    }
  }
  TouchedPages t;
  int next = 0;                                                // first page not listed yet
#ifdef __CUDA_ARCH__
#pragma unroll
#endif
  for (int i = 0; i < 3; ++i) {
    int a = from[i] >> page_shift, b = to[i] > from[i] ? ((to[i] - 1) >> page_shift) + 1 : a;
    if (a < next) a = next;
    if (b < a) b = a;
    t.first[i] = a;
    t.count[i] = b - a;
    if (b > a) next = b;
  }
  return t;
}
// no call of up to T tokens a sequence touches more pages than this (a run of m slots lies in at most m / P + 2 pages)
__host__ __device__ __forceinline__ int max_touched_pages(int64_t T, int sink, int window, int page_tokens) {
  const int64_t all = (static_cast<int64_t>(sink) + window + page_tokens - 1) / page_tokens;
  int64_t n = T / page_tokens + 6;
  if (n > T) n = T;
  return static_cast<int>(n < all ? n : all);
}

// Exponent of the smallest power-of-two scale under which a value of magnitude `amax` (finite, >= 0) fits e4m3, whose
// largest number is 448 = 1.75 * 2^8.
__host__ __device__ __forceinline__ int page_exponent(uint32_t amax_bits /* of the fp32 value */) {
  if (amax_bits == 0) return 0;
  const int biased = static_cast<int>(amax_bits >> 23);        // 0: subnormal, clamped below like all that small
  const int e = biased - 127 - 8 + ((amax_bits & 0x7fffffu) > 0x600000u ? 1 : 0);
  return e < kPageMinExp ? kPageMinExp : e;
}

// What a chunk attends to, as one sequence in time order: `kept` rows with the tokens that the cache holds (the sink, then the ring from its
// oldest token on), then the chunk's own rows.  A sequence that holds fewer than `kept` tokens has a gap between its sink and the rest (or
// behind all it holds): distances, which the window goes by, are right behind the gap, and in the sink they do not count.
struct ChunkSeq {
  int held;                  // tokens that the cache holds
  int ring0;                 // ring offset of the oldest token behind the sink
  int phase;                 // position of a row behind the gap, less its row, modulo the window's block
  int seen;                  // first row that the chunk's first token sees behind the sink
};
struct ChunkView {           // what the attention kernel asks of a sequence
  int first;                 // first row behind the gap (0: no gap)
  int sink_end;              // rows of the sink that hold a token
  int phase, pad;
};
__host__ __device__ __forceinline__ ChunkView chunk_view(int kept, int sink, const ChunkSeq& s) {
  if (s.held == kept) return ChunkView{0, sink, s.phase, 0};
  return ChunkView{kept - (s.held > sink ? s.held - sink : 0), s.held < sink ? s.held : sink, s.phase, 0};
}
// Whether the 64 rows of block kb hold a row that a chunk may attend to.
__host__ __device__ __forceinline__ bool chunk_block_held(const ChunkView& v, int sink, int kb) {
  return kb * 64 < sink ? kb * 64 < v.sink_end : (kb + 1) * 64 > v.first;
}

}  // namespace lg
