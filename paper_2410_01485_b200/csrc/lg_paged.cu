// The rolling-buffer cache of the paper's Section 3.2 in 8 bits and in pages: block tables and slot maps built from
// request lengths, an append that quantises, single-token attention over the pages, and a read-back in bf16.
//
// Numbers.  A page holds page_tokens slots of one kv head as e4m3 codes and one fp32 scale, the power of two that
// page_exponent() gives.  A power of two and a floating code: when a page's largest value changes, its other tokens are
// rescaled by exponents alone, which is exact but for codes below the normal range (values under 2^-14 of the largest),
// where scales of amax / 448 would round every token of the page anew with every append.  e4m3 keeps 4 significant bits
// wherever a value lies in its 15 octaves, so nothing is lost by a scale up to twice as large.
#include <math.h>

#include "lg_common.cuh"
#include "lg_decode.cuh"
#include "lg_host.h"
#include "lg_paged.cuh"

namespace lg {

// ---- e4m3 -------------------------------------------------------------------------------
// Round to nearest even; beyond 448 (infinities) the largest code, NaN stays NaN.
__device__ __forceinline__ uint32_t f32x2_to_e4m3x2(float lo, float hi) {
  uint16_t r;
  asm("cvt.rn.satfinite.e4m3x2.f32 %0, %1, %2;" : "=h"(r) : "f"(hi), "f"(lo));
  return r;
}
__device__ __forceinline__ float bf16_lo(uint32_t w) { return __uint_as_float(w << 16); }
__device__ __forceinline__ float bf16_hi(uint32_t w) { return __uint_as_float(w & 0xffff0000u); }

// ---- block tables and slot maps ------------------------------------------------------------
// A CTA works `rows` consecutive sequences and kExtendCols table columns of their new pages; where a sequence's pages
// start in the free list is the sum over the sequences before it, which every CTA adds up for itself (12 bytes a
// sequence out of the L2; a scan across CTAs would cost more round trips than it saves).
constexpr int kExtendThreads = 256, kExtendMaxRows = 32, kExtendCols = 1024;

struct ExtendArgs {
  const int64_t* n_before;
  const int32_t* n_new;      // or null: T_new for all
  const int32_t* free_pages;
  const int32_t* free_start;
  int32_t* table;
  int32_t* free_next;
  int B, T_new, n_free, sink, window, page_shift, stride, rows;
};

__device__ __forceinline__ int new_tokens(const int32_t* n_new, int b, int T) {
  if (!n_new) return T;
  const int t = n_new[b];
  return t < 0 ? 0 : t < T ? t : T;
}

__global__ void __launch_bounds__(kExtendThreads) table_extend_kernel(const ExtendArgs a) {
  pdl_trigger();
  __shared__ int64_t warp_sum[kExtendThreads / 32];
  __shared__ int have[kExtendMaxRows], need[kExtendMaxRows];
  __shared__ int64_t from[kExtendMaxRows];
  const int tid = threadIdx.x, lane = tid & 31, warp = tid >> 5;
  const int b0 = blockIdx.x * a.rows, nb = min(a.rows, a.B - b0);
  pdl_wait();
  auto pages = [&](int b, int& had) {
    const int64_t n = a.n_before[b];
    had = pages_of(n, a.sink, a.window, a.page_shift);
    return n < 0 ? 0 : pages_of(n + new_tokens(a.n_new, b, a.T_new), a.sink, a.window, a.page_shift);
  };
  int64_t sum = 0;
  for (int b = tid; b < b0; b += kExtendThreads) { int h; const int m = pages(b, h); sum += m - h; }
#pragma unroll
  for (int o = 16; o > 0; o >>= 1) sum += __shfl_xor_sync(0xffffffffu, sum, o);
  if (lane == 0) warp_sum[warp] = sum;
  __syncthreads();
  if (warp == 0) {
    int64_t base = a.free_start[0];
    for (int w = 0; w < kExtendThreads / 32; ++w) base += warp_sum[w];
    int h = 0, m = 0;
    if (lane < nb) m = pages(b0 + lane, h);
    int64_t incl = m - h;
#pragma unroll
    for (int o = 1; o < 32; o <<= 1) { const int64_t t = __shfl_up_sync(0xffffffffu, incl, o); if (lane >= o) incl += t; }
    if (lane < nb) { have[lane] = h; need[lane] = m; from[lane] = base + incl - (m - h); }
    if (lane == nb - 1 && b0 + nb == a.B && blockIdx.y == 0) {
      const int64_t next = base + incl;
      a.free_next[0] = static_cast<int32_t>(next < 0x7fffffffll ? next : 0x7fffffffll);
    }
  }
  __syncthreads();
  for (int r = 0; r < nb; ++r) {
    const int n = need[r] - have[r];
    int32_t* row = a.table + static_cast<int64_t>(b0 + r) * a.stride + have[r];
    for (int i = blockIdx.y * kExtendCols + tid; i < min(n, static_cast<int>(blockIdx.y + 1) * kExtendCols); i += kExtendThreads) {
      const int64_t f = from[r] + i;
      row[i] = f >= 0 && f < a.n_free ? a.free_pages[f] : -1;
    }
  }
}

struct SlotMapArgs {
  const int64_t* n_tokens;
  const int64_t* first;
  const int32_t* count;      // or null: T for all
  const int32_t* table;
  int64_t* slot_map;         // [B, T]
  int B, T, sink, window, page_shift, num_pages, stride;
};
constexpr int kSlotMapThreads = 256, kSlotMapPer = 4;   // tokens of a thread, side by side

// A thread's tokens follow each other in the ring, so one 64-bit division (200 cycles) places all of them; 8 bytes are written a
// token, and a page's entry comes out of the L1.
__global__ void __launch_bounds__(kSlotMapThreads) slot_map_kernel(const SlotMapArgs a) {
  pdl_trigger();
  const int b = blockIdx.y, t0 = (blockIdx.x * kSlotMapThreads + threadIdx.x) * kSlotMapPer;
  pdl_wait();
  if (t0 >= a.T) return;
  const int64_t n = a.n_tokens[b], first = a.first[b];
  const int count = new_tokens(a.count, b, a.T);
  const int32_t* table = a.table + static_cast<int64_t>(b) * a.stride;
  // position p of the ring is held iff n - window <= p < n
  const int64_t p0 = first + t0;
  int ring = p0 >= a.sink ? slot_of(p0, 0, a.window) - static_cast<int>(a.sink % a.window) : 0;   // ring offset of p0, (p0 - sink) mod window
  if (ring < 0) ring += a.window;
  int64_t out[kSlotMapPer];
#pragma unroll
  for (int x = 0; x < kSlotMapPer; ++x) {
    const int64_t p = p0 + x;
    out[x] = -1;
    if (t0 + x < count && p >= 0 && p < n && (p < a.sink || p >= n - a.window)) {
      const int slot = p < a.sink ? static_cast<int>(p) : a.sink + ring;
      const int page = checked_page(table[slot >> a.page_shift], a.num_pages);
      if (page >= 0) out[x] = (static_cast<int64_t>(page) << a.page_shift) + (slot & ((1 << a.page_shift) - 1));
    }
    if (p >= a.sink) ring = ring + 1 == a.window ? 0 : ring + 1;
  }
  int64_t* to = a.slot_map + static_cast<int64_t>(b) * a.T + t0;
  if ((reinterpret_cast<uintptr_t>(to) & 15) == 0 && t0 + kSlotMapPer <= a.T) {
#pragma unroll
    for (int x = 0; x < kSlotMapPer; x += 2) *reinterpret_cast<longlong2*>(to + x) = make_longlong2(out[x], out[x + 1]);
  } else {
#pragma unroll
    for (int x = 0; x < kSlotMapPer; ++x)
      if (t0 + x < a.T) to[x] = out[x];
  }
}

// ---- append -----------------------------------------------------------------------------------
struct AppendArgs {
  uint8_t* pool[2];          // K, V: [num_pages, Hkv, P, D]
  float* scale[2];           // [num_pages, Hkv]
  const __nv_bfloat16* rows[2];
  const int32_t* table;
  const int64_t* n_before;
  const int32_t* n_new;      // or null
  int64_t stride_b, stride_h, stride_t;
  int B, Hkv, T, sink, window, page_shift, num_pages, stride, max_touched;
  int units, groups;         // many tokens: (K or V, kv head) pairs a CTA works, CTAs per page
};

// Largest magnitudes: of two bf16 each (low and high half on their own; infinities and NaN count until finite_top has looked), of the codes (4
// to a word; NaN codes do not count).
__device__ __forceinline__ uint32_t top_of_new(uint4 v, uint32_t top) {
  return __vmaxu2(__vmaxu2(__vmaxu2(top, v.x & 0x7fff7fffu), __vmaxu2(v.y & 0x7fff7fffu, v.z & 0x7fff7fffu)), v.w & 0x7fff7fffu);
}
__device__ __forceinline__ bool finite_top(uint32_t top) { return (top & 0x7f80u) != 0x7f80u && (top & 0x7f800000u) != 0x7f800000u; }
__device__ __forceinline__ uint32_t finite_top_of(uint4 v, uint32_t top) {
  const uint32_t w[4] = {v.x, v.y, v.z, v.w};
#pragma unroll
  for (int j = 0; j < 4; ++j) {
    const uint32_t m = w[j] & 0x7fff7fffu;
    if ((m & 0xffffu) < 0x7f80u) top = max(top & 0xffffu, m & 0xffffu) | (top & 0xffff0000u);
    if (m < 0x7f800000u) top = max(top & 0xffff0000u, m & 0xffff0000u) | (top & 0xffffu);
  }
  return top;
}
__device__ __forceinline__ uint32_t top_of_old(uint2 v, uint32_t top) {
  const uint32_t a = v.x & 0x7f7f7f7fu, b = v.y & 0x7f7f7f7fu;
  return __vmaxu4(top, __vmaxu4(a & ~__vcmpeq4(a, 0x7f7f7f7fu), b & ~__vcmpeq4(b, 0x7f7f7f7fu)));
}
// both as the bits of an fp32 magnitude (their order is that of the magnitudes)
__device__ __forceinline__ uint32_t top_bits(uint32_t top_new, uint32_t top_old, float was) {
  uint32_t c = __vmaxu4(top_old, top_old >> 16);
  c = max(c & 0xffu, (c >> 8) & 0xffu);
  const uint32_t old_bits = __float_as_uint(f16x2_to_f32x2(e4m3x2_to_f16x2(c)).x * was);
  return max(max(top_new << 16, top_new & 0xffff0000u), c == 0 ? 0u : old_bits);
}
// (times a power of two in bf16: exact, but for results so small that they become codes of zero)
__device__ __forceinline__ uint32_t code_new2(uint32_t w, uint32_t inv2) {
  uint32_t r;
  asm("mul.rn.bf16x2 %0, %1, %2;" : "=r"(r) : "r"(w), "r"(inv2));
  return f32x2_to_e4m3x2(bf16_lo(r), bf16_hi(r));
}
__device__ __forceinline__ uint2 code_new(uint4 v, float inv) {
  const uint32_t inv2 = __byte_perm(__float_as_uint(inv), 0, 0x3232);   // a power of two is its upper half
  return make_uint2(__byte_perm(code_new2(v.x, inv2), code_new2(v.y, inv2), 0x5410), __byte_perm(code_new2(v.z, inv2), code_new2(v.w, inv2), 0x5410));
}
// (two products: was * inv may leave the range of fp32 where every code is zero)
__device__ __forceinline__ uint32_t recode4(uint32_t c, float was, float inv) {
  const float2 p = f16x2_to_f32x2(e4m3x2_to_f16x2(c)), q = f16x2_to_f32x2(e4m3x2_hi_to_f16x2(c));
  return f32x2_to_e4m3x2(p.x * was * inv, p.y * was * inv) | f32x2_to_e4m3x2(q.x * was * inv, q.y * was * inv) << 16;
}
__device__ __forceinline__ void scale_of(uint32_t bits, float& now, float& inv) {
  const int e = page_exponent(bits);
  now = __uint_as_float(static_cast<uint32_t>(127 + e) << 23);
  inv = __uint_as_float(static_cast<uint32_t>(127 - e) << 23);
}

// One token a sequence: a CTA per (sequence, kv head) of K or of V holds the codes of the page that the token goes to (NU units of 8 a
// thread) and the token's row, finds the largest magnitude and writes the token and, where the scale changed, the others.  What it takes is
// round trips: count, table entry, codes and scale.  Count and entry are read before the wait of an overlapped launch too, so that
// behind it all three travel at once; only where one has changed do they follow each other.
template <int D, int NU>
__global__ void __launch_bounds__(128) paged_append_one_kernel(const AppendArgs a) {
  pdl_trigger();
  constexpr int kThreads = 128, kPerRow = D / 8, kRows = NU * kThreads / kPerRow;
  __shared__ uint32_t warp_max[2][kThreads / 32];
  const int tid = threadIdx.x;
  const uint32_t x = blockIdx.x >> 1, kv = blockIdx.x & 1, b = x / static_cast<uint32_t>(a.Hkv), h = x - b * a.Hkv;
  const int t = a.n_new ? -1 : 1;
  auto count = [&]() { return __ldcg(reinterpret_cast<const long long*>(a.n_before) + b); };
  auto entry = [&](int64_t n) { return n < 0 ? -1 : __ldcg(a.table + static_cast<int64_t>(b) * a.stride + (slot_of(n, a.sink, a.window) >> a.page_shift)); };
  int64_t n0 = count();
  int lp_entry = entry(n0);
  pdl_wait();
#pragma unroll 1
  for (int round = 0; round < 4; ++round) {   // (the second is the last, unless someone writes the counts meanwhile)
    const int64_t n_seen = n0;
    const int entry_seen = lp_entry;
    n0 = count();
    lp_entry = entry(n_seen);
    const bool none = t < 0 && a.n_new[b] < 1;
    const int slot = n_seen < 0 ? 0 : slot_of(n_seen, a.sink, a.window), page = checked_page(entry_seen, a.num_pages);
    const int at = slot & (kRows - 1);                                   // the token's row in its page
    const int64_t after = n_seen + 1, cap = static_cast<int64_t>(a.sink) + a.window;
    const int held = static_cast<int>((after < cap ? after : cap) - (slot - at));   // slots of the page, from its first one on, that hold a token
    const int64_t unit = static_cast<int64_t>(page < 0 ? 0 : page) * a.Hkv + h;
    uint8_t* codes = (kv ? a.pool[1] : a.pool[0]) + unit * (kRows * D);
    float* scale = (kv ? a.scale[1] : a.scale[0]) + unit;
    const uint4 row = *reinterpret_cast<const uint4*>((kv ? a.rows[1] : a.rows[0]) + b * a.stride_b + h * a.stride_h + tid % kPerRow * 8);
    const float was = *scale;
    uint2 v[NU];
    uint32_t top = top_of_new(row, 0u), top_old = 0;                     // (every row's threads look at the whole token)
    if (!finite_top(top)) top = finite_top_of(row, 0u);
#pragma unroll
    for (int u = 0; u < NU; ++u) {
      const int e = u * kThreads + tid, rr = e / kPerRow;
      v[u] = rr < held && rr != at ? *reinterpret_cast<const uint2*>(codes + e * 8) : make_uint2(0u, 0u);
    }
#pragma unroll
    for (int u = 0; u < NU; ++u) top_old = top_of_old(v[u], top_old);
    uint32_t bits = __reduce_max_sync(0xffffffffu, top_bits(top, top_old, was));
    if (__any_sync(0xffffffffu, n0 != n_seen || lp_entry != entry_seen)) bits = 0xffffffffu;   // the plan was of another time
    if ((tid & 31) == 0) warp_max[round & 1][tid >> 5] = bits;
    __syncthreads();
    bits = 0;
#pragma unroll
    for (int w = 0; w < kThreads / 32; ++w) bits = max(bits, warp_max[round & 1][w]);
    if (bits == 0xffffffffu) {
      if (n0 != n_seen) lp_entry = entry(n0);
      continue;
    }
    if (n_seen < 0 || none || page < 0) return;
    float now, inv;
    scale_of(bits, now, inv);
    const bool rescale = held > 1 && was != now;
#pragma unroll
    for (int u = 0; u < NU; ++u) {
      const int e = u * kThreads + tid, rr = e / kPerRow;
      if (rr == at) *reinterpret_cast<uint2*>(codes + e * 8) = code_new(row, inv);
      else if (rescale && rr < held) *reinterpret_cast<uint2*>(codes + e * 8) = make_uint2(recode4(v[u].x, was, inv), recode4(v[u].y, was, inv));
    }
    if (tid == 0) *scale = now;
    return;
  }
}

// Several tokens a sequence: a CTA takes one page that a sequence's tokens go to, for some of the (K or V, kv head) pairs one after
// the other.  It holds a pair's new rows (bf16) and its kept old ones (codes) in registers, finds the largest magnitude, and writes codes and
// scale, while the next pair's rows are on their way.  Old rows are written only where the scale changed, and a page whose live tokens are all
// new is not read.  HBM-bound, with the conversions not far behind: 32K tokens into 32 heads 134 us, 805 MB at 6.0 TB/s; 142 us with four
// warps fewer an SM, 154 us with the products in fp32 and a test for infinities in the maximum of every word.
template <int D, int NU, int kThreads>   // NU units of 8 elements a thread: page_tokens = NU * 8 * kThreads / D
__global__ void __launch_bounds__(kThreads) paged_append_kernel(const AppendArgs a) {
  pdl_trigger();
  constexpr int kPerRow = D / 8, kRows = NU * kThreads / kPerRow;
  static_assert(kRows <= kThreads, "a thread per slot of the page");
  __shared__ int src[kRows];                 // new token of each slot; -1: kept old one; -2: nothing
  __shared__ uint32_t warp_max[2][kThreads / 32];
  const int tid = threadIdx.x;
  uint32_t x = blockIdx.x;
  const int g = x % a.groups; x /= a.groups;
  const int i = x % a.max_touched, b = x / a.max_touched;
  pdl_wait();
  const int64_t n0 = a.n_before[b];
  if (n0 < 0) return;                        // a negative count addresses nothing: the sequence is skipped
  const int64_t n1 = n0 + new_tokens(a.n_new, b, a.T);
  const RingHead head = ring_head(n1, a.sink, a.window);
  const TouchedPages t = touched_pages(n0, n1, head, a.sink, a.window, a.page_shift);
  if (i >= t.total()) return;
  const int lp = t.page(i);
  const int page = checked_page(a.table[static_cast<int64_t>(b) * a.stride + lp], a.num_pages);
  bool old = false;
  if (tid < kRows) {
    const int64_t pos = held_position(lp * kRows + tid, n1, head, a.sink, a.window);
    src[tid] = pos < 0 ? -2 : pos < n0 ? -1 : static_cast<int>(pos - n0);
    old = pos >= 0 && pos < n0;
  }
  const bool any_old = __syncthreads_or(old) != 0;
  if (page < 0) return;
  int from[NU];                              // src of my units
#pragma unroll
  for (int u = 0; u < NU; ++u) from[u] = src[(u * kThreads + tid) / kPerRow];
  const int last = min((g + 1) * a.units, 2 * a.Hkv);
  uint4 next[NU], v[NU];
  float was_next = 0.f, was;
  auto load = [&](int pair) {                // 8 new values a unit, or 8 old codes in (x, y)
    const int kv = pair >= a.Hkv, h = pair - (kv ? a.Hkv : 0);
    const int64_t unit = static_cast<int64_t>(page) * a.Hkv + h;
    const __nv_bfloat16* rows = (kv ? a.rows[1] : a.rows[0]) + b * a.stride_b + h * a.stride_h;
    const uint8_t* codes = (kv ? a.pool[1] : a.pool[0]) + unit * (kRows * D);
#pragma unroll
    for (int u = 0; u < NU; ++u) {
      const int e = u * kThreads + tid;
      next[u] = make_uint4(0, 0, 0, 0);
      if (from[u] >= 0) next[u] = *reinterpret_cast<const uint4*>(rows + from[u] * a.stride_t + e % kPerRow * 8);
      else if (from[u] == -1) { const uint2 c = *reinterpret_cast<const uint2*>(codes + e * 8); next[u].x = c.x; next[u].y = c.y; }
    }
    if (any_old) was_next = (kv ? a.scale[1] : a.scale[0])[unit];
  };
  load(g * a.units);
#pragma unroll 1
  for (int pair = g * a.units; pair < last; ++pair) {
#pragma unroll
    for (int u = 0; u < NU; ++u) v[u] = next[u];
    was = was_next;
    if (pair + 1 < last) load(pair + 1);
    uint32_t top = 0, top_old = 0;
#pragma unroll
    for (int u = 0; u < NU; ++u) {
      if (from[u] >= 0) top = top_of_new(v[u], top);
      else if (from[u] == -1) top_old = top_of_old(make_uint2(v[u].x, v[u].y), top_old);
    }
    if (!finite_top(top)) {
      top = 0;
#pragma unroll
      for (int u = 0; u < NU; ++u)
        if (from[u] >= 0) top = finite_top_of(v[u], top);
    }
    uint32_t bits = __reduce_max_sync(0xffffffffu, top_bits(top, top_old, was));
    if ((tid & 31) == 0) warp_max[pair & 1][tid >> 5] = bits;
    __syncthreads();
    bits = 0;
#pragma unroll
    for (int w = 0; w < kThreads / 32; ++w) bits = max(bits, warp_max[pair & 1][w]);
    float now, inv;
    scale_of(bits, now, inv);
    const bool rescale = any_old && was != now;
    const int kv = pair >= a.Hkv, h = pair - (kv ? a.Hkv : 0);
    const int64_t unit = static_cast<int64_t>(page) * a.Hkv + h;
    uint8_t* codes = (kv ? a.pool[1] : a.pool[0]) + unit * (kRows * D);
#pragma unroll
    for (int u = 0; u < NU; ++u) {
      uint2* to = reinterpret_cast<uint2*>(codes + (u * kThreads + tid) * 8);
      if (from[u] >= 0) *to = code_new(v[u], inv);
      else if (from[u] == -1 && rescale) *to = make_uint2(recode4(v[u].x, was, inv), recode4(v[u].y, was, inv));
    }
    if (tid == 0) (kv ? a.scale[1] : a.scale[0])[unit] = now;
  }
}

// ---- rows of the cache in bf16 ---------------------------------------------------------------
struct GatherArgs {
  const uint8_t* pool[2];
  const float* scale[2];
  const int64_t* slot_map;   // [B, T]
  uint4* out[2];             // [B, Hkv, T, D]
  int Hkv, T, page_shift, num_pages;
};

// A thread takes 16 elements of a token's K, then of its V: the slot, then scale and codes, then two 16-byte pieces of the row.  HBM-bound: 3
// bytes an element, two thirds of them written (32K tokens of 32 heads 126 us, 805 MB at 6.4 TB/s; with K and V or several tokens side by
// side in a thread 139-145 us: what the thread has in flight is not what counts, and the rows are then written further apart).
template <int D>
__global__ void __launch_bounds__(kGatherThreads) paged_gather_kernel(const GatherArgs a) {
  pdl_trigger();
  constexpr int kPerRow = D / 16;
  const int t = blockIdx.x * (kGatherThreads / kPerRow) + threadIdx.x / kPerRow, c = threadIdx.x % kPerRow, h = blockIdx.y, b = blockIdx.z;
  if (t >= a.T) return;
  pdl_wait();
  const int64_t slot = a.slot_map[static_cast<int64_t>(b) * a.T + t];
  const int64_t page = slot >> a.page_shift;
  const bool on = slot >= 0 && page < a.num_pages;
  const int64_t unit = on ? page * a.Hkv + h : 0;
  const int64_t at = ((unit << a.page_shift) + (slot & ((1 << a.page_shift) - 1))) * kPerRow + c;
  const int64_t to = ((static_cast<int64_t>(b) * a.Hkv + h) * a.T + t) * kPerRow + c;
#pragma unroll
  for (int x = 0; x < 2; ++x) {
    uint4 lo = make_uint4(0, 0, 0, 0), hi = lo;
    if (on) dequant16(*(reinterpret_cast<const uint4*>(a.pool[x]) + at), a.scale[x][unit], lo, hi);
    a.out[x][to * 2] = lo;
    a.out[x][to * 2 + 1] = hi;
  }
}

// ---- single-token attention ---------------------------------------------------------------------
// The 32-token tiles of all (sequence, kv head, group of <= 8 query heads) units form one sequence that is cut into slices, one per CTA
// (kMergeTiles), and these into equal runs, one per warp.  A warp streams its run through a ring of its own of
// kPagedSlots half tiles, K and V in turn (cp.async, 16-byte pieces XOR-swizzled by the row, so that fragments are read without
// bank conflicts); the ring runs on from one unit to the next, so the latencies of a unit (its pages, its scales, its tiles) are
// paid behind the tiles of the one before.  A unit that lies inside a run is finished by its warp; of the others a warp has
// at most two pieces, which the CTA merges in shared memory when its runs are done, and units that several CTAs share go through
// records in the workspace, which the CTA that delivers the last one merges in order.
// Scores are S^T = K Q^T and outputs O^T = V^T P^T on mma.sync m16n8k16 with f16 operands: an e4m3 code is an f16 number, so K
// and V enter without rounding, and q (8 significant bits) does not lose any either once its row is scaled by a power of
// two.  A contraction 8 heads wide is far below a tcgen05 tile.
// (K as e4m3 in products of its own kind, with q as the sum of two e4m3 numbers, needs no conversion but was slower: one sequence over 4224
// slots 14.0 us against 12.4 with its append, 16 over 60-131 thousand 1.06 times as long.)
// A page's K scale multiplies its scores; that of V goes into the weights, w_j = p_j vs / vs_ref with the largest scale of the unit so far, so that
// they fit f16 (kWeightTop), while the row sum is kept in fp32.  Where the scales of a unit's pages lie more than 2^6 apart that would
// cost bits, and the weights get a running reference of their own, w_j = 2^(s_j - m + log2 vs - r), r relative to the probabilities' m (log2 vs
// added to a large score would be rounded away).
// The instructions of a tile count although HBM bounds the kernel: in a loop of tens of milliseconds the board is at its power limit, and the clock
// that it takes back is the SMs'.  16 sequences over 60-131 thousand slots, 3.13 GB a step: 502 us (6.2 TB/s) at 1965 MHz, 518-522 us (6.0 TB/s) at the
// 1580 MHz of thousands of steps in a row; there a maximum and a rescaling in every tile and two exponentials a weight cost 4 % more.
constexpr int kPagedTile = 32, kPagedHalf = 16;   // tokens of a tile, and of what lies in one page whatever its size
constexpr int kPagedSlots = 5;          // 4 KB each at D = 128: three tiles' K and two tiles' V, or the other way round
constexpr int kPagedMaxB = 4096;        // sequences of one launch (their prefix sums lie in shared memory)
// Slices that cut across units make some CTA merge the records of two of them, one after the other, and wait twice: about what kMergeTiles
// tiles of a CTA take, half of that where units are still shared by several CTAs of their own.  So a CTA gets a unit whole, or an equal share of
// one, where the largest share is at most that, or a fifth, above the average one.  Decode and append, cut evenly across units | so:
//   one CTA a unit      16 sequences x 8 kv heads x 4224 slots 33.7 | 31.5 us, 14 x 8 x 1024 16.0 | 13.2, 48 x 4 x 1088 (D = 64) 15.6 | 13.2, 24 x 8 x 512 (D = 64)
//                       13.6 | 9.7 (10 x 8 x 4224, where the share is 132 tiles and the average 72, would be 23.8 | 30.4, and is cut evenly)
//   several             1 x 8 x 4224 12.4 | 11.2, 1 x 4 x 8192 13.6 | 11.2, 4 x 8 x 4224 16.3 | 15.2, 9 x 8 x 4224 22.5 | 21.3
//   several units a CTA, if alike   32 x 8 x 4224 58.4 | 56.1, 200 x 8 x 1024 94.2 | 90.3
constexpr uint32_t kMergeTiles = 16;
// The weights' place in f16, log2: they stay below 2^kWeightTop (f16 ends just under 2^16), and a reference that moves puts the maximum at
// 2^kWeightMax.  The row sum counts weights that an f16 of theirs drops, and beside one large weight (a sink's) there may be 10^5 of them: so the
// maximum lies high, not at 1, and they keep 11 bits down to 2^-25 of it and something down to 2^-36.  The room above spares moves: maximum at 2^7 | 2^11 |
// 2^13, 1 and 16 sequences over 4224 slots 11.16 32.2 | 11.15 32.2 | 11.15 32.4 us with their append, 48 small ones 12.6 | 12.6 | 12.7.
constexpr float kWeightTop = 15.f, kWeightMax = 11.f;
constexpr float kNoScore = -3.4e38f;    // the reference of a row that has attended nothing

struct PagedDecodeArgs {
  const __nv_bfloat16* q;        // [B, Hq, D]
  const float* scale[2];         // K, V: [num_pages, Hkv]
  const uint8_t* pool[2];
  const int32_t* table;          // [B, stride]
  const int64_t* n_tokens;       // [B]
  float* part;
  __nv_bfloat16* o;
  float* lse;
  unsigned int* unit_count;
  unsigned int* error_word;
  int B, Hq, Hkv, G, HG, C;
  int sink, block_tokens;
  int page_shift, num_pages, stride;
  float scale_log2;
};

template <int BYTES>
__device__ __forceinline__ void copy_async(uint32_t smem_dst, const void* src) {
  if (BYTES == 16) asm volatile("cp.async.cg.shared.global [%0], [%1], 16;" ::"r"(smem_dst), "l"(src) : "memory");
  else asm volatile("cp.async.ca.shared.global [%0], [%1], 4;" ::"r"(smem_dst), "l"(src) : "memory");
}
__device__ __forceinline__ void copy_commit() { asm volatile("cp.async.commit_group;" ::: "memory"); }
template <int N>
__device__ __forceinline__ void copy_wait() { asm volatile("cp.async.wait_group %0;" ::"n"(N) : "memory"); }
__device__ __forceinline__ void prefetch_l1(const void* p) { asm volatile("prefetch.global.L1 [%0];" ::"l"(p)); }
__device__ __forceinline__ void mma16816_f16(float* c, uint32_t a0, uint32_t a1, uint32_t a2, uint32_t a3, uint32_t b0,
                                             uint32_t b1) {
  asm volatile(
      "mma.sync.aligned.m16n8k16.row.col.f32.f16.f16.f32 {%0, %1, %2, %3}, {%4, %5, %6, %7}, {%8, %9}, {%0, %1, %2, %3};"
      : "+f"(c[0]), "+f"(c[1]), "+f"(c[2]), "+f"(c[3])
      : "r"(a0), "r"(a1), "r"(a2), "r"(a3), "r"(b0), "r"(b1));
}
__device__ __forceinline__ uint32_t pack_f16(float lo, float hi) {
  uint32_t r;
  asm("cvt.rn.f16x2.f32 %0, %1, %2;" : "=r"(r) : "f"(hi), "f"(lo));
  return r;
}
__device__ __forceinline__ float fast_log2(float x) {   // (exact for the powers of two of our own scales)
  float y;
  asm("lg2.approx.ftz.f32 %0, %1;" : "=f"(y) : "f"(x));
  return y;
}

__device__ __forceinline__ float min_nan(float a, float b) {   // the smaller one; NaN if either is
  float r;
  asm("min.NaN.f32 %0, %1, %2;" : "=f"(r) : "f"(a), "f"(b));
  return r;
}

template <int D>
struct PagedSmem {
  static constexpr int kSlot = kPagedTile * D;                          // K (or V) of a tile
  static constexpr int kRing = kPagedSlots * kSlot;                     // of a warp
  static constexpr int kPiece = kDecHeads * (D + 2) * 4;                // a piece of a unit: O of 8 heads, (m, l) behind each
  static constexpr int kPieces = kDecWarps * kRing;                     // the piece with which a warp's run begins
  static constexpr int kScales = kPieces + kDecWarps * kPiece;          // per warp, of three tiles: (K, V) scale of both halves
  static constexpr int kMeta = kScales + kDecWarps * 3 * 16;            // the units of the warps' pieces: (number, b, k, -), number -1: none
  static constexpr int kShare = kMeta + kDecWarps * 2 * 16;             // the CTA's first and last unit: (number, first CTA, CTAs, row of its first head), its heads
  static constexpr int kCum = kShare + 2 * 32;
  static_assert(kPiece <= kRing && kScales % 16 == 0, "the piece with which a run ends lies over the warp's ring");
  static int bytes(int B) { return kCum + (B + 1) * 4 + B; }
};

// byte offset of 16-byte chunk c of row r in a slot
template <int D>
__device__ __forceinline__ uint32_t tile_offset(int r, int c) {
  return r * D + ((c ^ (D == 128 ? r & 7 : (r >> 1) & 3)) << 4);
}

// tokens that sequence b holds (through the L2: read before and again behind the wait of an overlapped launch)
__device__ __forceinline__ int paged_valid(const PagedDecodeArgs& a, int b) {
  const int64_t n = __ldcg(reinterpret_cast<const long long*>(a.n_tokens) + b);
  return static_cast<int>(n < a.C ? (n < 0 ? 0 : n) : a.C);
}

// cum[b] = tiles of the sequences before b, b = 0 .. B, and behind them a byte per sequence: empty places of its last tile.
// Returns whether some sequence holds no token; mine: tokens of the thread's first sequence.  All threads.
__device__ __forceinline__ bool paged_build_cum(const PagedDecodeArgs& a, int* cum, int& mine) {
  __shared__ int warp_sum[kDecWarps];
  const int tid = threadIdx.x, lane = tid & 31, warp = tid >> 5;
  const int each = (a.B + kDecThreads - 1) / kDecThreads, b0 = tid * each, b1 = min(a.B, b0 + each);
  int local = 0;
  bool empty = false;
  mine = 0;
#pragma unroll 1
  for (int b = b0; b < b1; ++b) {
    const int v = paged_valid(a, b), n = (v + kPagedTile - 1) / kPagedTile;
    if (b == b0) mine = v;
    cum[b + 1] = n;
    reinterpret_cast<uint8_t*>(cum + a.B + 1)[b] = static_cast<uint8_t>(n * kPagedTile - v);
    local += n;
    empty |= n == 0;
  }
  int run = local;
#pragma unroll
  for (int o = 1; o < 32; o <<= 1) { const int t = __shfl_up_sync(0xffffffffu, run, o); if (lane >= o) run += t; }
  if (lane == 31) warp_sum[warp] = run;
  __syncthreads();
  run -= local;
#pragma unroll
  for (int w = 0; w < kDecWarps; ++w) run += w < warp ? warp_sum[w] : 0;
#pragma unroll 1
  for (int b = b0; b < b1; ++b) { run += cum[b + 1]; cum[b + 1] = run; }
  if (tid == 0) cum[0] = 0;
  return __syncthreads_or(empty) != 0;
}

// a place in the sequence of tiles: tile t of the nt of unit (b, kv head, group of query heads)
struct TilePos {
  int b, kvh, hg, t, nt;
  __device__ __forceinline__ void next_unit(const int* cum, int Hkv, int HG) {
    t = 0;
    if (++hg < HG) return;
    hg = 0;
    if (++kvh < Hkv) return;
    kvh = 0;
    do ++b; while (cum[b + 1] == cum[b]);
    nt = cum[b + 1] - cum[b];
  }
};

// The pages of up to 16 tiles of one unit, one half tile per lane.
constexpr int kNoToken = -2147483647 - 1;   // in place of a table entry: a half tile that holds no token
struct PageBatch {
  TilePos at;       // its first tile
  int count, page;  // tiles; the lane's table entry
};

// Block-aligned window: the ring's oldest tokens that it leaves out, (first ring offset, number), cyclic.  (Out of line: 64-bit divisions that
// most calls do not come by.)
static __device__ __noinline__ int2 left_out(int64_t n, int C, int sink, int block_tokens) {
  const int w = C - sink;
  if (n <= C) return make_int2(0, 0);
  const int64_t first_held = n - w, first_kept = ((n - 1) / block_tokens - w / block_tokens + 1) * block_tokens;
  if (first_kept <= first_held) return make_int2(0, 0);
  return make_int2(static_cast<int>((first_held - sink) % w), static_cast<int>(first_kept - first_held));
}

// (A sum of zero: nothing was attended.  One that is NaN stays NaN.)
__device__ __forceinline__ float lse_of(float m, float l) { return l != 0.f ? (m + fast_log2(l)) * 0.6931471805599453f : -INFINITY; }

// The records of a unit, one per CTA from first_cta on, merged in that order into o and lse: a warp per head, a lane per record's weight.
// The records sit in the L2, a round trip of a microsecond away: the values of up to 32 travel together, and their weights with them.
// (One sequence, 8 kv heads, 17 records a unit: in two batches of 16 the merge took 4.6 of the kernel's 10.1 us.)
template <int D>
__device__ __forceinline__ void merge_records(const PagedDecodeArgs& a, int64_t qh0 /* row of the unit's first head */, int heads, int u, int first_cta, int n_rec) {
  constexpr int V = D / 32;                  // values of a lane
  const int lane = threadIdx.x & 31, head = threadIdx.x >> 5;
  if (head >= heads) return;
  constexpr int kRec = kDecHeads * (D + 2);
  const float* recs = a.part + (static_cast<int64_t>(first_cta) + u) * kRec;
  const float* mine = recs + head * D + lane * V;
  float m = -INFINITY, l = 0.f, acc[V] = {};
#pragma unroll 1
  for (int i0 = 0; i0 < n_rec; i0 += 32) {   // (more than 32 records: the sums move to the larger of the maxima)
    float2 ml = make_float2(-INFINITY, 0.f);
    if (i0 + lane < n_rec) ml = __ldcg(reinterpret_cast<const float2*>(recs + static_cast<int64_t>(i0 + lane) * kRec + kDecHeads * D) + head);
    float v[32][V];
#pragma unroll
    for (int x = 0; x < 32; ++x) {
      const float* src = mine + static_cast<int64_t>(i0 + x) * kRec;
#pragma unroll
      for (int z = 0; z < V; ++z) v[x][z] = 0.f;
      if (i0 + x >= n_rec) continue;
      if (V == 4) {
        const float4 t = __ldcg(reinterpret_cast<const float4*>(src));
        v[x][0] = t.x; v[x][1] = t.y; v[x][V - 2] = t.z; v[x][V - 1] = t.w;
      } else {
        const float2 t = __ldcg(reinterpret_cast<const float2*>(src));
        v[x][0] = t.x; v[x][1] = t.y;
      }
    }
    float mn = fmaxf(m, ml.x);
#pragma unroll
    for (int o = 16; o > 0; o >>= 1) mn = fmaxf(mn, __shfl_xor_sync(0xffffffffu, mn, o));
    const float mu = mn == -INFINITY ? 0.f : mn, moved = fast_exp2(m - mu), f = fast_exp2(ml.x - mu);
    m = mn;
    l = l * moved + f * ml.y;
#pragma unroll
    for (int z = 0; z < V; ++z) acc[z] *= moved;
#pragma unroll
    for (int x = 0; x < 32; ++x) {
      const float fx = __shfl_sync(0xffffffffu, f, x);
#pragma unroll
      for (int z = 0; z < V; ++z) acc[z] += fx * v[x][z];
    }
  }
#pragma unroll
  for (int o = 16; o > 0; o >>= 1) l += __shfl_xor_sync(0xffffffffu, l, o);
  const float inv = l != 0.f ? __fdividef(1.f, l) : 0.f;
#pragma unroll
  for (int z = 0; z < V; z += 2)
    reinterpret_cast<uint32_t*>(a.o + (qh0 + head) * D + lane * V)[z / 2] = l != 0.f ? pack_bf16(acc[z] * inv, acc[z + 1] * inv) : 0u;
  if (lane == 0 && a.lse) a.lse[qh0 + head] = lse_of(m, l);
}

// (The size of this kernel's code is a time of its own: what a small decode runs once it also fetches once, about 130 cycles for 8
// instructions.  Hence single copies of what several places need, 32-bit arithmetic, one reciprocal a row.)
template <int D>
__global__ void __launch_bounds__(kDecThreads, D == 64 ? 2 : 1) paged_decode_kernel(const PagedDecodeArgs a) {
  extern __shared__ __align__(128) uint8_t sm[];
  using SM = PagedSmem<D>;
  int* cum = reinterpret_cast<int*>(sm + SM::kCum);
  int4* meta = reinterpret_cast<int4*>(sm + SM::kMeta);
  const int warp = threadIdx.x >> 5, lane = threadIdx.x & 31, r = lane >> 2, c = lane & 3;
  const int ups = a.Hkv * a.HG, me = blockIdx.x;
  pdl_trigger();

  uint32_t per = 1, f0 = 0, f1 = 0, g0 = 0, g1 = 0;                     // tiles: of a CTA, my CTA's, my warp's (the host sees to it that all fit 31 bits)
  auto valid_of = [&](const TilePos& p) { return p.nt * kPagedTile - reinterpret_cast<const uint8_t*>(cum + a.B + 1)[p.b]; };
  auto find = [&](uint32_t g) {                                         // the place of tile g
    int lo = 0, hi = a.B;                                               // cum[lo] * ups <= g < cum[hi] * ups
#pragma unroll 1
    while (hi - lo > 1) {
      const int mid = (lo + hi) >> 1;
      if (static_cast<uint32_t>(cum[mid]) * ups <= g) lo = mid; else hi = mid;
    }
    TilePos p;
    p.b = lo;
    p.nt = cum[lo + 1] - cum[lo];
    const uint32_t rel = g - static_cast<uint32_t>(cum[lo]) * ups, k = rel / static_cast<uint32_t>(p.nt);
    p.t = static_cast<int>(rel - k * p.nt);
    p.kvh = a.HG == 1 ? static_cast<int>(k) : static_cast<int>(k / static_cast<uint32_t>(a.HG));
    p.hg = static_cast<int>(k) - p.kvh * a.HG;
    return p;
  };
  auto fetch = [&](PageBatch& p, uint32_t left) {                       // count and page of a batch whose place is known
    p.count = static_cast<int>(min(static_cast<uint32_t>(min(16, p.at.nt - p.at.t)), left));
    const int slot = p.at.t * kPagedTile + lane * kPagedHalf;           // (the last half tile may hold no token)
    p.page = lane < 2 * p.count && slot < valid_of(p.at) ? __ldcg(a.table + static_cast<int64_t>(p.at.b) * a.stride + (slot >> a.page_shift)) : kNoToken;
  };
  const int in_page = (1 << a.page_shift) - 1;
  auto row_of = [&](const PageBatch& p, int page) {                     // of the pool: the lane's half tile in that page
    return ((page * a.Hkv + p.at.kvh) << a.page_shift) + (p.at.t * kPagedTile + lane * kPagedHalf & in_page);
  };
  PageBatch next{};                                                     // what is asked for next
  // the thread's pieces of q: dims 16 k + 4 c to + 3 of head r of the unit's group
  uint2 qw[D / 16];
  auto load_q = [&](const TilePos& p) {
    const int head = p.hg * kDecHeads + r;
    const uint2* qrow = reinterpret_cast<const uint2*>(a.q + (static_cast<int64_t>(p.b) * a.Hq + p.kvh * a.G + min(head, a.G - 1)) * D) + c;
#pragma unroll
    for (int k = 0; k < D / 16; ++k) qw[k] = qrow[4 * k];
  };

  // Before the wait: the plan from the counts and the table as they stand, and my first tiles asked into the L2, while the kernel before
  // (an append) still runs.  What is read here is used for addresses inside the pools only; behind the wait counts and table
  // are read again, in one trip with q, and the plan is made anew where a count has changed.
  bool any_empty = false;
#pragma unroll 1
  for (int round = a.B <= kDecThreads ? 0 : 1; round < 2; ++round) {
    int mine = 0;
    if (round == 1) pdl_wait();
    any_empty = paged_build_cum(a, cum, mine);
    const uint32_t total = static_cast<uint32_t>(cum[a.B]) * ups;
    per = max(1u, (total + gridDim.x - 1) / gridDim.x);
    f0 = min(total, per * me);
    f1 = min(total, f0 + per);
    int mates = 0, ahead = 0;                                           // CTAs that share my only unit, those of them before me (0: slices across units)
    // slices that keep to units (kMergeTiles)
    if (a.B <= 2 * kSms) {
      const uint32_t grid = gridDim.x, units = ups * a.B, all = cum[a.B];
      auto tiles_of = [&](int b) { return b < a.B ? static_cast<uint32_t>(cum[b + 1] - cum[b]) : 0u; };
      uint32_t most = 0, cut = 0;
#pragma unroll 1
      for (int b = lane; b < a.B; b += 32) most = max(most, tiles_of(b));
      most = __reduce_max_sync(0xffffffffu, most);
      const uint32_t held = (units + grid - 1) / grid * most;
      if (held <= max(per + kMergeTiles, per + per / 5)) {              // units whole
        if (units <= grid) cut = most;
        else if (most * a.B == all) { per = held; f0 = min(total, per * me); f1 = min(total, f0 + per); }   // (several a CTA: alike ones only)
      } else if (2 * units <= grid) {                                   // several CTAs a unit: shares of up to `cut` tiles, as small as all fit
        const uint32_t slices = grid / ups, room = max(per + kMergeTiles / 2, per + per / 5);   // (of a kv head's units together)
        cut = (all + slices - 1) / slices;
#pragma unroll 1
        for (int tries = 0; cut <= room; ++tries) {
          uint32_t sum = 0, next_cut = most;                            // CTAs; the smallest cut with which a unit takes one less
#pragma unroll 1
          for (int b = lane; b < a.B; b += 32) {
            const uint32_t nt = tiles_of(b), n = (nt + cut - 1) / cut;
            sum += n;
            if (n > 1) next_cut = min(next_cut, (nt + n - 2) / (n - 1));
          }
          if (__reduce_add_sync(0xffffffffu, sum) <= slices) break;
          cut = tries < 8 ? max(__reduce_min_sync(0xffffffffu, next_cut), cut + cut / 32) : most;
        }
        if (cut > room) cut = 0;
      }
      if (cut > 0) {
        f0 = f1 = total;
        uint32_t before = 0;                                            // CTAs of the sequences before b0
#pragma unroll 1
        for (int b0 = 0; b0 < a.B; b0 += 32) {                          // (a lane per sequence)
          const uint32_t nt = tiles_of(b0 + lane), n = (nt + cut - 1) / cut;
          uint32_t upto = n * ups;
#pragma unroll
          for (int o = 1; o < 32; o <<= 1) { const uint32_t t = __shfl_up_sync(0xffffffffu, upto, o); if (lane >= o) upto += t; }
          upto += before;
          const unsigned past = __ballot_sync(0xffffffffu, upto > static_cast<uint32_t>(me));
          if (past == 0) { before = __shfl_sync(0xffffffffu, upto, 31); continue; }
          const int y = __ffs(past) - 1;
          const uint32_t nb = __shfl_sync(0xffffffffu, n, y), ntb = __shfl_sync(0xffffffffu, nt, y), at = me - (__shfl_sync(0xffffffffu, upto, y) - nb * ups);
          const uint32_t k = at / nb, each = ntb / nb, more = ntb - each * nb;   // (the first `more` CTAs of a unit take one tile more)
          mates = nb; ahead = at - k * nb;
          f0 = static_cast<uint32_t>(cum[b0 + y]) * ups + k * ntb + ahead * each + min(static_cast<uint32_t>(ahead), more);
          f1 = f0 + each + (static_cast<uint32_t>(ahead) < more ? 1 : 0);
          break;
        }
      }
    }
    g0 = f0 + (f1 - f0) * warp / kDecWarps;
    g1 = f0 + (f1 - f0) * (warp + 1) / kDecWarps;
    if (g0 < g1) { next.at = find(g0); fetch(next, g1 - g0); }
    if (warp < 2 && f0 < f1) {                                          // who shares my CTA's first (warp 0) and last unit
      const TilePos p = find(warp ? f1 - 1 : f0);
      const uint32_t k = p.kvh * a.HG + p.hg, first = static_cast<uint32_t>(cum[p.b]) * ups + k * p.nt;
      const int c_lo = mates > 0 ? me - ahead : static_cast<int>(first / per), c_hi = mates > 0 ? c_lo + mates - 1 : static_cast<int>((first + p.nt - 1) / per);
      if (lane == 0) {
        reinterpret_cast<int4*>(sm + SM::kShare)[2 * warp] = make_int4(p.b * ups + k, c_lo, c_hi - c_lo + 1, p.b * a.Hq + p.kvh * a.G + p.hg * kDecHeads);
        reinterpret_cast<int4*>(sm + SM::kShare)[2 * warp + 1].x = min(kDecHeads, a.G - p.hg * kDecHeads);
      }
    }
    if (round == 0) {
      const int page = checked_page(next.page, a.num_pages);
      if (g0 < g1 && lane < 2 * min(next.count, 3) && page >= 0) {
        const int64_t row = row_of(next, page);
        prefetch_l2(a.pool[0] + row * D, kPagedHalf * D);
        prefetch_l2(a.pool[1] + row * D, kPagedHalf * D);
      }
      pdl_wait();
      if (g0 < g1) fetch(next, g1 - g0);
    }
    if (g0 < g1) load_q(next.at);
    if (!__syncthreads_or(round == 0 && threadIdx.x < a.B && paged_valid(a, threadIdx.x) != mine)) break;
  }
  if (any_empty) {                                                      // sequences without tokens: their empty results
#pragma unroll 1
    for (int b = me; b < a.B; b += gridDim.x) {
      if (cum[b + 1] != cum[b]) continue;
#pragma unroll 1
      for (int x = threadIdx.x; x < a.Hq * (D / 2); x += kDecThreads) {
        reinterpret_cast<uint32_t*>(a.o + static_cast<int64_t>(b) * a.Hq * D)[x] = 0u;
        if (a.lse && x < a.Hq) a.lse[static_cast<int64_t>(b) * a.Hq + x] = -INFINITY;
      }
    }
  }
  if (f0 >= f1) return;

  // ---- my run
  const uint32_t ring = smem_u32(sm) + warp * SM::kRing, scale_ring = smem_u32(sm + SM::kScales) + warp * 48;
  TilePos cur = next.at;                                                // what is being worked
  PageBatch ask = next;                                                 // what is being asked for (empty so far); `next` comes behind it
  ask.count = 0;
  uint32_t behind = g0;                                                 // first tile behind `ask`
  // a copy instruction of the warp brings 512 bytes, 4 rows at D = 128 (whose swizzle alternates from one instruction to the next),
  // 8 rows at D = 64
  const uint32_t lane_at = D == 128 ? (lane >> 3) * 128 + (((lane & 7) ^ (lane >> 3)) << 4) : (lane >> 2) * 64 + (((lane & 3) ^ ((lane >> 3) & 3)) << 4);
  int row = -1;                                                         // of the pool, of the lane's half tile in `ask`; -1: nothing there
  int asked = 0, row0 = -1, row1 = -1, ask_slot = 0, ask_scale = 0;     // tiles of `ask` asked for; the last one's rows
  auto ask_k = [&]() {                                                  // the next tile's pages and scales
    if (asked == ask.count) {
      const bool first = ask.count == 0;
      ask = next;
      asked = 0;
      const int page = checked_page(ask.page, a.num_pages);
      if (page < 0 && ask.page != kNoToken) atomicCAS(a.error_word, 0u, kPageError);
      row = page < 0 ? -1 : row_of(ask, page);
      if (ask.at.t == 0 && !first) {                                    // another unit begins: its q into the L1
        constexpr int kLines = kDecHeads * D * 2 / 128;
        if (lane < min(kLines, (a.G - ask.at.hg * kDecHeads) * D * 2 / 128))
          prefetch_l1(reinterpret_cast<const uint8_t*>(a.q + (static_cast<int64_t>(ask.at.b) * a.Hq + ask.at.kvh * a.G + ask.at.hg * kDecHeads) * D) + lane * 128);
      }
      behind += ask.count;
      if (behind < g1) {
        next.at.t += ask.count;
        if (next.at.t == next.at.nt) next.at.next_unit(cum, a.Hkv, a.HG);
        fetch(next, g1 - behind);
      }
    }
    row0 = __shfl_sync(0xffffffffu, row, 2 * asked);
    row1 = __shfl_sync(0xffffffffu, row, 2 * asked + 1);
    ++asked;
    if (lane < 4) {
      const int rw = lane < 2 ? row0 : row1;
      const uint32_t to = scale_ring + ask_scale + lane * 4;
      if (rw >= 0) copy_async<4>(to, (lane & 1 ? a.scale[1] : a.scale[0]) + (rw >> a.page_shift));
      else asm volatile("st.shared.f32 [%0], %1;" ::"r"(to), "f"(-1.f) : "memory");   // (a negative scale: nothing there)
    }
    ask_scale = ask_scale == 32 ? 0 : ask_scale + 16;
  };
  auto copy_tile = [&](const uint8_t* pool) {                           // K or V of the tile whose pages were asked for last
#pragma unroll
    for (int h = 0; h < 2; ++h) {
      const int rw = h ? row1 : row0;
      if (rw < 0) continue;
      const uint32_t to = ring + ask_slot + h * (kPagedHalf * D);
      const uint8_t* from = pool + static_cast<int64_t>(rw) * D + lane * 16;
#pragma unroll
      for (int x = 0; x < kPagedHalf * D / 512; ++x)
        copy_async<16>(D == 128 ? to + x / 2 * 1024 + (x & 1 ? 512 + (lane_at ^ 64) : lane_at) : to + x * 512 + lane_at, from + x * 512);
    }
    ask_slot = ask_slot == SM::kRing - SM::kSlot ? 0 : ask_slot + SM::kSlot;
  };

  uint32_t qf[D / 16][2];
  float qs0 = 0.f, qs1 = 0.f;                // what a product is multiplied by, heads 2c, 2c+1
  float m_run[2], l_run[2];                  // reference of the probabilities (log2 domain), the thread's share of their sum
  float oacc[D / 16][4];
  float vs_ref = -1.f, vs_inv = 0.f, vs_min = 0.f;   // largest V scale so far, its reciprocal, the smallest one
  bool own = false;                          // the V scales lie too far apart: the weights have a reference of their own
  float r_run[2];                            // ... this one (relative to m_run)
  int nvalid = 0, ex0 = 0, ex_cnt = 0, first_t = 0;
  const int ring_w = a.C - a.sink;
  auto attended = [&](int slot) {
    if (slot >= nvalid) return false;
    if (ex_cnt == 0 || slot < a.sink) return true;
    int d = slot - a.sink - ex0;
    if (d < 0) d += ring_w;
    return d >= ex_cnt;
  };
  int4 piece[2] = {make_int4(-1, 0, 0, 0), make_int4(-1, 0, 0, 0)};     // the units of my pieces: (number, b, kv head, group)
  const int n_run = static_cast<int>(g1 - g0);
  int slot = 0, scale_at = 0;
  const int frag_row = ((lane >> 3) & 1) * 8 + (lane & 7);
  auto next_slot = [&]() { slot = slot == SM::kRing - SM::kSlot ? 0 : slot + SM::kSlot; };
  // three tiles' K and two tiles' V
#pragma unroll 1
  for (int x = 0; x < 3; ++x) {
    if (x < n_run) { ask_k(); copy_tile(a.pool[0]); }
    copy_commit();
    if (x == 2) break;
    if (x < n_run) copy_tile(a.pool[1]);
    copy_commit();
  }
#pragma unroll 1
  for (int i = 0; i < n_run; ++i) {
    const int first_slot = cur.t * kPagedTile;
    if (i == 0 || cur.t == 0) {
      // A unit begins.  q in f16, its row scaled by a power of two to at most 2^11: b0 = dims 16 k + 4 c, +1, b1 = the next two (the
      // pieces of a row that ldmatrix hands to a thread are four neighbouring bytes, and the order of a product's terms is free).
      if (i > 0) load_q(cur);
      nvalid = valid_of(cur);
      ex_cnt = 0;
      if (a.block_tokens > 0) {
        const int2 x = left_out(a.n_tokens[cur.b], a.C, a.sink, a.block_tokens);
        ex0 = x.x; ex_cnt = x.y;
      }
      uint32_t top = 0;                     // magnitudes of finite values
#pragma unroll
      for (int k = 0; k < D / 16; ++k) {
#pragma unroll
        for (int j = 0; j < 2; ++j) {
          uint32_t w = (j ? qw[k].y : qw[k].x) & 0x7fff7fffu;
          w &= ~__vcmpgeu2(w, 0x7f807f80u);
          top = __vmaxu2(top, w);
        }
      }
      top = max(top >> 16, top & 0xffffu);
      top = max(top, __shfl_xor_sync(0xffffffffu, top, 1));
      top = max(top, __shfl_xor_sync(0xffffffffu, top, 2));
      const int e = top == 0 ? 0 : min(126, 137 - static_cast<int>(top >> 7));   // the largest value becomes 2^10 to 2^11
      const float mul = __uint_as_float(static_cast<uint32_t>(127 + e) << 23);
      const float q_mul = __uint_as_float(static_cast<uint32_t>(127 - e) << 23) * a.scale_log2;
#pragma unroll
      for (int k = 0; k < D / 16; ++k) {
        qf[k][0] = pack_f16(bf16_lo(qw[k].x) * mul, bf16_hi(qw[k].x) * mul);
        qf[k][1] = pack_f16(bf16_lo(qw[k].y) * mul, bf16_hi(qw[k].y) * mul);
      }
      qs0 = __shfl_sync(0xffffffffu, q_mul, 8 * c);
      qs1 = __shfl_sync(0xffffffffu, q_mul, 8 * c + 4);
      m_run[0] = m_run[1] = kNoScore;
      l_run[0] = l_run[1] = 0.f;
#pragma unroll
      for (int x = 0; x < D / 16; ++x) oacc[x][0] = oacc[x][1] = oacc[x][2] = oacc[x][3] = 0.f;
      own = false;
      vs_ref = -1.f;
      vs_min = 3.4e38f;
      first_t = cur.t;
    }
    copy_wait<kPagedSlots - 1>();
    __syncwarp();                           // K of the tile and its scales are there
    const float4 sc = *reinterpret_cast<const float4*>(sm + SM::kScales + warp * 48 + scale_at);   // (K, V) scale of the first half, of the second
    scale_at = scale_at == 32 ? 0 : scale_at + 16;
    const bool in0 = sc.y >= 0.f, in1 = sc.w >= 0.f;
    bool edge = first_slot + kPagedTile > nvalid || !in0 || !in1;
    if (ex_cnt > 0 && first_slot + kPagedTile > a.sink) {
      int d = max(first_slot, a.sink) - a.sink - ex0;  // the tile's first ring slot from the first one left out
      if (d < 0) d += ring_w;
      edge |= d < ex_cnt || d + kPagedTile > ring_w;
    }

    // ---- S^T[32 tokens, 8 heads] = K Q^T
    float s[2][4] = {};
    const uint32_t sk = ring + slot;
#pragma unroll
    for (int k = 0; k < D / 16; k += 2) {
#pragma unroll
      for (int x = 0; x < 2; ++x) {
        uint32_t x0, x1, x2, x3;            // rows 0-7 and 8-15 of chunk k, the same of chunk k + 1
        ldsm_x4(sk + tile_offset<D>(16 * x + frag_row, k + (lane >> 4)), x0, x1, x2, x3);
        mma16816_f16(s[x], e4m3x2_to_f16x2(x0), e4m3x2_to_f16x2(x1), e4m3x2_hi_to_f16x2(x0), e4m3x2_hi_to_f16x2(x1), qf[k][0], qf[k][1]);
        mma16816_f16(s[x], e4m3x2_to_f16x2(x2), e4m3x2_to_f16x2(x3), e4m3x2_hi_to_f16x2(x2), e4m3x2_hi_to_f16x2(x3), qf[k + 1][0], qf[k + 1][1]);
      }
    }
    next_slot();
    __syncwarp();                           // K has been read
    if (i + 2 < n_run) copy_tile(a.pool[1]);   // V of the tile whose K was asked for last
    copy_commit();

    // s[x][0, 1]: token 16 x + r, heads 2c, 2c+1; s[x][2, 3]: token 16 x + r + 8.  A score is s times its scales, which together are kept
    // finite and above zero (1e-30: what is cut there is a score below 1e-22), so that a score of zero stays zero and -inf stays -inf.
    float sc0[2], sc1[2];
#pragma unroll
    for (int x = 0; x < 2; ++x) {
      const float kk = x ? sc.z : sc.x;
      sc0[x] = fminf(fmaxf(qs0 * kk, 1e-30f), 3.4e38f);
      sc1[x] = fminf(fmaxf(qs1 * kk, 1e-30f), 3.4e38f);
    }
    if (edge) {
#pragma unroll
      for (int x = 0; x < 2; ++x) {
        const bool in = x ? in1 : in0;
        if (!in || !attended(first_slot + 16 * x + r)) s[x][0] = s[x][1] = -INFINITY;
        if (!in || !attended(first_slot + 16 * x + r + 8)) s[x][2] = s[x][3] = -INFINITY;
      }
    }
    float w[2][4];
    auto scores = [&](float sub0, float sub1) {   // less a reference
#pragma unroll
      for (int x = 0; x < 2; ++x) {
        w[x][0] = fmaf(s[x][0], sc0[x], -sub0); w[x][1] = fmaf(s[x][1], sc1[x], -sub1);
        w[x][2] = fmaf(s[x][2], sc0[x], -sub0); w[x][3] = fmaf(s[x][3], sc1[x], -sub1);
      }
    };
    float t0, t1;
    auto top = [&]() {
      t0 = fmaxf(fmaxf(w[0][0], w[0][2]), fmaxf(w[1][0], w[1][2]));
      t1 = fmaxf(fmaxf(w[0][1], w[0][3]), fmaxf(w[1][1], w[1][3]));
    };
    auto over_tokens = [&]() {
#pragma unroll
      for (int o = 4; o < 32; o <<= 1) {
        t0 = fmaxf(t0, __shfl_xor_sync(0xffffffffu, t0, o));
        t1 = fmaxf(t1, __shfl_xor_sync(0xffffffffu, t1, o));
      }
    };
    // Scores relative to a reference that was taken from them.  Where fp32 holds them in steps of 2 and more (from 2^24 on) the reference is as coarse,
    // and the largest score's weight may come out above the largest f16, hence the minimum.  The scores are rounded before the difference is
    // taken: in one step with the product, whose unrounded value may be half a step below, it could come out as 0.
    auto less = [&](float ref0, float ref1) {
#pragma unroll
      for (int x = 0; x < 2; ++x)
#pragma unroll
        for (int y = 0; y < 4; ++y) w[x][y] = min_nan(w[x][y] - (y & 1 ? ref1 : ref0), kWeightTop);
    };
    float be0 = 1.f, be1 = 1.f;               // what O is multiplied by
    const float was0 = m_run[0], was1 = m_run[1];
    bool moved = false;
    scores(m_run[0], m_run[1]);
    top();
    if (__any_sync(0xffffffffu, fmaxf(t0, t1) > kWeightTop)) {
      scores(0.f, 0.f);
      top();
      over_tokens();
      t0 = fmaxf(m_run[0], t0 - kWeightMax); t1 = fmaxf(m_run[1], t1 - kWeightMax);
      const float al0 = fast_exp2(m_run[0] - t0), al1 = fast_exp2(m_run[1] - t1);
      m_run[0] = t0; m_run[1] = t1;
      l_run[0] *= al0; l_run[1] *= al1;
      if (!own) { be0 = al0; be1 = al1; moved = true; }
      else { r_run[0] = fmaxf(r_run[0] + (was0 - t0), kNoScore); r_run[1] = fmaxf(r_run[1] + (was1 - t1), kNoScore); }
      less(t0, t1);
    }
    float pr[2][4];
#pragma unroll
    for (int x = 0; x < 2; ++x)
#pragma unroll
      for (int y = 0; y < 4; ++y) pr[x][y] = fast_exp2(w[x][y]);
    l_run[0] += (pr[0][0] + pr[0][2]) + (pr[1][0] + pr[1][2]);
    l_run[1] += (pr[0][1] + pr[0][3]) + (pr[1][1] + pr[1][3]);
    // The pages' V scales relative to the largest so far (a half that is not there has no weights).
    const float v0 = in0 ? sc.y : in1 ? sc.w : vs_ref, v1 = in1 ? sc.w : v0;
    if (!own && v0 > 0.f && (fmaxf(v0, v1) > vs_ref || fminf(v0, v1) < vs_min)) {
      const float most = fmaxf(vs_ref, fmaxf(v0, v1));
      vs_min = fminf(vs_min, fminf(v0, v1));
      own = vs_min * 64.f < most;
      if (own) {                              // O keeps the reference that it had: what moved m may weigh little, having a small scale
        const float lr = fast_log2(vs_ref);
        r_run[0] = vs_ref > 0.f ? fmaxf(was0 - m_run[0] + lr, kNoScore) : kNoScore;
        r_run[1] = vs_ref > 0.f ? fmaxf(was1 - m_run[1] + lr, kNoScore) : kNoScore;
        be0 = be1 = 1.f;
      } else if (most != vs_ref) {
        if (vs_ref > 0.f) { be0 *= vs_ref / most; be1 *= vs_ref / most; moved = true; }
        vs_inv = 1.f / most;
      }
      vs_ref = most;
    }
    if (!own) {
      const float h0 = v0 * vs_inv, h1 = v1 * vs_inv;
#pragma unroll
      for (int y = 0; y < 4; ++y) { w[0][y] = pr[0][y] * h0; w[1][y] = pr[1][y] * h1; }
    } else {
      const float lv0 = fast_log2(v0), lv1 = fast_log2(v1);
#pragma unroll
      for (int y = 0; y < 4; ++y) { w[0][y] += lv0; w[1][y] += lv1; }
      top();
      over_tokens();
      t0 = fmaxf(r_run[0], t0 - kWeightTop); t1 = fmaxf(r_run[1], t1 - kWeightTop);
      be0 *= fast_exp2(r_run[0] - t0); be1 *= fast_exp2(r_run[1] - t1);
      r_run[0] = t0; r_run[1] = t1;
      moved = true;
      less(t0, t1);
#pragma unroll
      for (int x = 0; x < 2; ++x)
#pragma unroll
        for (int y = 0; y < 4; ++y) w[x][y] = fast_exp2(w[x][y]);
    }
    if (moved) {
#pragma unroll
      for (int x = 0; x < D / 16; ++x) { oacc[x][0] *= be0; oacc[x][1] *= be1; oacc[x][2] *= be0; oacc[x][3] *= be1; }
    }
    uint32_t pb[2][2];                      // P^T as the B operand: tokens 2c, +1 of head r, then 8 + 2c, +1
#pragma unroll
    for (int x = 0; x < 2; ++x) {
      pb[x][0] = movmatrix_t(pack_f16(w[x][0], w[x][1]));
      pb[x][1] = movmatrix_t(pack_f16(w[x][2], w[x][3]));
    }

    copy_wait<kPagedSlots - 1>();
    __syncwarp();                           // V of the tile is there
    const uint32_t sv = ring + slot;
    if (edge) {   // rows that are not attended hold anything at all: a weight of zero does not silence a NaN of V, so those rows are zeroed
      if (!((lane < kPagedHalf ? in0 : in1) && attended(first_slot + lane))) {
#pragma unroll
        for (int x = 0; x < D / 16; ++x)
          asm volatile("st.shared.v4.b32 [%0], {%1, %1, %1, %1};" ::"r"(sv + lane * D + x * 16), "r"(0) : "memory");
      }
      __syncwarp();
    }
    // ---- O^T[D, 8 heads] += V^T P^T.  Transposed, a thread's 32 bits are dims 2r, 2r+1 of tokens 2c and 2c+1: the even dims are
    // the product's rows 0-7, the odd ones its rows 8-15.
#pragma unroll
    for (int x = 0; x < 2; ++x) {
#pragma unroll
      for (int k = 0; k < D / 16; k += 2) {
        uint32_t x0, x1, x2, x3;            // tokens 0-7 and 8-15 of chunk k, the same of chunk k + 1
        ldsm_x4_t(sv + tile_offset<D>(16 * x + frag_row, k + (lane >> 4)), x0, x1, x2, x3);
        x0 = __byte_perm(x0, 0, 0x3120); x1 = __byte_perm(x1, 0, 0x3120);
        x2 = __byte_perm(x2, 0, 0x3120); x3 = __byte_perm(x3, 0, 0x3120);
        mma16816_f16(oacc[k], e4m3x2_to_f16x2(x0), e4m3x2_hi_to_f16x2(x0), e4m3x2_to_f16x2(x1), e4m3x2_hi_to_f16x2(x1), pb[x][0], pb[x][1]);
        mma16816_f16(oacc[k + 1], e4m3x2_to_f16x2(x2), e4m3x2_hi_to_f16x2(x2), e4m3x2_to_f16x2(x3), e4m3x2_hi_to_f16x2(x3), pb[x][0], pb[x][1]);
      }
    }
    next_slot();
    __syncwarp();                           // V has been read
    if (i + 3 < n_run) { ask_k(); copy_tile(a.pool[0]); }
    copy_commit();
    ++cur.t;
    const bool tail = cur.t == cur.nt;
    if (tail || i + 1 == n_run) {
      // The unit, or my run, ends: the whole unit's result, or a piece (O relative to m).
#pragma unroll
      for (int o = 4; o < 32; o <<= 1) {
        l_run[0] += __shfl_xor_sync(0xffffffffu, l_run[0], o);
        l_run[1] += __shfl_xor_sync(0xffffffffu, l_run[1], o);
      }
      float g[2];
#pragma unroll
      for (int x = 0; x < 2; ++x) g[x] = own ? fast_exp2(r_run[x]) : vs_ref;
      if (first_t == 0 && tail) {
#pragma unroll
        for (int x = 0; x < 2; ++x) {
          const int gh = cur.hg * kDecHeads + 2 * c + x;
          if (gh >= a.G) continue;
          const int64_t qh = static_cast<int64_t>(cur.b) * a.Hq + cur.kvh * a.G + gh;
          const float f = l_run[x] != 0.f ? g[x] * __fdividef(1.f, l_run[x]) : 0.f;
          uint32_t* to = reinterpret_cast<uint32_t*>(a.o + qh * D) + r;
#pragma unroll
          for (int y = 0; y < D / 16; ++y) to[8 * y] = pack_bf16(oacc[y][x] * f, oacc[y][2 + x] * f);
          if (r == 0 && a.lse) a.lse[qh] = lse_of(m_run[x], l_run[x]);
        }
      } else {
        piece[tail ? 0 : 1] = make_int4(cur.b * ups + cur.kvh * a.HG + cur.hg, cur.b, cur.kvh, cur.hg);
        float* p = reinterpret_cast<float*>(tail ? sm + SM::kPieces + warp * SM::kPiece : sm + warp * SM::kRing) + (2 * c) * (D + 2);
#pragma unroll
        for (int y = 0; y < D / 16; ++y) {
          *reinterpret_cast<float2*>(p + 16 * y + 2 * r) = make_float2(oacc[y][0] * g[0], oacc[y][2] * g[0]);
          *reinterpret_cast<float2*>(p + D + 2 + 16 * y + 2 * r) = make_float2(oacc[y][1] * g[1], oacc[y][3] * g[1]);
        }
        if (r == 0) {
          *reinterpret_cast<float2*>(p + D) = make_float2(m_run[0], l_run[0]);
          *reinterpret_cast<float2*>(p + 2 * D + 2) = make_float2(m_run[1], l_run[1]);
        }
      }
      if (tail && i + 1 < n_run) cur.next_unit(cum, a.Hkv, a.HG);
    }
  }
  if (lane == 0) { meta[2 * warp] = piece[0]; meta[2 * warp + 1] = piece[1]; }
  __syncthreads();

  // ---- the pieces of my CTA's warps, unit by unit (a warp per head); what is not a whole unit becomes a record
  const int4 mine_of = lane < 2 * kDecWarps ? meta[lane] : make_int4(-1, 0, 0, 0);
  const int4 sh0 = reinterpret_cast<const int4*>(sm + SM::kShare)[0], sh1 = reinterpret_cast<const int4*>(sm + SM::kShare)[2];
  const float* heads = reinterpret_cast<const float*>(sm) + warp * (D + 2);
  auto piece_at = [&](int y) { return heads + ((y & 1) ? (y >> 1) * (SM::kRing / 4) : SM::kPieces / 4 + (y >> 1) * (SM::kPiece / 4)); };
#pragma unroll 1
  for (unsigned left = __ballot_sync(0xffffffffu, mine_of.x >= 0); left != 0;) {
    const int y0 = __ffs(left) - 1, u = __shfl_sync(0xffffffffu, mine_of.x, y0);
    const unsigned mask = __ballot_sync(0xffffffffu, mine_of.x == u);
    left &= ~mask;
    float2 ml[2 * kDecWarps];
    float m = -INFINITY, l = 0.f, acc[D / 32] = {};
#pragma unroll
    for (int y = 0; y < 2 * kDecWarps; ++y)
      if (mask >> y & 1) { ml[y] = *reinterpret_cast<const float2*>(piece_at(y) + D); m = fmaxf(m, ml[y].x); }
    const float mu = m == -INFINITY ? 0.f : m;
#pragma unroll
    for (int y = 0; y < 2 * kDecWarps; ++y) {
      if (!(mask >> y & 1)) continue;
      const float f = fast_exp2(ml[y].x - mu);
      l += f * ml[y].y;
#pragma unroll
      for (int x = 0; x < D / 32; x += 2) {
        const float2 v = *reinterpret_cast<const float2*>(piece_at(y) + lane * 2 + 32 * x);
        acc[x] += f * v.x;
        acc[x + 1] += f * v.y;
      }
    }
    if ((u == sh0.x && sh0.z > 1) || (u == sh1.x && sh1.z > 1)) {
      float* out = a.part + (static_cast<int64_t>(me) + u) * (kDecHeads * (D + 2));
#pragma unroll
      for (int x = 0; x < D / 32; x += 2) *reinterpret_cast<float2*>(out + warp * D + lane * 2 + 32 * x) = make_float2(acc[x], acc[x + 1]);
      if (lane == 0) *reinterpret_cast<float2*>(out + kDecHeads * D + 2 * warp) = make_float2(m, l);
      continue;
    }
    const int b = __shfl_sync(0xffffffffu, mine_of.y, y0), kvh = __shfl_sync(0xffffffffu, mine_of.z, y0);
    const int gh = __shfl_sync(0xffffffffu, mine_of.w, y0) * kDecHeads + warp;
    if (gh >= a.G) continue;
    const int64_t qh = static_cast<int64_t>(b) * a.Hq + kvh * a.G + gh;
    const float inv = l != 0.f ? __fdividef(1.f, l) : 0.f;
#pragma unroll
    for (int x = 0; x < D / 32; x += 2)
      *reinterpret_cast<uint32_t*>(a.o + qh * D + lane * 2 + 32 * x) = l != 0.f ? pack_bf16(acc[x] * inv, acc[x + 1] * inv) : 0u;
    if (lane == 0 && a.lse) a.lse[qh] = lse_of(m, l);
  }

  // ---- units that several CTAs share: the one that delivers the last record merges them, in order, and re-arms the counter.  The ticket
  // releases the CTA's record (its stores are ordered before by the barrier) and acquires the others'.
  __shared__ int s_last[2];
  __syncthreads();
  if (threadIdx.x < 2) {
    const int4 sh = threadIdx.x ? sh1 : sh0;
    bool last = false;
    if (sh.z > 1 && (threadIdx.x == 0 || sh1.x != sh0.x)) {
      unsigned int* count = unit_counter(a.unit_count, a.B * ups, sh.x, sh.y);
      last = ticket_add(count) + 1u == static_cast<unsigned>(sh.z);
      if (last) *count = 0u;
    }
    s_last[threadIdx.x] = last;
  }
  __syncthreads();
#pragma unroll 1
  for (int x = 0; x < 2; ++x) {
    if (!s_last[x]) continue;
    const int4 sh = x ? sh1 : sh0;
    merge_records<D>(a, sh.w, reinterpret_cast<const int4*>(sm + SM::kShare)[2 * x + 1].x, sh.x, sh.y, sh.z);
  }
}

// ---- host side -------------------------------------------------------------------------------------
static int table_columns(const lg_paged_params* p) {
  return static_cast<int>((static_cast<int64_t>(p->sink_tokens) + p->window_tokens + p->page_tokens - 1) / p->page_tokens);
}
int paged_table_stride(const lg_paged_params* p) { return p->table_stride > 0 ? p->table_stride : table_columns(p); }
int page_shift(int page_tokens) { return page_tokens == 16 ? 4 : page_tokens == 32 ? 5 : page_tokens == 64 ? 6 : 7; }

lg_status check_paged(const lg_paged_params* p) {
  if (!p) return LG_ERR_INVALID_ARG;
  if (p->B < 1 || p->Hq < 1 || p->Hkv < 1 || p->Hq % p->Hkv != 0) return LG_ERR_INVALID_ARG;
  if (p->sink_tokens < 0 || p->window_tokens < 1 || p->block_tokens < 0) return LG_ERR_INVALID_ARG;
  if (p->block_tokens > 0 && (p->window_tokens % p->block_tokens != 0 || p->sink_tokens % p->block_tokens != 0))
    return LG_ERR_INVALID_ARG;
  if (!(p->scale >= 0.f) || isinf(p->scale)) return LG_ERR_INVALID_ARG;
  if (p->page_tokens != 16 && p->page_tokens != 32 && p->page_tokens != 64 && p->page_tokens != 128) return LG_ERR_INVALID_ARG;
  if (p->num_pages < 1 || p->table_stride < 0) return LG_ERR_INVALID_ARG;
  if (p->D != 64 && p->D != 128) return LG_ERR_UNSUPPORTED;
  if (static_cast<int64_t>(p->sink_tokens) + p->window_tokens > (1ll << 30)) return LG_ERR_UNSUPPORTED;
  if (p->table_stride > 0 && p->table_stride < table_columns(p)) return LG_ERR_INVALID_ARG;
  // the decode numbers the rows of a pool in 32 bits
  if (static_cast<int64_t>(p->num_pages) * p->Hkv * p->page_tokens > 0x7fffffffll) return LG_ERR_UNSUPPORTED;
  return LG_OK;
}

// (A decode's CTA takes nearly all shared memory of an SM, and an SM changes its split of shared memory and L1 only when it is empty: with the
// same split an overlapped decode gets onto its SM while the append still runs.)
template <int D, int NU>
static lg_status launch_append_one(const AppendArgs& a, unsigned blocks, cudaStream_t stream) {
  static std::atomic<bool> done[kMaxDevices];
  auto kern = paged_append_one_kernel<D, NU>;
  int dev = -1;
  if (cudaGetDevice(&dev) != cudaSuccess) return LG_ERR_CUDA;
  if (dev >= 0 && dev < kMaxDevices && !done[dev].load(std::memory_order_acquire)) {
    if (cudaFuncSetAttribute(kern, cudaFuncAttributePreferredSharedMemoryCarveout, cudaSharedmemCarveoutMaxShared) != cudaSuccess) cudaGetLastError();
    done[dev].store(true, std::memory_order_release);
  }
  return launch_kernel(true, kern, dim3(blocks), 128, 0, stream, a) == cudaSuccess ? LG_OK : LG_ERR_CUDA;
}

static bool aligned(const void* p, uintptr_t n) { return (reinterpret_cast<uintptr_t>(p) & (n - 1)) == 0; }
static bool bad_pools(const void* k_pool, const void* v_pool, const void* k_scale, const void* v_scale) {
  return !k_pool || !v_pool || !k_scale || !v_scale || !aligned16(k_pool) || !aligned16(v_pool) || !aligned(k_scale, 4) || !aligned(v_scale, 4);
}

// The decode kernels may use the dynamic shared memory of their largest batch; said once per device.
static lg_status allow_decode_smem() {
  static std::atomic<bool> done[kMaxDevices];
  int dev = -1;
  if (cudaGetDevice(&dev) != cudaSuccess) return LG_ERR_CUDA;
  if (dev < 0 || dev >= kMaxDevices) return LG_ERR_UNSUPPORTED;
  if (done[dev].load(std::memory_order_acquire)) return LG_OK;
  if (cudaFuncSetAttribute(paged_decode_kernel<128>, cudaFuncAttributeMaxDynamicSharedMemorySize, PagedSmem<128>::bytes(kPagedMaxB)) != cudaSuccess ||
      cudaFuncSetAttribute(paged_decode_kernel<64>, cudaFuncAttributeMaxDynamicSharedMemorySize, PagedSmem<64>::bytes(kPagedMaxB)) != cudaSuccess) {
    cudaGetLastError();
    return LG_ERR_CUDA;
  }
  done[dev].store(true, std::memory_order_release);
  return LG_OK;
}

struct PagedDecodePlan { int HG, slice, n_cta; int64_t units; size_t total_bytes; };
static PagedDecodePlan plan_paged_decode(const lg_paged_params* p) {
  PagedDecodePlan w;
  w.HG = (p->Hq / p->Hkv + kDecHeads - 1) / kDecHeads;
  // sequences of one launch: their prefix sums lie in shared memory, and the kernel counts their tiles in 31 bits
  const int64_t C = static_cast<int64_t>(p->sink_tokens) + p->window_tokens, seq_units = static_cast<int64_t>(p->Hkv) * w.HG;
  const int64_t seq_tiles = seq_units * ((C + kPagedTile - 1) / kPagedTile);
  int64_t most_b = 0x7fffffffll / (seq_tiles + kDecMaxCtas);
  if (most_b > kPagedMaxB) most_b = kPagedMaxB;
  w.slice = static_cast<int>(p->B < most_b ? p->B : most_b);      // (0: one sequence is too long)
  w.units = w.slice * seq_units;
  w.total_bytes = kDecRecordOffset + align_up((static_cast<size_t>(kDecMaxCtas) + w.units) * kDecHeads * (p->D + 2) * sizeof(float), 256);
  // as many CTAs as fit an SM (D = 64: two), each with at least a tile for every second of its warps
  const int64_t tiles = w.slice * seq_tiles;
  int64_t n = (tiles + kDecWarps / 2 - 1) / (kDecWarps / 2);
  const int64_t most = (p->D == 64 ? 2 : 1) * kSms;
  if (n > most) n = most;
  w.n_cta = static_cast<int>(n < 1 ? 1 : n);
  return w;
}

}  // namespace lg

using namespace lg;

extern "C" {

lg_status lg_paged_table_extend(const lg_paged_params* p, const int64_t* n_tokens_before, const int32_t* n_new, int32_t T_new,
                                const int32_t* free_pages, int32_t n_free, const int32_t* free_start, int32_t* block_table,
                                int32_t* free_next, void* stream) {
  LG_RANGE("lg_paged_table_extend");
  lg_status s = check_paged(p);
  if (s != LG_OK) return s;
  if (T_new < 0 || n_free < 0) return LG_ERR_INVALID_ARG;
  if (!n_tokens_before || !free_start || !block_table || !free_next || (n_free > 0 && !free_pages)) return LG_ERR_INVALID_ARG;
  if (!aligned(n_tokens_before, 8) || !aligned(n_new, 4) || !aligned(free_pages, 4) || !aligned(free_start, 4) || !aligned(block_table, 4) ||
      !aligned(free_next, 4) || free_start == free_next)
    return LG_ERR_INVALID_ARG;
  if ((s = check_arch()) != LG_OK) return s;
  ExtendArgs a;
  a.n_before = n_tokens_before; a.n_new = n_new; a.free_pages = free_pages; a.free_start = free_start;
  a.table = block_table; a.free_next = free_next;
  a.B = p->B; a.T_new = T_new; a.n_free = n_free;
  a.sink = p->sink_tokens; a.window = p->window_tokens; a.page_shift = page_shift(p->page_tokens); a.stride = paged_table_stride(p);
  a.rows = (p->B + 2 * kSms - 1) / (2 * kSms);
  if (a.rows > kExtendMaxRows) a.rows = kExtendMaxRows;
  int64_t most = static_cast<int64_t>(T_new) / p->page_tokens + 1;       // new pages of a sequence
  if (most > table_columns(p)) most = table_columns(p);
  const int64_t cols = (most + kExtendCols - 1) / kExtendCols;
  if (cols > 65535) return LG_ERR_UNSUPPORTED;
  return launch_kernel(true, table_extend_kernel, dim3((p->B + a.rows - 1) / a.rows, static_cast<unsigned>(cols)), kExtendThreads, 0,
                       static_cast<cudaStream_t>(stream), a) == cudaSuccess ? LG_OK : LG_ERR_CUDA;
}

lg_status lg_paged_slot_map(const lg_paged_params* p, const int64_t* n_tokens, const int64_t* first, const int32_t* count, int32_t T,
                            const int32_t* block_table, int64_t* slot_map, void* stream) {
  LG_RANGE("lg_paged_slot_map");
  lg_status s = check_paged(p);
  if (s != LG_OK) return s;
  if (T < 0) return LG_ERR_INVALID_ARG;
  if (T == 0) return LG_OK;
  if (!n_tokens || !first || !block_table || !slot_map) return LG_ERR_INVALID_ARG;
  if (!aligned(n_tokens, 8) || !aligned(first, 8) || !aligned(count, 4) || !aligned(block_table, 4) || !aligned(slot_map, 8))
    return LG_ERR_INVALID_ARG;
  const int64_t blocks = (static_cast<int64_t>(T) + kSlotMapThreads * kSlotMapPer - 1) / (kSlotMapThreads * kSlotMapPer);
  if (p->B > 65535 || T > (1 << 30)) return LG_ERR_UNSUPPORTED;
  if ((s = check_arch()) != LG_OK) return s;
  SlotMapArgs a;
  a.n_tokens = n_tokens; a.first = first; a.count = count; a.table = block_table; a.slot_map = slot_map;
  a.B = p->B; a.T = T; a.sink = p->sink_tokens; a.window = p->window_tokens;
  a.page_shift = page_shift(p->page_tokens); a.num_pages = p->num_pages; a.stride = paged_table_stride(p);
  return launch_kernel(true, slot_map_kernel, dim3(static_cast<unsigned>(blocks), p->B), kSlotMapThreads, 0, static_cast<cudaStream_t>(stream), a) ==
                 cudaSuccess ? LG_OK : LG_ERR_CUDA;
}

lg_status lg_paged_append(const lg_paged_params* p, void* k_pool, void* v_pool, float* k_scale, float* v_scale, const int32_t* block_table,
                          const void* k_new, const void* v_new, const int64_t* new_strides, int32_t T_new, const int64_t* n_tokens_before,
                          const int32_t* n_new, void* stream) {
  LG_RANGE("lg_paged_append");
  lg_status s = check_paged(p);
  if (s != LG_OK) return s;
  if (T_new < 0) return LG_ERR_INVALID_ARG;
  if (T_new == 0) return LG_OK;
  if (bad_pools(k_pool, v_pool, k_scale, v_scale) || !block_table || !k_new || !v_new || !n_tokens_before) return LG_ERR_INVALID_ARG;
  if (!aligned(block_table, 4) || !aligned16(k_new) || !aligned16(v_new) || !aligned(n_tokens_before, 8) || !aligned(n_new, 4))
    return LG_ERR_INVALID_ARG;
  if (k_pool == v_pool || k_scale == v_scale) return LG_ERR_INVALID_ARG;   // K and V are written side by side
  AppendArgs a;
  a.stride_t = p->D;
  a.stride_h = static_cast<int64_t>(T_new) * p->D;
  a.stride_b = a.stride_h * p->Hkv;
  if (new_strides) {
    for (int i = 0; i < 3; ++i)
      if (new_strides[i] <= 0 || new_strides[i] % 8 != 0) return LG_ERR_INVALID_ARG;
    a.stride_b = new_strides[0]; a.stride_h = new_strides[1]; a.stride_t = new_strides[2];
    if (a.stride_t < p->D) return LG_ERR_INVALID_ARG;
  }
  a.pool[0] = static_cast<uint8_t*>(k_pool); a.pool[1] = static_cast<uint8_t*>(v_pool);
  a.scale[0] = k_scale; a.scale[1] = v_scale;
  a.rows[0] = static_cast<const __nv_bfloat16*>(k_new); a.rows[1] = static_cast<const __nv_bfloat16*>(v_new);
  a.table = block_table; a.n_before = n_tokens_before; a.n_new = n_new;
  a.B = p->B; a.Hkv = p->Hkv; a.T = T_new; a.sink = p->sink_tokens; a.window = p->window_tokens;
  a.page_shift = page_shift(p->page_tokens); a.num_pages = p->num_pages; a.stride = paged_table_stride(p);
  a.max_touched = max_touched_pages(T_new, p->sink_tokens, p->window_tokens, p->page_tokens);
  // one token: a CTA per (K or V, kv head).  Several: as many of them one after the other as leave eight CTAs an SM (a CTA's counts and table
  // entry are two round trips that the next pair's rows do not wait for)
  const int64_t pages = static_cast<int64_t>(p->B) * a.max_touched, pairs = 2ll * p->Hkv;
  int64_t units = T_new == 1 ? 1 : pages * pairs / (8 * kSms);
  units = units < 1 ? 1 : units > pairs ? pairs : units;
  a.units = static_cast<int>(units);
  a.groups = static_cast<int>((pairs + units - 1) / units);
  const int64_t blocks = pages * a.groups;
  if (blocks > 0x7fffffff) return LG_ERR_UNSUPPORTED;
  if ((s = check_arch()) != LG_OK) return s;
  const unsigned grid = static_cast<unsigned>(blocks);
  const int elements = p->page_tokens * p->D;
  cudaStream_t st = static_cast<cudaStream_t>(stream);
#define LG_APPEND_CASE(DD, PP, TT)                                                                \
  if (p->D == DD && elements == DD * PP) {                                                        \
    if (T_new == 1) return launch_append_one<DD, DD * PP / 1024>(a, grid, st);                    \
    return launch_kernel(true, paged_append_kernel<DD, DD * PP / 8 / TT, TT>, dim3(grid), TT, 0, st, a) == cudaSuccess ? LG_OK : LG_ERR_CUDA; \
  }
  LG_APPEND_CASE(128, 16, 128)
  LG_APPEND_CASE(128, 32, 128)
  LG_APPEND_CASE(128, 64, 256)
  LG_APPEND_CASE(128, 128, 512)
  LG_APPEND_CASE(64, 16, 128)
  LG_APPEND_CASE(64, 32, 128)
  LG_APPEND_CASE(64, 64, 128)
  LG_APPEND_CASE(64, 128, 256)
#undef LG_APPEND_CASE
  return LG_ERR_UNSUPPORTED;
}

lg_status lg_paged_gather(const lg_paged_params* p, const void* k_pool, const void* v_pool, const float* k_scale, const float* v_scale,
                          const int64_t* slot_map, int32_t T, void* k_out, void* v_out, void* stream) {
  LG_RANGE("lg_paged_gather");
  lg_status s = check_paged(p);
  if (s != LG_OK) return s;
  if (T < 0) return LG_ERR_INVALID_ARG;
  if (T == 0) return LG_OK;
  if (bad_pools(k_pool, v_pool, k_scale, v_scale) || !slot_map || !k_out || !v_out) return LG_ERR_INVALID_ARG;
  if (!aligned(slot_map, 8) || !aligned16(k_out) || !aligned16(v_out)) return LG_ERR_INVALID_ARG;
  const int rows = kGatherThreads / (p->D / 16);   // tokens of a block
  if (T > (1 << 30) || p->Hkv > 65535 || p->B > 65535) return LG_ERR_UNSUPPORTED;
  if ((s = check_arch()) != LG_OK) return s;
  GatherArgs a;
  a.pool[0] = static_cast<const uint8_t*>(k_pool); a.pool[1] = static_cast<const uint8_t*>(v_pool);
  a.scale[0] = k_scale; a.scale[1] = v_scale; a.slot_map = slot_map;
  a.out[0] = static_cast<uint4*>(k_out); a.out[1] = static_cast<uint4*>(v_out);
  a.Hkv = p->Hkv; a.T = T; a.page_shift = page_shift(p->page_tokens); a.num_pages = p->num_pages;
  return launch_kernel(true, p->D == 128 ? paged_gather_kernel<128> : paged_gather_kernel<64>, dim3((T + rows - 1) / rows, p->Hkv, p->B), kGatherThreads, 0,
                       static_cast<cudaStream_t>(stream), a) == cudaSuccess ? LG_OK : LG_ERR_CUDA;
}

size_t lg_paged_decode_workspace_bytes(const lg_paged_params* p) {
  if (check_paged(p) != LG_OK) return 0;
  const PagedDecodePlan w = plan_paged_decode(p);
  return w.slice > 0 ? w.total_bytes : 0;
}

lg_status lg_paged_decode(const lg_paged_params* p, const void* q, const void* k_pool, const void* v_pool, const float* k_scale,
                          const float* v_scale, const int32_t* block_table, const int64_t* n_tokens, void* o, float* lse, void* workspace,
                          size_t workspace_bytes, void* stream) {
  LG_RANGE("lg_paged_decode");
  lg_status s = check_paged(p);
  if (s != LG_OK) return s;
  if (bad_pools(k_pool, v_pool, k_scale, v_scale) || !q || !block_table || !n_tokens || !o || !workspace) return LG_ERR_INVALID_ARG;
  if (!aligned16(q) || !aligned16(o) || !aligned(block_table, 4) || !aligned(n_tokens, 8) || !aligned(lse, 4) || !aligned(workspace, 256))
    return LG_ERR_INVALID_ARG;
  const PagedDecodePlan w = plan_paged_decode(p);
  if (w.slice < 1) return LG_ERR_UNSUPPORTED;
  if (workspace_bytes < w.total_bytes) return LG_ERR_WORKSPACE;
  if ((s = check_arch()) != LG_OK) return s;
  PagedDecodeArgs a;
  a.scale[0] = k_scale; a.scale[1] = v_scale;
  a.pool[0] = static_cast<const uint8_t*>(k_pool); a.pool[1] = static_cast<const uint8_t*>(v_pool);
  uint8_t* ws = static_cast<uint8_t*>(workspace);
  a.error_word = reinterpret_cast<unsigned int*>(ws);
  a.unit_count = reinterpret_cast<unsigned int*>(ws + kDecCountOffset);
  a.part = reinterpret_cast<float*>(ws + kDecRecordOffset);
  a.Hq = p->Hq; a.Hkv = p->Hkv; a.G = p->Hq / p->Hkv; a.HG = w.HG;
  a.C = p->sink_tokens + p->window_tokens;
  a.sink = p->sink_tokens; a.block_tokens = p->block_tokens;
  a.page_shift = page_shift(p->page_tokens); a.num_pages = p->num_pages; a.stride = paged_table_stride(p);
  a.scale_log2 = (p->scale > 0.f ? p->scale : 1.0f / sqrtf(static_cast<float>(p->D))) * 1.4426950408889634f;
  if ((s = allow_decode_smem()) != LG_OK) return s;
  for (int b = 0; b < p->B; b += w.slice) {   // (larger batches: launch by launch, over the same records)
    a.B = p->B - b < w.slice ? p->B - b : w.slice;
    a.q = static_cast<const __nv_bfloat16*>(q) + static_cast<int64_t>(b) * p->Hq * p->D;
    a.o = static_cast<__nv_bfloat16*>(o) + static_cast<int64_t>(b) * p->Hq * p->D;
    a.lse = lse ? lse + static_cast<int64_t>(b) * p->Hq : nullptr;
    a.table = block_table + static_cast<int64_t>(b) * a.stride;
    a.n_tokens = n_tokens + b;
    const cudaError_t e = p->D == 128 ? launch_kernel(true, paged_decode_kernel<128>, dim3(w.n_cta), kDecThreads, PagedSmem<128>::bytes(a.B),
                                                      static_cast<cudaStream_t>(stream), a)
                                      : launch_kernel(true, paged_decode_kernel<64>, dim3(w.n_cta), kDecThreads, PagedSmem<64>::bytes(a.B),
                                                      static_cast<cudaStream_t>(stream), a);
    if (e != cudaSuccess) return LG_ERR_CUDA;
  }
  return LG_OK;
}

}  // extern "C"
