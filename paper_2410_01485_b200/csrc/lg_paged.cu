// The rolling-buffer cache of the paper's Section 3.2 in 8 bits and in pages: block tables and slot maps built from
// request lengths, an append that quantises, single-token attention over the pages, and a read-back in bf16.
//
// Numbers.  A page holds page_tokens slots of one kv head as e4m3 codes and one fp32 scale, the power of two that
// page_exponent() gives.  A power of two and a floating code: when a page's largest value changes, its other tokens are
// rescaled by exponents alone, which is exact but for codes below the normal range (values under 2^-14 of the largest),
// where scales of amax / 448 would round every token of the page anew with every append.  e4m3 keeps 4 significant bits
// wherever a value lies in its 15 octaves, so nothing is lost by a scale up to twice as large.
#include <cuda.h>
#include <cuda_fp16.h>
#include <math.h>

#include "lg_common.cuh"
#include "lg_decode.cuh"
#include "lg_host.h"
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
// Round to nearest even; beyond 448 (infinities) the largest code, NaN stays NaN.
__device__ __forceinline__ uint32_t f32x2_to_e4m3x2(float lo, float hi) {
  uint16_t r;
  asm("cvt.rn.satfinite.e4m3x2.f32 %0, %1, %2;" : "=h"(r) : "f"(hi), "f"(lo));
  return r;
}
__device__ __forceinline__ float2 f16x2_to_f32x2(uint32_t h) {
  return __half22float2(*reinterpret_cast<const __half2*>(&h));
}
__device__ __forceinline__ float bf16_lo(uint32_t w) { return __uint_as_float(w << 16); }
__device__ __forceinline__ float bf16_hi(uint32_t w) { return __uint_as_float(w & 0xffff0000u); }

// The page of a table entry, or -1 where the entry names no page of the pool.
__device__ __forceinline__ int checked_page(int page, int num_pages) { return page >= 0 && page < num_pages ? page : -1; }

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
  int B, T_new, n_free, sink, window, page_tokens, stride, rows;
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
    had = pages_of(n, a.sink, a.window, a.page_tokens);
    return n < 0 ? 0 : pages_of(n + new_tokens(a.n_new, b, a.T_new), a.sink, a.window, a.page_tokens);
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
constexpr int kSlotMapThreads = 256;

__global__ void __launch_bounds__(kSlotMapThreads) slot_map_kernel(const SlotMapArgs a) {
  pdl_trigger();
  const int64_t i = static_cast<int64_t>(blockIdx.x) * kSlotMapThreads + threadIdx.x;
  if (i >= static_cast<int64_t>(a.B) * a.T) return;
  const int b = static_cast<int>(i / a.T), t = static_cast<int>(i - static_cast<int64_t>(b) * a.T);
  pdl_wait();
  const int64_t n = a.n_tokens[b], pos = a.first[b] + t;
  int64_t out = -1;
  if (t < new_tokens(a.count, b, a.T) && pos >= 0 && pos < n) {
    const int slot = slot_of(pos, a.sink, a.window);
    if (held_position(slot, n, a.sink, a.window) == pos) {
      const int page = checked_page(a.table[static_cast<int64_t>(b) * a.stride + (slot >> a.page_shift)], a.num_pages);
      if (page >= 0) out = (static_cast<int64_t>(page) << a.page_shift) + (slot & ((1 << a.page_shift) - 1));
    }
  }
  a.slot_map[i] = out;
}

// ---- append -----------------------------------------------------------------------------------
// A CTA owns one (sequence, touched page, kv head) of K or of V: it holds the page's new rows (bf16) and its kept old ones
// (codes) in registers, finds the largest magnitude, and writes codes and scale.  Old rows are written only where the
// scale changed, and a page whose every live token is new is not read.  HBM-bound for prompts; one round trip for the
// counts and the table entry, one for the rows and one barrier for a single token.
struct AppendArgs {
  uint8_t* pool[2];          // K, V: [num_pages, Hkv, P, D]
  float* scale[2];           // [num_pages, Hkv]
  const __nv_bfloat16* rows[2];
  const int32_t* table;
  const int64_t* n_before;
  const int32_t* n_new;      // or null
  int64_t stride_b, stride_h, stride_t;
  int B, Hkv, T, sink, window, page_tokens, num_pages, stride, max_touched;
};
constexpr int kAppendThreads = 128;

template <int D, int NU>     // NU units of 8 elements a thread: page_tokens = NU * 8 * kAppendThreads / D
__global__ void __launch_bounds__(kAppendThreads) paged_append_kernel(const AppendArgs a) {
  pdl_trigger();
  constexpr int kPerRow = D / 8, kRows = NU * kAppendThreads / kPerRow;
  static_assert(kRows <= kAppendThreads, "a thread per slot of the page");
  __shared__ int src[kRows];                 // new token of each slot; -1: kept old one; -2: nothing
  __shared__ uint32_t warp_max[kAppendThreads / 32];
  const int tid = threadIdx.x;
  uint32_t x = blockIdx.x;
  const int kv = x & 1; x >>= 1;
  const int h = x % a.Hkv; x /= a.Hkv;
  const int i = x % a.max_touched, b = x / a.max_touched;
  pdl_wait();
  const int64_t n0 = a.n_before[b];
  if (n0 < 0) return;                        // a negative count addresses nothing: the sequence is skipped
  const int64_t n1 = n0 + new_tokens(a.n_new, b, a.T);
  const TouchedPages t = touched_pages(n0, n1, a.sink, a.window, a.page_tokens);
  if (i >= t.total()) return;
  const int lp = t.page(i);
  const int page = checked_page(a.table[static_cast<int64_t>(b) * a.stride + lp], a.num_pages);
  if (page < 0) return;
  bool old = false;
  if (tid < kRows) {
    const int64_t pos = held_position(static_cast<int64_t>(lp) * kRows + tid, n1, a.sink, a.window);
    src[tid] = pos < 0 ? -2 : pos < n0 ? -1 : static_cast<int>(pos - n0);
    old = pos >= 0 && pos < n0;
  }
  const bool any_old = __syncthreads_or(old) != 0;
  const int64_t unit = static_cast<int64_t>(page) * a.Hkv + h;
  uint8_t* codes = a.pool[kv] + unit * (kRows * D);
  const float was = any_old ? a.scale[kv][unit] : 0.f;
  const __nv_bfloat16* rows = a.rows[kv] + b * a.stride_b + h * a.stride_h;
  uint4 v[NU];                               // 8 new values, or 8 old codes in (x, y)
  uint32_t top = 0, top_code = 0;            // largest finite magnitude: bf16 bits, code
#pragma unroll
  for (int u = 0; u < NU; ++u) {
    const int e = u * kAppendThreads + tid, s = src[e / kPerRow];
    v[u] = make_uint4(0, 0, 0, 0);
    if (s >= 0) v[u] = *reinterpret_cast<const uint4*>(rows + s * a.stride_t + e % kPerRow * 8);
    else if (s == -1) { const uint2 c = *reinterpret_cast<const uint2*>(codes + e * 8); v[u].x = c.x; v[u].y = c.y; }
  }
#pragma unroll
  for (int u = 0; u < NU; ++u) {
    const int s = src[(u * kAppendThreads + tid) / kPerRow];
    if (s >= 0) {
      const uint32_t w[4] = {v[u].x, v[u].y, v[u].z, v[u].w};
#pragma unroll
      for (int j = 0; j < 4; ++j) {
        const uint32_t lo = w[j] & 0x7fffu, hi = (w[j] >> 16) & 0x7fffu;   // infinities and NaN do not count
        if (lo < 0x7f80u) top = max(top, lo);
        if (hi < 0x7f80u) top = max(top, hi);
      }
    } else if (s == -1) {
#pragma unroll
      for (int j = 0; j < 2; ++j) {
        uint32_t c = (j ? v[u].y : v[u].x) & 0x7f7f7f7fu;
        c &= ~__vcmpeq4(c, 0x7f7f7f7fu);                                   // NaN codes do not count
        const uint32_t m = __vmaxu4(c, c >> 16);
        top_code = max(top_code, max(m & 0xffu, (m >> 8) & 0xffu));
      }
    }
  }
  const float old_top = f16x2_to_f32x2(e4m3x2_to_f16x2(top_code)).x * was;
  uint32_t bits = max(top << 16, __float_as_uint(old_top));                // magnitudes: order of the bits
  bits = __reduce_max_sync(0xffffffffu, bits);
  if ((tid & 31) == 0) warp_max[tid >> 5] = bits;
  __syncthreads();
  bits = 0;
#pragma unroll
  for (int w = 0; w < kAppendThreads / 32; ++w) bits = max(bits, warp_max[w]);
  const int e2 = page_exponent(bits);
  const float now = __uint_as_float(static_cast<uint32_t>(e2 + 127) << 23), inv = __uint_as_float(static_cast<uint32_t>(127 - e2) << 23);
  const bool rescale = any_old && was != now;
#pragma unroll
  for (int u = 0; u < NU; ++u) {
    const int e = u * kAppendThreads + tid, s = src[e / kPerRow];
    uint2 out;
    if (s >= 0) {
      out.x = f32x2_to_e4m3x2(bf16_lo(v[u].x) * inv, bf16_hi(v[u].x) * inv) | f32x2_to_e4m3x2(bf16_lo(v[u].y) * inv, bf16_hi(v[u].y) * inv) << 16;
      out.y = f32x2_to_e4m3x2(bf16_lo(v[u].z) * inv, bf16_hi(v[u].z) * inv) | f32x2_to_e4m3x2(bf16_lo(v[u].w) * inv, bf16_hi(v[u].w) * inv) << 16;
      *reinterpret_cast<uint2*>(codes + e * 8) = out;
    } else if (s == -1 && rescale) {
      const float2 p = f16x2_to_f32x2(e4m3x2_to_f16x2(v[u].x)), q = f16x2_to_f32x2(e4m3x2_hi_to_f16x2(v[u].x));
      const float2 r = f16x2_to_f32x2(e4m3x2_to_f16x2(v[u].y)), w = f16x2_to_f32x2(e4m3x2_hi_to_f16x2(v[u].y));
      // (two products: was * inv may leave the range of fp32 where every code is zero)
      out.x = f32x2_to_e4m3x2(p.x * was * inv, p.y * was * inv) | f32x2_to_e4m3x2(q.x * was * inv, q.y * was * inv) << 16;
      out.y = f32x2_to_e4m3x2(r.x * was * inv, r.y * was * inv) | f32x2_to_e4m3x2(w.x * was * inv, w.y * was * inv) << 16;
      *reinterpret_cast<uint2*>(codes + e * 8) = out;
    }
  }
  if (tid == 0) a.scale[kv][unit] = now;
}

// ---- rows of the cache in bf16 ---------------------------------------------------------------
// 16 codes times the page's scale (exact for a power-of-two scale: 4 significant bits) as two 16-byte pieces.
__device__ __forceinline__ void dequant16(uint4 c, float s, uint4& lo, uint4& hi) {
  auto two = [s](uint32_t h) { const float2 f = f16x2_to_f32x2(h); return pack_bf16(f.x * s, f.y * s); };
  lo = make_uint4(two(e4m3x2_to_f16x2(c.x)), two(e4m3x2_hi_to_f16x2(c.x)), two(e4m3x2_to_f16x2(c.y)), two(e4m3x2_hi_to_f16x2(c.y)));
  hi = make_uint4(two(e4m3x2_to_f16x2(c.z)), two(e4m3x2_hi_to_f16x2(c.z)), two(e4m3x2_to_f16x2(c.w)), two(e4m3x2_hi_to_f16x2(c.w)));
}

struct GatherArgs {
  const uint8_t* pool[2];
  const float* scale[2];
  const int64_t* slot_map;   // [B, T]
  uint4* out[2];             // [B, Hkv, T, D]
  int Hkv, T, D, page_shift, num_pages;
};
constexpr int kGatherThreads = 256;

__global__ void __launch_bounds__(kGatherThreads) paged_gather_kernel(const GatherArgs a) {
  pdl_trigger();
  const int per_row = a.D / 16;
  const int64_t i = static_cast<int64_t>(blockIdx.x) * kGatherThreads + threadIdx.x;
  const int64_t t = i / per_row;
  const int c = static_cast<int>(i - t * per_row), h = blockIdx.y, b = blockIdx.z;
  if (t >= a.T) return;
  pdl_wait();
  const int64_t slot = a.slot_map[static_cast<int64_t>(b) * a.T + t];
  const int64_t page = slot >> a.page_shift;
  const bool on = slot >= 0 && page < a.num_pages;
  const int64_t unit = on ? page * a.Hkv + h : 0;
  const int64_t at = ((unit << a.page_shift) + (slot & ((1 << a.page_shift) - 1))) * per_row + c;
  const int64_t to = ((static_cast<int64_t>(b) * a.Hkv + h) * a.T + t) * per_row + c;
#pragma unroll
  for (int x = 0; x < 2; ++x) {
    uint4 lo = make_uint4(0, 0, 0, 0), hi = lo;
    if (on) dequant16(*(reinterpret_cast<const uint4*>(a.pool[x]) + at), a.scale[x][unit], lo, hi);
    a.out[x][to * 2] = lo;
    a.out[x][to * 2 + 1] = hi;
  }
}

// What a chunk attends to, as one sequence in time order: the `kept` tokens that the cache holds after n tokens (the sink, then
// the ring from its oldest token on, ring0 of the sequence), then the chunk's own rows.  Rows whose page is absent are zeros and the status
// word says so: the attention kernel behind then does nothing.
__global__ void __launch_bounds__(kGatherThreads) paged_linearise_kernel(const PagedLinearise a) {
  pdl_trigger();
  const int per_row = a.D / 16, L = a.kept + a.T;
  const int64_t i = static_cast<int64_t>(blockIdx.x) * kGatherThreads + threadIdx.x;
  const int64_t v = i / per_row;
  const int c = static_cast<int>(i - v * per_row), h = blockIdx.y, b = blockIdx.z;
  if (v >= L) return;
  pdl_wait();
  const int64_t bh = static_cast<int64_t>(b) * a.Hkv + h;
  uint4 lo[2], hi[2];
  if (v < a.kept) {
    int slot = static_cast<int>(v);
    if (v >= a.sink) {
      slot = a.ring0[b] + static_cast<int>(v) - a.sink;
      if (slot >= a.window) slot -= a.window;
      slot += a.sink;
    }
    const int page = checked_page(a.table[static_cast<int64_t>(b) * a.stride + (slot >> a.page_shift)], a.num_pages);
    const int64_t unit = (page < 0 ? 0 : page) * static_cast<int64_t>(a.Hkv) + h;
    const int64_t at = ((unit << a.page_shift) + (slot & ((1 << a.page_shift) - 1))) * per_row + c;
    if (page < 0) atomicCAS(a.error_word, 0u, kPageError);
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

lg_status launch_paged_linearise(const PagedLinearise& a, int B, cudaStream_t stream) {
  const int64_t blocks = (static_cast<int64_t>(a.kept + a.T) * (a.D / 16) + kGatherThreads - 1) / kGatherThreads;
  if (blocks > 0x7fffffff || a.Hkv > 65535 || B > kLineariseSeqs) return LG_ERR_UNSUPPORTED;
  return launch_kernel(true, paged_linearise_kernel, dim3(static_cast<unsigned>(blocks), a.Hkv, B), kGatherThreads, 0, stream, a) == cudaSuccess
             ? LG_OK : LG_ERR_CUDA;
}

// ---- single-token attention ---------------------------------------------------------------------
// The 32-token tiles of all (sequence, kv head, group of <= 8 query heads) units form one sequence that is cut into equal
// slices, one per CTA; each of a CTA's warps streams a run of tiles through a ring of its own, filled by TMA from the
// pages (128-byte or, at D = 64, 64-byte swizzle, so that the fragments are read without bank conflicts).  Scores are
// S^T = K Q^T and outputs O^T = V^T P^T on mma.sync m16n8k16 with f16 operands: an e4m3 code is an f16 number, so K and V
// enter without rounding, and q (8 significant bits) does not lose any either once its row is scaled by a power of two.
// The tensor-core time is far below the HBM's (16 products of 16 x 8 x 16 and 64 conversions per 4 KB of cache, about 80 of
// 178 cycles of an SM at full bandwidth), a contraction 8 heads wide is far below a tcgen05 tile.
// A page's scale multiplies its scores; that of V goes into the weights: w_j = 2^(s_j + log2 vs - r) with a running
// reference r of its own, so that w fits f16 (11 bits) whatever the scales of the pages are, while the row sum is kept in fp32
// relative to the running maximum m of the scores alone.
constexpr int kPagedTile = 32;
constexpr int kPagedMaxB = 4096;        // sequences of one launch (their prefix sums lie in shared memory)
constexpr int kPagedMaxCtas = 320;

struct PagedDecodeArgs {
  const __nv_bfloat16* q;        // [B, Hq, D]
  const float* k_scale;          // [num_pages, Hkv]
  const float* v_scale;
  const int32_t* table;          // [B, stride]
  const int64_t* n_tokens;       // [B]
  float* part;
  __nv_bfloat16* o;
  float* lse;
  unsigned int* unit_count;
  unsigned int* error_word;
  int B, Hq, Hkv, G, HG, C;
  int sink, block_tokens;
  int page_shift, num_pages, stride, box_rows;
  float scale_log2;
};

__device__ __forceinline__ void tma_load_2d(uint32_t smem_dst, const void* tmap, uint32_t bar, int c0, int c1) {
  asm volatile(
      "cp.async.bulk.tensor.2d.shared::cluster.global.mbarrier::complete_tx::bytes [%0], [%1, {%3, %4}], [%2];" ::"r"(smem_dst),
      "l"(reinterpret_cast<uint64_t>(tmap)), "r"(bar), "r"(c0), "r"(c1)
      : "memory");
}
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

template <int D>
struct PagedSmem {
  static constexpr int kTileBytes = kPagedTile * D;                     // K (or V) of a tile
  static constexpr int kPipe = kDecWarps * kDecStages * 2 * kTileBytes;
  static constexpr int kBars = kPipe;                                   // a barrier per warp and stage
  static constexpr int kScales = kBars + kDecWarps * kDecStages * 8;    // (k scale, v scale) of a tile's two halves
  static constexpr int kCum = kScales + kDecWarps * kDecStages * 16;
  static_assert(kDecWarps * kDecHeads * (D + 2) * 4 <= kPipe, "the merge lies over the rings");
  static int bytes(int B) { return 1024 /* alignment */ + kCum + (B + 1) * 4; }
};

// byte offset of 16-byte chunk c of row r in a tile as TMA lays it out
template <int D>
__device__ __forceinline__ uint32_t tile_offset(int r, int c) {
  return r * D + ((c ^ (D == 128 ? r & 7 : (r >> 1) & 3)) << 4);
}

// One segment: the CTA's warps stream tiles [tb, te) each of unit (b, kvh, hg) and leave their partial results in shared
// memory; `it` counts the warp's tiles over all segments.
template <int D>
__device__ __forceinline__ bool paged_run_segment(const PagedDecodeArgs& a, const CUtensorMap& tk, const CUtensorMap& tv, uint8_t* sm, int b,
                                                  int kvh, int hg, int nvalid, int tb, int te, uint32_t& it) {
  using SM = PagedSmem<D>;
  const int warp = threadIdx.x >> 5, lane = threadIdx.x & 31;
  const int r = lane >> 2, c = lane & 3;
  const uint32_t ring = smem_u32(sm) + warp * (kDecStages * 2 * SM::kTileBytes);
  uint64_t* bars = reinterpret_cast<uint64_t*>(sm + SM::kBars) + warp * kDecStages;
  float2* scales = reinterpret_cast<float2*>(sm + SM::kScales) + warp * kDecStages * 2;
  bool ok = true;

  // block-aligned window: the ring's oldest tokens that it leaves out (ex_cnt slots from ring offset ex0 on, cyclic)
  int ex0 = 0, ex_cnt = 0;
  const int ring_w = a.C - a.sink;
  if (a.block_tokens > 0) {
    const int64_t n = a.n_tokens[b];
    if (n > a.C) {
      const int64_t first_held = n - ring_w;
      const int64_t first_kept = ((n - 1) / a.block_tokens - ring_w / a.block_tokens + 1) * a.block_tokens;
      if (first_kept > first_held) {
        ex_cnt = static_cast<int>(first_kept - first_held);
        ex0 = static_cast<int>((first_held - a.sink) % ring_w);
      }
    }
  }
  auto attended = [&](int slot) {
    if (slot >= nvalid) return false;
    if (ex_cnt == 0 || slot < a.sink) return true;
    int d = slot - a.sink - ex0;
    if (d < 0) d += ring_w;
    return d >= ex_cnt;
  };

  // q in f16, its row scaled by a power of two to at most 2^11: b0 = dims 16 k + 4 c, +1, b1 = the next two (the pieces of a
  // row that ldmatrix hands to a thread are four neighbouring bytes, and the order of a product's terms is free)
  uint32_t qf[D / 16][2];
  float q_mul;
  {
    const int head = hg * kDecHeads + r;
    const bool on = head < a.G;
    const uint2* qrow = reinterpret_cast<const uint2*>(a.q + (static_cast<int64_t>(b) * a.Hq + kvh * a.G + (on ? head : 0)) * D);
    uint2 w[D / 16];
    uint32_t top = 0;
#pragma unroll
    for (int k = 0; k < D / 16; ++k) {
      w[k] = on ? qrow[4 * k + c] : make_uint2(0u, 0u);
#pragma unroll
      for (int j = 0; j < 4; ++j) {
        const uint32_t m = ((j & 2 ? w[k].y : w[k].x) >> (16 * (j & 1))) & 0x7fffu;
        if (m < 0x7f80u) top = max(top, m);
      }
    }
    top = max(top, __shfl_xor_sync(0xffffffffu, top, 1));
    top = max(top, __shfl_xor_sync(0xffffffffu, top, 2));
    int e = 137 - static_cast<int>(top >> 7);       // exponent of the factor: the largest value becomes 2^10 to 2^11
    if (e > 126 || top == 0) e = top == 0 ? 0 : 126;
    const float mul = __uint_as_float(static_cast<uint32_t>(127 + e) << 23);
    q_mul = __uint_as_float(static_cast<uint32_t>(127 - e) << 23);
#pragma unroll
    for (int k = 0; k < D / 16; ++k) {
      qf[k][0] = pack_f16(bf16_lo(w[k].x) * mul, bf16_hi(w[k].x) * mul);
      qf[k][1] = pack_f16(bf16_lo(w[k].y) * mul, bf16_hi(w[k].y) * mul);
    }
  }
  const float qs0 = __shfl_sync(0xffffffffu, q_mul, 8 * c) * a.scale_log2;
  const float qs1 = __shfl_sync(0xffffffffu, q_mul, 8 * c + 4) * a.scale_log2;

  float m_run[2] = {-INFINITY, -INFINITY};   // heads 2c, 2c+1: maximum of the scores (log2 domain)
  float r_run[2] = {-INFINITY, -INFINITY};   // reference of the weights
  float l_run[2] = {0.f, 0.f};
  float oacc[D / 16][4];
#pragma unroll
  for (int i = 0; i < D / 16; ++i) oacc[i][0] = oacc[i][1] = oacc[i][2] = oacc[i][3] = 0.f;

  // pages and scales of the next 32 half tiles to be asked for, one per lane
  int pg = -1;
  float ks = 0.f, vs = 0.f;
  int batch = tb;                            // the tile the batch starts at
  auto load_batch = [&](int t) {
    batch = t;
    const int slot = (2 * t + lane) * (kPagedTile / 2);
    pg = -1; ks = 0.f; vs = -1.f;            // (a negative scale marks an absent half)
    if (t + lane / 2 < te && slot < nvalid) {
      pg = checked_page(a.table[static_cast<int64_t>(b) * a.stride + (slot >> a.page_shift)], a.num_pages);
      if (pg >= 0) {
        const int64_t unit = static_cast<int64_t>(pg) * a.Hkv + kvh;
        ks = a.k_scale[unit];
        vs = a.v_scale[unit];
      } else {
        atomicCAS(a.error_word, 0u, kPageError);
      }
    }
  };
  uint32_t asked = it;
  auto issue_tile = [&](int t) {
    if (t - batch >= 16) load_batch(t);
    const int x = 2 * (t - batch);
    const uint32_t stage = asked % kDecStages;
    const int p0 = __shfl_sync(0xffffffffu, pg, x), p1 = __shfl_sync(0xffffffffu, pg, x + 1);
    const float k1 = __shfl_sync(0xffffffffu, ks, x + (lane & 1)), v1 = __shfl_sync(0xffffffffu, vs, x + (lane & 1));
    if (lane < 2) scales[stage * 2 + lane] = make_float2(k1, v1);
    if (lane == 0) {
      const int slot = t * kPagedTile, mask = (1 << a.page_shift) - 1;
      const uint32_t sk = ring + stage * 2 * SM::kTileBytes, sv = sk + SM::kTileBytes, bar = smem_u32(bars + stage);
      const int r0 = ((p0 * a.Hkv + kvh) << a.page_shift) + (slot & mask);
      if (a.box_rows == kPagedTile) {
        mbar_expect_tx(bars + stage, p0 >= 0 ? 2 * SM::kTileBytes : 0);
        if (p0 >= 0) { tma_load_2d(sk, &tk, bar, 0, r0); tma_load_2d(sv, &tv, bar, 0, r0); }
      } else {
        const int r1 = ((p1 * a.Hkv + kvh) << a.page_shift) + ((slot + kPagedTile / 2) & mask);
        mbar_expect_tx(bars + stage, ((p0 >= 0) + (p1 >= 0)) * SM::kTileBytes);
        if (p0 >= 0) { tma_load_2d(sk, &tk, bar, 0, r0); tma_load_2d(sv, &tv, bar, 0, r0); }
        if (p1 >= 0) {
          tma_load_2d(sk + SM::kTileBytes / 2, &tk, bar, 0, r1);
          tma_load_2d(sv + SM::kTileBytes / 2, &tv, bar, 0, r1);
        }
      }
    }
    ++asked;
  };

  load_batch(tb);
  for (int t = tb; t < min(te, tb + kDecStages - 1); ++t) issue_tile(t);
  __syncwarp();                          // the scales of the first tiles

  for (int t = tb; t < te; ++t) {
    const uint32_t stage = it % kDecStages;
    ok = ok && mbar_wait_warp(bars + stage, (it / kDecStages) & 1, a.error_word, 20);
    ++it;
    if (!ok) break;
    const uint32_t sk = ring + stage * 2 * SM::kTileBytes, sv = sk + SM::kTileBytes;
    const float2 sc0 = scales[stage * 2], sc1 = scales[stage * 2 + 1];
    const bool in0 = sc0.y >= 0.f, in1 = sc1.y >= 0.f;

    // rows that are not attended hold anything at all: a weight of zero does not silence a NaN of V, so those rows are zeroed
    const int slot0 = t * kPagedTile;
    const bool edge = slot0 + kPagedTile > nvalid || ex_cnt > 0 || !in0 || !in1;
    if (edge) {
      const bool on = attended(slot0 + lane) && (lane < kPagedTile / 2 ? in0 : in1);
      if (!on) {
#pragma unroll
        for (int x = 0; x < D / 16; ++x)
          asm volatile("st.shared.v4.b32 [%0], {%1, %1, %1, %1};" ::"r"(sv + lane * D + x * 16), "r"(0) : "memory");
      }
      __syncwarp();
    }

    // ---- S^T[32 tokens, 8 heads] = K Q^T
    float s[2][4] = {};
    const int row = ((lane >> 3) & 1) * 8 + (lane & 7);
#pragma unroll
    for (int x = 0; x < 2; ++x) {
#pragma unroll
      for (int k = 0; k < D / 16; k += 2) {
        uint32_t x0, x1, x2, x3;              // rows 0-7 and 8-15 of chunk k, the same of chunk k + 1
        ldsm_x4(sk + tile_offset<D>(16 * x + row, k + (lane >> 4)), x0, x1, x2, x3);
        mma16816_f16(s[x], e4m3x2_to_f16x2(x0), e4m3x2_to_f16x2(x1), e4m3x2_hi_to_f16x2(x0), e4m3x2_hi_to_f16x2(x1), qf[k][0], qf[k][1]);
        mma16816_f16(s[x], e4m3x2_to_f16x2(x2), e4m3x2_to_f16x2(x3), e4m3x2_hi_to_f16x2(x2), e4m3x2_hi_to_f16x2(x3), qf[k + 1][0], qf[k + 1][1]);
      }
    }
    // s[x][0, 1]: token 16 x + r, heads 2c, 2c+1; s[x][2, 3]: token 16 x + r + 8.  (Two products: the scales together may leave
    // the range of fp32 where the score does not.)
#pragma unroll
    for (int x = 0; x < 2; ++x) {
      const float kk = x ? sc1.x : sc0.x;
      s[x][0] = s[x][0] * qs0 * kk; s[x][1] = s[x][1] * qs1 * kk;
      s[x][2] = s[x][2] * qs0 * kk; s[x][3] = s[x][3] * qs1 * kk;
    }
    if (edge) {
#pragma unroll
      for (int x = 0; x < 2; ++x) {
        const bool in = x ? in1 : in0;
        if (!in || !attended(slot0 + 16 * x + r)) s[x][0] = s[x][1] = -INFINITY;
        if (!in || !attended(slot0 + 16 * x + r + 8)) s[x][2] = s[x][3] = -INFINITY;
      }
    }
    // (exact for powers of two; an absent half has no weights)
    const float lv0 = in0 ? log2f(sc0.y) : in1 ? log2f(sc1.y) : 0.f, lv1 = in1 ? log2f(sc1.y) : lv0;
    float a0 = fmaxf(s[0][0], s[0][2]), a1 = fmaxf(s[0][1], s[0][3]), b0 = fmaxf(s[1][0], s[1][2]), b1 = fmaxf(s[1][1], s[1][3]);
    float t0 = fmaxf(a0, b0), t1 = fmaxf(a1, b1);
#pragma unroll
    for (int o = 4; o < 32; o <<= 1) {
      t0 = fmaxf(t0, __shfl_xor_sync(0xffffffffu, t0, o));
      t1 = fmaxf(t1, __shfl_xor_sync(0xffffffffu, t1, o));
    }
    float u0 = t0 + lv0, u1 = t1 + lv0;
    if (lv0 != lv1) {                                                  // the halves lie in pages of different scales
      u0 = fmaxf(a0 + lv0, b0 + lv1); u1 = fmaxf(a1 + lv0, b1 + lv1);
#pragma unroll
      for (int o = 4; o < 32; o <<= 1) {
        u0 = fmaxf(u0, __shfl_xor_sync(0xffffffffu, u0, o));
        u1 = fmaxf(u1, __shfl_xor_sync(0xffffffffu, u1, o));
      }
    }
    const float mn0 = fmaxf(m_run[0], t0), mn1 = fmaxf(m_run[1], t1), rn0 = fmaxf(r_run[0], u0), rn1 = fmaxf(r_run[1], u1);
    const float mu0 = mn0 == -INFINITY ? 0.f : mn0, mu1 = mn1 == -INFINITY ? 0.f : mn1;
    const float ru0 = rn0 == -INFINITY ? 0.f : rn0, ru1 = rn1 == -INFINITY ? 0.f : rn1;
    const float al0 = fast_exp2(m_run[0] - mu0), al1 = fast_exp2(m_run[1] - mu1);
    const float be0 = fast_exp2(r_run[0] - ru0), be1 = fast_exp2(r_run[1] - ru1);
    m_run[0] = mn0; m_run[1] = mn1; r_run[0] = rn0; r_run[1] = rn1;
    l_run[0] *= al0; l_run[1] *= al1;
    uint32_t pb[2][2];                                                 // P^T as the B operand: tokens 2c, +1 of head r, then 8 + 2c, +1
#pragma unroll
    for (int x = 0; x < 2; ++x) {
      l_run[0] += fast_exp2(s[x][0] - mu0) + fast_exp2(s[x][2] - mu0);
      l_run[1] += fast_exp2(s[x][1] - mu1) + fast_exp2(s[x][3] - mu1);
      const float lv = x ? lv1 : lv0, d0 = lv - ru0, d1 = lv - ru1;
      pb[x][0] = movmatrix_t(pack_f16(fast_exp2(s[x][0] + d0), fast_exp2(s[x][1] + d1)));
      pb[x][1] = movmatrix_t(pack_f16(fast_exp2(s[x][2] + d0), fast_exp2(s[x][3] + d1)));
    }
    if (__any_sync(0xffffffffu, be0 != 1.f || be1 != 1.f)) {
#pragma unroll
      for (int i = 0; i < D / 16; ++i) { oacc[i][0] *= be0; oacc[i][1] *= be1; oacc[i][2] *= be0; oacc[i][3] *= be1; }
    }

    // ---- O^T[D, 8 heads] += V^T P^T.  Transposed, a thread's 32 bits are dims 2r, 2r+1 of tokens 2c and 2c+1: the even dims are
    // the product's rows 0-7, the odd ones its rows 8-15.
#pragma unroll
    for (int x = 0; x < 2; ++x) {
#pragma unroll
      for (int k = 0; k < D / 16; k += 2) {
        uint32_t x0, x1, x2, x3;              // tokens 0-7 and 8-15 of chunk k, the same of chunk k + 1
        ldsm_x4_t(sv + tile_offset<D>(16 * x + row, k + (lane >> 4)), x0, x1, x2, x3);
        x0 = __byte_perm(x0, 0, 0x3120); x1 = __byte_perm(x1, 0, 0x3120);
        x2 = __byte_perm(x2, 0, 0x3120); x3 = __byte_perm(x3, 0, 0x3120);
        mma16816_f16(oacc[k], e4m3x2_to_f16x2(x0), e4m3x2_hi_to_f16x2(x0), e4m3x2_to_f16x2(x1), e4m3x2_hi_to_f16x2(x1), pb[x][0], pb[x][1]);
        mma16816_f16(oacc[k + 1], e4m3x2_to_f16x2(x2), e4m3x2_hi_to_f16x2(x2), e4m3x2_to_f16x2(x3), e4m3x2_hi_to_f16x2(x3), pb[x][0], pb[x][1]);
      }
    }
    if (edge) asm volatile("fence.proxy.async.shared::cta;" ::: "memory");   // the zeroed rows before the next copy into them
    __syncwarp();
    if (t + kDecStages - 1 < te) issue_tile(t + kDecStages - 1);
  }
  if (!ok)                                                             // the copies in flight end before the CTA goes on
    for (; it != asked; ++it) mbar_wait_warp(bars + it % kDecStages, (it / kDecStages) & 1, a.error_word, 21);

  // from the reference of the weights to that of the sums: O relative to m
#pragma unroll
  for (int o = 4; o < 32; o <<= 1) {
    l_run[0] += __shfl_xor_sync(0xffffffffu, l_run[0], o);
    l_run[1] += __shfl_xor_sync(0xffffffffu, l_run[1], o);
  }
  const float g0 = m_run[0] == -INFINITY ? 0.f : fast_exp2(r_run[0] - m_run[0]), g1 = m_run[1] == -INFINITY ? 0.f : fast_exp2(r_run[1] - m_run[1]);
  __syncthreads();                       // everyone is done with the rings
  float* mine = reinterpret_cast<float*>(sm) + warp * kDecHeads * (D + 2);
#pragma unroll
  for (int i = 0; i < D / 16; ++i) {
    *reinterpret_cast<float2*>(mine + (2 * c) * (D + 2) + 16 * i + 2 * r) = make_float2(oacc[i][0] * g0, oacc[i][2] * g0);
    *reinterpret_cast<float2*>(mine + (2 * c + 1) * (D + 2) + 16 * i + 2 * r) = make_float2(oacc[i][1] * g1, oacc[i][3] * g1);
  }
  if (r == 0) {
    *reinterpret_cast<float2*>(mine + (2 * c) * (D + 2) + D) = make_float2(m_run[0], l_run[0]);
    *reinterpret_cast<float2*>(mine + (2 * c + 1) * (D + 2) + D) = make_float2(m_run[1], l_run[1]);
  }
  __syncthreads();
  return ok;
}

// cum[b] = tiles of the sequences before b, b = 0 .. B; returns whether some sequence holds no token.  All threads.
__device__ __forceinline__ int paged_valid(const PagedDecodeArgs& a, int b) {
  const int64_t n = a.n_tokens[b];
  return static_cast<int>(n < a.C ? (n < 0 ? 0 : n) : a.C);
}
__device__ __forceinline__ bool paged_build_cum(const PagedDecodeArgs& a, int* cum) {
  __shared__ int warp_sum[kDecWarps];
  const int tid = threadIdx.x, lane = tid & 31, warp = tid >> 5;
  const int each = (a.B + kDecThreads - 1) / kDecThreads, b0 = tid * each, b1 = min(a.B, b0 + each);
  int local = 0;
  bool empty = false;
  for (int b = b0; b < b1; ++b) {
    const int n = (paged_valid(a, b) + kPagedTile - 1) / kPagedTile;
    cum[b + 1] = n;
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
  for (int b = b0; b < b1; ++b) { run += cum[b + 1]; cum[b + 1] = run; }
  if (tid == 0) cum[0] = 0;
  return __syncthreads_or(empty) != 0;
}

template <int D>
__global__ void __launch_bounds__(kDecThreads) paged_decode_kernel(const __grid_constant__ CUtensorMap tk, const __grid_constant__ CUtensorMap tv,
                                                                   const PagedDecodeArgs a) {
  extern __shared__ uint8_t dyn[];
  using SM = PagedSmem<D>;
  uint8_t* sm = dyn + ((1024u - (smem_u32(dyn) & 1023u)) & 1023u);      // (the swizzles repeat every 1024 or 512 bytes)
  int* cum = reinterpret_cast<int*>(sm + SM::kCum);
  pdl_trigger();
  if (threadIdx.x < kDecWarps * kDecStages) mbar_init(reinterpret_cast<uint64_t*>(sm + SM::kBars) + threadIdx.x, 1);
  if (threadIdx.x == 0) { mbar_fence_init(); tma_prefetch_desc(&tk); tma_prefetch_desc(&tv); }
  pdl_wait();
  const bool any_empty = paged_build_cum(a, cum);                       // (its barriers order the mbarriers' initialisation too)
  const int ups = a.Hkv * a.HG, n_cta = gridDim.x, me = blockIdx.x, warp = threadIdx.x >> 5;
  const int64_t total = static_cast<int64_t>(cum[a.B]) * ups;
  const bool narrow = total * n_cta <= 0xffffffffll;                    // 64-bit divisions take 200 cycles each
  auto start_of = [&](int64_t x) -> int64_t {
    return narrow ? static_cast<uint32_t>(total) * static_cast<uint32_t>(x) / static_cast<uint32_t>(n_cta) : total * x / n_cta;
  };
  auto cta_of = [&](int64_t f) {
    int64_t x = narrow ? static_cast<uint32_t>(f) * static_cast<uint32_t>(n_cta) / static_cast<uint32_t>(total) : f * n_cta / total;
    while (x + 1 < n_cta && start_of(x + 1) <= f) ++x;
    while (x > 0 && start_of(x) > f) --x;
    return static_cast<int>(x);
  };
  const int64_t f0 = start_of(me), f1 = start_of(me + 1);
  for (int e = 0; any_empty && e < a.B; ++e) {                          // sequences without tokens: their empty results
    if (cum[e + 1] != cum[e]) continue;
    for (int x = 0; x < ups; ++x) {
      const int64_t u = static_cast<int64_t>(e) * ups + x;
      if (u % n_cta == me) decode_merge_unit<D>(a, reinterpret_cast<float*>(sm), e, x, u, 0, 0, total, n_cta);
    }
  }
  __shared__ int s_last;
  uint32_t it = 0;
  int b = 0;
  if (f0 < f1) {
    int lo = 0, hi = a.B;                                               // cum[lo] * ups <= f0 < cum[hi] * ups
    while (hi - lo > 1) {
      const int mid = (lo + hi) >> 1;
      if (static_cast<int64_t>(cum[mid]) * ups <= f0) lo = mid; else hi = mid;
    }
    b = lo;
  }
  for (int64_t pos = f0; pos < f1;) {
    while (static_cast<int64_t>(cum[b + 1]) * ups <= pos) ++b;
    const int nt = cum[b + 1] - cum[b];
    const int64_t before = static_cast<int64_t>(cum[b]) * ups, rel = pos - before;
    const int k = narrow ? static_cast<int>(static_cast<uint32_t>(rel) / static_cast<uint32_t>(nt)) : static_cast<int>(rel / nt);
    const int t0 = static_cast<int>(rel - static_cast<int64_t>(k) * nt);
    const int n = static_cast<int>(min(static_cast<int64_t>(nt - t0), f1 - pos));
    const int64_t first = before + static_cast<int64_t>(k) * nt, u = static_cast<int64_t>(b) * ups + k;
    const int tb = t0 + static_cast<int>(static_cast<int64_t>(n) * warp / kDecWarps);
    const int te = t0 + static_cast<int>(static_cast<int64_t>(n) * (warp + 1) / kDecWarps);
    asm volatile("fence.proxy.async.shared::cta;" ::: "memory");        // what was written over the rings, before the copies into them
    __syncthreads();
    const bool direct = t0 == 0 && n == nt;
    paged_run_segment<D>(a, tk, tv, sm, b, k / a.HG, k % a.HG, paged_valid(a, b), tb, te, it);
    decode_merge_warps<D>(a, reinterpret_cast<float*>(sm), b, k / a.HG, k % a.HG, a.part + (me + u) * (kDecHeads * (D + 2)), direct);
    pos += n;
    if (direct) continue;
    // the CTA that delivers a unit's last record merges them, in index order, and re-arms the counter
    const int c_lo = t0 == 0 ? me : cta_of(first), c_hi = t0 + n == nt ? me : cta_of(first + nt - 1);
    int pieces = c_hi - c_lo + 1;
    if (total < n_cta)
      for (int x = c_lo; x <= c_hi; ++x) pieces -= start_of(x) == start_of(x + 1) ? 1 : 0;
    __syncthreads();
    if (threadIdx.x == 0) {
      const bool last = ticket_add(a.unit_count + u) + 1u == static_cast<unsigned>(pieces);
      s_last = last;
      if (last) a.unit_count[u] = 0u;
    }
    __syncthreads();
    if (s_last) decode_merge_unit<D>(a, reinterpret_cast<float*>(sm), b, k, u, c_lo, c_hi - c_lo + 1, total, n_cta);
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
  // rows of a pool are addressed by TMA coordinates of 32 bits
  if (static_cast<int64_t>(p->num_pages) * p->Hkv * p->page_tokens > 0x7fffffffll) return LG_ERR_UNSUPPORTED;
  return LG_OK;
}

static bool aligned(const void* p, uintptr_t n) { return (reinterpret_cast<uintptr_t>(p) & (n - 1)) == 0; }
static bool bad_pools(const void* k_pool, const void* v_pool, const void* k_scale, const void* v_scale) {
  return !k_pool || !v_pool || !k_scale || !v_scale || !aligned16(k_pool) || !aligned16(v_pool) || !aligned(k_scale, 4) || !aligned(v_scale, 4);
}

// a pool as rows of D bytes, boxes of box_rows rows
static lg_status pool_tmap(CUtensorMap* out, const void* base, int64_t rows, int D, int box_rows) {
  const cuuint64_t dims[2] = {static_cast<cuuint64_t>(D), static_cast<cuuint64_t>(rows)};
  const cuuint64_t strides[1] = {static_cast<cuuint64_t>(D)};
  const cuuint32_t box[2] = {static_cast<cuuint32_t>(D), static_cast<cuuint32_t>(box_rows)};
  return encode_tmap_u8(out, base, 2, dims, strides, box, D == 128 ? CU_TENSOR_MAP_SWIZZLE_128B : CU_TENSOR_MAP_SWIZZLE_64B);
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

struct PagedDecodePlan { int HG, slice, n_cta; int64_t units; size_t count_bytes, total_bytes; };
static PagedDecodePlan plan_paged_decode(const lg_paged_params* p, int sms) {
  PagedDecodePlan w;
  w.HG = (p->Hq / p->Hkv + kDecHeads - 1) / kDecHeads;
  w.slice = p->B < kPagedMaxB ? p->B : kPagedMaxB;
  w.units = static_cast<int64_t>(w.slice) * p->Hkv * w.HG;
  w.count_bytes = align_up(static_cast<size_t>(w.units) * sizeof(unsigned int), 256);
  w.total_bytes = sizeof(WsHeader) + w.count_bytes +
                  align_up((static_cast<size_t>(kPagedMaxCtas) + w.units) * kDecHeads * (p->D + 2) * sizeof(float), 256);
  // a CTA has at least a tile for each two of its warps; as many as fit an SM (D = 64: two), and a whole number of them per unit
  // where that costs at most a quarter of them (equal lengths then make one segment of every slice)
  const int64_t C = static_cast<int64_t>(p->sink_tokens) + p->window_tokens;
  const int64_t tiles = w.units * ((C + kPagedTile - 1) / kPagedTile);
  int64_t n = (tiles + kDecWarps / 2 - 1) / (kDecWarps / 2);
  const int64_t most = (p->D == 64 ? 2 : 1) * static_cast<int64_t>(sms);
  if (n > most) n = most;
  if (n > kPagedMaxCtas) n = kPagedMaxCtas;
  if (n > w.units && (n / w.units) * w.units * 4 >= n * 3) n = (n / w.units) * w.units;
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
  a.sink = p->sink_tokens; a.window = p->window_tokens; a.page_tokens = p->page_tokens; a.stride = paged_table_stride(p);
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
  const int64_t blocks = (static_cast<int64_t>(p->B) * T + kSlotMapThreads - 1) / kSlotMapThreads;
  if (blocks > 0x7fffffff) return LG_ERR_UNSUPPORTED;
  if ((s = check_arch()) != LG_OK) return s;
  SlotMapArgs a;
  a.n_tokens = n_tokens; a.first = first; a.count = count; a.table = block_table; a.slot_map = slot_map;
  a.B = p->B; a.T = T; a.sink = p->sink_tokens; a.window = p->window_tokens;
  a.page_shift = page_shift(p->page_tokens); a.num_pages = p->num_pages; a.stride = paged_table_stride(p);
  return launch_kernel(true, slot_map_kernel, dim3(static_cast<unsigned>(blocks)), kSlotMapThreads, 0, static_cast<cudaStream_t>(stream), a) ==
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
  AppendArgs a;
  a.stride_t = p->D;
  a.stride_h = static_cast<int64_t>(T_new) * p->D;
  a.stride_b = a.stride_h * p->Hkv;
  if (new_strides && (new_strides[0] || new_strides[1] || new_strides[2])) {
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
  a.page_tokens = p->page_tokens; a.num_pages = p->num_pages; a.stride = paged_table_stride(p);
  a.max_touched = max_touched_pages(T_new, p->sink_tokens, p->window_tokens, p->page_tokens);
  const int64_t blocks = static_cast<int64_t>(p->B) * a.max_touched * p->Hkv * 2;
  if (blocks > 0x7fffffff) return LG_ERR_UNSUPPORTED;
  if ((s = check_arch()) != LG_OK) return s;
  const int nu = p->page_tokens * p->D / 8 / kAppendThreads;
  auto run = [&](auto kern) {
    return launch_kernel(true, kern, dim3(static_cast<unsigned>(blocks)), kAppendThreads, 0, static_cast<cudaStream_t>(stream), a) == cudaSuccess
               ? LG_OK : LG_ERR_CUDA;
  };
  if (p->D == 128)
    return nu == 2 ? run(paged_append_kernel<128, 2>) : nu == 4 ? run(paged_append_kernel<128, 4>)
         : nu == 8 ? run(paged_append_kernel<128, 8>) : run(paged_append_kernel<128, 16>);
  return nu == 1 ? run(paged_append_kernel<64, 1>) : nu == 2 ? run(paged_append_kernel<64, 2>)
       : nu == 4 ? run(paged_append_kernel<64, 4>) : run(paged_append_kernel<64, 8>);
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
  const int64_t blocks = (static_cast<int64_t>(T) * (p->D / 16) + kGatherThreads - 1) / kGatherThreads;
  if (blocks > 0x7fffffff || p->Hkv > 65535 || p->B > 65535) return LG_ERR_UNSUPPORTED;
  if ((s = check_arch()) != LG_OK) return s;
  GatherArgs a;
  a.pool[0] = static_cast<const uint8_t*>(k_pool); a.pool[1] = static_cast<const uint8_t*>(v_pool);
  a.scale[0] = k_scale; a.scale[1] = v_scale; a.slot_map = slot_map;
  a.out[0] = static_cast<uint4*>(k_out); a.out[1] = static_cast<uint4*>(v_out);
  a.Hkv = p->Hkv; a.T = T; a.D = p->D; a.page_shift = page_shift(p->page_tokens); a.num_pages = p->num_pages;
  return launch_kernel(true, paged_gather_kernel, dim3(static_cast<unsigned>(blocks), p->Hkv, p->B), kGatherThreads, 0,
                       static_cast<cudaStream_t>(stream), a) == cudaSuccess ? LG_OK : LG_ERR_CUDA;
}

size_t lg_paged_decode_workspace_bytes(const lg_paged_params* p) {
  return check_paged(p) == LG_OK ? plan_paged_decode(p, kSms).total_bytes : 0;
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
  const PagedDecodePlan w = plan_paged_decode(p, kSms);
  if (workspace_bytes < w.total_bytes) return LG_ERR_WORKSPACE;
  if (w.units > 0x7fffffff) return LG_ERR_UNSUPPORTED;
  if ((s = check_arch()) != LG_OK) return s;
  PagedDecodeArgs a;
  a.k_scale = k_scale; a.v_scale = v_scale;
  uint8_t* ws = static_cast<uint8_t*>(workspace);
  a.error_word = reinterpret_cast<unsigned int*>(ws);
  a.unit_count = reinterpret_cast<unsigned int*>(ws + sizeof(WsHeader));
  a.part = reinterpret_cast<float*>(ws + sizeof(WsHeader) + w.count_bytes);
  a.Hq = p->Hq; a.Hkv = p->Hkv; a.G = p->Hq / p->Hkv; a.HG = w.HG;
  a.C = p->sink_tokens + p->window_tokens;
  a.sink = p->sink_tokens; a.block_tokens = p->block_tokens;
  a.page_shift = page_shift(p->page_tokens); a.num_pages = p->num_pages; a.stride = paged_table_stride(p);
  a.box_rows = p->page_tokens < kPagedTile ? p->page_tokens : kPagedTile;
  a.scale_log2 = (p->scale > 0.f ? p->scale : 1.0f / sqrtf(static_cast<float>(p->D))) * 1.4426950408889634f;
  CUtensorMap tk, tv;
  const int64_t rows = static_cast<int64_t>(p->num_pages) * p->Hkv * p->page_tokens;
  if ((s = pool_tmap(&tk, k_pool, rows, p->D, a.box_rows)) != LG_OK) return s;
  if ((s = pool_tmap(&tv, v_pool, rows, p->D, a.box_rows)) != LG_OK) return s;
  if ((s = allow_decode_smem()) != LG_OK) return s;
  for (int b = 0; b < p->B; b += kPagedMaxB) {   // (larger batches: launch by launch, over the same records)
    a.B = p->B - b < kPagedMaxB ? p->B - b : kPagedMaxB;
    a.q = static_cast<const __nv_bfloat16*>(q) + static_cast<int64_t>(b) * p->Hq * p->D;
    a.o = static_cast<__nv_bfloat16*>(o) + static_cast<int64_t>(b) * p->Hq * p->D;
    a.lse = lse ? lse + static_cast<int64_t>(b) * p->Hq : nullptr;
    a.table = block_table + static_cast<int64_t>(b) * a.stride;
    a.n_tokens = n_tokens + b;
    const cudaError_t e = p->D == 128 ? launch_kernel(true, paged_decode_kernel<128>, dim3(w.n_cta), kDecThreads, PagedSmem<128>::bytes(a.B),
                                                      static_cast<cudaStream_t>(stream), tk, tv, a)
                                      : launch_kernel(true, paged_decode_kernel<64>, dim3(w.n_cta), kDecThreads, PagedSmem<64>::bytes(a.B),
                                                      static_cast<cudaStream_t>(stream), tk, tv, a);
    if (e != cudaSuccess) return LG_ERR_CUDA;
  }
  return LG_OK;
}

}  // extern "C"
