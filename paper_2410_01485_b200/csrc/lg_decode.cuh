// What the two decode kernels share (bf16 ring, paged 8-bit cache): warp-level building blocks and the merges of
// partial results.  A partial result is a record of 8 heads: O [8][D] relative to each head's running maximum, then the
// (maximum, sum) pairs [8][2], all fp32.
#pragma once
#include <math.h>

#include "lg_common.cuh"

namespace lg {

constexpr int kDecWarps = 8;          // warps per CTA, each with its own pipeline of tiles
constexpr int kDecThreads = kDecWarps * 32;
constexpr int kDecStages = 3;
constexpr int kDecHeads = 8;          // query heads per CTA (mma N)

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
__device__ __forceinline__ void mma16816(float* c, uint32_t a0, uint32_t a1, uint32_t a2, uint32_t a3, uint32_t b0,
                                         uint32_t b1) {
  asm volatile(
      "mma.sync.aligned.m16n8k16.row.col.f32.bf16.bf16.f32 {%0, %1, %2, %3}, {%4, %5, %6, %7}, {%8, %9}, "
      "{%0, %1, %2, %3};"
      : "+f"(c[0]), "+f"(c[1]), "+f"(c[2]), "+f"(c[3])
      : "r"(a0), "r"(a1), "r"(a2), "r"(a3), "r"(b0), "r"(b1));
}

// The warps' partial results of a segment, [warp][head 8][D + 2] in shared memory (each head's O, then its maximum and sum), merged in warp order.
// `direct`: the segment is the whole unit, so the result is final and goes straight to o / lse; otherwise it is the CTA's
// record for the merge across CTAs.  kDecThreads threads.
template <int D, typename Args>
__device__ __forceinline__ void decode_merge_warps(const Args& a, float* red, int b, int kvh, int hg, float* out, bool direct) {
  constexpr int kRec = D + 2;
  const int warp = threadIdx.x >> 5, lane = threadIdx.x & 31;
  {   // a warp per head: its weights once per thread, then D / 32 values of a lane, two neighbours at a time (four: two-way conflicts)
    static_assert(kDecWarps == kDecHeads && (D / 32) % 2 == 0, "a warp per head");
    constexpr int V = D / 32;
    const int head = warp, d = lane * 2;                 // values d, d + 1, and every 64 on
    const float* mine = red + head * kRec;               // the head's row of warp 0's record
    float f[kDecWarps], m = -INFINITY, l = 0.f, acc[V] = {};
#pragma unroll
    for (int w = 0; w < kDecWarps; ++w) { f[w] = mine[w * kDecHeads * kRec + D]; m = fmaxf(m, f[w]); }
    const float mu = m == -INFINITY ? 0.f : m;
#pragma unroll
    for (int w = 0; w < kDecWarps; ++w) {
      f[w] = fast_exp2(f[w] - mu);
      l += f[w] * mine[w * kDecHeads * kRec + D + 1];
#pragma unroll
      for (int x = 0; x < V; x += 2) {
        const float2 o2 = *reinterpret_cast<const float2*>(mine + w * kDecHeads * kRec + d + 32 * x);
        acc[x] += f[w] * o2.x;
        acc[x + 1] += f[w] * o2.y;
      }
    }
    if (direct) {
      const int gh = hg * kDecHeads + head;
      if (gh < a.G) {
        const int64_t qh = static_cast<int64_t>(b) * a.Hq + kvh * a.G + gh;
#pragma unroll
        for (int x = 0; x < V; x += 2)
          *reinterpret_cast<uint32_t*>(a.o + qh * D + d + 32 * x) = l > 0.f ? pack_bf16(acc[x] / l, acc[x + 1] / l) : 0u;
        if (lane == 0 && a.lse) a.lse[qh] = l > 0.f ? (m + log2f(l)) * 0.6931471805599453f : -INFINITY;
      }
    } else {
#pragma unroll
      for (int x = 0; x < V; x += 2) *reinterpret_cast<float2*>(out + head * D + d + 32 * x) = make_float2(acc[x], acc[x + 1]);
      if (lane == 0) { out[kDecHeads * D + 2 * head] = m; out[kDecHeads * D + 2 * head + 1] = l; }
    }
  }
}

// Merge the records of unit (b, k): CTAs first_cta .. first_cta + n_rec - 1, in that order (whichever CTA happens
// to run this, the summation order is the same).  kDecThreads threads; `scratch`: shared memory, 8 (n_rec + 1)
// pairs of floats.  The records sit in L2, so what this takes is round trips: one for all (max, sum) pairs, one
// for eight records' values at a time (read record by record it was a chain of 2 n_rec dependent round trips:
// one sequence of 8 kv heads, 16 records a unit, 24.5 -> 12.2 us for the kernel).
template <int D, typename Args>
__device__ __forceinline__ void decode_merge_unit(const Args& a, float* scratch, int b, int k, int64_t u, int first_cta,
                                                  int n_rec, int64_t total, int n_cta) {
  constexpr int kRec = D + 2;
  static_assert(kDecWarps == kDecHeads, "a warp per head");
  const int kvh = k / a.HG, hg = k % a.HG, tid = threadIdx.x, lane = tid & 31;
  const float* recs = a.part + (static_cast<int64_t>(first_cta) + u) * (kDecHeads * kRec);
  // a CTA with an empty slice (possible only with fewer tiles than CTAs) wrote no record
  const bool sparse_slices = total < n_cta;
  auto absent = [&](int c) { return sparse_slices && total * c / n_cta == total * (c + 1) / n_cta; };
  float2* ml = reinterpret_cast<float2*>(scratch);           // [n_rec][8]: (max, sum), then x becomes the record's weight
  // the first records' values travel together with the pairs (four values of one head a thread)
  constexpr int kBatch = 8;
  const int idx = tid * 4;
  float4 v[kBatch];
  auto load_batch = [&](int i0) {
#pragma unroll
    for (int x = 0; x < kBatch; ++x)
      v[x] = (idx < kDecHeads * D && i0 + x < n_rec && !absent(first_cta + i0 + x))
                 ? __ldcg(reinterpret_cast<const float4*>(recs + static_cast<int64_t>(i0 + x) * (kDecHeads * kRec) + idx))
                 : make_float4(0.f, 0.f, 0.f, 0.f);
  };
  load_batch(0);
  __syncthreads();                                           // scratch: whoever used this shared memory is done
  for (int e = tid; e < n_rec * kDecHeads; e += kDecThreads) {
    const int i = e / kDecHeads;
    ml[e] = absent(first_cta + i) ? make_float2(-INFINITY, 0.f)
                                  : __ldcg(reinterpret_cast<const float2*>(recs + static_cast<int64_t>(i) * (kDecHeads * kRec) +
                                                                           kDecHeads * D) + e % kDecHeads);
  }
  __syncthreads();
  {
    const int head = tid >> 5;
    float m = -INFINITY, l = 0.f;
    for (int i = lane; i < n_rec; i += 32) m = fmaxf(m, ml[i * kDecHeads + head].x);
#pragma unroll
    for (int o = 16; o > 0; o >>= 1) m = fmaxf(m, __shfl_xor_sync(0xffffffffu, m, o));
    const float mu = m == -INFINITY ? 0.f : m;
    for (int i = lane; i < n_rec; i += 32) {
      const float f = fast_exp2(ml[i * kDecHeads + head].x - mu);
      l += f * ml[i * kDecHeads + head].y;
      ml[i * kDecHeads + head].x = f;
    }
#pragma unroll
    for (int o = 16; o > 0; o >>= 1) l += __shfl_xor_sync(0xffffffffu, l, o);
    if (lane == 0) ml[n_rec * kDecHeads + head] = make_float2(m, l);
  }
  __syncthreads();
  static_assert(kDecHeads * 128 <= kDecThreads * 4, "one piece of a head per thread");
  if (idx < kDecHeads * D) {
    const int head = idx / D, gh = hg * kDecHeads + head;
    float4 acc = make_float4(0.f, 0.f, 0.f, 0.f);
    for (int i0 = 0;;) {
#pragma unroll
      for (int x = 0; x < kBatch; ++x) {
        const float f = i0 + x < n_rec ? ml[(i0 + x) * kDecHeads + head].x : 0.f;
        acc.x += f * v[x].x; acc.y += f * v[x].y; acc.z += f * v[x].z; acc.w += f * v[x].w;
      }
      i0 += kBatch;
      if (i0 >= n_rec) break;
      load_batch(i0);
    }
    if (gh < a.G) {
      const float m = ml[n_rec * kDecHeads + head].x, l = ml[n_rec * kDecHeads + head].y;
      const int64_t qh = static_cast<int64_t>(b) * a.Hq + kvh * a.G + gh;
      uint2 out;
      out.x = l > 0.f ? pack_bf16(acc.x / l, acc.y / l) : 0u;
      out.y = l > 0.f ? pack_bf16(acc.z / l, acc.w / l) : 0u;
      *reinterpret_cast<uint2*>(a.o + qh * D + idx % D) = out;
      if (idx % D == 0 && a.lse) a.lse[qh] = l > 0.f ? (m + log2f(l)) * 0.6931471805599453f : -INFINITY;
    }
  }
}

}  // namespace lg
