"""Index arithmetic of the paged cache (csrc/lg_paged.h), compiled for the host, against token-by-token simulation, and the
arithmetic of the reference that the GPU tests compare with.  No GPU."""
import os
import shutil
import subprocess

import numpy as np
import pytest

from paper_2410_01485_b200 import build
from tests import paged_reference as R

SOURCE = r"""
#define __forceinline__ inline
#include "lg_paged.h"
#include <cmath>
#include <cstdio>
#include <cstdlib>
#include <cstring>
#include <map>
#include <set>
using namespace lg;
int main() {
  std::srand(3);
  for (int i = 0; i < 4000; ++i) {
    const int sink = std::rand() % 3 == 0 ? 0 : std::rand() % 90, window = 1 + std::rand() % 200, shift = 4 + std::rand() % 4, P = 1 << shift;
    const int64_t n0 = std::rand() % 700, T = std::rand() % 3 == 0 ? 1 : std::rand() % 500, n1 = n0 + T;
    std::map<int, int64_t> held;
    for (int64_t j = 0; j < n1; ++j) held[slot_of(j, sink, window)] = j;
    std::set<int> pages;
    const RingHead head = ring_head(n1, sink, window);
    for (int s = 0; s < sink + window + 5; ++s) {
      const int64_t want = held.count(s) ? held[s] : -1;
      if (held_position(s, n1, head, sink, window) != want) { std::printf("held\n"); return 1; }
      if (want >= n0) pages.insert(s / P);
    }
    const TouchedPages t = touched_pages(n0, n1, head, sink, window, shift);
    if (t.total() != (int)pages.size() || t.total() > max_touched_pages(T, sink, window, P)) { std::printf("count\n"); return 1; }
    int x = 0;
    for (int p : pages) if (t.page(x++) != p) { std::printf("page\n"); return 1; }
    if (pages_of(n1, sink, window, shift) != (int)((held.size() + P - 1) / P)) { std::printf("pages_of\n"); return 1; }
  }
  // far positions: 64-bit counts, on both sides of 2^32 and far behind
  for (const int64_t far : {(1ll << 32) - 150, (1ll << 32) + 3, (1ll << 40) + 12345}) {
    for (int r = 0; r < 300; ++r) {
      const int s = slot_of(far + r, 7, 300);
      if (held_position(s, far + 300, ring_head(far + 300, 7, 300), 7, 300) != far + r) { std::printf("far\n"); return 1; }
    }
    const TouchedPages t = touched_pages(far, far + 1, ring_head(far + 1, 7, 300), 7, 300, 6);
    if (t.total() != 1 || t.page(0) != slot_of(far, 7, 300) / 64) { std::printf("far pages\n"); return 1; }
  }
  if (pages_of(-5, 4, 100, 4) != 0) { std::printf("negative\n"); return 1; }
  // exponents: the smallest one that covers, over all magnitudes of bf16 and the borders
  for (uint32_t b = 0; b < 0x7f80u; ++b) {
    uint32_t bits = b << 16;
    float v;
    std::memcpy(&v, &bits, 4);
    const int e = page_exponent(bits);
    const double fit = std::ldexp(448.0, e), below = std::ldexp(448.0, e - 1);
    if (v == 0 ? e != 0 : !(v <= fit && (e == kPageMinExp || v > below))) { std::printf("exponent %u %d\n", b, e); return 1; }
  }
  std::printf("ok\n");
  return 0;
}
"""


@pytest.mark.skipif(shutil.which("g++") is None, reason="needs a host compiler")
def test_closed_forms_against_simulation(tmp_path):
    src, exe = tmp_path / "t.cpp", tmp_path / "t"
    src.write_text(SOURCE)
    cuda = os.environ.get("CUDA_HOME", "/usr/local/cuda")
    subprocess.run(["g++", "-O1", "-std=c++17", "-I", build.CSRC, "-I", os.path.join(cuda, "include"), str(src), "-o",
                    str(exe)], check=True)
    out = subprocess.run([str(exe)], capture_output=True, text=True)
    assert out.stdout.split() == ["ok"] and out.returncode == 0


def test_reference_codes_against_torch():
    import torch
    x = torch.cat([torch.linspace(-448, 448, 20011), torch.randn(20000) * 0.01, torch.randn(5000) * 2.0 ** -9, torch.zeros(3)])
    want = x.to(torch.float8_e4m3fn).view(torch.uint8).numpy()
    assert np.array_equal(R.encode_e4m3(x.double().numpy()) & 127, want & 127)
    codes = np.arange(256, dtype=np.uint8)
    back = torch.from_numpy(codes).view(torch.float8_e4m3fn).double().numpy()
    assert np.array_equal(np.nan_to_num(R.decode_e4m3(codes), nan=1e9), np.nan_to_num(back, nan=1e9))
    assert np.array_equal(R.encode_e4m3(R.decode_e4m3(codes))[codes & 127 != 127], codes[codes & 127 != 127])


def test_reference_scale_is_the_smallest_that_covers():
    for v in (448.0, 449.0, 1.0, 1e-30, 3e38, 447.9, 896.0):
        s = R.scale_for(np.array([0.0, -v, np.inf, np.nan]))
        assert v <= 448 * s and v > 224 * s
    assert R.scale_for(np.zeros(4)) == 1.0 and R.scale_for(np.array([np.nan])) == 1.0 and R.scale_for(np.array([1e-40])) == 2.0 ** -120


CHUNK_SOURCE = r"""
#define __forceinline__ inline
#include "lg_paged.h"
#include <cstdio>
#include <cstdlib>
using namespace lg;
// The virtual sequence of a chunk (kept rows, then its own): which position a row stands for, and that what the attention kernel
// derives from the rows is what the positions say.
int main() {
  std::srand(5);
  int gaps = 0, short_sinks = 0;
  for (int i = 0; i < 3000; ++i) {
    const int sink = 64 * (std::rand() % 3), block = std::rand() % 2 ? 0 : (std::rand() % 2 ? 64 : 16), window = 64 * (1 + std::rand() % 4);
    const int cap = sink + window, T = 1 + std::rand() % (block ? window - block + 1 : window);      // (no more than a sequence without its sink allows)
    const int64_t n = std::rand() % 4 == 0 ? std::rand() % (sink + 1) : std::rand() % 1500;
    const int held = n < cap ? n : cap;
    int kept = held;
    if (held < cap && std::rand() % 4) { kept = held + std::rand() % (cap - held + 1); if (kept != held && kept < sink) kept = sink; }
    ChunkSeq s;
    s.held = held;
    s.ring0 = (n - held) % window;
    s.phase = block ? (((n - kept) % block) + block) % block : 0;
    s.seen = 0;
    const ChunkView view = chunk_view(kept, sink, s);
    gaps += kept > held; short_sinks += kept > held && held < sink;
    const int first = view.first > sink ? view.first : sink;
    int found = 0;
    for (int v = 0; v < kept + T; ++v) {
      // the position that row v holds (-1: none)
      int64_t pos = -1;
      if (v >= kept) pos = n + v - kept;
      else if (v < sink) pos = v < view.sink_end ? v : -1;
      else if (v >= first) pos = n - (kept - v);
      if (pos >= 0 && v < kept) {
        ++found;
        if (pos >= n || (v >= sink && (pos < sink || slot_of(pos, sink, window) != sink + (s.ring0 + v - first) % window))) { std::printf("row %d\n", v); return 1; }
        if (!chunk_block_held(view, sink, v / 64)) { std::printf("block %d\n", v / 64); return 1; }
      }
      for (int t = 0; t < T; t += 1 + T / 7) {
        const int q = kept + t;
        const int64_t at = n + t;
        const int lo0 = block ? ((q + s.phase) / block - window / block + 1) * block - s.phase : q - window + 1;
        const int lo = v < sink ? 0 : (lo0 > view.first ? lo0 : view.first), end = v < sink && view.sink_end < q + 1 ? view.sink_end : q + 1;
        const bool kernel = v >= lo && v < end;
        const bool near = block ? at / block - pos / block < window / block : at - pos < window;
        const bool want = pos >= 0 && pos <= at && (near || pos < sink);
        if (kernel != want) { std::printf("row %d of query %d: %d, sink %d window %d block %d n %d kept %d\n", v, t, kernel, sink, window, block, (int)n, kept); return 1; }
      }
    }
    if (found != held && !(kept == held && held < sink)) { std::printf("held %d of %d\n", found, held); return 1; }
  }
  std::printf(gaps > 500 && short_sinks > 100 ? "ok\n" : "few\n");
  return 0;
}
"""


@pytest.mark.skipif(shutil.which("g++") is None, reason="needs a host compiler")
def test_rows_of_a_chunk_against_positions(tmp_path):
    src, exe = tmp_path / "t.cpp", tmp_path / "t"
    src.write_text(CHUNK_SOURCE)
    cuda = os.environ.get("CUDA_HOME", "/usr/local/cuda")
    subprocess.run(["g++", "-O1", "-std=c++17", "-I", build.CSRC, "-I", os.path.join(cuda, "include"), str(src), "-o",
                    str(exe)], check=True)
    out = subprocess.run([str(exe)], capture_output=True, text=True)
    assert out.stdout.split() == ["ok"] and out.returncode == 0, out.stdout
