// chunk_mask.cuh -- which cached rows a token of a chunk sees.  Token i of
// sequence b (n rows cached before the chunk, C tokens in it, N = n + C)
// sits at row p = n + i and sees rows lo <= j < hi,
//   hi = N (mask_block 0), else min(N, (p / mask_block + 1) mask_block),
//   lo = max(0, key_start, p + 1 - window where window > 0);
// both grow with p, so a range of tokens sees [lo of the first, hi of the last).
// With `sinks` the rows ks <= j < min(ks + sinks, hi), ks = max(0, key_start),
// stay visible to it through the window.
#pragma once
#include "common.cuh"
#include "kernels.h"
#include "ragged.cuh"

namespace simsd {

struct ChunkSeq {
  int start, C, n, ks;
  bool bad;      // prefix length out of range: its rows are zero
  bool bad_off;  // token offsets out of range: no rows
};

__device__ __forceinline__ ChunkSeq chunk_seq(const ChunkArgs& a, int b) {
  ChunkSeq s;
  const Chunk c = chunk_of(a.token_start, b, a.T);
  s.start = c.start;
  s.C = c.count;
  s.bad_off = c.bad;
  s.n = a.prefix_len[b];
  s.ks = a.key_start ? max(0, a.key_start[b]) : 0;
  s.bad = s.n < 0 || static_cast<long long>(s.n) + s.C > static_cast<long long>(a.max_pages) * a.page_size;
  return s;
}

__device__ __forceinline__ int key_hi(const ChunkArgs& a, const ChunkSeq& s, int i) {
  const int N = s.n + s.C;
  if (a.mask_block == 0) return N;
  const int p = s.n + i;
  if (a.mask_block == 1) return p + 1;
  const long long h = static_cast<long long>(p / a.mask_block + 1) * a.mask_block;
  return static_cast<int>(min(static_cast<long long>(N), h));
}

__device__ __forceinline__ int key_lo(const ChunkArgs& a, const ChunkSeq& s, int i) {
  return a.window > 0 ? max(s.ks, s.n + i + 1 - a.window) : s.ks;
}

// End of the first rows that stay visible to a token that sees rows below hi.
__device__ __forceinline__ int sink_end(const ChunkArgs& a, const ChunkSeq& s, int hi) {
  return static_cast<int>(min(static_cast<long long>(hi), static_cast<long long>(s.ks) + a.sinks));
}

}  // namespace simsd
