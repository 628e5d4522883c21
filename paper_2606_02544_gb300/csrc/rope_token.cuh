// rope_token.cuh -- where a token of a chunk lies: its position and its row
// in the paged cache.
#pragma once
#include "common.cuh"
#include "kernels.h"
#include "ragged.cuh"

namespace simsd {

// A token of a block: its position, destination row of the cache in rows
// of a head at KV head 0 (-1: not written), and what its q row becomes
struct Token {
  long long row;
  int pos;
  int state;  // 0: outside every sequence (untouched), 1: rotated, 2: zeroed
};

// `append`: the token goes to the cache (else it is only rotated).  A warp.
__device__ __forceinline__ Token resolve(const RopeArgs& a, int tok, bool append) {
  Token t;
  t.row = -1;
  t.pos = 0;
  t.state = 0;
  if (!append) {
    t.pos = a.positions[tok];
    t.state = 1;
    return t;
  }
  const int lane = threadIdx.x & 31;
  const int b = warp_find_seq(a.token_start, a.Bt, tok);
  if (b < 0) return t;
  const Chunk c = chunk_of(a.token_start, b, a.T);
  if (c.bad) return t;
  const int n = a.prefix_len[b], i = tok - c.start;
  if (n < 0 || static_cast<long long>(n) + c.count > static_cast<long long>(a.max_pages) * a.page_size) {
    if (lane == 0) raise_error(a.err_word, SIMSD_EW_PREFIX_LEN);
    t.state = 2;
    return t;
  }
  t.state = 1;
  const int dst = n + i, pi = dst / a.page_size;
  t.pos = a.positions ? a.positions[tok] : dst;
  const int pg = a.block_table[static_cast<size_t>(b) * a.max_pages + pi];
  if (pg < 0 || pg >= a.num_pages) {
    if (lane == 0) raise_error(a.err_word, SIMSD_EW_PAGE);
    return t;
  }
  t.row = static_cast<long long>(pg) * a.Hkv * a.page_size + (dst - pi * a.page_size);
  return t;
}

}  // namespace simsd
