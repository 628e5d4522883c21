// ragged.cuh -- chunks of new tokens packed end to end: the tokens of
// sequence b are rows token_start[b] .. token_start[b+1]-1 of a [T] array.
#pragma once
#include <cstdint>

namespace simsd {

// The sequence that holds token `tok`, found by a whole warp (32 probes a
// step); -1 when no sequence holds it.  Offsets that are not in order give
// some sequence or -1, never an index outside [0, Bt).
__device__ __forceinline__ int warp_find_seq(const int32_t* __restrict__ token_start, int Bt, int tok) {
  const unsigned full = 0xffffffffu;
  const int lane = threadIdx.x & 31;
  int lo = 0, n = Bt;  // the answer, if any, is the last b in [lo, lo + n) with start[b] <= tok
  while (n > 1) {
    const int step = (n + 31) >> 5;
    const int i = lane * step;
    const bool le = i < n && token_start[lo + i] <= tok;
    const unsigned m = __ballot_sync(full, le);
    const int k = m ? 31 - __clz(m) : 0;
    lo += k * step;
    n = min(step, n - k * step);
  }
  const int s0 = token_start[lo], s1 = token_start[lo + 1];
  return s0 <= tok && tok < s1 ? lo : -1;
}

// Host and device agree on what a sequence's chunk is: rows [start, start +
// count) within [0, T); a pair of offsets outside that is an empty chunk.
struct Chunk {
  int start, count;
  bool bad;
};
__device__ __forceinline__ Chunk chunk_of(const int32_t* token_start, int b, int T) {
  Chunk c;
  const int s0 = token_start[b], s1 = token_start[b + 1];
  c.bad = s0 < 0 || s1 < s0 || s1 > T;
  c.start = c.bad ? 0 : s0;
  c.count = c.bad ? 0 : s1 - s0;
  return c;
}

}  // namespace simsd
