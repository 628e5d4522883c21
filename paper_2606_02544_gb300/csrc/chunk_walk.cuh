// chunk_walk.cuh -- how the work of an attention call over ragged chunks is
// cut into equal runs, shared by the kernels that walk such runs.
//
// A unit is (KV head, sequence, `ub` tokens); its key tiles, of kTile rows,
// are those that any of its tokens sees.  The tiles of all units end to end
// (KV head slowest, so that CTAs work on one head's K/V at a time) are cut
// into equal runs, one per CTA.  Lengths are only known on the device, so
// every CTA sums them up itself and finds where its run starts.
#pragma once
#include "chunk_mask.cuh"

namespace simsd {

// The rows that a range of tokens sees: [lo, se) and [w0, hi), se <= w0; the
// first part (rows that stay visible through a window) is empty without SINKS.
struct Keys {
  int lo, se, w0, hi;
};
template <bool SINKS>
__device__ __forceinline__ Keys keys_of(const ChunkArgs& a, const ChunkSeq& s, int i0, int i1) {
  if (s.bad) return Keys{0, 0, 0, 0};
  const int w0 = key_lo(a, s, i0), hi = key_hi(a, s, i1 - 1);
  if (w0 >= hi) return Keys{0, 0, 0, 0};
  if constexpr (SINKS) return Keys{s.ks, min(sink_end(a, s, hi), w0), w0, hi};
  return Keys{w0, w0, w0, hi};
}

// Its tiles, counted from lo / kTile on without those between the two parts:
// tile t covers the rows from tile_row(t) on.  (0 tiles where nothing is seen.)
template <bool SINKS, int kTile>
__device__ __forceinline__ int tiles_skipped(const Keys& k) {
  return SINKS ? max(0, k.w0 / kTile - (k.se + kTile - 1) / kTile) : 0;
}
template <bool SINKS, int kTile>
__device__ __forceinline__ int tiles_of(const Keys& k) {
  return k.hi > 0 ? (k.hi + kTile - 1) / kTile - k.lo / kTile - tiles_skipped<SINKS, kTile>(k) : 0;
}

// A unit's weight in the walk: its key tiles, one where it sees none
// (somebody has to zero its rows).
template <bool SINKS, int kTile>
__device__ __forceinline__ int unit_weight(const ChunkArgs& a, const ChunkSeq& s, int ub, int j) {
  const int i0 = j * ub, i1 = min(s.C, i0 + ub);
  return max(1, tiles_of<SINKS, kTile>(keys_of<SINKS>(a, s, i0, i1)));
}

// Tiles of every sequence in `tiles` (shared, kChunkMaxSeqs ints).  Every
// thread of the block takes part.
template <bool SINKS, int kTile, int kThreads>
__device__ __forceinline__ void plan_tiles(const ChunkArgs& a, int ub, int32_t* tiles) {
  const int tid = threadIdx.x, warp = tid >> 5, lane = tid & 31;
  uint32_t err = 0;
  bool is_long = false;
  // short chunks: a thread per sequence; chunks of more than two units: a warp
  for (int b = tid; b < a.Bt; b += kThreads) {
    const ChunkSeq s = chunk_seq(a, b);
    err |= (s.bad_off ? SIMSD_EW_TOKENS : 0u) | (s.bad && s.C > 0 ? SIMSD_EW_PREFIX_LEN : 0u);
    int v = 0;
    if (s.C > 2 * ub) {
      v = -1;
      is_long = true;
    } else if (s.C > 0) {
      v = unit_weight<SINKS, kTile>(a, s, ub, 0);
      if (s.C > ub) v += unit_weight<SINKS, kTile>(a, s, ub, 1);
    }
    tiles[b] = v;
  }
  if (err && blockIdx.x == 0) raise_error(a.err_word, err);
  if (__syncthreads_or(is_long)) {
    for (int b = warp; b < a.Bt; b += kThreads / 32) {
      if (tiles[b] >= 0) continue;
      const ChunkSeq s = chunk_seq(a, b);
      const int units = (s.C + ub - 1) / ub;
      int v = 0;
      for (int j = lane; j < units; j += 32) v += unit_weight<SINKS, kTile>(a, s, ub, j);
#pragma unroll
      for (int o = 16; o > 0; o >>= 1) v += __shfl_xor_sync(0xffffffffu, v, o);
      if (lane == 0) tiles[b] = v;
    }
  }
  // The host's bound on the tiles of a call holds for offsets in order; those
  // that are not may make chunks overlap beyond it, and then nothing is done.
  // (Checked only where some are not: in plan_start, for every call, long
  // prompts came out 5 to 9% slower.)
  if (!__syncthreads_or(err & SIMSD_EW_TOKENS)) return;
  long long all = 0;
  for (int b = 0; b < a.Bt; ++b) all += tiles[b];
  __syncthreads();
  if (all * a.Hkv >= (1ll << 31))
    for (int b = tid; b < a.Bt; b += kThreads) tiles[b] = 0;
  __syncthreads();
}

__device__ __forceinline__ int warp_inclusive(int v) {
  const int lane = threadIdx.x & 31;
#pragma unroll
  for (int o = 1; o < 32; o <<= 1) {
    const int y = __shfl_up_sync(0xffffffffu, v, o);
    if (lane >= o) v += y;
  }
  return v;
}

// A place in the walk: tile t of unit (b, j) for a KV head.
struct Place {
  int b, j, kvh, t;
};

// The total (per KV head), and the place of the CTA's run start.  One warp.
template <bool SINKS, int kTile>
__device__ __forceinline__ Place plan_start(const ChunkArgs& a, int ub, int ctas, const int32_t* tiles, int& total,
                                            ChunkSeq& s) {
  const unsigned full = 0xffffffffu;
  const int lane = threadIdx.x & 31;
  int sum = 0;
  for (int b = lane; b < a.Bt; b += 32) sum += tiles[b];
#pragma unroll
  for (int o = 16; o > 0; o >>= 1) sum += __shfl_xor_sync(full, sum, o);
  total = sum;
  Place w{0, 0, 0, 0};
  const int all = sum * a.Hkv, W = (all + ctas - 1) / ctas;
  const long long R0 = static_cast<long long>(W) * blockIdx.x;
  if (R0 >= all) return w;
  w.kvh = static_cast<int>(R0) / sum;
  int at = static_cast<int>(R0) - w.kvh * sum;  // tiles before the run within the head
  for (int b0 = 0; b0 < a.Bt; b0 += 32) {
    const int v = b0 + lane < a.Bt ? tiles[b0 + lane] : 0;
    const int inc = warp_inclusive(v);
    const unsigned m = __ballot_sync(full, inc > at);
    if (m) {
      const int k = __ffs(m) - 1;
      w.b = b0 + k;
      at -= __shfl_sync(full, inc - v, k);
      break;
    }
    at -= __shfl_sync(full, inc, 31);
  }
  s = chunk_seq(a, w.b);
  for (int j0 = 0; j0 * ub < s.C; j0 += 32) {
    const int v = (j0 + lane) * ub < s.C ? unit_weight<SINKS, kTile>(a, s, ub, j0 + lane) : 0;
    const int inc = warp_inclusive(v);
    const unsigned m = __ballot_sync(full, inc > at);
    if (m) {
      const int k = __ffs(m) - 1;
      w.j = j0 + k;
      w.t = at - __shfl_sync(full, inc - v, k);
      break;
    }
    at -= __shfl_sync(full, inc, 31);
  }
  return w;
}

// The run [R0, R1) of a CTA piece by piece: from the first unit that starts in
// it to R1, then the unit cut at R0, so that both pieces of a cut unit are
// written near the end of the launch.
template <bool SINKS, int kTile>
struct Walk {
  Place start, w;
  ChunkSeq seq, s;
  int left, head, total, W, all;
  long long R0;
  bool first;

  struct Step {
    Keys keys;
    int tiles, weight, take;  // the unit's key tiles (those from w.t on are left), its weight, what the piece takes
    int slot, last;           // slot 0: the piece at the start of the run; last: of the CTA
  };

  __device__ __forceinline__ void begin(const ChunkArgs& a, int ub, int ctas, const Place& place, const ChunkSeq& sq,
                                        int sum) {
    start = w = place;
    seq = s = sq;
    total = sum;
    all = total * a.Hkv;
    W = (all + ctas - 1) / ctas;
    R0 = static_cast<long long>(W) * blockIdx.x;
    left = R0 < all ? min(W, all - static_cast<int>(R0)) : 0;
    head = 0;
    first = true;
    if (left > 0 && w.t > 0) {
      head = min(left, unit_weight<SINKS, kTile>(a, s, ub, w.j) - w.t);
      left -= head;
      first = false;
      if (left > 0) advance(a, ub);
    }
  }
  // The next piece, of unit (w.kvh, w.b, w.j) of sequence s; false: no more.
  __device__ __forceinline__ bool peek(const ChunkArgs& a, int ub, Step& p) {
    if (left == 0 && head > 0) {
      left = head;
      head = 0;
      w = start;
      s = seq;
      first = true;
    }
    if (left == 0) return false;
    const int i0 = w.j * ub;
    p.keys = keys_of<SINKS>(a, s, i0, min(s.C, i0 + ub));
    p.tiles = tiles_of<SINKS, kTile>(p.keys);
    p.weight = max(1, p.tiles);
    p.take = min(p.weight - w.t, left);
    p.slot = first ? 0 : 1;
    p.last = left == p.take && head == 0;
    return true;
  }
  __device__ __forceinline__ void pop(const ChunkArgs& a, int ub, const Step& p) {
    first = false;
    left -= p.take;
    if (left > 0) advance(a, ub);
  }
  // to the next unit that exists
  __device__ __forceinline__ void advance(const ChunkArgs& a, int ub) {
    ++w.j;
    w.t = 0;
    if (w.j * ub < s.C) return;
    w.j = 0;
    do {
      if (++w.b == a.Bt) {
        w.b = 0;
        if (++w.kvh == a.Hkv) return;
      }
      s = chunk_seq(a, w.b);
    } while (s.C == 0);
  }
};

// A unit cut by the ends of runs: its pieces are those of CTAs c0 .. c1, c0's
// in `slot`.  ntok 0: the boundary cuts no unit, or not as the first.
struct Record {
  int tok0, ntok, kvh, c0;
  int c1, slot, pad0, pad1;
};
// The record of run boundary blockIdx.x: the unit that it is the first to cut.
template <bool SINKS, int kTile>
__device__ __forceinline__ Record boundary_record(const Walk<SINKS, kTile>& k, const ChunkArgs& a, int ub) {
  Record rec{};
  if (k.R0 < k.all && k.start.t > 0) {
    const int weight = unit_weight<SINKS, kTile>(a, k.seq, ub, k.start.j);
    const int begin = static_cast<int>(k.R0) - k.start.t, c0 = begin / k.W;
    if (c0 + 1 == static_cast<int>(blockIdx.x)) {
      rec.tok0 = k.seq.start + k.start.j * ub;
      rec.ntok = min(ub, k.seq.C - k.start.j * ub);
      rec.kvh = k.start.kvh;
      rec.c0 = c0;
      rec.c1 = (begin + weight - 1) / k.W;
      rec.slot = begin != c0 * k.W ? 1 : 0;
    }
  }
  return rec;
}

}  // namespace simsd
