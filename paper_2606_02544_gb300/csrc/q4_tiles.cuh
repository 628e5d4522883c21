// q4_tiles.cuh -- tiles of a cache in 4 bits on their way to shared memory,
// shared by the kernels that read one: what the walking warp says of a tile,
// and the copies that bring its codes and scales.
#pragma once
#include <cmath>

#include "chunk_walk.cuh"
#include "ptx.cuh"
#include "q4.cuh"

namespace simsd {

constexpr int kQ4Tile = 128;  // keys per tile

enum : int {
  kFirst = 1,       // of a piece
  kLast = 2,        // of a piece
  kLastPiece = 4,   // and that the CTA's last one
  kFull = 8,        // every row sees every key
  kEmpty = 16,      // no row sees any key
  kEnd = 32,        // no tile: the end of the run
  kPart = 64,       // the piece leaves partial results,
  kSlot1 = 128,     // those of slot 1
  kBad = 256        // a page id of the piece (so far) is out of range
};
struct alignas(16) TileInfo {
  int flags, key0, ntok, tok0;
  int kvh, i0, n, C;
  int lo, se, w0, hi;  // keys that any row of the unit sees
  int ks, pad0, pad1, pad2;
};

template <int D>
struct alignas(128) Stage {
  uint8_t kc[kQ4Tile * D / 2], vc[kQ4Tile * D / 2];
  uint8_t ks[kQ4Tile * D / kQ4Group], vs[kQ4Tile * D / kQ4Group];
};

__device__ __forceinline__ void bulk_load(uint32_t dst, const void* src, uint32_t bytes, uint32_t bar) {
  asm volatile("cp.async.bulk.shared::cluster.global.mbarrier::complete_tx::bytes [%0], [%1], %2, [%3];" ::"r"(dst),
               "l"(src), "r"(bytes), "r"(bar)
               : "memory");
}

// The pieces of a run, tile by tile.  One warp; `sub`: keys per copy (a page,
// or part of one).
template <int D, bool SINKS>
struct TileWalk {
  Walk<SINKS, kQ4Tile> k;
  typename Walk<SINKS, kQ4Tile>::Step piece;
  TileInfo u;
  int ub, sub, flags, skip, tse, all_lo, all_hi, all_se, t0;
  int win_base, win;  // lane i holds the page id of page win_base + i
  const int32_t* bt;
  // this lane's copy of the tile: its first key is u.key0 + at, row off of page
  // pi (kept from tile to tile, of which each is pages, rest further: a divide
  // would be a good part of the walk's time)
  bool load;
  int at, pi, off, pages, rest;
  size_t row;  // in the pool, in rows of a head

  // Tokens of a unit, keys of a copy, and the page size that they hold for.
  __device__ __forceinline__ void sizes(int unit_tokens, int copy_keys, int P) {
    ub = unit_tokens;
    sub = copy_keys;
    at = min(static_cast<int>(threadIdx.x & 31), kQ4Tile / sub - 1) * sub;
    pages = kQ4Tile / P;
    rest = kQ4Tile - pages * P;
  }

  __device__ __forceinline__ bool next_piece(const ChunkArgs& a) {
    if (!k.peek(a, ub, piece)) return false;
    u.i0 = k.w.j * ub;
    u.tok0 = k.s.start + u.i0;
    u.ntok = min(ub, k.s.C - u.i0);
    u.kvh = k.w.kvh;
    u.lo = piece.keys.lo;
    u.se = piece.keys.se;
    u.w0 = piece.keys.w0;
    u.hi = piece.keys.hi;
    u.n = k.s.n;
    u.C = k.s.C;
    u.ks = k.s.ks;
    const bool empty = piece.tiles == 0;
    flags = (empty ? kEmpty : 0) | (piece.take < piece.weight ? kPart : 0) | (piece.slot ? kSlot1 : 0);
    // rows that every token of the unit sees
    all_lo = empty ? 0 : key_lo(a, k.s, u.i0 + u.ntok - 1);
    all_hi = empty ? 0 : key_hi(a, k.s, u.i0);
    all_se = SINKS && !empty ? sink_end(a, k.s, all_hi) : 0;
    skip = tiles_skipped<SINKS, kQ4Tile>(piece.keys);
    tse = (u.se + kQ4Tile - 1) / kQ4Tile;
    bt = a.block_table + static_cast<size_t>(k.w.b) * a.max_pages;
    t0 = u.lo / kQ4Tile + k.w.t;
    win_base = -(1 << 30);
    return true;
  }
  // Tile i of the piece: u, and the lane's copy.
  __device__ __forceinline__ void tile(const ChunkArgs& a, int i) {
    const unsigned full = 0xffffffffu;
    const int lane = threadIdx.x & 31, P = a.page_size, t = t0 + i;
    const bool empty = flags & kEmpty;
    const int before = u.key0;
    u.key0 = (t + (SINKS && t >= tse ? skip : 0)) * kQ4Tile;
    const bool all = !empty && ((u.key0 >= all_lo && u.key0 + kQ4Tile <= all_hi) ||
                                (SINKS && u.key0 >= u.ks && u.key0 + kQ4Tile <= all_se));
    // copy s of the tile is lane s's
    const int key = u.key0 + at;
    if (i == 0 || u.key0 != before + kQ4Tile) {
      pi = key / P;
      off = key - pi * P;
    } else {
      pi += pages;
      off += rest;
      if (off >= P) {
        off -= P;
        ++pi;
      }
    }
    if (__any_sync(full, static_cast<unsigned>(pi - win_base) >= 32u)) {
      win_base = __shfl_sync(full, pi, 0);
      win = win_base + lane < a.max_pages ? bt[win_base + lane] : -1;
    }
    const int pg = __shfl_sync(full, win, (pi - win_base) & 31);
    load = !empty && lane * sub < kQ4Tile && key + sub > u.lo && key < u.hi && (!SINKS || key < u.se || key + sub > u.w0);
    const bool wrong = load && (pg < 0 || pg >= a.num_pages);
    load = load && !wrong;
    if (__any_sync(full, wrong)) {
      if (lane == 0) raise_error(a.err_word, SIMSD_EW_PAGE);
      flags |= kBad;
    }
    row = (static_cast<size_t>(pg) * a.Hkv + u.kvh) * P + off;
    u.flags = flags | (i == 0 ? kFirst : 0) | (i + 1 == piece.take ? kLast | (piece.last ? kLastPiece : 0) : 0) | (all ? kFull : 0);
  }
  // Bytes of all lanes' copies of K, or of V; then the copies themselves.
  __device__ __forceinline__ uint32_t bytes() const {
    return __popc(__ballot_sync(0xffffffffu, load)) * static_cast<uint32_t>(sub * (D / 2 + D / kQ4Group));
  }
  __device__ __forceinline__ void copy_k(const simsd_q4_cache& c, Stage<D>& s, uint32_t bar) const {
    copy(c.k_codes, c.k_scales, s.kc, s.ks, bar);
  }
  __device__ __forceinline__ void copy_v(const simsd_q4_cache& c, Stage<D>& s, uint32_t bar) const {
    copy(c.v_codes, c.v_scales, s.vc, s.vs, bar);
  }
  __device__ __forceinline__ void copy(const void* codes, const void* scales, uint8_t* to_codes, uint8_t* to_scales,
                                       uint32_t bar) const {
    if (!load) return;
    const int at = (threadIdx.x & 31) * sub;
    bulk_load(smem_u32(to_codes + at * (D / 2)), static_cast<const uint8_t*>(codes) + row * (D / 2),
              static_cast<uint32_t>(sub * (D / 2)), bar);
    bulk_load(smem_u32(to_scales + at * (D / kQ4Group)), static_cast<const uint8_t*>(scales) + row * (D / kQ4Group),
              static_cast<uint32_t>(sub * (D / kQ4Group)), bar);
  }
};

// What turns products of codes' values into scores in log2 units, m 2^e with m
// in [1, 2]: the softmax scale, the keys' unit and log2(e).
struct ScoreScale {
  float m;
  int e;
};
inline ScoreScale score_scale(float softmax_scale, float k_unit) {
  int e;
  const double m = std::frexp(static_cast<double>(softmax_scale) * k_unit * 1.4426950408889634, &e);
  return ScoreScale{static_cast<float>(2.0 * m), e - 1};
}
// A power of two, `down`, that brings a row's largest component to [1, 4), from
// that component's bf16 bits without the sign, and the factor of the row's
// scores, which undoes it.  The factor stays among fp32's normal numbers: as 0
// (a row of zeros has the largest power, and a unit may be 2^-64) it would turn
// hidden keys' -inf into NaN, as inf scores of 0.  Nothing is lost by it: below
// 2^-126 all scores of a row are 0 in fp32's sense (under 2^-104), above 2^126
// two that differ do so by more than 2^90.
__device__ __forceinline__ float q_factor(uint32_t top, const ScoreScale& s, float& down) {
  const int ex = min(max(static_cast<int>(top >> 7), 1), 253);  // 2^(ex - 127) <= the largest < 2^(ex - 126)
  down = __uint_as_float(static_cast<uint32_t>(254 - ex) << 23);
  return __uint_as_float(static_cast<uint32_t>(min(max(ex + s.e, 1), 253)) << 23) * s.m;
}
// Probabilities in fp16 have 2^-24 as their smallest number: with a weight of 1
// for the largest, keys 2^25 times smaller would count in the sum and not in
// the output (2^18 of them at 2^-25.5, 0.5% of a row).  So a reference is set
// kHeadroom below the maximum, for which the largest weighs 2^7, and is left
// until a score is kMoveAbove above it: 2^15, below fp16's 65504.
constexpr float kHeadroom = 7.0f, kMoveAbove = 15.0f;  // log2 units
__device__ __forceinline__ uint32_t pack_f16x2(float lo, float hi) {
  uint32_t r;
  asm("cvt.rn.f16x2.f32 %0, %1, %2;" : "=r"(r) : "f"(hi), "f"(lo));
  return r;
}

}  // namespace simsd
