// chunk_attention_tc.cu -- bf16 attention of a chunk of new tokens over the
// paged cache on the sm_103a tensor cores (Sec. 3.3: prompt and earlier
// blocks are read from the KV cache; here they are also what fills it).
//
// Mathematics.  Row (token, query head): o = sum_j e^(s_j - M) v_j / sum_j
// e^(s_j - M), s_j = scale q.k_j over the rows lo <= j < hi of chunk_mask.cuh,
// in one pass over the keys with a running reference maximum and sum (fp32;
// the reference moves only when a score exceeds it by 2^8, so O is rarely
// rescaled).  Probabilities are rounded to bf16 for the tensor cores, their
// sum is not; O is accumulated in fp32 and rounded once.
//
// A unit is (sequence, KV head, up to 256 query rows): the g = Hq / Hkv
// heads of floor(128 / g) tokens make one row block, a unit holds two, so a
// K/V tile of 128 keys crosses L2 once for both and feeds four MMAs: S_A =
// Q_A K^T, S_B = Q_B K^T, O_A += P_A V, O_B += P_B V.
//
// Work.  The key tiles of all units end to end (KV head slowest, so that
// CTAs work on one head's K/V at a time) are cut into equal runs, one per
// CTA (one CTA per SM); lengths are only known on the device, so every CTA
// sums them up itself and finds where its run starts.  A unit cut by a
// run's end leaves partial (O, m, l), which a second launch merges.  Long
// prompts (compute-bound) and single tokens over long caches (memory-bound)
// so load every SM alike.
//
// Warp roles (384 threads): warps 0-3 softmax of row block A, 4-7 of B
// (thread i of a block owns query row i = TMEM lane i); warp 8 TMA producer
// of Q, K and V; warps 9 and 10 issue the MMAs of block A and of block B;
// warp 11 walks the run and passes unit by unit to the others through shared
// memory.  An MMA warp keeps the order PV(i) S(i+1) of its block, S as soon
// as PV (whose P lies in the same columns) is done; the two warps are not
// tied to each other and settle in antiphase, one block's products under the
// other's softmax (about 2530 cycles for a tile of both; made to take turns,
// 3150).  A softmax warp begins with the probabilities of the first half of
// the keys before the tile's maximum is known, against the old reference,
// and starts again where the reference has to move.
//
// Bound: the softmax (exponentials, conversions and maxima of 2 x 128 x 128
// scores: about 2000 of the 2530 cycles, the two products 1024) for prompts,
// HBM for single tokens.  Measured, 32 heads on 8, d 128: 8192 tokens of one
// prompt 434 us (1.3 PFLOP/s of the two products, causal), 2048 after 32768
// 765 us (1.5); 64 single tokens over 2048 to 8192 rows 214 us (6.3 TB/s); 8
// over 512 to 1024, 16 heads, 20 us, most of it one CTA's chain from the
// tokens' offsets to its first tile and the second launch.
// TMEM (512 columns): S_A [0,128), S_B [128,256), O_A [256,384), O_B
// [384,512); P (bf16) overwrites the first 64 columns of its S.
// Shared memory: Q of both blocks, a ring of 128-key K tiles and one of V.
//
// Every mbarrier wait is bounded; after one expires the CTA raises
// SIMSD_EW_TIMEOUT, every role leaves its loops, drains its copies and MMAs
// and frees TMEM.
#include <cuda.h>
#include <cuda_bf16.h>
#include <cuda_runtime.h>

#include <algorithm>
#include <mutex>

#include "chunk_mask.cuh"
#include "common.cuh"
#include "kernels.h"
#include "ptx_chunk.cuh"

namespace simsd {
namespace {

constexpr int kTile = 128;     // keys per tile
constexpr int kSub = 64;       // keys per copy (a page, or part of one)
constexpr int kRows = 128;     // query rows per row block (MMA M)
constexpr int kThreads = 384;
constexpr int kWarpProducer = 8, kWarpMma = 9, kWarpWalk = 11;  // (warp 10: the MMAs of block B)
constexpr uint32_t kTmemCols = 512;
constexpr uint32_t kColS = 0, kColO = 256;  // + 128 per row block
constexpr int kHalfBytes = kTile * 128;     // 128 rows x 64 bf16
constexpr int kQueue = 4;                   // units passed on but not taken by all roles
constexpr int kQueueReaders = 11;           // 8 softmax warps, the producer, 2 MMA warps
constexpr int kFlags = 8;                   // more than the pieces that tiles in the rings can span
constexpr float kRescaleThreshold = 8.0f;   // log2 units
constexpr float kLn2 = 0.6931471805599453f;

struct ChunkTcParams {
  ChunkArgs a;
  int g, tb;          // heads per KV head, tokens per row block
  int ctas;           // grid size
  int wide_out;       // the output is 32-byte aligned
  float scale_log2;
};

// Key tiles [t0, t0 + tiles) of a unit, or of the CTA's piece of it.
struct alignas(16) Piece {
  int tok0, ntok;      // first token of the unit in the chunk array, tokens of it
  int kvh, b;
  int t0, tiles;       // this piece's key tiles; tiles 0: the rows are zero; -1: no more pieces
  int lo, hi;          // keys that the unit's tokens see
  int n, C, ks, i0;    // the sequence (chunk_mask.cuh) and the unit's first token in it
  int part, slot;      // writes partial results (slot 0: the piece at the start of the run)
  int last, flag;      // the CTA's last piece; its entry in `bad`
};

template <int D>
struct alignas(1024) SmemChunk {
  static constexpr int kHalves = D / 64;
  static constexpr int kTileBytes = kHalves * kHalfBytes;  // one K or V tile
  // K and V have rings of their own: the producer and the MMA warps wait for
  // every use of a slot in turn, so they never read a parity a phase early (the
  // softmax warps wait for V only where they zero rows, and after the tile's S)
  static constexpr int kStagesK = D == 128 ? 3 : 5, kStagesV = D == 128 ? 2 : 5;
  static constexpr int kStages = kStagesK + kStagesV;
  uint8_t ring[kStages][kTileBytes];  // K, then V
  uint8_t q[2][kTileBytes];
  uint64_t bar_full[kStages], bar_free[kStages];
  uint64_t bar_q[2], bar_qfree[2];
  uint64_t bar_s[2], bar_p[2][2], bar_pv[2], bar_ofree[2];
  uint64_t bar_msg[kQueue], bar_msgfree[kQueue];
  uint64_t bar_drain[2];
  Piece queue[kQueue];
  int bad[kFlags];     // a page id of the piece is out of range (written by the producer)
  uint32_t tmem_base;
  int abort_flag;
};
template <int D>
constexpr size_t smem_bytes() {
  return sizeof(SmemChunk<D>) + 1024;
}
static_assert(smem_bytes<128>() <= 232448 && smem_bytes<64>() <= 232448, "one CTA per SM");
static_assert(SmemChunk<128>::kStages * SmemChunk<128>::kTileBytes >= kChunkMaxSeqs * 4 &&
                  SmemChunk<64>::kStages * SmemChunk<64>::kTileBytes >= kChunkMaxSeqs * 4,
              "the ring holds the tile counts of all sequences while runs are planned");

template <int D>
__device__ __forceinline__ void signal_abort(SmemChunk<D>& sm, int32_t* err_word) {
  raise_error(err_word, SIMSD_EW_TIMEOUT);
  *reinterpret_cast<volatile int*>(&sm.abort_flag) = 1;
}

// The keys that unit j of a sequence sees, and its weight in the walk: its
// key tiles, one where it sees none (somebody has to zero its rows).
struct Range {
  int lo, hi;
};
__device__ __forceinline__ Range unit_range(const ChunkTcParams& p, const ChunkSeq& s, int j) {
  if (s.bad) return Range{0, 0};
  const int ub = 2 * p.tb, i0 = j * ub, i1 = min(s.C, i0 + ub);
  const int lo = key_lo(p.a, s, i0), hi = key_hi(p.a, s, i1 - 1);
  return lo < hi ? Range{lo, hi} : Range{0, 0};
}
__device__ __forceinline__ int range_tiles(const Range& r) {
  return r.hi > 0 ? (r.hi + kTile - 1) / kTile - r.lo / kTile : 0;
}
__device__ __forceinline__ int unit_weight(const ChunkTcParams& p, const ChunkSeq& s, int j) {
  return max(1, range_tiles(unit_range(p, s, j)));
}

// Tiles of every sequence in `tiles` (shared, kChunkMaxSeqs ints).  Every
// thread of the block takes part.
__device__ __forceinline__ void plan_tiles(const ChunkTcParams& p, int32_t* tiles) {
  const int tid = threadIdx.x, warp = tid >> 5, lane = tid & 31;
  const int ub = 2 * p.tb;
  uint32_t err = 0;
  bool is_long = false;
  // short chunks: a thread per sequence; chunks of more than two units: a warp
  for (int b = tid; b < p.a.Bt; b += kThreads) {
    const ChunkSeq s = chunk_seq(p.a, b);
    err |= (s.bad_off ? SIMSD_EW_TOKENS : 0u) | (s.bad && s.C > 0 ? SIMSD_EW_PREFIX_LEN : 0u);
    int v = 0;
    if (s.C > 2 * ub) {
      v = -1;
      is_long = true;
    } else if (s.C > 0) {
      v = unit_weight(p, s, 0);
      if (s.C > ub) v += unit_weight(p, s, 1);
    }
    tiles[b] = v;
  }
  if (err && blockIdx.x == 0) raise_error(p.a.err_word, err);
  if (__syncthreads_or(is_long)) {
    for (int b = warp; b < p.a.Bt; b += kThreads / 32) {
      if (tiles[b] >= 0) continue;
      const ChunkSeq s = chunk_seq(p.a, b);
      const int units = (s.C + ub - 1) / ub;
      int v = 0;
      for (int j = lane; j < units; j += 32) v += unit_weight(p, s, j);
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
  for (int b = 0; b < p.a.Bt; ++b) all += tiles[b];
  __syncthreads();
  if (all * p.a.Hkv >= (1ll << 31))
    for (int b = tid; b < p.a.Bt; b += kThreads) tiles[b] = 0;
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
__device__ __forceinline__ Place plan_start(const ChunkTcParams& p, const int32_t* tiles, int& total, ChunkSeq& s) {
  const unsigned full = 0xffffffffu;
  const int lane = threadIdx.x & 31, ub = 2 * p.tb;
  int sum = 0;
  for (int b = lane; b < p.a.Bt; b += 32) sum += tiles[b];
#pragma unroll
  for (int o = 16; o > 0; o >>= 1) sum += __shfl_xor_sync(full, sum, o);
  total = sum;
  Place w{0, 0, 0, 0};
  const int all = sum * p.a.Hkv, W = (all + p.ctas - 1) / p.ctas;
  const long long R0 = static_cast<long long>(W) * blockIdx.x;
  if (R0 >= all) return w;
  w.kvh = static_cast<int>(R0) / sum;
  int at = static_cast<int>(R0) - w.kvh * sum;  // tiles before the run within the head
  for (int b0 = 0; b0 < p.a.Bt; b0 += 32) {
    const int v = b0 + lane < p.a.Bt ? tiles[b0 + lane] : 0;
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
  s = chunk_seq(p.a, w.b);
  for (int j0 = 0; j0 * ub < s.C; j0 += 32) {
    const int v = (j0 + lane) * ub < s.C ? unit_weight(p, s, j0 + lane) : 0;
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

// Partial results: O (unnormalised, fp32) as [ctas * 4 entries][D / 4][128
// rows] vectors of four (a warp's 32 rows are adjacent, so they are written
// and read in whole lines), (m, l) [entries][128], entry (cta * 2 + slot) * 2
// + block, m in log2 units, l = -1 where a page id of the piece is out of
// range (the row is zero then); then one record per run boundary.
struct Record {
  int tok0, ntok, kvh, c0;  // ntok 0: the boundary cuts no unit, or not as the first
  int c1, slot, pad0, pad1;
};
template <int D>
__device__ __forceinline__ float4* partial_o(const ChunkTcParams& p, int entry, int col4, int row) {
  return static_cast<float4*>(p.a.workspace) + (static_cast<size_t>(entry) * (D / 4) + col4) * kRows + row;
}
template <int D>
__device__ __forceinline__ float2* partial_ml(const ChunkTcParams& p, int entry, int row) {
  return reinterpret_cast<float2*>(static_cast<float4*>(p.a.workspace) +
                                   static_cast<size_t>(p.ctas) * 4 * (D / 4) * kRows) +
         static_cast<size_t>(entry) * kRows + row;
}
template <int D>
__device__ __forceinline__ Record* records(const ChunkTcParams& p) {
  return reinterpret_cast<Record*>(static_cast<float*>(p.a.workspace) +
                                   static_cast<size_t>(p.ctas) * 4 * kRows * (D + 2));
}

__device__ __forceinline__ void st_global_256(void* p, const uint32_t (&v)[8]) {
  asm volatile("st.global.v8.b32 [%0], {%1,%2,%3,%4,%5,%6,%7,%8};" ::"l"(p), "r"(v[0]), "r"(v[1]), "r"(v[2]),
               "r"(v[3]), "r"(v[4]), "r"(v[5]), "r"(v[6]), "r"(v[7])
               : "memory");
}

// The next message of the unit queue, copied to the registers of a warp;
// false when a wait expired.
template <int D>
__device__ __forceinline__ bool next_piece(SmemChunk<D>& sm, uint32_t& at, Piece& u) {
  volatile int* abort_flag = &sm.abort_flag;
  const uint32_t st = at % kQueue, par = (at / kQueue) & 1;
  if (!mbar_wait_warp(smem_u32(&sm.bar_msg[st]), par, abort_flag)) return false;
  const int4* src = reinterpret_cast<const int4*>(&sm.queue[st]);
  const int4 a = src[0], b = src[1], c = src[2], d = src[3];
  u.tok0 = a.x;
  u.ntok = a.y;
  u.kvh = a.z;
  u.b = a.w;
  u.t0 = b.x;
  u.tiles = b.y;
  u.lo = b.z;
  u.hi = b.w;
  u.n = c.x;
  u.C = c.y;
  u.ks = c.z;
  u.i0 = c.w;
  u.part = d.x;
  u.slot = d.y;
  u.last = d.z;
  u.flag = d.w;
  __syncwarp();
  if ((threadIdx.x & 31) == 0) mbar_arrive(smem_u32(&sm.bar_msgfree[st]));
  ++at;
  return true;
}

template <int D>
__global__ void __launch_bounds__(kThreads, 1)
    chunk_tc_kernel(const __grid_constant__ CUtensorMap tm_q, const __grid_constant__ CUtensorMap tm_k,
                    const __grid_constant__ CUtensorMap tm_v, const __grid_constant__ ChunkTcParams p) {
  using Smem = SmemChunk<D>;
  constexpr int kHalves = Smem::kHalves, kStages = Smem::kStages, kStagesK = Smem::kStagesK, kStagesV = Smem::kStagesV;
  extern __shared__ uint8_t smem_raw[];
  Smem& sm = *reinterpret_cast<Smem*>((reinterpret_cast<uintptr_t>(smem_raw) + 1023) & ~static_cast<uintptr_t>(1023));
  volatile int* abort_flag = &sm.abort_flag;
  const int tid = threadIdx.x, warp = tid >> 5, lane = tid & 31;

  if (tid == 0) {
    sm.abort_flag = 0;
    for (int s = 0; s < kStages; ++s) {
      mbar_init(smem_u32(&sm.bar_full[s]), 1);
      mbar_init(smem_u32(&sm.bar_free[s]), 2);  // one commit per row block
    }
    for (int x = 0; x < 2; ++x) {
      mbar_init(smem_u32(&sm.bar_q[x]), 1);
      mbar_init(smem_u32(&sm.bar_qfree[x]), 1);
      mbar_init(smem_u32(&sm.bar_s[x]), 1);
      mbar_init(smem_u32(&sm.bar_p[x][0]), 4);
      mbar_init(smem_u32(&sm.bar_p[x][1]), 4);
      mbar_init(smem_u32(&sm.bar_pv[x]), 1);
      mbar_init(smem_u32(&sm.bar_ofree[x]), 4);
    }
    for (int s = 0; s < kQueue; ++s) {
      mbar_init(smem_u32(&sm.bar_msg[s]), 1);
      mbar_init(smem_u32(&sm.bar_msgfree[s]), kQueueReaders);
    }
    mbar_init(smem_u32(&sm.bar_drain[0]), 1);
    mbar_init(smem_u32(&sm.bar_drain[1]), 1);
    fence_mbar_init();
  }
  if (warp == kWarpMma) {
    tmem_alloc(smem_u32(&sm.tmem_base), kTmemCols);
    tmem_relinquish();
  }
  if (warp == kWarpProducer && lane == 0) {
    tma_prefetch_desc(&tm_q);
    tma_prefetch_desc(&tm_k);
    tma_prefetch_desc(&tm_v);
  }
  pdl_wait();
  int32_t* tiles = reinterpret_cast<int32_t*>(sm.ring[0]);
  plan_tiles(p, tiles);
  Place start{0, 0, 0, 0};
  int total = 0;
  ChunkSeq seq{};
  if (warp == kWarpWalk) start = plan_start(p, tiles, total, seq);
  fence_proxy_async_smem();  // the ring was written here and is filled by TMA next
  tc_fence_before();
  __syncthreads();
  tc_fence_after();
  const uint32_t tmem = sm.tmem_base;

  // register split: 2 x 128 x 208 + 128 x 88 = 64,512 = the launch's 384 x 168
  if (warp >= 8) {
    asm volatile("setmaxnreg.dec.sync.aligned.u32 88;");
    if (warp == kWarpWalk) {
      // ---------------------------------------------------------------- walk
      // the run [R0, R1): from the first unit that starts in it to R1, then
      // the unit cut at R0, so that both pieces of a cut unit are written
      // near the end of the launch
      const int all = total * p.a.Hkv, W = (all + p.ctas - 1) / p.ctas;
      const long long R0 = static_cast<long long>(W) * blockIdx.x;
      int left = R0 < all ? min(W, all - static_cast<int>(R0)) : 0;
      Place w = start;
      ChunkSeq s = seq;
      int head = 0;
      bool first = true;
      auto advance = [&]() {
        // to the next unit that exists
        ++w.j;
        w.t = 0;
        if (w.j * 2 * p.tb < s.C) return;
        w.j = 0;
        do {
          if (++w.b == p.a.Bt) {
            w.b = 0;
            if (++w.kvh == p.a.Hkv) return;
          }
          s = chunk_seq(p.a, w.b);
        } while (s.C == 0);
      };
      if (left > 0 && w.t > 0) {
        head = min(left, unit_weight(p, s, w.j) - w.t);
        left -= head;
        first = false;
        if (left > 0) advance();
      }
      uint32_t at = 0;
      bool ok = true;
      for (;;) {
        if (left == 0 && head > 0) {
          left = head;
          head = 0;
          w = start;
          s = seq;
          first = true;
        }
        Piece u;
        u.tiles = -1;
        if (left > 0) {
          const Range r = unit_range(p, s, w.j);
          const int n = range_tiles(r), weight = max(1, n), take = min(weight - w.t, left);
          u.i0 = w.j * 2 * p.tb;
          u.tok0 = s.start + u.i0;
          u.ntok = min(2 * p.tb, s.C - u.i0);
          u.kvh = w.kvh;
          u.b = w.b;
          u.t0 = r.lo / kTile + w.t;
          u.tiles = n == 0 ? 0 : take;
          u.lo = r.lo;
          u.hi = r.hi;
          u.n = s.n;
          u.C = s.C;
          u.ks = s.ks;
          u.part = take < weight;
          u.slot = first ? 0 : 1;
          first = false;
          left -= take;
          u.last = left == 0 && head == 0;
          u.flag = at % kFlags;
          if (left > 0) advance();
        }
        const uint32_t st = at % kQueue, use = at / kQueue;
        if (use > 0) ok = mbar_wait_warp(smem_u32(&sm.bar_msgfree[st]), (use - 1) & 1, abort_flag);
        if (!ok) break;
        if (lane == 0) {
          sm.queue[st] = u;
          mbar_arrive(smem_u32(&sm.bar_msg[st]));
        }
        ++at;
        if (u.tiles < 0) break;
      }
      if (!ok && lane == 0) signal_abort(sm, p.a.err_word);
      // the record of run boundary blockIdx.x: the unit that it is the first to cut
      if (lane == 0 && blockIdx.x > 0) {
        Record rec{};
        if (R0 < all && start.t > 0) {
          const int weight = unit_weight(p, seq, start.j), begin = static_cast<int>(R0) - start.t, c0 = begin / W;
          if (c0 + 1 == static_cast<int>(blockIdx.x)) {
            rec.tok0 = seq.start + start.j * 2 * p.tb;
            rec.ntok = min(2 * p.tb, seq.C - start.j * 2 * p.tb);
            rec.kvh = start.kvh;
            rec.c0 = c0;
            rec.c1 = (begin + weight - 1) / W;
            rec.slot = begin != c0 * W ? 1 : 0;
          }
        }
        records<D>(p)[blockIdx.x] = rec;
      }
    } else if (warp == kWarpProducer) {
      // ------------------------------------------------------------ producer
      uint32_t at = 0, jq[2] = {0, 0};
      uint32_t slot[2] = {0, 0}, par[2] = {0, 0}, used[2] = {0, 0};  // K, V: next slot, its parity, slots filled
      bool ok = true;
      Piece u;
      while (ok && (ok = next_piece<D>(sm, at, u)) && u.tiles >= 0) {
        if (u.tiles == 0) continue;
        const int nblk = u.ntok > p.tb ? 2 : 1;
        if (lane == 0) {
#pragma unroll
          for (int x = 0; x < 2; ++x) {
            if (x >= nblk || !ok) continue;
            if (jq[x] > 0 && !mbar_wait(smem_u32(&sm.bar_qfree[x]), (jq[x] - 1) & 1, abort_flag)) {
              ok = false;
              continue;
            }
            const uint32_t bq = smem_u32(&sm.bar_q[x]);
            mbar_arrive_expect_tx(bq, static_cast<uint32_t>(kHalves * p.g * p.tb) * 128u);
#pragma unroll
            for (int hf = 0; hf < kHalves; ++hf)
              tma_load_3d(smem_u32(sm.q[x]) + hf * kHalfBytes, &tm_q, bq, 64 * hf, u.kvh * p.g, u.tok0 + x * p.tb);
            ++jq[x];
          }
        }
        ok = __shfl_sync(0xffffffffu, ok, 0);
        if (!ok) break;
        const int32_t* bt = p.a.block_table + static_cast<size_t>(u.b) * p.a.max_pages;
        const int P = p.a.page_size, sub = min(P, kSub);
        int win_base = -(1 << 30), win = -1;  // lane i holds the page id of page win_base + i
        bool bad = false;
        for (int t = u.t0; ok && t < u.t0 + u.tiles; ++t) {
          const int key0 = t * kTile, valid = min(kTile, u.hi - key0);
          const int nsub = (valid + sub - 1) / sub;
          const int pi0 = key0 / P, pi1 = (key0 + valid - 1) / P;  // at most 16 pages a tile
          if (pi0 < win_base || pi1 >= win_base + 32) {
            win_base = pi0;
            const int pi = win_base + lane;
            win = pi < p.a.max_pages ? bt[pi] : -1;
          }
          // lane s issues the copies of sub-tile s
          const int key = key0 + min(lane, nsub - 1) * sub, pi = key / P;
          int pg = __shfl_sync(0xffffffffu, win, (pi - win_base) & 31);
          // a page id out of range is replaced by page 0, and the softmax
          // warps, which see this flag no later than the S of this tile, zero
          // the piece's rows (hidden keys before the first need no page)
          const bool wrong = (pg < 0 || pg >= p.a.num_pages) && key + sub > u.lo;
          if (pg < 0 || pg >= p.a.num_pages) pg = 0;
          bad |= __any_sync(0xffffffffu, wrong);
          if (lane == 0 && (t == u.t0 || bad)) {
            if (bad) raise_error(p.a.err_word, SIMSD_EW_PAGE);
            *reinterpret_cast<volatile int*>(&sm.bad[u.flag]) = bad;
          }
          const int row = (pg * p.a.Hkv + u.kvh) * P + (key - pi * P);
#pragma unroll
          for (int kv = 0; kv < 2; ++kv) {
            const uint32_t slots = kv == 0 ? kStagesK : kStagesV, st = (kv == 0 ? 0 : kStagesK) + slot[kv];
            if (lane == 0 && ok && used[kv] >= slots && !mbar_wait(smem_u32(&sm.bar_free[st]), par[kv] ^ 1, abort_flag))
              ok = false;
            ok = __shfl_sync(0xffffffffu, ok, 0);
            if (!ok) break;
            const uint32_t bar = smem_u32(&sm.bar_full[st]);
            if (lane == 0) mbar_arrive_expect_tx(bar, static_cast<uint32_t>(nsub * kHalves * sub) * 128u);
            __syncwarp();
            if (lane < nsub) {
              const uint32_t dst = smem_u32(sm.ring[st]) + static_cast<uint32_t>(lane * sub) * 128u;
#pragma unroll
              for (int hf = 0; hf < kHalves; ++hf)
                tma_load_2d(dst + hf * kHalfBytes, kv == 0 ? &tm_k : &tm_v, bar, 64 * hf, row);
            }
            ++used[kv];
            if (++slot[kv] == slots) {
              slot[kv] = 0;
              par[kv] ^= 1;
            }
          }
        }
      }
      if (!ok && lane == 0) signal_abort(sm, p.a.err_word);
      // every issued load must have landed before the CTA may exit
      if (lane == 0) {
#pragma unroll
        for (int kv = 0; kv < 2; ++kv) {
          const uint32_t slots = kv == 0 ? kStagesK : kStagesV, slot0 = kv == 0 ? 0 : kStagesK;
          for (uint32_t it = used[kv] > slots ? used[kv] - slots : 0; it < used[kv]; ++it)
            mbar_wait(smem_u32(&sm.bar_full[slot0 + it % slots]), (it / slots) & 1, nullptr);
        }
        for (int x = 0; x < 2; ++x)
          if (jq[x] > 0) mbar_wait(smem_u32(&sm.bar_q[x]), (jq[x] - 1) & 1, nullptr);
      }
      __syncwarp();
    } else {
      // ---------------------------------------------------------- MMA issuers
      // One warp per row block, in the order S(0) PV(0) S(1) PV(1) ...: S is
      // issued once the PV before it (whose P lies in the same columns) is
      // done.  The warp stays converged (every lane waits) and one lane
      // issues, from descriptors whose low halves are one addition away from
      // a tile's base: an MMA takes 64 cycles and must not take more to issue.
      const int x = warp - kWarpMma;
      constexpr uint32_t kIdescQK = idesc_bf16_f32(kRows, kTile, 0, 0);
      constexpr uint32_t kIdescPV = idesc_bf16_f32(kRows, D, 0, 1);
      const uint64_t dq = sdesc_sw128(smem_u32(sm.q[x]), 16, 1024), dk = sdesc_sw128(smem_u32(sm.ring[0]), 16, 1024),
                     dv = sdesc_sw128(smem_u32(sm.ring[kStagesK]), kHalfBytes, 1024);
      const uint32_t q_lo = static_cast<uint32_t>(dq), k_lo = static_cast<uint32_t>(dk), v_lo = static_cast<uint32_t>(dv);
      const uint32_t k_hi = static_cast<uint32_t>(dk >> 32), v_hi = static_cast<uint32_t>(dv >> 32);
      constexpr uint32_t kTileStep = Smem::kTileBytes >> 4;
      const uint32_t scol = tmem + kColS + 128u * x, ocol = tmem + kColO + 128u * x;
      const bool leader = elect_one();
      uint32_t c = 0, ju = 0;   // tiles and units this block has worked on
      uint32_t ks = 0, kp = 0;  // ring slot and parity of the next K tile
      uint32_t vs = 0, vp = 0;  // of the next V tile
      uint32_t at = 0;
      auto wait = [&](uint64_t& bar, uint32_t parity) { return mbar_wait_poll(smem_u32(&bar), parity, abort_flag); };
      auto step_k = [&]() {
        if (++ks == kStagesK) {
          ks = 0;
          kp ^= 1;
        }
      };
      auto step_v = [&]() {
        if (++vs == kStagesV) {
          vs = 0;
          vp ^= 1;
        }
      };
      // S for the K tile in slot ks; `qdone`: Q has no further reader
      auto issue_s = [&](bool qdone) -> bool {
        if (!wait(sm.bar_full[ks], kp)) return false;
        if (c > 0 && !wait(sm.bar_pv[x], (c - 1) & 1)) return false;
        __syncwarp();
        const uint32_t b = k_lo + ks * kTileStep;
        if (leader) {
          tc_fence_after();
#pragma unroll
          for (int kk = 0; kk < D / 16; ++kk) {
            const uint32_t off = ((kk >> 2) * kHalfBytes + (kk & 3) * 32) >> 4;
            tc_mma_ss_lh(scol, q_lo + off, k_hi, b + off, k_hi, kIdescQK, kk > 0);
          }
          tc_commit(smem_u32(&sm.bar_s[x]));
          tc_commit(smem_u32(&sm.bar_free[ks]));
          if (qdone) tc_commit(smem_u32(&sm.bar_qfree[x]));
        }
        __syncwarp();
        step_k();
        return true;
      };
      Piece u;
      bool ok = true;
      while (ok && (ok = next_piece<D>(sm, at, u)) && u.tiles >= 0) {
        const int n = u.tiles;
        if (n == 0) continue;
        if (x == 1 && u.ntok <= p.tb) {
          // a unit of few tokens has no second row block: its tiles are only
          // passed on (each tile's release counts both blocks)
          for (int i = 0; ok && i < n; ++i) {
            ok = wait(sm.bar_full[ks], kp);
            if (ok && leader) tc_commit(smem_u32(&sm.bar_free[ks]));
            step_k();
            ok = ok && wait(sm.bar_full[kStagesK + vs], vp);
            if (ok && leader) tc_commit(smem_u32(&sm.bar_free[kStagesK + vs]));
            step_v();
          }
          continue;
        }
        ok = wait(sm.bar_q[x], ju & 1);
        ok = ok && issue_s(n == 1);
        for (int i = 0; ok && i < n; ++i) {
          ok = wait(sm.bar_full[kStagesK + vs], vp);
          // the unit's first PV overwrites O: the epilogue of the unit before has read it
          if (ok && i == 0 && ju > 0) ok = wait(sm.bar_ofree[x], (ju - 1) & 1);
          const uint32_t b = v_lo + vs * kTileStep;
#pragma unroll
          for (int hp = 0; hp < 2; ++hp) {
            ok = ok && wait(sm.bar_p[x][hp], c & 1);
            __syncwarp();
            if (ok && leader) {
              tc_fence_after();
#pragma unroll
              for (int kk = 4 * hp; kk < 4 * hp + 4; ++kk)
                tc_mma_ts_lh(ocol, scol + 8 * kk, b + kk * 128, v_hi, kIdescPV, (i == 0 && kk == 0) ? 0u : 1u);
              if (hp == 1) {
                tc_commit(smem_u32(&sm.bar_pv[x]));
                tc_commit(smem_u32(&sm.bar_free[kStagesK + vs]));
              }
            }
            __syncwarp();
          }
          if (!ok) break;
          ++c;
          step_v();
          if (i + 1 < n) ok = issue_s(i + 2 == n);
        }
        ++ju;
      }
      if (!ok && lane == 0) signal_abort(sm, p.a.err_word);
      if (leader) {
        tc_commit(smem_u32(&sm.bar_drain[x]));
        mbar_wait(smem_u32(&sm.bar_drain[x]), 0, nullptr);
      }
      __syncwarp();
    }
  } else {
    asm volatile("setmaxnreg.inc.sync.aligned.u32 208;");
    // -------------------------------------------------------------- softmax
    const int x = warp >> 2;
    const int row = tid & (kRows - 1);
    const int tl = row / p.g, hl = row - tl * p.g;
    const uint32_t lane_tmem = tmem + (static_cast<uint32_t>((warp & 3) * 32) << 16);
    const uint32_t s_tmem = lane_tmem + kColS + 128u * x, o_tmem = lane_tmem + kColO + 128u * x;
    uint32_t g = 0, c = 0, at = 0;
    bool ok = true;
    Piece u;
    while ((ok = ok && next_piece<D>(sm, at, u)) && u.tiles >= 0) {
      const int xt = x * p.tb + tl;  // token of this row within the unit
      const bool row_exists = tl < p.tb && xt < u.ntok;
      const bool has = x == 0 || u.ntok > p.tb;
      const bool active = row_exists && u.tiles > 0;
      int klo = 0, khi = 0;  // this row's keys
      if (active) {
        ChunkSeq s;
        s.n = u.n;
        s.C = u.C;
        s.ks = u.ks;
        klo = key_lo(p.a, s, u.i0 + xt);
        khi = key_hi(p.a, s, u.i0 + xt);
      }
      const bool seen = klo < khi;
      // a warp without a row that sees a key only keeps the hand-offs going
      const bool work = __any_sync(0xffffffffu, seen);
      // tiles [full0, full1) lie inside every row's keys
      const int wlo = __reduce_max_sync(0xffffffffu, klo), whi = __reduce_min_sync(0xffffffffu, seen ? khi : (work ? 0x7fffffff : 0));
      float m_ref = -INFINITY, l_sum = 0.f;
      bool have_o = false;
      if (u.tiles > 0 && has) {
        for (int i = 0; i < u.tiles; ++i, ++c) {
          const int key0 = (u.t0 + i) * kTile;
          if (!mbar_wait_warp(smem_u32(&sm.bar_s[x]), c & 1, abort_flag)) {
            ok = false;
            break;
          }
          // Rows of V outside the unit's keys may hold anything: zeroed, so
          // that 0 * NaN cannot reach O.  Both blocks write the same zeros,
          // so each block's PV sees them.  Not before S of the tile: block
          // B's warps skip units that have no block B without a wait, and
          // then lag behind the ring by many uses of a slot, which a parity
          // does not tell apart.  The block's MMA warp, which has waited for
          // every use of V in turn, issues this S after the last one before
          // this tile's, so from here the parity names one use.
          if (key0 < u.lo || key0 + kTile > u.hi) {
            const uint32_t gt = g + i, vst = kStagesK + gt % kStagesV;  // the tile's V slot
            if (!mbar_wait_warp(smem_u32(&sm.bar_full[vst]), (gt / kStagesV) & 1, abort_flag)) {
              ok = false;
              break;
            }
            if (key0 + row < u.lo || key0 + row >= u.hi) {
              const uint4 z = make_uint4(0u, 0u, 0u, 0u);
#pragma unroll
              for (int hf = 0; hf < kHalves; ++hf) {
                uint4* r0 = reinterpret_cast<uint4*>(sm.ring[vst] + hf * kHalfBytes + row * 128);
#pragma unroll
                for (int k = 0; k < 8; ++k) r0[k] = z;
              }
            }
            fence_proxy_async_smem();
          }
          if (!work) {
            __syncwarp();
            if (lane == 0) {
              mbar_arrive(smem_u32(&sm.bar_p[x][0]));
              mbar_arrive(smem_u32(&sm.bar_p[x][1]));
            }
            continue;
          }
          tc_fence_after();
          uint32_t xs[4][32];
#pragma unroll
          for (int ch = 0; ch < 4; ++ch) tmem_ld32(s_tmem + 32 * ch, xs[ch]);
          tmem_wait_ld();
          if (key0 < wlo || key0 + kTile > whi) {
            // this row's keys within the tile
            const int from = min(max(klo - key0, 0), kTile), to = min(max(khi - key0, 0), kTile);
#pragma unroll
            for (int wd = 0; wd < 4; ++wd) {
              const int f = min(max(from - 32 * wd, 0), 32), e = min(max(to - 32 * wd, 0), 32);
              // bits f .. e-1
              const uint32_t keep = e > f ? (0xffffffffu >> (32 - (e - f))) << f : 0u;
#pragma unroll
              for (int k = 0; k < 32; ++k) xs[wd][k] = (keep >> k) & 1u ? xs[wd][k] : 0xff800000u;
            }
          }
          // The half's probabilities against the reference that the row has,
          // and beside them the row's maximum, which tells whether that
          // reference still serves (scores at most 2^8 above it).  It rarely
          // does not; then, and on a piece's first tile, the half is done
          // (again) with the reference moved.
          const unsigned long long sc2 = f32x2(p.scale_log2, p.scale_log2);
          unsigned long long acc[2], nm2;
          auto half = [&](int hp) {
#pragma unroll
            for (int q = 0; q < 2; ++q) {
              uint32_t pk[16];
#pragma unroll
              for (int k = 0; k < 16; ++k) {
                float e0, e1;
                f32x2_split(fma_f32x2(f32x2(__uint_as_float(xs[2 * hp + q][2 * k]), __uint_as_float(xs[2 * hp + q][2 * k + 1])),
                                      sc2, nm2),
                            e0, e1);
                const float p0 = fast_exp2(e0), p1 = fast_exp2(e1);
                acc[k & 1] = add_f32x2(acc[k & 1], f32x2(p0, p1));
                pk[k] = pack_bf16x2(p0, p1);
              }
              tmem_st16(s_tmem + 32 * hp + 16 * q, pk);
            }
          };
          auto row_max = [&]() {
            float r[8];
#pragma unroll
            for (int k = 0; k < 8; ++k)
              r[k] = fmax3(__uint_as_float(xs[0][k]), __uint_as_float(xs[0][k + 8]), __uint_as_float(xs[0][k + 16]));
#pragma unroll
            for (int k = 0; k < 8; ++k) r[k] = fmax3(r[k], __uint_as_float(xs[0][k + 24]), __uint_as_float(xs[1][k]));
#pragma unroll
            for (int k = 0; k < 8; ++k)
              r[k] = fmax3(r[k], __uint_as_float(xs[1][k + 8]), __uint_as_float(xs[1][k + 16]));
#pragma unroll
            for (int k = 0; k < 8; ++k) r[k] = fmax3(r[k], __uint_as_float(xs[1][k + 24]), __uint_as_float(xs[2][k]));
#pragma unroll
            for (int k = 0; k < 8; ++k)
              r[k] = fmax3(r[k], __uint_as_float(xs[2][k + 8]), __uint_as_float(xs[2][k + 16]));
#pragma unroll
            for (int k = 0; k < 8; ++k) r[k] = fmax3(r[k], __uint_as_float(xs[2][k + 24]), __uint_as_float(xs[3][k]));
#pragma unroll
            for (int k = 0; k < 8; ++k)
              r[k] = fmax3(r[k], __uint_as_float(xs[3][k + 8]), __uint_as_float(xs[3][k + 16]));
#pragma unroll
            for (int k = 0; k < 8; ++k) r[k] = fmaxf(r[k], __uint_as_float(xs[3][k + 24]));
            return fmax3(fmax3(r[0], r[1], r[2]), fmax3(r[3], r[4], r[5]), fmaxf(r[6], r[7])) * p.scale_log2;
          };
          auto start_half = [&]() {
            const float neg_m = m_ref != -INFINITY ? -m_ref : 0.f;
            nm2 = f32x2(neg_m, neg_m);
            acc[0] = acc[1] = f32x2(0.f, 0.f);
          };
          start_half();
          half(0);
          const float mx = row_max();
          const bool move = seen && mx != -INFINITY && (m_ref == -INFINITY || mx > m_ref + kRescaleThreshold);
          if (__any_sync(0xffffffffu, move)) {
            // the first stores of the half are complete before those that
            // replace them are issued (stores to TMEM are asynchronous, and
            // only a wait orders two of them)
            tmem_wait_st();
            // O holds the piece's earlier tiles, all complete (S of this tile
            // was issued after the PV before it had finished)
            const float f = move && m_ref != -INFINITY ? fast_exp2(m_ref - mx) : 1.0f;
            l_sum *= f;
            if (move) m_ref = mx;
            if (i > 0) {
#pragma unroll 1
              for (int ch = 0; ch < D / 16; ++ch) {
                uint32_t o[16];
                tmem_ld16(o_tmem + 16 * ch, o);
                tmem_wait_ld();
#pragma unroll
                for (int k = 0; k < 16; ++k) o[k] = __float_as_uint(__uint_as_float(o[k]) * f);
                tmem_st16(o_tmem + 16 * ch, o);
              }
            }
            start_half();
            half(0);
          }
          auto hand_over = [&](int hp) {
            tmem_wait_st();
            tc_fence_before();
            __syncwarp();
            if (lane == 0) mbar_arrive(smem_u32(&sm.bar_p[x][hp]));
          };
          hand_over(0);
          half(1);
          hand_over(1);
          {
            float s0, s1;
            f32x2_split(add_f32x2(acc[0], acc[1]), s0, s1);
            l_sum += s0 + s1;
          }
        }
        if (u.last) pdl_launch_next();
        have_o = ok && mbar_wait_warp(smem_u32(&sm.bar_pv[x]), (c - 1) & 1, abort_flag);
        if (!have_o) ok = false;
        if (have_o) tc_fence_after();
      } else if (u.last) {
        pdl_launch_next();
      }
      g += u.tiles;
      if (!has) continue;
      // ---- epilogue (a sum that is NaN is passed on, not hidden)
      const bool poison = u.tiles > 0 && *reinterpret_cast<volatile int*>(&sm.bad[u.flag]) != 0;
      const bool any = have_o && seen && l_sum != 0.f && !poison;
      const float inv = any ? 1.0f / l_sum : 0.f;
      const int entry = (static_cast<int>(blockIdx.x) * 2 + u.slot) * 2 + x;
      const size_t out_row = static_cast<size_t>(u.tok0 + (row_exists ? xt : 0)) * p.a.Hq + u.kvh * p.g + hl;
      uint8_t* orow = static_cast<uint8_t*>(p.a.out) + out_row * (2 * D);
#pragma unroll 1
      for (int ch = 0; ch < D / 16; ++ch) {
        uint32_t o[16];
        if (have_o) {
          tmem_ld16(o_tmem + 16 * ch, o);
          tmem_wait_ld();
        }
        if (ch == D / 16 - 1 && u.tiles > 0) {
          // O may be overwritten by the next unit's first PV
          tc_fence_before();
          __syncwarp();
          if (lane == 0) mbar_arrive(smem_u32(&sm.bar_ofree[x]));
        }
        if (!row_exists) continue;
        if (u.part) {
#pragma unroll
          for (int k = 0; k < 4; ++k)
            *partial_o<D>(p, entry, 4 * ch + k, row) =
                any ? make_float4(__uint_as_float(o[4 * k]), __uint_as_float(o[4 * k + 1]),
                                  __uint_as_float(o[4 * k + 2]), __uint_as_float(o[4 * k + 3]))
                    : make_float4(0.f, 0.f, 0.f, 0.f);
        } else {
          uint32_t wv[8];
#pragma unroll
          for (int e = 0; e < 8; ++e)
            wv[e] = any ? pack_bf16x2(__uint_as_float(o[2 * e]) * inv, __uint_as_float(o[2 * e + 1]) * inv) : 0u;
          if (p.wide_out) {
            st_global_256(orow + 32 * ch, wv);
          } else {
            reinterpret_cast<uint4*>(orow + 32 * ch)[0] = make_uint4(wv[0], wv[1], wv[2], wv[3]);
            reinterpret_cast<uint4*>(orow + 32 * ch)[1] = make_uint4(wv[4], wv[5], wv[6], wv[7]);
          }
        }
      }
      if (row_exists && u.part) *partial_ml<D>(p, entry, row) = make_float2(any ? m_ref : -INFINITY, any ? l_sum : poison ? -1.f : 0.f);
      if (row_exists && !u.part && p.a.lse) p.a.lse[out_row] = any ? (m_ref + log2f(l_sum)) * kLn2 : -INFINITY;
    }
    if (!ok && lane == 0) signal_abort(sm, p.a.err_word);
  }

  tc_fence_before();
  __syncthreads();
  if (warp == kWarpMma) {
    tc_fence_after();
    tmem_dealloc(tmem, kTmemCols);
  }
}

// Merge of cut units: O = sum_i 2^(m_i - M) O_i / sum_i 2^(m_i - M) l_i over
// a unit's pieces.  Block (c - 1, y) takes run boundary c and, of its unit's
// query rows, groups of 8 rows y, y + gridDim.y, ...; a thread owns four
// columns of a row (8 rows x 16 bytes of a partial are one line).
template <int D>
__global__ void __launch_bounds__(2 * D) chunk_merge_kernel(const __grid_constant__ ChunkTcParams p) {
  pdl_wait();
  const Record rec = records<D>(p)[blockIdx.x + 1];
  const int np = rec.c1 - rec.c0 + 1, rows = rec.ntok * p.g;
  const int r8 = threadIdx.x & 7, col4 = threadIdx.x >> 3;
  for (int e = blockIdx.y * 8 + r8; e < rows; e += gridDim.y * 8) {
    const int x = e >= p.tb * p.g ? 1 : 0, row = e - x * p.tb * p.g;
    const int tl = row / p.g, hl = row - tl * p.g;
    auto entry = [&](int j) { return ((rec.c0 + j) * 2 + (j == 0 ? rec.slot : 0)) * 2 + x; };
    const size_t out_row = static_cast<size_t>(rec.tok0 + x * p.tb + tl) * p.a.Hq + rec.kvh * p.g + hl;
    uint2* dst = reinterpret_cast<uint2*>(static_cast<__nv_bfloat16*>(p.a.out) + out_row * D) + col4;
    if (np == 2) {
      // cut once, as nearly always: all loads together
      const float2 ma = *partial_ml<D>(p, entry(0), row), mb = *partial_ml<D>(p, entry(1), row);
      const float4 oa = *partial_o<D>(p, entry(0), col4, row), ob = *partial_o<D>(p, entry(1), col4, row);
      const bool ha = ma.y != 0.f, hb = mb.y != 0.f, poison = ma.y == -1.f || mb.y == -1.f;
      const float M = fmaxf(ha ? ma.x : -INFINITY, hb ? mb.x : -INFINITY);
      const float wa = ha && !poison ? exp2f(ma.x - M) : 0.f, wb = hb && !poison ? exp2f(mb.x - M) : 0.f;
      const float L = fmaf(wa, ma.y, wb * mb.y), inv = L != 0.f ? 1.f / L : 0.f;
      *dst = L == 0.f ? make_uint2(0u, 0u)
                      : make_uint2(pack_bf16x2(fmaf(wa, oa.x, wb * ob.x) * inv, fmaf(wa, oa.y, wb * ob.y) * inv),
                                   pack_bf16x2(fmaf(wa, oa.z, wb * ob.z) * inv, fmaf(wa, oa.w, wb * ob.w) * inv));
      if (p.a.lse && col4 == 0) p.a.lse[out_row] = L != 0.f ? (M + log2f(L)) * kLn2 : -INFINITY;
      continue;
    }
    float M = -INFINITY;
    bool poison = false;
#pragma unroll 4
    for (int j = 0; j < np; ++j) {
      const float2 ml = *partial_ml<D>(p, entry(j), row);
      if (ml.y != 0.f) M = fmaxf(M, ml.x);
      poison |= ml.y == -1.f;
    }
    float L = 0.f;
    float4 acc = make_float4(0.f, 0.f, 0.f, 0.f);
#pragma unroll 4
    for (int j = 0; j < np; ++j) {
      const float2 ml = *partial_ml<D>(p, entry(j), row);
      const float4 o = *partial_o<D>(p, entry(j), col4, row);
      const float w = ml.y != 0.f && !poison ? exp2f(ml.x - M) : 0.f;
      L = fmaf(w, ml.y, L);
      acc.x = fmaf(w, o.x, acc.x);
      acc.y = fmaf(w, o.y, acc.y);
      acc.z = fmaf(w, o.z, acc.z);
      acc.w = fmaf(w, o.w, acc.w);
    }
    const float inv = L != 0.f ? 1.f / L : 0.f;
    *dst = L == 0.f ? make_uint2(0u, 0u)
                    : make_uint2(pack_bf16x2(acc.x * inv, acc.y * inv), pack_bf16x2(acc.z * inv, acc.w * inv));
    if (p.a.lse && col4 == 0) p.a.lse[out_row] = L != 0.f ? (M + log2f(L)) * kLn2 : -INFINITY;
  }
  pdl_launch_next();
}

template <int D>
cudaError_t launch_d(const ChunkArgs& a, int num_sms, EncodeTiledFn encode, cudaStream_t stream) {
  ChunkTcParams p{};
  p.a = a;
  p.g = a.Hq / a.Hkv;
  p.tb = kRows / p.g;
  p.ctas = num_sms;
  p.wide_out = (reinterpret_cast<uintptr_t>(a.out) & 31u) == 0;
  p.scale_log2 = a.scale * 1.4426950408889634f;
  CUtensorMap tq, tk, tv;
  {
    const cuuint64_t dims[3] = {D, static_cast<cuuint64_t>(a.Hq), static_cast<cuuint64_t>(a.T)};
    const cuuint64_t strides[2] = {D * 2ull, static_cast<cuuint64_t>(a.q_stride) * 2ull};
    const cuuint32_t box[3] = {64u, static_cast<cuuint32_t>(p.g), static_cast<cuuint32_t>(p.tb)};
    if (!make_bf16_map(encode, &tq, a.q, 3, dims, strides, box)) return cudaErrorInvalidValue;
  }
  {
    const cuuint64_t dims[2] = {D, std::max<cuuint64_t>(1, static_cast<cuuint64_t>(a.num_pages) * a.Hkv * a.page_size)};
    const cuuint64_t strides[1] = {D * 2ull};
    const cuuint32_t box[2] = {64u, static_cast<cuuint32_t>(std::min(a.page_size, kSub))};
    if (!make_bf16_map(encode, &tk, a.k_cache, 2, dims, strides, box)) return cudaErrorInvalidValue;
    if (!make_bf16_map(encode, &tv, a.v_cache, 2, dims, strides, box)) return cudaErrorInvalidValue;
  }
  {
    // the shared-memory attribute, once per device
    static std::mutex mu;
    static bool done[64] = {};
    int dev = 0;
    cudaError_t e = cudaGetDevice(&dev);
    if (e != cudaSuccess) return e;
    if (dev < 0 || dev >= 64) return cudaErrorInvalidDevice;
    std::lock_guard<std::mutex> lk(mu);
    if (!done[dev]) {
      e = cudaFuncSetAttribute(chunk_tc_kernel<D>, cudaFuncAttributeMaxDynamicSharedMemorySize,
                               static_cast<int>(smem_bytes<D>()));
      if (e != cudaSuccess) return e;
      done[dev] = true;
    }
  }
  cudaError_t e = launch_overlapped(chunk_tc_kernel<D>, dim3(static_cast<unsigned>(p.ctas)), dim3(kThreads),
                                    smem_bytes<D>(), stream, 1u, tq, tk, tv, p);
  if (e != cudaSuccess || p.ctas == 1) return e;
  // units of many rows: 16 blocks to a boundary (two passes over 256 rows; the
  // launch after an 8192-token prompt takes 8 us, with 4 blocks 24)
  const unsigned y = static_cast<long long>(a.T) * p.g > 32ll * a.Bt ? 16u : 2u;
  return launch_overlapped(chunk_merge_kernel<D>, dim3(static_cast<unsigned>(p.ctas - 1), y), dim3(2 * D), 0,
                           stream, 1u, p);
}

}  // namespace

size_t chunk_tc_workspace_bytes(int T, int Bt, int d, int num_sms) {
  if (T <= 0 || Bt <= 0) return 0;
  // two partial pieces per CTA, two row blocks each: O and (m, l) of 128
  // rows; then a record per run boundary
  return static_cast<size_t>(num_sms) * (4ull * kRows * (d + 2) * sizeof(float) + sizeof(Record));
}

cudaError_t launch_chunk_attention_tc(const ChunkArgs& a, int num_sms, EncodeTiledFn encode, cudaStream_t stream) {
  return a.d == 128 ? launch_d<128>(a, num_sms, encode, stream) : launch_d<64>(a, num_sms, encode, stream);
}

}  // namespace simsd
