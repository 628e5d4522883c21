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
// Q_A K^T, S_B = Q_B K^T, O_A += P_A V, O_B += P_B V.  While the softmax of
// one block runs, the MMAs of the other keep the tensor pipe busy.
//
// Work.  The key tiles of all units end to end (KV head slowest, so that
// CTAs work on one head's K/V at a time) are cut into equal runs, one per
// CTA (one CTA per SM); lengths are only known on the device, so every CTA
// sums them up itself and finds where its run starts, then walks unit by
// unit.  A unit cut by a run's end leaves partial (O, m, l), which a second
// launch merges.  Long prompts (compute-bound) and single tokens over long
// caches (memory-bound) so load every SM alike.
//
// Warp roles (512 threads): warps 0-3 softmax of row block A, 4-7 of B
// (thread i of a block owns query row i = TMEM lane i); warp 8 TMA producer
// of Q and K, warp 11 of V; warps 9, 10 issue S of A and B, warps 12, 13 PV
// of A and B (a thread that issues a tcgen05.mma is held about as long as
// the MMA runs, so each stream has its own).
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
#include "ptx.cuh"

namespace simsd {
namespace {

constexpr int kTile = 128;     // keys per tile
constexpr int kSub = 64;       // keys per copy (a page, or part of one)
constexpr int kRows = 128;     // query rows per row block (MMA M)
constexpr int kThreads = 512;  // warps 14-15 only meet the final barrier
constexpr int kSoftmaxThreads = 256;
constexpr int kWarpProducer = 8, kWarpMma = 9, kWarpProducerV = 11, kWarpPv = 12;
constexpr uint32_t kTmemCols = 512;
constexpr uint32_t kColS = 0, kColO = 256;  // + 128 per row block
constexpr int kHalfBytes = kTile * 128;     // 128 rows x 64 bf16
constexpr float kRescaleThreshold = 8.0f;   // log2 units
constexpr float kLn2 = 0.6931471805599453f;

struct ChunkTcParams {
  ChunkArgs a;
  int g, tb;          // heads per KV head, tokens per row block
  int ctas;           // grid size
  float scale_log2;
};

template <int D>
struct alignas(1024) SmemChunk {
  static constexpr int kHalves = D / 64;
  static constexpr int kTileBytes = kHalves * kHalfBytes;  // one K or V tile
  // K and V have rings of their own: whoever waits on a slot's barrier waits
  // for every use of it in turn, so a parity is never read a phase early
  static constexpr int kStagesK = D == 128 ? 3 : 5, kStagesV = D == 128 ? 2 : 5;
  static constexpr int kStages = kStagesK + kStagesV;
  uint8_t ring[kStages][kTileBytes];  // K, then V
  uint8_t q[2][kTileBytes];
  uint64_t bar_full[kStages], bar_free[kStages];
  uint64_t bar_q, bar_qfree;
  uint64_t bar_s[2], bar_p[2][2], bar_pv[2], bar_ofree[2];
  uint64_t bar_drain[4];
  uint32_t tmem_base;
  int abort_flag;
  int bad[2];          // per unit parity: a needed page id is out of range
  long long total;     // key tiles of all units of one KV head
  int start[4];        // where the CTA's run starts: sequence, unit of it, KV head, tile
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

// Key tiles [t0, t0 + tiles) that unit j of a sequence sees; a unit that
// sees none (or whose sequence is bad) still counts one tile in the walk,
// as somebody has to zero its rows.
struct Range {
  int t0, tiles, lo, hi;
};
__device__ __forceinline__ Range unit_range(const ChunkTcParams& p, const ChunkSeq& s, int j) {
  Range r{0, 0, 0, 0};
  if (s.bad) return r;
  const int ub = 2 * p.tb, i0 = j * ub, i1 = min(s.C, i0 + ub);
  const int lo = key_lo(p.a, s, i0), hi = key_hi(p.a, s, i1 - 1);
  if (lo >= hi) return r;
  r.lo = lo;
  r.hi = hi;
  r.t0 = lo / kTile;
  r.tiles = (hi + kTile - 1) / kTile - r.t0;
  return r;
}
__device__ __forceinline__ int unit_weight(const ChunkTcParams& p, const ChunkSeq& s, int j) {
  return max(1, unit_range(p, s, j).tiles);
}

// A piece: key tiles [t0, t0 + tiles) of a unit.
struct Piece {
  int b, j, kvh;
  ChunkSeq s;
  Range r;     // the whole unit's
  int t0, tiles;
  bool part;   // writes partial results
  int slot;    // 0: the piece at the start of the CTA's run
  bool last;   // the CTA's last piece
};

// A CTA's walk over its run [R0, R1): from the first unit that starts in it
// to R1, then the unit cut at R0, so that both pieces of a cut unit are
// written near the end of the launch.
struct Walk {
  int b, j, kvh, t;    // next piece (t: tile of the unit, in walk weight)
  long long left;      // tiles left of the current phase
  int hb, hj, hk, ht;  // the run's start
  long long head;      // tiles of the unit cut at the run's start
  int phase;
  bool first;          // the next piece begins at the run's start
};

template <int D>
__device__ __forceinline__ void walk_advance(const ChunkTcParams& p, Walk& w) {
  // to the next unit that exists
  ++w.j;
  w.t = 0;
  for (;;) {
    const Chunk c = chunk_of(p.a.token_start, w.b, p.a.T);
    if (w.j * 2ll * p.tb < c.count) return;
    w.j = 0;
    if (++w.b == p.a.Bt) {
      w.b = 0;
      if (++w.kvh == p.a.Hkv) return;
    }
    if (chunk_of(p.a.token_start, w.b, p.a.T).count > 0) return;
  }
}

template <int D>
__device__ __forceinline__ Walk walk_begin(const ChunkTcParams& p, const SmemChunk<D>& sm) {
  Walk w;
  const long long total = sm.total * p.a.Hkv, W = (total + p.ctas - 1) / p.ctas;
  const long long R0 = min(total, W * blockIdx.x), R1 = min(total, R0 + W);
  w.b = w.hb = sm.start[0];
  w.j = w.hj = sm.start[1];
  w.kvh = w.hk = sm.start[2];
  w.t = w.ht = sm.start[3];
  w.phase = 0;
  w.left = R1 - R0;
  w.head = 0;
  w.first = true;
  if (w.left > 0 && w.t > 0) {
    const int weight = unit_weight(p, chunk_seq(p.a, w.b), w.j);
    w.head = min(w.left, static_cast<long long>(weight - w.t));
    w.left -= w.head;
    w.first = false;
    if (w.left > 0) walk_advance<D>(p, w);
  }
  return w;
}

template <int D>
__device__ __forceinline__ bool walk_next(const ChunkTcParams& p, Walk& w, Piece& u) {
  if (w.phase == 0 && w.left == 0) {
    w.phase = 1;
    w.left = w.head;
    w.b = w.hb;
    w.j = w.hj;
    w.kvh = w.hk;
    w.t = w.ht;
    w.first = true;
  }
  if (w.left == 0) return false;
  u.b = w.b;
  u.j = w.j;
  u.kvh = w.kvh;
  u.s = chunk_seq(p.a, w.b);
  u.r = unit_range(p, u.s, w.j);
  const int weight = max(1, u.r.tiles);
  const int take = static_cast<int>(min(static_cast<long long>(weight - w.t), w.left));
  u.t0 = u.r.t0 + w.t;
  u.tiles = u.r.tiles == 0 ? 0 : take;
  u.part = take < weight;
  u.slot = w.first ? 0 : 1;
  w.first = false;
  w.left -= take;
  u.last = w.left == 0 && (w.phase == 1 || w.head == 0);
  if (w.left > 0) walk_advance<D>(p, w);
  return true;
}

// Where runs start.  Every thread of the block takes part; `tiles` (shared,
// kChunkMaxSeqs ints) holds each sequence's key tiles, then their running
// sum modulo 2^32 (a sequence is found by its exact 64-bit sum per round).
template <int D>
__device__ void plan_run(const ChunkTcParams& p, SmemChunk<D>& sm, int32_t* tiles) {
  const int tid = threadIdx.x, warp = tid >> 5, lane = tid & 31;
  const unsigned full = 0xffffffffu;
  const int ub = 2 * p.tb;
  uint32_t err = 0;
  // short chunks: a thread per sequence; chunks of more than two units: a warp
  for (int b = tid; b < p.a.Bt; b += kThreads) {
    const ChunkSeq s = chunk_seq(p.a, b);
    err |= (s.bad_off ? SIMSD_EW_TOKENS : 0u) | (s.bad && s.C > 0 ? SIMSD_EW_PREFIX_LEN : 0u);
    const int units = (s.C + ub - 1) / ub;
    int v = -1;
    if (units <= 2) {
      v = units > 0 ? unit_weight(p, s, 0) : 0;
      if (units > 1) v += unit_weight(p, s, 1);
    }
    tiles[b] = v;
  }
  if (err && blockIdx.x == 0) raise_error(p.a.err_word, err);
  __syncthreads();
  for (int b = warp; b < p.a.Bt; b += kThreads / 32) {
    if (tiles[b] >= 0) continue;
    const ChunkSeq s = chunk_seq(p.a, b);
    const int units = (s.C + ub - 1) / ub;
    int v = 0;
    for (int j = lane; j < units; j += 32) v += unit_weight(p, s, j);
#pragma unroll
    for (int o = 16; o > 0; o >>= 1) v += __shfl_xor_sync(full, v, o);
    if (lane == 0) tiles[b] = v;
  }
  __syncthreads();
  // warp 0: the total, then the sequence that holds the run's start
  if (warp == 0) {
    long long sum = 0;
    for (int b = lane; b < p.a.Bt; b += 32) sum += tiles[b];
#pragma unroll
    for (int o = 16; o > 0; o >>= 1) sum += __shfl_xor_sync(full, sum, o);
    const long long all = sum * p.a.Hkv, W = (all + p.ctas - 1) / p.ctas;
    const long long R0 = min(all, W * blockIdx.x);
    int kvh = 0, b = 0, j = 0, t = 0;
    if (R0 < all) {
      kvh = static_cast<int>(R0 / sum);
      long long at = R0 - kvh * sum;  // tiles before the run within the head
      for (int b0 = 0; b0 < p.a.Bt; b0 += 32) {
        const int v = b0 + lane < p.a.Bt ? tiles[b0 + lane] : 0;
        long long inc = v;
#pragma unroll
        for (int o = 1; o < 32; o <<= 1) {
          const long long y = __shfl_up_sync(full, inc, o);
          if (lane >= o) inc += y;
        }
        const unsigned m = __ballot_sync(full, inc > at);
        if (m) {
          const int k = __ffs(m) - 1;
          b = b0 + k;
          at -= __shfl_sync(full, inc - v, k);
          break;
        }
        at -= __shfl_sync(full, inc, 31);
      }
      const ChunkSeq s = chunk_seq(p.a, b);
      const int units = (s.C + ub - 1) / ub;
      for (int j0 = 0; j0 < units; j0 += 32) {
        const int v = j0 + lane < units ? unit_weight(p, s, j0 + lane) : 0;
        int inc = v;
#pragma unroll
        for (int o = 1; o < 32; o <<= 1) {
          const int y = __shfl_up_sync(full, inc, o);
          if (lane >= o) inc += y;
        }
        const unsigned m = __ballot_sync(full, inc > at);
        if (m) {
          const int k = __ffs(m) - 1;
          j = j0 + k;
          t = static_cast<int>(at) - __shfl_sync(full, inc - v, k);
          break;
        }
        at -= __shfl_sync(full, inc, 31);
      }
    }
    if (lane == 0) {
      sm.total = sum;
      sm.start[0] = b;
      sm.start[1] = j;
      sm.start[2] = kvh;
      sm.start[3] = t;
    }
  }
  __syncthreads();
}

// Partial results: O (unnormalised, fp32) [ctas * 4][128][D], (m, l)
// [ctas * 4][128][2], entry (cta * 2 + slot) * 2 + block, m in log2 units;
// then one record per run boundary.
struct Record {
  int tok0, ntok, kvh, c0;  // ntok 0: boundary cuts no unit, or not as the first
  int c1, slot, pad0, pad1;
};
template <int D>
__device__ __forceinline__ float* partial_o(const ChunkTcParams& p, size_t entry, int row) {
  return static_cast<float*>(p.a.workspace) + (entry * kRows + row) * D;
}
template <int D>
__device__ __forceinline__ float2* partial_ml(const ChunkTcParams& p, size_t entry, int row) {
  return reinterpret_cast<float2*>(static_cast<float*>(p.a.workspace) + static_cast<size_t>(p.ctas) * 4 * kRows * D) +
         entry * kRows + row;
}
template <int D>
__device__ __forceinline__ Record* records(const ChunkTcParams& p) {
  return reinterpret_cast<Record*>(static_cast<float*>(p.a.workspace) +
                                   static_cast<size_t>(p.ctas) * 4 * kRows * (D + 2));
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
    sm.bad[0] = sm.bad[1] = 0;
    for (int s = 0; s < kStages; ++s) {
      mbar_init(smem_u32(&sm.bar_full[s]), 1);
      mbar_init(smem_u32(&sm.bar_free[s]), 2);  // one commit per row block
    }
    mbar_init(smem_u32(&sm.bar_q), 1);
    mbar_init(smem_u32(&sm.bar_qfree), 2);
    for (int x = 0; x < 2; ++x) {
      mbar_init(smem_u32(&sm.bar_s[x]), 1);
      mbar_init(smem_u32(&sm.bar_p[x][0]), 4);
      mbar_init(smem_u32(&sm.bar_p[x][1]), 4);
      mbar_init(smem_u32(&sm.bar_pv[x]), 1);
      mbar_init(smem_u32(&sm.bar_ofree[x]), 4);
    }
    for (int d = 0; d < 4; ++d) mbar_init(smem_u32(&sm.bar_drain[d]), 1);
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
  plan_run<D>(p, sm, reinterpret_cast<int32_t*>(sm.ring[0]));
  fence_proxy_async_smem();  // the ring was written here and is filled by TMA next
  tc_fence_before();
  __syncthreads();
  tc_fence_after();
  const uint32_t tmem = sm.tmem_base;

  // register split: 2 x 128 x 200 + 2 x 128 x 56 = 65,536, the launch's 512 x 128
  if (warp >= 8) {
    asm volatile("setmaxnreg.dec.sync.aligned.u32 56;");
    if (warp == kWarpProducer || warp == kWarpProducerV) {
      // ----------------------------------------------------------- producers
      // warp 8 fills the K slots (and Q), warp 11 the V slots
      const int kv = warp == kWarpProducer ? 0 : 1;
      const uint32_t slots = kv == 0 ? kStagesK : kStagesV, slot0 = kv == 0 ? 0 : kStagesK;
      const CUtensorMap* m = kv == 0 ? &tm_k : &tm_v;
      uint32_t g = 0, jq = 0;
      bool ok = true;
      Walk w = walk_begin<D>(p, sm);
      Piece u;
      while (ok && walk_next<D>(p, w, u)) {
        if (u.tiles == 0) continue;
        if (kv == 0) {
          if (lane == 0) {
            if (jq > 0 && !mbar_wait(smem_u32(&sm.bar_qfree), (jq - 1) & 1, abort_flag)) {
              ok = false;
            } else {
              const uint32_t bq = smem_u32(&sm.bar_q);
              const int nblk = (u.s.C - u.j * 2 * p.tb) > p.tb ? 2 : 1;
              mbar_arrive_expect_tx(bq, static_cast<uint32_t>(nblk * kHalves * p.g * p.tb) * 128u);
              for (int x = 0; x < nblk; ++x)
                for (int hf = 0; hf < kHalves; ++hf)
                  tma_load_3d(smem_u32(sm.q[x]) + hf * kHalfBytes, &tm_q, bq, 64 * hf, u.kvh * p.g,
                              u.s.start + (u.j * 2 + x) * p.tb);
            }
          }
          ok = __shfl_sync(0xffffffffu, ok, 0);
          if (!ok) break;
          ++jq;
        }
        const int32_t* bt = p.a.block_table + static_cast<size_t>(u.b) * p.a.max_pages;
        const int P = p.a.page_size, sub = min(P, kSub);
        int win_base = -(1 << 30), win = -1;  // lane i holds the page id of page win_base + i
        for (int t = u.t0; t < u.t0 + u.tiles; ++t) {
          const uint32_t st = slot0 + g % slots, use = g / slots;
          const int key0 = t * kTile, valid = min(kTile, u.r.hi - key0);
          const int nsub = (valid + sub - 1) / sub;
          const int pi0 = key0 / P;
          if (lane == 0 && use > 0 && !mbar_wait(smem_u32(&sm.bar_free[st]), (use - 1) & 1, abort_flag)) ok = false;
          ok = __shfl_sync(0xffffffffu, ok, 0);
          if (!ok) break;
          const int pi1 = (key0 + valid - 1) / P;  // at most 16 pages a tile
          if (pi0 < win_base || pi1 >= win_base + 32) {
            win_base = pi0;
            const int pi = win_base + lane;
            win = pi < p.a.max_pages ? bt[pi] : -1;
          }
          const uint32_t bar = smem_u32(&sm.bar_full[st]);
          if (lane == 0) mbar_arrive_expect_tx(bar, static_cast<uint32_t>(nsub * kHalves * sub) * 128u);
          __syncwarp();
          // lane s issues the copies of sub-tile s
          {
            const int key = key0 + min(lane, nsub - 1) * sub, pi = key / P;
            int pg = __shfl_sync(0xffffffffu, win, (pi - win_base) & 31);
            // a page id out of range is replaced by page 0 (the softmax warps
            // zero the unit's output and raise the error)
            if (pg < 0 || pg >= p.a.num_pages) pg = 0;
            if (lane < nsub) {
              const int row = (pg * p.a.Hkv + u.kvh) * P + (key - pi * P);
              const uint32_t dst = smem_u32(sm.ring[st]) + static_cast<uint32_t>(lane * sub) * 128u;
              for (int hf = 0; hf < kHalves; ++hf) tma_load_2d(dst + hf * kHalfBytes, m, bar, 64 * hf, row);
            }
          }
          ++g;
        }
      }
      if (!ok && lane == 0) signal_abort(sm, p.a.err_word);
      // every issued load must have landed before the CTA may exit
      if (lane == 0) {
        for (uint32_t it = g > slots ? g - slots : 0; it < g; ++it)
          mbar_wait(smem_u32(&sm.bar_full[slot0 + it % slots]), (it / slots) & 1, nullptr);
        if (kv == 0 && jq > 0) mbar_wait(smem_u32(&sm.bar_q), (jq - 1) & 1, nullptr);
      }
      __syncwarp();
    } else if (warp >= kWarpMma && warp <= kWarpPv + 1) {
      // ---------------------------------------------------------- MMA issuers
      const bool is_s = warp < kWarpProducerV;
      const int x = is_s ? warp - kWarpMma : warp - kWarpPv;
      if (lane == 0) {
        constexpr uint32_t kIdescQK = idesc_bf16_f32(kRows, kTile, 0, 0);
        constexpr uint32_t kIdescPV = idesc_bf16_f32(kRows, D, 0, 1);
        const uint32_t qb = smem_u32(sm.q[x]);
        const uint32_t scol = tmem + kColS + 128u * x, ocol = tmem + kColO + 128u * x;
        uint32_t g = 0;         // tiles of the walk
        uint32_t c = 0, jc = 0;  // tiles and units this row block has worked on
        uint32_t jq = 0;
        bool ok = true;
        Walk w = walk_begin<D>(p, sm);
        Piece u;
        while (ok && walk_next<D>(p, w, u)) {
          if (u.tiles == 0) continue;
          // a unit of few tokens has no second row block: its issuers only
          // pass the tiles on (each tile's release counts both blocks)
          const bool has = x == 0 || u.s.C - u.j * 2 * p.tb > p.tb;
          ++jq;
          if (is_s) {
            ok = mbar_wait(smem_u32(&sm.bar_q), (jq - 1) & 1, abort_flag);
            for (int i = 0; ok && i < u.tiles; ++i, ++g) {
              const uint32_t st = g % kStagesK;
              // S(t) needs K(t), and the PV of the tile before, whose P lies in S
              ok = mbar_wait_poll(smem_u32(&sm.bar_full[st]), (g / kStagesK) & 1, abort_flag) &&
                   (!has || c == 0 || mbar_wait_poll(smem_u32(&sm.bar_pv[x]), (c - 1) & 1, abort_flag));
              if (!ok) break;
              if (has) {
                tc_fence_after();
                const uint32_t kb = smem_u32(sm.ring[st]);
#pragma unroll
                for (int kk = 0; kk < D / 16; ++kk) {
                  const uint32_t off = (kk >> 2) * kHalfBytes + (kk & 3) * 32;
                  tc_mma_ss(scol, sdesc_sw128(qb + off, 16, 1024), sdesc_sw128(kb + off, 16, 1024), kIdescQK, kk > 0);
                }
                tc_commit(smem_u32(&sm.bar_s[x]));
                ++c;
              }
              tc_commit(smem_u32(&sm.bar_free[st]));
            }
            if (ok) tc_commit(smem_u32(&sm.bar_qfree));
          } else {
            for (int i = 0; ok && i < u.tiles; ++i, ++g) {
              const uint32_t st = kStagesK + g % kStagesV;
              ok = mbar_wait_poll(smem_u32(&sm.bar_full[st]), (g / kStagesV) & 1, abort_flag);
              if (ok && has) {
                // the unit's first PV overwrites O: the epilogue of the unit before has read it
                if (i == 0 && jc > 0) ok = mbar_wait_poll(smem_u32(&sm.bar_ofree[x]), (jc - 1) & 1, abort_flag);
                const uint32_t vb = smem_u32(sm.ring[st]);
#pragma unroll
                for (int hp = 0; hp < 2; ++hp) {
                  ok = ok && mbar_wait_poll(smem_u32(&sm.bar_p[x][hp]), c & 1, abort_flag);
                  if (!ok) break;
                  tc_fence_after();
#pragma unroll
                  for (int kk = 4 * hp; kk < 4 * hp + 4; ++kk)
                    tc_mma_ts(ocol, scol + 8 * kk, sdesc_sw128(vb + kk * 2048, kHalfBytes, 1024), kIdescPV,
                              (i == 0 && kk == 0) ? 0u : 1u);
                }
                if (ok) tc_commit(smem_u32(&sm.bar_pv[x]));
                ++c;
              }
              if (ok) tc_commit(smem_u32(&sm.bar_free[st]));
            }
            if (has) ++jc;
          }
        }
        if (!ok) signal_abort(sm, p.a.err_word);
        const int d = (is_s ? 0 : 2) + x;
        tc_commit(smem_u32(&sm.bar_drain[d]));
        mbar_wait(smem_u32(&sm.bar_drain[d]), 0, nullptr);
      }
      __syncwarp();
    }
  } else {
    asm volatile("setmaxnreg.inc.sync.aligned.u32 200;");
    // -------------------------------------------------------------- softmax
    const int x = warp >> 2;
    const int row = tid & (kRows - 1);
    const int tl = row / p.g, hl = row - tl * p.g;
    const uint32_t lane_tmem = tmem + (static_cast<uint32_t>((warp & 3) * 32) << 16);
    const uint32_t s_tmem = lane_tmem + kColS + 128u * x, o_tmem = lane_tmem + kColO + 128u * x;
    uint32_t g = 0, c = 0, mu = 0;
    bool ok = true;
    Walk w = walk_begin<D>(p, sm);
    Piece u;
    for (; walk_next<D>(p, w, u); ++mu) {
      const int par = mu & 1;
      // every softmax thread is done with the unit before: its flag is cleared
      asm volatile("bar.sync 1, 256;" ::: "memory");
      if (tid == 0) sm.bad[par ^ 1] = 0;
      if (u.tiles > 0) {
        const int32_t* bt = p.a.block_table + static_cast<size_t>(u.b) * p.a.max_pages;
        bool bad = false;
        for (int i = u.r.lo / p.a.page_size + tid; i <= (u.r.hi - 1) / p.a.page_size; i += kSoftmaxThreads) {
          const int pg = bt[i];
          bad |= pg < 0 || pg >= p.a.num_pages;
        }
        if (bad) {
          atomicOr(&sm.bad[par], 1);
          raise_error(p.a.err_word, SIMSD_EW_PAGE);
        }
      }
      asm volatile("bar.sync 1, 256;" ::: "memory");
      const int i_tok = (u.j * 2 + x) * p.tb + tl;  // token of this row within its sequence
      const bool row_exists = tl < p.tb && i_tok < u.s.C;
      const bool has = x == 0 || u.s.C - u.j * 2 * p.tb > p.tb;
      const bool active = row_exists && u.tiles > 0 && sm.bad[par] == 0;
      const int klo = active ? key_lo(p.a, u.s, i_tok) : 0, khi = active ? key_hi(p.a, u.s, i_tok) : 0;
      const bool seen = klo < khi;
      const size_t out_row = (static_cast<size_t>(u.s.start) + (row_exists ? i_tok : 0)) * p.a.Hq + u.kvh * p.g + hl;
      float m_ref = -INFINITY, l_sum = 0.f;
      bool have_o = false;
      if (u.tiles > 0 && has) {
        for (int i = 0; ok && i < u.tiles; ++i, ++c) {
          const uint32_t gt = g + i, vst = kStagesK + gt % kStagesV;  // the tile's V slot
          if (!mbar_wait_warp(smem_u32(&sm.bar_s[x]), c & 1, abort_flag)) {
            ok = false;
            break;
          }
          tc_fence_after();
          float xs[kTile];
#pragma unroll
          for (int ch = 0; ch < 4; ++ch) tmem_ld32(s_tmem + 32 * ch, *reinterpret_cast<uint32_t(*)[32]>(xs + 32 * ch));
          tmem_wait_ld();
          const int key0 = (u.t0 + i) * kTile;
          // this row's keys within the tile
          const int from = min(max(klo - key0, 0), kTile), to = min(max(khi - key0, 0), kTile);
          if (__any_sync(0xffffffffu, from > 0 || to < kTile)) {
#pragma unroll
            for (int wd = 0; wd < 4; ++wd) {
              const int f = min(max(from - 32 * wd, 0), 32), e = min(max(to - 32 * wd, 0), 32);
              // bits f .. e-1
              const uint32_t keep = e > f ? (0xffffffffu >> (32 - (e - f))) << f : 0u;
#pragma unroll
              for (int k = 0; k < 32; ++k) xs[32 * wd + k] = (keep >> k) & 1u ? xs[32 * wd + k] : -INFINITY;
            }
          }
          float mx;
          {
            float r[8];
#pragma unroll
            for (int k = 0; k < 8; ++k) r[k] = fmaxf(xs[k], xs[k + 8]);
#pragma unroll
            for (int k = 16; k < kTile; k += 16)
#pragma unroll
              for (int q = 0; q < 8; ++q) r[q] = fmax3(r[q], xs[k + q], xs[k + q + 8]);
            mx = fmax3(fmax3(r[0], r[1], r[2]), fmax3(r[3], r[4], r[5]), fmaxf(r[6], r[7])) * p.scale_log2;
          }
          bool need = false;
          if (seen && mx != -INFINITY) {
            if (m_ref == -INFINITY)
              m_ref = mx;
            else if (mx > m_ref + kRescaleThreshold)
              need = true;
          }
          if (__any_sync(0xffffffffu, need)) {
            // O holds the unit's earlier tiles, all complete (S of this tile
            // was issued after the PV before it had finished)
            const float f = need ? fast_exp2(m_ref - mx) : 1.0f;
            if (need) {
              l_sum *= f;
              m_ref = mx;
            }
            if (i > 0) {
#pragma unroll 1
              for (int ch = 0; ch < D / 32; ++ch) {
                uint32_t o[32];
                tmem_ld32(o_tmem + 32 * ch, o);
                tmem_wait_ld();
#pragma unroll
                for (int k = 0; k < 32; ++k) o[k] = __float_as_uint(__uint_as_float(o[k]) * f);
                tmem_st32(o_tmem + 32 * ch, o);
              }
            }
          }
          // rows of V outside the unit's keys may hold anything: zeroed, so
          // that 0 * NaN cannot reach O.  The first two warps of each block
          // write the same zeros, so each block's PV sees them.
          const int vlo = max(u.r.lo - key0, 0), vhi = min(u.r.hi - key0, kTile);
          if (vlo > 0 || vhi < kTile) {
            if (!mbar_wait_warp(smem_u32(&sm.bar_full[vst]), (gt / kStagesV) & 1, abort_flag)) {
              ok = false;
              break;
            }
            if (row < vlo || row >= vhi) {
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
          const float neg_m = (seen && m_ref != -INFINITY) ? -m_ref : 0.f;
          const unsigned long long sc2 = f32x2(p.scale_log2, p.scale_log2), nm2 = f32x2(neg_m, neg_m);
          unsigned long long acc[4] = {f32x2(0.f, 0.f), f32x2(0.f, 0.f), f32x2(0.f, 0.f), f32x2(0.f, 0.f)};
#pragma unroll
          for (int hp = 0; hp < 2; ++hp) {
#pragma unroll
            for (int q = 0; q < 2; ++q) {
              uint32_t pk[16];
#pragma unroll
              for (int k = 0; k < 16; ++k) {
                const int col = 64 * hp + 32 * q + 2 * k;
                float e0, e1;
                f32x2_split(fma_f32x2(f32x2(xs[col], xs[col + 1]), sc2, nm2), e0, e1);
                const float p0 = fast_exp2(e0), p1 = fast_exp2(e1);
                acc[k & 3] = add_f32x2(acc[k & 3], f32x2(p0, p1));
                pk[k] = pack_bf16x2(p0, p1);
              }
              tmem_st16(s_tmem + 32 * hp + 16 * q, pk);
            }
            tmem_wait_st();
            tc_fence_before();
            __syncwarp();
            if (lane == 0) mbar_arrive(smem_u32(&sm.bar_p[x][hp]));
          }
          {
            float s0, s1;
            f32x2_split(add_f32x2(add_f32x2(acc[0], acc[1]), add_f32x2(acc[2], acc[3])), s0, s1);
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
      // ---- epilogue
      // (a sum that is NaN is passed on, not hidden)
      const bool any = have_o && seen && l_sum != 0.f;
      const float inv = any ? 1.0f / l_sum : 0.f;
      const size_t entry = (static_cast<size_t>(blockIdx.x) * 2 + u.slot) * 2 + x;
      if (has) {
        const bool full_write = row_exists && !u.part;
        __nv_bfloat16* orow = static_cast<__nv_bfloat16*>(p.a.out) + out_row * D;
#pragma unroll 1
        for (int ch = 0; ch < D / 32; ++ch) {
          uint32_t o[32];
          if (have_o) {
            tmem_ld32(o_tmem + 32 * ch, o);
            tmem_wait_ld();
          }
          if (row_exists && u.part) {
            float4* dst = reinterpret_cast<float4*>(partial_o<D>(p, entry, row) + 32 * ch);
#pragma unroll
            for (int k = 0; k < 8; ++k)
              dst[k] = any ? make_float4(__uint_as_float(o[4 * k]), __uint_as_float(o[4 * k + 1]),
                                         __uint_as_float(o[4 * k + 2]), __uint_as_float(o[4 * k + 3]))
                           : make_float4(0.f, 0.f, 0.f, 0.f);
          } else if (full_write) {
            uint4* dst = reinterpret_cast<uint4*>(orow + 32 * ch);
#pragma unroll
            for (int k = 0; k < 4; ++k) {
              uint32_t wv[4];
#pragma unroll
              for (int e = 0; e < 4; ++e)
                wv[e] = any ? pack_bf16x2(__uint_as_float(o[8 * k + 2 * e]) * inv,
                                          __uint_as_float(o[8 * k + 2 * e + 1]) * inv)
                            : 0u;
              dst[k] = make_uint4(wv[0], wv[1], wv[2], wv[3]);
            }
          }
        }
        if (row_exists && u.part) *partial_ml<D>(p, entry, row) = make_float2(any ? m_ref : -INFINITY, any ? l_sum : 0.f);
        if (full_write && p.a.lse) p.a.lse[out_row] = any ? (m_ref + log2f(l_sum)) * kLn2 : -INFINITY;
        if (u.tiles > 0) {
          // O may be overwritten by the next unit's first PV
          tc_fence_before();
          __syncwarp();
          if (lane == 0) mbar_arrive(smem_u32(&sm.bar_ofree[x]));
        }
      }
    }
    if (!ok && lane == 0) signal_abort(sm, p.a.err_word);
  }

  tc_fence_before();
  __syncthreads();
  if (warp == kWarpMma) {
    tc_fence_after();
    tmem_dealloc(tmem, kTmemCols);
  }
  // the record of run boundary blockIdx.x: the unit that it is the first to cut
  if (tid == 0 && blockIdx.x > 0 && p.a.workspace) {
    Record rec{};
    const long long total = sm.total * p.a.Hkv, W = (total + p.ctas - 1) / p.ctas, G = W * blockIdx.x;
    if (G < total && sm.start[3] > 0) {
      const ChunkSeq s = chunk_seq(p.a, sm.start[0]);
      const int weight = unit_weight(p, s, sm.start[1]);
      const long long begin = G - sm.start[3], c0 = begin / W;
      if (c0 + 1 == static_cast<long long>(blockIdx.x)) {
        rec.tok0 = s.start + sm.start[1] * 2 * p.tb;
        rec.ntok = min(2 * p.tb, s.C - sm.start[1] * 2 * p.tb);
        rec.kvh = sm.start[2];
        rec.c0 = static_cast<int>(c0);
        rec.c1 = static_cast<int>((begin + weight - 1) / W);
        rec.slot = begin != c0 * W ? 1 : 0;
      }
    }
    records<D>(p)[blockIdx.x] = rec;
  }
}

// Merge of cut units: O = sum_i 2^(m_i - M) O_i / sum_i 2^(m_i - M) l_i over
// a unit's pieces.  Block (c - 1, x, z) takes run boundary c, row block x,
// rows 16 z .. 16 z + 15, four per warp, lanes over the head dimension.
constexpr int kMergeRows = 4;
template <int D>
__global__ void __launch_bounds__(128) chunk_merge_kernel(const __grid_constant__ ChunkTcParams p) {
  constexpr int E = D / 32;  // elements of a lane
  pdl_wait();
  const unsigned full = 0xffffffffu;
  const Record rec = records<D>(p)[blockIdx.x + 1];
  const int x = blockIdx.y, lane = threadIdx.x & 31, warp = threadIdx.x >> 5;
  const int np = rec.c1 - rec.c0 + 1;
  auto entry = [&](int j) { return (static_cast<size_t>(rec.c0 + j) * 2 + (j == 0 ? rec.slot : 0)) * 2 + x; };
  for (int k = 0; k < kMergeRows; ++k) {
    const int row = static_cast<int>(blockIdx.z) * 16 + warp * kMergeRows + k;
    const int tl = row / p.g, tok = x * p.tb + tl;
    if (tl >= p.tb || tok >= rec.ntok) continue;  // (warp-uniform)
    float M = -INFINITY;
    for (int j = lane; j < np; j += 32) {
      const float2 ml = *partial_ml<D>(p, entry(j), row);
      if (ml.y != 0.f) M = fmaxf(M, ml.x);
    }
#pragma unroll
    for (int o = 16; o > 0; o >>= 1) M = fmaxf(M, __shfl_xor_sync(full, M, o));
    float L = 0.f, acc[E];
#pragma unroll
    for (int e = 0; e < E; ++e) acc[e] = 0.f;
    for (int j0 = 0; j0 < np; j0 += 32) {
      float wj = 0.f;
      if (j0 + lane < np) {
        const float2 ml = *partial_ml<D>(p, entry(j0 + lane), row);
        if (ml.y != 0.f) {
          wj = exp2f(ml.x - M);
          L = fmaf(wj, ml.y, L);
        }
      }
      const int cnt = min(32, np - j0);
#pragma unroll 4
      for (int i = 0; i < cnt; ++i) {
        const float* o = partial_o<D>(p, entry(j0 + i), row);
        const float wt = __shfl_sync(full, wj, i);
#pragma unroll
        for (int e = 0; e < E; ++e) acc[e] = fmaf(wt, o[lane * E + e], acc[e]);
      }
    }
#pragma unroll
    for (int o = 16; o > 0; o >>= 1) L += __shfl_xor_sync(full, L, o);
    const float inv = L != 0.f ? 1.f / L : 0.f;
    const size_t out_row = static_cast<size_t>(rec.tok0 + tok) * p.a.Hq + rec.kvh * p.g + (row - tl * p.g);
    uint32_t* dst = reinterpret_cast<uint32_t*>(static_cast<__nv_bfloat16*>(p.a.out) + out_row * D);
#pragma unroll
    for (int e = 0; e < E; e += 2) dst[lane * (E / 2) + e / 2] = pack_bf16x2(acc[e] * inv, acc[e + 1] * inv);
    if (p.a.lse && lane == 0) p.a.lse[out_row] = L != 0.f ? (M + log2f(L)) * kLn2 : -INFINITY;
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
  return launch_overlapped(chunk_merge_kernel<D>, dim3(static_cast<unsigned>(p.ctas - 1), 2u, kRows / 16), dim3(128),
                           0, stream, 1u, p);
}

}  // namespace

size_t chunk_tc_workspace_bytes(int T, int Bt, int Hq, int Hkv, int d, long long max_keys, int num_sms) {
  if (T <= 0 || Bt <= 0) return 0;
  (void)Hq;
  (void)Hkv;
  (void)max_keys;
  // two partial pieces per CTA, two row blocks each: O and (m, l) of 128
  // rows; then a record per run boundary
  return static_cast<size_t>(num_sms) * (4ull * kRows * (d + 2) * sizeof(float) + sizeof(Record));
}

cudaError_t launch_chunk_attention_tc(const ChunkArgs& a, int num_sms, EncodeTiledFn encode, cudaStream_t stream) {
  return a.d == 128 ? launch_d<128>(a, num_sms, encode, stream) : launch_d<64>(a, num_sms, encode, stream);
}

}  // namespace simsd
