// chunk_attention_q4_tc.cu -- attention of short chunks over a paged cache in
// 4 bits on the sm_103a tensor cores (Sec. 3.3: the prefix is read from a KV
// cache).
//
// Mathematics.  As in chunk_attention_q4.cu: keys and values are exact in
// fp16, q is brought to fp16 by a power of two a row, probabilities are
// rounded to fp16, S and O are accumulated in fp32; the softmax is that of
// chunk_attention_tc.cu but for the place of its reference (q4_tiles.cuh).
//
// A unit is (KV head, sequence, up to 128 query rows), a tile 128 keys.  The
// codes and scales of a tile (18 KB) come by bulk copies; eight warps turn
// them into the fp16 tiles of K and V, each once, in the layout that the
// matrix instructions read (rows of 128 bytes, swizzled), and set the rows of
// V that no token sees to zero.  The walk of chunk_walk.cuh; units cut by the
// end of a run are merged by a second launch.
//
// A tile's softmax is one chain of waits, loads and exponentials a row, some
// 3800 cycles where a thread takes all 128 keys of a row.  So a row's keys are
// shared by two threads, 64 each, which have a reference and a sum of their
// own and are put together at the unit's end.  Lean units, of up to 64 rows,
// have their rows of Q twice, in the lanes 0-63 and 64-127 of tensor memory:
// the first take a tile's first 64 keys, the others the last 64, and set the P
// of the keys that are not theirs to zero.  All four partitions of the SM then
// share the exponentials, at the same number of matrix instructions.  Wider
// units have a second set of softmax warps for the last 64 keys, with an O of
// its own.  S has two buffers: S of the next tile is formed under the softmax
// of this one.
//
// Bound and measured.  32 blocks of 16 tokens over 4096 rows (32 heads on 8,
// D = 128; 155 MB, 23 us of copies) take 84 us, of 32 tokens 94.  The matrix
// instructions of a tile take half of its 2100 cycles; the rest are the chains
// beside them, each of which is about as long: one warp of an SM partition
// turns 32 rows of K and one 32 rows of V (29 instructions for 16 components),
// one does the softmax, one looks up pages and copies.  (With 47 instructions,
// by generic addresses, 95 us; then without the turning 80, without turning and
// softmax 71.)  Not faster: twelve turning warps
// and the softmax of a tile over eight warps (96: as many instructions more);
// more rows in flight for each turning warp (110 to 118).  Sets of softmax warps
// that took whole tiles in turns, each with one S: 106.
//
// Warp roles (640 threads): warps 0-3 softmax (thread i owns lane i of tensor
// memory, and turns its row of Q into fp16), warps 4-7 that of the last 64 keys
// of wide units; warps 8-11 K, 12-15 V; warps 16 and 19 walk the run and issue
// the copies of K and Q, and of V; warp 17 issues the products S, warp 18 P V.
// TMEM (512 columns): S [0,128), [128,256); O [256,384); [384,512) O of the
// second set, or the Q of lean units (else Q stays in shared memory); P (fp16)
// of each half of the keys overwrites the first 32 of its own 64 columns of S.
//
// Every mbarrier wait is bounded; after one expires the CTA raises
// SIMSD_EW_TIMEOUT, every role leaves its loops, drains its copies and MMAs
// and frees TMEM.
#include <cuda.h>
#include <cuda_bf16.h>
#include <cuda_fp16.h>
#include <cuda_runtime.h>

#include <algorithm>
#include <mutex>

#include "common.cuh"
#include "kernels.h"
#include "ptx_chunk.cuh"
#include "q4_tiles.cuh"

namespace simsd {
namespace {

constexpr int kTile = kQ4Tile;
constexpr int kRows = 128;  // query rows of a unit (MMA M)
constexpr int kThreads = 640;
constexpr int kWarpConvert = 8, kConvertWarps = 8,  // (half of them K, half V)
              kWarpWalk = 16, kWarpS = 17, kWarpPv = 18, kWarpWalkV = 19;
constexpr uint32_t kTmemCols = 512;
constexpr uint32_t kColO = 256;  // + 128 per set
constexpr uint32_t kColQ = 384;  // lean units: Q
constexpr int kHalfBytes = kTile * 128;  // 128 rows x 64 fp16
constexpr int kInfos = 8;                // tiles that the walk is ahead of the last reader
constexpr float kLn2 = 0.6931471805599453f;

struct Q4TcParams {
  ChunkArgs a;
  simsd_q4_cache c;
  int g, tb;          // heads per KV head, tokens of a unit
  int ctas, sub;      // grid size; keys per copy
  ScoreScale scale;   // of scores, in log2 units
};

template <int D, bool LEAN>
struct alignas(1024) SmemQ4Tc {
  static constexpr int kHalves = D / 64;
  static constexpr int kTileBytes = kHalves * kHalfBytes;
  static constexpr int kQHalf = LEAN ? kHalfBytes / 2 : kHalfBytes;
  static constexpr int kSlots = D == 128 ? 2 : 4;   // of K, and of V
  static constexpr int kStages = D == 64 ? 6 : 3;  // of codes
  static constexpr int kSoftmaxWarps = LEAN ? 4 : 8;
  uint8_t k[kSlots][kTileBytes], v[kSlots][kTileBytes];
  uint8_t q[kHalves * kQHalf];
  Stage<D> ring[kStages];
  TileInfo info[kInfos];
  uint64_t bar_code[kStages], bar_codefree[kStages];
  uint64_t bar_k[kSlots], bar_kfree[kSlots], bar_v[kSlots], bar_vfree[kSlots];
  uint64_t bar_info[kInfos], bar_infofree[kInfos];
  uint64_t bar_qraw, bar_q, bar_qfree;
  uint64_t bar_s[2], bar_p[2][2], bar_pv[2], bar_ofree, bar_meet, bar_drain[2];
  float2 ml[2][LEAN ? 1 : 2][kRows];  // (m, l) of the sets' lanes, for pieces in turns
  float q_factor[2][kRows];  // of the rows' scores, for units in turns
  // lean units: O of the upper lanes on its way to the lower ones, 16 columns
  // at a time, in two buffers
  float o[LEAN ? 2 : 1][16][kRows / 2];
  uint64_t bar_x[2], bar_xfree[2];
  uint32_t tmem_base;
  int abort_flag;
};
template <int D, bool LEAN>
constexpr size_t smem_bytes() {
  return sizeof(SmemQ4Tc<D, LEAN>) + 1024;
}
static_assert(smem_bytes<128, true>() <= 232448 && smem_bytes<64, true>() <= 232448 &&
                  smem_bytes<128, false>() <= 232448 && smem_bytes<64, false>() <= 232448, "one CTA per SM");
static_assert(2 * SmemQ4Tc<64, false>::kSlots * SmemQ4Tc<64, false>::kTileBytes >= kChunkMaxSeqs * 4 &&
                  2 * SmemQ4Tc<128, false>::kSlots * SmemQ4Tc<128, false>::kTileBytes >= kChunkMaxSeqs * 4,
              "the tiles of K and V hold the tile counts of all sequences while runs are planned");

// kind::f16 with fp16 A and B, fp32 accumulator
constexpr uint32_t idesc_f16_f32(int M, int N, int b_mn_major) {
  return (1u << 4) | (static_cast<uint32_t>(b_mn_major) << 16) | (static_cast<uint32_t>(N >> 3) << 17) |
         (static_cast<uint32_t>(M >> 4) << 24);
}

__device__ __forceinline__ uint2 lds64(uint32_t at) {
  uint2 v;
  asm volatile("ld.shared.v2.b32 {%0, %1}, [%2];" : "=r"(v.x), "=r"(v.y) : "r"(at) : "memory");
  return v;
}
__device__ __forceinline__ uint32_t lds8(uint32_t at) {
  uint32_t v;
  asm volatile("ld.shared.u8 %0, [%1];" : "=r"(v) : "r"(at) : "memory");
  return v;
}
__device__ __forceinline__ void sts128(uint32_t at, uint32_t a, uint32_t b, uint32_t c, uint32_t d) {
  asm volatile("st.shared.v4.b32 [%0], {%1, %2, %3, %4};" ::"r"(at), "r"(a), "r"(b), "r"(c), "r"(d) : "memory");
}

// Partial results: O (without the values' unit) as [ctas * 2 entries][D / 4]
// [128 rows] vectors of four, (m, l) [entries][128], entry cta * 2 + slot, m
// in log2 units, l = -1 where a page id of the piece is out of range; then one
// Record per run boundary.
template <int D>
__device__ __forceinline__ float4* partial_o(const Q4TcParams& p, int entry, int col4, int row) {
  return static_cast<float4*>(p.a.workspace) + (static_cast<size_t>(entry) * (D / 4) + col4) * kRows + row;
}
template <int D>
__device__ __forceinline__ float2* partial_ml(const Q4TcParams& p, int entry, int row) {
  return reinterpret_cast<float2*>(partial_o<D>(p, 2 * p.ctas, 0, 0)) + static_cast<size_t>(entry) * kRows + row;
}
template <int D>
__device__ __forceinline__ Record* records(const Q4TcParams& p) {
  return reinterpret_cast<Record*>(partial_ml<D>(p, 2 * p.ctas, 0));
}

template <int D, bool SINKS, bool LEAN>
__global__ void __launch_bounds__(kThreads, 1)
    chunk_q4_tc_kernel(const __grid_constant__ CUtensorMap tm_q, const __grid_constant__ Q4TcParams p) {
  using Smem = SmemQ4Tc<D, LEAN>;
  constexpr int kHalves = Smem::kHalves, kSlots = Smem::kSlots, kStages = Smem::kStages;
  extern __shared__ uint8_t smem_raw[];
  // (an offset from the array: through a number the compiler no longer knows that it is shared memory)
  Smem& sm = *reinterpret_cast<Smem*>(smem_raw + (0u - smem_u32(smem_raw) & 1023u));
  volatile int* abort_flag = &sm.abort_flag;
  const unsigned full = 0xffffffffu;
  const int tid = threadIdx.x, warp = tid >> 5, lane = tid & 31;
  if (tid == 0) {
    sm.abort_flag = 0;
    for (int s = 0; s < kStages; ++s) {
      mbar_init(smem_u32(&sm.bar_code[s]), 2);
      mbar_init(smem_u32(&sm.bar_codefree[s]), kConvertWarps);
    }
    for (int s = 0; s < kSlots; ++s) {
      mbar_init(smem_u32(&sm.bar_k[s]), kConvertWarps / 2);
      mbar_init(smem_u32(&sm.bar_v[s]), kConvertWarps / 2);
      mbar_init(smem_u32(&sm.bar_kfree[s]), 1);
      mbar_init(smem_u32(&sm.bar_vfree[s]), 1);
    }
    for (int s = 0; s < kInfos; ++s) {
      mbar_init(smem_u32(&sm.bar_info[s]), 1);
      mbar_init(smem_u32(&sm.bar_infofree[s]), Smem::kSoftmaxWarps + kConvertWarps + 2);
    }
    mbar_init(smem_u32(&sm.bar_qraw), 1);
    mbar_init(smem_u32(&sm.bar_q), 4);
    mbar_init(smem_u32(&sm.bar_qfree), LEAN ? 4 : 1);
    for (int x = 0; x < 2; ++x) {
      mbar_init(smem_u32(&sm.bar_s[x]), 1);
      mbar_init(smem_u32(&sm.bar_p[x][0]), 4);
      mbar_init(smem_u32(&sm.bar_p[x][1]), 4);
    }
    mbar_init(smem_u32(&sm.bar_pv[0]), 1);
    mbar_init(smem_u32(&sm.bar_pv[1]), 1);
    mbar_init(smem_u32(&sm.bar_ofree), Smem::kSoftmaxWarps);
    mbar_init(smem_u32(&sm.bar_meet), Smem::kSoftmaxWarps);
    mbar_init(smem_u32(&sm.bar_drain[0]), 1);
    mbar_init(smem_u32(&sm.bar_drain[1]), 1);
    for (int x = 0; x < 2; ++x) {
      mbar_init(smem_u32(&sm.bar_x[x]), 2);
      mbar_init(smem_u32(&sm.bar_xfree[x]), 2);
    }
    fence_mbar_init();
  }
  if (warp == kWarpS) {
    tmem_alloc(smem_u32(&sm.tmem_base), kTmemCols);
    tmem_relinquish();
  }
  if (warp == kWarpWalk && lane == 0) tma_prefetch_desc(&tm_q);
  pdl_wait();
  int32_t* tiles = reinterpret_cast<int32_t*>(sm.k[0]);
  plan_tiles<SINKS, kTile, kThreads>(p.a, p.tb, tiles);
  Place start{0, 0, 0, 0};
  int total = 0;
  ChunkSeq seq{};
  if (warp == kWarpWalk || warp == kWarpWalkV) start = plan_start<SINKS, kTile>(p.a, p.tb, p.ctas, tiles, total, seq);
  tc_fence_before();
  __syncthreads();
  tc_fence_after();
  const uint32_t tmem = sm.tmem_base;
  auto give_up = [&]() {
    if (lane == 0) {
      raise_error(p.a.err_word, SIMSD_EW_TIMEOUT);
      *abort_flag = 1;
    }
  };
  auto wait = [&](uint64_t& bar, uint32_t parity) { return mbar_wait_warp(smem_u32(&bar), parity, abort_flag); };
  auto arrive = [&](uint64_t& bar) {
    __syncwarp();
    if (lane == 0) mbar_arrive(smem_u32(&bar));
  };
  bool ok = true;

  // register split: 256 x 128 + 256 x 72 + 128 x 80 = 61,440 = the launch's 640 x 96
  if (warp >= kWarpWalk) {
    asm volatile("setmaxnreg.dec.sync.aligned.u32 80;");
    if (warp == kWarpWalk || warp == kWarpWalkV) {
      // ------------------------------------------------------ walk and copies
      // Both warps walk the run; one copies K and Q and tells the others of the
      // tiles, one copies V.
      const bool tells = warp == kWarpWalk;
      TileWalk<D, SINKS> tw;
      tw.sizes(p.tb, p.sub, p.a.page_size);
      tw.k.begin(p.a, p.tb, p.ctas, start, seq, total);
      uint32_t it = 0, codes = 0, units = 0;  // messages; tiles with copies; Q tiles
      auto say = [&](const TileInfo& u) {
        if (!tells) return;
        if (it >= kInfos) ok = wait(sm.bar_infofree[it % kInfos], ((it / kInfos) - 1) & 1);
        if (!ok) return;
        if (lane == 0) {
          sm.info[it % kInfos] = u;
          mbar_arrive(smem_u32(&sm.bar_info[it % kInfos]));
        }
        ++it;
      };
      while (ok && tw.next_piece(p.a)) {
        const bool empty = tw.flags & kEmpty;
        for (int i = 0; ok && i < tw.piece.take; ++i) {
          tw.tile(p.a, i);
          if (!empty) {
            const uint32_t st = codes % kStages;
            if (codes >= kStages) ok = wait(sm.bar_codefree[st], ((codes / kStages) - 1) & 1);
            if (!ok) break;
            const uint32_t bar = smem_u32(&sm.bar_code[st]), bytes = tw.bytes();
            if (lane == 0) mbar_arrive_expect_tx(bar, bytes);
            __syncwarp();
            if (tells) tw.copy_k(p.c, sm.ring[st], bar);
            else tw.copy_v(p.c, sm.ring[st], bar);
            ++codes;
            if (i == 0 && tells) {
              // Q, once the unit before has no use for its own any more
              if (units > 0) ok = wait(sm.bar_qfree, (units - 1) & 1);
              if (!ok) break;
              if (lane == 0) {
                const uint32_t bq = smem_u32(&sm.bar_qraw);
                mbar_arrive_expect_tx(bq, static_cast<uint32_t>(kHalves * p.g * p.tb) * 128u);
#pragma unroll
                for (int hf = 0; hf < kHalves; ++hf)
                  tma_load_3d(smem_u32(sm.q) + hf * Smem::kQHalf, &tm_q, bq, 64 * hf, tw.u.kvh * p.g, tw.u.tok0);
              }
              ++units;
            }
          }
          say(tw.u);
        }
        if (!ok) break;
        tw.k.pop(p.a, p.tb, tw.piece);
      }
      if (ok) {
        TileInfo u{};
        u.flags = kEnd;
        say(u);
      }
      if (!ok) give_up();
      if (tells && lane == 0 && blockIdx.x > 0) records<D>(p)[blockIdx.x] = boundary_record<SINKS, kTile>(tw.k, p.a, p.tb);
      // every copy must have landed before the CTA may exit
      if (lane == 0) {
        for (uint32_t j = codes > kStages ? codes - kStages : 0; j < codes; ++j)
          mbar_wait(smem_u32(&sm.bar_code[j % kStages]), (j / kStages) & 1, nullptr);
        if (units > 0) mbar_wait(smem_u32(&sm.bar_qraw), (units - 1) & 1, nullptr);
      }
      __syncwarp();
    } else if (warp <= kWarpPv) {
      // ------------------------------------------------------------- products
      // Tile n (counted over the run) has S buffer n & 1 and slots n % kSlots of
      // K and V.
      const bool leader = elect_one();
      auto poll = [&](uint64_t& bar, uint32_t parity) { return mbar_wait(smem_u32(&bar), parity, abort_flag); };
      constexpr uint32_t kTileStep = Smem::kTileBytes >> 4;
      uint32_t n = 0, units = 0;
      for (uint32_t it = 0; ok; ++it) {
        ok = poll(sm.bar_info[it % kInfos], (it / kInfos) & 1);
        if (!ok) break;
        const int flags = sm.info[it % kInfos].flags;
        arrive(sm.bar_infofree[it % kInfos]);
        if (flags & kEnd) break;
        if (flags & kEmpty) continue;
        const uint32_t slot = n % kSlots, buf = n & 1;
        if (warp == kWarpS) {
          constexpr uint32_t kIdesc = idesc_f16_f32(kRows, kTile, 0);
          const uint64_t dq = sdesc_sw128(smem_u32(sm.q), 16, 1024), dk = sdesc_sw128(smem_u32(sm.k[0]), 16, 1024);
          const uint32_t q_lo = static_cast<uint32_t>(dq), hi = static_cast<uint32_t>(dk >> 32);
          const uint32_t k_lo = static_cast<uint32_t>(dk) + slot * kTileStep;
          if (flags & kFirst) ok = poll(sm.bar_q, units & 1);
          ok = ok && poll(sm.bar_k[slot], (n / kSlots) & 1);
          // the PV whose P lies in the same columns is done
          if (n >= 2) ok = ok && poll(sm.bar_pv[buf], ((n >> 1) - 1) & 1);
          __syncwarp();
          if (ok && leader) {
            tc_fence_after();
#pragma unroll
            for (int kk = 0; kk < D / 16; ++kk) {
              const uint32_t off = ((kk >> 2) * kHalfBytes + (kk & 3) * 32) >> 4;
              if constexpr (LEAN) tc_mma_ts_lh(tmem + 128u * buf, tmem + kColQ + 8 * kk, k_lo + off, hi, kIdesc, kk > 0);
              else tc_mma_ss_lh(tmem + 128u * buf, q_lo + off, hi, k_lo + off, hi, kIdesc, kk > 0);
            }
            tc_commit(smem_u32(&sm.bar_s[buf]));
            tc_commit(smem_u32(&sm.bar_kfree[slot]));
            if (!LEAN && (flags & kLast)) tc_commit(smem_u32(&sm.bar_qfree));
          }
          __syncwarp();
        } else {
          constexpr uint32_t kIdesc = idesc_f16_f32(kRows, D, 1);
          const uint64_t dv = sdesc_sw128(smem_u32(sm.v[0]), kHalfBytes, 1024);
          const uint32_t v_lo = static_cast<uint32_t>(dv) + slot * kTileStep, hi = static_cast<uint32_t>(dv >> 32);
          ok = poll(sm.bar_v[slot], (n / kSlots) & 1);
          // the unit's first PV overwrites O: the epilogue of the unit before has read it
          if ((flags & kFirst) && units > 0) ok = ok && poll(sm.bar_ofree, (units - 1) & 1);
#pragma unroll
          for (int hp = 0; hp < 2; ++hp) {
            ok = ok && poll(sm.bar_p[buf][hp], (n >> 1) & 1);
            __syncwarp();
            if (ok && leader) {
              tc_fence_after();
#pragma unroll
              for (int kk = 4 * hp; kk < 4 * hp + 4; ++kk) {
                // (the first products of an O; wide units have one for each half of the keys)
                const bool first = (flags & kFirst) && (kk == 0 || (!LEAN && kk == 4));
                tc_mma_ts_lh(tmem + kColO + (LEAN ? 0u : 128u * hp), tmem + 128u * buf + 32 * hp + 8 * kk, v_lo + kk * 128, hi, kIdesc,
                             first ? 0u : 1u);
              }
              if (hp == 1) {
                tc_commit(smem_u32(&sm.bar_pv[buf]));
                tc_commit(smem_u32(&sm.bar_vfree[slot]));
              }
            }
            __syncwarp();
          }
        }
        ++n;
        if (flags & kLast) ++units;
      }
      if (!ok) give_up();
      if (leader) {
        uint64_t& drain = sm.bar_drain[warp - kWarpS];
        tc_commit(smem_u32(&drain));
        mbar_wait(smem_u32(&drain), 0, nullptr);
      }
      __syncwarp();
    }
  } else if (warp >= kWarpConvert) {
    asm volatile("setmaxnreg.dec.sync.aligned.u32 72;");
    // ------------------------------------------------- codes to tiles of K and V
    // A warp takes 32 rows; a lane one group of 16 components of a row at a
    // time: 8 bytes of codes, a scale, two chunks of 16 bytes.  Lanes of the
    // upper 64 components write their second chunk first: eight lanes then
    // fill eight different chunks of 128 bytes.
    constexpr int kGroups = D / kQ4Group, kRowsStep = 32 / kGroups;
    const int w = warp & 3, kv = (warp - kWarpConvert) >> 2, grp = lane & (kGroups - 1);
    const int half = grp >> 2, ch = (grp & 3) * 2;
    const int r0 = 32 * w + lane / kGroups;
    // Places of the lane's row r0 in a tile: of its first and its second chunk
    // (rows 4 and 8 further have them in the same column, of 8, or 4 columns on).
    const uint32_t to = static_cast<uint32_t>(half * kHalfBytes + r0 * 128), x = r0 & 7;
    const uint32_t to_a = to + (((ch + half) ^ x) << 4), to_b = to + (((ch + 1 - half) ^ x) << 4);
    uint32_t c = 0;
    for (uint32_t it = 0; ok; ++it) {
      ok = wait(sm.bar_info[it % kInfos], (it / kInfos) & 1);
      if (!ok) break;
      const TileInfo& info = sm.info[it % kInfos];
      const int flags = info.flags, key0 = info.key0, lo = info.lo, se = info.se, w0 = info.w0, hi = info.hi;
      arrive(sm.bar_infofree[it % kInfos]);
      if (flags & kEnd) break;
      if (flags & kEmpty) continue;
      const uint32_t st = c % kStages, slot = c % kSlots;
      const Stage<D>& s = sm.ring[st];
      ok = wait(sm.bar_code[st], (c / kStages) & 1);
      if (c >= kSlots) ok = ok && wait(kv ? sm.bar_vfree[slot] : sm.bar_kfree[slot], ((c / kSlots) - 1) & 1);
      if (!ok) break;
      {
        uint32_t codes = smem_u32(kv ? s.vc : s.kc) + r0 * (D / 2) + 8 * grp;
        uint32_t scales = smem_u32(kv ? s.vs : s.ks) + r0 * kGroups + grp;
        uint32_t tile = smem_u32(kv ? sm.v[slot] : sm.k[slot]);
        const bool zero = kv && !(flags & kFull);
        constexpr int kSteps = 16 / kRowsStep;
#pragma unroll 1
        for (int rb = 0; rb < 32; rb += 16) {
          uint2 cw[kSteps];
          uint32_t sc[kSteps];
#pragma unroll
          for (int j = 0; j < kSteps; ++j) {
            cw[j] = lds64(codes + kRowsStep * j * (D / 2));
            sc[j] = lds8(scales + kRowsStep * j * kGroups);
          }
          if (zero) {
            // values of rows that no token of the unit sees may be anything: 0
#pragma unroll
            for (int j = 0; j < kSteps; ++j) {
              const int key = key0 + r0 + rb + kRowsStep * j;
              if (key < lo || key >= hi || (SINKS && key >= se && key < w0)) sc[j] = 0u;
            }
          }
#pragma unroll
          for (int j = 0; j < kSteps; ++j) {
            const uint32_t f = q4_scale_pair(sc[j] * 0x101u);
            const uint32_t ca = half ? cw[j].y : cw[j].x, cb = half ? cw[j].x : cw[j].y;
            const uint32_t turn = kRowsStep == 4 && (j & 1) ? 64u : 0u, at = tile + 128 * kRowsStep * j;
            sts128(at + (to_a ^ turn), mul_f16x2(q4_pair<0>(ca), f), mul_f16x2(q4_pair<1>(ca), f), mul_f16x2(q4_pair<2>(ca), f),
                   mul_f16x2(q4_pair<3>(ca), f));
            sts128(at + (to_b ^ turn), mul_f16x2(q4_pair<0>(cb), f), mul_f16x2(q4_pair<1>(cb), f), mul_f16x2(q4_pair<2>(cb), f),
                   mul_f16x2(q4_pair<3>(cb), f));
          }
          codes += 16 * (D / 2);
          scales += 16 * kGroups;
          tile += 16 * 128;
        }
        fence_proxy_async_smem();
        arrive(kv ? sm.bar_v[slot] : sm.bar_k[slot]);
      }
      if (!ok) break;
      arrive(sm.bar_codefree[st]);
      ++c;
    }
    if (!ok) give_up();
  } else {
    asm volatile("setmaxnreg.inc.sync.aligned.u32 128;");
    // -------------------------------------------------------------- softmax
    // (lean units: the warps of the second set have nothing to do)
    const int set = warp >> 2, row = tid & (kRows - 1);        // row: the lane of tensor memory
    const int upper = LEAN ? row >> 6 : 0, half = LEAN ? upper : set;  // which 64 keys of a tile
    const int ur = LEAN ? row & 63 : row, tl = ur / p.g, hl = ur - tl * p.g;
    const uint32_t lane_tmem = tmem + (static_cast<uint32_t>((warp & 3) * 32) << 16);
    const uint32_t o_tmem = lane_tmem + kColO + 128u * set;
    uint32_t c = 0, units = 0, turns = 0;  // tiles; units; turns of the buffers that O passes through
    bool seen = false;  // the row sees a key
    float m_ref = -INFINITY, l_sum = 0.f, scale = 0.f;
    for (uint32_t it = 0; ok && (!LEAN || set == 0); ++it) {
      ok = wait(sm.bar_info[it % kInfos], (it / kInfos) & 1);
      if (!ok) break;
      const TileInfo& info = sm.info[it % kInfos];
      const int flags = info.flags;
      if (flags & kEnd) break;
      const bool empty = flags & kEmpty;
      // the keys that the row sees: [lo, hi), and of the first rows that stay visible those below se
      auto row_keys = [&](int& lo, int& hi, int& se) {
        lo = hi = se = 0;
        if (tl < p.tb && tl < info.ntok && !empty) {
          ChunkSeq s;
          s.n = info.n;
          s.C = info.C;
          s.ks = info.ks;
          lo = key_lo(p.a, s, info.i0 + tl);
          hi = key_hi(p.a, s, info.i0 + tl);
          if constexpr (SINKS) se = sink_end(p.a, s, hi);
        }
      };
      if (flags & kFirst) {
        int lo, hi, se;
        row_keys(lo, hi, se);
        seen = lo < hi;
        m_ref = -INFINITY;
        l_sum = 0.f;
        if (!empty) {
          // this thread's row of Q: the power of two that its components take,
          // and by the first set its fp16 form, in place of itself or in tensor
          // memory (the other set does not wait for the copy, which may be a unit
          // ahead of it)
          if (set == 0) ok = wait(sm.bar_qraw, units & 1);
          if (!ok) break;
          uint4* qr[kHalves];
          uint32_t top = 0;
#pragma unroll
          for (int hf = 0; hf < kHalves; ++hf) {
            qr[hf] = reinterpret_cast<uint4*>(sm.q + hf * Smem::kQHalf + (LEAN ? ur : row) * 128);
            if (set == 0) {
#pragma unroll
              for (int k = 0; k < 8; ++k) {
                const uint4 x = qr[hf][k ^ (row & 7)];
                const uint32_t a = max(max(x.x & 0x7fffu, x.x >> 16 & 0x7fffu), max(x.y & 0x7fffu, x.y >> 16 & 0x7fffu));
                const uint32_t b = max(max(x.z & 0x7fffu, x.z >> 16 & 0x7fffu), max(x.w & 0x7fffu, x.w >> 16 & 0x7fffu));
                top = max(top, max(a, b));
              }
            }
          }
          if (set == 0) {
            float down;
            sm.q_factor[units & 1][row] = q_factor(top, p.scale, down);
            auto half2_of = [&](uint32_t w) {
              return pack_f16x2(__uint_as_float(w << 16) * down, __uint_as_float(w & 0xffff0000u) * down);
            };
            if constexpr (LEAN) {
#pragma unroll
              for (int hf = 0; hf < kHalves; ++hf)
#pragma unroll
                for (int q = 0; q < 2; ++q) {
                  uint32_t w[16];
#pragma unroll
                  for (int k = 0; k < 4; ++k) {
                    const uint4 x = qr[hf][(4 * q + k) ^ (row & 7)];
                    w[4 * k] = half2_of(x.x);
                    w[4 * k + 1] = half2_of(x.y);
                    w[4 * k + 2] = half2_of(x.z);
                    w[4 * k + 3] = half2_of(x.w);
                  }
                  tmem_st16(lane_tmem + kColQ + 32 * hf + 16 * q, w);
                }
              arrive(sm.bar_qfree);
              tmem_wait_st();
              tc_fence_before();
            } else {
#pragma unroll
              for (int hf = 0; hf < kHalves; ++hf)
#pragma unroll
                for (int k = 0; k < 8; ++k) {
                  const uint4 x = qr[hf][k ^ (row & 7)];
                  qr[hf][k ^ (row & 7)] = make_uint4(half2_of(x.x), half2_of(x.y), half2_of(x.z), half2_of(x.w));
                }
              fence_proxy_async_smem();
            }
            arrive(sm.bar_q);
          } else {
            ok = wait(sm.bar_q, units & 1);
            if (!ok) break;
          }
          scale = sm.q_factor[units & 1][row];
          ++units;
        }
      }
      if (!empty) {
        const uint32_t buf = c & 1, s_tmem = lane_tmem + 128u * buf;
        ok = wait(sm.bar_s[buf], (c >> 1) & 1);
        if (!ok) break;
        // (a warp without a row that sees a key only keeps the hand-offs going)
        if (!__any_sync(full, seen)) {
          if constexpr (LEAN) arrive(sm.bar_p[buf][half ^ 1]);
          arrive(sm.bar_p[buf][half]);
        } else {
          tc_fence_after();
          // 64 columns of S, the keys that the row does not see at -inf
          uint32_t xs[2][32];
          tmem_ld32(s_tmem + 64 * half, xs[0]);
          tmem_ld32(s_tmem + 64 * half + 32, xs[1]);
          tmem_wait_ld();
          if (!(flags & kFull)) {
            int lo, hi, kse;
            row_keys(lo, hi, kse);
            const int key0 = info.key0 + 64 * half, ks = info.ks;
            const int from = min(max(lo - key0, 0), 64), to = min(max(hi - key0, 0), 64);
#pragma unroll
            for (int wd = 0; wd < 2; ++wd) {
              const int f = min(max(from - 32 * wd, 0), 32), e = min(max(to - 32 * wd, 0), 32);
              uint32_t keep = e > f ? (0xffffffffu >> (32 - (e - f))) << f : 0u;  // bits f .. e-1
              if constexpr (SINKS) {
                const int sf = min(max(ks - key0 - 32 * wd, 0), 32), se = min(max(kse - key0 - 32 * wd, 0), 32);
                keep |= se > sf ? (0xffffffffu >> (32 - (se - sf))) << sf : 0u;
              }
#pragma unroll
              for (int k = 0; k < 32; ++k) xs[wd][k] = (keep >> k) & 1u ? xs[wd][k] : 0xff800000u;
            }
          }
          auto max_of = [&]() {
            float r[8];
#pragma unroll
            for (int k = 0; k < 8; ++k) r[k] = fmax3(__uint_as_float(xs[0][k]), __uint_as_float(xs[0][k + 8]), __uint_as_float(xs[0][k + 16]));
#pragma unroll
            for (int k = 0; k < 8; ++k) r[k] = fmax3(r[k], __uint_as_float(xs[0][k + 24]), __uint_as_float(xs[1][k]));
#pragma unroll
            for (int k = 0; k < 8; ++k) r[k] = fmax3(r[k], __uint_as_float(xs[1][k + 8]), __uint_as_float(xs[1][k + 16]));
#pragma unroll
            for (int k = 0; k < 8; ++k) r[k] = fmaxf(r[k], __uint_as_float(xs[1][k + 24]));
            return fmax3(fmax3(r[0], r[1], r[2]), fmax3(r[3], r[4], r[5]), fmaxf(r[6], r[7]));
          };
          const float mx = max_of() * scale;
          // (by their difference: far from zero the sum of a reference and 15 is not)
          const bool move = seen && mx != -INFINITY && mx - m_ref > kMoveAbove;
          if (__any_sync(full, move)) {
            const float f = move && m_ref != -INFINITY ? fast_exp2(m_ref - (mx - kHeadroom)) : 1.0f;
            l_sum *= f;
            if (move) m_ref = mx - kHeadroom;
            if (!(flags & kFirst)) {
              // O holds the piece's earlier tiles once the PV before this one is done
              ok = wait(sm.bar_pv[buf ^ 1], ((c - 1) >> 1) & 1);
              if (!ok) break;
              tc_fence_after();
#pragma unroll 1
              for (int q = 0; q < D / 16; ++q) {
                uint32_t o[16];
                tmem_ld16(o_tmem + 16 * q, o);
                tmem_wait_ld();
#pragma unroll
                for (int k = 0; k < 16; ++k) o[k] = __float_as_uint(__uint_as_float(o[k]) * f);
                tmem_st16(o_tmem + 16 * q, o);
              }
            }
          }
          const float neg_m = m_ref != -INFINITY ? -m_ref : 0.f;
          const unsigned long long sc2 = f32x2(scale, scale), nm2 = f32x2(neg_m, neg_m), zero2 = f32x2(0.f, 0.f);
          unsigned long long acc[4] = {f32x2(0.f, 0.f), f32x2(0.f, 0.f), f32x2(0.f, 0.f), f32x2(0.f, 0.f)};
          if constexpr (LEAN) {
            // the keys of the other half of the lanes
            const uint32_t none[16] = {};
            tmem_st16(s_tmem + 64 * (1 - half), none);
            tmem_st16(s_tmem + 64 * (1 - half) + 16, none);
          }
#pragma unroll
          for (int q = 0; q < 2; ++q) {
            uint32_t pk[16];
#pragma unroll
            for (int k = 0; k < 16; ++k) {
              // Scores are rounded before the reference is taken off, as it was:
              // far from zero a product that is not would differ from it by more
              // than an exponent holds.  (In one step 1 to 2% faster; by a
              // branch that only such rows take, slower than by two steps.)
              float e0, e1;
              const unsigned long long s2 = fma_f32x2(f32x2(__uint_as_float(xs[q][2 * k]), __uint_as_float(xs[q][2 * k + 1])), sc2, zero2);
              f32x2_split(add_f32x2(s2, nm2), e0, e1);
              const float p0 = fast_exp2(e0), p1 = fast_exp2(e1);
              acc[k & 3] = add_f32x2(acc[k & 3], f32x2(p0, p1));
              pk[k] = pack_f16x2(p0, p1);
            }
            tmem_st16(s_tmem + 64 * half + 16 * q, pk);
          }
          tmem_wait_st();
          tc_fence_before();
          if constexpr (LEAN) arrive(sm.bar_p[buf][half ^ 1]);
          arrive(sm.bar_p[buf][half]);
          float s0, s1;
          f32x2_split(add_f32x2(add_f32x2(acc[0], acc[1]), add_f32x2(acc[2], acc[3])), s0, s1);
          l_sum += s0 + s1;
        }
        ++c;
      }
      if (flags & kLastPiece) pdl_launch_next();
      if (!(flags & kLast)) {
        arrive(sm.bar_infofree[it % kInfos]);
        continue;
      }

      // ---- epilogue: the sets' sums, and half the columns of O for each set
      // (a sum that is NaN is passed on, not hidden)
      const bool bad = flags & kBad, part = flags & kPart, row_exists = tl < p.tb && tl < info.ntok;
      const size_t out_row = static_cast<size_t>(info.tok0 + (row_exists ? tl : 0)) * p.a.Hq + info.kvh * p.g + hl;
      arrive(sm.bar_infofree[it % kInfos]);
      float M = -INFINITY, L = 0.f, mine = 0.f, theirs = 0.f;
      if (!empty) {
        auto& ml = sm.ml[units & 1];
        ml[set][row] = make_float2(m_ref, l_sum);
        arrive(sm.bar_meet);
        ok = wait(sm.bar_meet, (units - 1) & 1);
        ok = ok && wait(sm.bar_pv[(c - 1) & 1], ((c - 1) >> 1) & 1);
        if (!ok) break;
        tc_fence_after();
        const float2 x = ml[LEAN ? 0 : set ^ 1][LEAN ? row ^ 64 : row];
        M = fmaxf(m_ref, x.x);
        const float ref = M == -INFINITY ? 0.f : M;
        mine = fast_exp2(m_ref - ref);
        theirs = fast_exp2(x.x - ref);
        L = fmaf(mine, l_sum, theirs * x.y);
      }
      const bool any = !empty && seen && L != 0.f && !bad;
      const float norm = !any ? 0.f : part ? 1.f : p.c.v_unit / L;
      mine *= norm;
      theirs *= norm;
      const int entry = static_cast<int>(blockIdx.x) * 2 + (flags & kSlot1 ? 1 : 0);
      uint4* orow = reinterpret_cast<uint4*>(static_cast<uint8_t*>(p.a.out) + out_row * (2 * D));
#pragma unroll 1
      for (int q = LEAN ? 0 : set * (D / 32); q < (LEAN ? D / 16 : (set + 1) * (D / 32)); ++q) {
        float o[16];
        {
          uint32_t a[16], b[16];
          if (!empty) {
            tmem_ld16(o_tmem + 16 * q, a);
            if constexpr (!LEAN) tmem_ld16(lane_tmem + kColO + 128u * (set ^ 1) + 16 * q, b);
            tmem_wait_ld();
          }
#pragma unroll
          for (int k = 0; k < 16; ++k) {
            o[k] = empty ? 0.f : __uint_as_float(a[k]) * mine;
            if constexpr (!LEAN) o[k] = empty ? 0.f : fmaf(__uint_as_float(b[k]), theirs, o[k]);
          }
        }
        if (!empty && q == (LEAN ? D / 16 : (set + 1) * (D / 32)) - 1) {
          // O may be overwritten by the next unit's first PV
          tc_fence_before();
          arrive(sm.bar_ofree);
        }
        if constexpr (LEAN) {
          // the upper lanes' share goes to the lower ones
          if (!empty) {
            const uint32_t buf = turns & 1, use = turns >> 1;
            float(*to)[kRows / 2] = sm.o[buf];
            if (upper) {
              if (use > 0) ok = ok && wait(sm.bar_xfree[buf], (use - 1) & 1);
#pragma unroll
              for (int k = 0; k < 16; ++k) to[k][ur] = o[k];
              arrive(sm.bar_x[buf]);
            } else {
              ok = ok && wait(sm.bar_x[buf], use & 1);
#pragma unroll
              for (int k = 0; k < 16; ++k) o[k] += to[k][ur];
              arrive(sm.bar_xfree[buf]);
            }
            ++turns;
          }
          if (upper) continue;
        }
        if (!row_exists) continue;
        if (part) {
#pragma unroll
          for (int k = 0; k < 4; ++k)
            *partial_o<D>(p, entry, 4 * q + k, ur) =
                any ? make_float4(o[4 * k], o[4 * k + 1], o[4 * k + 2], o[4 * k + 3]) : make_float4(0.f, 0.f, 0.f, 0.f);
        } else {
          uint32_t wv[8];
#pragma unroll
          for (int e = 0; e < 8; ++e) wv[e] = any ? pack_bf16x2(o[2 * e], o[2 * e + 1]) : 0u;
          orow[2 * q] = make_uint4(wv[0], wv[1], wv[2], wv[3]);
          orow[2 * q + 1] = make_uint4(wv[4], wv[5], wv[6], wv[7]);
        }
      }
      if (row_exists && set == 0 && !upper) {
        if (part) *partial_ml<D>(p, entry, ur) = make_float2(any ? M : -INFINITY, any ? L : bad ? -1.f : 0.f);
        if (!part && p.a.lse) p.a.lse[out_row] = any ? (M + log2f(L)) * kLn2 : -INFINITY;
      }
    }
    if (!ok) give_up();
  }
  tc_fence_before();
  __syncthreads();
  if (warp == kWarpS) {
    tc_fence_after();
    tmem_dealloc(tmem, kTmemCols);
  }
}

// Merge of cut units: block (c - 1, y) takes run boundary c and, of its unit's
// query rows, every gridDim.y-th group of 8; a thread owns four columns of a
// row (8 rows x 16 bytes of a partial are one line).
template <int D>
__global__ void __launch_bounds__(2 * D) chunk_q4_tc_merge_kernel(const __grid_constant__ Q4TcParams p) {
  pdl_wait();
  pdl_launch_next();
  const Record rec = records<D>(p)[blockIdx.x + 1];
  const int np = rec.c1 - rec.c0 + 1, rows = rec.ntok * p.g;
  const int r8 = threadIdx.x & 7, col4 = threadIdx.x >> 3;
  for (int row = blockIdx.y * 8 + r8; row < rows; row += gridDim.y * 8) {
    auto entry = [&](int j) { return (rec.c0 + j) * 2 + (j == 0 ? rec.slot : 0); };
    float M = -INFINITY, L = 0.f;
    bool bad = false;
#pragma unroll 4
    for (int j = 0; j < np; ++j) {
      const float2 ml = *partial_ml<D>(p, entry(j), row);
      if (ml.y != 0.f) M = fmaxf(M, ml.x);
      bad |= ml.y == -1.f;
    }
    float4 acc = make_float4(0.f, 0.f, 0.f, 0.f);
#pragma unroll 4
    for (int j = 0; j < np; ++j) {
      const float2 ml = *partial_ml<D>(p, entry(j), row);
      const float4 o = *partial_o<D>(p, entry(j), col4, row);
      const float w = ml.y != 0.f && !bad ? exp2f(ml.x - (M == -INFINITY ? 0.f : M)) : 0.f;
      L = fmaf(w, ml.y, L);
      acc.x = fmaf(w, o.x, acc.x);
      acc.y = fmaf(w, o.y, acc.y);
      acc.z = fmaf(w, o.z, acc.z);
      acc.w = fmaf(w, o.w, acc.w);
    }
    const bool any = L != 0.f && !bad;
    const float inv = any ? p.c.v_unit / L : 0.f;
    const int tl = row / p.g;
    const size_t out_row = static_cast<size_t>(rec.tok0 + tl) * p.a.Hq + rec.kvh * p.g + (row - tl * p.g);
    reinterpret_cast<uint2*>(static_cast<__nv_bfloat16*>(p.a.out) + out_row * D)[col4] =
        any ? make_uint2(pack_bf16x2(acc.x * inv, acc.y * inv), pack_bf16x2(acc.z * inv, acc.w * inv)) : make_uint2(0u, 0u);
    if (p.a.lse && col4 == 0) p.a.lse[out_row] = any ? (M + log2f(L)) * kLn2 : -INFINITY;
  }
}

template <int D, bool SINKS, bool LEAN>
cudaError_t launch_lean(Q4TcParams p, int num_sms, EncodeTiledFn encode, cudaStream_t stream) {
  p.tb = (LEAN ? kRows / 2 : kRows) / p.g;
  CUtensorMap tq;
  const cuuint64_t dims[3] = {D, static_cast<cuuint64_t>(p.a.Hq), static_cast<cuuint64_t>(p.a.T)};
  const cuuint64_t strides[2] = {D * 2ull, static_cast<cuuint64_t>(p.a.q_stride) * 2ull};
  const cuuint32_t box[3] = {64u, static_cast<cuuint32_t>(p.g), static_cast<cuuint32_t>(p.tb)};
  if (!make_bf16_map(encode, &tq, p.a.q, 3, dims, strides, box)) return cudaErrorInvalidValue;
  constexpr size_t bytes = smem_bytes<D, LEAN>();
  static std::mutex mu;
  static bool done[64] = {};
  int dev = 0;
  cudaError_t e = cudaGetDevice(&dev);
  if (e != cudaSuccess) return e;
  if (dev < 0 || dev >= 64) return cudaErrorInvalidDevice;
  {
    std::lock_guard<std::mutex> lk(mu);
    if (!done[dev]) {
      e = cudaFuncSetAttribute(chunk_q4_tc_kernel<D, SINKS, LEAN>, cudaFuncAttributeMaxDynamicSharedMemorySize,
                               static_cast<int>(bytes));
      if (e != cudaSuccess) return e;
      done[dev] = true;
    }
  }
  p.ctas = num_sms;
  e = launch_overlapped(chunk_q4_tc_kernel<D, SINKS, LEAN>, dim3(static_cast<unsigned>(p.ctas)), dim3(kThreads), bytes,
                        stream, 1u, tq, p);
  if (e != cudaSuccess || p.ctas == 1) return e;
  return launch_overlapped(chunk_q4_tc_merge_kernel<D>, dim3(static_cast<unsigned>(p.ctas - 1), 8u), dim3(2 * D), 0,
                           stream, 1u, p);
}

// Lean units where a sequence has up to 64 query rows a KV head on average.
template <int D, bool SINKS>
cudaError_t launch_d(const Q4TcParams& p, int num_sms, EncodeTiledFn encode, cudaStream_t stream) {
  const bool lean = p.g <= kRows / 2 && static_cast<long long>(p.a.T) * p.g <= static_cast<long long>(kRows / 2) * p.a.Bt;
  return lean ? launch_lean<D, SINKS, true>(p, num_sms, encode, stream)
              : launch_lean<D, SINKS, false>(p, num_sms, encode, stream);
}

}  // namespace

size_t chunk_q4_tc_workspace_bytes(int d, int num_sms) {
  return static_cast<size_t>(num_sms) * (2ull * kRows * (d + 2) * sizeof(float) + sizeof(Record));
}

cudaError_t launch_chunk_attention_q4_tc(const ChunkArgs& a, const simsd_q4_cache& c, int num_sms, EncodeTiledFn encode,
                                         cudaStream_t stream) {
  Q4TcParams p{};
  p.a = a;
  p.c = c;
  p.g = a.Hq / a.Hkv;
  p.sub = a.page_size % kTile == 0 ? kTile : std::min(a.page_size, 64);
  p.scale = score_scale(a.scale, c.k_unit);
  if (a.sinks > 0) return a.d == 128 ? launch_d<128, true>(p, num_sms, encode, stream) : launch_d<64, true>(p, num_sms, encode, stream);
  return a.d == 128 ? launch_d<128, false>(p, num_sms, encode, stream) : launch_d<64, false>(p, num_sms, encode, stream);
}

}  // namespace simsd
