// chunk_attention_q4.cu -- attention of single tokens and short chunks over a
// paged cache in 4 bits (Sec. 3.3: the prefix is read from a KV cache).
//
// Mathematics.  As in chunk_attention_tc.cu: one pass over the keys with a
// running reference and sum (fp32; q4_tiles.cuh says where the reference lies
// and when it moves).  Keys and values are scale times code: 6
// significant bits, exact in fp16.  q is multiplied by a power of two that
// brings its row's largest component to [1, 4) and is then exact in fp16 too,
// but for components below 2^-14 of the largest (off by 2^-25 of it at most).
// Probabilities are rounded to fp16, their sum is not; products are
// accumulated in fp32.
//
// Few query rows meet many keys, so the keys are the wide side of the
// products: S^T = K Q^T and O^T += V^T P^T with 16 keys (channels) by 8 rows
// a matrix instruction, mma.sync m16n8k16.  Its operands come from registers:
// a thread turns 16 bytes of codes into the fragments of 8 instructions
// (convert, times scale) without a way through shared memory, where the
// tcgen05 instructions would have them, 64 KB a tile written and read again.
// The order of components within a product and of keys within 16 is free, so
// each thread takes the components, channels and keys that lie together.
//
// Work.  The walk of chunk_walk.cuh over units of (KV head, sequence, up to
// 16 query rows).  One warp walks the run and brings the tiles' codes and
// scales (128 keys, 18 KB) by bulk copies, each a page's contiguous rows of a
// head; four warps share a tile's keys, each with a softmax of its
// own, merged at the end of a unit through shared memory.  A unit cut by a
// run's end leaves partial (O, m, l), which a second launch merges.
//
// Bound: what twelve warps an SM can hide of their latencies: some 280
// instructions for 16 keys (64 conversions and 64 products with a scale among
// them) take 53% of the issue slots, the reads 56% of DRAM's rate.  64 single
// tokens over 2048 to 8192 rows, 32 heads on 8 of 128, read 377 MB in 79 us (4.8
// TB/s).
//
// Every mbarrier wait is bounded; after one expires the CTA raises
// SIMSD_EW_TIMEOUT, every warp leaves its loop and the copies in flight are
// waited for.
#include <cuda_bf16.h>
#include <cuda_fp16.h>
#include <cuda_runtime.h>

#include <algorithm>
#include <mutex>

#include "common.cuh"
#include "kernels.h"
#include "q4_tiles.cuh"

namespace simsd {
namespace {

constexpr int kTile = kQ4Tile;
constexpr int kMaxSeqs = 8192;  // their tile counts fit the ring
constexpr float kNoReference = -3.402823466e38f;  // of rows that have seen no key: the lowest number, below every score
constexpr float kLn2 = 0.6931471805599453f;

struct Q4Params {
  ChunkArgs a;
  simsd_q4_cache c;
  int g, ub, ctas;    // heads per KV head, tokens of a unit, grid size
  int sub;            // keys per copy: a page, or part of one
  ScoreScale scale;   // of scores, in log2 units
};

// NB blocks of 8 query rows.  CTAs of four warps, whose 32 keys a tile pay for
// what a tile costs beside its products; as many an SM as registers allow.
// One block, 64 single tokens over 2048 to 8192 rows: 79 us (77 when this was
// chosen; four CTAs, with 96
// registers a thread, 81; eight warps of 16 keys, two CTAs, then 113 for 87).  Two,
// 32 blocks of 4 tokens over these: 67 us (eight warps of 16 keys, one CTA, 84).
template <int D, int NB>
struct Cfg {
  static constexpr int kRows = 8 * NB;  // query rows of a unit
  static constexpr int kWarps = 4;
  static constexpr int kThreads = 32 * (kWarps + 1);
  static constexpr int kWarpKeys = kTile / kWarps;
  static constexpr int kCtas = NB == 1 ? 3 : 2;  // an SM
  static constexpr int kStages = (NB == 1 ? 3 : 4) * (128 / D);
};

template <int D, int NB>
struct SmemQ4 {
  using C = Cfg<D, NB>;
  Stage<D> ring[C::kStages];
  __nv_bfloat16 q[2][C::kRows * D];
  float4 fold[C::kWarps / 2][NB * (D / 16)][32];  // O of half the warps
  float2 ml[C::kWarps][8 * NB];
  float2 fin[C::kRows];
  TileInfo info[C::kStages];
  uint64_t bar_full[C::kStages], bar_free[C::kStages], bar_qfree[2], bar_merge[3];
  int abort_flag;
};

__device__ __forceinline__ void mma16816(float (&c)[4], uint32_t a0, uint32_t a1, uint32_t a2, uint32_t a3,
                                         uint32_t b0, uint32_t b1) {
  asm volatile(
      "mma.sync.aligned.m16n8k16.row.col.f32.f16.f16.f32 {%0,%1,%2,%3}, {%4,%5,%6,%7}, {%8,%9}, {%0,%1,%2,%3};"
      : "+f"(c[0]), "+f"(c[1]), "+f"(c[2]), "+f"(c[3])
      : "r"(a0), "r"(a1), "r"(a2), "r"(a3), "r"(b0), "r"(b1));
}
// The first of a sum's.
__device__ __forceinline__ void mma16816_first(float (&c)[4], uint32_t a0, uint32_t a1, uint32_t a2, uint32_t a3,
                                               uint32_t b0, uint32_t b1) {
  asm volatile(
      "mma.sync.aligned.m16n8k16.row.col.f32.f16.f16.f32 {%0,%1,%2,%3}, {%4,%5,%6,%7}, {%8,%9}, {%10,%10,%10,%10};"
      : "=f"(c[0]), "=f"(c[1]), "=f"(c[2]), "=f"(c[3])
      : "r"(a0), "r"(a1), "r"(a2), "r"(a3), "r"(b0), "r"(b1), "f"(0.f));
}
// The transpose of an 8 x 8 matrix of fp16, two neighbours of a row a thread.
__device__ __forceinline__ uint32_t transpose8(uint32_t x) {
  uint32_t y;
  asm volatile("movmatrix.sync.aligned.m8n8.trans.b16 %0, %1;" : "=r"(y) : "r"(x));
  return y;
}
// Partial results: O (without the values' unit) [entries][RB][D], then (m, l)
// [entries][RB], entry cta * 2 + slot, m in log2 units, l = -1 where a page id
// of the piece is out of range; then one Record per run boundary.
template <int D, int RB>
__device__ __forceinline__ float* partial_o(const Q4Params& p, int entry, int row) {
  return static_cast<float*>(p.a.workspace) + (static_cast<size_t>(entry) * RB + row) * D;
}
template <int D, int RB>
__device__ __forceinline__ float2* partial_ml(const Q4Params& p, int entry, int row) {
  return reinterpret_cast<float2*>(partial_o<D, RB>(p, 2 * p.ctas, 0)) + static_cast<size_t>(entry) * RB + row;
}
template <int D, int RB>
__device__ __forceinline__ Record* records(const Q4Params& p) {
  return reinterpret_cast<Record*>(partial_ml<D, RB>(p, 2 * p.ctas, 0));
}

// A thread's codes of K: the D / 4 components (D / 8 bytes) from t D / 4 on.
template <int D>
struct KCodes {
  uint32_t w[D / 32];
  uint32_t s;  // their scales, a byte each
};
template <int D>
__device__ __forceinline__ KCodes<D> load_k(const Stage<D>& st, int key, int t) {
  KCodes<D> c;
  if constexpr (D == 128) {
    const uint4 v = *reinterpret_cast<const uint4*>(&st.kc[key * 64 + 16 * t]);
    c.w[0] = v.x, c.w[1] = v.y, c.w[2] = v.z, c.w[3] = v.w;
    c.s = *reinterpret_cast<const uint16_t*>(&st.ks[key * 8 + 2 * t]);
  } else {
    const uint2 v = *reinterpret_cast<const uint2*>(&st.kc[key * 32 + 8 * t]);
    c.w[0] = v.x, c.w[1] = v.y;
    c.s = st.ks[key * 4 + t];
  }
  return c;
}
// The codes of V of one key, D / 8 channels from g D / 8 on.
template <int D>
struct VCodes {
  uint32_t w[D / 64];
};
template <int D>
__device__ __forceinline__ VCodes<D> load_v(const Stage<D>& st, int key, int g) {
  VCodes<D> c;
  if constexpr (D == 128) {
    const uint2 v = *reinterpret_cast<const uint2*>(&st.vc[key * 64 + 8 * g]);
    c.w[0] = v.x, c.w[1] = v.y;
  } else {
    c.w[0] = *reinterpret_cast<const uint32_t*>(&st.vc[key * 32 + 4 * g]);
  }
  return c;
}

template <int D, int NB, bool SINKS>
__global__ void __launch_bounds__(Cfg<D, NB>::kThreads, Cfg<D, NB>::kCtas) chunk_q4_kernel(const __grid_constant__ Q4Params p) {
  using C = Cfg<D, NB>;
  using Smem = SmemQ4<D, NB>;
  constexpr int RB = C::kRows, kStages = C::kStages, kWarps = C::kWarps;
  extern __shared__ uint8_t smem_raw[];
  // (an offset from the array: through a number the compiler no longer knows that it is shared memory)
  Smem& sm = *reinterpret_cast<Smem*>(smem_raw + (0u - smem_u32(smem_raw) & 127u));
  static_assert(sizeof(sm.ring) >= kMaxSeqs * 4, "the ring holds the tile counts of all sequences");
  volatile int* abort_flag = &sm.abort_flag;
  const unsigned full = 0xffffffffu;
  const int tid = threadIdx.x, warp = tid >> 5, lane = tid & 31;
  if (tid == 0) {
    sm.abort_flag = 0;
    for (int s = 0; s < kStages; ++s) {
      mbar_init(smem_u32(&sm.bar_full[s]), 1);
      mbar_init(smem_u32(&sm.bar_free[s]), kWarps);
    }
    mbar_init(smem_u32(&sm.bar_qfree[0]), kWarps);
    mbar_init(smem_u32(&sm.bar_qfree[1]), kWarps);
    for (int i = 0; i < 3; ++i) mbar_init(smem_u32(&sm.bar_merge[i]), kWarps);
    fence_mbar_init();
  }
  pdl_wait();
  int32_t* tiles = reinterpret_cast<int32_t*>(&sm.ring[0]);
  plan_tiles<SINKS, kTile, C::kThreads>(p.a, p.ub, tiles);
  Place start{0, 0, 0, 0};
  int total = 0;
  ChunkSeq seq{};
  if (warp == kWarps) start = plan_start<SINKS, kTile>(p.a, p.ub, p.ctas, tiles, total, seq);
  fence_proxy_async_smem();  // the ring was written here and is filled by bulk copies next
  __syncthreads();
  auto give_up = [&]() {
    if (lane == 0) {
      raise_error(p.a.err_word, SIMSD_EW_TIMEOUT);
      *abort_flag = 1;
    }
  };

  if (warp == kWarps) {
    // -------------------------------------------------------- walk and copies
    TileWalk<D, SINKS> tw;
    tw.sizes(p.ub, p.sub, p.a.page_size);
    tw.k.begin(p.a, p.ub, p.ctas, start, seq, total);
    uint32_t it = 0, units = 0;  // tiles passed on, of them with a Q
    bool ok = true;
    auto slot_free = [&]() {
      if (it >= kStages) ok = mbar_wait_warp(smem_u32(&sm.bar_free[it % kStages]), ((it / kStages) - 1) & 1, abort_flag);
      return ok;
    };
    while (ok && tw.next_piece(p.a)) {
      for (int i = 0; i < tw.piece.take; ++i) {
        const uint32_t st = it % kStages;
        tw.tile(p.a, i);
        if (!slot_free()) break;
        const bool with_q = i == 0 && !(tw.flags & kEmpty);
        const uint32_t qb = units & 1, q_bytes = static_cast<uint32_t>(p.g * D * 2);
        if (with_q && units >= 2) {
          ok = mbar_wait_warp(smem_u32(&sm.bar_qfree[qb]), ((units >> 1) - 1) & 1, abort_flag);
          if (!ok) break;
        }
        const uint32_t bar = smem_u32(&sm.bar_full[st]);
        const uint32_t bytes = 2 * tw.bytes() + (with_q ? tw.u.ntok * q_bytes : 0u);
        if (lane == 0) {
          sm.info[st] = tw.u;
          mbar_arrive_expect_tx(bar, bytes);
        }
        __syncwarp();
        tw.copy_k(p.c, sm.ring[st], bar);
        tw.copy_v(p.c, sm.ring[st], bar);
        if (with_q) {
          for (int x = lane; x < tw.u.ntok; x += 32)
            bulk_load(smem_u32(&sm.q[qb][x * p.g * D]),
                      static_cast<const __nv_bfloat16*>(p.a.q) + static_cast<long long>(tw.u.tok0 + x) * p.a.q_stride +
                          static_cast<long long>(tw.u.kvh) * p.g * D,
                      q_bytes, bar);
          ++units;
        }
        ++it;
      }
      if (!ok) break;
      tw.k.pop(p.a, p.ub, tw.piece);
    }
    if (ok && slot_free()) {
      // the end of the run
      if (lane == 0) {
        TileInfo u{};
        u.flags = kEnd;
        sm.info[it % kStages] = u;
        mbar_arrive(smem_u32(&sm.bar_full[it % kStages]));
      }
      ++it;
    }
    if (!ok) give_up();
    if (lane == 0 && blockIdx.x > 0) records<D, RB>(p)[blockIdx.x] = boundary_record<SINKS, kTile>(tw.k, p.a, p.ub);
    // every copy must have landed before the CTA may exit
    if (lane == 0)
      for (uint32_t j = it > kStages ? it - kStages : 0; j < it; ++j)
        mbar_wait(smem_u32(&sm.bar_full[j % kStages]), (j / kStages) & 1, nullptr);
    __syncwarp();
    return;
  }

  // ------------------------------------------------------------------ softmax
  const int g = lane >> 2, t = lane & 3;  // the thread's place in the fragments
  const int perm = g ^ ((g >> 1) & 1);    // place of key g among 8: neighbours in pairs, pairs turned in turns
  const int va = (2 * t) ^ (t & 1), vb = (2 * t + 1) ^ (t & 1);
  constexpr int kSteps = D / 16;          // products of 16 components; blocks of 16 channels
  constexpr int G = C::kWarpKeys / 16;
  uint32_t q[NB][kSteps][2];
  // m: the reference that the probabilities are formed against, in log2 units
  float o[NB][kSteps][4], m[NB][2], l[NB][2], rs[NB][2];
  uint32_t units = 0, pieces = 0;
  bool ok = true;
  for (uint32_t it = 0; ok; ++it) {
    const uint32_t st = it % kStages;
    if (!mbar_wait_warp(smem_u32(&sm.bar_full[st]), (it / kStages) & 1, abort_flag)) {
      ok = false;
      break;
    }
    const Stage<D>& s = sm.ring[st];
    const TileInfo& info = sm.info[st];
    const int4 head = *reinterpret_cast<const int4*>(&info);
    const int flags = head.x, key0 = head.y, ntok = head.z, tok0 = head.w;
    if (flags & kEnd) break;
    if (flags & kFirst) {
#pragma unroll
      for (int nb = 0; nb < NB; ++nb) {
#pragma unroll
        for (int k = 0; k < kSteps; ++k) o[nb][k][0] = o[nb][k][1] = o[nb][k][2] = o[nb][k][3] = 0.f;
        m[nb][0] = m[nb][1] = kNoReference;
        l[nb][0] = l[nb][1] = 0.f;
      }
      if (!(flags & kEmpty)) {
        const uint32_t qb = units & 1;
#pragma unroll
        for (int nb = 0; nb < NB; ++nb) {
          // row 8 nb + g: its components from t D / 4 on
          const int row = nb * 8 + g;
          const bool real = row < ntok * p.g;
          uint4 raw[D / 32];
          uint32_t top = 0;
#pragma unroll
          for (int j = 0; j < D / 32; ++j) {
            raw[j] = make_uint4(0u, 0u, 0u, 0u);
            if (real) raw[j] = *reinterpret_cast<const uint4*>(&sm.q[qb][row * D + t * (D / 4) + 8 * j]);
            const uint32_t w[4] = {raw[j].x, raw[j].y, raw[j].z, raw[j].w};
#pragma unroll
            for (int e = 0; e < 4; ++e) top = max(top, max(w[e] & 0x7fffu, w[e] >> 16 & 0x7fffu));
          }
          top = max(top, __shfl_xor_sync(full, top, 1));
          top = max(top, __shfl_xor_sync(full, top, 2));
          float down;
          const float factor = q_factor(top, p.scale, down);
#pragma unroll
          for (int j = 0; j < D / 32; ++j) {
            const uint32_t w[4] = {raw[j].x, raw[j].y, raw[j].z, raw[j].w};
#pragma unroll
            for (int e = 0; e < 4; ++e)
              q[nb][2 * j + e / 2][e & 1] = pack_f16x2(__uint_as_float(w[e] << 16) * down, __uint_as_float(w[e] & 0xffff0000u) * down);
          }
          // scores of rows 2t and 2t + 1, whose q lies with lanes of g = 2t and 2t + 1
          rs[nb][0] = __shfl_sync(full, factor, 8 * t);
          rs[nb][1] = __shfl_sync(full, factor, 8 * t + 4);
        }
        __syncwarp();
        if (lane == 0) mbar_arrive(smem_u32(&sm.bar_qfree[qb]));
        ++units;
      }
    }
    if (!(flags & kEmpty)) {
      const bool masked = !(flags & kFull);
      if (masked) {
        // values of rows that no token of the unit sees may be anything: their
        // scales, which only this warp reads, are set to 0
        const int lo = info.lo, se = info.se, w0 = info.w0, hi = info.hi;
#pragma unroll 1
        for (int i = warp * C::kWarpKeys + lane; i < (warp + 1) * C::kWarpKeys; i += 32) {
          const int key = key0 + i;
          if (key >= lo && key < hi && (!SINKS || key < se || key >= w0)) continue;
          uint32_t* row = reinterpret_cast<uint32_t*>(&sm.ring[st].vs[i * (D / kQ4Group)]);
#pragma unroll
          for (int k = 0; k < D / kQ4Group / 4; ++k) row[k] = 0u;
        }
        fence_proxy_async_smem();  // (the slot is filled by bulk copies next)
        __syncwarp();
      }
      const int kb = warp * C::kWarpKeys;
      // S^T of keys perm(g) and 8 + perm(g) of each 16, rows 2t and 2t + 1
      float sc[G][NB][4];
#pragma unroll
      for (int u = 0; u < G; ++u) {
        const KCodes<D> ka = load_k(s, kb + 16 * u + perm, t), kc = load_k(s, kb + 16 * u + 8 + perm, t);
        const uint32_t x = q4_scale_pair(ka.s), y = q4_scale_pair(kc.s);
        uint32_t sa[2], sb[2];
        sa[0] = __byte_perm(x, 0, 0x1010);
        sb[0] = __byte_perm(y, 0, 0x1010);
        sa[1] = __byte_perm(x, 0, 0x3232);  // (128 components: a thread's lie in two groups)
        sb[1] = __byte_perm(y, 0, 0x3232);
#pragma unroll
        for (int k = 0; k < kSteps; ++k) {
          const uint32_t wa = ka.w[k / 2], wb = kc.w[k / 2], fa = sa[k / 4], fb = sb[k / 4];
          const uint32_t a0 = mul_f16x2(k & 1 ? q4_pair<2>(wa) : q4_pair<0>(wa), fa);
          const uint32_t a1 = mul_f16x2(k & 1 ? q4_pair<2>(wb) : q4_pair<0>(wb), fb);
          const uint32_t a2 = mul_f16x2(k & 1 ? q4_pair<3>(wa) : q4_pair<1>(wa), fa);
          const uint32_t a3 = mul_f16x2(k & 1 ? q4_pair<3>(wb) : q4_pair<1>(wb), fb);
#pragma unroll
          for (int nb = 0; nb < NB; ++nb) {
            if (k == 0)
              mma16816_first(sc[u][nb], a0, a1, a2, a3, q[nb][k][0], q[nb][k][1]);
            else
              mma16816(sc[u][nb], a0, a1, a2, a3, q[nb][k][0], q[nb][k][1]);
          }
        }
      }
      if (masked) {
        ChunkSeq cs;
        cs.n = info.n;
        cs.C = info.C;
        cs.ks = info.ks;
#pragma unroll
        for (int nb = 0; nb < NB; ++nb)
#pragma unroll
          for (int e = 0; e < 2; ++e) {
            const int tl = info.i0 + min((nb * 8 + 2 * t + e) / p.g, ntok - 1);
            const int lo = key_lo(p.a, cs, tl), hi = key_hi(p.a, cs, tl), se = SINKS ? sink_end(p.a, cs, hi) : 0;
#pragma unroll
            for (int u = 0; u < G; ++u)
#pragma unroll
              for (int h = 0; h < 2; ++h) {
                const int key = key0 + kb + 16 * u + 8 * h + perm;
                if (!((key >= lo && key < hi) || (SINKS && key >= cs.ks && key < se))) sc[u][nb][2 * h + e] = -INFINITY;
              }
          }
      }
      // exponents; those of rows whose reference has to move again.  Scores are
      // rounded before the reference is taken off, as it was: far from zero a
      // product that is not would differ from it by more than an exponent holds
      float pr[G][NB][4];
      bool above = false;
#pragma unroll
      for (int u = 0; u < G; ++u)
#pragma unroll
        for (int nb = 0; nb < NB; ++nb)
#pragma unroll
          for (int e = 0; e < 4; ++e) {
            sc[u][nb][e] = __fmul_rn(sc[u][nb][e], rs[nb][e & 1]);
            pr[u][nb][e] = sc[u][nb][e] - m[nb][e & 1];
            above |= pr[u][nb][e] > kMoveAbove;
          }
      if (__any_sync(full, above)) {
#pragma unroll
        for (int nb = 0; nb < NB; ++nb)
#pragma unroll
          for (int e = 0; e < 2; ++e) {
            float mx = kNoReference;
#pragma unroll
            for (int u = 0; u < G; ++u) mx = fmaxf(mx, fmaxf(sc[u][nb][e], sc[u][nb][e + 2]));
            mx = fmaxf(mx, __shfl_xor_sync(full, mx, 4));
            mx = fmaxf(mx, __shfl_xor_sync(full, mx, 8));
            mx = fmaxf(mx, __shfl_xor_sync(full, mx, 16));
            mx = fmaxf(m[nb][e], mx - kHeadroom);
            const float f = fast_exp2(m[nb][e] - mx);
            m[nb][e] = mx;
            l[nb][e] *= f;
#pragma unroll
            for (int k = 0; k < kSteps; ++k) {
              o[nb][k][e] *= f;
              o[nb][k][e + 2] *= f;
            }
#pragma unroll
            for (int u = 0; u < G; ++u) {
              pr[u][nb][e] = sc[u][nb][e] - mx;
              pr[u][nb][e + 2] = sc[u][nb][e + 2] - mx;
            }
          }
      }
      uint32_t pb[G][NB][2];
#pragma unroll
      for (int u = 0; u < G; ++u)
#pragma unroll
        for (int nb = 0; nb < NB; ++nb) {
#pragma unroll
          for (int e = 0; e < 4; ++e) pr[u][nb][e] = fast_exp2(pr[u][nb][e]);
          l[nb][0] += pr[u][nb][0] + pr[u][nb][2];
          l[nb][1] += pr[u][nb][1] + pr[u][nb][3];
          pb[u][nb][0] = transpose8(pack_f16x2(pr[u][nb][0], pr[u][nb][1]));
          pb[u][nb][1] = transpose8(pack_f16x2(pr[u][nb][2], pr[u][nb][3]));
        }
#pragma unroll
      for (int u = 0; u < G; ++u) {
        // V^T of keys va, vb and 8 + va, 8 + vb, channels from g D / 8 on (all of one scale)
        const int kv = kb + 16 * u;
        const VCodes<D> v0 = load_v(s, kv + va, g), v1 = load_v(s, kv + vb, g);
        const VCodes<D> v2 = load_v(s, kv + 8 + va, g), v3 = load_v(s, kv + 8 + vb, g);
        constexpr int kScales = D / kQ4Group;
        const int vg = D == 128 ? g : g >> 1;
        const uint32_t s01 = s.vs[(kv + va) * kScales + vg] | s.vs[(kv + vb) * kScales + vg] << 8;
        const uint32_t s23 = s.vs[(kv + 8 + va) * kScales + vg] | s.vs[(kv + 8 + vb) * kScales + vg] << 8;
        const uint32_t f01 = q4_scale_pair(s01), f23 = q4_scale_pair(s23);
        constexpr uint32_t kLow = 0x0f0f0f0fu;
#pragma unroll
        for (int i = 0; i < D / 64; ++i) {
          // bytes of two keys' codes of one channel
          const uint32_t e01 = (v0.w[i] & kLow) | (v1.w[i] << 4 & ~kLow), d01 = (v0.w[i] >> 4 & kLow) | (v1.w[i] & ~kLow);
          const uint32_t e23 = (v2.w[i] & kLow) | (v3.w[i] << 4 & ~kLow), d23 = (v2.w[i] >> 4 & kLow) | (v3.w[i] & ~kLow);
          auto block = [&](int k, uint32_t a0, uint32_t a1, uint32_t a2, uint32_t a3) {
            a0 = mul_f16x2(a0, f01);
            a1 = mul_f16x2(a1, f01);
            a2 = mul_f16x2(a2, f23);
            a3 = mul_f16x2(a3, f23);
#pragma unroll
            for (int nb = 0; nb < NB; ++nb) mma16816(o[nb][k], a0, a1, a2, a3, pb[u][nb][0], pb[u][nb][1]);
          };
          block(4 * i, q4_pair<0>(e01), q4_pair<0>(d01), q4_pair<0>(e23), q4_pair<0>(d23));
          block(4 * i + 1, q4_pair<1>(e01), q4_pair<1>(d01), q4_pair<1>(e23), q4_pair<1>(d23));
          block(4 * i + 2, q4_pair<2>(e01), q4_pair<2>(d01), q4_pair<2>(e23), q4_pair<2>(d23));
          block(4 * i + 3, q4_pair<3>(e01), q4_pair<3>(d01), q4_pair<3>(e23), q4_pair<3>(d23));
        }
      }
    }
    // what the end of a piece needs is read before the slot is given back
    const bool part = flags & kPart, bad = flags & kBad;
    const int kvh = info.kvh, entry = static_cast<int>(blockIdx.x) * 2 + (flags & kSlot1 ? 1 : 0);
    __syncwarp();
    if (lane == 0) mbar_arrive(smem_u32(&sm.bar_free[st]));
    if (flags & kLastPiece) pdl_launch_next();
    if (!(flags & kLast)) continue;

    // ---- the warps' results, merged: maxima and sums first
    const uint32_t par = pieces & 1;
    auto meet = [&](int i) {
      __syncwarp();
      if (lane == 0) mbar_arrive(smem_u32(&sm.bar_merge[i]));
      ok = ok && mbar_wait_warp(smem_u32(&sm.bar_merge[i]), par, abort_flag);
    };
#pragma unroll
    for (int nb = 0; nb < NB; ++nb)
#pragma unroll
      for (int e = 0; e < 2; ++e) {
        float x = l[nb][e];
        x += __shfl_xor_sync(full, x, 4);
        x += __shfl_xor_sync(full, x, 8);
        x += __shfl_xor_sync(full, x, 16);
        if (g == 0) sm.ml[warp][8 * nb + 2 * t + e] = make_float2(m[nb][e], x);
      }
    meet(0);
    if (!ok) break;
#pragma unroll
    for (int nb = 0; nb < NB; ++nb)
#pragma unroll
      for (int e = 0; e < 2; ++e) {
        float M = kNoReference, L = 0.f;
#pragma unroll
        for (int w = 0; w < kWarps; ++w) M = fmaxf(M, sm.ml[w][8 * nb + 2 * t + e].x);
#pragma unroll
        for (int w = 0; w < kWarps; ++w) {
          const float2 x = sm.ml[w][8 * nb + 2 * t + e];
          L = fmaf(fast_exp2(x.x - M), x.y, L);
        }
        const float f = fast_exp2(m[nb][e] - M);
        if (warp == 0 && g == 0) sm.fin[nb * 8 + 2 * t + e] = make_float2(M, L);
#pragma unroll
        for (int k = 0; k < kSteps; ++k) {
          o[nb][k][e] *= f;
          o[nb][k][e + 2] *= f;
        }
      }
    // then O: the upper half of the warps' onto the lower half's, those summed by all
    constexpr int kHalf = kWarps / 2;
    float4(*fold)[32] = sm.fold[warp % kHalf];
    if (warp >= kHalf) {
#pragma unroll
      for (int nb = 0; nb < NB; ++nb)
#pragma unroll
        for (int k = 0; k < kSteps; ++k)
          fold[nb * kSteps + k][lane] = make_float4(o[nb][k][0], o[nb][k][1], o[nb][k][2], o[nb][k][3]);
    }
    meet(1);
    if (!ok) break;
    if (warp < kHalf) {
#pragma unroll
      for (int nb = 0; nb < NB; ++nb)
#pragma unroll
        for (int k = 0; k < kSteps; ++k) {
          float4 x = fold[nb * kSteps + k][lane];
          x.x += o[nb][k][0], x.y += o[nb][k][1], x.z += o[nb][k][2], x.w += o[nb][k][3];
          fold[nb * kSteps + k][lane] = x;
        }
    }
    meet(2);
    if (!ok) break;
    // two blocks of channels (four channels side by side) of two rows a turn
    const int rows = ntok * p.g;
    for (int i = tid; i < NB * (kSteps / 2) * 32; i += 32 * kWarps) {
      const int ln = i & 31, j = i >> 5, k2 = j % (kSteps / 2), nb = j / (kSteps / 2);
      float4 x = make_float4(0.f, 0.f, 0.f, 0.f), y = x;
#pragma unroll
      for (int w = 0; w < kHalf; ++w) {
        const float4 a = sm.fold[w][nb * kSteps + 2 * k2][ln], b = sm.fold[w][nb * kSteps + 2 * k2 + 1][ln];
        x.x += a.x, x.y += a.y, x.z += a.z, x.w += a.w;
        y.x += b.x, y.y += b.y, y.z += b.z, y.w += b.w;
      }
      const int ch = (ln >> 2) * (D / 8) + 4 * k2;
#pragma unroll
      for (int e = 0; e < 2; ++e) {
        const int row = nb * 8 + 2 * (ln & 3) + e;
        if (row >= rows) continue;
        const float2 ml = sm.fin[row];
        // (a sum that is NaN is passed on, not hidden)
        const bool any = ml.y != 0.f && !bad;
        const float o0 = e ? x.y : x.x, o1 = e ? x.w : x.z, o2 = e ? y.y : y.x, o3 = e ? y.w : y.z;
        if (part) {
          *reinterpret_cast<float4*>(partial_o<D, RB>(p, entry, row) + ch) = any ? make_float4(o0, o1, o2, o3) : make_float4(0.f, 0.f, 0.f, 0.f);
          if (ch == 0) *partial_ml<D, RB>(p, entry, row) = make_float2(any ? ml.x : -INFINITY, any ? ml.y : bad ? -1.f : 0.f);
        } else {
          const float inv = any ? p.c.v_unit / ml.y : 0.f;
          const int tl = row / p.g;
          const size_t out_row = static_cast<size_t>(tok0 + tl) * p.a.Hq + kvh * p.g + (row - tl * p.g);
          const __nv_bfloat162 lo2 = __floats2bfloat162_rn(o0 * inv, o1 * inv), hi2 = __floats2bfloat162_rn(o2 * inv, o3 * inv);
          *reinterpret_cast<uint2*>(static_cast<__nv_bfloat16*>(p.a.out) + out_row * D + ch) =
              any ? make_uint2(*reinterpret_cast<const uint32_t*>(&lo2), *reinterpret_cast<const uint32_t*>(&hi2)) : make_uint2(0u, 0u);
          if (p.a.lse && ch == 0) p.a.lse[out_row] = any ? (ml.x + log2f(ml.y)) * kLn2 : -INFINITY;
        }
      }
    }
    ++pieces;
  }
  if (!ok) give_up();
}

// Merge of cut units: block (c - 1, y) takes run boundary c and, of its unit's
// query rows, every gridDim.y-th group of 1024 / D; a thread owns four columns.
template <int D, int RB>
__global__ void __launch_bounds__(256) chunk_q4_merge_kernel(const __grid_constant__ Q4Params p) {
  pdl_wait();
  pdl_launch_next();
  const Record rec = records<D, RB>(p)[blockIdx.x + 1];
  const int np = rec.c1 - rec.c0 + 1, rows = rec.ntok * p.g, ch = 4 * (threadIdx.x % (D / 4));
  for (int row = blockIdx.y * (1024 / D) + threadIdx.x / (D / 4); row < rows; row += gridDim.y * (1024 / D)) {
    auto entry = [&](int j) { return (rec.c0 + j) * 2 + (j == 0 ? rec.slot : 0); };
    float M = -INFINITY, L = 0.f;
    bool bad = false;
#pragma unroll 4
    for (int j = 0; j < np; ++j) {
      const float2 ml = *partial_ml<D, RB>(p, entry(j), row);
      if (ml.y != 0.f) M = fmaxf(M, ml.x);
      bad |= ml.y == -1.f;
    }
    float4 acc = make_float4(0.f, 0.f, 0.f, 0.f);
#pragma unroll 4
    for (int j = 0; j < np; ++j) {
      const float2 ml = *partial_ml<D, RB>(p, entry(j), row);
      const float4 o = *reinterpret_cast<const float4*>(partial_o<D, RB>(p, entry(j), row) + ch);
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
    const __nv_bfloat162 lo2 = __floats2bfloat162_rn(acc.x * inv, acc.y * inv), hi2 = __floats2bfloat162_rn(acc.z * inv, acc.w * inv);
    *reinterpret_cast<uint2*>(static_cast<__nv_bfloat16*>(p.a.out) + out_row * D + ch) =
        any ? make_uint2(*reinterpret_cast<const uint32_t*>(&lo2), *reinterpret_cast<const uint32_t*>(&hi2)) : make_uint2(0u, 0u);
    if (p.a.lse && ch == 0) p.a.lse[out_row] = any ? (M + log2f(L)) * kLn2 : -INFINITY;
  }
}

// Query rows of a unit: 8 where they hold a token's heads and a sequence's rows
// on average, else 16.
int q4_rows(int T, int Bt, int g) { return g <= 8 && static_cast<long long>(T) * g <= 8ll * Bt ? 8 : 16; }
constexpr int q4_ctas(int rows, int num_sms) { return (rows == 8 ? Cfg<128, 1>::kCtas : Cfg<128, 2>::kCtas) * num_sms; }

template <int D, int NB, bool SINKS>
cudaError_t launch_rows(Q4Params p, int num_sms, cudaStream_t stream) {
  using C = Cfg<D, NB>;
  constexpr size_t bytes = sizeof(SmemQ4<D, NB>) + 128;
  static_assert(C::kCtas * (bytes + 1024) <= 228 * 1024, "shared memory of an SM");
  p.ub = C::kRows / p.g;
  p.ctas = C::kCtas * num_sms;
  static std::mutex mu;
  static bool done[64] = {};
  int dev = 0;
  cudaError_t e = cudaGetDevice(&dev);
  if (e != cudaSuccess) return e;
  if (dev < 0 || dev >= 64) return cudaErrorInvalidDevice;
  {
    std::lock_guard<std::mutex> lk(mu);
    if (!done[dev]) {
      e = cudaFuncSetAttribute(chunk_q4_kernel<D, NB, SINKS>, cudaFuncAttributeMaxDynamicSharedMemorySize,
                               static_cast<int>(bytes));
      if (e != cudaSuccess) return e;
      done[dev] = true;
    }
  }
  e = launch_overlapped(chunk_q4_kernel<D, NB, SINKS>, dim3(static_cast<unsigned>(p.ctas)), dim3(C::kThreads), bytes,
                        stream, 1u, p);
  if (e != cudaSuccess || p.ctas == 1) return e;
  return launch_overlapped(chunk_q4_merge_kernel<D, C::kRows>, dim3(static_cast<unsigned>(p.ctas - 1)), dim3(256), 0, stream, 1u, p);
}

template <int D, bool SINKS>
cudaError_t launch_d(const Q4Params& p, int num_sms, cudaStream_t stream) {
  return q4_rows(p.a.T, p.a.Bt, p.g) == 8 ? launch_rows<D, 1, SINKS>(p, num_sms, stream)
                                          : launch_rows<D, 2, SINKS>(p, num_sms, stream);
}

}  // namespace

// By the query rows that a sequence has for a KV head on average.  Up to 16:
// from the registers; up to 768, or 512 of heads of 64: by tiles; more: through
// the image, which costs one pass over the rows but then serves 256 of them a
// tile.  Heads of 128, 32 on 8: 32 sequences of 4096 rows, 20 query rows 95 us
// from the registers (in two blocks of 16) and 84 by tiles; 16 sequences, 256
// query rows 94 us by tiles and 139 through the image, 512 167 and 192, 768 240
// and 246, 1024 313 and 296.  Heads of 64, 28 on 4: 448 80 and 78, 511 97 and 95,
// 672 111 and 98 (by tiles there is no image to be held).
constexpr int kCodesRows = 16;
constexpr int tiles_rows(int d) { return d == 128 ? 768 : 512; }
Q4Way chunk_q4_way(int dtype, int T, int Bt, int Hq, int Hkv, int d) {
  if (dtype != SIMSD_BF16 || Bt > kChunkMaxSeqs) return Q4Way::kImage;
  const int g = Hq / Hkv;
  const long long rows = static_cast<long long>(T) * g;
  if (g <= kCodesRows && rows <= static_cast<long long>(kCodesRows) * Bt && Bt <= kMaxSeqs) return Q4Way::kCodes;
  return g <= 128 && rows <= static_cast<long long>(tiles_rows(d)) * Bt ? Q4Way::kTiles : Q4Way::kImage;
}

size_t chunk_q4_workspace_bytes(int T, int Bt, int Hq, int Hkv, int d, int num_sms) {
  const int rows = q4_rows(T, Bt, Hq / Hkv);
  return static_cast<size_t>(q4_ctas(rows, num_sms)) * (2ull * rows * (d + 2) * sizeof(float) + sizeof(Record));
}

cudaError_t launch_chunk_attention_q4(const ChunkArgs& a, const simsd_q4_cache& c, int num_sms, cudaStream_t stream) {
  Q4Params p{};
  p.a = a;
  p.c = c;
  p.g = a.Hq / a.Hkv;
  p.sub = a.page_size % kTile == 0 ? kTile : std::min(a.page_size, 64);
  p.scale = score_scale(a.scale, c.k_unit);
  if (a.sinks > 0) return a.d == 128 ? launch_d<128, true>(p, num_sms, stream) : launch_d<64, true>(p, num_sms, stream);
  return a.d == 128 ? launch_d<128, false>(p, num_sms, stream) : launch_d<64, false>(p, num_sms, stream);
}

}  // namespace simsd
