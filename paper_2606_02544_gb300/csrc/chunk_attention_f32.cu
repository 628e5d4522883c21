// chunk_attention_f32.cu -- fp32 attention of a chunk of new tokens over the
// paged cache, on the CUDA cores (fp32 throughout, as the fp32 verification).
//
// Mathematics: one pass over the keys with the running maximum and sum of a
// softmax, as in the bf16 kernel.
//
// A unit is (sequence, up to RB query rows of one KV head: the heads of
// RB / g tokens).  Its CTA holds Q in shared memory, streams tiles of 64 keys
// through it (K of the next tile is copied while the softmax and P V of this
// one run, V while its S does) and keeps O in registers: a thread owns RB /
// 16 rows and, of S, 4 columns, of O, d / 16 columns, so a value read from
// shared memory serves 4 to 8 products and the rows' rescaling is local.
// Bound by the FMA pipes where blocks are wide: 4 chunks of 512 tokens over
// 500 to 1000 keys, 32 heads, take 675 us, about 37 TFLOP/s of 74.  Few units
// are split over their keys into nsplit ranges, whose partial (O, m, l) a
// second launch merges.  Few rows have a kernel of their own (below).
#include <cuda_runtime.h>

#include <algorithm>
#include <mutex>

#include "chunk_mask.cuh"
#include "common.cuh"
#include "kernels.h"
#include "ptx.cuh"

namespace simsd {
namespace {

constexpr int kThreads = 256;
constexpr int kTile = 64;  // keys per tile
constexpr int kFewTile = kThreads;  // of the kernel for few rows

struct F32Params {
  ChunkArgs a;
  int g, gb;      // heads per KV head, of a unit
  int hblocks;    // units that the heads of a KV head make
  int tb;         // tokens of a unit
  int nsplit;
  int heads, units;  // CTAs of a token's heads, and of the call's tokens
};

template <int D, int RB>
struct SmemF32 {
  float q[RB][D];
  float k[kTile][D];  // 16-byte chunk c of row r lies at chunk c ^ (r & 7)
  float v[kTile][D];
  float p[RB][kTile];
  uint32_t row[2][kTile];  // per tile parity: the keys' rows in the pool
};

__device__ __forceinline__ void cp_async16(void* dst, const void* src, bool real) {
  // (src-size 0: sixteen zero bytes, nothing is read)
  asm volatile("cp.async.cg.shared.global [%0], [%1], 16, %2;" ::"r"(smem_u32(dst)), "l"(src), "r"(real ? 16 : 0)
               : "memory");
}
__device__ __forceinline__ void cp_async_commit() { asm volatile("cp.async.commit_group;" ::: "memory"); }
template <int N>
__device__ __forceinline__ void cp_async_wait() {
  asm volatile("cp.async.wait_group %0;" ::"n"(N) : "memory");
}

// Partials of split units: O [T][Hq][nsplit][D], then (m, l) [T][Hq][nsplit]
// (m as a score).
template <int D>
__device__ __forceinline__ float* partial_o(const F32Params& p, size_t row, int split) {
  return static_cast<float*>(p.a.workspace) + (row * p.nsplit + split) * D;
}
template <int D>
__device__ __forceinline__ float2* partial_ml(const F32Params& p, size_t row, int split) {
  return reinterpret_cast<float2*>(static_cast<float*>(p.a.workspace) +
                                   static_cast<size_t>(p.a.T) * p.a.Hq * p.nsplit * D) +
         row * p.nsplit + split;
}

// A CTA's share of the call: query rows of one sequence and KV head, and a
// range of key tiles.
struct Unit {
  ChunkSeq s;
  int i0, rows;       // row r: token i0 + r / gb, head h0 + r % gb (if below `heads`)
  int kvh, h0, heads;
  int lo, hi;         // keys that any of the rows sees
  int t_begin, t_end;
  const int32_t* bt;
};

// False: nothing to do.  Called by all threads.
__device__ __forceinline__ bool unit_of(const F32Params& p, const int tile, Unit& u) {
  __shared__ int unit_s[2];
  const ChunkArgs& a = p.a;
  const unsigned full = 0xffffffffu;
  const int tid = threadIdx.x, lane = tid & 31, warp = tid >> 5;
  if (blockIdx.x == 0 && blockIdx.z == 0) {
    uint32_t e = 0;
    for (int b = tid; b < a.Bt; b += kThreads) {
      const ChunkSeq s = chunk_seq(a, b);
      e |= (s.bad_off ? SIMSD_EW_TOKENS : 0u) | (s.bad && s.C > 0 ? SIMSD_EW_PREFIX_LEN : 0u);
    }
    if (e) raise_error(a.err_word, e);
  }
  // heads first, then units from the last down: the later tokens of a chunk
  // see more keys, and what starts last should be short
  const int head = blockIdx.x % p.heads;
  // the unit: sequences in turn, each of ceil(C / tb) units
  if (warp == 0) {
    int at = p.units - 1 - blockIdx.x / p.heads, b = -1, j = 0;
    for (int b0 = 0; b0 < a.Bt && b < 0; b0 += 32) {
      const int n = b0 + lane < a.Bt ? (chunk_of(a.token_start, b0 + lane, a.T).count + p.tb - 1) / p.tb : 0;
      int inc = n;
#pragma unroll
      for (int o = 1; o < 32; o <<= 1) {
        const int y = __shfl_up_sync(full, inc, o);
        if (lane >= o) inc += y;
      }
      const unsigned m = __ballot_sync(full, inc > at);
      if (m) {
        const int k = __ffs(m) - 1;
        b = b0 + k;
        j = at - __shfl_sync(full, inc - n, k);
      } else {
        at -= __shfl_sync(full, inc, 31);
      }
    }
    if (lane == 0) {
      unit_s[0] = b;
      unit_s[1] = j;
    }
  }
  __syncthreads();
  const int b = unit_s[0];
  if (b < 0) return false;
  u.s = chunk_seq(a, b);
  u.i0 = unit_s[1] * p.tb;
  const int i1 = min(u.s.C, u.i0 + p.tb);
  u.kvh = head / p.hblocks;
  u.h0 = u.kvh * p.g + (head - u.kvh * p.hblocks) * p.gb;
  u.heads = min(p.gb, u.kvh * p.g + p.g - u.h0);
  u.rows = (i1 - u.i0) * p.gb;
  u.lo = u.hi = 0;
  if (!u.s.bad) {
    u.lo = key_lo(a, u.s, u.i0);
    u.hi = key_hi(a, u.s, i1 - 1);
  }
  if (u.lo >= u.hi) u.lo = u.hi = 0;
  u.bt = a.block_table + static_cast<size_t>(b) * a.max_pages;
  bool bad = false;
  if (u.hi > u.lo)
    for (int i = u.lo / a.page_size + tid; i <= (u.hi - 1) / a.page_size; i += kThreads)
      bad |= u.bt[i] < 0 || u.bt[i] >= a.num_pages;
  bad = __syncthreads_or(bad);
  if (bad && tid == 0) raise_error(a.err_word, SIMSD_EW_PAGE);
  if (bad) u.hi = u.lo;
  const int T0 = u.lo / tile, nt = u.hi > u.lo ? (u.hi + tile - 1) / tile - T0 : 0;
  u.t_begin = T0 + static_cast<int>(static_cast<long long>(blockIdx.z) * nt / p.nsplit);
  u.t_end = T0 + static_cast<int>(static_cast<long long>(blockIdx.z + 1) * nt / p.nsplit);
  return true;
}

// The keys that row r of the unit sees.
__device__ __forceinline__ void row_keys(const F32Params& p, const Unit& u, int r, int& lo, int& hi) {
  const bool real = r < u.rows && u.hi > u.lo;
  lo = real ? key_lo(p.a, u.s, u.i0 + r / p.gb) : 0;
  hi = real ? key_hi(p.a, u.s, u.i0 + r / p.gb) : 0;
}

// A key's row in the pool (~0: not among [lo, hi); 2^32 rows would be a terabyte).
__device__ __forceinline__ uint32_t pool_row(const F32Params& p, const Unit& u, int key) {
  if (key < u.lo || key >= u.hi) return ~0u;
  const int pi = key / p.a.page_size;
  return (static_cast<uint32_t>(u.bt[pi]) * p.a.Hkv + u.kvh) * p.a.page_size + (key - pi * p.a.page_size);
}

template <int D, int RB>
__global__ void __launch_bounds__(kThreads) chunk_f32_kernel(const __grid_constant__ F32Params p) {
  constexpr int RT = RB / 16;   // rows of a thread
  constexpr int OC = D / 64;    // four-column groups of O of a thread
  extern __shared__ uint4 smem_raw[];
  SmemF32<D, RB>& sm = *reinterpret_cast<SmemF32<D, RB>*>(smem_raw);
  pdl_wait();
  pdl_launch_next();
  const ChunkArgs& a = p.a;
  const unsigned full = 0xffffffffu;
  const int tid = threadIdx.x;
  Unit u;
  if (!unit_of(p, kTile, u)) return;
  const ChunkSeq& s = u.s;
  const int t_begin = u.t_begin, t_end = u.t_end, rows = u.rows, heads = u.heads, h0 = u.h0, i0 = u.i0;

  // where the keys of tile t lie (the page arithmetic once a key, not once a copy)
  auto find_rows = [&](int t) {
    if (tid < kTile) sm.row[t & 1][tid] = pool_row(p, u, t * kTile + tid);
  };
  auto load_tile = [&](int t, bool is_k) {
    const float4* src = static_cast<const float4*>(is_k ? a.k_cache : a.v_cache);
    const int c = tid % (D / 4);
#pragma unroll 4
    for (int r = tid / (D / 4); r < kTile; r += kThreads / (D / 4)) {
      const uint32_t at = sm.row[t & 1][r];
      cp_async16(is_k ? &sm.k[r][4 * (c ^ (r & 7))] : &sm.v[r][4 * c], src + (at == ~0u ? 0 : static_cast<size_t>(at) * (D / 4) + c), at != ~0u);
    }
    cp_async_commit();
  };
  if (t_begin < t_end) find_rows(t_begin);
  __syncthreads();
  if (t_begin < t_end) load_tile(t_begin, true);
  for (int i = tid; i < RB * (D / 4); i += kThreads) {
    const int r = i / (D / 4), c = i - r * (D / 4), tl = r / p.gb, hh = r - tl * p.gb;
    const bool real = r < rows && hh < heads;
    const float4 x = real ? *reinterpret_cast<const float4*>(static_cast<const float*>(a.q) +
                                                            static_cast<long long>(s.start + i0 + tl) * a.q_stride +
                                                            static_cast<long long>(h0 + hh) * D + 4 * c)
                          : make_float4(0.f, 0.f, 0.f, 0.f);
    *reinterpret_cast<float4*>(&sm.q[r][4 * c]) = x;
  }
  if (t_begin < t_end) load_tile(t_begin, false);

  const int tx = tid & 15, ty = tid >> 4;
  int klo[RT], khi[RT];
  float m[RT], l[RT], o[RT][OC][4];
#pragma unroll
  for (int r = 0; r < RT; ++r) {
    row_keys(p, u, ty * RT + r, klo[r], khi[r]);
    m[r] = -INFINITY;
    l[r] = 0.f;
#pragma unroll
    for (int c = 0; c < OC; ++c)
#pragma unroll
      for (int e = 0; e < 4; ++e) o[r][c][e] = 0.f;
  }
  for (int t = t_begin; t < t_end; ++t) {
    cp_async_wait<1>();  // K of this tile (V may be on its way)
    __syncthreads();
    if (t + 1 < t_end) find_rows(t + 1);
    float sc[RT][4];
#pragma unroll
    for (int r = 0; r < RT; ++r)
#pragma unroll
      for (int j = 0; j < 4; ++j) sc[r][j] = 0.f;
#pragma unroll 4
    for (int c = 0; c < D / 4; ++c) {
      float4 kv[4];
#pragma unroll
      for (int j = 0; j < 4; ++j) kv[j] = *reinterpret_cast<const float4*>(&sm.k[tx + 16 * j][4 * (c ^ (tx & 7))]);
#pragma unroll
      for (int r = 0; r < RT; ++r) {
        const float4 qv = *reinterpret_cast<const float4*>(&sm.q[ty * RT + r][4 * c]);
#pragma unroll
        for (int j = 0; j < 4; ++j) {
          sc[r][j] = fmaf(qv.x, kv[j].x, sc[r][j]);
          sc[r][j] = fmaf(qv.y, kv[j].y, sc[r][j]);
          sc[r][j] = fmaf(qv.z, kv[j].z, sc[r][j]);
          sc[r][j] = fmaf(qv.w, kv[j].w, sc[r][j]);
        }
      }
    }
    __syncthreads();  // K has been read by all
    if (t + 1 < t_end)
      load_tile(t + 1, true);
    else
      cp_async_commit();  // (keeps the count of groups)
    // softmax of this thread's rows (sixteen lanes share a row)
#pragma unroll
    for (int r = 0; r < RT; ++r) {
      float mx = -INFINITY;
#pragma unroll
      for (int j = 0; j < 4; ++j) {
        const int key = t * kTile + tx + 16 * j;
        const bool in = key >= klo[r] && key < khi[r];
        sc[r][j] = in ? sc[r][j] * a.scale : -INFINITY;
        mx = fmaxf(mx, sc[r][j]);
      }
#pragma unroll
      for (int w = 8; w > 0; w >>= 1) mx = fmaxf(mx, __shfl_xor_sync(full, mx, w));
      const float m_new = fmaxf(m[r], mx);
      // (nothing seen so far: every weight is zero)
      const float ref = m_new == -INFINITY ? 0.f : m_new;
      const float corr = expf(m[r] - ref);
      float sum = 0.f;
#pragma unroll
      for (int j = 0; j < 4; ++j) {
        const float e = expf(sc[r][j] - ref);
        sum += e;
        sm.p[ty * RT + r][tx + 16 * j] = e;
      }
#pragma unroll
      for (int w = 8; w > 0; w >>= 1) sum += __shfl_xor_sync(full, sum, w);
      l[r] = fmaf(l[r], corr, sum);
      m[r] = m_new;
#pragma unroll
      for (int c = 0; c < OC; ++c)
#pragma unroll
        for (int e = 0; e < 4; ++e) o[r][c][e] *= corr;
    }
    cp_async_wait<1>();  // V of this tile
    __syncthreads();     // (P of a row is written and read by one warp)
#pragma unroll 4
    for (int k4 = 0; k4 < kTile / 4; ++k4) {
      float4 pv[RT];
#pragma unroll
      for (int r = 0; r < RT; ++r) pv[r] = *reinterpret_cast<const float4*>(&sm.p[ty * RT + r][4 * k4]);
#pragma unroll
      for (int e = 0; e < 4; ++e) {
#pragma unroll
        for (int c = 0; c < OC; ++c) {
          const float4 vv = *reinterpret_cast<const float4*>(&sm.v[4 * k4 + e][64 * c + 4 * tx]);
#pragma unroll
          for (int r = 0; r < RT; ++r) {
            const float w = e == 0 ? pv[r].x : e == 1 ? pv[r].y : e == 2 ? pv[r].z : pv[r].w;
            o[r][c][0] = fmaf(w, vv.x, o[r][c][0]);
            o[r][c][1] = fmaf(w, vv.y, o[r][c][1]);
            o[r][c][2] = fmaf(w, vv.z, o[r][c][2]);
            o[r][c][3] = fmaf(w, vv.w, o[r][c][3]);
          }
        }
      }
    }
    __syncthreads();  // V (and P) have been read by all
    if (t + 1 < t_end)
      load_tile(t + 1, false);
    else
      cp_async_commit();
  }
  cp_async_wait<0>();
#pragma unroll
  for (int r = 0; r < RT; ++r) {
    const int row = ty * RT + r, tl = row / p.gb, hh = row - tl * p.gb;
    if (row >= rows || hh >= heads) continue;
    const size_t out_row = static_cast<size_t>(s.start + i0 + tl) * a.Hq + h0 + hh;
    const bool part = p.nsplit > 1;
    const float inv = part ? 1.f : (l[r] != 0.f ? 1.f / l[r] : 0.f);
    float* dst = part ? partial_o<D>(p, out_row, blockIdx.z) : static_cast<float*>(a.out) + out_row * D;
#pragma unroll
    for (int c = 0; c < OC; ++c)
      *reinterpret_cast<float4*>(dst + 64 * c + 4 * tx) =
          l[r] != 0.f ? make_float4(o[r][c][0] * inv, o[r][c][1] * inv, o[r][c][2] * inv, o[r][c][3] * inv)
                      : make_float4(0.f, 0.f, 0.f, 0.f);
    if (tx == 0) {
      if (part)
        *partial_ml<D>(p, out_row, blockIdx.z) = make_float2(m[r], l[r]);
      else if (a.lse)
        a.lse[out_row] = l[r] != 0.f ? m[r] + logf(l[r]) : -INFINITY;
    }
  }
}

// Few rows (single tokens, short drafts): a warp takes keys for itself, four
// at a time, its lanes the columns, with Q, O and the running maximum and sum
// of R rows in registers; K and V go from the cache straight to registers,
// the next four keys' while these are worked on.  The warps' results are
// merged through shared memory.  Bound by memory and by the sums over the
// lanes (20 shuffles a key): 32 single tokens over 4096 keys, 32 heads on 8,
// read 1.07 GB in 266 us (4.0 TB/s); tiles of 16 rows took 650.
template <int D>
__global__ void __launch_bounds__(kThreads, 2) chunk_f32_few_kernel(const __grid_constant__ F32Params p) {
  constexpr int E = D / 32, kWarps = kThreads / 32, kKeys = 4, R = 4;
  struct alignas(4 * E) Vec {
    float x[E];
  };
  // (three: a warp may still be at a tile while another is past the barrier of the next)
  __shared__ uint32_t key_row[3][kFewTile];
  __shared__ alignas(16) float part_o[kWarps][R][D];
  __shared__ float part_m[kWarps][R], part_l[kWarps][R];
  __shared__ int2 sees[R];  // the keys that a row sees
  pdl_wait();
  pdl_launch_next();
  const ChunkArgs& a = p.a;
  const unsigned full = 0xffffffffu;
  const int tid = threadIdx.x, lane = tid & 31, warp = tid >> 5;
  Unit u;
  if (!unit_of(p, kFewTile, u)) return;
  Vec q[R], o[R];
  float m[R], l[R];
#pragma unroll
  for (int r = 0; r < R; ++r) {
    const int tl = r / p.gb, hh = r - tl * p.gb;
    const bool real = r < u.rows && hh < u.heads;
    if (real)
      q[r] = *reinterpret_cast<const Vec*>(static_cast<const float*>(a.q) +
                                           static_cast<long long>(u.s.start + u.i0 + tl) * a.q_stride +
                                           static_cast<long long>(u.h0 + hh) * D + E * lane);
    m[r] = -INFINITY;
    l[r] = 0.f;
#pragma unroll
    for (int e = 0; e < E; ++e) {
      o[r].x[e] = 0.f;
      q[r].x[e] = real ? q[r].x[e] * a.scale : 0.f;
    }
  }
  const Vec* kp = static_cast<const Vec*>(a.k_cache);
  const Vec* vp = static_cast<const Vec*>(a.v_cache);
  if (tid < R) row_keys(p, u, tid, sees[tid].x, sees[tid].y);
  if (u.t_begin < u.t_end) key_row[u.t_begin % 3][tid] = pool_row(p, u, u.t_begin * kFewTile + tid);
  __syncthreads();
  Vec k[kKeys], v[kKeys];
  // (hidden keys: zeros)
  auto load = [&](Vec (&to)[kKeys], const Vec* from, const uint32_t* rows) {
#pragma unroll
    for (int j = 0; j < kKeys; ++j) {
      const uint32_t at = rows[j];
#pragma unroll
      for (int e = 0; e < E; ++e) to[j].x[e] = 0.f;
      if (at != ~0u) to[j] = from[static_cast<size_t>(at) * 32 + lane];
    }
  };
  constexpr int kRun = kFewTile / kWarps;  // keys of a warp in a tile
  if (u.t_begin < u.t_end) {
    load(k, kp, &key_row[u.t_begin % 3][warp * kRun]);
    load(v, vp, &key_row[u.t_begin % 3][warp * kRun]);
  }
  for (int t = u.t_begin; t < u.t_end; ++t) {
    if (t + 1 < u.t_end) key_row[(t + 1) % 3][tid] = pool_row(p, u, (t + 1) * kFewTile + tid);
    __syncthreads();
#pragma unroll 1
    for (int c = 0; c < kRun; c += kKeys) {
      float sc[R][kKeys];
#pragma unroll
      for (int j = 0; j < kKeys; ++j) {
#pragma unroll
        for (int r = 0; r < R; ++r) {
          float x = 0.f;
#pragma unroll
          for (int e = 0; e < E; ++e) x = fmaf(q[r].x[e], k[j].x[e], x);
          sc[r][j] = x;
        }
      }
      const bool more = c + kKeys < kRun || t + 1 < u.t_end;
      const uint32_t* next = c + kKeys < kRun ? &key_row[t % 3][warp * kRun + c + kKeys] : &key_row[(t + 1) % 3][warp * kRun];
      if (more) load(k, kp, next);
      const int key0 = t * kFewTile + warp * kRun + c;
#pragma unroll
      for (int r = 0; r < R; ++r) {
        float mx = m[r];
#pragma unroll
        for (int j = 0; j < kKeys; ++j) {
#pragma unroll
          for (int w = 16; w > 0; w >>= 1) sc[r][j] += __shfl_xor_sync(full, sc[r][j], w);
          if (key0 + j < sees[r].x || key0 + j >= sees[r].y) sc[r][j] = -INFINITY;
          mx = fmaxf(mx, sc[r][j]);
        }
        // (nothing seen so far: every weight is zero)
        const float ref = mx == -INFINITY ? 0.f : mx, corr = expf(m[r] - ref);
        l[r] *= corr;
#pragma unroll
        for (int e = 0; e < E; ++e) o[r].x[e] *= corr;
#pragma unroll
        for (int j = 0; j < kKeys; ++j) {
          const float w = expf(sc[r][j] - ref);
          l[r] += w;
#pragma unroll
          for (int e = 0; e < E; ++e) o[r].x[e] = fmaf(w, v[j].x[e], o[r].x[e]);
        }
        m[r] = mx;
      }
      if (more) load(v, vp, next);
    }
  }
#pragma unroll
  for (int r = 0; r < R; ++r) {
    *reinterpret_cast<Vec*>(&part_o[warp][r][E * lane]) = o[r];
    if (lane == 0) {
      part_m[warp][r] = m[r];
      part_l[warp][r] = l[r];
    }
  }
  __syncthreads();
  for (int i = tid; i < R * D; i += kThreads) {
    const int r = i / D, c = i - r * D, tl = r / p.gb, hh = r - tl * p.gb;
    if (r >= u.rows || hh >= u.heads) continue;
    float M = -INFINITY, L = 0.f, acc = 0.f;
#pragma unroll
    for (int w = 0; w < kWarps; ++w) M = fmaxf(M, part_m[w][r]);
    const float ref = M == -INFINITY ? 0.f : M;
#pragma unroll
    for (int w = 0; w < kWarps; ++w) {
      const float x = expf(part_m[w][r] - ref);
      L = fmaf(x, part_l[w][r], L);
      acc = fmaf(x, part_o[w][r][c], acc);
    }
    const size_t out_row = static_cast<size_t>(u.s.start + u.i0 + tl) * a.Hq + u.h0 + hh;
    if (p.nsplit > 1) {
      partial_o<D>(p, out_row, blockIdx.z)[c] = L != 0.f ? acc : 0.f;
      if (c == 0) *partial_ml<D>(p, out_row, blockIdx.z) = make_float2(M, L);
    } else {
      static_cast<float*>(a.out)[out_row * D + c] = L != 0.f ? acc * (1.f / L) : 0.f;
      if (a.lse && c == 0) a.lse[out_row] = L != 0.f ? M + logf(L) : -INFINITY;
    }
  }
}

// A warp per (token, head): O = sum_i e^(m_i - M) O_i / sum_i e^(m_i - M) l_i.
template <int D>
__global__ void __launch_bounds__(128) chunk_f32_merge_kernel(const __grid_constant__ F32Params p) {
  constexpr int E = D / 32;
  pdl_wait();
  pdl_launch_next();
  const int lane = threadIdx.x & 31;
  const size_t row = static_cast<size_t>(blockIdx.x) * 4 + (threadIdx.x >> 5);
  if (row >= static_cast<size_t>(p.a.T) * p.a.Hq) return;
  const int b = warp_find_seq(p.a.token_start, p.a.Bt, static_cast<int>(row / p.a.Hq));
  if (b < 0 || chunk_of(p.a.token_start, b, p.a.T).bad) return;  // no chunk holds the token: untouched
  float M = -INFINITY, L = 0.f, acc[E];
#pragma unroll
  for (int e = 0; e < E; ++e) acc[e] = 0.f;
  for (int i = 0; i < p.nsplit; ++i) {
    const float2 ml = *partial_ml<D>(p, row, i);
    if (ml.y != 0.f) M = fmaxf(M, ml.x);
  }
#pragma unroll 4
  for (int i = 0; i < p.nsplit; ++i) {
    const float2 ml = *partial_ml<D>(p, row, i);
    const float w = ml.y != 0.f ? expf(ml.x - M) : 0.f;
    L = fmaf(w, ml.y, L);
    const float* o = partial_o<D>(p, row, i);
#pragma unroll
    for (int e = 0; e < E; ++e) acc[e] = fmaf(w, o[lane + 32 * e], acc[e]);
  }
  const float inv = L != 0.f ? 1.f / L : 0.f;
#pragma unroll
  for (int e = 0; e < E; ++e) static_cast<float*>(p.a.out)[row * D + lane + 32 * e] = acc[e] * inv;
  if (p.a.lse && lane == 0) p.a.lse[row] = L != 0.f ? M + logf(L) : -INFINITY;
}

static_assert(2 * (sizeof(SmemF32<128, 64>) + 1024 + 64) <= 228 * 1024, "two CTAs a SM");

struct F32Plan {
  int rb, gb, hblocks, tb, units, nsplit;
};

// Blocks of 4 rows (in registers) where a sequence has up to 8 query rows a KV
// head on average, of 16 up to 16, of 64 where it has more (K and V are read a
// quarter as often), of 128 where even such blocks are two a SM.  32 sequences
// over 4096 keys, 32 heads on 8: 2 tokens 505 us with 4 rows, 646 with 16; 4
// tokens 878 and 646.  4 chunks of 512 tokens: 675 us with 128 rows, 777 with
// 64.  Ranges of keys until about four CTAs a SM are at work, none shorter
// than 3 tiles (for 4 rows, one of theirs) of the longest possible key range.
F32Plan f32_plan(int T, int Bt, int Hq, int Hkv, long long max_keys, int num_sms) {
  F32Plan f;
  const int g = Hq / Hkv;
  auto lay = [&](int rb) {
    f.rb = rb;
    f.gb = std::min(g, rb);
    f.hblocks = (g + f.gb - 1) / f.gb;
    f.tb = rb / f.gb;
    f.units = static_cast<int>(std::min<long long>(T, T / f.tb + static_cast<long long>(Bt)));
    return static_cast<long long>(f.units) * Hkv * f.hblocks;
  };
  long long ctas = lay(128);
  if (ctas < 2ll * num_sms || static_cast<long long>(T) * g <= 64ll * Bt)
    ctas = lay(static_cast<long long>(T) * g > 16ll * Bt ? 64 : static_cast<long long>(T) * g > 8ll * Bt ? 16 : 4);
  const long long least = f.rb == 4 ? kFewTile : 3 * kTile;
  const long long most = std::max<long long>(1, (max_keys + least - 1) / least);
  f.nsplit = static_cast<int>(std::max<long long>(1, std::min<long long>({4ll * num_sms / ctas, most, 64})));
  return f;
}

template <int D, int RB>
cudaError_t launch_rb(const F32Params& p, const F32Plan& f, cudaStream_t stream) {
  const dim3 grid(static_cast<unsigned>(f.units) * static_cast<unsigned>(p.heads), 1u, static_cast<unsigned>(f.nsplit));
  cudaError_t e;
  if constexpr (RB == 4) {
    e = launch_overlapped(chunk_f32_few_kernel<D>, grid, dim3(kThreads), 0, stream, 1u, p);
  } else {
    static std::mutex mu;
    static bool done[64] = {};
    int dev = 0;
    e = cudaGetDevice(&dev);
    if (e != cudaSuccess) return e;
    if (dev < 0 || dev >= 64) return cudaErrorInvalidDevice;
    std::lock_guard<std::mutex> lk(mu);
    if (!done[dev]) {
      e = cudaFuncSetAttribute(chunk_f32_kernel<D, RB>, cudaFuncAttributeMaxDynamicSharedMemorySize,
                               static_cast<int>(sizeof(SmemF32<D, RB>)));
      if (e != cudaSuccess) return e;
      done[dev] = true;
    }
    e = launch_overlapped(chunk_f32_kernel<D, RB>, grid, dim3(kThreads), sizeof(SmemF32<D, RB>), stream, 1u, p);
  }
  if (e != cudaSuccess || f.nsplit == 1) return e;
  const unsigned blocks = static_cast<unsigned>((static_cast<long long>(p.a.T) * p.a.Hq + 3) / 4);
  return launch_overlapped(chunk_f32_merge_kernel<D>, dim3(blocks), dim3(128), 0, stream, 1u, p);
}

}  // namespace

size_t chunk_f32_workspace_bytes(int T, int Bt, int Hq, int Hkv, int d, long long max_keys, int num_sms) {
  if (T <= 0 || Bt <= 0) return 0;
  const F32Plan f = f32_plan(T, Bt, Hq, Hkv, max_keys, num_sms);
  return f.nsplit > 1 ? static_cast<size_t>(T) * Hq * f.nsplit * (d + 2) * sizeof(float) : 0;
}

cudaError_t launch_chunk_attention_f32(const ChunkArgs& a, int num_sms, cudaStream_t stream) {
  const F32Plan f =
      f32_plan(a.T, a.Bt, a.Hq, a.Hkv, static_cast<long long>(a.max_pages) * a.page_size, num_sms);
  F32Params p{};
  p.a = a;
  p.g = a.Hq / a.Hkv;
  p.gb = f.gb;
  p.hblocks = f.hblocks;
  p.tb = f.tb;
  p.nsplit = f.nsplit;
  p.heads = a.Hkv * f.hblocks;
  p.units = f.units;
  if (f.rb == 128)
    return a.d == 128 ? launch_rb<128, 128>(p, f, stream) : launch_rb<64, 128>(p, f, stream);
  if (f.rb == 64) return a.d == 128 ? launch_rb<128, 64>(p, f, stream) : launch_rb<64, 64>(p, f, stream);
  if (f.rb == 16) return a.d == 128 ? launch_rb<128, 16>(p, f, stream) : launch_rb<64, 16>(p, f, stream);
  return a.d == 128 ? launch_rb<128, 4>(p, f, stream) : launch_rb<64, 4>(p, f, stream);
}

}  // namespace simsd
