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
// RB is 64 for chunks of many rows (bound by the FMA pipes), 16 for single
// tokens (bound by memory, then by the reads of K and V from shared memory).
// Few units are split over their keys into nsplit ranges, whose partial
// (O, m, l) a second launch merges.
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
  long long row[2][kTile];  // per tile parity: a key's row in the pool, in 16-byte units (-1: hidden)
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

template <int D, int RB>
__global__ void __launch_bounds__(kThreads) chunk_f32_kernel(const __grid_constant__ F32Params p) {
  constexpr int RT = RB / 16;   // rows of a thread
  constexpr int OC = D / 64;    // four-column groups of O of a thread
  extern __shared__ uint4 smem_raw[];
  SmemF32<D, RB>& sm = *reinterpret_cast<SmemF32<D, RB>*>(smem_raw);
  __shared__ int unit_s[2];
  pdl_wait();
  pdl_launch_next();
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
  if (b < 0) return;
  const ChunkSeq s = chunk_seq(a, b);
  const int i0 = unit_s[1] * p.tb, i1 = min(s.C, i0 + p.tb);
  const int kvh = head / p.hblocks, h0 = kvh * p.g + (head - kvh * p.hblocks) * p.gb;
  const int heads = min(p.gb, kvh * p.g + p.g - h0);
  const int rows = (i1 - i0) * p.gb;  // row r: token i0 + r / gb, head h0 + r % gb (if below `heads`)
  int lo = 0, hi = 0;
  if (!s.bad) {
    lo = key_lo(a, s, i0);
    hi = key_hi(a, s, i1 - 1);
  }
  if (lo >= hi) lo = hi = 0;
  const int32_t* bt = a.block_table + static_cast<size_t>(b) * a.max_pages;
  bool bad = false;
  if (hi > lo)
    for (int i = lo / a.page_size + tid; i <= (hi - 1) / a.page_size; i += kThreads)
      bad |= bt[i] < 0 || bt[i] >= a.num_pages;
  bad = __syncthreads_or(bad);
  if (bad && tid == 0) raise_error(a.err_word, SIMSD_EW_PAGE);
  if (bad) hi = lo;
  // this CTA's tiles
  const int T0 = lo / kTile, nt = hi > lo ? (hi + kTile - 1) / kTile - T0 : 0;
  const int t_begin = T0 + static_cast<int>(static_cast<long long>(blockIdx.z) * nt / p.nsplit);
  const int t_end = T0 + static_cast<int>(static_cast<long long>(blockIdx.z + 1) * nt / p.nsplit);

  // where the keys of tile t lie (the page arithmetic once a key, not once a copy)
  auto find_rows = [&](int t) {
    if (tid < kTile) {
      const int key = t * kTile + tid;
      long long off = -1;
      if (key >= lo && key < hi) {
        const int pi = key / a.page_size;
        off = ((static_cast<long long>(bt[pi]) * a.Hkv + kvh) * a.page_size + (key - pi * a.page_size)) * (D / 4);
      }
      sm.row[t & 1][tid] = off;
    }
  };
  auto load_tile = [&](int t, bool is_k) {
    const float4* src = static_cast<const float4*>(is_k ? a.k_cache : a.v_cache);
    const int c = tid % (D / 4);
#pragma unroll 4
    for (int r = tid / (D / 4); r < kTile; r += kThreads / (D / 4)) {
      const long long off = sm.row[t & 1][r];
      cp_async16(is_k ? &sm.k[r][4 * (c ^ (r & 7))] : &sm.v[r][4 * c], src + (off < 0 ? 0 : off + c), off >= 0);
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
    const int row = ty * RT + r;
    const bool real = row < rows && nt > 0;
    klo[r] = real ? key_lo(a, s, i0 + row / p.gb) : 0;
    khi[r] = real ? key_hi(a, s, i0 + row / p.gb) : 0;
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

struct F32Plan {
  int rb, gb, hblocks, tb, units, nsplit;
};

// RB 16 where a sequence has up to 16 query rows a KV head on average, 64
// where it has more (the wider block reads K and V a quarter as often), 128
// where even such blocks are two a SM (4 chunks of 512 tokens, 32 heads: 675
// us, with 64 rows 777 us).  Ranges of keys until about two CTAs a SM are at
// work, none shorter than 4 tiles of the longest possible key range.
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
    ctas = lay(g > 16 || static_cast<long long>(T) * g > 16ll * Bt ? 64 : 16);
  const long long most = std::max<long long>(1, (max_keys + kTile - 1) / kTile / 4);
  f.nsplit = static_cast<int>(std::max<long long>(1, std::min<long long>({2ll * num_sms / ctas, most, 64})));
  return f;
}

template <int D, int RB>
cudaError_t launch_rb(const F32Params& p, const F32Plan& f, cudaStream_t stream) {
  {
    static std::mutex mu;
    static bool done[64] = {};
    int dev = 0;
    cudaError_t e = cudaGetDevice(&dev);
    if (e != cudaSuccess) return e;
    if (dev < 0 || dev >= 64) return cudaErrorInvalidDevice;
    std::lock_guard<std::mutex> lk(mu);
    if (!done[dev]) {
      e = cudaFuncSetAttribute(chunk_f32_kernel<D, RB>, cudaFuncAttributeMaxDynamicSharedMemorySize,
                               static_cast<int>(sizeof(SmemF32<D, RB>)));
      if (e != cudaSuccess) return e;
      done[dev] = true;
    }
  }
  const dim3 grid(static_cast<unsigned>(f.units) * static_cast<unsigned>(p.heads), 1u, static_cast<unsigned>(f.nsplit));
  cudaError_t e = launch_overlapped(chunk_f32_kernel<D, RB>, grid, dim3(kThreads), sizeof(SmemF32<D, RB>), stream, 1u, p);
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
  if (f.rb == 64)
    return a.d == 128 ? launch_rb<128, 64>(p, f, stream) : launch_rb<64, 64>(p, f, stream);
  return a.d == 128 ? launch_rb<128, 16>(p, f, stream) : launch_rb<64, 16>(p, f, stream);
}

}  // namespace simsd
