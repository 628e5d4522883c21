// sample.cu -- draws a token from each row of logits with a given random
// number, after temperature, top-k, top-p and min-p (Sec. 3.2: drafts come
// from the draft model's distribution).
//
// Mathematics.  w_v = exp((x_v - m) / T), m = max x.  The kept set is a
// prefix of the order (x falling, index rising): {x > kappa} and the tokens
// x = kappa up to some index, cut by w >= min_p.  Sums of weights are 64-bit
// integers in units of 2^-38 of the largest weight (a token whose number hangs
// on the last bits of a sum of 150,000 weights is still the right one).
//
// A row is read twice.  The first pass (from HBM) takes the maximum and, of
// an eighth of the row, counts and weights over bins 1/32 wide in x / T.
// From this sample the place of kappa is known within its statistical error;
// the second pass (from L2) adds up exactly what lies above that bracket and
// lists the tokens inside it, which tells whether kappa is there (else the
// row goes on to the searches below), and one CTA searches the list in shared
// memory.  A bracket with more tokens than the list holds is narrowed by
// another pass.  What no bracket settles (a bin with more tokens than the
// list, as at very high temperatures) goes through radix searches over the
// row.  The random number is placed by the weights of the row's segments (one
// per warp), and only the segment it falls in is read again.
//
// Bound by memory for many rows (HBM once, L2 once) and by the chain of
// passes and exchanges for few.  Counting an eighth of the row instead of
// all of it matters: shared-memory atomics run at about 4 tokens a cycle and
// SM, and HBM delivers 12.
//
// A thread-block cluster serves a row: one CTA where there are many rows,
// up to eight where there are few.
#include <cuda_bf16.h>
#include <cuda_runtime.h>

#include <algorithm>
#include <cfloat>
#include <cmath>
#include <mutex>

#include "common.cuh"
#include "kernels.h"
#include "ptx.cuh"

namespace simsd {
namespace {

typedef unsigned long long u64;

constexpr int kThreads = 512;
constexpr int kWarps = kThreads / 32;
constexpr int kMaxCluster = 8;
constexpr int kBatch = 16;         // elements of a lane in flight
constexpr int kCoarse = 2048;     // bins of the first pass
constexpr float kBinsPerUnit = 32.f;
constexpr int kSampleFrom = 16384;  // vocabularies from here on are sampled
constexpr int kList = 8192;       // tokens of the list
constexpr int kRegion = kList / kWarps;  // of a warp
constexpr int kAim = 2500;        // tokens that a bracket aims at where the sample is too coarse
constexpr int kFine = 2048;       // bins of the searches
constexpr int kFirst = 2048;      // elements that place the window of the first pass
constexpr float kUnit = 274877906944.0f;  // 2^38
constexpr unsigned kFull = 0xffffffffu;

// Ordered pattern: a < b as floats (-0 = +0) iff ordered(a) < ordered(b).
__device__ __forceinline__ uint32_t ordered(float x) {
  const uint32_t b = __float_as_uint(x + 0.0f);
  return b & 0x80000000u ? ~b : b | 0x80000000u;
}
__device__ __forceinline__ float from_ordered(uint32_t k) {
  return __uint_as_float(k & 0x80000000u ? k & 0x7fffffffu : ~k);
}
__device__ __forceinline__ u64 units(float w) { return __float2ull_rn(w * kUnit); }

// A sum of a batch of weights, exact to 2^-34: the parts of the weights that
// are multiples of 2^-13 add up exactly, the rests are below 2^-13.
struct BatchSum {
  float hi = 0.f, lo = 0.f;
  __device__ __forceinline__ void add(float w) {
    const float h = __fsub_rn(__fadd_rn(w, 1536.f), 1536.f);
    hi = __fadd_rn(hi, h);
    lo = __fadd_rn(lo, __fsub_rn(w, h));
  }
  __device__ __forceinline__ u64 total() const {
    return static_cast<u64>(__float2ll_rn(hi * kUnit) + __float2ll_rn(lo * kUnit));
  }
};

// A running sum of such batches' fp32 sums with its rounding errors (two-sum).
struct LongSum {
  float hi = 0.f, lo = 0.f;
  __device__ __forceinline__ void add(float x) {
    const float t = __fadd_rn(hi, x), z = __fsub_rn(t, hi);
    lo = __fadd_rn(lo, __fadd_rn(__fsub_rn(hi, __fsub_rn(t, z)), __fsub_rn(x, z)));
    hi = t;
  }
  __device__ __forceinline__ u64 total() const {
    return static_cast<u64>(__float2ll_rn(hi * kUnit) + __float2ll_rn(lo * kUnit));
  }
};

// The part f of a sum, f in [0, 1): floor and ceiling.
__device__ __forceinline__ u64 fraction(float f) { return __float2ull_rz(f * 18446744073709551616.0f); }
__device__ __forceinline__ u64 part_floor(float f, u64 sum) { return __umul64hi(sum, fraction(f)); }
__device__ __forceinline__ u64 part_ceil(float f, u64 sum) {
  const u64 q = fraction(f);
  return __umul64hi(sum, q) + (sum * q ? 1 : 0);
}
// Natural logarithm of a sum of weights in units of 2^-38 (no 64-bit floating point).
__device__ __forceinline__ float log_units(u64 sum) {
  const int e = 63 - __clzll(static_cast<long long>(sum));
  const float f = __ull2float_rn(sum) * exp2f(static_cast<float>(-e));  // [1, 2]
  return fmaf(static_cast<float>(e - 38), 0.693147180559945f, logf(f));
}

// z = (x - m) / T as a correctly rounded quotient (one Newton step on the
// product with 1 / T); infinite m: the tokens at m share the weight.
struct Weight {
  float m, T, inv;
  __device__ __forceinline__ float z(float x) const {
    const float d = x - m;
    const float q = d * inv;
    const float r = fmaf(-q, T, d);
    const float c = T > 1e-18f ? fmaf(r, inv, q) : d / T;
    return x == m ? 0.f : (isinf(d) ? d : c);
  }
  __device__ __forceinline__ float w(float x) const { return expf(z(x)); }
};

struct Kept {
  uint32_t kappa;
  int last;
  float min_p;
  // a higher kappa: an index limit among the ties of the old one does not hold there
  __device__ __forceinline__ void move_to(uint32_t key) {
    if (key != kappa) last = 0x7fffffff;
    kappa = key;
  }
  __device__ __forceinline__ bool in_prefix(uint32_t key, int idx) const {
    return key > kappa || (key == kappa && idx <= last);
  }
};

struct alignas(16) Smem {
  union {
    struct {
      float x[kList];
      int idx[kList];
    } list;
    u64 mass[kFine];  // searches over the row
  };
  uint32_t coarse[kCoarse], part[kCoarse];          // sample: counts, weights in 2^-16 of their bin's upper edge
  uint32_t count[kFine], low[kFine], high[kFine];   // searches: counts, weight units modulo 2^19 and above
  u64 seg[kMaxCluster * kWarps];  // weights of the row's segments (rank 0 holds all)
  u64 warp_a[kWarps], warp_b[kWarps], warp_c[kWarps];
  u64 x_max[kMaxCluster];                          // exchanges over the cluster: one slot per CTA
  u64 x_sum[4][kMaxCluster];
  u64 x_out[4];
  u64 found[5];
  int list_n[kWarps], pick_lo, pick_hi, token;
};

// ------------------------------------------------------------- the cluster
__device__ __forceinline__ uint32_t map_rank(const void* p, int rank) {
  uint32_t r;
  asm volatile("mapa.shared::cluster.u32 %0, %1, %2;" : "=r"(r) : "r"(smem_u32(p)), "r"(rank));
  return r;
}
__device__ __forceinline__ void st_rank(void* p, int rank, u64 v) {
  asm volatile("st.shared::cluster.u64 [%0], %1;" ::"r"(map_rank(p, rank)), "l"(v) : "memory");
}
__device__ __forceinline__ void st_rank(void* p, int rank, uint32_t v) {
  asm volatile("st.shared::cluster.u32 [%0], %1;" ::"r"(map_rank(p, rank)), "r"(v) : "memory");
}
__device__ __forceinline__ uint32_t ld_rank_u32(const void* p, int rank) {
  uint32_t v;
  asm volatile("ld.shared::cluster.u32 %0, [%1];" : "=r"(v) : "r"(map_rank(p, rank)) : "memory");
  return v;
}
__device__ __forceinline__ uint4 ld_rank_v4(const void* p, int rank) {
  uint4 v;
  asm volatile("ld.shared::cluster.v4.u32 {%0, %1, %2, %3}, [%4];"
               : "=r"(v.x), "=r"(v.y), "=r"(v.z), "=r"(v.w)
               : "r"(map_rank(p, rank))
               : "memory");
  return v;
}
__device__ __forceinline__ u64 ld_rank_u64(const void* p, int rank) {
  u64 v;
  asm volatile("ld.shared::cluster.u64 %0, [%1];" : "=l"(v) : "r"(map_rank(p, rank)) : "memory");
  return v;
}
__device__ __forceinline__ void sync_all(int CL) {
  if (CL > 1) {
    asm volatile("barrier.cluster.arrive.release;" ::: "memory");
    asm volatile("barrier.cluster.wait.acquire;" ::: "memory");
  } else {
    __syncthreads();
  }
}

// -------------------------------------------------------------------- rows
// The vectors [v0, v1) of a row belong to this CTA, and of those a run to
// each warp (a segment), so that a warp's elements are consecutive.
template <typename E>
struct Row {
  static constexpr int kVec = 16 / sizeof(E), kUnroll = kBatch / kVec;
  const E* base;  // 16-byte aligned; `lead` elements before the row
  int lead, V;
  int vecs, per, per_warp;  // vectors of the row, of a CTA, of a segment

  __device__ __forceinline__ void load(int v, float (&x)[kVec]) const {
    const int i0 = v * kVec - lead;
    const E* p = base + static_cast<size_t>(v) * kVec;
    if (i0 >= 0 && i0 + kVec <= V) {
      const uint4 q = *reinterpret_cast<const uint4*>(p);
      const uint32_t w[4] = {q.x, q.y, q.z, q.w};
#pragma unroll
      for (int e = 0; e < kVec; ++e)
        x[e] = sizeof(E) == 4 ? __uint_as_float(w[e])
                              : __uint_as_float(e & 1 ? w[e / 2] & 0xffff0000u : w[e / 2] << 16);
    } else {
#pragma unroll
      for (int e = 0; e < kVec; ++e) x[e] = i0 + e >= 0 && i0 + e < V ? static_cast<float>(p[e]) : -INFINITY;
    }
    // (elements outside the row and NaN count as -inf)
#pragma unroll
    for (int e = 0; e < kVec; ++e) x[e] = fmaxf(x[e], -INFINITY);
  }
  __device__ __forceinline__ int seg_begin(int rank, int warp) const {
    return min(min(vecs, rank * per + per), min(vecs, rank * per) + warp * per_warp);
  }
  // batches of kUnroll vectors of this thread's segment: f(x, first index of each vector)
  template <typename F>
  __device__ __forceinline__ void batches(int rank, F&& f) const {
    const int warp = threadIdx.x >> 5, lane = threadIdx.x & 31;
    const int a = seg_begin(rank, warp), b = min(seg_begin(rank, warp + 1), min(vecs, rank * per + per));
    // (all lanes stay in the loop: what it calls may exchange within the warp)
    for (int v = a + lane; v - lane < b; v += 32 * kUnroll) {
      float x[kUnroll][kVec];
#pragma unroll
      for (int i = 0; i < kUnroll; ++i) {
        if (v + 32 * i < b) {
          load(v + 32 * i, x[i]);
        } else {
#pragma unroll
          for (int e = 0; e < kVec; ++e) x[i][e] = -INFINITY;
        }
      }
      f(x, v * kVec - lead);
    }
  }
  // index of element e of vector i of the batch that starts at index i0
  __device__ static __forceinline__ int index(int i0, int i, int e) { return i0 + 32 * kVec * i + e; }
};

__device__ __forceinline__ u64 warp_sum(u64 v) {
#pragma unroll
  for (int o = 16; o > 0; o >>= 1) v += __shfl_xor_sync(kFull, v, o);
  return v;
}

// Sums over the cluster of four values; every CTA gets them.
__device__ __noinline__ void cluster_sum(Smem& sm, int CL, int rank, u64 (&v)[4]) {
  const int lane = threadIdx.x & 31, warp = threadIdx.x >> 5;
#pragma unroll
  for (int k = 0; k < 4; ++k) v[k] = warp_sum(v[k]);
  __syncthreads();
  if (lane == 0) {
    sm.warp_a[warp] = v[0];
    sm.warp_b[warp] = v[1];
    sm.warp_c[warp] = v[2];
    sm.found[0] = 0;
  }
  __syncthreads();
  if (lane == 0) atomicAdd(&sm.found[0], v[3]);
  __syncthreads();
  if (warp < 3) {
    const u64* src = warp == 0 ? sm.warp_a : warp == 1 ? sm.warp_b : sm.warp_c;
    const u64 x = warp_sum(lane < kWarps ? src[lane] : 0);
    if (lane < CL) {
      st_rank(&sm.x_sum[warp][rank], lane, x);
      if (warp == 0) st_rank(&sm.x_sum[3][rank], lane, sm.found[0]);
    }
  }
  sync_all(CL);
#pragma unroll
  for (int k = 0; k < 4; ++k) {
    v[k] = 0;
    for (int r = 0; r < CL; ++r) v[k] += sm.x_sum[k][r];
  }
  sync_all(CL);
}

// Exclusive scan over the block of (c, q) in thread order.
__device__ __forceinline__ void block_scan(Smem& sm, u64 c, u64 q, u64& pc, u64& pq) {
  const int lane = threadIdx.x & 31, warp = threadIdx.x >> 5;
  u64 ic = c, iq = q;
#pragma unroll
  for (int o = 1; o < 32; o <<= 1) {
    const u64 yc = __shfl_up_sync(kFull, ic, o), yq = __shfl_up_sync(kFull, iq, o);
    if (lane >= o) {
      ic += yc;
      iq += yq;
    }
  }
  __syncthreads();
  if (lane == 31) {
    sm.warp_a[warp] = ic;
    sm.warp_b[warp] = iq;
  }
  __syncthreads();
  u64 ta = lane < warp ? sm.warp_a[lane] : 0, tb = lane < warp ? sm.warp_b[lane] : 0;
#pragma unroll
  for (int o = 8; o > 0; o >>= 1) {
    ta += __shfl_xor_sync(kFull, ta, o);
    tb += __shfl_xor_sync(kFull, tb, o);
  }
  // (lanes 16 .. 31 hold nothing: kWarps is 16)
  pc = ic - c + __shfl_sync(kFull, ta, 0);
  pq = iq - q + __shfl_sync(kFull, tb, 0);
}
static_assert(kWarps == 16, "the scan of the warps' totals");

// What a search finds: the key at which the count (or the weight) from the
// highest key down first reaches the target, what lies above it, and at it.
struct Found {
  uint32_t key;
  u64 above_count, above_mass, at_count;
  bool ok;  // false: everything together does not reach the target
};

// Search over keys in [lo, hi], a digit of up to 11 bits per round.
// visit(f) calls f(key, weight units) for the elements.  kRow: every CTA of
// the cluster visits its own part of the row, and all get the result; else
// one CTA searches its list (at most kList elements, each below 2^51 units:
// their sums are kept as two 32-bit words).
template <bool kRow, typename Visit>
__device__ __forceinline__ Found search(Smem& sm, int CL, bool by_count, u64 target, uint32_t lo, uint32_t hi,
                                        Visit&& visit) {
  if (!kRow) CL = 1;
  Found f{0u, 0, 0, 0, true};
  for (;;) {
    const uint32_t span = hi - lo;
    const int bits = 32 - __clz(span);  // (clz(0) = 32)
    const int shift = max(0, bits - 11);
    sync_all(CL);
    for (int i = threadIdx.x; i < kFine; i += kThreads) {
      sm.count[i] = 0;
      if (kRow) {
        sm.mass[i] = 0;
      } else {
        sm.low[i] = 0;
        sm.high[i] = 0;
      }
    }
    sync_all(CL);
    visit([&](uint32_t key, u64 q) {
      if (key < lo || key > hi) return;
      const uint32_t bin = (key - lo) >> shift;
      atomicAdd(&sm.count[bin], 1u);
      if (q == 0) return;
      if (kRow) {
        atomicAdd(&sm.mass[bin], q);
      } else {
        atomicAdd(&sm.low[bin], static_cast<uint32_t>(q) & 0x7ffffu);
        atomicAdd(&sm.high[bin], static_cast<uint32_t>(q >> 19));
      }
    });
    sync_all(CL);
    // thread t: bins 4 t .. 4 t + 3 from the top
    u64 c[4], q[4], sc = 0, sq = 0;
#pragma unroll
    for (int e = 0; e < 4; ++e) {
      const int bin = kFine - 1 - (4 * static_cast<int>(threadIdx.x) + e);
      c[e] = q[e] = 0;
      if (!kRow) {
        c[e] = sm.count[bin];
        q[e] = (static_cast<u64>(sm.high[bin]) << 19) + sm.low[bin];
      } else {
        for (int r = 0; r < CL; ++r) {
          c[e] += ld_rank_u32(&sm.count[bin], r);
          q[e] += ld_rank_u64(&sm.mass[bin], r);
        }
      }
      sc += c[e];
      sq += q[e];
    }
    if (threadIdx.x == 0) sm.found[0] = ~0ull;
    u64 pc, pq;
    block_scan(sm, sc, sq, pc, pq);
    pc += f.above_count;
    pq += f.above_mass;
#pragma unroll
    for (int e = 0; e < 4; ++e) {
      const u64 before = by_count ? pc : pq, after = by_count ? pc + c[e] : pq + q[e];
      if (before < target && after >= target) {
        sm.found[0] = kFine - 1 - (4 * threadIdx.x + e);
        sm.found[1] = pc;
        sm.found[2] = pq;
        sm.found[3] = c[e];
      }
      pc += c[e];
      pq += q[e];
    }
    __syncthreads();
    const u64 bin = sm.found[0];
    if (bin == ~0ull) {
      f.ok = false;
      sync_all(CL);
      return f;
    }
    f.above_count = sm.found[1];
    f.above_mass = sm.found[2];
    f.at_count = sm.found[3];
    lo += static_cast<uint32_t>(bin) << shift;
    if (shift == 0) {
      f.key = lo;
      sync_all(CL);  // the histograms are read by all before anything else is written there
      return f;
    }
    hi = min(hi, lo + ((1u << shift) - 1u));
  }
}

template <typename E>
__global__ void __launch_bounds__(kThreads, 2) sample_kernel(const __grid_constant__ SampleArgs a, const int CL) {
  extern __shared__ uint4 smem_raw[];
  Smem& sm = *reinterpret_cast<Smem*>(smem_raw);
  constexpr int kVec = Row<E>::kVec, kUnroll = Row<E>::kUnroll;
  constexpr uint32_t kKeyMin = 0x00800000u;  // ordered(-inf) + 1: the lowest key a token can have
  const int tid = threadIdx.x, lane = tid & 31, warp = tid >> 5;
  const int r = blockIdx.x / CL, rank = blockIdx.x - r * CL;
  pdl_wait();
  Row<E> row;
  {
    const E* first = static_cast<const E*>(a.logits) + static_cast<size_t>(r) * static_cast<size_t>(a.row_stride);
    row.lead = static_cast<int>((reinterpret_cast<uintptr_t>(first) & 15u) / sizeof(E));
    row.base = first - row.lead;
    row.V = a.V;
    row.vecs = (a.V + row.lead + kVec - 1) / kVec;
    row.per = (row.vecs + CL - 1) / CL;
    row.per_warp = (row.per + kWarps - 1) / kWarps;
  }
  float T = a.temperature ? a.temperature[r] : 1.f, p = a.top_p ? a.top_p[r] : 1.f;
  const float mp = a.min_p ? fminf(a.min_p[r], 1.f) : 0.f;
  const float u = a.u[r];
  const bool bad_mp = a.min_p && a.min_p[r] != a.min_p[r];
  int k = a.top_k ? a.top_k[r] : 0;
  bool bad = !(T >= 0.f) || isinf(T) || !(u >= 0.f && u < 1.f) || p != p || bad_mp;
  if (T == 0.f) {  // greedy: the first token of the order alone
    T = 1.f;
    k = 1;
  }
  if (k < 1 || k >= a.V) k = 0;
  const bool cut = !bad && (k > 0 || p < 1.f);
  const float inv = 1.0f / T;

  // ---- pass 1: the maximum, and of a sample counts and weights over bins of x / T
  // sampled: the first vector of every other batch, about an eighth; fs: what
  // one sampled vector stands for
  const bool sampled = a.V >= kSampleFrom;
  float fs = 1.f;
  if (sampled) {
    int n = 0;
    for (int i = lane; i < CL * kWarps; i += 32) {
      const int rk = i / kWarps, w = i - rk * kWarps;
      const int len = min(row.seg_begin(rk, w + 1), min(row.vecs, rk * row.per + row.per)) - row.seg_begin(rk, w);
      const int pairs = len / (64 * kUnroll), rest = len - pairs * 64 * kUnroll;
      n += 32 * pairs + min(max(rest, 0), 32);
    }
#pragma unroll
    for (int o = 16; o > 0; o >>= 1) n += __shfl_xor_sync(kFull, n, o);
    fs = static_cast<float>(row.vecs) / static_cast<float>(max(n, 1));
  }
  const float scale = inv * kBinsPerUnit;
  float base = 0.f;
  if (cut) {
    for (int i = tid; i < kCoarse; i += kThreads) sm.coarse[i] = sm.part[i] = 0;
    // the window lies around the maximum of the row's first elements
    float f = -INFINITY;
    for (int i = tid; i < min(a.V, kFirst); i += kThreads)
      f = fmaxf(f, static_cast<float>(row.base[row.lead + i]));
#pragma unroll
    for (int o = 16; o > 0; o >>= 1) f = fmaxf(f, __shfl_xor_sync(kFull, f, o));
    if (lane == 0) sm.warp_a[warp] = __float_as_uint(f);
    __syncthreads();
    f = -INFINITY;
    for (int w = 0; w < kWarps; ++w) f = fmaxf(f, __uint_as_float(static_cast<uint32_t>(sm.warp_a[w])));
    base = isinf(f) ? 0.f : f;
    __syncthreads();
  }
  auto count_in = [&](float x) {
    const float y = fminf(fmaxf(fmaf(x - base, scale, 0.5f * kCoarse), 0.f), kCoarse - 0.01f);
    const float b = floorf(y), d = (b + 1.f - y) * (1.f / kBinsPerUnit);  // e^-d = 1 - d + d^2 / 2 to 5e-6
    const int bin = static_cast<int>(b);
    atomicAdd(&sm.coarse[bin], 1u);
    atomicAdd(&sm.part[bin], static_cast<uint32_t>(fmaf(d, fmaf(d, 0.5f, -1.f), 1.f) * 65536.f));
  };
  float mx = -INFINITY;
  {
    int nb = 0;
    row.batches(rank, [&](float (&x)[kUnroll][kVec], int) {
#pragma unroll
      for (int i = 0; i < kUnroll; ++i)
#pragma unroll
        for (int e = 0; e < kVec; ++e) mx = fmaxf(mx, x[i][e]);
      if (cut) {
        if (!sampled) {
#pragma unroll
          for (int i = 0; i < kUnroll; ++i)
#pragma unroll
            for (int e = 0; e < kVec; ++e)
              if (x[i][e] != -INFINITY) count_in(x[i][e]);
        } else if ((nb++ & 1) == 0) {
#pragma unroll
          for (int e = 0; e < kVec; ++e)
            if (x[0][e] != -INFINITY) count_in(x[0][e]);
        }
      }
    });
  }
#pragma unroll
  for (int o = 16; o > 0; o >>= 1) mx = fmaxf(mx, __shfl_xor_sync(kFull, mx, o));
  if (lane == 0) sm.warp_a[warp] = __float_as_uint(mx);
  __syncthreads();
  if (warp == 0) {
    mx = -INFINITY;
    for (int w = 0; w < kWarps; ++w) mx = fmaxf(mx, __uint_as_float(static_cast<uint32_t>(sm.warp_a[w])));
    if (lane < CL) st_rank(&sm.x_max[rank], lane, static_cast<u64>(__float_as_uint(mx)));
  }
  sync_all(CL);
  mx = -INFINITY;
  for (int q = 0; q < CL; ++q) mx = fmaxf(mx, __uint_as_float(static_cast<uint32_t>(sm.x_max[q])));
  const float m = mx + 0.0f;
  bad = bad || m == -INFINITY;
  if (bad) {
    if (rank == 0 && tid == 0) {
      raise_error(a.err_word, SIMSD_EW_SAMPLE);
      a.token[r] = -1;
      if (a.kept) a.kept[r] = 0;
      if (a.log_prob) a.log_prob[r] = -INFINITY;
    }
    if (a.log_probs)
      for (int i = rank * kThreads + tid; i < a.V; i += CL * kThreads)
        a.log_probs[static_cast<size_t>(r) * a.V + i] = -INFINITY;
    sync_all(CL);
    return;
  }
  const Weight wt{m, T, inv};
  Kept kept{kKeyMin, 0x7fffffff, mp};
  u64 set_mass = 0;     // of the tokens that top_p is a share of (0: not known yet)
  bool have_seg = false;  // the segments' weights (and the kept count) come from pass 2
  u64 kept_count = 0;

  // visits this CTA's elements that the prefix kept so far holds
  auto visit_row = [&](auto&& f) {
    row.batches(rank, [&](float (&x)[kUnroll][kVec], int i0) {
#pragma unroll
      for (int i = 0; i < kUnroll; ++i)
#pragma unroll
        for (int e = 0; e < kVec; ++e) {
          const uint32_t key = ordered(x[i][e]);
          if (x[i][e] != -INFINITY && kept.in_prefix(key, Row<E>::index(i0, i, e)))
            f(key, units(wt.w(x[i][e])));
        }
    });
  };
  const uint32_t key_max = ordered(m);

  // ---- the bracket of kappa, from the sample.  Thread t holds 4 bins from
  // the top; c and w: what the sample says of the whole row.
  struct Bracket {
    float x0, x1;  // tokens x0 <= x < x1 are to be listed
    bool all;      // x1 lies above all tokens
    bool listing;  // false: too many, their weight is taken to narrow the bracket
    bool ok;
  };
  float hc[4], hw[4];
  float hz = 0.f;  // weight of the whole row
  if (cut) {
    uint4 cn = make_uint4(0, 0, 0, 0), pn = cn;
    const int j4 = kCoarse - 4 - 4 * tid;  // bins j4 .. j4 + 3; entry e is bin j4 + 3 - e
#pragma unroll
    for (int h = 0; h < 2; ++h) {
      uint4 x[kMaxCluster];
#pragma unroll
      for (int q = 0; q < kMaxCluster; ++q)
        x[q] = q < CL ? ld_rank_v4(h == 0 ? &sm.coarse[j4] : &sm.part[j4], q) : make_uint4(0, 0, 0, 0);
      uint4& t = h == 0 ? cn : pn;
#pragma unroll
      for (int q = 0; q < kMaxCluster; ++q) t.x += x[q].x, t.y += x[q].y, t.z += x[q].z, t.w += x[q].w;
    }
    const uint32_t cs[4] = {cn.w, cn.z, cn.y, cn.x}, ps[4] = {pn.w, pn.z, pn.y, pn.x};
#pragma unroll
    for (int e = 0; e < 4; ++e) {
      // weight of the bin's upper edge (at most that of its tokens times e^(1/32))
      const float top = (static_cast<float>(j4 + 4 - e) - 0.5f * kCoarse) / kBinsPerUnit - (m - base) * inv;
      hc[e] = static_cast<float>(cs[e]);
      hw[e] = cs[e] ? static_cast<float>(ps[e]) * (1.f / 65536.f) * expf(fminf(top, 1.f)) : 0.f;
    }
  }
  auto edge = [&](int bin) { return base + (static_cast<float>(bin) - 0.5f * kCoarse) / scale; };
  const bool window_ok = scale < 1e30f && fmaf(m - base, scale, 0.5f * kCoarse) < kCoarse - 1;
  auto estimate = [&](bool by_count) {
    float sw = 0.f, sv = 0.f;
    u64 sc = 0;
#pragma unroll
    for (int e = 0; e < 4; ++e) {
      sc += static_cast<u64>(hc[e]);
      sw += hw[e];
      sv += hc[e] > 0.f ? hw[e] * hw[e] / hc[e] : 0.f;
    }
    u64 pc, pq, pv, none;
    block_scan(sm, sc, units(sw), pc, pq);
    __syncthreads();
    if (tid == kThreads - 1) {
      sm.found[3] = pq + units(sw);
      sm.pick_lo = sm.pick_hi = -1;
    }
    block_scan(sm, units(sv), 0, pv, none);
    if (tid == kThreads - 1) sm.found[4] = pv + units(sv);
    __syncthreads();
    const float all_w = __ull2float_rn(sm.found[3]) / kUnit, all_v = __ull2float_rn(sm.found[4]) / kUnit;
    hz = all_w * fs;
    // `lo`: the last bin by which the target is surely reached, `hi`: the
    // first where it may be (4 standard deviations of a count, 3 of a weight:
    // a miss costs another way through the row, not the result)
    const float pp = fmaxf(p, 0.f), noise = fs > 1.f ? fs * sqrtf(1.f - 1.f / fs) : 0.f;
    float rc = static_cast<float>(pc), rw = __ull2float_rn(pq) / kUnit, rv = __ull2float_rn(pv) / kUnit;
    float reach[4];
#pragma unroll
    for (int e = 0; e < 4; ++e) {
      rc += hc[e];
      rw += hw[e];
      rv += hc[e] > 0.f ? hw[e] * hw[e] / hc[e] : 0.f;
      const int bin = kCoarse - 1 - (4 * tid + e);
      float d, sd;
      if (by_count) {
        d = rc * fs - static_cast<float>(k);
        sd = 4.f * noise * sqrtf(rc);
      } else {
        d = (rw - pp * all_w) * fs;
        sd = 3.f * noise * sqrtf(fmaxf((1.f - pp) * (1.f - pp) * rv + pp * pp * (all_v - rv), 0.f)) + 1e-4f * hz;
      }
      reach[e] = rc * fs + 4.f * noise * sqrtf(rc);
      if (d + sd >= 0.f) atomicMax(&sm.pick_hi, bin);
      if (d - sd >= 0.f) atomicMax(&sm.pick_lo, bin);
    }
    __syncthreads();
    const int lo = sm.pick_lo, hi = sm.pick_hi;
    // tokens up to the bottom of the bracket: a list of all of them, where it fits
#pragma unroll
    for (int e = 0; e < 4; ++e)
    {
      const int bin = kCoarse - 1 - (4 * tid + e);
      if (bin == max(lo, 0)) sm.found[0] = static_cast<u64>(reach[e]);
      if (bin == max(hi, 0)) sm.found[1] = static_cast<u64>(fmaxf(reach[e] - hc[e] * fs, 0.f));
    }
    __syncthreads();
    Bracket b;
    b.all = lo > 0 && sm.found[0] + 64 <= (by_count ? kList / 2 : kList / 8);
    // (never -inf: what counts as -inf lies below every bracket)
    b.x0 = lo > 0 ? edge(lo) : -FLT_MAX;
    b.x1 = b.all || hi < 0 ? INFINITY : edge(hi + 1);
    b.listing = by_count || sm.found[0] - min(sm.found[0], sm.found[1]) <= 2 * kAim;
    b.ok = window_ok && hi > 0 && b.x0 < b.x1;
    __syncthreads();
    return b;
  };
  // A bracket of about kAim tokens inside b, whose weight (or count) is
  // `whole`: the target lies `part` below its top.
  auto narrow = [&](const Bracket& b, bool by_count, float part, float whole) {
    float in[4], n[4], si = 0.f, sn = 0.f;
#pragma unroll
    for (int e = 0; e < 4; ++e) {
      const int bin = kCoarse - 1 - (4 * tid + e);
      const bool inside = edge(bin) >= b.x0 && edge(bin) < b.x1;
      n[e] = inside ? hc[e] : 0.f;
      in[e] = inside ? (by_count ? hc[e] : hw[e]) : 0.f;
      si += in[e];
      sn += n[e];
    }
    u64 pi, pn;
    block_scan(sm, units(si), static_cast<u64>(sn), pi, pn);
    __syncthreads();
    if (tid == kThreads - 1) {
      sm.found[3] = pi + units(si);
      sm.pick_lo = kCoarse;
      sm.pick_hi = -1;
      sm.found[0] = 0;
    }
    __syncthreads();
    const float goal = part / whole * __ull2float_rn(sm.found[3]);
    float r = __ull2float_rn(pi), c = static_cast<float>(pn);
#pragma unroll
    for (int e = 0; e < 4; ++e) {
      if (r < goal && r + in[e] * kUnit >= goal) sm.found[0] = static_cast<u64>(c + 0.5f * n[e]) + 1;
      r += in[e] * kUnit;
      c += n[e];
    }
    __syncthreads();
    // half of kAim tokens to either side
    const float mid = static_cast<float>(sm.found[0]), half = 0.5f * kAim / fs;
    c = static_cast<float>(pn);
#pragma unroll
    for (int e = 0; e < 4; ++e) {
      const int bin = kCoarse - 1 - (4 * tid + e);
      if (n[e] > 0.f && c + n[e] >= mid - half && c <= mid + half) {
        atomicMax(&sm.pick_hi, bin);
        atomicMin(&sm.pick_lo, bin);
      }
      c += n[e];
    }
    __syncthreads();
    Bracket t;
    t.x0 = fmaxf(b.x0, edge(sm.pick_lo));
    t.x1 = fminf(b.x1, edge(sm.pick_hi + 1));
    t.all = false;
    t.listing = true;
    t.ok = sm.found[0] > 0 && t.x0 < t.x1;
    __syncthreads();
    return t;
  };

  // ---- pass 2: adds up the tokens x1 <= x < top (top: what is counted
  // already) and lists those in [x0, x1).  v: count and weight above, count
  // and weight of the list; `need_all`: v[1] is the row's whole weight and
  // what lies above is left in the segments alone.
  const float c_exp = inv * 1.4426950408889634f;
  u64 above_n = 0, above_q = 0;
  bool fits = false;  // the list holds all that it should
  auto pass = [&](const Bracket& b, float top, bool need_all, u64 (&v)[4]) {
    // fp32 weights: 2^((x - m) c) on tokens that are certain to be kept, or to
    // be part of a total (the list's are taken again with all their digits).
    // Straight code for every token, no branches but for the list's stores.
    LongSum fq, fa, fl;
    uint32_t n = 0, nl = 0;
    const float x0 = b.x0, x1 = b.x1;
    const bool listing = b.listing;
    int at = 0;  // tokens of the warp's region of the list
    row.batches(rank, [&](float (&x)[kUnroll][kVec], int i0) {
      float s = 0.f, sa = 0.f, sl = 0.f;
#pragma unroll
      for (int i = 0; i < kUnroll; ++i)
#pragma unroll
        for (int e = 0; e < kVec; ++e) {
          const float xe = x[i][e];
          const float w = fast_exp2((xe - m) * c_exp);
          const bool above = xe >= x1 && xe < top, in = xe >= x0 && xe < x1;
          sa += w;
          s += above ? w : 0.f;
          sl += in ? w : 0.f;
          n += above ? 1u : 0u;
          nl += in ? 1u : 0u;
          if (listing) {
            const unsigned who = __ballot_sync(kFull, in);
            if (who) {
              const int to = at + __popc(who & ((1u << lane) - 1u));
              if (in && to < kRegion) {
                sm.list.x[warp * kRegion + to] = xe;
                sm.list.idx[warp * kRegion + to] = Row<E>::index(i0, i, e);
              }
              at += __popc(who);
            }
          }
        }
      fq.add(s);
      fl.add(sl);
      fa.add(sa);
    });
    const u64 q = fq.total(), qa = fa.total(), ql = fl.total();
    if (lane == 0) sm.list_n[warp] = at;
    const u64 seg = warp_sum(q);
    if (lane == 0) {
      if (top == INFINITY)
        st_rank(&sm.seg[rank * kWarps + warp], 0, seg);
      else  // (only this warp writes its entry; rank 0 reads it after the exchange)
        st_rank(&sm.seg[rank * kWarps + warp], 0, seg + ld_rank_u64(&sm.seg[rank * kWarps + warp], 0));
    }
    // tokens listed, and (above 2^32) regions that overflowed
    v[0] = n;
    v[1] = q;
    v[2] = (lane == 0 && at > kRegion ? 1ull << 32 : 0ull) + nl;
    v[3] = need_all ? qa : ql;
    cluster_sum(sm, CL, rank, v);
    if (need_all) {  // the list's weight, in an exchange of its own
      u64 t[4] = {ql, 0, 0, 0};
      cluster_sum(sm, CL, rank, t);
      set_mass = v[3];
      v[3] = t[0];
    }
    fits = b.listing && v[2] >> 32 == 0 && v[2] <= kList;
    v[2] &= 0xffffffffull;
  };

  // The bracket of one limit, exact sums around it, and the search of the
  // list.  False: not settled (nothing changed).
  auto by_list = [&](bool by_count, bool& both) {
    Bracket b = estimate(by_count);
    if (!b.ok) return false;
    both = by_count && p < 1.f && b.all;
    float top = INFINITY;
    u64 v[4];
    above_n = above_q = 0;
    for (int round = 0;; ++round) {
      pass(b, top, !by_count && round == 0, v);
      above_n += v[0];
      above_q += v[1];
      const u64 target = by_count ? static_cast<u64>(k) : max(1ull, part_ceil(fmaxf(p, 0.f), set_mass));
      const u64 above = by_count ? above_n : above_q, upto = above + (by_count ? v[2] : v[3]);
      // kappa is in the list: less than the target lies above it, and no less with it
      const bool here = above < target && upto >= target;
      if (here && fits) break;
      if (round == 4) return false;
      both = false;
      // the part of the row that holds it, and its exact weight
      Bracket c = b;
      if (here) {
        top = b.x1;
        b = narrow(c, by_count, __ull2float_rn(target - above), __ull2float_rn(upto - above));
      } else {
        top = INFINITY;
        above_n = above_q = 0;
        if (above >= target) {
          c.x0 = b.x1;
          c.x1 = INFINITY;
          b = narrow(c, by_count, __ull2float_rn(target), __ull2float_rn(above));
        } else {
          // (the count of all tokens is not known: the histogram's will do)
          const float rest = by_count ? 0.f : __ull2float_rn(set_mass - min(set_mass, upto));
          c.x0 = -FLT_MAX;
          c.x1 = b.x0;
          if (!(rest > 0.f)) return false;
          b = narrow(c, by_count, __ull2float_rn(target - upto), rest);
        }
      }
      if (!b.ok) return false;
    }
    // this CTA's list without gaps
    {
      float lx[kWarps];
      int li[kWarps];
#pragma unroll
      for (int w = 0; w < kWarps; ++w)
        if (tid < sm.list_n[w]) {
          lx[w] = sm.list.x[w * kRegion + tid];
          li[w] = sm.list.idx[w * kRegion + tid];
        }
      __syncthreads();
      int to = 0;
#pragma unroll
      for (int w = 0; w < kWarps; ++w) {
        const int n = sm.list_n[w];
        if (tid < n) {
          sm.list.x[to + tid] = lx[w];
          sm.list.idx[to + tid] = li[w];
        }
        to += n;
      }
    }
    __syncthreads();
    // all lists go to rank 0, in the order of the CTAs
    if (CL > 1) {
      int own = 0;
      for (int w = 0; w < kWarps; ++w) own += sm.list_n[w];
      if (tid < CL) st_rank(&sm.x_sum[0][rank], tid, static_cast<u64>(own));
      sync_all(CL);
      int at = 0;
      for (int c = 0; c < rank; ++c) at += static_cast<int>(sm.x_sum[0][c]);
      if (rank > 0)
        for (int i = tid; i < own; i += kThreads) {
          st_rank(&sm.list.x[at + i], 0, __float_as_uint(sm.list.x[i]));
          st_rank(&sm.list.idx[at + i], 0, static_cast<uint32_t>(sm.list.idx[i]));
        }
      sync_all(CL);
    }
    if (rank == 0) {
      const int total = static_cast<int>(v[2]);
      const uint32_t key_lo = max(kKeyMin, ordered(b.x0));
      const uint32_t key_hi = b.x1 < m ? ordered(b.x1) : key_max;
      auto visit_list = [&](auto&& f) {
        for (int i = tid; i < total; i += kThreads) {
          const uint32_t key = ordered(sm.list.x[i]);
          if (kept.in_prefix(key, sm.list.idx[i])) f(key, units(wt.w(sm.list.x[i])));
        }
      };
      u64 set = set_mass;
      if (total <= kThreads) {
        // a thread per token: its rank and the weight before it, by comparing
        // it with all others (the histograms' memory holds keys and weights)
        u64* sk = reinterpret_cast<u64*>(sm.coarse);  // key, then lower index first
        u64* sq = reinterpret_cast<u64*>(sm.part);
        u64 mine = 0, own = 0;
        if (tid < total) {
          mine = static_cast<u64>(ordered(sm.list.x[tid])) << 32 | (0xffffffffu - static_cast<uint32_t>(sm.list.idx[tid]));
          own = units(wt.w(sm.list.x[tid]));
          sk[tid] = mine;
          sq[tid] = own;
        }
        __syncthreads();
        u64 before = 0;
        int place = 0;
        if (tid < total) {
#pragma unroll 8
          for (int j = 0; j < total; ++j) {
            const bool ahead = sk[j] > mine;
            place += ahead ? 1 : 0;
            before += ahead ? sq[j] : 0;
          }
        }
        const int limit = by_count ? static_cast<int>(min(static_cast<u64>(k) - above_n, static_cast<u64>(total))) : total;
        u64 none, s;
        block_scan(sm, 0, tid < total && place < limit ? own : 0, none, s);
        __syncthreads();
        if (tid == kThreads - 1) sm.found[4] = s + (tid < total && place < limit ? own : 0);
        __syncthreads();
        if (by_count) set = above_q + sm.found[4];
        u64 goal = ~0ull;
        if (!by_count || both) {
          goal = max(1ull, part_ceil(fmaxf(p, 0.f), set));
          goal = goal > above_q ? goal - above_q : 1;
        }
        // the last kept token: the last within the limit that begins before the goal
        const bool in = tid < total && place < limit && before < goal;
        if (tid == 0) sm.pick_lo = -1;
        __syncthreads();
        if (in) atomicMax(&sm.pick_lo, place);
        __syncthreads();
        if (in && place == sm.pick_lo) {
          sm.found[0] = mine;
          sm.pick_hi = place;
        }
        __syncthreads();
        kept.kappa = static_cast<uint32_t>(sm.found[0] >> 32);
        kept.last = static_cast<int>(0xffffffffu - static_cast<uint32_t>(sm.found[0]));
        if (in) {
          const int v2 = (sm.list.idx[tid] + row.lead) / kVec, c = v2 / row.per, w = (v2 - c * row.per) / row.per_warp;
          atomicAdd(&sm.seg[c * kWarps + w], own);
        }
        if (tid < CL) {
          st_rank(&sm.x_out[0], tid, sm.found[0] >> 32 << 32 | static_cast<uint32_t>(kept.last));
          st_rank(&sm.x_out[1], tid, set);
          st_rank(&sm.x_out[2], tid, above_n + sm.pick_hi + 1);
        }
      } else {
      // keep `quota` of the tokens at kappa: the lowest indices
      auto take = [&](const Found& f, u64 quota) {
        kept.move_to(f.key);
        if (quota >= f.at_count) return;
        const uint32_t kappa = f.key;
        auto visit_ties = [&](auto&& g) {
          for (int i = tid; i < total; i += kThreads)
            if (ordered(sm.list.x[i]) == kappa && sm.list.idx[i] <= kept.last)
              g(0xffffffffu - static_cast<uint32_t>(sm.list.idx[i]), 0ull);
        };
        const Found t =
            search<false>(sm, 1, true, quota, 0xffffffffu - static_cast<uint32_t>(a.V), 0xffffffffu, visit_ties);
        kept.last = static_cast<int>(0xffffffffu - t.key);
      };
      bool p_left = !by_count;
      if (by_count) {
        const u64 rest = static_cast<u64>(k) - above_n;
        const Found f = search<false>(sm, 1, true, rest, key_lo, key_hi, visit_list);
        if (f.ok) take(f, rest - f.above_count);
        p_left = both;
        // weight of the kept part of the list
        u64 s = 0, none, before;
        visit_list([&](uint32_t, u64 q2) { s += q2; });
        block_scan(sm, 0, s, none, before);
        __syncthreads();
        if (tid == kThreads - 1) sm.found[4] = before + s;
        __syncthreads();
        set = above_q + sm.found[4];
        __syncthreads();
      }
      if (p_left) {
        const u64 goal = max(1ull, part_ceil(fmaxf(p, 0.f), set));
        const u64 target = goal > above_q ? goal - above_q : 1;
        const Found f = search<false>(sm, 1, false, target, key_lo, key_hi, visit_list);
        if (f.ok) {
          const u64 one = max(units(wt.w(from_ordered(f.key))), 1ull);
          take(f, (target - f.above_mass + one - 1) / one);
        }
      }
      // the kept part of the list joins its segments
      // (neighbours in the list are mostly of one segment: one atomic a warp)
      u64 cnt = 0, none, before;
      for (int i0 = 32 * warp; i0 < total; i0 += kThreads) {
        const int i = i0 + lane;
        const bool in = i < total && kept.in_prefix(ordered(sm.list.x[i]), sm.list.idx[i]);
        const u64 one = in ? units(wt.w(sm.list.x[i])) : 0;
        int to = -1;
        if (in) {
          const int v2 = (sm.list.idx[i] + row.lead) / kVec, c = v2 / row.per;
          to = c * kWarps + (v2 - c * row.per) / row.per_warp;
        }
        cnt += in ? 1 : 0;
        const int first = __reduce_max_sync(kFull, to);
        if (first < 0) continue;
        if (__all_sync(kFull, !in || to == first)) {
          const u64 sum = warp_sum(one);
          if (lane == 0) atomicAdd(&sm.seg[first], sum);
        } else if (in) {
          atomicAdd(&sm.seg[to], one);
        }
      }
      block_scan(sm, cnt, 0, before, none);
      if (tid == kThreads - 1) {
        const u64 all = above_n + before + cnt;
        for (int c = 0; c < CL; ++c) {
          st_rank(&sm.x_out[0], c, static_cast<u64>(kept.kappa) << 32 | static_cast<uint32_t>(kept.last));
          st_rank(&sm.x_out[1], c, set);
          st_rank(&sm.x_out[2], c, all);
        }
      }
      }
    }
    sync_all(CL);
    kept.kappa = static_cast<uint32_t>(sm.x_out[0] >> 32);
    kept.last = static_cast<int>(static_cast<uint32_t>(sm.x_out[0]));
    set_mass = sm.x_out[1];
    kept_count = sm.x_out[2];
    have_seg = true;
    sync_all(CL);
    return true;
  };

  // the same by radix searches over the row
  auto by_row = [&](bool by_count) {
    have_seg = false;
    u64 target = static_cast<u64>(k);
    if (!by_count) {
      if (set_mass == 0) {
        u64 v[4] = {0, 0, 0, 0};
        visit_row([&](uint32_t, u64 w) { v[0] += w; });
        cluster_sum(sm, CL, rank, v);
        set_mass = v[0];
      }
      target = max(1ull, part_ceil(fmaxf(p, 0.f), set_mass));
    }
    const Found f = search<true>(sm, CL, by_count, target, kKeyMin, key_max, visit_row);
    if (!f.ok) return;
    const u64 one = max(units(wt.w(from_ordered(f.key))), 1ull);
    const u64 quota = by_count ? target - f.above_count : (target - f.above_mass + one - 1) / one;
    set_mass = f.above_mass + min(quota, f.at_count) * units(wt.w(from_ordered(f.key)));
    kept.move_to(f.key);
    if (quota < f.at_count) {
      auto visit_ties = [&](auto&& g) {
        row.batches(rank, [&](float (&x)[kUnroll][kVec], int i0) {
#pragma unroll
          for (int i = 0; i < kUnroll; ++i)
#pragma unroll
            for (int e = 0; e < kVec; ++e) {
              const int idx = Row<E>::index(i0, i, e);
              if (x[i][e] != -INFINITY && ordered(x[i][e]) == f.key && idx <= kept.last)
                g(0xffffffffu - static_cast<uint32_t>(idx), 0ull);
            }
        });
      };
      const Found t =
          search<true>(sm, CL, true, quota, 0xffffffffu - static_cast<uint32_t>(a.V), 0xffffffffu, visit_ties);
      kept.last = static_cast<int>(0xffffffffu - t.key);
    }
  };

  if (k > 0) {
    bool both = false;
    if (!by_list(true, both)) {
      both = false;
      by_row(true);
    }
    if (p < 1.f && !both) by_row(false);
  } else if (p < 1.f) {
    bool both = false;
    if (!by_list(false, both)) {
      set_mass = 0;
      by_row(false);
    }
  }

  // ---- the segments' weights, where pass 2 has not left them or min_p cuts
  if (!have_seg || mp > 0.f) {
    u64 n = 0, q = 0;
    const float least = from_ordered(kept.kappa);
    row.batches(rank, [&](float (&x)[kUnroll][kVec], int i0) {
      float any = -INFINITY;
#pragma unroll
      for (int i = 0; i < kUnroll; ++i)
#pragma unroll
        for (int e = 0; e < kVec; ++e) any = fmaxf(any, x[i][e]);
      if (any < least) return;
      BatchSum s;
      int cnt = 0;
#pragma unroll
      for (int i = 0; i < kUnroll; ++i)
#pragma unroll
        for (int e = 0; e < kVec; ++e) {
          const float w = wt.w(x[i][e]);
          const bool in = x[i][e] != -INFINITY && w >= mp &&
                          kept.in_prefix(ordered(x[i][e]), Row<E>::index(i0, i, e));
          s.add(in ? w : 0.f);
          cnt += in ? 1 : 0;
        }
      n += cnt;
      q += s.total();
    });
    const u64 seg = warp_sum(q);
    if (lane == 0) st_rank(&sm.seg[rank * kWarps + warp], 0, seg);
    u64 v[4] = {n, 0, 0, 0};
    cluster_sum(sm, CL, rank, v);
    kept_count = v[0];
  }

  // ---- rank 0 places the random number
  if (rank == 0) {
    // every warp for itself: lane i sums segments 4 i .. 4 i + 3
    u64 four[4], own4 = 0;
#pragma unroll
    for (int e = 0; e < 4; ++e) {
      four[e] = 4 * lane + e < CL * kWarps ? sm.seg[4 * lane + e] : 0;
      own4 += four[e];
    }
    u64 inc = own4;
#pragma unroll
    for (int o = 1; o < 32; o <<= 1) {
      const u64 y = __shfl_up_sync(kFull, inc, o);
      if (lane >= o) inc += y;
    }
    const u64 all = __shfl_sync(kFull, inc, 31);
    const float logz = log_units(all);
    const u64 thr = part_floor(u, all);
    const int who = __ffs(__ballot_sync(kFull, inc > thr)) - 1;  // (thr < all)
    u64 at = inc - own4;
    int s = 4 * lane;
#pragma unroll
    for (int e = 0; e < 3; ++e)
      if (s == 4 * lane + e && thr >= at + four[e]) {
        at += four[e];
        ++s;
      }
    at = __shfl_sync(kFull, at, who);
    s = __shfl_sync(kFull, s, who);
    if (tid == 0) {
      sm.token = -1;
      sm.pick_lo = -1;
      if (a.kept) a.kept[r] = static_cast<int>(kept_count);
      for (int c = 0; c < CL; ++c) st_rank(&sm.x_out[3], c, static_cast<u64>(__float_as_uint(logz)));
    }
    __syncthreads();
    const int sr = s / kWarps, sw = s - sr * kWarps;
    const int va = row.seg_begin(sr, sw), vb = min(row.seg_begin(sr, sw + 1), min(row.vecs, sr * row.per + row.per));
    for (int v0 = va; v0 < vb; v0 += kThreads) {
      const int v = v0 + tid;
      float x[kVec];
      u64 own = 0, q[kVec];
      int last = -1;
      if (v < vb) row.load(v, x);
#pragma unroll
      for (int e = 0; e < kVec; ++e) {
        q[e] = 0;
        const int idx = v * kVec - row.lead + e;
        if (v < vb && x[e] != -INFINITY && kept.in_prefix(ordered(x[e]), idx)) {
          const float w = wt.w(x[e]);
          if (w >= mp) {
            q[e] = units(w);
            if (q[e]) last = idx;
          }
        }
        own += q[e];
      }
      if (last >= 0) atomicMax(&sm.pick_lo, last);  // the last kept token of the segment
      u64 before, none;
      block_scan(sm, own, 0, before, none);
      before += at;
      if (own && thr >= before && thr < before + own) {
#pragma unroll
        for (int e = 0; e < kVec; ++e) {
          if (q[e] && thr >= before && thr < before + q[e]) sm.token = v * kVec - row.lead + e;
          before += q[e];
        }
      }
      __syncthreads();
      if (sm.token >= 0) break;
      // the sum so far, from the warps' totals of the scan
      u64 t = lane < kWarps ? sm.warp_a[lane] : 0;
      t = warp_sum(t);
      at += t;
    }
    __syncthreads();
    if (tid == 0) {
      // rounding of the segment's sum may leave the number just past its last token
      const int tok = sm.token >= 0 ? sm.token : sm.pick_lo;
      a.token[r] = tok;
      if (a.log_prob) a.log_prob[r] = wt.z(static_cast<float>(row.base[row.lead + tok])) - logz;
    }
  }
  if (a.log_probs) {
    sync_all(CL);
    const float logz = __uint_as_float(static_cast<uint32_t>(sm.x_out[3]));
    float* out = a.log_probs + static_cast<size_t>(r) * a.V;
    row.batches(rank, [&](float (&x)[kUnroll][kVec], int i0) {
#pragma unroll
      for (int i = 0; i < kUnroll; ++i)
#pragma unroll
        for (int e = 0; e < kVec; ++e) {
          const int idx = Row<E>::index(i0, i, e);
          // (vectors past the segment's end hold -inf but are not this warp's)
          const int v = (idx + row.lead) / kVec;
          if (idx < 0 || idx >= a.V || v >= min(row.seg_begin(rank, warp + 1), min(row.vecs, rank * row.per + row.per)))
            continue;
          const float z = wt.z(x[i][e]);
          const bool in = x[i][e] != -INFINITY && kept.in_prefix(ordered(x[i][e]), idx) && (mp <= 0.f || expf(z) >= mp);
          out[idx] = in ? z - logz : -INFINITY;
        }
    });
  }
  pdl_launch_next();
  sync_all(CL);  // no CTA leaves while another may write to its shared memory
}

template <typename E>
cudaError_t launch_e(const SampleArgs& a, int num_sms, cudaStream_t stream) {
  {
    static std::mutex mu;
    static bool done[64] = {};
    int dev = 0;
    cudaError_t e = cudaGetDevice(&dev);
    if (e != cudaSuccess) return e;
    if (dev < 0 || dev >= 64) return cudaErrorInvalidDevice;
    std::lock_guard<std::mutex> lk(mu);
    if (!done[dev]) {
      e = cudaFuncSetAttribute(sample_kernel<E>, cudaFuncAttributeMaxDynamicSharedMemorySize,
                               static_cast<int>(sizeof(Smem)));
      if (e != cudaSuccess) return e;
      done[dev] = true;
    }
  }
  // Two CTAs fit a SM: as many CTAs a row as fit at once, none for less than
  // 4096 tokens.  (More CTAs for many rows would keep the rows in work within
  // L2 between the passes, but cost more in exchanges than that gains: 1024
  // rows of 151936 take 0.87 ms with one, 0.95 ms with two, 1.27 ms with four.)
  int CL = kMaxCluster;
  while (CL > 1 && (a.R * static_cast<long long>(CL) > 2ll * num_sms || a.V < 4096 * CL)) CL >>= 1;
  return launch_overlapped(sample_kernel<E>, dim3(static_cast<unsigned>(a.R) * CL), dim3(kThreads), sizeof(Smem),
                           stream, static_cast<unsigned>(CL), a, CL);
}

}  // namespace

cudaError_t launch_sample(int elem_bytes, const SampleArgs& a, int num_sms, cudaStream_t stream) {
  return elem_bytes == 4 ? launch_e<float>(a, num_sms, stream) : launch_e<__nv_bfloat16>(a, num_sms, stream);
}

}  // namespace simsd
