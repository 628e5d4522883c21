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
// A row is read twice.  The first pass (from HBM) takes the maximum and a
// histogram of counts over bins 1/128 wide in x / T.  A bin's weights differ
// by less than a factor rho = e^(1/128), so the histogram brackets kappa: to
// the bin that holds the k-th count, or to the bins where the cumulative
// weight, known within rho, can reach top_p of the total.  The second pass
// (from L2) sums the weights above the bracket and lists the tokens inside
// it; one CTA then searches that list in shared memory.  Rows whose bracket
// holds more than kList tokens (very flat ones with top_p near 1) go through
// a radix search over the row instead (3 more passes).  The random number is
// placed by the weights of the row's segments (one per warp), and only the
// segment it falls in is read again.
//
// A thread-block cluster serves a row: one CTA where there are many rows,
// up to eight where there are few.
#include <cuda_bf16.h>
#include <cuda_runtime.h>

#include <algorithm>
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
constexpr int kUnroll = 4;        // vectors of a lane in flight
constexpr int kCoarse = 8192;     // bins of the first pass
constexpr float kBinsPerUnit = 128.f;
constexpr float kRho = 1.0080f;   // above e^(1/128) = 1.00784, with room for rounding
constexpr int kList = 8192;       // tokens inside the bracket
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
    uint32_t coarse[kCoarse];
    struct {
      float x[kList];
      int idx[kList];
    } list;
  };
  u64 mass[kFine];
  uint32_t count[kFine];
  u64 seg[kMaxCluster * kWarps];  // weights of the row's segments (rank 0 holds all)
  u64 warp_a[kWarps], warp_b[kWarps];
  u64 x_max[kMaxCluster];                          // exchanges over the cluster: one slot per CTA
  u64 x_sum[3][kMaxCluster];
  u64 x_out[4];
  u64 found[5];
  int list_n, pick_lo, pick_hi, token;
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
  static constexpr int kVec = 16 / sizeof(E);
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
    for (int e = 0; e < kVec; ++e) x[e] = x[e] == x[e] ? x[e] : -INFINITY;
  }
  __device__ __forceinline__ int seg_begin(int rank, int warp) const {
    return min(min(vecs, rank * per + per), min(vecs, rank * per) + warp * per_warp);
  }
  // batches of kUnroll vectors of this thread's segment: f(x, first index of each vector)
  template <typename F>
  __device__ __forceinline__ void batches(int rank, F&& f) const {
    const int warp = threadIdx.x >> 5, lane = threadIdx.x & 31;
    const int a = seg_begin(rank, warp), b = min(seg_begin(rank, warp + 1), min(vecs, rank * per + per));
    for (int v = a + lane; v < b; v += 32 * kUnroll) {
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

// Sums over the cluster of up to three values that each warp's lane 0 has
// left in seg_a / seg_b / seg_c (arrays of kWarps); slot arrays x_sum.
// Returns with all CTAs knowing all sums; the caller may reuse the slots
// after the next sync_all.
__device__ void cluster_sum3(Smem& sm, int CL, int rank, u64 a, u64 b, u64 c, u64 (&out)[3]) {
  const int lane = threadIdx.x & 31, warp = threadIdx.x >> 5;
  a = warp_sum(a);
  b = warp_sum(b);
  c = warp_sum(c);
  if (lane == 0) {
    sm.warp_a[warp] = a;
    sm.warp_b[warp] = b;
    sm.mass[warp] = c;
  }
  __syncthreads();
  if (warp == 0) {
    u64 x = lane < kWarps ? sm.warp_a[lane] : 0, y = lane < kWarps ? sm.warp_b[lane] : 0;
    u64 z = lane < kWarps ? sm.mass[lane] : 0;
    x = warp_sum(x);
    y = warp_sum(y);
    z = warp_sum(z);
    if (lane < CL) {
      st_rank(&sm.x_sum[0][rank], lane, x);
      st_rank(&sm.x_sum[1][rank], lane, y);
      st_rank(&sm.x_sum[2][rank], lane, z);
    }
  }
  sync_all(CL);
  for (int s = 0; s < 3; ++s) {
    u64 v = 0;
    for (int r = 0; r < CL; ++r) v += sm.x_sum[s][r];
    out[s] = v;
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
  pc = ic - c;
  pq = iq - q;
  for (int w = 0; w < warp; ++w) {
    pc += sm.warp_a[w];
    pq += sm.warp_b[w];
  }
}

// What a search finds: the key at which the count (or the weight) from the
// highest key down first reaches the target, what lies above it, and at it.
struct Found {
  uint32_t key;
  u64 above_count, above_mass, at_count;
  bool ok;  // false: everything together does not reach the target
};

// Search over keys in [lo, hi], a digit of up to 11 bits per round.
// visit(f) calls f(key, weight units) for the elements; CL > 1: every CTA
// of the cluster visits its own, and all get the result.
template <typename Visit>
__device__ Found search(Smem& sm, int CL, bool by_count, u64 target, uint32_t lo, uint32_t hi, Visit&& visit) {
  Found f{0u, 0, 0, 0, true};
  for (;;) {
    const uint32_t span = hi - lo;
    const int bits = 32 - __clz(span);  // (clz(0) = 32)
    const int shift = max(0, bits - 11);
    for (int i = threadIdx.x; i < kFine; i += kThreads) {
      sm.count[i] = 0;
      sm.mass[i] = 0;
    }
    sync_all(CL);
    visit([&](uint32_t key, u64 q) {
      if (key < lo || key > hi) return;
      const uint32_t bin = (key - lo) >> shift;
      atomicAdd(&sm.count[bin], 1u);
      if (q) atomicAdd(&sm.mass[bin], q);
    });
    sync_all(CL);
    // thread t: bins 4 t .. 4 t + 3 from the top
    u64 c[4], q[4], sc = 0, sq = 0;
#pragma unroll
    for (int e = 0; e < 4; ++e) {
      const int bin = kFine - 1 - (4 * static_cast<int>(threadIdx.x) + e);
      c[e] = q[e] = 0;
      if (CL == 1) {
        c[e] = sm.count[bin];
        q[e] = sm.mass[bin];
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
    sync_all(CL);  // the histograms are read by all before they are cleared
    lo += static_cast<uint32_t>(bin) << shift;
    if (shift == 0) {
      f.key = lo;
      return f;
    }
    hi = min(hi, lo + ((1u << shift) - 1u));
  }
}

template <typename E>
__global__ void __launch_bounds__(kThreads, 2) sample_kernel(const __grid_constant__ SampleArgs a, const int CL) {
  extern __shared__ uint4 smem_raw[];
  Smem& sm = *reinterpret_cast<Smem*>(smem_raw);
  constexpr int kVec = Row<E>::kVec;
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

  // ---- pass 1: the maximum, and counts over bins of x / T
  float base = 0.f;
  if (cut) {
    for (int i = tid; i < kCoarse; i += kThreads) sm.coarse[i] = 0;
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
  // bin of x: floor of y(x), not falling in x
  const float scale = inv * kBinsPerUnit;
  auto yof = [&](float x) {
    return fminf(fmaxf(fmaf(x - base, scale, 0.5f * kCoarse), 0.f), static_cast<float>(kCoarse - 1));
  };
  float mx = -INFINITY;
  if (cut) {
    row.batches(rank, [&](float (&x)[kUnroll][kVec], int) {
#pragma unroll
      for (int i = 0; i < kUnroll; ++i)
#pragma unroll
        for (int e = 0; e < kVec; ++e) {
          mx = fmaxf(mx, x[i][e]);
          atomicAdd(&sm.coarse[__float2int_rd(yof(x[i][e]))], 1u);
        }
    });
  } else {
    row.batches(rank, [&](float (&x)[kUnroll][kVec], int) {
#pragma unroll
      for (int i = 0; i < kUnroll; ++i)
#pragma unroll
        for (int e = 0; e < kVec; ++e) mx = fmaxf(mx, x[i][e]);
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

  // ---- one stage for top_k (by_count), one for top_p
  auto stage = [&](bool by_count) {
    // the bracket, from the histogram: bins [pick_lo, pick_hi]; thread t
    // holds 16 bins from the top
    constexpr int kPer = kCoarse / kThreads;
    float c[kPer], w[kPer];
    float sw = 0.f;
    u64 sc = 0;
#pragma unroll
    for (int e = 0; e < kPer; ++e) {
      const int bin = kCoarse - 1 - (kPer * tid + e);
      uint32_t n = 0;
      if (CL == 1)
        n = sm.coarse[bin];
      else
        for (int q = 0; q < CL; ++q) n += ld_rank_u32(&sm.coarse[bin], q);
      c[e] = static_cast<float>(n);
      // weight of the bin's lower edge (of the window's ends: of nothing)
      const float edge = (static_cast<float>(bin) - 0.5f * kCoarse) / kBinsPerUnit - (m - base) * inv;
      w[e] = n ? static_cast<float>(n) * expf(fminf(edge, 0.f)) : 0.f;
      sc += n;
      sw += w[e];
    }
    // (weights as units of 2^-38, as the sums are)
    u64 pc, pq, all_q;
    block_scan(sm, sc, units(sw), pc, pq);
    if (tid == kThreads - 1) sm.found[4] = pq + units(sw);
    if (tid == 0) {
      sm.pick_hi = -1;
      sm.pick_lo = -1;
      sm.list_n = 0;
    }
    __syncthreads();
    all_q = sm.found[4];
    // early: the first bin by which the target may be reached; late: the
    // first by which it must have been
    const float part = fmaxf(p, 0.f) * __ull2float_rn(all_q);
    const u64 t_early = by_count ? static_cast<u64>(k) : __float2ull_rz(part * (0.9999f / kRho));
    const u64 t_late = by_count ? static_cast<u64>(k) : __float2ull_rz(part * (1.0001f * kRho)) + 1;
    float run = 0.f;
#pragma unroll
    for (int e = 0; e < kPer; ++e) {
      const int bin = kCoarse - 1 - (kPer * tid + e);
      const u64 b0 = by_count ? pc : pq + units(run);
      pc += static_cast<u64>(c[e]);
      run += w[e];
      const u64 b1 = by_count ? pc : pq + units(run);
      if (c[e] > 0.f || bin == 0) {
        if (b0 <= t_early && (b1 > t_early || (by_count && b1 >= t_early))) atomicMax(&sm.pick_hi, bin);
        if (b0 < t_late && b1 >= t_late) atomicMax(&sm.pick_lo, bin);
      }
    }
    __syncthreads();
    int hi = sm.pick_hi, lo = sm.pick_lo;
    if (hi < 0) hi = kCoarse - 1;
    // not reached for certain, or weights that the window does not bound
    if (lo < 0 || !(scale < 1e30f) || !(fmaf(m - base, scale, 0.5f * kCoarse) < kCoarse - 1)) lo = 0;
    // both limits: with all of the top_k in the list top_p needs no pass of its own
    const bool both = by_count && p < 1.f;
    // tokens in bins lo .. hi and lo .. top
    u64 n_in = 0, n_up = 0;
    {
      u64 in = 0, up = 0;
#pragma unroll
      for (int e = 0; e < kPer; ++e) {
        const int bin = kCoarse - 1 - (kPer * tid + e);
        if (bin >= lo) up += static_cast<u64>(c[e]);
        if (bin >= lo && bin <= hi) in += static_cast<u64>(c[e]);
      }
      u64 ex_in, ex_up;
      block_scan(sm, in, up, ex_in, ex_up);
      if (tid == kThreads - 1) {
        sm.found[0] = ex_in + in;
        sm.found[1] = ex_up + up;
      }
      __syncthreads();
      n_in = sm.found[0];
      n_up = sm.found[1];
    }
    sync_all(CL);  // the histogram is read by all; the list may take its place
    return make_int4(lo, both && n_up <= kList ? kCoarse - 1 : hi,
                     static_cast<int>(min(both && n_up <= kList ? n_up : n_in, static_cast<u64>(0x7fffffff))), both && n_up <= kList);
  };

  // pass 2 and the search of the list.  Returns false where the list would
  // not hold the bracket (nothing done).
  auto by_list = [&](bool by_count, int4 br) {
    if (br.z > kList || br.x == 0) return false;  // (bin 0 also holds -inf and all below the window)
    const float y0 = static_cast<float>(br.x), y1 = static_cast<float>(br.y + 1);
    const bool need_all = !by_count && set_mass == 0;
    u64 n = 0, q = 0, qa = 0;
    row.batches(rank, [&](float (&x)[kUnroll][kVec], int i0) {
      BatchSum s, sa;
      int cnt = 0;
#pragma unroll
      for (int i = 0; i < kUnroll; ++i)
#pragma unroll
        for (int e = 0; e < kVec; ++e) {
          const float y = yof(x[i][e]);
          const bool above = y >= y1;
          if (need_all || above) {
            const float w = wt.w(x[i][e]);
            sa.add(w);
            s.add(above ? w : 0.f);
          }
          cnt += above ? 1 : 0;
          if (!above && y >= y0) {
            const int at = atomicAdd(&sm.list_n, 1);
            sm.list.x[at] = x[i][e];
            sm.list.idx[at] = Row<E>::index(i0, i, e);
          }
        }
      n += cnt;
      q += s.total();
      qa += sa.total();
    });
    const u64 seg = warp_sum(q);
    if (lane == 0) st_rank(&sm.seg[rank * kWarps + warp], 0, seg);
    u64 out[3];
    cluster_sum3(sm, CL, rank, n, q, qa, out);
    // all lists go to rank 0, in the order of the CTAs
    const int own = sm.list_n;
    if (CL > 1) {
      if (tid < CL) st_rank(&sm.x_sum[0][rank], tid, static_cast<u64>(own));
      sync_all(CL);
      int at = 0, all = 0;
      for (int c = 0; c < CL; ++c) {
        if (c < rank) at += static_cast<int>(sm.x_sum[0][c]);
        all += static_cast<int>(sm.x_sum[0][c]);
      }
      if (rank > 0)
        for (int i = tid; i < own; i += kThreads) {
          st_rank(&sm.list.x[at + i], 0, __float_as_uint(sm.list.x[i]));
          st_rank(&sm.list.idx[at + i], 0, static_cast<uint32_t>(sm.list.idx[i]));
        }
      sync_all(CL);
      if (rank == 0 && tid == 0) sm.list_n = all;
    }
    __syncthreads();
    if (rank == 0) {
      const int total = sm.list_n;
      auto visit_list = [&](auto&& f) {
        for (int i = tid; i < total; i += kThreads) {
          const uint32_t key = ordered(sm.list.x[i]);
          if (kept.in_prefix(key, sm.list.idx[i])) f(key, units(wt.w(sm.list.x[i])));
        }
      };
      u64 set = set_mass;
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
        const Found t = search(sm, 1, true, quota, 0xffffffffu - static_cast<uint32_t>(a.V), 0xffffffffu, visit_ties);
        kept.last = static_cast<int>(0xffffffffu - t.key);
      };
      bool p_left = !by_count;
      if (by_count) {
        const Found f = search(sm, 1, true, static_cast<u64>(k) - out[0], kKeyMin, key_max, visit_list);
        if (f.ok) take(f, static_cast<u64>(k) - out[0] - f.above_count);
        p_left = br.w != 0;
        // weight of the kept part of the list
        u64 s = 0, none, before;
        visit_list([&](uint32_t, u64 q2) { s += q2; });
        block_scan(sm, 0, s, none, before);
        if (tid == kThreads - 1) sm.found[4] = before + s;
        __syncthreads();
        set = out[1] + sm.found[4];
        __syncthreads();
      } else if (need_all) {
        set = out[2];
      }
      if (p_left) {
        u64 target = max(1ull, part_ceil(fmaxf(p, 0.f), set));
        target = target > out[1] ? target - out[1] : 1;
        const Found f = search(sm, 1, false, target, kKeyMin, key_max, visit_list);
        if (f.ok) {
          const u64 one = max(units(wt.w(from_ordered(f.key))), 1ull);
          take(f, (target - f.above_mass + one - 1) / one);
        }
      }
      // the kept part of the list joins its segments
      u64 cnt = 0, none, before;
      for (int i = tid; i < total; i += kThreads) {
        const uint32_t key = ordered(sm.list.x[i]);
        if (!kept.in_prefix(key, sm.list.idx[i])) continue;
        ++cnt;
        const int v = (sm.list.idx[i] + row.lead) / kVec, c = v / row.per, w = (v - c * row.per) / row.per_warp;
        atomicAdd(&sm.seg[c * kWarps + w], units(wt.w(sm.list.x[i])));
      }
      block_scan(sm, cnt, 0, before, none);
      if (tid == kThreads - 1) {
        const u64 all = out[0] + before + cnt;
        for (int c = 0; c < CL; ++c) {
          st_rank(&sm.x_out[0], c, static_cast<u64>(kept.kappa) << 32 | static_cast<uint32_t>(kept.last));
          st_rank(&sm.x_out[1], c, set);
          st_rank(&sm.x_out[2], c, all);
        }
      }
    }
    sync_all(CL);
    kept.kappa = static_cast<uint32_t>(sm.x_out[0] >> 32);
    kept.last = static_cast<int>(static_cast<uint32_t>(sm.x_out[0]));
    set_mass = sm.x_out[1];
    kept_count = sm.x_out[2];
    have_seg = true;
    return true;
  };

  // the same by radix searches over the row
  auto by_row = [&](bool by_count) {
    have_seg = false;
    u64 target = static_cast<u64>(k);
    if (!by_count) {
      if (set_mass == 0) {
        u64 q = 0, out[3];
        visit_row([&](uint32_t, u64 w) { q += w; });
        cluster_sum3(sm, CL, rank, q, 0, 0, out);
        set_mass = out[0];
      }
      target = max(1ull, part_ceil(fmaxf(p, 0.f), set_mass));
    }
    const Found f = search(sm, CL, by_count, target, kKeyMin, key_max, visit_row);
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
      const Found t = search(sm, CL, true, quota, 0xffffffffu - static_cast<uint32_t>(a.V), 0xffffffffu, visit_ties);
      kept.last = static_cast<int>(0xffffffffu - t.key);
    }
  };

  if (k > 0) {
    const int4 br = stage(true);
    const bool listed = by_list(true, br);
    if (!listed) by_row(true);
    if (p < 1.f && !(listed && br.w)) by_row(false);
  } else if (p < 1.f) {
    const int4 br = stage(false);
    if (!by_list(false, br)) by_row(false);
  }

  // ---- the segments' weights, where pass 2 has not left them or min_p cuts
  if (!have_seg || mp > 0.f) {
    u64 n = 0, q = 0;
    row.batches(rank, [&](float (&x)[kUnroll][kVec], int i0) {
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
    u64 out[3];
    cluster_sum3(sm, CL, rank, n, 0, 0, out);
    kept_count = out[0];
  }

  // ---- rank 0 places the random number
  if (rank == 0) {
    u64 all = 0;
    for (int s = 0; s < CL * kWarps; ++s) all += sm.seg[s];
    const float logz = log_units(all);
    const u64 thr = part_floor(u, all);
    int s = 0;
    u64 at = 0;
    while (s < CL * kWarps - 1 && thr >= at + sm.seg[s]) at += sm.seg[s++];
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
      for (int w = 0; w < kWarps; ++w) at += sm.warp_a[w];
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
  // two CTAs a SM: as many CTAs a row as make about four rounds of them, but
  // none for less than 2048 tokens
  int CL = kMaxCluster;
  while (CL > 1 && (static_cast<long long>(a.R) * CL > 8ll * num_sms || a.V < 2048 * CL)) CL >>= 1;
  return launch_overlapped(sample_kernel<E>, dim3(static_cast<unsigned>(a.R) * CL), dim3(kThreads), sizeof(Smem),
                           stream, static_cast<unsigned>(CL), a, CL);
}

}  // namespace

cudaError_t launch_sample(int elem_bytes, const SampleArgs& a, int num_sms, cudaStream_t stream) {
  return elem_bytes == 4 ? launch_e<float>(a, num_sms, stream) : launch_e<__nv_bfloat16>(a, num_sms, stream);
}

}  // namespace simsd
