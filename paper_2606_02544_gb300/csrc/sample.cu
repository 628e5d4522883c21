// sample.cu -- draws a token from each row of logits with a given random
// number, after temperature, top-k, top-p and min-p (Sec. 3.2: drafts come
// from the draft model's distribution).
//
// Mathematics.  w_v = exp((x_v - m) / T), m = max x.  The kept set is a
// prefix of the order (x falling, index rising): {x > kappa} and the tokens
// x = kappa up to some index, cut by w >= min_p.  The sums that top_p decides
// by are 64-bit integers in units of 2^-38 of the largest weight; the random
// number is placed in units of 2^-88, so that the smallest weights have their
// share of it.
//
// A row is read twice.  The first pass (from HBM) takes the maximum and a
// histogram over 2048 bins of x / T: counts for top_k, weights to 2^-17 of
// themselves for top_p.  That names the bin of kappa (a bracket of a few where
// top_p falls near a bin's edge).  The second pass (the last vectors first,
// which are still in L2) adds up what lies above the bin and lists the tokens
// inside it; one CTA sorts the list (bitonic, mostly in registers) and cuts
// it.  Sums that contradict the histogram, or more tokens in the bin than the
// list holds (many equal logits), send the row through radix searches (400
// rows of 151936 equal logits: 1.9 ms); a row whose open tokens the sample
// missed, as nearly all are masked, has its histogram taken once more around
// the maximum (8 rows with 10 open tokens: 45 us).  The random number is placed
// by the weights of the row's segments (one per warp), and only the segment it
// falls in is read again.
//
// The second pass takes a weight as 2^(c (x - m)), c = log2(e) / T in fp32,
// which is good to (|z| + 1) 2^-22 of itself, z = (x - m) / T; the list, the
// searches and the place within a segment take e^z of the correctly rounded z.
// Against 64-bit sums, normal logits in rows of 1066 to 151936: all of 8192
// random numbers gave the same token; under top_p 12 of 5096 rows kept one
// token more or less.
//
// Counting all of a row costs one shared-memory reduction a token, which HBM
// can feed; counts of an eighth of it left brackets of thousands of tokens
// under heavy-tailed weights and a third pass over the row (1024 rows of
// 151936: 898 us, this way 320).
//
// Measured, 151936 logits of fp32: 1024 rows 320 us (1.9 TB/s of the bytes
// read once, 3.8 of those read; each pass about 70% of the time in the
// instructions of a token, 16 and 11, and HBM), 8 rows 23 us (a chain of
// passes and exchanges over a cluster); 132 rows of 32003 in bf16 with their
// distribution 51 us.
//
// A thread-block cluster serves a row: one CTA where there are many rows (of
// 256 threads where they are short), up to eight where there are few.
#include <cuda_bf16.h>
#include <cuda_runtime.h>

#include <algorithm>
#include <cfloat>
#include <cmath>
#include <mutex>
#include <type_traits>

#include "common.cuh"
#include "kernels.h"
#include "ptx.cuh"

namespace simsd {
namespace {

typedef unsigned long long u64;
typedef unsigned __int128 u128;

constexpr int kMaxWarps = 16;    // of a CTA: 512 threads (NT) for few rows, 256 for many
constexpr int kMaxCluster = 8;
constexpr int kBatch = 16;         // elements of a lane in flight
constexpr int kBins = 2048;       // bins of the first pass
constexpr int kLower = 1536;      // of them below the base, over at most kBelow in x / T ...
constexpr float kBelow = 48.f, kAbove = 48.f;  // ... the others above it, over kAbove
constexpr int kList = 4096;       // tokens of the list
constexpr int kAll = 512;         // a list of no more tokens may hold all of the set
constexpr int kSmallV = 32768;
constexpr int kFine = 2048;       // bins of the searches
constexpr int kUnitBits = 38;
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

// What the random number is placed by: units of 2^-88, so that tokens far
// below the largest keep their share (a row may be one token of weight 1 and
// 150,000 of 2^-40: the first 2^-24 of the random numbers fall on those), as
// whole units of 2^-38 and the rest where they are added up apart.
constexpr int kFineBits = 50;
struct Parts {
  u64 coarse, fine;
};
__device__ __forceinline__ Parts parts(float w) {
  const float t = w * kUnit, f = floorf(t);
  return Parts{__float2ull_rz(f), __float2ull_rn((t - f) * 1125899906842624.0f)};
}
// (added up modulo 2^64, the rests as signed numbers: they may have come out negative)
__device__ __forceinline__ Parts parts(const LongSum& s) {
  const Parts h = parts(s.hi), l = parts(fabsf(s.lo));
  return s.lo < 0.f ? Parts{h.coarse - l.coarse, h.fine - l.fine} : Parts{h.coarse + l.coarse, h.fine + l.fine};
}
__device__ __forceinline__ u128 join(u64 coarse, u64 fine) {
  return (static_cast<u128>(coarse) << kFineBits) + static_cast<u128>(static_cast<__int128>(static_cast<long long>(fine)));
}
// The floor of a sum's part f, f in [0, 1), exact: the 24 bits of f times the
// sum, which is below 2^112, shifted by the exponent.
__device__ __forceinline__ u128 part_floor(float f, u128 sum) {
  const uint32_t b = __float_as_uint(f) & 0x7fffffffu;  // (-0 is in range)
  const int shift = b >> 23 ? 150 - static_cast<int>(b >> 23) : 149;  // 24 .. 149
  const uint32_t m = (b & 0x7fffffu) | (b >> 23 ? 0x800000u : 0u);
  const u128 low = static_cast<u128>(static_cast<u64>(sum)) * m, high = static_cast<u128>(static_cast<u64>(sum >> 64)) * m;
  return shift < 64 ? (high << (64 - shift)) + (low >> shift) : (high + (low >> 64)) >> (shift - 64);
}

// The part f of a sum in units of 2^-38, f in [0, 1): ceiling.
__device__ __forceinline__ u64 fraction(float f) { return __float2ull_rz(f * 18446744073709551616.0f); }
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
// product with 1 / T, where that has not passed the largest number, as with
// masks of the type's lowest value and T < 1); infinite m: the tokens at m
// share the weight.
struct Weight {
  float m, T, inv;
  __device__ __forceinline__ float z(float x) const {
    const float d = x - m;
    const float q = d * inv;
    const float r = fmaf(-q, T, d);
    const float c = T > 1e-18f ? (isinf(q) ? q : fmaf(r, inv, q)) : d / T;
    return x == m ? 0.f : c;
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

template <int NT>
struct alignas(16) Smem {
  static constexpr int kWarps = NT / 32;
  union {
    u64 list[kList];  // ordered pattern, then the lower index first
    u64 mass[kFine];  // searches over the row
  };
  uint32_t hist[kBins];  // pass 1: counts, or weights in 2^-16 of their bin's middle
  uint32_t count[kFine];
  u64 seg[kMaxCluster * kMaxWarps];  // weights of the row's segments (rank 0 holds all): units of 2^-38 ...
  u64 seg_fine[kMaxCluster * kMaxWarps];  // ... and of 2^-88
  u64 warp_a[kWarps], warp_b[kWarps], warp_v[4][kWarps];
  u64 x_max[kMaxCluster];                          // exchanges over the cluster: one slot per CTA
  u64 x_sum[2][4][kMaxCluster];                    // (in turn, so that a sum costs one barrier)
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
template <typename E, int NT>
struct Row {
  static constexpr int kVec = 16 / sizeof(E), kUnroll = kBatch / kVec;
  const E* base;  // 16-byte aligned; `lead` elements before the row
  int lead, V;
  int vecs, per, per_warp;  // vectors of the row, of a CTA, of a segment

  // (a NaN counts as -inf)
  __device__ static __forceinline__ void unpack(const uint4& q, float (&x)[kVec]) {
    const uint32_t w[4] = {q.x, q.y, q.z, q.w};
#pragma unroll
    for (int e = 0; e < kVec; ++e)
      x[e] = fmaxf(sizeof(E) == 4 ? __uint_as_float(w[e])
                                  : __uint_as_float(e & 1 ? w[e / 2] & 0xffff0000u : w[e / 2] << 16),
                   -INFINITY);
  }
  __device__ __forceinline__ uint4 vector(int v) const { return reinterpret_cast<const uint4*>(base)[v]; }
  // (elements outside the row count as -inf)
  __device__ __forceinline__ void load(int v, float (&x)[kVec]) const {
    const int i0 = v * kVec - lead;
    if (i0 >= 0 && i0 + kVec <= V) {
      unpack(vector(v), x);
    } else {
      const E* p = base + static_cast<size_t>(v) * kVec;
#pragma unroll
      for (int e = 0; e < kVec; ++e)
        x[e] = i0 + e >= 0 && i0 + e < V ? fmaxf(static_cast<float>(p[e]), -INFINITY) : -INFINITY;
    }
  }
  __device__ __forceinline__ int seg_begin(int rank, int warp) const {
    return min(min(vecs, rank * per + per), min(vecs, rank * per) + warp * per_warp);
  }
  // batches of kUnroll vectors of this thread's segment: f(x, first index of each vector);
  // kBack: the last first
  template <bool kBack = false, typename F>
  __device__ __forceinline__ void batches(int rank, F&& f) const {
    const int warp = threadIdx.x >> 5, lane = threadIdx.x & 31;
    const int a = seg_begin(rank, warp), b = min(seg_begin(rank, warp + 1), min(vecs, rank * per + per));
    const int whole = min(b, (V + lead) / kVec);  // vectors with nothing past the row's end
    // (all lanes stay in the loop: what it calls may exchange within the warp)
    const int step = 32 * kUnroll, runs = b > a ? (b - a + step - 1) / step : 0;
    for (int run = 0; run < runs; ++run) {
      const int v = a + lane + (kBack ? runs - 1 - run : run) * step;
      float x[kUnroll][kVec];
      const int v0 = v - lane;
      if (v0 * kVec >= lead && v0 + 32 * kUnroll <= whole) {
        uint4 q[kUnroll];
#pragma unroll
        for (int i = 0; i < kUnroll; ++i) q[i] = vector(v + 32 * i);
#pragma unroll
        for (int i = 0; i < kUnroll; ++i) unpack(q[i], x[i]);
      } else {
#pragma unroll
        for (int i = 0; i < kUnroll; ++i) {
          if (v + 32 * i < b) {
            load(v + 32 * i, x[i]);
          } else {
#pragma unroll
            for (int e = 0; e < kVec; ++e) x[i][e] = -INFINITY;
          }
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

// A segment's weight, from its warp's lanes to rank 0.
template <int NT>
__device__ __forceinline__ void put_segment(Smem<NT>& sm, int rank, const LongSum& own) {
  const Parts p = parts(own);
  const u64 coarse = warp_sum(p.coarse), fine = warp_sum(p.fine);
  if ((threadIdx.x & 31) == 0) {
    const int i = rank * (NT / 32) + (threadIdx.x >> 5);
    st_rank(&sm.seg[i], 0, coarse);
    st_rank(&sm.seg_fine[i], 0, fine);
  }
}

// Sums over the cluster of four values: the CTAs' own sums in x_sum[turn] of
// every CTA, which sum_of adds up.  A buffer's next use lies behind the next
// sum's barrier.  (By value, and the sums left in shared memory: with an array
// by reference the fp32 kernel of 256 threads, which spills, went on with a
// wrong low half of one of them.)
template <int NT>
__device__ __noinline__ void cluster_sum(Smem<NT>& sm, int CL, int rank, int turn, u64 a, u64 b, u64 c, u64 d) {
  constexpr int kWarps = NT / 32;
  const int lane = threadIdx.x & 31, warp = threadIdx.x >> 5;
  a = warp_sum(a);
  b = warp_sum(b);
  c = warp_sum(c);
  d = warp_sum(d);
  if (lane == 0) {
    sm.warp_v[0][warp] = a;
    sm.warp_v[1][warp] = b;
    sm.warp_v[2][warp] = c;
    sm.warp_v[3][warp] = d;
  }
  __syncthreads();
  if (warp < 4) {
    const u64 x = warp_sum(lane < kWarps ? sm.warp_v[warp][lane] : 0);
    if (lane < CL) st_rank(&sm.x_sum[turn][warp][rank], lane, x);
  }
  sync_all(CL);
}
template <int NT>
__device__ __forceinline__ u64 sum_of(const Smem<NT>& sm, int CL, int turn, int k) {
  u64 s = 0;
  for (int r = 0; r < CL; ++r) s += sm.x_sum[turn][k][r];
  return s;
}

// Exclusive scan over the block of (c, q) in thread order.
template <int NT>
__device__ __forceinline__ void block_scan(Smem<NT>& sm, u64 c, u64 q, u64& pc, u64& pq) {
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
  // (lanes 16 .. 31 hold nothing)
  pc = ic - c + __shfl_sync(kFull, ta, 0);
  pq = iq - q + __shfl_sync(kFull, tb, 0);
}

// What a search finds: the key at which the count (or the weight) from the
// highest key down first reaches the target, what lies above it, and at it.
struct Found {
  uint32_t key;
  u64 above_count, above_mass, at_count;
  bool ok;  // false: everything together does not reach the target
};

// Search over keys in [lo, hi], a digit of up to 11 bits per round.
// visit(f) calls f(counts, key, weight units) for the elements of this CTA's part of
// the row; all CTAs of the cluster get the result.
template <int NT, typename Visit>
__device__ __forceinline__ Found search(Smem<NT>& sm, int CL, bool by_count, u64 target, uint32_t lo, uint32_t hi,
                                        Visit&& visit) {
  Found f{0u, 0, 0, 0, true};
  for (;;) {
    const uint32_t span = hi - lo;
    const int bits = 32 - __clz(span);  // (clz(0) = 32)
    const int shift = max(0, bits - 11);
    sync_all(CL);
    for (int i = threadIdx.x; i < kFine; i += NT) {
      sm.count[i] = 0;
      sm.mass[i] = 0;
    }
    sync_all(CL);
    // (all lanes call it.  Where they agree on a bin, as many equal tokens do,
    // one adds for all: a 64-bit sum in shared memory is a loop of exchanges)
    visit([&](bool real, uint32_t key, u64 q) {
      const int bin = real && key >= lo && key <= hi ? static_cast<int>((key - lo) >> shift) : -1;
      const unsigned who = __ballot_sync(kFull, bin >= 0);
      if (!who) return;
      const int first = __shfl_sync(kFull, bin, __ffs(who) - 1);
      if (__all_sync(kFull, bin < 0 || bin == first)) {
        const u64 sum = warp_sum(bin >= 0 ? q : 0);
        if ((threadIdx.x & 31) == __ffs(who) - 1) {
          atomicAdd(&sm.count[bin], static_cast<uint32_t>(__popc(who)));
          if (sum) atomicAdd(&sm.mass[bin], sum);
        }
      } else if (bin >= 0) {
        atomicAdd(&sm.count[bin], 1u);
        if (q) atomicAdd(&sm.mass[bin], q);
      }
    });
    sync_all(CL);
    // thread t: bins B t .. B t + B - 1 from the top
    constexpr int B = kFine / NT;
    u64 c[B], q[B], sc = 0, sq = 0;
#pragma unroll
    for (int e = 0; e < B; ++e) {
      const int bin = kFine - 1 - (B * static_cast<int>(threadIdx.x) + e);
      c[e] = q[e] = 0;
      for (int r = 0; r < CL; ++r) {
        c[e] += ld_rank_u32(&sm.count[bin], r);
        q[e] += ld_rank_u64(&sm.mass[bin], r);
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
    for (int e = 0; e < B; ++e) {
      const u64 before = by_count ? pc : pq, after = by_count ? pc + c[e] : pq + q[e];
      if (before < target && after >= target) {
        sm.found[0] = kFine - 1 - (B * threadIdx.x + e);
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
    hi = lo + min(hi - lo, (1u << shift) - 1u);  // (lo plus a bin may pass 2^32)
  }
}

// Sorts n keys, the highest first (n: a power of two, 32 K to 512 K): a
// bitonic network.  A warp takes strides below 32 K in registers, its lanes
// holding K keys of a run of 32 K; longer ones go through shared memory.
// (132 rows with lists of about 1000 tokens: 53.8 us, with K = 1 throughout 58.7.)
template <int K, int NT>
__device__ __noinline__ void sort_keys(u64* key, int n) {
  const int lane = threadIdx.x & 31, first = (threadIdx.x >> 5) * 32 * K;
  u64 x[K];
  auto in_warp = [&](int size) {
#pragma unroll
    for (int stride = 16 * K; stride > 0; stride >>= 1) {
      if (stride >= size) continue;
      if (stride >= 32) {
#pragma unroll
        for (int e = 0; e < K; ++e) {
          const int f = e ^ (stride / 32);
          if (f > e && f < K) {
            const bool down = ((first + 32 * e) & size) == 0;
            if ((x[e] < x[f]) == down) {
              const u64 t = x[e];
              x[e] = x[f];
              x[f] = t;
            }
          }
        }
      } else {
#pragma unroll
        for (int e = 0; e < K; ++e) {
          const int i = first + 32 * e + lane;
          const u64 y = __shfl_xor_sync(kFull, x[e], stride);
          const bool high = ((i & stride) == 0) == ((i & size) == 0);
          x[e] = (x[e] < y) == high ? y : x[e];
        }
      }
    }
  };
  __syncthreads();
  for (int size = 2; size <= n; size <<= 1) {
    for (int stride = size / 2; stride >= 32 * K; stride >>= 1) {
      __syncthreads();
#pragma unroll
      for (int k = 0; k < K; ++k) {
        const int i = threadIdx.x + k * NT;
        if (i >= n / 2) break;
        const int lo = 2 * i - (i & (stride - 1)), hi = lo + stride;
        const u64 a = key[lo], b = key[hi];
        if ((a < b) == ((lo & size) == 0)) {
          key[lo] = b;
          key[hi] = a;
        }
      }
    }
    if (size == 2 || size > 32 * K) {
      __syncthreads();
      if (first < n)
#pragma unroll
        for (int e = 0; e < K; ++e) x[e] = key[first + 32 * e + lane];
    }
    if (first < n) in_warp(size);
    if (size >= 32 * K && first < n)
#pragma unroll
      for (int e = 0; e < K; ++e) key[first + 32 * e + lane] = x[e];
  }
  __syncthreads();
}

template <typename E, int NT>
__global__ void __launch_bounds__(NT, 1024 / NT) sample_kernel(const __grid_constant__ SampleArgs a, const int CL) {
  extern __shared__ uint4 smem_raw[];
  Smem<NT>& sm = *reinterpret_cast<Smem<NT>*>(smem_raw);
  constexpr int kWarps = NT / 32;
  constexpr int kVec = Row<E, NT>::kVec, kUnroll = Row<E, NT>::kUnroll;
  constexpr uint32_t kKeyMin = 0x00800000u;  // ordered(-inf) + 1: the lowest key a token can have
  const int tid = threadIdx.x, lane = tid & 31, warp = tid >> 5;
  const int r = blockIdx.x / CL, rank = blockIdx.x - r * CL;
  // (no CTA writes to another before that one has begun)
  if (CL > 1) asm volatile("barrier.cluster.arrive.release;" ::: "memory");
  pdl_wait();
  Row<E, NT> row;
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

  // ---- pass 1: the maximum, and counts or weights over bins of x / T.  The
  // bins are laid by a vector a thread from all over the row: the base is their
  // maximum, the lower bins end three times as far below it as they lie on
  // average (a flat row has narrower bins), the upper ones reach far up (the
  // few tokens above a sample's maximum, and a single one far above all).
  const bool by_count = k > 0;
  float base = 0.f, below = kBelow;
  if (cut) {
    for (int i = tid; i < kBins; i += NT) sm.hist[i] = 0;
    float x[kVec], f = -INFINITY, d = 0.f;
    row.load(static_cast<int>(static_cast<long long>(tid) * row.vecs / NT), x);
#pragma unroll
    for (int e = 0; e < kVec; ++e) f = fmaxf(f, x[e]);
#pragma unroll
    for (int o = 16; o > 0; o >>= 1) f = fmaxf(f, __shfl_xor_sync(kFull, f, o));
    if (lane == 0) sm.warp_a[warp] = __float_as_uint(f);
    __syncthreads();
    f = __uint_as_float(static_cast<uint32_t>(sm.warp_a[lane & (kWarps - 1)]));
#pragma unroll
    for (int o = kWarps / 2; o > 0; o >>= 1) f = fmaxf(f, __shfl_xor_sync(kFull, f, o));
    base = isinf(f) ? 0.f : f;
    // (what lies below every window does not count)
    int n = 0;
#pragma unroll
    for (int e = 0; e < kVec; ++e) {
      const float z = (base - x[e]) * inv;
      if (z >= 0.f && z < kBelow) {
        d += z;
        ++n;
      }
    }
#pragma unroll
    for (int o = 16; o > 0; o >>= 1) {
      d += __shfl_xor_sync(kFull, d, o);
      n += __shfl_xor_sync(kFull, n, o);
    }
    if (lane == 0) sm.warp_b[warp] = static_cast<u64>(__float_as_uint(d)) << 32 | static_cast<uint32_t>(n);
    __syncthreads();
    const u64 dn = sm.warp_b[lane & (kWarps - 1)];
    d = __uint_as_float(static_cast<uint32_t>(dn >> 32));
    n = static_cast<int>(static_cast<uint32_t>(dn));
#pragma unroll
    for (int o = kWarps / 2; o > 0; o >>= 1) {
      d += __shfl_xor_sync(kFull, d, o);
      n += __shfl_xor_sync(kFull, n, o);
    }
    // (few tokens say nothing: most are masked)
    if (n >= 32) below = fminf(fmaxf(3.f * d / static_cast<float>(n), 1e-3f), kBelow);
  }
  // bins per unit of x, their width in x / T; in units of the whole window
  // (so that one instruction clamps: bin b holds what rounds to b, and a
  // token's weight is taken against its middle)
  const float scale_hi = inv * ((kBins - kLower) / kAbove), width_hi = kAbove / (kBins - kLower);
  const float s_hi = scale_hi / (kBins - 1), c_hi = width_hi * 1.4426950408889634f;
  float scale_lo, width_lo, s_lo, c_lo;
  auto lay = [&] {
    scale_lo = inv * (kLower / below);
    width_lo = below / kLower;
    s_lo = scale_lo / (kBins - 1);
    c_lo = width_lo * 1.4426950408889634f;
  };
  lay();
  float mx = -INFINITY;
  // the last bits of a sum with 2^23 are an integer (a conversion is four
  // times as dear): the bin's address is those bits, shifted, and a constant
  const uint32_t at = smem_u32(sm.hist) - (0x4b000000u << 2);
  auto count_in = [&](float x, bool count) {
    const float t = x - base;  // (first: base and x may be large against a bin)
    const bool upper = t >= 0.f;
    const float y = __saturatef(fmaf(t, upper ? s_hi : s_lo, static_cast<float>(kLower) / (kBins - 1)));
    const float f = fmaf(y, static_cast<float>(kBins - 1), 8388608.f);
    uint32_t q = 1;
    if (!count) {
      const float r = fmaf(y, static_cast<float>(kBins - 1), 8388608.f - f);
      q = __float_as_uint(fmaf(fast_exp2(r * (upper ? c_hi : c_lo)), 65536.f, 8388608.f)) & 0x3ffffu;
    }
    // (what lies below the window, as masked tokens do, is left out)
    asm volatile("{\n\t.reg .pred p;\n\tsetp.gt.f32 p, %2, 0f00000000;\n\t@p red.shared.add.u32 [%0], %1;\n\t}" ::"r"(
                     at + (__float_as_uint(f) << 2)),
                 "r"(q), "f"(y)
                 : "memory");
  };
  auto one = [&](auto kind) {
    row.batches(rank, [&](float (&x)[kUnroll][kVec], int) {
#pragma unroll
      for (int i = 0; i < kUnroll; ++i)
#pragma unroll
        for (int e = 0; e < kVec; ++e) {
          mx = fmaxf(mx, x[i][e]);
          if (decltype(kind)::value) count_in(x[i][e], decltype(kind)::value == 1);
        }
    });
  };
  if (!cut)
    one(std::integral_constant<int, 0>{});
  else if (by_count)
    one(std::integral_constant<int, 1>{});
  else
    one(std::integral_constant<int, 2>{});
#pragma unroll
  for (int o = 16; o > 0; o >>= 1) mx = fmaxf(mx, __shfl_xor_sync(kFull, mx, o));
  if (lane == 0) sm.warp_a[warp] = __float_as_uint(mx);
  __syncthreads();
  if (CL > 1) asm volatile("barrier.cluster.wait.acquire;" ::: "memory");
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
      for (int i = rank * NT + tid; i < a.V; i += CL * NT)
        a.log_probs[static_cast<size_t>(r) * a.V + i] = -INFINITY;
    sync_all(CL);
    return;
  }
  const Weight wt{m, T, inv};
  Kept kept{kKeyMin, 0x7fffffff, mp};
  u64 set_mass = 0;     // of the tokens that top_p is a share of (0: not known yet)
  bool have_seg = false;  // the segments' weights (and the kept count) come from pass 2
  u64 kept_count = 0;
  int turn = 0;         // of cluster_sum

  // visits this CTA's elements that the prefix kept so far holds
  auto visit_row = [&](auto&& f) {
    row.batches(rank, [&](float (&x)[kUnroll][kVec], int i0) {
#pragma unroll
      for (int i = 0; i < kUnroll; ++i)
#pragma unroll
        for (int e = 0; e < kVec; ++e) {
          const uint32_t key = ordered(x[i][e]);
          const bool in = x[i][e] != -INFINITY && kept.in_prefix(key, Row<E, NT>::index(i0, i, e));
          f(in, key, in ? units(wt.w(x[i][e])) : 0);
        }
    });
  };
  const uint32_t key_max = ordered(m);

  // ---- the bracket of kappa.  Thread t holds B bins from the top.
  struct Bracket {
    float x0, x1;  // tokens x0 <= x < x1 are to be listed
    bool all;      // x1 lies above all tokens
    bool few;      // fewer than top_k tokens have a weight: top_p cuts among them
    bool ok;
  };
  auto edge = [&](int bin) {
    const float y = static_cast<float>(bin - kLower) - 0.5f;  // (its lower edge)
    return base + y / (y > 0.f ? scale_hi : scale_lo);
  };
  auto estimate = [&] {
    constexpr int B = kBins / NT;        // bins of a thread
    const int first = kBins - B - B * tid;  // entry e is bin first + B - 1 - e
    uint32_t h[B] = {};
#pragma unroll
    for (int f = 0; f < B / 4; ++f) {
      uint4 x[kMaxCluster];
#pragma unroll
      for (int q = 0; q < kMaxCluster; ++q)
        x[q] = q < CL ? ld_rank_v4(&sm.hist[first + 4 * f], q) : make_uint4(0, 0, 0, 0);
#pragma unroll
      for (int q = 0; q < kMaxCluster; ++q) {
        h[B - 1 - 4 * f] += x[q].x;
        h[B - 2 - 4 * f] += x[q].y;
        h[B - 3 - 4 * f] += x[q].z;
        h[B - 4 - 4 * f] += x[q].w;
      }
    }
    u64 c[B], w[B], sc = 0, sw = 0;
#pragma unroll
    for (int e = 0; e < B; ++e) {
      // a bin's weight is its sum times that of its middle (kLower's has two halves, and its
      // middle is the base), its count at most the sum times e^(width / 2)
      const int up = first + B - 1 - e - kLower;
      const float mid = static_cast<float>(up) * (up > 0 ? width_hi : width_lo) - (m - base) * inv;
      const float share = static_cast<float>(h[e]) * (1.f / 65536.f);
      c[e] = by_count ? h[e] : static_cast<u64>(share * 1.1f);
      w[e] = by_count || h[e] == 0 ? 0 : units(share * expf(fminf(mid, 1.f)));
      sc += c[e];
      sw += w[e];
    }
    u64 pc, pw;
    block_scan(sm, sc, sw, pc, pw);
    if (tid == NT - 1) {
      sm.found[3] = by_count ? pc + sc : pw + sw;
      sm.found[0] = 0;
      sm.pick_lo = sm.pick_hi = -1;
    }
    __syncthreads();
    // kappa's bin is the first by which the target is reached; a weight is
    // known to 2^-16.8, and the bins that this leaves open are listed too
    // (a miss costs the searches over the row, not the result)
    const u64 all_w = sm.found[3], slack = by_count ? 0 : all_w >> 16;  // (top_k: all tokens of the window)
    const u64 goal = by_count ? static_cast<u64>(k) : max(1ull, part_ceil(fmaxf(p, 0.f), all_w));
#pragma unroll
    for (int e = 0; e < B; ++e) {
      const u64 before = by_count ? pc : pw, after = by_count ? pc + c[e] : pw + w[e];
      if (before < goal + slack && after >= goal + slack) {
        sm.pick_lo = first + B - 1 - e;
        sm.found[0] = pc + c[e];
      }
      if (before + slack < goal && after + slack >= goal) sm.pick_hi = first + B - 1 - e;
      pc += c[e];
      pw += w[e];
    }
    __syncthreads();
    // (the target lies so near the whole weight that only the lowest token is certain to reach it)
    const int lo = sm.pick_lo, hi = sm.pick_hi;
    Bracket b;
    // tokens down to the bottom of the bracket: a list of all of them, where it fits
    b.all = hi >= 0 && lo >= 0 && sm.found[0] <= (by_count ? kList : kAll);
    // (never -inf: what counts as -inf lies below every bracket)
    b.x0 = lo >= 0 ? edge(lo) : -FLT_MAX;
    // (a window of kBelow under the maximum ends where weights do)
    b.few = by_count && lo < 0 && base == m && below == kBelow && p < 1.f && all_w <= kList;
    if (b.few) {
      b.x0 = edge(0);
      b.all = true;
    }
    b.x1 = b.all || hi == kBins - 1 ? INFINITY : edge(hi + 1);
    b.ok = (hi >= 0 || b.few) && (lo >= 0 || b.few || !by_count) && b.x0 < b.x1 && scale_lo < 1e30f && m < INFINITY;
    return b;
  };

  auto key_x = [](u64 key) { return from_ordered(static_cast<uint32_t>(key >> 32)); };

  // ---- pass 2: adds up the tokens x1 <= x and lists those in [x0, x1).
  // Sums: count above (and, above 2^32, of the list), weight above, weight of the
  // list, weight of the row (the last three only where they are used).
  const float c_exp = inv * 1.4426950408889634f;
  auto pass = [&](const Bracket& b) {
    if (tid == 0) sm.list_n = 0;
    __syncthreads();
    const float x0 = b.x0, x1 = b.x1;
    auto list = [&](float x, int idx) {
      const int to = atomicAdd(&sm.list_n, 1);
      if (to < kList) sm.list[to] = static_cast<u64>(ordered(x)) << 32 | ~static_cast<uint32_t>(idx);
    };
    // fp32 weights: 2^((x - m) c) on tokens that are certain to be kept, or to
    // be part of a total (the list's are taken with all their digits).
    LongSum fq, fa;
    uint32_t n = 0;
    if (b.all && by_count) {
      row.template batches<true>(rank, [&](float (&x)[kUnroll][kVec], int i0) {
#pragma unroll
        for (int i = 0; i < kUnroll; ++i)
#pragma unroll
          for (int e = 0; e < kVec; ++e)
            if (x[i][e] >= x0) list(x[i][e], Row<E, NT>::index(i0, i, e));
      });
    } else {
      row.template batches<true>(rank, [&](float (&x)[kUnroll][kVec], int i0) {
        float s = 0.f, sa = 0.f;
#pragma unroll
        for (int i = 0; i < kUnroll; ++i) {
          bool some = false;
#pragma unroll
          for (int e = 0; e < kVec; ++e) {
            const float xe = x[i][e], w = fast_exp2((xe - m) * c_exp);
            sa += w;
            if (xe >= x1) {
              s += w;
              ++n;
            }
            some |= xe >= x0 && xe < x1;
          }
          if (some) {
#pragma unroll
            for (int e = 0; e < kVec; ++e)
              if (x[i][e] >= x0 && x[i][e] < x1) list(x[i][e], Row<E, NT>::index(i0, i, e));
          }
        }
        fq.add(s);
        fa.add(sa);
      });
    }
    const u64 q = fq.total();
    put_segment(sm, rank, fq);
    __syncthreads();
    u64 ql = 0;
    const int own = sm.list_n;
    if (!by_count)
      for (int i = tid; i < min(own, kList); i += NT) ql += units(wt.w(key_x(sm.list[i])));
    turn ^= 1;
    cluster_sum(sm, CL, rank, turn, n + (tid == 0 ? static_cast<u64>(own) << 32 : 0), q, ql, fa.total());
  };

  // The bracket of a limit, exact sums around it, and the search of the list.
  // False: not settled (nothing changed).
  auto by_list = [&](bool& both) {
    const Bracket b = estimate();
    if (!b.ok) return false;
    pass(b);
    const u64 counts = sum_of(sm, CL, turn, 0), above_n = counts & 0xffffffffull;
    const u64 above_q = sum_of(sm, CL, turn, 1);
    const int total = static_cast<int>(counts >> 32);
    if (!by_count) set_mass = sum_of(sm, CL, turn, 3);
    {
      // kappa is in the list: less than the target lies above it, and no less with it
      const u64 target = by_count ? static_cast<u64>(b.few ? min(k, total) : k)
                                  : max(1ull, part_ceil(fmaxf(p, 0.f), set_mass));
      const u64 above = by_count ? above_n : above_q, upto = above + (by_count ? total : sum_of(sm, CL, turn, 2));
      if (total > kList || above >= target || upto < target) return false;
    }
    both = by_count && p < 1.f && b.all;
    // min_p cuts below all that lies above the list: the list settles it
    // (not where top_p is still to look at the whole set)
    const bool min_p_too = mp > 0.f && (b.all || wt.w(b.x1) >= mp) && (!by_count || p >= 1.f || both);
    // all lists go to rank 0, in the order of the CTAs
    if (CL > 1) {
      int at = 0;
      for (int c = 0; c < rank; ++c) at += static_cast<int>(sm.x_sum[turn][0][c] >> 32);
      if (rank > 0)
        for (int i = tid; i < sm.list_n; i += NT) st_rank(&sm.list[at + i], 0, sm.list[i]);
      sync_all(CL);
    }
    if (rank == 0) {
      // the list in order, a run of it to each thread
      int n2 = 32;
      while (n2 < total) n2 <<= 1;
      for (int i = total + tid; i < n2; i += NT) sm.list[i] = 0;
      // (a warp's run as long as keeps all warps at work)
      if (n2 <= NT)
        sort_keys<1, NT>(sm.list, n2);
      else if (n2 == 2 * NT)
        sort_keys<2, NT>(sm.list, n2);
      else if (n2 == 4 * NT)
        sort_keys<4, NT>(sm.list, n2);
      else if (n2 == 8 * NT)
        sort_keys<8, NT>(sm.list, n2);
      else
        sort_keys<kList / NT, NT>(sm.list, n2);
      const int each = max(1, n2 / NT), i0 = tid * each, i1 = min(total, i0 + each);
      const int limit = by_count ? min(static_cast<int>(static_cast<u64>(k) - above_n), total) : total;
      u64 own = 0, in_limit = 0, before, rest;
      for (int i = i0; i < i1; ++i) {
        const u64 q = units(wt.w(key_x(sm.list[i])));
        own += q;
        in_limit += i < limit ? q : 0;
      }
      block_scan(sm, own, in_limit, before, rest);
      if (tid == NT - 1) {
        sm.found[4] = rest + in_limit;
        sm.pick_lo = -1;
      }
      __syncthreads();
      const u64 set = by_count ? above_q + sm.found[4] : set_mass;
      u64 goal = ~0ull;
      if (!by_count || both) {
        goal = max(1ull, part_ceil(fmaxf(p, 0.f), set));
        goal = goal > above_q ? goal - above_q : 1;
      }
      // the last kept token: the last within the limit that begins before the
      // goal (and, where that settles it, is not below min_p)
      int mine = -1;
      for (int i = i0; i < min(i1, limit) && before < goal; ++i) {
        const float w = wt.w(key_x(sm.list[i]));
        if (min_p_too && w < mp) break;
        const u64 q = units(w);
        before += q;
        mine = i;
        const int v2 = (static_cast<int>(~static_cast<uint32_t>(sm.list[i])) + row.lead) / kVec, c = v2 / row.per;
        const int seg = c * kWarps + (v2 - c * row.per) / row.per_warp;
        if (w >= 0x1p-15f) {
          atomicAdd(&sm.seg[seg], q);  // (a whole number of units)
        } else {
          const Parts f = parts(w);
          atomicAdd(&sm.seg[seg], f.coarse);
          atomicAdd(&sm.seg_fine[seg], f.fine);
        }
      }
      if (mine >= 0) atomicMax(&sm.pick_lo, mine);
      __syncthreads();
      if (tid < CL) {
        // (none: min_p cuts between the list and what lies above it)
        const int last = sm.pick_lo;
        st_rank(&sm.x_out[0], tid, last >= 0 ? sm.list[last] : static_cast<u64>(ordered(b.x1)) << 32 | 0x80000000u);
        st_rank(&sm.x_out[1], tid, set);
        st_rank(&sm.x_out[2], tid, above_n + static_cast<u64>(last + 1));
      }
    }
    sync_all(CL);
    kept.kappa = static_cast<uint32_t>(sm.x_out[0] >> 32);
    kept.last = static_cast<int>(~static_cast<uint32_t>(sm.x_out[0]));
    set_mass = sm.x_out[1];
    kept_count = sm.x_out[2];
    have_seg = mp <= 0.f || min_p_too;
    return true;
  };

  // the same by radix searches over the row
  auto by_row = [&](bool count) {
    have_seg = false;
    u64 target = static_cast<u64>(k);
    if (!count) {
      if (set_mass == 0) {
        u64 all = 0;
        visit_row([&](bool, uint32_t, u64 w) { all += w; });
        turn ^= 1;
        cluster_sum(sm, CL, rank, turn, all, 0, 0, 0);
        set_mass = sum_of(sm, CL, turn, 0);
      }
      target = max(1ull, part_ceil(fmaxf(p, 0.f), set_mass));
    }
    const Found f = search(sm, CL, count, target, kKeyMin, key_max, visit_row);
    if (!f.ok) return;
    const u64 one = max(units(wt.w(from_ordered(f.key))), 1ull);
    const u64 quota = count ? target - f.above_count : (target - f.above_mass + one - 1) / one;
    set_mass = f.above_mass + min(quota, f.at_count) * units(wt.w(from_ordered(f.key)));
    kept.move_to(f.key);
    if (quota < f.at_count) {
      auto visit_ties = [&](auto&& g) {
        row.batches(rank, [&](float (&x)[kUnroll][kVec], int i0) {
#pragma unroll
          for (int i = 0; i < kUnroll; ++i)
#pragma unroll
            for (int e = 0; e < kVec; ++e) {
              const int idx = Row<E, NT>::index(i0, i, e);
              g(x[i][e] != -INFINITY && ordered(x[i][e]) == f.key && idx <= kept.last,
                0xffffffffu - static_cast<uint32_t>(idx), 0ull);
            }
        });
      };
      const Found t =
          search(sm, CL, true, quota, 0xffffffffu - static_cast<uint32_t>(a.V), 0xffffffffu, visit_ties);
      kept.last = static_cast<int>(0xffffffffu - t.key);
    }
  };

  // the histogram once more, around the maximum itself
  auto again = [&] {
    base = m;
    below = kBelow;
    lay();
    sync_all(CL);  // the first one is read by all
    for (int i = tid; i < kBins; i += NT) sm.hist[i] = 0;
    __syncthreads();
    row.batches(rank, [&](float (&x)[kUnroll][kVec], int) {
#pragma unroll
      for (int i = 0; i < kUnroll; ++i)
#pragma unroll
        for (int e = 0; e < kVec; ++e) count_in(x[i][e], by_count);
    });
    sync_all(CL);
  };

  if (cut) {
    bool both = false;
    for (int round = 0; !by_list(both); ++round) {
      // (nearly all masked, and no open token in the sample)
      if (round == 0 && m < INFINITY) {
        again();
        continue;
      }
      both = false;
      set_mass = 0;
      by_row(by_count);
      break;
    }
    if (by_count && p < 1.f && !both) by_row(false);
  }

  // ---- the segments' weights, where pass 2 has not left them or min_p cuts
  if (!have_seg) {
    u64 n = 0;
    LongSum sum;
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
                          kept.in_prefix(ordered(x[i][e]), Row<E, NT>::index(i0, i, e));
          s.add(in ? w : 0.f);
          cnt += in ? 1 : 0;
        }
      n += cnt;
      sum.add(s.hi);
      sum.add(s.lo);
    });
    put_segment(sm, rank, sum);
    turn ^= 1;
    cluster_sum(sm, CL, rank, turn, n, 0, 0, 0);
    kept_count = sum_of(sm, CL, turn, 0);
  }

  // ---- rank 0 places the random number
  if (rank == 0) {
    if (warp == 0) {
      // lane i: segments 4 i .. 4 i + 3
      u128 four[4], own4 = 0;
#pragma unroll
      for (int e = 0; e < 4; ++e) {
        four[e] = 4 * lane + e < CL * kWarps ? join(sm.seg[4 * lane + e], sm.seg_fine[4 * lane + e]) : 0;
        own4 += four[e];
      }
      u128 inc = own4;
#pragma unroll
      for (int o = 1; o < 32; o <<= 1) {
        const u64 yl = __shfl_up_sync(kFull, static_cast<u64>(inc), o);
        const u64 yh = __shfl_up_sync(kFull, static_cast<u64>(inc >> 64), o);
        if (lane >= o) inc += static_cast<u128>(yh) << 64 | yl;
      }
      const u128 all = static_cast<u128>(__shfl_sync(kFull, static_cast<u64>(inc >> 64), 31)) << 64 |
                       __shfl_sync(kFull, static_cast<u64>(inc), 31);
      const float logz = log_units(static_cast<u64>(all >> kFineBits));
      if (lane < CL) st_rank(&sm.x_out[3], lane, static_cast<u64>(__float_as_uint(logz)));
      const u128 thr = part_floor(u, all);
      if (lane == __ffs(__ballot_sync(kFull, inc > thr)) - 1) {  // (thr < all)
        u128 rem = thr - (inc - own4), sum = four[0];
        int s = 0;
#pragma unroll
        for (int e = 0; e < 3; ++e)
          if (s == e && rem >= four[e]) {
            rem -= four[e];
            sum = four[e + 1];
            ++s;
          }
        // within the segment: units in which its sum has 62 bits
        const u64 top = static_cast<u64>(sum >> 62);
        const int drop = top ? 64 - __clzll(static_cast<long long>(top)) : 0;
        sm.found[0] = thr == 0 ? ~0ull : static_cast<u64>(4 * lane + s);
        sm.found[1] = static_cast<u64>(rem >> drop);
        sm.found[2] = static_cast<u64>(drop);
        sm.token = sm.pick_lo = -1;
        sm.pick_hi = 0x7fffffff;
        if (a.kept) a.kept[r] = static_cast<int>(kept_count);
      }
    }
    __syncthreads();
    const bool nought = sm.found[0] == ~0ull;  // below the smallest unit
    const int s = nought ? 0 : static_cast<int>(sm.found[0]);
    u64 left = sm.found[1];  // of the number, in the segment
    const float unit = exp2f(static_cast<float>(kUnitBits + kFineBits - static_cast<int>(sm.found[2])));
    const float logz = __uint_as_float(static_cast<uint32_t>(sm.x_out[3]));
    // a token's weight among the kept
    auto kept_weight = [&](float x, int idx) {
      const float w = wt.w(x);
      return x != -INFINITY && w >= mp && kept.in_prefix(ordered(x), idx) ? w : 0.f;
    };
    const int sr = s / kWarps, sw = s - sr * kWarps;
    const int va = row.seg_begin(sr, sw), vb = min(row.seg_begin(sr, sw + 1), min(row.vecs, sr * row.per + row.per));
    for (int v0 = va; !nought && v0 < vb; v0 += NT) {
      const int v = v0 + tid;
      float x[kVec];
      u64 own = 0;
      int last = -1;
      if (v < vb) {
        row.load(v, x);
#pragma unroll
        for (int e = 0; e < kVec; ++e) {
          const int idx = v * kVec - row.lead + e;
          x[e] = kept_weight(x[e], idx);
          if (x[e] > 0.f) last = idx;
          own += __float2ull_rn(x[e] * unit);
        }
      }
      if (last >= 0) atomicMax(&sm.pick_lo, last);  // the last kept token of the segment
      u64 before, none;
      block_scan(sm, own, 0, before, none);
      if (left >= before && left - before < own) {
#pragma unroll
        for (int e = 0; e < kVec; ++e) {
          const u64 q = __float2ull_rn(x[e] * unit);
          if (left >= before && left - before < q) sm.token = v * kVec - row.lead + e;
          before += q;
        }
      }
      __syncthreads();
      if (sm.token >= 0) break;
      // what is left of the number, from the warps' totals of the scan
      left -= warp_sum(lane < kWarps ? sm.warp_a[lane] : 0);
    }
    // rounding of the segment's sum may leave the number just past its last token
    int tok = sm.token >= 0 ? sm.token : sm.pick_lo;
    if (tok < 0) {
      // Zero (or what is below the smallest unit) falls on the first kept token
      // that has a weight at all; the row's maximum has one.
      for (int v0 = 0; v0 < row.vecs; v0 += NT) {
        const int v = v0 + tid;
        int first = -1;
        if (v < row.vecs) {
          float x[kVec];
          row.load(v, x);
#pragma unroll
          for (int e = kVec - 1; e >= 0; --e) {
            const int idx = v * kVec - row.lead + e;
            if (kept_weight(x[e], idx) > 0.f) first = idx;
          }
        }
        if (first >= 0) atomicMin(&sm.pick_hi, first);
        if (__syncthreads_or(first >= 0)) break;
      }
      tok = sm.pick_hi;
    }
    if (tid == 0) {
      a.token[r] = tok;
      if (a.log_prob) a.log_prob[r] = wt.z(static_cast<float>(row.base[row.lead + tok])) - logz;
    }
  }
  if (a.log_probs) {
    sync_all(CL);
    const float logz = __uint_as_float(static_cast<uint32_t>(sm.x_out[3]));
    float* out = a.log_probs + static_cast<size_t>(r) * a.V;
    // (element by element: rows of the result need not begin at a vector)
    const E* from = row.base + row.lead;
    for (int i0 = rank * NT + tid; i0 < a.V; i0 += kBatch * CL * NT) {
      float x[kBatch];
#pragma unroll
      for (int j = 0; j < kBatch; ++j) {
        const int idx = i0 + j * CL * NT;
        x[j] = idx < a.V ? fmaxf(static_cast<float>(from[idx]), -INFINITY) : -INFINITY;
      }
#pragma unroll
      for (int j = 0; j < kBatch; ++j) {
        const int idx = i0 + j * CL * NT;
        const float z = wt.z(x[j]);
        const bool in = x[j] != -INFINITY && kept.in_prefix(ordered(x[j]), idx) && (mp <= 0.f || expf(z) >= mp);
        if (idx < a.V) out[idx] = in ? z - logz : -INFINITY;
      }
    }
  }
  pdl_launch_next();
  sync_all(CL);  // no CTA leaves while another may write to its shared memory
}

template <typename E, int NT>
cudaError_t launch_nt(const SampleArgs& a, int CL, cudaStream_t stream) {
  {
    static std::mutex mu;
    static bool done[64] = {};
    int dev = 0;
    cudaError_t e = cudaGetDevice(&dev);
    if (e != cudaSuccess) return e;
    if (dev < 0 || dev >= 64) return cudaErrorInvalidDevice;
    std::lock_guard<std::mutex> lk(mu);
    if (!done[dev]) {
      e = cudaFuncSetAttribute(sample_kernel<E, NT>, cudaFuncAttributeMaxDynamicSharedMemorySize,
                               static_cast<int>(sizeof(Smem<NT>)));
      if (e != cudaSuccess) return e;
      done[dev] = true;
    }
  }
  return launch_overlapped(sample_kernel<E, NT>, dim3(static_cast<unsigned>(a.R) * CL), dim3(NT), sizeof(Smem<NT>),
                           stream, static_cast<unsigned>(CL), a, CL);
}

template <typename E>
cudaError_t launch_e(const SampleArgs& a, int num_sms, cudaStream_t stream) {
  // Short rows that are more than two CTAs a SM: their time is the chain of
  // steps of a row, of which four CTAs of 256 threads overlap more (1783 rows
  // of 1066: 81 us, with 512 threads 132; 2000 of 32003: 204, 230; but 610 of
  // 65536: 118, 113; 1024 of 151936: 356, 330, as fewer rows stay in L2).
  // Four CTAs a SM leave a thread 64 registers, with spills of about 490 bytes
  // stored and 800 loaded (512 threads: 28); three, with a fifth of the spills,
  // take 5% longer.
  if (a.R > 2ll * num_sms && a.V <= kSmallV) return launch_nt<E, 256>(a, 1, stream);
  // Two CTAs fit a SM: as many CTAs a row as fit at once, none for less than
  // 4096 tokens.  (More CTAs for many rows would keep the rows in work within
  // L2 between the passes, but cost more in exchanges than that gains: 1024
  // rows of 151936 take 321 us with one, 380 with two, 537 with four; 400 rows
  // 165, 169 and 224.)
  int CL = kMaxCluster;
  while (CL > 1 && (a.R * static_cast<long long>(CL) > 2ll * num_sms || a.V < 4096 * CL)) CL >>= 1;
  return launch_nt<E, 512>(a, CL, stream);
}

}  // namespace

cudaError_t launch_sample(int elem_bytes, const SampleArgs& a, int num_sms, cudaStream_t stream) {
  return elem_bytes == 4 ? launch_e<float>(a, num_sms, stream) : launch_e<__nv_bfloat16>(a, num_sms, stream);
}

}  // namespace simsd
