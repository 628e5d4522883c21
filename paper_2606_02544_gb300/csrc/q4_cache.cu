// q4_cache.cu -- the way of a chunk of tokens into a paged cache in 4 bits,
// and the rows of such a cache written out again (Sec. 3.3: the prefix is
// read from a KV cache; keys are cached rotated).
//
// Mathematics.  The rotation is that of rope_append.cu.  A group of 16
// components becomes s = (max |x| / 6) to nearest in 8 bits and codes (x / s)
// to nearest in 4 bits; the rotated key is taken as it is in fp32, without a
// rounding to the type before.  x / s is x fl(1 / s) with one step of
// correction by its residual (Markstein 1990), which makes it correctly
// rounded, so that ties of 16-bit values go to the even code; max |x| / 6 is
// formed the same way.
// Written out, s times a code has 6 significant bits: exact in fp16 and bf16.
//
// A thread owns eight components: a row of 128 is half a warp's (of 64, a
// quarter), a group two lanes', so that a rotation's partner comes by shuffle
// and a group's largest by one.  A token's angles are formed once a warp,
// one or two a lane, and serve every head that the warp visits (through
// shared memory; four angles formed by each lane for itself, with four
// components a lane and quotients by division, took 200 us for 16384 tokens).
//
// Bound by memory: a token reads (Hq + 2 Hkv) d elements and writes Hq d and
// 2 Hkv (d / 2 + d / 16) bytes.  16404 tokens of 32 heads on 8 of 128 in bf16
// (355 MB) take 78 us, 4.5 TB/s, and the cache written out again as keys and
// values (86 MB) 12 us (7 TB/s, its reads from L2); a single token a sequence takes as long as the
// host's two calls, 15 us.
#include <cuda_bf16.h>
#include <cuda_fp16.h>
#include <cuda_runtime.h>

#include <algorithm>

#include "chunk_walk.cuh"
#include "common.cuh"
#include "kernels.h"
#include "q4.cuh"
#include "rope_token.cuh"

namespace simsd {
namespace {

constexpr int kThreads = 256;
constexpr int kMaxTokens = 64;  // tokens of a block

// Eight components as they lie in memory.
template <typename E>
struct Raw8 {
  uint4 v[sizeof(E) / 2];
};
template <typename E>
__device__ __forceinline__ Raw8<E> load8(const E* p) {
  Raw8<E> r;
#pragma unroll
  for (int i = 0; i < static_cast<int>(sizeof(E) / 2); ++i) r.v[i] = reinterpret_cast<const uint4*>(p)[i];
  return r;
}
__device__ __forceinline__ void unpack8(const Raw8<float>& r, float (&x)[8]) {
#pragma unroll
  for (int i = 0; i < 2; ++i) {
    x[4 * i] = __uint_as_float(r.v[i].x);
    x[4 * i + 1] = __uint_as_float(r.v[i].y);
    x[4 * i + 2] = __uint_as_float(r.v[i].z);
    x[4 * i + 3] = __uint_as_float(r.v[i].w);
  }
}
__device__ __forceinline__ void unpack8(const Raw8<__nv_bfloat16>& r, float (&x)[8]) {
  const uint32_t w[4] = {r.v[0].x, r.v[0].y, r.v[0].z, r.v[0].w};
#pragma unroll
  for (int e = 0; e < 4; ++e) {
    x[2 * e] = __uint_as_float(w[e] << 16);
    x[2 * e + 1] = __uint_as_float(w[e] & 0xffff0000u);
  }
}
__device__ __forceinline__ void store8(float* p, const float (&x)[8]) {
  reinterpret_cast<float4*>(p)[0] = make_float4(x[0], x[1], x[2], x[3]);
  reinterpret_cast<float4*>(p)[1] = make_float4(x[4], x[5], x[6], x[7]);
}
__device__ __forceinline__ void store8(__nv_bfloat16* p, const float (&x)[8]) {
  uint32_t w[4];
#pragma unroll
  for (int e = 0; e < 4; ++e) {
    const __nv_bfloat162 b = __floats2bfloat162_rn(x[2 * e], x[2 * e + 1]);
    w[e] = *reinterpret_cast<const uint32_t*>(&b);
  }
  *reinterpret_cast<uint4*>(p) = make_uint4(w[0], w[1], w[2], w[3]);
}

// The ways in which pairs can lie: rotate-half with halves of whole vectors of
// eight, interleaved with a rotated part of whole vectors, anything else.
enum { kHalves = 0, kPairs = 1, kOther = 2 };

// A lane's share of a rotation: components comp .. comp + 7 of a row.
template <int kWay>
struct Turner {
  float cs[8], sn[8];  // x turned: x cs + partner sn (the partner's sign in sn)
  int comp, lane, base, r, half, partner;
  bool by_half;

  __device__ __forceinline__ void set(const float2* angles) {
#pragma unroll
    for (int e = 0; e < 8; ++e) {
      const int k = comp + e;
      cs[e] = 1.f;
      sn[e] = 0.f;
      if (k < r) {
        const float2 x = angles[by_half ? (k < half ? k : k - half) : k >> 1];
        cs[e] = x.x;
        sn[e] = (by_half ? k < half : (k & 1) == 0) ? -x.y : x.y;
      }
    }
  }
  __device__ __forceinline__ void turn(float (&x)[8]) const {
    const unsigned full = 0xffffffffu;
    float o[8];
    if constexpr (kWay == kPairs) {
#pragma unroll
      for (int e = 0; e < 8; ++e) o[e] = x[e ^ 1];
    } else if constexpr (kWay == kHalves) {
#pragma unroll
      for (int e = 0; e < 8; ++e) o[e] = __shfl_sync(full, x[e], partner);
    } else if (!by_half) {
#pragma unroll
      for (int e = 0; e < 8; ++e) o[e] = x[e ^ 1];
    } else {
      // the partner's place within its vector differs from the component's
#pragma unroll
      for (int e = 0; e < 8; ++e) {
        const int p = comp + e < half ? comp + e + half : comp + e < r ? comp + e - half : comp + e;
        o[e] = 0.f;
#pragma unroll
        for (int j = 0; j < 8; ++j) {
          const float t = __shfl_sync(full, x[j], base + (p >> 3));
          if (j == (p & 7)) o[e] = t;
        }
      }
    }
    if (kWay == kOther || comp < r) {
#pragma unroll
      for (int e = 0; e < 8; ++e)
        if (kWay != kOther || comp + e < r) x[e] = x[e] * cs[e] + o[e] * sn[e];
    }
  }
};

// Warp item (token, group of heads): of the token's q rows, then of its keys
// and values, every groups-th step of kRows rows.
template <typename E, int D, int kWay>
__global__ void __launch_bounds__(kThreads, 3) rope_q4_kernel(const __grid_constant__ RopeArgs a,
                                                              const __grid_constant__ simsd_q4_cache c) {
  constexpr int kLanes = D / 8, kRows = 32 / kLanes;  // lanes of a row, rows of a warp
  constexpr int kInFlight = 8 / sizeof(E);            // steps of q whose loads are issued together
  __shared__ Token toks[kMaxTokens];
  __shared__ float2 angles[kThreads / 32][D / 2];  // a warp's token: (cos, sin) of each pair
  pdl_wait();
  pdl_launch_next();
  const unsigned full = 0xffffffffu;
  const int warp = threadIdx.x >> 5, lane = threadIdx.x & 31;
  const int tok0 = blockIdx.x * a.tokens_block;
  if (blockIdx.x == 0) {
    bool bad = false;
    for (int b = threadIdx.x; b < a.Bt; b += kThreads) bad |= chunk_of(a.token_start, b, a.T).bad;
    if (bad) raise_error(a.err_word, SIMSD_EW_TOKENS);
  }
  for (int i = warp; i < a.tokens_block && tok0 + i < a.T; i += kThreads / 32) {
    const Token t = resolve(a, tok0 + i, true);
    if (lane == 0) toks[i] = t;
  }
  __syncthreads();
  const int at = lane & (kLanes - 1), sub = lane / kLanes;
  Turner<kWay> tr;
  tr.r = a.plan.rot_dim;
  tr.half = tr.r / 2;
  tr.by_half = kWay == kHalves || (kWay == kOther && a.plan.layout == SIMSD_ROPE_HALF);
  tr.lane = lane;
  tr.base = lane - at;
  tr.comp = 8 * at;
  tr.partner = tr.comp < tr.half ? lane + tr.half / 8 : tr.comp < tr.r ? lane - tr.half / 8 : lane;
  for (int w = warp; w < a.tokens_block * a.groups; w += kThreads / 32) {
    const int i = w / a.groups, grp = w - i * a.groups, tok = tok0 + i;
    if (tok >= a.T) break;
    const Token tk = toks[i];
    if (tk.state == 0) continue;
    const E* q = static_cast<const E*>(a.q) + static_cast<long long>(tok) * a.q_stride + tr.comp;
    E* q_out = static_cast<E*>(a.q_out) + static_cast<long long>(tok) * a.q_out_stride + tr.comp;
    if (tk.state == 2) {
      const float zero[8] = {};
      for (int h = grp * kRows + sub; h < a.Hq; h += a.groups * kRows) store8(q_out + h * D, zero);
      continue;
    }
    __syncwarp();
    for (int pair = lane; pair < tr.half; pair += 32) {
      const unsigned long long turn = static_cast<unsigned long long>(static_cast<long long>(tk.pos)) * a.plan.turn[pair];
      float2 cs;
      sincospif(static_cast<float>(static_cast<int32_t>(turn >> 32)) * 0x1p-31f, &cs.y, &cs.x);
      angles[warp][pair] = make_float2(cs.x * a.plan.magnitude, cs.y * a.plan.magnitude);
    }
    __syncwarp();
    tr.set(angles[warp]);
    // the first keys and values are on their way while q is turned
    const E* k = static_cast<const E*>(a.k) + static_cast<long long>(tok) * a.k_stride + tr.comp;
    const E* v = static_cast<const E*>(a.v) + static_cast<long long>(tok) * a.v_stride + tr.comp;
    Raw8<E> rk{}, rv{};
    auto fetch = [&](int h) {
      if (h < a.Hkv) {
        rk = load8(k + h * D);
        rv = load8(v + h * D);
      }
    };
    if (tk.row >= 0) fetch(grp * kRows + sub);
    for (int h0 = grp * kRows; h0 < a.Hq; h0 += a.groups * kRows * kInFlight) {
      Raw8<E> raw[kInFlight];
#pragma unroll
      for (int j = 0; j < kInFlight; ++j) {
        const int h = h0 + j * a.groups * kRows + sub;
        if (h < a.Hq) raw[j] = load8(q + h * D);
      }
#pragma unroll
      for (int j = 0; j < kInFlight; ++j) {
        const int h = h0 + j * a.groups * kRows + sub;
        if (h - sub >= a.Hq) break;  // (the warp's lanes agree)
        float x[8];
        unpack8(raw[j], x);
        tr.turn(x);
        if (h < a.Hq) store8(q_out + h * D, x);
      }
    }
    if (tk.row < 0) continue;
    auto put = [&](float (&x)[8], int h, float unit, void* codes, void* scales) {
      if (unit != 1.f) {
        // (correctly rounded as the quotients below; what passes fp32 stays an infinity)
        const float inv = 1.f / unit;
#pragma unroll
        for (int e = 0; e < 8; ++e) {
          const float y = x[e] * inv, z = fmaf(fmaf(-y, unit, x[e]), inv, y);
          x[e] = fabsf(y) < INFINITY ? z : y;
        }
      }
      uint32_t top = 0;  // as bits: a NaN is above every number
#pragma unroll
      for (int e = 0; e < 8; ++e) top = max(top, __float_as_uint(x[e]) & 0x7fffffffu);
      top = max(top, __shfl_xor_sync(full, top, 1));
      const uint32_t sc = q4_scale(__uint_as_float(top));
      const float s = q4_scale_value(sc), s_inv = __frcp_rn(s);
      if (top >= 0x7f800000u) {
        // infinities have no residual: the largest numbers go to 6 as well
#pragma unroll
        for (int e = 0; e < 8; ++e) x[e] = fminf(fmaxf(x[e], -3.4e38f), 3.4e38f);
      }
      uint32_t code = 0;
#pragma unroll
      for (int e = 0; e < 8; ++e) {
        const float y = x[e] * s_inv;
        x[e] = fmaf(fmaf(-y, s, x[e]), s_inv, y);
      }
#pragma unroll
      for (int e = 0; e < 4; ++e) code |= q4_codes(x[2 * e], x[2 * e + 1]) << (8 * e);
      if (h >= a.Hkv) return;
      const long long row = tk.row + static_cast<long long>(h) * a.page_size;
      static_cast<uint32_t*>(codes)[row * (D / 8) + at] = code;
      if ((at & 1) == 0) static_cast<uint8_t*>(scales)[row * (D / kQ4Group) + (at >> 1)] = static_cast<uint8_t>(sc);
    };
    for (int h0 = grp * kRows; h0 < a.Hkv; h0 += a.groups * kRows) {
      const int h = h0 + sub;
      float x[8], y[8];
      unpack8(rk, x);
      unpack8(rv, y);
      fetch(h + a.groups * kRows);  // the next ones
      tr.turn(x);
      put(x, h, c.k_unit, c.k_codes, c.k_scales);
      put(y, h, c.v_unit, c.v_codes, c.v_scales);
    }
  }
}

template <typename E, int D>
cudaError_t launch_d(RopeArgs a, const simsd_q4_cache& c, int num_sms, cudaStream_t stream) {
  constexpr int kRows = 32 / (D / 8), kWarps = kThreads / 32;
  const int steps = (std::max(a.Hq, a.Hkv) + kRows - 1) / kRows;
  // two full waves of warps where there are that many steps, more steps to a
  // warp (fewer angles formed) beyond, half a token's at most (so that the
  // items of a block divide among its warps)
  const long long want = 2ll * 64 * num_sms;
  a.groups = static_cast<int>(std::min<long long>(steps, std::max<long long>(2, want / std::max(1, a.T))));
  // items for every warp of a block, and of many tokens so many that the
  // blocks (three an SM) make one wave (finding a token's sequence and page is
  // a chain of loads)
  a.tokens_block = std::max((kWarps + a.groups - 1) / a.groups, (a.T + 3 * num_sms - 1) / (3 * num_sms));
  a.tokens_block = std::min(kMaxTokens, a.tokens_block);
  const unsigned blocks = static_cast<unsigned>((a.T + a.tokens_block - 1) / a.tokens_block);
  const int r = a.plan.rot_dim;
  auto* kern = a.plan.layout == SIMSD_ROPE_HALF && r % 16 == 0  ? rope_q4_kernel<E, D, kHalves>
               : a.plan.layout != SIMSD_ROPE_HALF && r % 8 == 0 ? rope_q4_kernel<E, D, kPairs>
                                                                : rope_q4_kernel<E, D, kOther>;
  return launch_overlapped(kern, dim3(blocks), dim3(kThreads), 0, stream, 1u, a, c);
}

// ------------------------------------------------------------------ expand
struct ExpandTo {
  simsd_q4_cache c;
  const int32_t* block_table;
  void *k, *v;
  int num_pages, max_pages, page_size, Bt, Hkv;
  int32_t* err_word;  // null: nothing is raised
  int wide;           // k and v are 32-byte aligned
  int round;          // pages whose (page, head) are counted in 2^30 (nearly always all)
};

__device__ __forceinline__ void st_global_256(void* p, const uint32_t (&v)[8]) {
  asm volatile("st.global.v8.b32 [%0], {%1,%2,%3,%4,%5,%6,%7,%8};" ::"l"(p), "r"(v[0]), "r"(v[1]), "r"(v[2]), "r"(v[3]),
               "r"(v[4]), "r"(v[5]), "r"(v[6]), "r"(v[7])
               : "memory");
}
// 32 bytes; in one store where they are a whole sector (two of 16, with other
// lanes' between them, cost L2 a partial sector each).
__device__ __forceinline__ void put32(void* to, const uint32_t (&o)[8], bool wide) {
  if (wide) {
    st_global_256(to, o);
  } else {
    static_cast<uint4*>(to)[0] = make_uint4(o[0], o[1], o[2], o[3]);
    static_cast<uint4*>(to)[1] = make_uint4(o[4], o[5], o[6], o[7]);
  }
}
__device__ __forceinline__ void put16(float* to, const uint32_t (&h)[8], float unit, bool wide) {
#pragma unroll
  for (int i = 0; i < 2; ++i) {
    uint32_t o[8];
#pragma unroll
    for (int k = 0; k < 4; ++k) {
      const float2 a = __half22float2(*reinterpret_cast<const __half2*>(&h[4 * i + k]));
      o[2 * k] = __float_as_uint(a.x * unit);
      o[2 * k + 1] = __float_as_uint(a.y * unit);
    }
    put32(to + 8 * i, o, wide);
  }
}
__device__ __forceinline__ void put16(__nv_bfloat16* to, const uint32_t (&h)[8], float unit, bool wide) {
  uint32_t o[8];
#pragma unroll
  for (int i = 0; i < 8; ++i) {
    const float2 a = __half22float2(*reinterpret_cast<const __half2*>(&h[i]));
    const __nv_bfloat162 b = __floats2bfloat162_rn(a.x * unit, a.y * unit);
    o[i] = *reinterpret_cast<const uint32_t*>(&b);
  }
  put32(to, o, wide);
}

// One group: 8 bytes of codes and a scale to 16 values.
__device__ __forceinline__ void group_values(uint2 w, uint32_t scale, uint32_t (&h)[8]) {
  const uint32_t s = q4_scale_pair(scale | scale << 8);
  h[0] = mul_f16x2(q4_pair<0>(w.x), s);
  h[1] = mul_f16x2(q4_pair<1>(w.x), s);
  h[2] = mul_f16x2(q4_pair<2>(w.x), s);
  h[3] = mul_f16x2(q4_pair<3>(w.x), s);
  h[4] = mul_f16x2(q4_pair<0>(w.y), s);
  h[5] = mul_f16x2(q4_pair<1>(w.y), s);
  h[6] = mul_f16x2(q4_pair<2>(w.y), s);
  h[7] = mul_f16x2(q4_pair<3>(w.y), s);
}

// Rows [r0, r1) of a sequence, by (page, head): 256 threads to one, or where
// pages are small as many as it has groups.  (One running index over pages,
// heads, rows and groups costs a 64-bit division a group: 293 instructions
// for 32 of them, 23 us for 16404 tokens of 8 heads.)
template <typename E, int D>
__device__ __forceinline__ void expand_rows(const ExpandTo& t, const int32_t* table, int r0, int r1) {
  constexpr int G = D / kQ4Group;
  const int P = t.page_size, per = P * G;
  const int wide = min(per, kThreads), sub = threadIdx.x / wide, at = threadIdx.x - sub * wide, turn = kThreads / wide;
  const int end = (r1 - 1) / P + 1;
  for (int k0 = r0 / P; k0 < end; k0 += min(t.round, end - k0)) {
    const int units = min(t.round, end - k0) * t.Hkv;
    for (int u = blockIdx.x * turn + sub; u < units; u += gridDim.x * turn) {
      const int k = u / t.Hkv, pg = table[k0 + k];
      if (pg < 0 || pg >= t.num_pages) {
        if (t.err_word) raise_error(t.err_word, SIMSD_EW_PAGE);
        continue;
      }
      // (the page's rows of the range; page k0 + k < 2^31 / P)
      const int first = (k0 + k) * P, lo = max(0, r0 - first) * G, hi = min(P, r1 - first) * G;
      const long long base = (static_cast<long long>(pg) * t.Hkv + (u - k * t.Hkv)) * per;
      constexpr int U = 2;  // groups of a thread whose loads are issued together
      for (int i0 = at; i0 < hi; i0 += U * wide) {
        uint2 kw[U], vw[U];
        uint32_t ks[U], vs[U];
#pragma unroll
        for (int j = 0; j < U; ++j) {
          const int i = i0 + j * wide;
          const long long g = base + (i >= lo && i < hi ? i : max(lo, i0));  // (a row of the range in any case)
          kw[j] = static_cast<const uint2*>(t.c.k_codes)[g];
          vw[j] = static_cast<const uint2*>(t.c.v_codes)[g];
          ks[j] = static_cast<const uint8_t*>(t.c.k_scales)[g];
          vs[j] = static_cast<const uint8_t*>(t.c.v_scales)[g];
        }
#pragma unroll
        for (int j = 0; j < U; ++j) {
          const int i = i0 + j * wide;
          if (i < lo || i >= hi) continue;
          uint32_t h[8];
          group_values(kw[j], ks[j], h);
          put16(static_cast<E*>(t.k) + (base + i) * kQ4Group, h, t.c.k_unit, t.wide);
          group_values(vw[j], vs[j], h);
          put16(static_cast<E*>(t.v) + (base + i) * kQ4Group, h, t.c.v_unit, t.wide);
        }
      }
    }
  }
}

template <typename E, int D>
__global__ void __launch_bounds__(kThreads) expand_kernel(const __grid_constant__ ExpandTo t, const int32_t* first,
                                                          const int32_t* last) {
  pdl_wait();
  pdl_launch_next();
  for (int b = blockIdx.y; b < t.Bt; b += gridDim.y) {
    const int r0 = first[b], r1 = last[b];
    if (r0 >= r1) continue;
    if (r0 < 0 || r1 > static_cast<long long>(t.max_pages) * t.page_size) {
      if (blockIdx.x == 0 && threadIdx.x == 0 && t.err_word) raise_error(t.err_word, SIMSD_EW_PREFIX_LEN);
      continue;
    }
    expand_rows<E, D>(t, t.block_table + static_cast<size_t>(b) * t.max_pages, r0, r1);
  }
}

// The rows that a call of attention sees.
template <typename E, int D>
__global__ void __launch_bounds__(kThreads) expand_seen_kernel(const __grid_constant__ ExpandTo t,
                                                               const __grid_constant__ ChunkArgs a) {
  pdl_wait();
  pdl_launch_next();
  for (int b = blockIdx.y; b < t.Bt; b += gridDim.y) {
    const ChunkSeq s = chunk_seq(a, b);
    if (s.C == 0) continue;
    const Keys k = keys_of<true>(a, s, 0, s.C);
    const int32_t* table = t.block_table + static_cast<size_t>(b) * t.max_pages;
    if (k.lo < k.se) expand_rows<E, D>(t, table, k.lo, k.se);
    if (k.w0 < k.hi) expand_rows<E, D>(t, table, k.w0, k.hi);
  }
}

int wide_ok(const void* k, const void* v) { return ((reinterpret_cast<uintptr_t>(k) | reinterpret_cast<uintptr_t>(v)) & 31u) == 0; }

// About 16 blocks an SM over all sequences.
dim3 expand_grid(int Bt, int num_sms) {
  const int y = std::min(Bt, 65535);
  return dim3(static_cast<unsigned>(std::max(1, (16 * num_sms + y - 1) / y)), static_cast<unsigned>(y));
}

}  // namespace

cudaError_t launch_rope_q4(int elem_bytes, const RopeArgs& a, const simsd_q4_cache& c, int num_sms,
                           cudaStream_t stream) {
  if (elem_bytes == 4) return a.d == 128 ? launch_d<float, 128>(a, c, num_sms, stream) : launch_d<float, 64>(a, c, num_sms, stream);
  return a.d == 128 ? launch_d<__nv_bfloat16, 128>(a, c, num_sms, stream)
                    : launch_d<__nv_bfloat16, 64>(a, c, num_sms, stream);
}

cudaError_t launch_q4_expand(int elem_bytes, const ExpandArgs& a, int num_sms, cudaStream_t stream) {
  const ExpandTo t{a.c, a.block_table, a.k_cache, a.v_cache, a.num_pages, a.max_pages, a.page_size, a.Bt, a.Hkv, a.err_word,
                   wide_ok(a.k_cache, a.v_cache), (1 << 30) / a.Hkv};
  auto* kern = elem_bytes == 4 ? (a.d == 128 ? expand_kernel<float, 128> : expand_kernel<float, 64>)
                               : (a.d == 128 ? expand_kernel<__nv_bfloat16, 128> : expand_kernel<__nv_bfloat16, 64>);
  return launch_overlapped(kern, expand_grid(a.Bt, num_sms), dim3(kThreads), 0, stream, 1u, t, a.first, a.last);
}

cudaError_t launch_q4_expand_seen(int elem_bytes, const ChunkArgs& a, const simsd_q4_cache& c, void* k_image,
                                  void* v_image, int num_sms, cudaStream_t stream) {
  const ExpandTo t{c, a.block_table, k_image, v_image, a.num_pages, a.max_pages, a.page_size, a.Bt, a.Hkv, nullptr,
                   wide_ok(k_image, v_image), (1 << 30) / a.Hkv};
  auto* kern = elem_bytes == 4
                   ? (a.d == 128 ? expand_seen_kernel<float, 128> : expand_seen_kernel<float, 64>)
                   : (a.d == 128 ? expand_seen_kernel<__nv_bfloat16, 128> : expand_seen_kernel<__nv_bfloat16, 64>);
  return launch_overlapped(kern, expand_grid(a.Bt, num_sms), dim3(kThreads), 0, stream, 1u, t, a);
}

}  // namespace simsd
