// rope_append.cu -- rotary positions of a chunk of tokens, and the chunk's
// way into the paged cache (Sec. 3.1 "Position Encoding Alignment": keys are
// cached rotated; Sec. 3.3: the prefix is read from the cache).
//
// Mathematics.  The pair i < r/2 of a token at position p turns by p f_i
// (rotary embedding of RoFormer over the first r components; f_i as scaled
// by simsd_rope_plan_init).  The plan holds F_i = round(2^64 f_i / 2 pi), f_i
// a double, and p F_i mod 2^64 is the fraction of a turn.  That product is
// exact; what is lost is the double's rounding, about 4 2^-53 f_i p radians
// (f_i <= 1): below fp32's last bit up to p = 2^27, 2^-20 at p = 2^31.  Its top
// 32 bits, read as a signed number of 2^-31 half turns, go to sincospif.
// Products and sums are fp32, rounded once to the type.
//
// Bound by memory: a token reads and writes (Hq + 2 Hkv) d elements.  A
// thread owns one pair of VE-wide vectors (the two halves of VE pairs, or
// two vectors of interleaved pairs) of one token and walks over heads, so
// the VE angles it forms serve every head it visits; kHeadsInFlight heads'
// loads are issued together (two: with four the registers leave half the
// threads, 108 us instead of 85 for 16384 tokens of 32/8 heads, bf16; angles
// formed once a block in shared memory, 91 us).  Few tokens are spread over
// more threads by giving each fewer heads (down to one).  403 MB in 85 us:
// 4.7 TB/s; what remains is the latency of a thread's loads.
#include <cuda_bf16.h>
#include <cuda_runtime.h>

#include <algorithm>

#include "common.cuh"
#include "kernels.h"
#include "ragged.cuh"

namespace simsd {
namespace {

constexpr int kThreads = 256;
constexpr int kMaxTokens = 64;  // tokens of a block
constexpr int kHeadsInFlight = 2;

template <typename E, int VE>
struct alignas(sizeof(E) * VE) Vec {
  E e[VE];
};

__device__ __forceinline__ float to_f32(float x) { return x; }
__device__ __forceinline__ float to_f32(__nv_bfloat16 x) { return __bfloat162float(x); }
__device__ __forceinline__ void from_f32(float x, float& y) { y = x; }
__device__ __forceinline__ void from_f32(float x, __nv_bfloat16& y) { y = __float2bfloat16_rn(x); }

// a token of the block: its position, destination row of the cache in rows
// of d elements at KV head 0 (-1: not written), and what its q row becomes
struct Token {
  long long row;
  int pos;
  int state;  // 0: outside every sequence (untouched), 1: rotated, 2: zeroed
};

__device__ Token resolve(const RopeArgs& a, int tok) {
  Token t;
  t.row = -1;
  t.pos = 0;
  t.state = 0;
  if (!a.k_cache) {
    t.pos = a.positions[tok];
    t.state = 1;
    return t;
  }
  const int lane = threadIdx.x & 31;
  const int b = warp_find_seq(a.token_start, a.Bt, tok);
  if (b < 0) return t;
  const Chunk c = chunk_of(a.token_start, b, a.T);
  if (c.bad) return t;
  const int n = a.prefix_len[b], i = tok - c.start;
  if (n < 0 || static_cast<long long>(n) + c.count > static_cast<long long>(a.max_pages) * a.page_size) {
    if (lane == 0) raise_error(a.err_word, SIMSD_EW_PREFIX_LEN);
    t.state = 2;
    return t;
  }
  t.state = 1;
  const int dst = n + i, pi = dst / a.page_size;
  t.pos = a.positions ? a.positions[tok] : dst;
  const int pg = a.block_table[static_cast<size_t>(b) * a.max_pages + pi];
  if (pg < 0 || pg >= a.num_pages) {
    if (lane == 0) raise_error(a.err_word, SIMSD_EW_PAGE);
    return t;
  }
  t.row = static_cast<long long>(pg) * a.Hkv * a.page_size + (dst - pi * a.page_size);
  return t;
}

// Thread (token, head group, task): task t of a row is the vectors t and
// t + R of the rotated part (R = r / (2 VE) tasks; 2t and 2t + 1 where
// interleaved pairs are taken one component at a time), then pairs of
// vectors of the rest; a row of V is copied over the same tasks.
template <typename E, int VE>
__global__ void __launch_bounds__(kThreads, 3) rope_kernel(const __grid_constant__ RopeArgs a) {
  using V = Vec<E, VE>;
  __shared__ Token toks[kMaxTokens];
  pdl_wait();
  pdl_launch_next();
  const int warp = threadIdx.x >> 5, lane = threadIdx.x & 31;
  const int tok0 = blockIdx.x * a.tokens_block;
  if (a.k_cache && blockIdx.x == 0) {
    bool bad = false;
    for (int b = threadIdx.x; b < a.Bt; b += kThreads) bad |= chunk_of(a.token_start, b, a.T).bad;
    if (bad) raise_error(a.err_word, SIMSD_EW_TOKENS);
  }
  for (int i = warp; i < a.tokens_block && tok0 + i < a.T; i += kThreads / 32) {
    const Token t = resolve(a, tok0 + i);
    if (lane == 0) toks[i] = t;
  }
  __syncthreads();
  const int R = a.plan.rot_dim / (2 * VE);          // rotating tasks of a row
  const int nvec = a.d / VE, rest = nvec - 2 * R;   // vectors of a row; those not rotated
  const int tasks = R + (rest + 1) / 2;
  const int per_token = tasks * a.groups;
  const int heads = a.Hq + (a.v ? 2 : 1) * a.Hkv;
  const bool half = a.plan.layout == SIMSD_ROPE_HALF;
  for (int w = threadIdx.x; w < a.tokens_block * per_token; w += kThreads) {
    const int i = w / per_token, u = w - i * per_token, grp = u / tasks, t = u - grp * tasks;
    const int tok = tok0 + i;
    if (tok >= a.T) break;
    const Token tk = toks[i];
    if (tk.state == 0) continue;
    const bool turns = t < R;
    // vectors of this task: in the rotated part t and t + R, else two of the
    // rest; of a V row the same two
    const bool split = half || VE == 1;  // a pair's components lie in two vectors
    const int va = turns && (half || VE > 1) ? t : 2 * t, vb = turns && (half || VE > 1) ? t + R : va + 1;
    const bool two = vb < nvec;
    float cs[VE], sn[VE];
    if (turns) {
#pragma unroll
      for (int e = 0; e < VE; ++e) {
        // half: pairs VE t + e; interleaved: the pairs of vector t, then those of vector t + R
        const int pair = split ? VE * t + e : (VE * (e < VE / 2 ? t : t + R)) / 2 + (e < VE / 2 ? e : e - VE / 2);
        const unsigned long long turn =
            static_cast<unsigned long long>(static_cast<long long>(tk.pos)) * a.plan.turn[pair];
        sincospif(static_cast<float>(static_cast<int32_t>(turn >> 32)) * 0x1p-31f, &sn[e], &cs[e]);
        sn[e] *= a.plan.magnitude;
        cs[e] *= a.plan.magnitude;
      }
    }
    for (int h0 = grp; h0 < heads; h0 += a.groups * kHeadsInFlight) {
      V xa[kHeadsInFlight], xb[kHeadsInFlight];
      E* dst[kHeadsInFlight];
#pragma unroll
      for (int k = 0; k < kHeadsInFlight; ++k) {
        const int h = h0 + k * a.groups;
        dst[k] = nullptr;
        if (h < heads) {
          const E* src;
          if (h < a.Hq) {
            src = static_cast<const E*>(a.q) + static_cast<long long>(tok) * a.q_stride + static_cast<long long>(h) * a.d;
            dst[k] = static_cast<E*>(a.q_out) + static_cast<long long>(tok) * a.q_out_stride + static_cast<long long>(h) * a.d;
          } else {
            const int kv = h - a.Hq, hk = kv < a.Hkv ? kv : kv - a.Hkv;
            const bool isv = kv >= a.Hkv;
            src = static_cast<const E*>(isv ? a.v : a.k) + static_cast<long long>(tok) * (isv ? a.v_stride : a.k_stride) +
                  static_cast<long long>(hk) * a.d;
            if (!a.k_cache)
              dst[k] = static_cast<E*>(a.k_out) + static_cast<long long>(tok) * a.k_out_stride + static_cast<long long>(hk) * a.d;
            else if (tk.row >= 0)
              dst[k] = static_cast<E*>(isv ? a.v_cache : a.k_cache) +
                       (tk.row + static_cast<long long>(hk) * a.page_size) * a.d;
          }
          xa[k] = reinterpret_cast<const V*>(src)[va];
          if (two) xb[k] = reinterpret_cast<const V*>(src)[vb];
        }
      }
#pragma unroll
      for (int k = 0; k < kHeadsInFlight; ++k) {
        const int h = h0 + k * a.groups;
        if (h < heads && dst[k]) {
          if (tk.state == 2) {
#pragma unroll
            for (int e = 0; e < VE; ++e) {
              from_f32(0.f, xa[k].e[e]);
              from_f32(0.f, xb[k].e[e]);
            }
          } else if (turns && h < a.Hq + a.Hkv) {
            if (split) {
#pragma unroll
              for (int e = 0; e < VE; ++e) {
                const float x = to_f32(xa[k].e[e]), y = to_f32(xb[k].e[e]);
                from_f32(x * cs[e] - y * sn[e], xa[k].e[e]);
                from_f32(x * sn[e] + y * cs[e], xb[k].e[e]);
              }
            } else {
#pragma unroll
              for (int e = 0; e + 1 < VE; e += 2) {
                const float x = to_f32(xa[k].e[e]), y = to_f32(xa[k].e[e + 1]);
                from_f32(x * cs[e / 2] - y * sn[e / 2], xa[k].e[e]);
                from_f32(x * sn[e / 2] + y * cs[e / 2], xa[k].e[e + 1]);
                const float x2 = to_f32(xb[k].e[e]), y2 = to_f32(xb[k].e[e + 1]);
                from_f32(x2 * cs[VE / 2 + e / 2] - y2 * sn[VE / 2 + e / 2], xb[k].e[e]);
                from_f32(x2 * sn[VE / 2 + e / 2] + y2 * cs[VE / 2 + e / 2], xb[k].e[e + 1]);
              }
            }
          }
          reinterpret_cast<V*>(dst[k])[va] = xa[k];
          if (two) reinterpret_cast<V*>(dst[k])[vb] = xb[k];
        }
      }
    }
  }
}

template <typename E, int VE>
cudaError_t launch_ve(RopeArgs a, int num_sms, cudaStream_t stream) {
  const int R = a.plan.rot_dim / (2 * VE), tasks = R + (a.d / VE - 2 * R + 1) / 2;
  const int heads = a.Hq + (a.v ? 2 : 1) * a.Hkv;
  // Threads for about two full waves of the GPU (2048 a SM) if there are
  // that many (token, task, head) triples; more heads to a thread (fewer
  // angles formed) beyond that.
  const long long want = 2ll * 2048 * num_sms;
  const long long per_head = std::max<long long>(1, static_cast<long long>(a.T) * tasks);
  a.groups = static_cast<int>(std::min<long long>(heads, std::max<long long>(1, want / per_head)));
  // a block's threads all busy, and of many tokens so many that the blocks
  // (three a SM) make one wave: finding a token's sequence and page is a
  // chain of loads, on which a block of few tokens spends most of its time
  a.tokens_block = std::max(kThreads / (tasks * a.groups), (a.T + 3 * num_sms - 1) / (3 * num_sms));
  a.tokens_block = std::max(1, std::min(kMaxTokens, a.tokens_block));
  const unsigned blocks = static_cast<unsigned>((a.T + a.tokens_block - 1) / a.tokens_block);
  return launch_overlapped(rope_kernel<E, VE>, dim3(blocks), dim3(kThreads), 0, stream, 1u, a);
}

}  // namespace

cudaError_t launch_rope(int elem_bytes, const RopeArgs& a, int num_sms, cudaStream_t stream) {
  // the widest vector that divides the rotated part into pairs of vectors
  // (and with it the row): 16 bytes for the usual head sizes, less for a
  // rotated part of, say, 24 components
  const int r = a.plan.rot_dim;
  auto fits = [&](int ve) { return r % (2 * ve) == 0 && a.d % ve == 0; };
  if (elem_bytes == 4) {
    if (fits(4)) return launch_ve<float, 4>(a, num_sms, stream);
    if (fits(2)) return launch_ve<float, 2>(a, num_sms, stream);
    return launch_ve<float, 1>(a, num_sms, stream);
  }
  if (fits(8)) return launch_ve<__nv_bfloat16, 8>(a, num_sms, stream);
  if (fits(4)) return launch_ve<__nv_bfloat16, 4>(a, num_sms, stream);
  if (fits(2)) return launch_ve<__nv_bfloat16, 2>(a, num_sms, stream);
  return launch_ve<__nv_bfloat16, 1>(a, num_sms, stream);
}

}  // namespace simsd
