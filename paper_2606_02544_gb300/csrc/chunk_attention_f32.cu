// chunk_attention_f32.cu -- fp32 attention of a chunk of new tokens over the
// paged cache, on the CUDA cores.  One CTA per query row; its warps take the
// visible keys in chunks of 32 (a key per lane), fold each chunk into their
// running maximum and sum, and are merged at the end.
#include <cuda_runtime.h>

#include "chunk_mask.cuh"
#include "common.cuh"
#include "kernels.h"

namespace simsd {
namespace {

constexpr int kWarps = 4;

template <int DPL>  // head-dim elements per lane (d = 32 * DPL)
__global__ void __launch_bounds__(kWarps * 32) chunk_f32_kernel(const __grid_constant__ ChunkArgs a) {
  constexpr int d = 32 * DPL;
  __shared__ __align__(16) float q_s[d];
  __shared__ float acc_s[kWarps][d];
  __shared__ float m_s[kWarps], l_s[kWarps];
  pdl_wait();
  pdl_launch_next();
  const unsigned full = 0xffffffffu;
  const int lane = threadIdx.x & 31, warp = threadIdx.x >> 5;
  const int tok = blockIdx.x / a.Hq, h = blockIdx.x - tok * a.Hq, kvh = h / (a.Hq / a.Hkv);
  if (blockIdx.x == 0) {
    uint32_t e = 0;
    for (int b = threadIdx.x; b < a.Bt; b += blockDim.x) {
      const ChunkSeq s = chunk_seq(a, b);
      e |= (s.bad_off ? SIMSD_EW_TOKENS : 0u) | (s.bad && s.C > 0 ? SIMSD_EW_PREFIX_LEN : 0u);
    }
    if (e) raise_error(a.err_word, e);
  }
  const int b = warp_find_seq(a.token_start, a.Bt, tok);
  if (b < 0) return;
  const ChunkSeq s = chunk_seq(a, b);
  if (s.bad_off) return;
  const size_t row = static_cast<size_t>(tok) * a.Hq + h;
  float* o = static_cast<float*>(a.out) + row * d;
  const int i = tok - s.start;
  const int lo = s.bad ? 0 : key_lo(a, s, i), hi = s.bad ? 0 : key_hi(a, s, i);
  const int32_t* bt = a.block_table + static_cast<size_t>(b) * a.max_pages;
  bool bad_page = false;
  if (hi > lo)
    for (int p = lo / a.page_size + lane; p <= (hi - 1) / a.page_size; p += 32)
      bad_page |= bt[p] < 0 || bt[p] >= a.num_pages;
  bad_page = __any_sync(full, bad_page);
  if (bad_page && threadIdx.x == 0) raise_error(a.err_word, SIMSD_EW_PAGE);
  for (int c = threadIdx.x; c < d; c += blockDim.x)
    q_s[c] = static_cast<const float*>(a.q)[static_cast<long long>(tok) * a.q_stride + static_cast<long long>(h) * d + c];
  __syncthreads();
  float acc[DPL];
#pragma unroll
  for (int c = 0; c < DPL; ++c) acc[c] = 0.f;
  float m = -INFINITY, l = 0.f;
  if (!bad_page) {
    for (int base = lo + 32 * warp; base < hi; base += 32 * kWarps) {
      const int j = base + lane;
      long long off = 0;
      float sc = -INFINITY;
      if (j < hi) {
        const int pi = j / a.page_size;
        off = ((static_cast<long long>(bt[pi]) * a.Hkv + kvh) * a.page_size + (j - pi * a.page_size)) * d;
        const float4* k4 = reinterpret_cast<const float4*>(static_cast<const float*>(a.k_cache) + off);
        const float4* q4 = reinterpret_cast<const float4*>(q_s);
        float dot = 0.f;
#pragma unroll 8
        for (int c = 0; c < d / 4; ++c) {
          const float4 kv = k4[c], qv = q4[c];
          dot = fmaf(qv.x, kv.x, dot);
          dot = fmaf(qv.y, kv.y, dot);
          dot = fmaf(qv.z, kv.z, dot);
          dot = fmaf(qv.w, kv.w, dot);
        }
        sc = dot * a.scale;
      }
      float mc = sc;
#pragma unroll
      for (int w = 16; w > 0; w >>= 1) mc = fmaxf(mc, __shfl_xor_sync(full, mc, w));
      const float m_new = fmaxf(m, mc);
      if (m_new == -INFINITY) continue;
      const float corr = expf(m - m_new), pr = expf(sc - m_new);
      float ps = pr;
#pragma unroll
      for (int w = 16; w > 0; w >>= 1) ps += __shfl_xor_sync(full, ps, w);
      l = l * corr + ps;
#pragma unroll
      for (int c = 0; c < DPL; ++c) acc[c] *= corr;
      const int cnt = min(32, hi - base);
      for (int u = 0; u < cnt; ++u) {
        const float* vr = static_cast<const float*>(a.v_cache) + __shfl_sync(full, off, u);
        const float pu = __shfl_sync(full, pr, u);
#pragma unroll
        for (int c = 0; c < DPL; ++c) acc[c] = fmaf(pu, vr[lane + 32 * c], acc[c]);
      }
      m = m_new;
    }
  }
  if (lane == 0) {
    m_s[warp] = m;
    l_s[warp] = l;
  }
#pragma unroll
  for (int c = 0; c < DPL; ++c) acc_s[warp][lane + 32 * c] = acc[c];
  __syncthreads();
  float M = -INFINITY, L = 0.f, f[kWarps];
#pragma unroll
  for (int w = 0; w < kWarps; ++w) M = fmaxf(M, m_s[w]);
#pragma unroll
  for (int w = 0; w < kWarps; ++w) {
    f[w] = m_s[w] == -INFINITY ? 0.f : expf(m_s[w] - M);
    L = fmaf(f[w], l_s[w], L);
  }
  const float inv = L > 0.f ? 1.f / L : 0.f;
  for (int c = threadIdx.x; c < d; c += blockDim.x) {
    float v = 0.f;
#pragma unroll
    for (int w = 0; w < kWarps; ++w) v = fmaf(f[w], acc_s[w][c], v);
    o[c] = v * inv;
  }
  if (a.lse && threadIdx.x == 0) a.lse[row] = L > 0.f ? M + logf(L) : -INFINITY;
}

}  // namespace

cudaError_t launch_chunk_attention_f32(const ChunkArgs& a, cudaStream_t stream) {
  const unsigned blocks = static_cast<unsigned>(static_cast<long long>(a.T) * a.Hq);
  if (a.d == 64)
    return launch_overlapped(chunk_f32_kernel<2>, dim3(blocks), dim3(kWarps * 32), 0, stream, 1u, a);
  return launch_overlapped(chunk_f32_kernel<4>, dim3(blocks), dim3(kWarps * 32), 0, stream, 1u, a);
}

}  // namespace simsd
