// pages.cu -- the pages of a paged cache: forking, extending and releasing
// sequences, and making the pool dense again (Sec. 3.3: the prefix is read
// from a KV cache; these calls say which pages hold it).
//
// State.  refs[p] counts the block-table entries that name page p; a page is
// free where it is 0.  There is no list of free pages besides: every call
// finds the lowest free ones in refs itself, so the result of a call depends
// on the tables and counts alone, and a pool is made by zeroing them.
//
// Each call that takes pages has one CTA count what is wanted, look for free
// pages (16384 counts a step) and hand them out in order; nothing is changed
// where they do not suffice.  Contents (fork: the pages that are filled in
// part, compact: the live pages above the count of live ones) are copied by a
// second launch over all SMs from a list in the workspace.
//
// Bound: the copies by memory (each byte read once, where a source page is
// copied many times from L2, and written once), the bookkeeping by the
// latency of a chain of dependent loads and barriers in one CTA, some 8 us.
// 32 forks of a sequence whose last page is filled in part, 268 MB, copy in 46 us
// (5.8 TB/s), 500 pages, 457 MB read and written, in 66 (6.9 TB/s).
#include <cuda_runtime.h>

#include <algorithm>

#include "common.cuh"
#include "kernels.h"

namespace simsd {
namespace {

constexpr int kPlanThreads = 1024;
constexpr int kPerThread = 16;  // counts of a thread in a step of the search
constexpr int kStep = kPlanThreads * kPerThread;
constexpr int kList = 4096;     // free pages handed out in a round
constexpr int kCopyThreads = 256;
constexpr int kVecs = 8;        // 16-byte vectors of a thread in flight
constexpr int kChunk = kCopyThreads * kVecs * 16;  // bytes of a block's turn

// Inclusive sum over the block; every thread gets the total as well.
struct BlockSum {
  int part[kPlanThreads / 32 + 1];
};
__device__ __forceinline__ int block_inclusive(BlockSum& sm, int v, int& total) {
  const unsigned full = 0xffffffffu;
  const int lane = threadIdx.x & 31, warp = threadIdx.x >> 5;
#pragma unroll
  for (int o = 1; o < 32; o <<= 1) {
    const int y = __shfl_up_sync(full, v, o);
    if (lane >= o) v += y;
  }
  __syncthreads();  // (part has been read by all of the last call)
  if (lane == 31) sm.part[warp] = v;
  __syncthreads();
  int w = sm.part[lane];
#pragma unroll
  for (int o = 1; o < 32; o <<= 1) {
    const int y = __shfl_up_sync(full, w, o);
    if (lane >= o) w += y;
  }
  total = __shfl_sync(full, w, 31);
  const int before = __shfl_sync(full, w, (warp - 1) & 31);
  return v + (warp > 0 ? before : 0);
}

// Bit i of the result: page p0 + i is free (below n).
__device__ __forceinline__ uint32_t free_bits(const int32_t* refs, int p0, int n) {
  uint32_t m = 0;
  int4 r[kPerThread / 4];
#pragma unroll
  for (int k = 0; k < kPerThread / 4; ++k) {
    const int p = p0 + 4 * k;
    r[k] = make_int4(1, 1, 1, 1);
    if (p + 3 < n) {
      r[k] = *reinterpret_cast<const int4*>(refs + p);
    } else {
      if (p < n) r[k].x = refs[p];
      if (p + 1 < n) r[k].y = refs[p + 1];
      if (p + 2 < n) r[k].z = refs[p + 2];
    }
  }
#pragma unroll
  for (int k = 0; k < kPerThread / 4; ++k)
    m |= (r[k].x <= 0 ? 1u : 0u) << (4 * k) | (r[k].y <= 0 ? 2u : 0u) << (4 * k) |
         (r[k].z <= 0 ? 4u : 0u) << (4 * k) | (r[k].w <= 0 ? 8u : 0u) << (4 * k);
  return m;
}

// The search for free pages of one CTA: `list` gets the ids of the free pages
// numbered base .. base + kList - 1 from the lowest on.  Returns how many free
// pages there are, counted only as far as `most`.  first: the thread's bits of
// the first step, loaded while other loads were on their way.
struct Free {
  BlockSum sum;
  int list[kList];
};
__device__ __forceinline__ uint32_t step_bits(const int32_t* refs, int num_pages, long long s0) {
  const long long p0 = s0 + static_cast<long long>(threadIdx.x) * kPerThread;
  return p0 < num_pages ? free_bits(refs, static_cast<int>(p0), num_pages) : 0u;
}
__device__ int find_free(Free& sm, const int32_t* refs, int num_pages, uint32_t first, int base, int most) {
  int found = 0;
  for (long long s0 = 0; s0 < num_pages && found < most; s0 += kStep) {
    const int p0 = static_cast<int>(s0) + threadIdx.x * kPerThread;
    uint32_t m = s0 == 0 ? first : step_bits(refs, num_pages, s0);
    const int c = __popc(m);
    int total;
    int at = found + block_inclusive(sm.sum, c, total) - c - base;
    while (m) {
      const int i = __ffs(m) - 1;
      m &= m - 1;
      if (at >= 0 && at < kList) sm.list[at] = p0 + i;
      ++at;
    }
    found += total;
  }
  __syncthreads();
  return found;
}

// ------------------------------------------------------------------ extend
// Wanted pages of sequence b: entries of its rows [len, len + add) that name none.
struct Span {
  int first, last;  // entries
  bool bad;
};
__device__ __forceinline__ Span span_of(const PagesArgs& a, int b) {
  Span s{0, 0, false};
  const long long n = a.lens[b], add = a.add[b];
  s.bad = n < 0 || add < 0 || n + add > static_cast<long long>(a.max_pages) * a.page_size;
  if (s.bad || add == 0) return s;
  s.first = static_cast<int>(n / a.page_size);
  s.last = static_cast<int>((n + add + a.page_size - 1) / a.page_size);
  return s;
}

// How many entries of the span name no page; 0 where the span is refused (a
// page in it is shared, or none of the pool's).
constexpr int kShort = 8;  // entries that a thread looks at by itself, at once
__device__ __forceinline__ uint32_t entry_error(const PagesArgs& a, int pg) {
  if (pg == -1) return 0u;
  if (pg < 0 || pg >= a.num_pages) return SIMSD_EW_PAGE;
  return a.refs[pg] > 1 ? SIMSD_EW_SHARED : 0u;
}
__device__ __forceinline__ int wanted(const PagesArgs& a, int b, const Span& s, uint32_t* err) {
  const unsigned full = 0xffffffffu;
  const int lane = threadIdx.x & 31, len = s.last - s.first;
  int n = 0;
  if (len > 0 && len <= kShort) {
    const int32_t* row = a.block_table + static_cast<size_t>(b) * a.max_pages + s.first;
    int pg[kShort];
    uint32_t e = 0;
#pragma unroll
    for (int k = 0; k < kShort; ++k) pg[k] = k < len ? row[k] : 0;
#pragma unroll
    for (int k = 0; k < kShort; ++k) {
      if (k >= len) continue;
      n += pg[k] == -1;
      e |= entry_error(a, pg[k]);
    }
    *err |= e;
    if (e) n = 0;
  }
  // longer spans: the warp together
  for (unsigned m = __ballot_sync(full, len > kShort); m; m &= m - 1) {
    const int who = __ffs(m) - 1;
    const int bb = __shfl_sync(full, b, who), first = __shfl_sync(full, s.first, who), last = __shfl_sync(full, s.last, who);
    const int32_t* row = a.block_table + static_cast<size_t>(bb) * a.max_pages;
    int c = 0;
    uint32_t e = 0;
    for (int k = first + lane; k < last; k += 32) {
      const int pg = row[k];
      c += pg == -1;
      e |= entry_error(a, pg);
    }
    c = __reduce_add_sync(full, c);
    e = __reduce_or_sync(full, e);
    if (lane == who) {
      n = e ? 0 : c;
      *err |= e;
    }
  }
  return n;
}

__global__ void __launch_bounds__(kPlanThreads, 1) extend_kernel(const __grid_constant__ PagesArgs a) {
  __shared__ Free sm;
  pdl_wait();
  pdl_launch_next();
  const unsigned full = 0xffffffffu;
  const int tid = threadIdx.x, lane = tid & 31;
  const uint32_t first = step_bits(a.refs, a.num_pages, 0);
  // a thread per sequence, in rounds; of the first round it keeps what it found
  uint32_t err = 0;
  Span mine{0, 0, true};
  int mine_n = 0, mine_at = 0, total = 0;
  // (granted: whether a sequence was refused is said as soon as that is known,
  // too few free pages for those that want one below)
  auto say = [&](int b, bool ok) {
    if (a.granted && b < a.Bt) a.granted[b] = ok ? a.lens[b] : -1;
  };
  auto look = [&](int b, Span& s, uint32_t* e) {
    s = Span{0, 0, true};
    if (b < a.Bt) {
      s = span_of(a, b);
      if (s.bad) *e |= SIMSD_EW_PREFIX_LEN;
    }
    return wanted(a, b, s, e);
  };
  for (int b0 = 0; b0 < a.Bt; b0 += kPlanThreads) {
    Span s;
    uint32_t here = 0;
    const int n = look(b0 + tid, s, &here);
    say(b0 + tid, here == 0);
    err |= here;
    int turn;
    const int at = total + block_inclusive(sm.sum, n, turn) - n;
    if (b0 == 0) {
      mine = s;
      mine_n = n;
      mine_at = at;
    }
    total += turn;
  }
  if (err) raise_error(a.err_word, err);
  if (total == 0) return;
  if (find_free(sm, a.refs, a.num_pages, first, 0, total) < total) {
    if (tid == 0) raise_error(a.err_word, SIMSD_EW_POOL);
    for (int b0 = 0; a.granted && b0 < a.Bt; b0 += kPlanThreads) {
      Span s;
      uint32_t ignored = 0;
      if (look(b0 + tid, s, &ignored) > 0) say(b0 + tid, false);
    }
    return;
  }
  // Requests are numbered by sequence, then entry.  A round hands out the
  // pages of the list, requests base .. base + kList - 1.
  for (int base = 0; base < total; base += kList) {
    if (base > 0) {
      // (the pages of the last round are taken now, and its entries want none
      // any more: list and requests are numbered anew)
      __syncthreads();
      find_free(sm, a.refs, a.num_pages, step_bits(a.refs, a.num_pages, 0), 0, total - base);
    }
    const int room = min(kList, total - base);
    int before = 0;
    for (int b0 = 0; b0 < a.Bt && before < room; b0 += kPlanThreads) {
      const int b = b0 + tid;
      Span s = mine;
      int n = mine_n, at = mine_at, turn = 0;
      if (base > 0 || b0 > 0) {
        uint32_t ignored = 0;
        n = look(b, s, &ignored);
        at = before + block_inclusive(sm.sum, n, turn) - n;
      } else if (a.Bt > kPlanThreads) {
        block_inclusive(sm.sum, n, turn);
      }
      const int len = s.last - s.first;
      if (n > 0 && len <= kShort) {
        int32_t* row = a.block_table + static_cast<size_t>(b) * a.max_pages + s.first;
        for (int k = 0, j = at; k < len; ++k) {
          if (row[k] != -1) continue;
          if (j < room) {
            row[k] = sm.list[j];
            a.refs[sm.list[j]] = 1;
          }
          ++j;
        }
      }
      for (unsigned m = __ballot_sync(full, n > 0 && len > kShort); m; m &= m - 1) {
        const int who = __ffs(m) - 1;
        int32_t* row = a.block_table + static_cast<size_t>(__shfl_sync(full, b, who)) * a.max_pages;
        const int from = __shfl_sync(full, s.first, who), last = __shfl_sync(full, s.last, who);
        int j0 = __shfl_sync(full, at, who);
        for (int k0 = from; k0 < last; k0 += 32) {
          const int k = k0 + lane;
          const bool none = k < last && row[k] == -1;
          const unsigned w = __ballot_sync(full, none);
          const int j = j0 + __popc(w & ((1u << lane) - 1u));
          if (none && j < room) {
            row[k] = sm.list[j];
            a.refs[sm.list[j]] = 1;
          }
          j0 += __popc(w);
        }
      }
      before += turn;
      if (a.Bt <= kPlanThreads) break;
    }
  }
}

// ----------------------------------------------------------------- release
// Block (i, y): entries of sequence seq[i] whose pages lie wholly within rows
// [first[i], last[i]).  An entry is taken by exchange, so that a sequence
// named twice is released once.
__global__ void __launch_bounds__(256) release_kernel(const __grid_constant__ PagesArgs a) {
  pdl_wait();
  pdl_launch_next();
  for (int i = blockIdx.x; i < a.n; i += gridDim.x) {
    const int b = a.seq ? a.seq[i] : i;
    if (b < 0 || b >= a.Bt) {
      if (threadIdx.x == 0) raise_error(a.err_word, SIMSD_EW_SEQ);
      continue;
    }
    const long long f = max(0, a.first[i]), l = a.last[i];
    const int k0 = static_cast<int>(min(static_cast<long long>(a.max_pages), (f + a.page_size - 1) / a.page_size));
    const int k1 = static_cast<int>(min(static_cast<long long>(a.max_pages), max(0ll, l / a.page_size)));
    int32_t* row = a.block_table + static_cast<size_t>(b) * a.max_pages;
    for (int k = k0 + blockIdx.y * 256 + threadIdx.x; k < k1; k += gridDim.y * 256) {
      if (row[k] == -1) continue;
      const int pg = atomicExch(&row[k], -1);
      if (pg == -1) continue;
      if (pg < 0 || pg >= a.num_pages) {
        raise_error(a.err_word, SIMSD_EW_PAGE);
      } else if (atomicSub(&a.refs[pg], 1) <= 0) {
        atomicAdd(&a.refs[pg], 1);  // counted too low before: stays as it was
        raise_error(a.err_word, SIMSD_EW_PAGE);
      }
    }
  }
}

// -------------------------------------------------------------------- fork
// Workspace of fork and compact: {count of moves, live pages, 0, 0}, then the
// moves (from, to); fork: then per pair its state; compact: then where each
// page goes.
struct Header {
  int moves, live, pad0, pad1;
};
__device__ __forceinline__ Header* header(const PagesArgs& a) { return static_cast<Header*>(a.workspace); }
__device__ __forceinline__ int2* moves_of(const PagesArgs& a) { return reinterpret_cast<int2*>(header(a) + 1); }

// state of a pair: -1 nothing is done, 0 no page is filled in part, else the
// new page + 1
__device__ __forceinline__ int* pair_state(const PagesArgs& a) { return reinterpret_cast<int*>(moves_of(a) + a.n); }

__global__ void __launch_bounds__(kPlanThreads, 1) fork_plan_kernel(const __grid_constant__ PagesArgs a) {
  __shared__ Free sm;
  extern __shared__ uint32_t marks[];  // [words] a source, [words] a destination, [words] one twice
  const int words = (a.Bt + 31) / 32;
  uint32_t *is_src = marks, *is_dst = marks + words, *twice = marks + 2 * words;
  const int tid = threadIdx.x;
  for (int i = tid; i < 3 * words; i += kPlanThreads) marks[i] = 0u;
  __syncthreads();
  pdl_wait();
  pdl_launch_next();
  const uint32_t first = step_bits(a.refs, a.num_pages, 0);
  auto inside = [&](int b) { return b >= 0 && b < a.Bt; };
  for (int i = tid; i < a.n; i += kPlanThreads) {
    const int s = a.src[i], d = a.dst[i];
    if (inside(s)) atomicOr(&is_src[s >> 5], 1u << (s & 31));
    if (inside(d) && (atomicOr(&is_dst[d >> 5], 1u << (d & 31)) >> (d & 31) & 1u)) atomicOr(&twice[d >> 5], 1u << (d & 31));
  }
  __syncthreads();
  const long long most = static_cast<long long>(a.max_pages) * a.page_size;
  uint32_t err = 0;
  // a pair's source page that is filled in part (-1: none), or -2: refused
  auto partial = [&](int i) {
    const int s = a.src[i], d = a.dst[i];
    if (!inside(s) || !inside(d) || (is_src[d >> 5] >> (d & 31) & 1u) || (twice[d >> 5] >> (d & 31) & 1u)) {
      err |= SIMSD_EW_SEQ;
      return -2;
    }
    const int n = a.lens[s];
    if (n < 0 || n > most) {
      err |= SIMSD_EW_PREFIX_LEN;
      return -2;
    }
    if (n % a.page_size == 0) return -1;
    const int pg = a.block_table[static_cast<size_t>(s) * a.max_pages + n / a.page_size];
    if (pg < -1 || pg >= a.num_pages) {
      err |= SIMSD_EW_PAGE;
      return -2;
    }
    return pg;
  };
  // (of the first round a thread keeps what it found)
  int total = 0, mine = -2, mine_at = 0;
  for (int i0 = 0; i0 < a.n; i0 += kPlanThreads) {
    const int pg = i0 + tid < a.n ? partial(i0 + tid) : -2;
    int turn;
    const int at = total + block_inclusive(sm.sum, pg >= 0, turn) - 1;
    if (i0 == 0) {
      mine = pg;
      mine_at = at;
    }
    total += turn;
  }
  if (err) raise_error(a.err_word, err);
  const int have = total ? find_free(sm, a.refs, a.num_pages, first, 0, total) : 0;
  const bool short_of = have < total;
  if (tid == 0) {
    if (short_of) raise_error(a.err_word, SIMSD_EW_POOL);
    *header(a) = Header{short_of ? 0 : total, 0, 0, 0};
  }
  int before = 0, base = 0;
  for (int i0 = 0; i0 < a.n; i0 += kPlanThreads) {
    const int i = i0 + tid;
    int pg = mine, at = mine_at, turn = 0;
    if (a.n > kPlanThreads) {
      pg = i < a.n ? partial(i) : -2;
      at = before + block_inclusive(sm.sum, pg >= 0, turn) - 1;
      if (!short_of && before + turn > base + kList) {
        // (a turn wants at most 1024 pages, the list holds 4096)
        base = before;
        find_free(sm, a.refs, a.num_pages, first, base, base + kList);
      }
    }
    if (i < a.n) {
      int st = pg == -2 || short_of ? -1 : 0;
      if (st == 0 && pg >= 0) {
        const int to = sm.list[at - base];
        moves_of(a)[at] = make_int2(pg, to);
        if (a.n <= kPlanThreads) a.refs[to] = 1;
        st = to + 1;
      }
      pair_state(a)[i] = st;
    }
    before += turn;
  }
  // the pages are taken once nobody looks for free ones any more
  __syncthreads();
  if (!short_of && a.n > kPlanThreads)
    for (int i = tid; i < total; i += kPlanThreads) a.refs[moves_of(a)[i].y] = 1;
}

// Copies the contents of the listed pages in every layer of every array.
__device__ __forceinline__ void copy_pages(const PagesArgs& a, int moves) {
  // turns: for each layer of an array, for each chunk of a page, the moves
  // (the copies of one source follow each other)
  long long turns = 0;
  for (int k = 0; k < a.pages.n; ++k)
    turns += static_cast<long long>(a.pages.array[k].layers) * ((a.pages.array[k].page_bytes + kChunk - 1) / kChunk);
  turns *= moves;
  const int2* list = moves_of(a);
  for (long long u = blockIdx.x; u < turns; u += gridDim.x) {
    long long t = u / moves;
    const int2 mv = list[u - t * moves];
    int k = 0;
    long long chunks = 0;
    for (; k < a.pages.n; ++k) {
      chunks = (a.pages.array[k].page_bytes + kChunk - 1) / kChunk;
      const long long here = a.pages.array[k].layers * chunks;
      if (t < here) break;
      t -= here;
    }
    const simsd_page_array& x = a.pages.array[k];
    const long long layer = t / chunks, off = (t - layer * chunks) * kChunk;
    uint8_t* plane = static_cast<uint8_t*>(x.base) + layer * x.layer_bytes + off;
    const uint4* from = reinterpret_cast<const uint4*>(plane + mv.x * x.page_bytes);
    uint4* to = reinterpret_cast<uint4*>(plane + mv.y * x.page_bytes);
    const int vecs = static_cast<int>(min(static_cast<long long>(kChunk), x.page_bytes - off) / 16);
    uint4 v[kVecs];
#pragma unroll
    for (int j = 0; j < kVecs; ++j) {
      const int i = j * kCopyThreads + threadIdx.x;
      if (i < vecs) v[j] = from[i];
    }
#pragma unroll
    for (int j = 0; j < kVecs; ++j) {
      const int i = j * kCopyThreads + threadIdx.x;
      if (i < vecs) to[i] = v[j];
    }
  }
}

__global__ void __launch_bounds__(kCopyThreads) fork_kernel(const __grid_constant__ PagesArgs a) {
  pdl_wait();
  pdl_launch_next();
  const int moves = header(a)->moves;
  // tables, lengths and counts: a block per pair
  for (int i = blockIdx.x; i < a.n; i += gridDim.x) {
    const int st = pair_state(a)[i];
    if (st < 0) continue;
    const int s = a.src[i], d = a.dst[i], n = a.lens[s], whole = n / a.page_size;
    const int32_t* from = a.block_table + static_cast<size_t>(s) * a.max_pages;
    int32_t* to = a.block_table + static_cast<size_t>(d) * a.max_pages;
    for (int k = threadIdx.x; k < a.max_pages; k += kCopyThreads) {
      const int old = to[k];
      int pg = k < whole ? from[k] : k == whole && st > 0 ? st - 1 : -1;
      if (pg < -1 || pg >= a.num_pages) {
        raise_error(a.err_word, SIMSD_EW_PAGE);
        pg = -1;
      }
      if (k < whole && pg >= 0) atomicAdd(&a.refs[pg], 1);
      if (old != -1) {
        if (old < 0 || old >= a.num_pages) {
          raise_error(a.err_word, SIMSD_EW_PAGE);
        } else if (atomicSub(&a.refs[old], 1) <= 0) {
          atomicAdd(&a.refs[old], 1);
          raise_error(a.err_word, SIMSD_EW_PAGE);
        }
      }
      if (pg != old) to[k] = pg;
    }
    if (threadIdx.x == 0) a.lens[d] = n;
  }
  copy_pages(a, moves);
}

// ----------------------------------------------------------------- compact
__device__ __forceinline__ int* where_to(const PagesArgs& a) { return reinterpret_cast<int*>(moves_of(a) + a.num_pages); }

// The k-th live page above the count of live ones goes to the k-th free one
// below it.
__global__ void __launch_bounds__(kPlanThreads, 1) compact_plan_kernel(const __grid_constant__ PagesArgs a) {
  __shared__ Free sm;
  pdl_wait();
  pdl_launch_next();
  const int tid = threadIdx.x;
  // the free pages of a step, loaded again only where there are more steps
  const uint32_t first = step_bits(a.refs, a.num_pages, 0);
  auto bits = [&](long long s0) { return s0 == 0 ? first : step_bits(a.refs, a.num_pages, s0); };
  int free_pages = 0;
  for (long long s0 = 0; s0 < a.num_pages; s0 += kStep) free_pages += __popc(bits(s0));
  int total_free;
  block_inclusive(sm.sum, free_pages, total_free);
  const int live = a.num_pages - total_free;
  int2* moves = moves_of(a);
  int* to = where_to(a);
  // bit i: page p0 + i lies below the count of live ones
  auto below = [&](long long p0) { return p0 + kPerThread <= live ? (1u << kPerThread) - 1u : p0 < live ? (1u << (live - p0)) - 1u : 0u; };
  // holes first (they all lie below the pages that fill them), then movers
  int holes = 0;
  for (long long s0 = 0; s0 < live; s0 += kStep) {
    const long long p0 = s0 + static_cast<long long>(tid) * kPerThread;
    uint32_t m = bits(s0) & below(p0);
    const int c = __popc(m);
    int turn, at = holes + block_inclusive(sm.sum, c, turn) - c;
    for (; m; m &= m - 1, ++at) {
      const int p = static_cast<int>(p0) + __ffs(m) - 1;
      moves[at].y = p;
      if (at < kList) sm.list[at] = p;
    }
    holes += turn;
  }
  __syncthreads();
  int moved = 0;
  for (long long s0 = live / kStep * static_cast<long long>(kStep); s0 < a.num_pages; s0 += kStep) {
    const long long p0 = s0 + static_cast<long long>(tid) * kPerThread;
    const int n = p0 < a.num_pages ? static_cast<int>(min(static_cast<long long>(kPerThread), a.num_pages - p0)) : 0;
    const uint32_t above = ~below(p0) & ((1u << n) - 1u), used = n > 0 ? ~bits(s0) & above : 0u;
    const int c = __popc(used);
    int turn, at = moved + block_inclusive(sm.sum, c, turn) - c;
    for (uint32_t m = above; m; m &= m - 1) {
      const int i = __ffs(m) - 1, p = static_cast<int>(p0) + i;
      int dst = p;
      if (used >> i & 1u) {
        dst = at < kList ? sm.list[at] : moves[at].y;
        moves[at++].x = p;
        a.refs[dst] = a.refs[p];
        a.refs[p] = 0;
      }
      to[p] = dst;
    }
    moved += turn;
  }
  if (tid == 0) {
    *header(a) = Header{moved, live, 0, 0};
    if (a.live) *a.live = live;
  }
}

__global__ void __launch_bounds__(kCopyThreads) compact_kernel(const __grid_constant__ PagesArgs a) {
  pdl_wait();
  pdl_launch_next();
  const Header h = *header(a);
  const long long entries = static_cast<long long>(a.Bt) * a.max_pages;
  for (long long i = static_cast<long long>(blockIdx.x) * kCopyThreads + threadIdx.x; i < entries;
       i += static_cast<long long>(gridDim.x) * kCopyThreads) {
    const int pg = a.block_table[i];
    if (pg < -1 || pg >= a.num_pages)
      raise_error(a.err_word, SIMSD_EW_PAGE);
    else if (pg >= h.live)
      a.block_table[i] = where_to(a)[pg];
  }
  copy_pages(a, h.moves);
}

// Blocks of the second launch: eight an SM at most (full occupancy), and no
// more than there can be turns.
unsigned copy_blocks(const PagesArgs& a, long long most_moves, long long others, int num_sms) {
  long long turns = 0;
  for (int k = 0; k < a.pages.n; ++k)
    turns += static_cast<long long>(a.pages.array[k].layers) * ((a.pages.array[k].page_bytes + kChunk - 1) / kChunk);
  return static_cast<unsigned>(std::max<long long>(1, std::min<long long>(8ll * num_sms, std::max(turns * most_moves, others))));
}

}  // namespace

size_t pages_workspace_bytes(int num_pages, int pairs) {
  const size_t fork = static_cast<size_t>(pairs) * (sizeof(int2) + sizeof(int));
  const size_t compact = static_cast<size_t>(num_pages) * (sizeof(int2) + sizeof(int));
  return sizeof(Header) + std::max(fork, compact);
}

cudaError_t launch_pages_extend(const PagesArgs& a, cudaStream_t stream) {
  return launch_overlapped(extend_kernel, dim3(1), dim3(kPlanThreads), 0, stream, 1u, a);
}

cudaError_t launch_pages_release(const PagesArgs& a, int num_sms, cudaStream_t stream) {
  const unsigned x = static_cast<unsigned>(std::min(a.n, 64 * num_sms));
  const unsigned y = static_cast<unsigned>(std::max(1, std::min((a.max_pages + 255) / 256, 4 * num_sms / static_cast<int>(x))));
  return launch_overlapped(release_kernel, dim3(x, y), dim3(256), 0, stream, 1u, a);
}

cudaError_t launch_pages_fork(const PagesArgs& a, int num_sms, cudaStream_t stream) {
  const size_t marks = 3 * sizeof(uint32_t) * static_cast<size_t>((a.Bt + 31) / 32);
  cudaError_t e = launch_overlapped(fork_plan_kernel, dim3(1), dim3(kPlanThreads), marks, stream, 1u, a);
  if (e != cudaSuccess) return e;
  return launch_overlapped(fork_kernel, dim3(copy_blocks(a, a.n, a.n, num_sms)), dim3(kCopyThreads), 0, stream, 1u, a);
}

cudaError_t launch_pages_compact(const PagesArgs& a, int num_sms, cudaStream_t stream) {
  cudaError_t e = launch_overlapped(compact_plan_kernel, dim3(1), dim3(kPlanThreads), 0, stream, 1u, a);
  if (e != cudaSuccess) return e;
  const long long rows = (static_cast<long long>(a.Bt) * a.max_pages + kCopyThreads - 1) / kCopyThreads;
  return launch_overlapped(compact_kernel, dim3(copy_blocks(a, a.num_pages / 2 + 1, rows, num_sms)), dim3(kCopyThreads), 0,
                           stream, 1u, a);
}

}  // namespace simsd
