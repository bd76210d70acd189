// Page pool of the K/V caches (gfx950): which sequence holds which page, and
// the copies of pages that are shared or moved.
//
// The state is a reference count per page (0: free) and each sequence's run of
// page-table entries; those past the run are -1, so that nothing is stored
// through them into a page that another sequence has.  Free pages are given out
// lowest first, in the order of the requests, by one workgroup that walks the
// counts 8192 at a time with ballots: whole-number work with one result however
// the waves run.  Only counts are added to with atomics, and sums of ones have
// no order.
//
// The bookkeeping is a few launches of a few microseconds (15 forks of a prompt
// of 1003 entries in 32 layers: kernels of 2.4 and 4.0 us, and the copy of 15.7 MB
// 5.4); copies run at the rate of a plain copy.
#include <algorithm>

#include "bounds.h"
#include "common.h"
#include "kernels.h"
#include "kvq.h"

namespace sb {
namespace {

typedef uint32_t u32x4 __attribute__((ext_vector_type(4)));

constexpr int kChunk = 8192;          // pages that one workgroup walks at a time
// scratch: number of moves; live pages per chunk; sources; targets; new number
// of every page
constexpr int kCounts = 16, kLists = kCounts + 256;
// entries of a list: a compaction moves at most half of the pages, a fork copies
// at most a page for each of 64 children (of a small pool, more than half)
__host__ __device__ inline size_t list_ints(int n) { return n < 128 ? 64 : (size_t)n / 2; }
__host__ __device__ inline size_t src_at() { return kLists; }
__host__ __device__ inline size_t dst_at(int n) { return kLists + list_ints(n); }
__host__ __device__ inline size_t map_at(int n) { return kLists + 2 * list_ints(n); }

// Walks pages base .. base + kChunk - 1 with 1024 threads: fn(page, rank) for
// each with pred(page), rank counting from `before` in page order.  Returns
// before plus their number.  `cnt`: 128 ints of LDS.
template <typename Pred, typename Fn>
__device__ __forceinline__ int walk_chunk(int base, int n_pages, int before,
                                          int* cnt, Pred pred, Fn fn) {
  const int lane = threadIdx.x & 63;
  const int wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
  unsigned long long mask[8];
#pragma unroll
  for (int j = 0; j < 8; ++j) {
    const int pg = base + j * 1024 + (int)threadIdx.x;
    mask[j] = __ballot(pg < n_pages && pred(pg));
  }
  __syncthreads();                    // (the previous walk's readers are done)
  if (lane == 0)
#pragma unroll
    for (int j = 0; j < 8; ++j) cnt[j * 16 + wave] = __popcll(mask[j]);
  __syncthreads();
  // every wave scans the 128 counts, two a lane (each at most 64)
  const int2 c = reinterpret_cast<const int2*>(cnt)[lane];
  int total;
  const int excl = wave_excl_scan_small<8>(c.x + c.y, total);
  int mine[8];
#pragma unroll
  for (int j = 0; j < 8; ++j) {
    const int i = (j * 16 + wave) >> 1;
    mine[j] = __builtin_amdgcn_readlane(excl, i) +
              (wave & 1 ? __builtin_amdgcn_readlane(c.x, i) : 0);
  }
#pragma unroll
  for (int j = 0; j < 8; ++j) {
    if ((mask[j] >> lane) & 1ull) {
      const int below = (int)__builtin_amdgcn_mbcnt_hi(
          (unsigned)(mask[j] >> 32), __builtin_amdgcn_mbcnt_lo((unsigned)mask[j], 0u));
      fn(base + j * 1024 + (int)threadIdx.x, before + mine[j] + below);
    }
  }
  return before + total;
}

__global__ __launch_bounds__(1024) void pool_reset_kernel(sb_pool p, int max_seqs,
                                                          int max_pages) {
  const size_t step = (size_t)gridDim.x * 1024;
  const size_t i0 = (size_t)blockIdx.x * 1024 + threadIdx.x;
  for (size_t i = i0; i < (size_t)max_seqs * max_pages; i += step) p.page_table[i] = -1;
  for (size_t i = i0; i < (size_t)p.n_pages; i += step) p.refs[i] = 0;
  if (i0 < (size_t)max_seqs) p.held[i0] = 0;
  if (i0 == 0) *p.refused = 0;
}

// Gives `total` free pages, lowest first, to the requests off[i] .. off[i + 1]
// (fn(page, rank)); returns how many there were.
template <typename Fn>
__device__ __forceinline__ int take_pages(const sb_pool& p, int total, int* cnt, Fn fn) {
  int found = 0;
  for (int base = 0; base < p.n_pages && found < total; base += kChunk)
    found = walk_chunk(
        base, p.n_pages, found, cnt, [&](int pg) { return p.refs[pg] <= 0; },
        [&](int pg, int rank) {
          if (rank < total) fn(pg, rank);
        });
  return min(found, total);
}

// the request that rank belongs to: the last i with off[i] <= rank
__device__ __forceinline__ int request_of(const int* off, int n, int rank) {
  int lo = 0, hi = n - 1;
  while (lo < hi) {
    const int m = (lo + hi + 1) >> 1;
    if (off[m] <= rank) lo = m;
    else hi = m - 1;
  }
  return lo;
}

__global__ __launch_bounds__(1024) void pool_grow_kernel(sb_pool p, int n_seqs,
                                                         const int* __restrict__ len,
                                                         int extra, int max_pages) {
  __shared__ __attribute__((aligned(8))) int cnt[128], off[65], have[64], over[64];
  const int t = threadIdx.x;
  if (t < 64) {
    int need = 0;
    have[t] = over[t] = 0;
    if (t < n_seqs) {
      const long long want = (max(0LL, (long long)len[t] + extra) + 15) / 16;
      have[t] = min(max(p.held[t], 0), max_pages);
      over[t] = want > max_pages;
      need = max(0, (int)min(want, (long long)max_pages) - have[t]);
    }
    int incl = need;
    for (int d = 1; d < 64; d <<= 1) {
      const int o = __shfl_up(incl, d, 64);
      if (t >= d) incl += o;
    }
    off[t + 1] = incl;
    if (t == 0) off[0] = 0;
  }
  __syncthreads();
  const int found = take_pages(p, off[64], cnt, [&](int pg, int rank) {
    const int s = request_of(off, 64, rank);
    p.page_table[(size_t)s * max_pages + have[s] + rank - off[s]] = pg;
    p.refs[pg] = 1;
  });
  if (t < n_seqs) {
    const int need = off[t + 1] - off[t];
    const int got = min(need, max(0, found - off[t]));
    if (need > 0) p.held[t] = have[t] + got;
    if (over[t] || got < need) atomicAdd(p.refused, 1);
  }
}

// One workgroup per listed sequence (l.b: the children of a fork).
__global__ __launch_bounds__(1024) void pool_release_kernel(sb_pool p, PoolList l,
                                                            int children,
                                                            int max_pages) {
  const int s = children ? l.b[blockIdx.x] : l.a[blockIdx.x];
  const int n = min(p.held[s], max_pages);
  for (int j = threadIdx.x; j < n; j += 1024) {
    int* e = p.page_table + (size_t)s * max_pages + j;
    atomicAdd(&p.refs[checked_index(*e, p.n_pages, nullptr, kDevPage)], -1);
    *e = -1;
  }
  __syncthreads();
  if (threadIdx.x == 0) p.held[s] = 0;
}

// Workgroup 0 takes the pages for the copies; workgroup 1 + i shares the full
// pages of pair i.  (A shared page's count is at least 1 throughout, so the
// search for free pages does not depend on the sharing.)
__global__ __launch_bounds__(1024) void pool_fork_kernel(sb_pool p, PoolList l,
                                                         const int* __restrict__ len,
                                                         int max_pages) {
  __shared__ __attribute__((aligned(8))) int cnt[128], off[65], full[64];
  const int t = threadIdx.x;
  auto length = [&](int i) {
    const int s = l.a[i];
    return min(max(len[s], 0), min(max(p.held[s], 0), max_pages) * 16);
  };
  if (blockIdx.x > 0) {
    const int i = blockIdx.x - 1, n = length(i) >> 4;
    const int* from = p.page_table + (size_t)l.a[i] * max_pages;
    int* to = p.page_table + (size_t)l.b[i] * max_pages;
    for (int j = t; j < n; j += 1024) {
      const int pg = from[j];
      to[j] = pg;
      atomicAdd(&p.refs[checked_index(pg, p.n_pages, nullptr, kDevPage)], 1);
    }
    return;
  }
  if (t < 64) {
    int need = 0;
    if (t < l.n) {
      const int L = length(t);
      full[t] = L >> 4;
      need = (L & 15) != 0;
    }
    const unsigned long long m = __ballot(need != 0);
    off[t] = (int)__builtin_amdgcn_mbcnt_hi(
        (unsigned)(m >> 32), __builtin_amdgcn_mbcnt_lo((unsigned)m, 0u));
    if (t == 0) off[64] = __popcll(m);
  }
  __syncthreads();
  const int total = off[64];
  int* scr = p.scratch;
  const int found = take_pages(p, total, cnt, [&](int pg, int rank) {
    // the pair that asks for its rank-th page: the last i with off[i] == rank
    const int i = request_of(off, l.n, rank);
    const int src = checked_index(p.page_table[(size_t)l.a[i] * max_pages + full[i]],
                                  p.n_pages, nullptr, kDevPage);
    p.page_table[(size_t)l.b[i] * max_pages + full[i]] = pg;
    p.refs[pg] = 1;
    scr[src_at() + rank] = src;
    scr[dst_at(p.n_pages) + rank] = pg;
  });
  if (t == 0) scr[0] = found;
  if (t < l.n) {
    const int need = (t + 1 < 64 ? off[t + 1] : total) - off[t];
    const bool got = need != 0 && off[t] < found;
    p.held[l.b[t]] = full[t] + (got ? 1 : 0);
    if (need != 0 && !got) atomicAdd(p.refused, 1);
  }
}

// Copies the listed pages in every layer of the caches, a (page, layer) of K
// and V at a time: 32 KiB in an 8-bit cache of 8 x 128 heads, eight 16-byte
// loads a thread before the first store, past the caches (954 MB read and
// written: 209 us through them, 196 past them, means of three runs of each in
// turn; a plain copy of as much takes 203).  moved: the counts and new numbers
// of the pages are set, too.
__global__ __launch_bounds__(256) void pool_copy_kernel(sb_pool p, PoolRegions rg,
                                                        int units, int moved) {
  const int n = p.scratch[0];
  const int* src = p.scratch + src_at();
  const int* dst = p.scratch + dst_at(p.n_pages);
  const long long total = (long long)n * units;
  for (long long u = blockIdx.x; u < total; u += gridDim.x) {
    const int i = (int)(u / units);
    int k = (int)(u - (long long)i * units);
    const int a = src[i], b = dst[i];
    if (moved && k == 0 && threadIdx.x == 0) {
      p.scratch[map_at(p.n_pages) + a] = b;
      p.refs[b] = p.refs[a];
      p.refs[a] = 0;
    }
    if (rg.n == 0) continue;
    const bool second = k >= rg.r[0].n_layers;
    if (second) k -= rg.r[0].n_layers;
    const PoolRegion g = second ? rg.r[1] : rg.r[0];
    const size_t layer = (size_t)k * p.n_pages;
    const int m = (int)(g.page_bytes >> 4);
    const u32x4* ks = reinterpret_cast<const u32x4*>(g.k) + (layer + a) * m;
    const u32x4* vs = reinterpret_cast<const u32x4*>(g.v) + (layer + a) * m;
    u32x4* kd = reinterpret_cast<u32x4*>(g.k) + (layer + b) * m;
    u32x4* vd = reinterpret_cast<u32x4*>(g.v) + (layer + b) * m;
    for (int e = threadIdx.x; e < m; e += 1024) {
      u32x4 x[4], y[4];
#pragma unroll
      for (int j = 0; j < 4; ++j) {
        const int c = min(e + 256 * j, m - 1);
        x[j] = __builtin_nontemporal_load(ks + c);
        y[j] = __builtin_nontemporal_load(vs + c);
      }
#pragma unroll
      for (int j = 0; j < 4; ++j) {
        const int c = e + 256 * j;
        if (c < m) {
          __builtin_nontemporal_store(x[j], kd + c);
          __builtin_nontemporal_store(y[j], vd + c);
        }
      }
    }
    if (g.exp_bytes > 0 && (int)threadIdx.x < 2 * g.exp_bytes) {
      const int h = (int)threadIdx.x % g.exp_bytes;
      uint8_t* x = (int)threadIdx.x < g.exp_bytes ? g.k_exp : g.v_exp;
      x[(layer + b) * g.exp_bytes + h] = x[(layer + a) * g.exp_bytes + h];
    }
  }
}

__global__ __launch_bounds__(1024) void pool_count_kernel(sb_pool p) {
  __shared__ __attribute__((aligned(8))) int cnt[128];
  const int n = walk_chunk(
      blockIdx.x * kChunk, p.n_pages, 0, cnt, [&](int pg) { return p.refs[pg] > 0; },
      [](int, int) {});
  if (threadIdx.x == 0) p.scratch[kCounts + blockIdx.x] = n;
}

// Lists the pages in use at or above their number n, and the free ones below.
__global__ __launch_bounds__(1024) void pool_moves_kernel(sb_pool p) {
  __shared__ __attribute__((aligned(8))) int cnt[128], red[3];
  const int t = threadIdx.x, nb = gridDim.x, base = blockIdx.x * kChunk;
  if (t < 3) red[t] = 0;
  __syncthreads();
  if (t < nb) {
    const int c = p.scratch[kCounts + t];
    atomicAdd(&red[0], c);
    if (t < (int)blockIdx.x) atomicAdd(&red[1], c);
  }
  __syncthreads();
  const int n = red[0], before = red[1];      // in use; in use below this chunk
  // in use below page n
  const int bb = n / kChunk;
  if (t < min(bb, nb)) atomicAdd(&red[2], p.scratch[kCounts + t]);
  int some = 0;
#pragma unroll
  for (int j = 0; j < kChunk / 1024; ++j) {
    const int pg = bb * kChunk + j * 1024 + t;
    some += __popcll(__ballot(pg < min(n, p.n_pages) && p.refs[pg] > 0));
  }
  if ((t & 63) == 0) atomicAdd(&red[2], some);
  __syncthreads();
  const int low = red[2];
  int* src = p.scratch + src_at();
  int* dst = p.scratch + dst_at(p.n_pages);
  int* map = p.scratch + map_at(p.n_pages);
  if (blockIdx.x == 0 && t == 0) p.scratch[0] = n - low;
  for (int j = 0; j < kChunk / 1024; ++j) {
    const int pg = base + j * 1024 + t;
    if (pg < p.n_pages) map[pg] = pg;
  }
  walk_chunk(
      base, p.n_pages, before, cnt, [&](int pg) { return p.refs[pg] > 0; },
      [&](int pg, int rank) {
        if (pg >= n) src[rank - low] = pg;
      });
  walk_chunk(
      base, p.n_pages, base - before, cnt, [&](int pg) { return p.refs[pg] <= 0; },
      [&](int pg, int rank) {
        if (pg < n) dst[rank] = pg;
      });
}

__global__ __launch_bounds__(256) void pool_tables_kernel(sb_pool p, int max_pages) {
  const int s = blockIdx.y, j = blockIdx.x * 256 + threadIdx.x;
  if (j >= min(p.held[s], max_pages)) return;
  int* e = p.page_table + (size_t)s * max_pages + j;
  *e = p.scratch[map_at(p.n_pages) + checked_index(*e, p.n_pages, nullptr, kDevPage)];
}

void copy_pages(const sb_pool& p, const PoolRegions& rg, int most, bool moved,
                hipStream_t st) {
  int units = 0;
  for (int r = 0; r < rg.n; ++r) units += rg.r[r].n_layers;
  if (units == 0) {
    if (!moved) return;
    units = 1;
  }
  const long long total = (long long)most * units;
  pool_copy_kernel<<<(int)std::min<long long>(total, 4096), 256, 0, st>>>(
      p, rg, units, moved ? 1 : 0);
}

}  // namespace

void launch_pool_reset(const sb_pool& p, int max_seqs, int max_pages,
                       hipStream_t st) {
  const size_t n = std::max((size_t)max_seqs * max_pages, (size_t)p.n_pages);
  pool_reset_kernel<<<(int)std::min<size_t>((n + 1023) / 1024, 1024), 1024, 0, st>>>(
      p, max_seqs, max_pages);
}
void launch_pool_grow(const sb_pool& p, int n_seqs, const int* len, int extra,
                      int max_pages, hipStream_t st) {
  pool_grow_kernel<<<1, 1024, 0, st>>>(p, n_seqs, len, extra, max_pages);
}
void launch_pool_release(const sb_pool& p, const PoolList& l, bool children,
                         int max_pages, hipStream_t st) {
  pool_release_kernel<<<l.n, 1024, 0, st>>>(p, l, children ? 1 : 0, max_pages);
}
void launch_pool_fork(const sb_pool& p, const PoolList& l, const int* len,
                      const PoolRegions& rg, int max_pages, hipStream_t st) {
  launch_pool_release(p, l, true, max_pages, st);
  pool_fork_kernel<<<1 + l.n, 1024, 0, st>>>(p, l, len, max_pages);
  copy_pages(p, rg, l.n, false, st);
}
void launch_pool_compact(const sb_pool& p, const PoolRegions& rg, int max_seqs,
                         int max_pages, hipStream_t st) {
  const int nb = (p.n_pages + kChunk - 1) / kChunk;
  pool_count_kernel<<<nb, 1024, 0, st>>>(p);
  pool_moves_kernel<<<nb, 1024, 0, st>>>(p);
  copy_pages(p, rg, std::max(1, p.n_pages / 2), true, st);
  pool_tables_kernel<<<dim3((max_pages + 255) / 256, max_seqs), 256, 0, st>>>(
      p, max_pages);
}

}  // namespace sb

extern "C" size_t sb_pool_scratch_ints(int32_t n_pages) {
  if (n_pages < 1 || n_pages > (1 << 20)) return 0;
  return sb::map_at(n_pages) + (size_t)n_pages;
}
