// Storing into the 8-bit K/V cache (gfx950): entries of an elem cache, or the
// accepted nodes of a verified tree.
//
// A wave owns the K or the V block of one (layer, page, KV head): 16 x hd
// values.  It finds the largest finite |x| of the entries that it stores,
// takes the least exponent e with |x| <= 448 2^e (bit arithmetic on the fp32
// value: 448 = 1.75 * 2^8), at least the page's own where it holds earlier
// entries, and writes x 2^-e as e4m3, ties to even; held codes follow a risen
// exponent.  The products with powers of two are exact, so a value is rounded
// once, whoever computes it.
//
// HBM bound: es + 1 bytes per value.  The loads of a wave cover whole
// contiguous runs (K: 1 KiB per instruction; V: lane (a, r) reads slots 4 a ..
// 4 a + 3 of column 16 c + r, 512 B per instruction for bf16), and V's stores
// are hd / 4 consecutive bytes a lane.
#include <algorithm>

#include "bounds.h"
#include "common.h"
#include "kernels.h"
#include "kvq.h"

namespace sb {
namespace {

// Entries of a paged elem cache.
template <typename T>
struct CacheSource {
  const T* k;
  const T* v;
  const int* table;      // [n_seqs][max_pages]
  int max_pages;
  int n_pages;
  const int* first;
  const int* last;
  int max_entries;
  // range of entries of sequence s, cut to the table and the host's bound
  __device__ __forceinline__ void range(int s, int& a, int& z) const {
    a = max(first[s], 0);
    z = min(last[s], max_pages * 16);
    if (z > a) z = (int)min((long long)z, (long long)a + max_entries);
  }
  struct Page {
    const T* k;
    const T* v;
  };
  __device__ __forceinline__ Page page(int l, int s, int j, int kh, int Hkv,
                                       int hd, int) const {
    const int pg = checked_index(table[(size_t)s * max_pages + j], n_pages,
                                 nullptr, kDevPage);
    const size_t off = (((size_t)l * n_pages + pg) * Hkv + kh) * 16 * hd;
    return Page{k + off, v + off};
  }
  // eight K values of slot t, four V values of slots t .. t + 3
  __device__ __forceinline__ void k8(const Page& p, int t, int c, int hd,
                                     bool, float (&x)[8]) const {
    Frag8<T> f;
    f.load(p.k + t * hd + c);
    if constexpr (sizeof(T) == 2) {
      const uint32_t w[4] = {f.v.x, f.v.y, f.v.z, f.v.w};
#pragma unroll
      for (int e = 0; e < 4; ++e) {
        x[2 * e] = __uint_as_float(w[e] << 16);
        x[2 * e + 1] = __uint_as_float(w[e] & 0xFFFF0000u);
      }
    } else {
      x[0] = f.a.x; x[1] = f.a.y; x[2] = f.a.z; x[3] = f.a.w;
      x[4] = f.b.x; x[5] = f.b.y; x[6] = f.b.z; x[7] = f.b.w;
    }
  }
  __device__ __forceinline__ void v4(const Page& p, int t, int c, int,
                                     uint32_t, float (&x)[4]) const {
    if constexpr (sizeof(T) == 2) {
      const uint2 w = *reinterpret_cast<const uint2*>(p.v + c * 16 + t);
      x[0] = __uint_as_float(w.x << 16);
      x[1] = __uint_as_float(w.x & 0xFFFF0000u);
      x[2] = __uint_as_float(w.y << 16);
      x[3] = __uint_as_float(w.y & 0xFFFF0000u);
    } else {
      const float4 w = *reinterpret_cast<const float4*>(p.v + c * 16 + t);
      x[0] = w.x; x[1] = w.y; x[2] = w.z; x[3] = w.w;
    }
  }
};

// The root and the accepted nodes of a verified tree: entry T + j is segment
// slot 0 (j = 0) or path[j - 1].
template <typename T>
struct PathSource {
  const T* k;            // [n_layers][pool_seqs][seg_pages] pages
  const T* v;
  int seg_pages;
  int pool_seqs;
  const int* T_old;
  const int* a;
  const int* path;       // [n_seqs][path_cap]
  int path_cap;
  __device__ __forceinline__ void range(int s, int& lo, int& hi) const {
    const int t = T_old[s];
    lo = max(t, 0);
    // (a table's end is the kernel's own bound)
    hi = t < 0 ? 0 : (int)min((long long)t + 1 + min(max(a[s], 0), path_cap),
                              (long long)0x7FFFFFF0);
  }
  struct Page {
    const T* k;
    const T* v;
    const int* path;
    int e0;              // first entry of the page, from T
    size_t step;         // elements per segment page
  };
  __device__ __forceinline__ Page page(int l, int s, int j, int kh, int Hkv,
                                       int hd, int) const {
    const size_t off = (((size_t)l * pool_seqs + s) * seg_pages * Hkv + kh) * 16 * hd;
    return Page{k + off, v + off, path + (size_t)s * path_cap, 16 * j - T_old[s],
                (size_t)Hkv * 16 * hd};
  }
  __device__ __forceinline__ int slot(const Page& p, int t) const {
    const int j = p.e0 + t;
    return min(max(j <= 0 ? 0 : p.path[j - 1], 0), seg_pages * 16 - 1);
  }
  __device__ __forceinline__ void k8(const Page& p, int t, int c, int hd,
                                     bool use, float (&x)[8]) const {
#pragma unroll
    for (int e = 0; e < 8; ++e) x[e] = 0.f;
    if (!use) return;
    const int sl = slot(p, t);
    const T* r = p.k + (sl >> 4) * p.step + (sl & 15) * hd + c;
#pragma unroll
    for (int e = 0; e < 8; ++e) x[e] = Elem<T>::to_f32(r[e]);
  }
  __device__ __forceinline__ void v4(const Page& p, int t, int c, int,
                                     uint32_t use, float (&x)[4]) const {
#pragma unroll
    for (int e = 0; e < 4; ++e) {
      x[e] = 0.f;
      if (!((use >> e) & 1u)) continue;
      const int sl = slot(p, t + e);
      x[e] = Elem<T>::to_f32(p.v[(sl >> 4) * p.step + c * 16 + (sl & 15)]);
    }
  }
};

// |x| for the largest value: infinities and NaN do not set the scale
__device__ __forceinline__ float finite_abs(float x) {
  const float a = fabsf(x);
  return a < __builtin_inff() ? a : 0.f;
}
// the least e >= -126 with amax <= 448 * 2^e
__device__ __forceinline__ int exponent_for(float amax) {
  const uint32_t u = __float_as_uint(amax);
  const int E = (int)(u >> 23) - 127;
  return max(E - ((u & 0x7FFFFFu) <= 0x600000u ? 8 : 7), -126);
}
// four values to codes; what is not finite becomes NaN
__device__ __forceinline__ uint32_t codes4(float a, float b, float c, float d) {
  auto clean = [](float x) {
    return fabsf(x) < __builtin_inff() ? x : __builtin_nanf("");
  };
  int w = __builtin_amdgcn_cvt_pk_fp8_f32(clean(a), clean(b), 0, false);
  return (uint32_t)__builtin_amdgcn_cvt_pk_fp8_f32(clean(c), clean(d), w, true);
}
// held codes times 2^d (d <= 0), rounded again
__device__ __forceinline__ uint32_t lower4(uint32_t w, float f) {
  const auto lo = __builtin_amdgcn_cvt_pk_f32_fp8(w, false);
  const auto hi = __builtin_amdgcn_cvt_pk_f32_fp8(w, true);
  return codes4(lo[0] * f, lo[1] * f, hi[0] * f, hi[1] * f);
}
__device__ __forceinline__ uint32_t byte_mask(uint32_t bits4) {
  return (bits4 & 1u ? 0xFFu : 0u) | (bits4 & 2u ? 0xFF00u : 0u) |
         (bits4 & 4u ? 0xFF0000u : 0u) | (bits4 & 8u ? 0xFF000000u : 0u);
}

template <typename T, int HD, typename Source>
__global__ __launch_bounds__(256) void kvq_store_kernel(Source src, sb_kvq dst,
                                                        int max_pages, int Hkv,
                                                        int* err) {
  const int s = blockIdx.y, l = blockIdx.z;
  const int lane = threadIdx.x & 63;
  const int task = blockIdx.x * 4 + (threadIdx.x >> 6);
  const bool is_v = task & 1;
  const int kh = (task >> 1) % Hkv, jp = (task >> 1) / Hkv;
  int a, z;
  src.range(s, a, z);
  z = min(z, max_pages * 16);
  const long long j64 = (long long)(a >> 4) + jp;
  if (z <= a || j64 * 16 >= z) return;
  const int j = (int)j64;
  // slots t0 .. t1 - 1 of the page are stored, slots below t0 are held
  const int t0 = max(a - 16 * j, 0), t1 = min(z - 16 * j, 16);
  const uint32_t fresh = (t1 >= 16 ? 0xFFFFu : (1u << t1) - 1u) & ~((1u << t0) - 1u);
  const int pg = checked_index(dst.page_table[(size_t)s * max_pages + j],
                               dst.n_pages, err, kDevPage);
  const size_t block = ((size_t)l * dst.n_pages + pg) * Hkv + kh;
  uint8_t* code = (is_v ? dst.v : dst.k) + block * 16 * HD;
  uint8_t* expo = (is_v ? dst.v_exp : dst.k_exp) + block;
  const auto page = src.page(l, s, j, kh, Hkv, HD, 0);
  constexpr int NW = HD / 16;      // words of four codes a lane owns
  float x[NW][4];
  float amax = 0.f;
  const int va = lane >> 4, vr = lane & 15;
  if (is_v) {
    const uint32_t use = (fresh >> (4 * va)) & 15u;
#pragma unroll
    for (int c = 0; c < NW; ++c) src.v4(page, 4 * va, 16 * c + vr, HD, use, x[c]);
#pragma unroll
    for (int c = 0; c < NW; ++c)
#pragma unroll
      for (int e = 0; e < 4; ++e)
        if ((use >> e) & 1u) amax = fmaxf(amax, finite_abs(x[c][e]));
  } else {
#pragma unroll
    for (int i = 0; i < NW / 2; ++i) {
      const int e0 = (i * 64 + lane) * 8, t = e0 / HD;
      float y[8];
      src.k8(page, t, e0 % HD, HD, (fresh >> t) & 1u, y);
#pragma unroll
      for (int e = 0; e < 8; ++e) {
        x[2 * i + (e >> 2)][e & 3] = y[e];
        if ((fresh >> t) & 1u) amax = fmaxf(amax, finite_abs(y[e]));
      }
    }
  }
  amax = wave_max(amax);
  int e = exponent_for(amax), drop = 0;
  if (t0 > 0) {
    const int was = min((int)*expo - 127, 127);
    drop = max(was - e, 0);          // the page's own is the larger one
    e += drop;
    drop = was - e;                  // <= 0: held codes go down by this
  }
  const float f = __uint_as_float((uint32_t)(127 - e) << 23);
  const float g = __uint_as_float((uint32_t)(127 + max(drop, -60)) << 23);
  const bool whole = fresh == 0xFFFFu;
  if (is_v) {
    uint32_t w[NW];
    uint32_t* o = reinterpret_cast<uint32_t*>(code) + lane * NW;
    const uint32_t mf = byte_mask((fresh >> (4 * va)) & 15u);
    const uint32_t mh = byte_mask((((1u << t0) - 1u) >> (4 * va)) & 15u);
#pragma unroll
    for (int c = 0; c < NW; ++c)
      w[c] = codes4(x[c][0] * f, x[c][1] * f, x[c][2] * f, x[c][3] * f);
    if (!whole) {
#pragma unroll
      for (int c = 0; c < NW; ++c) {
        const uint32_t old = o[c];
        const uint32_t h = drop < 0 ? lower4(old, g) : old;
        w[c] = (w[c] & mf) | (h & mh) | (old & ~(mf | mh));
      }
    }
#pragma unroll
    for (int c = 0; c < NW; c += 4)
      *reinterpret_cast<uint4*>(o + c) = make_uint4(w[c], w[c + 1], w[c + 2], w[c + 3]);
  } else {
#pragma unroll
    for (int i = 0; i < NW / 2; ++i) {
      const int e0 = (i * 64 + lane) * 8, t = e0 / HD;
      uint2* o = reinterpret_cast<uint2*>(code + e0);
      if ((fresh >> t) & 1u) {
        const float(&p)[4] = x[2 * i];
        const float(&q)[4] = x[2 * i + 1];
        *o = make_uint2(codes4(p[0] * f, p[1] * f, p[2] * f, p[3] * f),
                        codes4(q[0] * f, q[1] * f, q[2] * f, q[3] * f));
      } else if (t < t0 && drop < 0) {
        const uint2 old = *o;
        *o = make_uint2(lower4(old.x, g), lower4(old.y, g));
      }
    }
  }
  if (lane == 0) *expo = (uint8_t)(e + 127);
}

template <typename T, typename Source>
void launch_store(const Source& src, const sb_kvq& dst, int max_pages, int Hkv,
                  int hd, int n_seqs, int pages, int* err, hipStream_t st) {
  const dim3 grid((pages * Hkv * 2 + 3) / 4, n_seqs, dst.n_layers);
  if (hd == 128)
    kvq_store_kernel<T, 128, Source><<<grid, 256, 0, st>>>(src, dst, max_pages, Hkv, err);
  else
    kvq_store_kernel<T, 64, Source><<<grid, 256, 0, st>>>(src, dst, max_pages, Hkv, err);
}

}  // namespace

template <typename T>
void launch_kvq_store(const T* src_k, const T* src_v, const int* src_table,
                      int src_pages, const sb_kvq& dst, int max_pages,
                      int n_seqs, const int* first, const int* last,
                      int max_entries, int Hkv, int hd, hipStream_t st) {
  const CacheSource<T> src{src_k, src_v, src_table, max_pages, src_pages,
                           first, last, max_entries};
  // a run of n entries touches at most this many pages
  const int pages = (int)std::min<long long>(((long long)max_entries + 30) / 16,
                                             max_pages);
  launch_store<T>(src, dst, max_pages, Hkv, hd, n_seqs, pages, nullptr, st);
}

template <typename T>
void launch_kvq_commit(const T* seg_k, const T* seg_v, int seg_pages,
                       int pool_seqs, const sb_kvq& dst, int max_pages,
                       int n_seqs, const int* T_old, const int* a,
                       const int* path, int path_cap, int Hkv, int hd, int* err,
                       hipStream_t st) {
  const PathSource<T> src{seg_k, seg_v, seg_pages, pool_seqs, T_old, a, path, path_cap};
  launch_store<T>(src, dst, max_pages, Hkv, hd, n_seqs, (path_cap + 1 + 30) / 16,
                  err, st);
}

#define SB_KVQ(T)                                                              \
  template void launch_kvq_store<T>(const T*, const T*, const int*, int,       \
                                    const sb_kvq&, int, int, const int*,       \
                                    const int*, int, int, int, hipStream_t);   \
  template void launch_kvq_commit<T>(const T*, const T*, int, int,             \
                                     const sb_kvq&, int, int, const int*,      \
                                     const int*, const int*, int, int, int,    \
                                     int*, hipStream_t);
SB_KVQ(float)
SB_KVQ(bf16_t)
#undef SB_KVQ

}  // namespace sb
