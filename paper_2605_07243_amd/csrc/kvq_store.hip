// Storing into the 8-bit K/V cache (gfx950): entries of an elem cache, or the
// accepted nodes of a verified tree.
//
// A wave owns the K or the V block of one (layer, page, KV head): 16 x hd
// values.  It finds the largest finite |x| of the entries that it stores,
// takes the least exponent e with |x| <= 448 2^e (bit arithmetic on the fp32
// value: 448 = 1.75 * 2^8), at least the page's own where it holds earlier
// entries, and writes x 2^-e as e4m3, ties to even.  The products with powers of
// two are exact, so the call rounds a value once.  Held codes follow a risen
// exponent: those that stay at or above the least normal code exactly, the others
// rounded to the new scale's 2^-9 2^e steps; over any number of rises a held value
// is within 2^-4 |x| + 2^-9 2^e of what was stored.
//
// HBM bound: es + 1 bytes per value.  The loads of a wave cover whole
// contiguous runs (K: 1 KiB per instruction; V: lane (a, r) reads slots 4 a ..
// 4 a + 3 of column 16 c + r, 512 B per instruction for bf16), and V's stores
// are hd / 4 consecutive bytes a lane.  16 prompts of 512 to 2048 entries in 8
// layers of 8 x 128 heads: 183-208 us, 4.8 to 5.5 TB/s.  The few entries of one
// iteration (16 sequences, 32 layers) take 13 us: a launch and the chain
// bounds -> page -> scale and codes, each step a trip to memory.
#include <algorithm>

#include "bounds.h"
#include "common.h"
#include "kernels.h"
#include "kvq.h"

namespace sb {
namespace {

typedef uint32_t u32x4 __attribute__((ext_vector_type(4)));
typedef uint32_t u32x2 __attribute__((ext_vector_type(2)));
typedef uint16_t u16x2 __attribute__((ext_vector_type(2)));
typedef short s16x2 __attribute__((ext_vector_type(2)));

// Four values as they are stored.  top: the largest bits of |x|, non-finite
// ones included (bf16: of even and odd values, as halves); code: e4m3 of
// x / scale, ties to even, what is not finite as NaN (v_cvt_scalef32_pk_fp8:
// two values an instruction; checked exact for every bf16 value and the scale
// range in use).
template <typename T> struct Quad;
template <> struct Quad<bf16_t> {
  u32x2 w;
  __device__ __forceinline__ void set(int e, bf16_t v) {
    w[e >> 1] |= (uint32_t)v << (16 * (e & 1));
  }
  __device__ __forceinline__ void keep(uint32_t use) {
    w[0] &= (use & 1u ? 0xFFFFu : 0u) | (use & 2u ? 0xFFFF0000u : 0u);
    w[1] &= (use & 4u ? 0xFFFFu : 0u) | (use & 8u ? 0xFFFF0000u : 0u);
  }
  __device__ __forceinline__ static uint32_t join(uint32_t a, uint32_t b) {
    return __builtin_bit_cast(uint32_t,
                              __builtin_elementwise_max(__builtin_bit_cast(u16x2, a),
                                                        __builtin_bit_cast(u16x2, b)));
  }
  __device__ __forceinline__ uint32_t top(uint32_t t) const {
    return join(t, join(w[0] & 0x7FFF7FFFu, w[1] & 0x7FFF7FFFu));
  }
  __device__ __forceinline__ static uint32_t bits(uint32_t t) {
    return max(t & 0xFFFFu, t >> 16) << 16;
  }
  __device__ __forceinline__ float at(int e) const {
    return __uint_as_float(e & 1 ? w[e >> 1] & 0xFFFF0000u : w[e >> 1] << 16);
  }
  __device__ __forceinline__ uint32_t code(float scale) const {
    const uint32_t lo = w[0], hi = w[1];   // (an element cannot be bit-cast itself)
    s16x2 r = {0, 0};
    r = __builtin_amdgcn_cvt_scalef32_pk_fp8_bf16(r, __builtin_bit_cast(bf16x2_t, lo),
                                                  scale, false);
    r = __builtin_amdgcn_cvt_scalef32_pk_fp8_bf16(r, __builtin_bit_cast(bf16x2_t, hi),
                                                  scale, true);
    return __builtin_bit_cast(uint32_t, r);
  }
};
template <> struct Quad<float> {
  u32x4 w;
  __device__ __forceinline__ void set(int e, float v) { w[e] = __float_as_uint(v); }
  __device__ __forceinline__ void keep(uint32_t use) {
#pragma unroll
    for (int e = 0; e < 4; ++e)
      if (!((use >> e) & 1u)) w[e] = 0u;
  }
  __device__ __forceinline__ uint32_t top(uint32_t t) const {
#pragma unroll
    for (int e = 0; e < 4; ++e) t = max(t, w[e] & 0x7FFFFFFFu);
    return t;
  }
  __device__ __forceinline__ static uint32_t bits(uint32_t t) { return t; }
  __device__ __forceinline__ float at(int e) const { return __uint_as_float(w[e]); }
  __device__ __forceinline__ uint32_t code(float scale) const {
    s16x2 r = {0, 0};
    r = __builtin_amdgcn_cvt_scalef32_pk_fp8_f32(r, at(0), at(1), scale, false);
    r = __builtin_amdgcn_cvt_scalef32_pk_fp8_f32(r, at(2), at(3), scale, true);
    return __builtin_bit_cast(uint32_t, r);
  }
};

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
  // eight K values of slot t; four V values of slots t .. t + 3 (zeros where
  // none is used)
  __device__ __forceinline__ void k8(const Page& p, int t, int c, int hd,
                                     bool use, Quad<T> (&x)[2]) const {
    x[0] = x[1] = Quad<T>{};
    if (use) {
      const Quad<T>* q = reinterpret_cast<const Quad<T>*>(p.k + t * hd + c);
      if constexpr (sizeof(T) == 2) {   // (one 16-byte load)
        const u32x4 w = *reinterpret_cast<const u32x4*>(q);
        x[0].w = w.xy;
        x[1].w = w.zw;
      } else {
        x[0] = q[0];
        x[1] = q[1];
      }
    }
  }
  __device__ __forceinline__ Quad<T> v4(const Page& p, int t, int c,
                                        uint32_t use) const {
    Quad<T> x{};
    if (use) x = *reinterpret_cast<const Quad<T>*>(p.v + c * 16 + t);
    return x;
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
                                     bool use, Quad<T> (&x)[2]) const {
    x[0] = x[1] = Quad<T>{};
    if (!use) return;
    const int sl = slot(p, t);
    const Quad<T>* q = reinterpret_cast<const Quad<T>*>(
        p.k + (sl >> 4) * p.step + (sl & 15) * hd + c);
    x[0] = q[0];
    x[1] = q[1];
  }
  __device__ __forceinline__ Quad<T> v4(const Page& p, int t, int c,
                                        uint32_t use) const {
    Quad<T> x{};
#pragma unroll
    for (int e = 0; e < 4; ++e) {
      if (!((use >> e) & 1u)) continue;
      const int sl = slot(p, t + e);
      x.set(e, p.v[(sl >> 4) * p.step + c * 16 + (sl & 15)]);
    }
    return x;
  }
};

// the least e >= -126 with amax <= 448 * 2^e (bits of amax >= 0, finite)
__device__ __forceinline__ int exponent_for(uint32_t u) {
  const int E = (int)(u >> 23) - 127;
  return max(E - ((u & 0x7FFFFFu) <= 0x600000u ? 8 : 7), -126);
}
// held codes over 2^n (scale = 2^n, n >= 0), rounded again
__device__ __forceinline__ uint32_t lower4(uint32_t w, float scale) {
  const auto lo = __builtin_amdgcn_cvt_pk_f32_fp8(w, false);
  const auto hi = __builtin_amdgcn_cvt_pk_f32_fp8(w, true);
  s16x2 r = {0, 0};
  r = __builtin_amdgcn_cvt_scalef32_pk_fp8_f32(r, lo[0], lo[1], scale, false);
  r = __builtin_amdgcn_cvt_scalef32_pk_fp8_f32(r, hi[0], hi[1], scale, true);
  return __builtin_bit_cast(uint32_t, r);
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
  const int task = blockIdx.x * 4 + __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
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
  const int pg = page_to_store(dst.page_table[(size_t)s * max_pages + j],
                               dst.n_pages, err, kDevPage);
  if (pg < 0) return;
  const size_t block = ((size_t)l * dst.n_pages + pg) * Hkv + kh;
  uint8_t* code = (is_v ? dst.v : dst.k) + block * 16 * HD;
  uint8_t* expo = (is_v ? dst.v_exp : dst.k_exp) + block;
  const auto page = src.page(l, s, j, kh, Hkv, HD, 0);
  constexpr int NW = HD / 16;      // words of four codes a lane owns
  Quad<T> x[NW];
  const int va = lane >> 4, vr = lane & 15;
  // V: which of the lane's four slots are stored, and which are held; what is
  // there already is loaded with the new values (one round trip)
  const uint32_t use = (fresh >> (4 * va)) & 15u;
  const uint32_t kept = (((1u << t0) - 1u) >> (4 * va)) & 15u;
  const int own = t0 > 0 ? min((int)*expo - 127, 127) : -126;
  u32x4 was[NW / 4];
#pragma unroll
  for (int c = 0; c < NW / 4; ++c) was[c] = u32x4{0, 0, 0, 0};
  if (is_v) {
    if (use != 15u && (use | kept) != 0) {
#pragma unroll
      for (int c = 0; c < NW / 4; ++c)
        was[c] = reinterpret_cast<const u32x4*>(code)[lane * (NW / 4) + c];
    }
#pragma unroll
    for (int c = 0; c < NW; ++c) x[c] = src.v4(page, 4 * va, 16 * c + vr, use);
    if (use != 15u) {
#pragma unroll
      for (int c = 0; c < NW; ++c) x[c].keep(use);
    }
  } else {
#pragma unroll
    for (int i = 0; i < NW / 2; ++i) {
      const int e0 = (i * 64 + lane) * 8, t = e0 / HD;
      Quad<T> y[2];
      src.k8(page, t, e0 % HD, HD, (fresh >> t) & 1u, y);
      x[2 * i] = y[0];
      x[2 * i + 1] = y[1];
    }
  }
  uint32_t top = 0;
#pragma unroll
  for (int c = 0; c < NW; ++c) top = x[c].top(top);
  // (bits of non-negative floats are ordered as integers)
  top = (uint32_t)-wave_min_i(-(int)Quad<T>::bits(top));
  if (top >= 0x7F800000u) {            // what is not finite sets no scale
    uint32_t m = 0;
#pragma unroll
    for (int c = 0; c < NW; ++c)
#pragma unroll
      for (int e = 0; e < 4; ++e) {
        const uint32_t u = __float_as_uint(x[c].at(e)) & 0x7FFFFFFFu;
        m = max(m, u < 0x7F800000u ? u : 0u);
      }
    top = (uint32_t)-wave_min_i(-(int)m);
  }
  const int e = max(exponent_for(top), own);
  const bool rise = t0 > 0 && e > own;
  const float scale = __uint_as_float((uint32_t)(127 + e) << 23);
  const float down = __uint_as_float((uint32_t)(127 + min(e - own, 60)) << 23);
  if (lane == 0) *expo = (uint8_t)(e + 127);
  if (is_v) {
    // groups of four slots without a new value whose codes stay are not touched
    if (use == 0 && (kept == 0 || !rise)) return;
    uint32_t w[NW];
#pragma unroll
    for (int c = 0; c < NW; ++c) w[c] = x[c].code(scale);
    if (use != 15u) {
      const uint32_t mf = byte_mask(use), mh = byte_mask(kept);
#pragma unroll
      for (int c = 0; c < NW; ++c) {
        const uint32_t old = was[c / 4][c % 4];
        const uint32_t h = rise ? lower4(old, down) : old;
        w[c] = (w[c] & mf) | (h & mh) | (old & ~(mf | mh));
      }
    }
#pragma unroll
    for (int c = 0; c < NW / 4; ++c)
      reinterpret_cast<u32x4*>(code)[lane * (NW / 4) + c] =
          u32x4{w[4 * c], w[4 * c + 1], w[4 * c + 2], w[4 * c + 3]};
  } else {
#pragma unroll
    for (int i = 0; i < NW / 2; ++i) {
      const int e0 = (i * 64 + lane) * 8, t = e0 / HD;
      u32x2* o = reinterpret_cast<u32x2*>(code + e0);
      if ((fresh >> t) & 1u) {
        *o = u32x2{x[2 * i].code(scale), x[2 * i + 1].code(scale)};
      } else if (t < t0 && rise) {
        const u32x2 old = *o;
        *o = u32x2{lower4(old[0], down), lower4(old[1], down)};
      }
    }
  }
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
