// Row-wise kernels around the projections: embedding gather, RMSNorm,
// residual add of split-K partials, RoPE + K/V segment write, SwiGLU, the
// layer-wise shift operand and the drafter input fusion operand.
// One workgroup per call row; the active row count is read on the device.
#include <cmath>

#include "bounds.h"
#include "common.h"
#include "kernels.h"

namespace sb {

// Four consecutive elements of a row as floats (16 B of float, 8 B of bf16).
template <typename T>
__device__ __forceinline__ float4 load4(const T* p);
template <>
__device__ __forceinline__ float4 load4<float>(const float* p) {
  return *reinterpret_cast<const float4*>(p);
}
template <>
__device__ __forceinline__ float4 load4<bf16_t>(const bf16_t* p) {
  const uint2 u = *reinterpret_cast<const uint2*>(p);
  return make_float4(__uint_as_float(u.x << 16), __uint_as_float(u.x & 0xFFFF0000u),
                     __uint_as_float(u.y << 16), __uint_as_float(u.y & 0xFFFF0000u));
}

__device__ __forceinline__ float sumsq4(float4 v) {
  return v.x * v.x + v.y * v.y + v.z * v.z + v.w * v.w;
}

__device__ __forceinline__ float4 scale4(float4 v, float r, float4 g) {
  return make_float4(v.x * r * g.x, v.y * r * g.y, v.z * r * g.z, v.w * r * g.w);
}

// Row kernels below use 1024 threads per row: thread t owns float4 columns
// t and t + 1024 (d <= 8192), loaded before any reduction.
constexpr int kRowThreads = 1024;
constexpr int kRowVec = 2;

template <typename T>
__device__ __forceinline__ void store4(T* p, float4 v);

// x = embedding row of the call row's token, out = rmsnorm(x) * g as T (one
// launch: the row is still in registers when its norm is taken).
template <typename T>
__global__ __launch_bounds__(kRowThreads) void embed_norm_kernel(
    const int* __restrict__ n, const int* __restrict__ tok,
    const T* __restrict__ E, int d, const float* __restrict__ g, float eps,
    float* __restrict__ x, T* __restrict__ out) {
  __shared__ float red[16];
  const int i = blockIdx.x;
  if (i >= *n) return;
  const T* e = E + (size_t)tok[i] * d;
  float4* xr = reinterpret_cast<float4*>(x + (size_t)i * d);
  float4 v[kRowVec], gv[kRowVec];
  float ss = 0.f;
#pragma unroll
  for (int q = 0; q < kRowVec; ++q) {
    const int c = threadIdx.x + q * kRowThreads;
    const bool ok = c < d / 4;
    v[q] = ok ? load4<T>(e + 4 * c) : make_float4(0.f, 0.f, 0.f, 0.f);
    gv[q] = ok ? reinterpret_cast<const float4*>(g)[c]
               : make_float4(0.f, 0.f, 0.f, 0.f);
  }
#pragma unroll
  for (int q = 0; q < kRowVec; ++q) {
    const int c = threadIdx.x + q * kRowThreads;
    if (c < d / 4) xr[c] = v[q];
    ss += sumsq4(v[q]);
  }
  ss = block_sum(ss, red);
  const float r = 1.0f / sqrtf(ss / (float)d + eps);
  T* o = out + (size_t)i * d;
#pragma unroll
  for (int q = 0; q < kRowVec; ++q) {
    const int c = threadIdx.x + q * kRowThreads;
    if (c < d / 4) store4<T>(o + 4 * c, scale4(v[q], r, gv[q]));
  }
}

template <typename T>
void launch_embed_norm(const CallPlan& p, const T* embed, int d,
                       const float* g, float eps, float* x, T* out,
                       hipStream_t st) {
  embed_norm_kernel<T><<<p.cap, kRowThreads, 0, st>>>(p.n, p.token, embed, d,
                                                      g, eps, x, out);
}

template <>
__device__ __forceinline__ void store4<float>(float* p, float4 v) {
  *reinterpret_cast<float4*>(p) = v;
}
template <>
__device__ __forceinline__ void store4<bf16_t>(bf16_t* p, float4 v) {
  uint2 u;
  u.x = pack_bf16x2(v.x, v.y);
  u.y = pack_bf16x2(v.z, v.w);
  *reinterpret_cast<uint2*>(p) = u;
}

__device__ __forceinline__ float4 add4(float4 a, float4 b) {
  return make_float4(a.x + b.x, a.y + b.y, a.z + b.z, a.w + b.w);
}

// sum_{s < ks} P[s] at float4 offset `off` (ks <= 16).  The partials were
// just written by the projection (most reads miss the local L2), so up to
// eight loads are issued before the first add: one memory latency per eight
// partials rather than one per partial.
__device__ __forceinline__ float4 sum_parts(const float* __restrict__ P,
                                            size_t part_stride, int ks,
                                            size_t off) {
  float4 a = make_float4(0.f, 0.f, 0.f, 0.f);
  for (int s0 = 0; s0 < ks; s0 += 8) {
    float4 v[8];
#pragma unroll
    for (int u = 0; u < 8; ++u)
      v[u] = s0 + u < ks
                 ? *reinterpret_cast<const float4*>(P + (s0 + u) * part_stride + off)
                 : make_float4(0.f, 0.f, 0.f, 0.f);
#pragma unroll
    for (int u = 0; u < 8; ++u) a = add4(a, v[u]);
  }
  return a;
}

// The same for two offsets at once (sixteen loads in flight).
__device__ __forceinline__ void sum_parts2(const float* __restrict__ P,
                                           size_t part_stride, int ks,
                                           size_t off_a, size_t off_b,
                                           float4& a, float4& b) {
  a = make_float4(0.f, 0.f, 0.f, 0.f);
  b = a;
  for (int s0 = 0; s0 < ks; s0 += 8) {
    float4 va[8], vb[8];
#pragma unroll
    for (int u = 0; u < 8; ++u) {
      const bool ok = s0 + u < ks;
      const float* q = P + (s0 + u) * part_stride;
      va[u] = ok ? *reinterpret_cast<const float4*>(q + off_a)
                 : make_float4(0.f, 0.f, 0.f, 0.f);
      vb[u] = ok ? *reinterpret_cast<const float4*>(q + off_b)
                 : make_float4(0.f, 0.f, 0.f, 0.f);
    }
#pragma unroll
    for (int u = 0; u < 8; ++u) {
      a = add4(a, va[u]);
      b = add4(b, vb[u]);
    }
  }
}

// One workgroup of 1024 threads per row: thread t owns float4 columns
// t, t + 1024 (d <= 8192), summed over the partials in one pass.
// add_rows != nullptr adds row add_rows[add_idx[i] - 1] (fp32 [.][d]) to
// the partial sum.
// Row grids up to this size issue their loads before the live row count
// arrives (the EARLY forms of residual_kernel and qkv_post_kernel).
constexpr int kEarlyRows = 128;

template <typename T, bool EARLY>
__global__ __launch_bounds__(1024) void residual_kernel(
    const float* __restrict__ P, const int* n, float* __restrict__ x,
    size_t part_stride, int ks, int d, const float* __restrict__ g,
    int accumulate, float eps, T* __restrict__ out, int ldo,
    float* __restrict__ taps, int tap_mask, const int* __restrict__ out_row,
    const float* __restrict__ add_rows, const int* __restrict__ add_idx) {
  constexpr int MAXV = 2;
  __shared__ float red[16];
  const int i = blockIdx.x;
  // EARLY (small grids: few rows, bound by latency): the live row count is
  // waited for only at the exit test further down.  The partial sums, the
  // residual and the gains of row i < grid size are in their buffers
  // whether or not the row is live, so their loads go out together with
  // the count's (one round trip after the kernel boundary instead of two).
  // The count is read with a vector load (the empty asm before it rules out
  // a scalar one, whose wait would also be taken for the kernel arguments
  // read next), older than the partial loads, so the waits for those cover
  // it; the second empty asm keeps the loads, and the test, in their
  // places.  Otherwise (a large grid has many rows past the live count,
  // which then exit before loading anything) the count is tested first.
  int nrows = 0;
  if constexpr (EARLY) {
    __asm__ volatile("" ::: "memory");
    nrows = *n;
  } else {
    if (i >= *n) return;
  }
  float* xr = x + (size_t)i * d;
  const float4* ar = nullptr;
  float* tr = nullptr;
  auto row_extras = [&] {
    if (add_rows != nullptr)
      ar = reinterpret_cast<const float4*>(add_rows + (size_t)(add_idx[i] - 1) * d);
    if (taps != nullptr && tap_mask != 0 && out_row[i] >= 0)
      tr = taps + (size_t)out_row[i] * 3 * d;
  };
  if constexpr (!EARLY) row_extras();
  const int nv = d >> 2;
  float4 v[MAXV];
  float ss = 0.f;
  // the norm gains are loaded with the partials (not after the reduction)
  float4 gv[MAXV];
#pragma unroll
  for (int q = 0; q < MAXV; ++q) {
    const int c = threadIdx.x + q * 1024;
    gv[q] = (g != nullptr && c < nv) ? reinterpret_cast<const float4*>(g)[c]
                                     : make_float4(0.f, 0.f, 0.f, 0.f);
  }
  if (nv > 1024) {
    // second column only where it exists (else a repeat of the first)
    const int c1 = threadIdx.x + 1024 < nv ? threadIdx.x + 1024 : threadIdx.x;
    sum_parts2(P, part_stride, ks, (size_t)i * d + 4 * threadIdx.x,
               (size_t)i * d + 4 * c1, v[0], v[1]);
  } else {
    v[0] = threadIdx.x < nv
               ? sum_parts(P, part_stride, ks, (size_t)i * d + 4 * threadIdx.x)
               : make_float4(0.f, 0.f, 0.f, 0.f);
  }
  float4 xv[MAXV];
  if constexpr (EARLY) {
#pragma unroll
    for (int q = 0; q < MAXV; ++q) {
      const int c = threadIdx.x + q * 1024;
      xv[q] = (accumulate && c < nv) ? reinterpret_cast<const float4*>(xr)[c]
                                     : make_float4(0.f, 0.f, 0.f, 0.f);
    }
    // (the count passes through the asm so that its test, and the wait for
    // it, stay here)
    __asm__ volatile("" : "+v"(nrows)::"memory");
    if (i >= nrows) {   // no load in flight past the end of the program
      __builtin_amdgcn_s_waitcnt(0);
      return;
    }
    row_extras();
  }
#pragma unroll
  for (int q = 0; q < MAXV; ++q) {
    const int c = threadIdx.x + q * 1024;
    if (c < nv) {
      float4 a = v[q];
      if (ar != nullptr) a = add4(a, ar[c]);
      if (accumulate)
        a = add4(a, EARLY ? xv[q] : reinterpret_cast<const float4*>(xr)[c]);
      reinterpret_cast<float4*>(xr)[c] = a;
      if (tr) {
        if (tap_mask & 1) reinterpret_cast<float4*>(tr)[c] = a;
        if (tap_mask & 2) reinterpret_cast<float4*>(tr + d)[c] = a;
        if (tap_mask & 4) reinterpret_cast<float4*>(tr + 2 * d)[c] = a;
      }
      ss += a.x * a.x + a.y * a.y + a.z * a.z + a.w * a.w;
      v[q] = a;
    }
  }
  if (g == nullptr) return;
  ss = block_sum(ss, red);
  const float rs = 1.0f / sqrtf(ss / (float)d + eps);
  T* o = out + (size_t)i * ldo;
#pragma unroll
  for (int q = 0; q < MAXV; ++q) {
    const int c = threadIdx.x + q * 1024;
    if (c < nv) {
      const float4 gg = gv[q];
      store4<T>(o + 4 * c, make_float4(v[q].x * rs * gg.x, v[q].y * rs * gg.y,
                                       v[q].z * rs * gg.z, v[q].w * rs * gg.w));
    }
  }
}

namespace {
thread_local bool g_rows_likely_empty = false;
}  // namespace

void set_rows_likely_empty(bool v) { g_rows_likely_empty = v; }
bool rows_likely_empty() { return g_rows_likely_empty; }

template <typename T>
void launch_residual(float* x, const float* P, int ks, size_t part_stride,
                     const int* n, int cap, int d, bool accumulate,
                     const float* g, float eps, T* out, int ldo, float* taps,
                     int tap_mask, const int* out_row, hipStream_t st,
                     const float* add_rows, const int* add_idx) {
  auto k = cap <= kEarlyRows && !g_rows_likely_empty ? residual_kernel<T, true>
                                                     : residual_kernel<T, false>;
  k<<<cap, 1024, 0, st>>>(P, n, x, part_stride, ks, d, g, accumulate ? 1 : 0,
                          eps, out, ldo, taps, tap_mask, out_row, add_rows,
                          add_idx);
}

// cos and sin of pos theta^(-2t/hd), freq_step = log2(theta) (-2 / hd).  The
// frequency is 2^n (1 + r) with the Taylor series of 2^f, |f| <= 1/2, to
// f^13 (1e-17), and the angle is reduced in double, in revolutions, to an
// eighth of a turn either way; there sine and cosine take the single-precision
// polynomials of Moshier's Cephes library (sinf, cosf).  The library's exp,
// log and sincosf did the same in three times the code, which a launch of
// few rows spends its time fetching.
__device__ __forceinline__ void rope_angle(double pos, double freq_step, int t,
                                           float& c, float& s) {
  const double e = freq_step * (double)t;
  const double n = __builtin_rint(e);
  const double f = (e - n) * 0.693147180559945309417232;   // ln 2
  constexpr double kInvFact[14] = {
      1.0, 1.0, 1.0 / 2, 1.0 / 6, 1.0 / 24, 1.0 / 120, 1.0 / 720, 1.0 / 5040,
      1.0 / 40320, 1.0 / 362880, 1.0 / 3628800, 1.0 / 39916800,
      1.0 / 479001600, 1.0 / 6227020800.0};
  double w = kInvFact[13];
#pragma unroll
  for (int k = 12; k >= 0; --k) w = __builtin_fma(w, f, kInvFact[k]);
  constexpr double kInv2Pi = 0.159154943091895335768884;
  const double rev = pos * (__builtin_amdgcn_ldexp(w, (int)n) * kInv2Pi);
  const double r4 = 4.0 * (rev - __builtin_rint(rev));     // quarter turns
  const double qd = __builtin_rint(r4);
  const float x = (float)((r4 - qd) * 1.570796326794896619231322);
  const int qi = (int)qd & 3;
  const float z = x * x;
  const float sp =
      ((-1.9515295891e-4f * z + 8.3321608736e-3f) * z - 1.6666654611e-1f) * z * x + x;
  const float cp =
      ((2.443315711809948e-5f * z - 1.388731625493765e-3f) * z +
       4.166664568298827e-2f) * z * z - 0.5f * z + 1.0f;
  const float a = (qi & 1) ? cp : sp, b = (qi & 1) ? sp : cp;
  s = (qi & 2) ? -a : a;
  c = (qi == 1 || qi == 2) ? -b : b;
}

// RoPE (rotate-half pairs (j, j + hd/2), angle pos * theta^(-2j/hd)) on the
// Q and K heads of the summed QKV projection; Q -> q [cap][H][hd], K and V ->
// the row's slot of its sequence's segment pages, or, for a prefill pass,
// straight into the row's cache entry (no copy from a segment afterwards, and
// the later pieces of the pass find them there).  Grid (rows, item blocks):
// an item is four rotation pairs of one Q/K head, or four V columns; one
// item per thread, its partials summed in one pass.
template <typename T, bool EARLY>
__global__ __launch_bounds__(256) void qkv_post_kernel(
    const float* __restrict__ P, int ks, size_t part_stride, CallPlan p, int H,
    int Hkv, int hd, double freq_step, T* __restrict__ q, KVView kv) {
  __shared__ __attribute__((aligned(16))) float cs[128];
  __shared__ __attribute__((aligned(16))) float sn[128];
  const int i = blockIdx.x;
  // EARLY: the live row count is waited for only after this thread's
  // partial loads are issued (rows below the grid size are in the partial
  // slabs whether or not they are live), as in residual_kernel
  int nrows = 0;
  if constexpr (EARLY) {
    __asm__ volatile("" ::: "memory");
    nrows = *p.n;
  } else {
    if (i >= *p.n) return;
  }
  const int half = hd >> 1;
  const int q4 = half >> 2;
  const int n_rot = (H + Hkv) * q4;
  const int n_items = n_rot + Hkv * (hd >> 2);
  const int idx = blockIdx.y * blockDim.x + threadIdx.x;
  const int ncol = (H + 2 * Hkv) * hd;
  const size_t row = (size_t)i * ncol;
  float4 a = make_float4(0.f, 0.f, 0.f, 0.f), b = a;
  int head = 0, j = 0;
  if (idx < n_rot) {
    head = div_small(idx, q4);
    j = (idx - head * q4) * 4;
    sum_parts2(P, part_stride, ks, row + head * hd + j,
               row + head * hd + j + half, a, b);
  } else if (idx < n_items) {
    const int v = idx - n_rot;
    head = div_small(v, hd >> 2);
    j = (v - head * (hd >> 2)) * 4;
    a = sum_parts(P, part_stride, ks, row + (H + Hkv) * hd + head * hd + j);
  }
  if constexpr (EARLY) {
    __asm__ volatile("" : "+v"(nrows)::"memory");
    if (i >= nrows) {
      __builtin_amdgcn_s_waitcnt(0);
      return;
    }
  }
  // where the row's K/V go: segment slot and / or cache entry (one outside
  // the page table, or without a page, is not written: a sequence may have
  // outgrown its table or its pool)
  const int seq = p.seq[i];
  T* kseg = nullptr;
  T* vseg = nullptr;
  T* kcache = nullptr;
  T* vcache = nullptr;
  int sl = 0, cl = 0;
  if (p.kv_row == nullptr) {
    const int slot = p.slot[i];
    const size_t page = ((size_t)seq * kv.seg_pages + (slot >> 4)) * Hkv;
    sl = slot & 15;
    kseg = static_cast<T*>(kv.seg_k) + page * 16 * hd;
    vseg = static_cast<T*>(kv.seg_v) + page * 16 * hd;
  }
  if (p.kv_row != nullptr || p.write_through) {
    const int e = p.kv_dst[i];
    if (e >= 0 && (e >> 4) < kv.max_pages) {
      const int pg = page_to_store(kv.page_table[(size_t)seq * kv.max_pages + (e >> 4)],
                                   kv.n_pages, kv.err, kDevPage);
      if (pg >= 0) {
        const size_t page = (size_t)pg * Hkv;
        cl = e & 15;
        kcache = static_cast<T*>(kv.k) + page * 16 * hd;
        vcache = static_cast<T*>(kv.v) + page * 16 * hd;
      }
    }
  }
  const double pos = (double)p.pos[i];
  for (int t = threadIdx.x; t < half; t += blockDim.x)
    rope_angle(pos, freq_step, t, cs[t], sn[t]);
  __syncthreads();
  if (idx < n_rot) {
    const float4 c4 = *reinterpret_cast<const float4*>(&cs[j]);
    const float4 s4 = *reinterpret_cast<const float4*>(&sn[j]);
    const float4 ra = make_float4(a.x * c4.x - b.x * s4.x, a.y * c4.y - b.y * s4.y,
                                  a.z * c4.z - b.z * s4.z, a.w * c4.w - b.w * s4.w);
    const float4 rb = make_float4(b.x * c4.x + a.x * s4.x, b.y * c4.y + a.y * s4.y,
                                  b.z * c4.z + a.z * s4.z, b.w * c4.w + a.w * s4.w);
    if (head < H) {
      T* dst = q + ((size_t)i * H + head) * hd + j;
      store4<T>(dst, ra);
      store4<T>(dst + half, rb);
      return;
    }
    if (kseg != nullptr) {
      T* dst = kseg + ((head - H) * 16 + sl) * hd + j;
      store4<T>(dst, ra);
      store4<T>(dst + half, rb);
    }
    if (kcache != nullptr) {
      T* dst = kcache + ((head - H) * 16 + cl) * hd + j;
      store4<T>(dst, ra);
      store4<T>(dst + half, rb);
    }
  } else if (idx < n_items) {
    const T v[4] = {Elem<T>::from_f32(a.x), Elem<T>::from_f32(a.y),
                    Elem<T>::from_f32(a.z), Elem<T>::from_f32(a.w)};
#pragma unroll
    for (int e = 0; e < 4; ++e) {
      if (vseg != nullptr) vseg[(head * hd + j + e) * 16 + sl] = v[e];
      if (vcache != nullptr) vcache[(head * hd + j + e) * 16 + cl] = v[e];
    }
  }
}

template <typename T>
void launch_qkv_post(const float* P, int ks, size_t part_stride,
                     const CallPlan& p, int H, int Hkv, int hd, float theta,
                     T* q, const KVView& kv, hipStream_t st) {
  const int items = (H + Hkv) * (hd / 8) + Hkv * (hd / 4);
  auto k = p.cap <= kEarlyRows && !g_rows_likely_empty
               ? qkv_post_kernel<T, true>
               : qkv_post_kernel<T, false>;
  k<<<dim3(p.cap, (items + 255) / 256), 256, 0, st>>>(
      P, ks, part_stride, p, H, Hkv, hd,
      std::log2((double)theta) * (-2.0 / (double)hd), q, kv);
}

// out = silu(gate) * up, four columns per thread; grid (rows, F / 1024).
template <typename T>
__global__ __launch_bounds__(256) void swiglu_kernel(
    const float* __restrict__ P, int ks, size_t part_stride,
    const int* __restrict__ n, int F, T* __restrict__ out) {
  const int i = blockIdx.x;
  if (i >= *n) return;
  const int j = (blockIdx.y * 256 + threadIdx.x) * 4;
  if (j >= F) return;
  const size_t row = (size_t)i * 2 * F;
  const float4 gt = sum_parts(P, part_stride, ks, row + j);
  const float4 up = sum_parts(P, part_stride, ks, row + F + j);
  const float4 r = make_float4(gt.x / (1.0f + expf(-gt.x)) * up.x,
                               gt.y / (1.0f + expf(-gt.y)) * up.y,
                               gt.z / (1.0f + expf(-gt.z)) * up.z,
                               gt.w / (1.0f + expf(-gt.w)) * up.w);
  store4<T>(out + (size_t)i * F + j, r);
}

template <typename T>
void launch_swiglu(const float* P, int ks, size_t part_stride, const int* n,
                   int cap, int F, T* out, hipStream_t st) {
  swiglu_kernel<T><<<dim3(cap, (F + 1023) / 1024), 256, 0, st>>>(
      P, ks, part_stride, n, F, out);
}

// Layer-wise shift operand (Eq. 3): [h_k, h_{k-1}] with h_0 := h_1.
template <typename T>
__global__ __launch_bounds__(kRowThreads) void shift_prep_kernel(
    const float* __restrict__ h, const int* __restrict__ n,
    const int* __restrict__ pred, int d, T* __restrict__ out) {
  const int i = blockIdx.x;
  if (i >= *n) return;
  const float4* a = reinterpret_cast<const float4*>(h + (size_t)i * d);
  const float4* b = reinterpret_cast<const float4*>(h + (size_t)pred[i] * d);
  T* o = out + (size_t)i * 2 * d;
  float4 va[kRowVec], vb[kRowVec];
#pragma unroll
  for (int q = 0; q < kRowVec; ++q) {
    const int c = threadIdx.x + q * kRowThreads;
    if (c < d / 4) {
      va[q] = a[c];
      vb[q] = b[c];
    }
  }
#pragma unroll
  for (int q = 0; q < kRowVec; ++q) {
    const int c = threadIdx.x + q * kRowThreads;
    if (c < d / 4) {
      store4<T>(o + 4 * c, va[q]);
      store4<T>(o + d + 4 * c, vb[q]);
    }
  }
}

template <typename T>
void launch_shift_prep(const float* h, const CallPlan& p, int d, T* out,
                       hipStream_t st) {
  shift_prep_kernel<T><<<p.cap, kRowThreads, 0, st>>>(h, p.n, p.pred, d, out);
}

// Drafter input fusion operand (Eq. 2): [norm_c(c), norm_e(embed(x)),
// norm_q(q_k)], each an RMSNorm with its own gain; all three rows are
// loaded at once and their sums of squares reduced together.
// With parts == 2 only [norm_c(c), norm_e(embed(x))] is written (row stride
// 2d): the norm_q(q_k) third is then applied through cached rows (Eq. 2's
// split of W_fuse, see the engine).
template <typename T>
__global__ __launch_bounds__(kRowThreads) void fuse_prep_kernel(
    const float* __restrict__ cond, CallPlan p, const T* __restrict__ E,
    const T* __restrict__ Q, const float* __restrict__ gc,
    const float* __restrict__ ge, const float* __restrict__ gq, float eps,
    int d, T* __restrict__ out, int parts) {
  __shared__ float red[3][16];
  const int i = blockIdx.x;
  if (i >= *p.n) return;
  const int ci = p.cond[i];
  const float4* cr = reinterpret_cast<const float4*>(cond + (size_t)max(ci, 0) * d);
  const T* er = E + (size_t)p.token[i] * d;
  const T* qr = Q + (size_t)(p.k[i] - 1) * d;
  float4 vc[kRowVec], ve[kRowVec], vq[kRowVec];
  float s[3] = {0.f, 0.f, 0.f};
#pragma unroll
  for (int q = 0; q < kRowVec; ++q) {
    const int c = threadIdx.x + q * kRowThreads;
    const bool ok = c < d / 4;
    vc[q] = ok && ci >= 0 ? cr[c] : make_float4(0.f, 0.f, 0.f, 0.f);
    ve[q] = ok ? load4<T>(er + 4 * c) : make_float4(0.f, 0.f, 0.f, 0.f);
    vq[q] = ok ? load4<T>(qr + 4 * c) : make_float4(0.f, 0.f, 0.f, 0.f);
    s[0] += sumsq4(vc[q]);
    s[1] += sumsq4(ve[q]);
    s[2] += sumsq4(vq[q]);
  }
  const int lane = threadIdx.x & 63, w = threadIdx.x >> 6;
#pragma unroll
  for (int j = 0; j < 3; ++j) {
    const float t = wave_sum(s[j]);
    if (lane == 0) red[j][w] = t;
  }
  __syncthreads();
  float r[3];
#pragma unroll
  for (int j = 0; j < 3; ++j) {
    float t = 0.f;
    for (int q = 0; q < (int)(blockDim.x >> 6); ++q) t += red[j][q];
    r[j] = 1.0f / sqrtf(t / (float)d + eps);
  }
  T* o = out + (size_t)i * parts * d;
#pragma unroll
  for (int q = 0; q < kRowVec; ++q) {
    const int c = threadIdx.x + q * kRowThreads;
    if (c < d / 4) {
      // a zero condition stays zero (0 * finite scale)
      store4<T>(o + 4 * c, scale4(vc[q], r[0], reinterpret_cast<const float4*>(gc)[c]));
      store4<T>(o + d + 4 * c, scale4(ve[q], r[1], reinterpret_cast<const float4*>(ge)[c]));
      if (parts == 3)
        store4<T>(o + 2 * d + 4 * c, scale4(vq[q], r[2], reinterpret_cast<const float4*>(gq)[c]));
    }
  }
}

// out[k] = rmsnorm(src[k]) * g as T for the first n rows of src (T rows).
template <typename T>
__global__ __launch_bounds__(kRowThreads) void norm_rows_kernel(
    const T* __restrict__ src, int d, const float* __restrict__ g, float eps,
    T* __restrict__ out) {
  __shared__ float red[16];
  const int i = blockIdx.x;
  const T* sr = src + (size_t)i * d;
  float4 v[kRowVec];
  float ss = 0.f;
#pragma unroll
  for (int q = 0; q < kRowVec; ++q) {
    const int c = threadIdx.x + q * kRowThreads;
    v[q] = c < d / 4 ? load4<T>(sr + 4 * c) : make_float4(0.f, 0.f, 0.f, 0.f);
    ss += sumsq4(v[q]);
  }
  ss = block_sum(ss, red);
  const float r = 1.0f / sqrtf(ss / (float)d + eps);
  T* o = out + (size_t)i * d;
#pragma unroll
  for (int q = 0; q < kRowVec; ++q) {
    const int c = threadIdx.x + q * kRowThreads;
    if (c < d / 4)
      store4<T>(o + 4 * c, scale4(v[q], r, reinterpret_cast<const float4*>(g)[c]));
  }
}

template <typename T>
void launch_norm_rows(const T* src, int n_rows, int d, const float* g,
                      float eps, T* out, hipStream_t st) {
  norm_rows_kernel<T><<<n_rows, kRowThreads, 0, st>>>(src, d, g, eps, out);
}

template <typename T>
void launch_fuse_prep(const float* cond, const CallPlan& p, const T* embed,
                      const T* pos_query, const float* gc, const float* ge,
                      const float* gq, float eps, int d, T* out, int parts,
                      hipStream_t st) {
  fuse_prep_kernel<T><<<p.cap, kRowThreads, 0, st>>>(cond, p, embed, pos_query,
                                                     gc, ge, gq, eps, d, out,
                                                     parts);
}

// out[i] = T(src[idx[i]]) (idx null: identity), rows of w floats; one
// float4 per thread, grid (rows, w / 1024).
template <typename T>
__global__ __launch_bounds__(256) void rows_to_elem_kernel(
    const float* __restrict__ src, const int* __restrict__ idx,
    const int* __restrict__ n, int w, T* __restrict__ out) {
  const int i = blockIdx.x;
  if (i >= *n) return;
  const int c = blockIdx.y * 256 + threadIdx.x;
  if (c >= w / 4) return;
  const float* s = src + (size_t)(idx ? idx[i] : i) * w;
  store4<T>(out + (size_t)i * w + 4 * c, reinterpret_cast<const float4*>(s)[c]);
}

template <typename T>
void launch_rows_to_elem(const float* src, const int* idx, const int* n,
                         int cap, int w, T* out, hipStream_t st) {
  rows_to_elem_kernel<T><<<dim3(cap, (w / 4 + 255) / 256), 256, 0, st>>>(
      src, idx, n, w, out);
}

#define SB_INST(T)                                                             \
  template void launch_embed_norm<T>(const CallPlan&, const T*, int,           \
                                     const float*, float, float*, T*,          \
                                     hipStream_t);                             \
  template void launch_residual<T>(float*, const float*, int, size_t,          \
                                   const int*, int, int, bool, const float*,   \
                                   float, T*, int, float*, int, const int*,    \
                                   hipStream_t, const float*, const int*);     \
  template void launch_norm_rows<T>(const T*, int, int, const float*, float,   \
                                    T*, hipStream_t);                          \
  template void launch_qkv_post<T>(const float*, int, size_t, const CallPlan&, \
                                   int, int, int, float, T*, const KVView&,    \
                                   hipStream_t);                               \
  template void launch_swiglu<T>(const float*, int, size_t, const int*, int,   \
                                 int, T*, hipStream_t);                        \
  template void launch_shift_prep<T>(const float*, const CallPlan&, int, T*,   \
                                     hipStream_t);                             \
  template void launch_fuse_prep<T>(const float*, const CallPlan&, const T*,   \
                                    const T*, const float*, const float*,      \
                                    const float*, float, int, T*, int,         \
                                    hipStream_t);                              \
  template void launch_rows_to_elem<T>(const float*, const int*, const int*,   \
                                       int, int, T*, hipStream_t);
SB_INST(float)
SB_INST(bf16_t)
#undef SB_INST

}  // namespace sb
