// Attention over an 8-bit paged K/V cache (gfx950).
//
// Row i of sequence s attends to the cache entries e < T_s with e < sinks or
// e > pos_i - window (window 0: all of them) and to the segment slots whose
// visibility bit is set:  o = sum_e softmax_e(q . k_e / sqrt(hd)) v_e.  Cache
// entries are e4m3 codes times a power of two per page of 16 entries, KV head
// and K / V; the segment is in the element type.
//
// Both products run on the matrix cores in the element type: e4m3 values and
// powers of two are exact in bf16 and fp32, so the codes are converted in
// registers (v_cvt_scalef32_pk_bf16_fp8, two values an instruction) and
// nothing is lost; K's scale is applied to the fp32 scores.  With 16 keys of a
// page as MFMA rows and 16 query vectors as columns, S^T = K Q^T leaves lane
// (r = lane % 16, g = lane / 16) the scores of query r for keys 4 g .. 4 g + 3
// of the page, which is the B operand of O^T += V^T P^T with the keys in that
// order; the V pages are stored so that lane (r, g) finds columns 16 c + r of
// those keys in hd / 4 consecutive bytes, and a K row's quarter g is hd / 4
// consecutive bytes too: two 16-byte loads each for 128-wide heads, straight
// into registers, 2 KiB contiguous per wave.
//
// The softmax reference m moves only when a score exceeds it by 8 (in log2
// units): the probabilities stay below 2^8 and the sums in fp32.  P is rounded
// to bf16 for the bf16 product (2^-9 relative each, averaged over the keys);
// its sum is taken before the rounding, in fp32.
#include <hip/hip_ext.h>

#include <algorithm>

#include "bounds.h"
#include "common.h"
#include "kernels.h"
#include "kvq.h"

namespace sb {
namespace {

// softmax reference of a row that has seen nothing: below every score, and
// finite, so that exp2(score - reference) of a hidden key (-inf) is 0
constexpr float kLow = -3.0e38f;
constexpr float kLog2e = 1.4426950408889634f;
// waves of a workgroup; each takes every kWaves-th tile of 32 keys
constexpr int kWaves = 4;
constexpr int kMaxSplit = 64;

__device__ __forceinline__ float byte_scale(int b) {
  return __uint_as_float(b > 0 ? (uint32_t)b << 23 : 0x00400000u);
}

// Eight values along the contraction from two words of codes.
__device__ __forceinline__ uint32_t cvt2_bf16(uint32_t w, float s, bool hi) {
  return __builtin_bit_cast(
      uint32_t, hi ? __builtin_amdgcn_cvt_scalef32_pk_bf16_fp8(w, s, true)
                   : __builtin_amdgcn_cvt_scalef32_pk_bf16_fp8(w, s, false));
}
__device__ __forceinline__ void cvt8(Frag8<bf16_t>& f, uint32_t w0, float s0,
                                     uint32_t w1, float s1) {
  f.v = make_uint4(cvt2_bf16(w0, s0, false), cvt2_bf16(w0, s0, true),
                   cvt2_bf16(w1, s1, false), cvt2_bf16(w1, s1, true));
}
__device__ __forceinline__ float4 cvt4_f32(uint32_t w, float s) {
  const auto lo = __builtin_amdgcn_cvt_pk_f32_fp8(w, false);
  const auto hi = __builtin_amdgcn_cvt_pk_f32_fp8(w, true);
  return make_float4(lo[0] * s, lo[1] * s, hi[0] * s, hi[1] * s);
}
__device__ __forceinline__ void cvt8(Frag8<float>& f, uint32_t w0, float s0,
                                     uint32_t w1, float s1) {
  f.a = cvt4_f32(w0, s0);
  f.b = cvt4_f32(w1, s1);
}

// P fragment of eight probabilities
__device__ __forceinline__ void pack8(Frag8<bf16_t>& f, const float (&p)[8]) {
  f.v = make_uint4(pack_bf16x2(p[0], p[1]), pack_bf16x2(p[2], p[3]),
                   pack_bf16x2(p[4], p[5]), pack_bf16x2(p[6], p[7]));
}
__device__ __forceinline__ void pack8(Frag8<float>& f, const float (&p)[8]) {
  f.a = make_float4(p[0], p[1], p[2], p[3]);
  f.b = make_float4(p[4], p[5], p[6], p[7]);
}
__device__ __forceinline__ void unpack8(const Frag8<bf16_t>& f, float (&v)[8]) {
  const uint32_t w[4] = {f.v.x, f.v.y, f.v.z, f.v.w};
#pragma unroll
  for (int e = 0; e < 4; ++e) {
    v[2 * e] = __uint_as_float(w[e] << 16);
    v[2 * e + 1] = __uint_as_float(w[e] & 0xFFFF0000u);
  }
}
__device__ __forceinline__ void unpack8(const Frag8<float>& f, float (&v)[8]) {
  v[0] = f.a.x; v[1] = f.a.y; v[2] = f.a.z; v[3] = f.a.w;
  v[4] = f.b.x; v[5] = f.b.y; v[6] = f.b.z; v[7] = f.b.w;
}

// What a hidden key may not do to the rows that do not see it: its probability
// is 0, but 0 times a NaN or an infinity is NaN, and the product takes every
// key for every row.  In a tile that some row does not see whole, such values
// are taken out of the operand, and added to the rows that see their keys: +inf
// and NaN through one product of indicators, -inf and NaN through another.
// (not zero: a value of the fragment has all exponent bits set)
__device__ __forceinline__ uint32_t bad_bits(const Frag8<bf16_t>& f) {
  auto w = [](uint32_t x) { return ((x & 0x7F807F80u) + 0x00800080u) & 0x80008000u; };
  return w(f.v.x) | w(f.v.y) | w(f.v.z) | w(f.v.w);
}
__device__ __forceinline__ uint32_t bad_bits(const Frag8<float>& f) {
  auto w = [](float x) {
    return ((__float_as_uint(x) & 0x7F800000u) + 0x00800000u) & 0x80000000u;
  };
  return w(f.a.x) | w(f.a.y) | w(f.a.z) | w(f.a.w) | w(f.b.x) | w(f.b.y) |
         w(f.b.z) | w(f.b.w);
}
// keeps what follows from being computed ahead of the rare path it is in
__device__ __forceinline__ void pin(Frag8<bf16_t>& f) {
  __asm__ volatile("" : "+v"(f.v.x), "+v"(f.v.y), "+v"(f.v.z), "+v"(f.v.w));
}
__device__ __forceinline__ void pin(Frag8<float>& f) {
  __asm__ volatile("" : "+v"(f.a.x), "+v"(f.a.y), "+v"(f.a.z), "+v"(f.a.w),
                   "+v"(f.b.x), "+v"(f.b.y), "+v"(f.b.z), "+v"(f.b.w));
}
template <typename T>
struct BadParts {
  Frag8<T> up, dn;
};
template <typename T>
__device__ __forceinline__ BadParts<T> take_bad(Frag8<T>& f) {
  float v[8], up[8], dn[8];
  pin(f);
  unpack8(f, v);
#pragma unroll
  for (int e = 0; e < 8; ++e) {
    const uint32_t u = __float_as_uint(v[e]);
    const bool bad = (u & 0x7F800000u) == 0x7F800000u;
    const bool nan = (u & 0x007FFFFFu) != 0;
    const bool neg = (int)u < 0;
    up[e] = bad & (nan | !neg) ? 1.f : 0.f;
    dn[e] = bad & (nan | neg) ? 1.f : 0.f;
    v[e] = bad ? 0.f : v[e];
  }
  pack8(f, v);
  BadParts<T> b;
  pack8(b.up, up);
  pack8(b.dn, dn);
  return b;
}
template <typename T>
__device__ __forceinline__ f32x4_t add_bad(const BadParts<T>& b, uint32_t seen,
                                           f32x4_t acc) {
  float one[8];
#pragma unroll
  for (int e = 0; e < 8; ++e) one[e] = (seen >> e) & 1u ? 1.f : 0.f;
  Frag8<T> fs;
  pack8(fs, one);
  const f32x4_t z = {0.f, 0.f, 0.f, 0.f};
  const f32x4_t nu = mma_16x16x32(b.up, fs, z), nd = mma_16x16x32(b.dn, fs, z);
#pragma unroll
  for (int j = 0; j < 4; ++j) {
    if (nu[j] > 0.f) acc[j] += __builtin_inff();
    if (nd[j] > 0.f) acc[j] -= __builtin_inff();
  }
  return acc;
}
// The pages of one sequence that a group of rows reads, as a list: the sinks'
// pages, then from the first page of the earliest window on.  Tiles (pairs of
// listed pages) full0 .. full1 - 1 hold nothing that any row does not see.
struct Span {
  int nsp, w0;   // sink pages; first page after them
  int n;         // pages
  int full0, full1;
  __device__ __forceinline__ int page(int v) const {
    return v < nsp ? v : v - nsp + w0;
  }
};
__device__ __forceinline__ Span make_span(int T, int sinks, int lo_min, int lo_max) {
  Span s;
  s.nsp = lo_min > 0 ? (min(sinks, T) + 15) >> 4 : 0;
  s.w0 = max(lo_min >> 4, s.nsp);
  s.n = s.nsp + max(0, ((T + 15) >> 4) - s.w0);
  const int whole = s.nsp + max(0, ((lo_max + 15) >> 4) - s.w0);
  s.full0 = (whole + 1) >> 1;
  s.full1 = max(s.full0, (s.nsp + max(0, (T >> 4) - s.w0)) >> 1);
  return s;
}
__device__ __forceinline__ int prefix_of(const QRows& r, const QView& kv, int s) {
  return max(0, min(min(r.prefix_len[s], kv.max_pages * 16), r.max_prefix));
}
// Splits of a sequence with T entries (the same in the merge).
__device__ __forceinline__ int splits_of(const QRows& r, int T, int n_split,
                                         int split_tokens) {
  if (r.window > 0) T = (int)min((long long)T, (long long)r.window + r.sinks + 32);
  return max(1, min(n_split, (T + split_tokens - 1) / split_tokens));
}
__device__ __forceinline__ void rows_of(const QRows& r, int s, int& row0, int& n) {
  row0 = max(0, min(r.row_off[s], r.n_rows));
  const int row1 = max(row0, min(r.row_off[s + 1], r.n_rows));
  n = min(row1 - row0, r.rows_per_seq);
}
__device__ __forceinline__ int wave_max_i(int v) { return -wave_min_i(-v); }

// A workgroup: QT tiles of 16 query vectors of one KV head, one split of the
// prefix; the last split also takes the segment.  Each of the four waves holds
// all of the workgroup's queries and takes every fourth tile of 32 keys (no
// barrier in the loop), one tile of loads ahead; their (O, m, l) meet in LDS at
// the end.  A tile's codes are converted once for the QT query tiles.
template <typename T, int HD, int QT>
__global__ __launch_bounds__(kWaves * 64, 2) void kvq_attn_kernel(
    const T* __restrict__ q, QRows r, QView kv, int H, int Hkv, int n_split,
    int split_tokens, float scale, float* __restrict__ o_part,
    float* __restrict__ ml, T* __restrict__ out) {
  constexpr int NK = HD / 32;          // contraction steps of a score
  constexpr int NC = HD / 16;          // output column blocks
  constexpr int W4 = HD / 64;          // 16-byte loads per page half
  constexpr int LDO = HD + 4;
  __shared__ __attribute__((aligned(16))) float osh[kWaves][16][LDO];
  __shared__ float msh[QT][kWaves][16], lsh[QT][kWaves][16];
  int bx = blockIdx.x, by = blockIdx.y, bz = blockIdx.z;
  {
    // the query groups of a split on one XCD: they read the same pages
    const int gx = gridDim.x, gz = gridDim.z;
    const int l = xcd_grouped(bx + gx * (by + (int)gridDim.y * bz),
                              gx * (int)gridDim.y * gz);
    bx = l % gx;
    bz = (l / gx) % gz;
    by = l / (gx * gz);
  }
  const int s = by / Hkv, kh = by % Hkv, G = H / Hkv;
  int row0, n_rows;
  rows_of(r, s, row0, n_rows);
  const int nq = n_rows * G, q0 = bx * 16 * QT;
  if (q0 >= nq) return;
  const int Tp = prefix_of(r, kv, s);
  const int ns = splits_of(r, Tp, n_split, split_tokens);
  if (bz >= ns) return;
  const int tid = threadIdx.x, lane = tid & 63;
  const int wave = __builtin_amdgcn_readfirstlane(tid >> 6);
  const int c16 = lane & 15, g = lane >> 4;
  int row[QT], lo[QT];
  Frag8<T> qf[QT][NK];
#pragma unroll
  for (int j = 0; j < QT; ++j) {
    const int qv = q0 + 16 * j + c16;
    const bool valid = qv < nq;
    const int rq = valid ? div_small(qv, G) : 0;
    row[j] = row0 + rq;
    const int head = kh * G + (valid ? qv - rq * G : 0);
#pragma unroll
    for (int i = 0; i < NK; ++i) {
      qf[j][i].load(q + ((size_t)row[j] * H + head) * HD + g * (HD / 4) + 8 * i);
      if (!valid) qf[j][i].zero();
    }
    // first entry of the row's window
    lo[j] = 0;
    if (r.window > 0)
      lo[j] = (int)max(0LL, min((long long)r.pos[row[j]] - (r.window - 1), (long long)Tp));
  }
  int lo_min = 0, lo_max = 0;
  if (r.window > 0) {
    lo_min = lo_max = lo[0];
#pragma unroll
    for (int j = 1; j < QT; ++j) {
      lo_min = min(lo_min, lo[j]);
      lo_max = max(lo_max, lo[j]);
    }
    lo_min = __builtin_amdgcn_readfirstlane(wave_min_i(lo_min));
    lo_max = __builtin_amdgcn_readfirstlane(wave_max_i(lo_max));
    if (lo_max <= r.sinks) {     // the sinks reach into every window
      lo_min = lo_max = 0;
#pragma unroll
      for (int j = 0; j < QT; ++j) lo[j] = 0;
    }
  }
  const Span sp = make_span(Tp, r.sinks, lo_min, lo_max);
  const int* ptab = kv.page_table + (size_t)s * kv.max_pages;
  const int tiles = (sp.n + 1) >> 1, per = (tiles + ns - 1) / ns;
  const int t0 = bz * per, t1 = max(t0, min(tiles, t0 + per));
  // this split's whole tiles, and what is left before and after them
  const int f0 = min(max(sp.full0, t0), t1), f1 = max(f0, min(sp.full1, t1));
  scale *= kLog2e;

  float m[QT], l[QT];
  f32x4_t acc[QT][NC];
#pragma unroll
  for (int j = 0; j < QT; ++j) {
    m[j] = kLow;
    l[j] = 0.f;
#pragma unroll
    for (int c = 0; c < NC; ++c) acc[j][c] = f32x4_t{0.f, 0.f, 0.f, 0.f};
  }

  // softmax step: raw scores of the two halves times k0, k1 (> 0) ->
  // probabilities, packed
  auto soften = [&](f32x4_t (&sc)[QT][2], float k0, float k1, Frag8<T> (&pf)[QT]) {
    // (compared with the raw scores: a maximum of matrix results costs two
    // instructions each; the border need not be exact)
    const float r0 = __builtin_amdgcn_rcpf(k0), r1 = __builtin_amdgcn_rcpf(k1);
    bool up = false;
#pragma unroll
    for (int j = 0; j < QT; ++j) {
      const float b0 = (m[j] + 8.f) * r0, b1 = (m[j] + 8.f) * r1;
#pragma unroll
      for (int e = 0; e < 4; ++e) up |= (sc[j][0][e] > b0) | (sc[j][1][e] > b1);
    }
    if (__ballot(up) != 0) {
#pragma unroll
      for (int j = 0; j < QT; ++j) {
        const float mx = fmaxf(
            k0 * fmaxf(fmaxf(sc[j][0][0], sc[j][0][1]), fmaxf(sc[j][0][2], sc[j][0][3])),
            k1 * fmaxf(fmaxf(sc[j][1][0], sc[j][1][1]), fmaxf(sc[j][1][2], sc[j][1][3])));
        const float m2 = fmaxf(m[j], max_x32(max_x16(mx)));
        const float a = __builtin_amdgcn_exp2f(m[j] - m2);
        m[j] = m2;
        l[j] *= a;
#pragma unroll
        for (int c = 0; c < NC; ++c) acc[j][c] *= a;
      }
    }
#pragma unroll
    for (int j = 0; j < QT; ++j) {
      float p[8];
#pragma unroll
      for (int e = 0; e < 8; ++e) {
        p[e] = __builtin_amdgcn_exp2f(
            __builtin_fmaf(sc[j][e >> 2][e & 3], e < 4 ? k0 : k1, -m[j]));
        l[j] += p[e];
      }
      pack8(pf[j], p);
    }
  };

  const size_t page_bytes = (size_t)Hkv * 16 * HD;
  const uint8_t* kbase = kv.k + (size_t)kh * 16 * HD + (size_t)(c16 * 4 + g) * (HD / 4);
  const uint8_t* vbase = kv.v + (size_t)kh * 16 * HD + (size_t)lane * (HD / 4);
  auto load_page = [&](int pg, uint4 (&kd)[W4], uint4 (&vd)[W4]) {
    const uint8_t* kp = kbase + (size_t)pg * page_bytes;
    const uint8_t* vp = vbase + (size_t)pg * page_bytes;
#pragma unroll
    for (int j = 0; j < W4; ++j) {
      kd[j] = *reinterpret_cast<const uint4*>(kp + 16 * j);
      vd[j] = *reinterpret_cast<const uint4*>(vp + 16 * j);
    }
  };

  // whole tiles, 32 of this wave's at a time: lane 2 n + h holds page h of
  // tile n
  uint4 kr[2][2][W4], vr[2][2][W4];
  for (int n0 = 0; f0 + wave + kWaves * n0 < f1; n0 += 32) {
    const int cnt = min(32, (f1 - f0 - wave + kWaves - 1) / kWaves - n0);
    const int v_l = min(2 * (f0 + wave + kWaves * (n0 + (lane >> 1))) + (lane & 1),
                        sp.n - 1);
    const int pid = checked_index(ptab[sp.page(v_l)], kv.n_pages, kv.err, kDevPage);
    const int ke_l = kv.k_exp[(size_t)pid * Hkv + kh];
    const int ve_l = kv.v_exp[(size_t)pid * Hkv + kh];
    auto issue = [&](int n, uint4 (&kd)[2][W4], uint4 (&vd)[2][W4]) {
#pragma unroll
      for (int h = 0; h < 2; ++h)
        load_page(__builtin_amdgcn_readlane(pid, 2 * n + h), kd[h], vd[h]);
    };
    auto compute = [&](int n, const uint4 (&kd)[2][W4], const uint4 (&vd)[2][W4]) {
      f32x4_t sc[QT][2];
#pragma unroll
      for (int h = 0; h < 2; ++h) {
#pragma unroll
        for (int j = 0; j < QT; ++j) sc[j][h] = f32x4_t{0.f, 0.f, 0.f, 0.f};
        const uint32_t* w = reinterpret_cast<const uint32_t*>(&kd[h][0]);
#pragma unroll
        for (int i = 0; i < NK; ++i) {
          Frag8<T> kf;
          cvt8(kf, w[2 * i], 1.f, w[2 * i + 1], 1.f);
#pragma unroll
          for (int j = 0; j < QT; ++j) sc[j][h] = mma_16x16x32(kf, qf[j][i], sc[j][h]);
        }
      }
      Frag8<T> pf[QT];
      soften(sc, byte_scale(__builtin_amdgcn_readlane(ke_l, 2 * n)) * scale,
             byte_scale(__builtin_amdgcn_readlane(ke_l, 2 * n + 1)) * scale, pf);
      const float vs0 = byte_scale(__builtin_amdgcn_readlane(ve_l, 2 * n));
      const float vs1 = byte_scale(__builtin_amdgcn_readlane(ve_l, 2 * n + 1));
      const uint32_t* w0 = reinterpret_cast<const uint32_t*>(&vd[0][0]);
      const uint32_t* w1 = reinterpret_cast<const uint32_t*>(&vd[1][0]);
#pragma unroll
      for (int c = 0; c < NC; ++c) {
        Frag8<T> vf;
        cvt8(vf, w0[c], vs0, w1[c], vs1);
#pragma unroll
        for (int j = 0; j < QT; ++j) acc[j][c] = mma_16x16x32(vf, pf[j], acc[j][c]);
      }
    };
    issue(0, kr[0], vr[0]);
    for (int n = 0; n < cnt; n += 2) {
      issue(min(n + 1, cnt - 1), kr[1], vr[1]);
      compute(n, kr[0], vr[0]);
      if (n + 1 >= cnt) break;
      issue(min(n + 2, cnt - 1), kr[0], vr[0]);
      compute(n + 1, kr[1], vr[1]);
    }
  }

  // the other tiles: those that some row does not see whole, and, after the
  // last split's share of the prefix, the segment
  const int n_left = f0 - t0, n_pre = n_left + t1 - f1;
  int L = 0;
  if (bz == ns - 1 && kv.seg_pages > 0 && r.vis_words > 0)
    L = max(0, min(min(r.seg_len[s], kv.seg_pages * 16), r.vis_words * 32));
  const int n_gen = n_pre + ((L + 31) >> 5);
  for (int i = (wave + kWaves - (f1 - f0) % kWaves) % kWaves; i < n_gen; i += kWaves) {
    Frag8<T> vf[NC];
    f32x4_t sc[QT][2];
    float ks[2];
    uint32_t seen[QT];
#pragma unroll
    for (int j = 0; j < QT; ++j) {
      seen[j] = 0;
      sc[j][0] = sc[j][1] = f32x4_t{0.f, 0.f, 0.f, 0.f};
    }
    if (i < n_pre) {
      const int v0 = 2 * (i < n_left ? t0 + i : f1 + i - n_left);
      int first[2];                    // entry number of each half
      uint4 kd[2][W4], vd[2][W4];
      float vs[2];
#pragma unroll
      for (int h = 0; h < 2; ++h) {
        const int ap = sp.page(min(v0 + h, sp.n - 1));
        first[h] = v0 + h < sp.n ? ap * 16 : Tp;
        const int pg = checked_index(ptab[ap], kv.n_pages, kv.err, kDevPage);
        load_page(pg, kd[h], vd[h]);
        ks[h] = byte_scale(kv.k_exp[(size_t)pg * Hkv + kh]) * scale;
        vs[h] = byte_scale(kv.v_exp[(size_t)pg * Hkv + kh]);
      }
#pragma unroll
      for (int h = 0; h < 2; ++h) {
        const uint32_t* w = reinterpret_cast<const uint32_t*>(&kd[h][0]);
#pragma unroll
        for (int c = 0; c < NK; ++c) {
          Frag8<T> kf;
          cvt8(kf, w[2 * c], 1.f, w[2 * c + 1], 1.f);
#pragma unroll
          for (int j = 0; j < QT; ++j) sc[j][h] = mma_16x16x32(kf, qf[j][c], sc[j][h]);
        }
      }
      const uint32_t* w0 = reinterpret_cast<const uint32_t*>(&vd[0][0]);
      const uint32_t* w1 = reinterpret_cast<const uint32_t*>(&vd[1][0]);
#pragma unroll
      for (int c = 0; c < NC; ++c) cvt8(vf[c], w0[c], vs[0], w1[c], vs[1]);
#pragma unroll
      for (int j = 0; j < QT; ++j)
#pragma unroll
        for (int e = 0; e < 8; ++e) {
          const int key = first[e >> 2] + 4 * g + (e & 3);
          seen[j] |= (uint32_t)(key < Tp && (key < r.sinks || key >= lo[j])) << e;
        }
    } else {
      const int t = i - n_pre;
      const T* kp[2];
      const T* vp[2];
#pragma unroll
      for (int h = 0; h < 2; ++h) {
        const int pg = min(2 * t + h, kv.seg_pages - 1);
        const size_t at = (((size_t)s * kv.seg_pages + pg) * Hkv + kh) * 16 * HD;
        kp[h] = static_cast<const T*>(kv.seg_k) + at + c16 * HD + g * (HD / 4);
        vp[h] = static_cast<const T*>(kv.seg_v) + at + c16 * 16 + 4 * g;
        ks[h] = scale;
#pragma unroll
        for (int c = 0; c < NK; ++c) {
          Frag8<T> kf;
          kf.load(kp[h] + 8 * c);
#pragma unroll
          for (int j = 0; j < QT; ++j) sc[j][h] = mma_16x16x32(kf, qf[j][c], sc[j][h]);
        }
      }
#pragma unroll
      for (int c = 0; c < NC; ++c) {
        if constexpr (sizeof(T) == 2) {
          const uint2 a = *reinterpret_cast<const uint2*>(vp[0] + 256 * c);
          const uint2 b = *reinterpret_cast<const uint2*>(vp[1] + 256 * c);
          vf[c].v = make_uint4(a.x, a.y, b.x, b.y);
        } else {
          vf[c].a = *reinterpret_cast<const float4*>(vp[0] + 256 * c);
          vf[c].b = *reinterpret_cast<const float4*>(vp[1] + 256 * c);
        }
      }
#pragma unroll
      for (int j = 0; j < QT; ++j) {
        const uint32_t word = r.vis[(size_t)row[j] * r.vis_words + t];
#pragma unroll
        for (int e = 0; e < 8; ++e) {
          const int slot = 16 * (e >> 2) + 4 * g + (e & 3);
          seen[j] |= (uint32_t)(((word >> slot) & 1u) && 32 * t + slot < L) << e;
        }
      }
    }
#pragma unroll
    for (int j = 0; j < QT; ++j)
#pragma unroll
      for (int h = 0; h < 2; ++h)
#pragma unroll
        for (int e = 0; e < 4; ++e)
          sc[j][h][e] = (seen[j] >> (4 * h + e)) & 1u ? sc[j][h][e] : -__builtin_inff();
    Frag8<T> pf[QT];
    soften(sc, ks[0], ks[1], pf);
    uint32_t bad = 0;
#pragma unroll
    for (int c = 0; c < NC; ++c) bad |= bad_bits(vf[c]);
    if (__ballot(bad != 0) != 0) {
#pragma unroll
      for (int c = 0; c < NC; ++c) {
        const BadParts<T> b = take_bad(vf[c]);
#pragma unroll
        for (int j = 0; j < QT; ++j) acc[j][c] = add_bad(b, seen[j], acc[j][c]);
        __builtin_amdgcn_sched_barrier(0);   // (one column block at a time)
      }
    }
#pragma unroll
    for (int c = 0; c < NC; ++c)
#pragma unroll
      for (int j = 0; j < QT; ++j) acc[j][c] = mma_16x16x32(vf[c], pf[j], acc[j][c]);
  }

  // the waves' shares, one query tile after the other
#pragma unroll
  for (int j = 0; j < QT; ++j) {
    l[j] = sum_x32(sum_x16(l[j]));
    if (g == 0) {
      msh[j][wave][c16] = m[j];
      lsh[j][wave][c16] = l[j];
    }
  }
  const int qj = tid >> 4, part16 = tid & 15;
#pragma unroll
  for (int j = 0; j < QT; ++j) {
    if (q0 + 16 * j >= nq) break;      // uniform
    if (j > 0) __syncthreads();
#pragma unroll
    for (int c = 0; c < NC; ++c)
      *reinterpret_cast<float4*>(&osh[wave][c16][16 * c + 4 * g]) =
          make_float4(acc[j][c][0], acc[j][c][1], acc[j][c][2], acc[j][c][3]);
    __syncthreads();
    const int qv = q0 + 16 * j + qj;
    if (qv >= nq) continue;
    float M = kLow, L = 0.f, wt[kWaves];
#pragma unroll
    for (int w = 0; w < kWaves; ++w) M = fmaxf(M, msh[j][w][qj]);
#pragma unroll
    for (int w = 0; w < kWaves; ++w) {
      wt[w] = __builtin_amdgcn_exp2f(msh[j][w][qj] - M);
      L += wt[w] * lsh[j][w][qj];
    }
    const int rq = div_small(qv, G);
    const int orow = row0 + rq, ohead = kh * G + qv - rq * G;
    const float inv = L == 0.f ? 0.f : 1.0f / L;
    const size_t at = (size_t)orow * H + ohead;
#pragma unroll
    for (int e = 0; e < HD / 64; ++e) {
      const int col = part16 * 4 + e * 64;
      float4 o = make_float4(0.f, 0.f, 0.f, 0.f);
#pragma unroll
      for (int w = 0; w < kWaves; ++w) {
        const float4 x = *reinterpret_cast<const float4*>(&osh[w][qj][col]);
        o.x += wt[w] * x.x;
        o.y += wt[w] * x.y;
        o.z += wt[w] * x.z;
        o.w += wt[w] * x.w;
      }
      if (ns > 1) {
        *reinterpret_cast<float4*>(
            o_part + ((size_t)bz * r.n_rows * H + at) * HD + col) = o;
      } else if constexpr (sizeof(T) == 2) {
        *reinterpret_cast<uint2*>(out + at * HD + col) =
            make_uint2(pack_bf16x2(o.x * inv, o.y * inv),
                       pack_bf16x2(o.z * inv, o.w * inv));
      } else {
        *reinterpret_cast<float4*>(out + at * HD + col) =
            make_float4(o.x * inv, o.y * inv, o.z * inv, o.w * inv);
      }
    }
    if (ns > 1 && part16 == 0)
      *reinterpret_cast<float2*>(ml + ((size_t)bz * r.n_rows * H + at) * 2) =
          make_float2(M, L);
  }
}

// Rows of sequences with several splits: o = sum_z w_z O_z / sum_z w_z l_z,
// w_z = 2^(m_z - max m).  Four columns of one head per thread.
template <typename T>
__global__ __launch_bounds__(256) void kvq_merge_kernel(
    QRows r, QView kv, int H, int hd, int n_split, int split_tokens,
    const float* __restrict__ o_part, const float* __restrict__ ml,
    T* __restrict__ out) {
  const int s = blockIdx.z;
  int row0, n_rows;
  rows_of(r, s, row0, n_rows);
  if ((int)blockIdx.y >= n_rows) return;
  const int ns = splits_of(r, prefix_of(r, kv, s), n_split, split_tokens);
  const int c = blockIdx.x * 256 + threadIdx.x;
  if (ns == 1 || c * 4 >= H * hd) return;
  const size_t row = row0 + blockIdx.y;
  const int head = c * 4 / hd;
  const size_t step = (size_t)r.n_rows * H;
  const float2* mlp = reinterpret_cast<const float2*>(ml) + row * H + head;
  const float4* op = reinterpret_cast<const float4*>(o_part) + row * H * hd / 4 + c;
  float M = kLow, L = 0.f;
  float4 o = make_float4(0.f, 0.f, 0.f, 0.f);
#pragma unroll 4
  for (int z = 0; z < ns; ++z) M = fmaxf(M, mlp[z * step].x);
#pragma unroll 4
  for (int z = 0; z < ns; ++z) {
    const float2 e = mlp[z * step];
    const float4 x = op[z * step * hd / 4];
    const float w = __builtin_amdgcn_exp2f(e.x - M);
    L += w * e.y;
    o.x += w * x.x;
    o.y += w * x.y;
    o.z += w * x.z;
    o.w += w * x.w;
  }
  const float inv = L == 0.f ? 0.f : 1.0f / L;
  T* dst = out + row * H * hd + 4 * c;
  if constexpr (sizeof(T) == 2)
    *reinterpret_cast<uint2*>(dst) = make_uint2(
        pack_bf16x2(o.x * inv, o.y * inv), pack_bf16x2(o.z * inv, o.w * inv));
  else
    *reinterpret_cast<float4*>(dst) =
        make_float4(o.x * inv, o.y * inv, o.z * inv, o.w * inv);
}

int cdiv(long a, long b) { return (int)((a + b - 1) / b); }

}  // namespace

// Two query tiles a workgroup where there are more than one (a tile's codes
// are converted once for both: 16 trees of up to 64 nodes 74 -> 49 us, a tree
// of 512 nodes over 8192 entries 179 -> 102; four do not fit the registers: 60
// and 128).  Enough workgroups for two on every CU, cut no shorter than 256
// entries (60 nodes over 1024: 13.5 us, with 128 17.1); beyond that long
// prefixes are cut to 4096 entries so that ragged batches end together.
QPlan kvq_attn_plan(int n_seqs, int rows_per_seq, int max_prefix, int window,
                    int sinks, int H, int Hkv, int hd, int es, int max_split) {
  long eff = max_prefix;
  if (window > 0) eff = std::min(eff, (long)window + sinks + 32);
  const long nq = (long)rows_per_seq * (H / Hkv);
  const int qt = es == 4 || nq <= 16 ? 1 : 2;
  const long items = (long)cdiv(nq, 16 * qt) * n_seqs * Hkv;
  int nz = std::min(cdiv(512, items), std::max(1, (int)(eff / 256)));
  nz = std::max(nz, cdiv(eff, 4096));
  nz = std::max(1, std::min({nz, max_split, kMaxSplit}));
  return QPlan{nz, std::max(32, cdiv(cdiv(eff, nz), 32) * 32), qt};
}

template <typename T>
void launch_kvq_attn(const T* q, const QRows& r, const QView& kv, int H,
                     int Hkv, int hd, const QPlan& plan, float* o_part,
                     float* ml, T* out, hipStream_t st) {
  const float scale = 1.0f / sqrtf((float)hd);
  const dim3 grid(cdiv((long)r.rows_per_seq * (H / Hkv), 16 * plan.qt),
                  r.n_seqs * Hkv, plan.n_split);
  auto k = hd == 128 ? kvq_attn_kernel<T, 128, 1> : kvq_attn_kernel<T, 64, 1>;
  if constexpr (sizeof(T) == 2) {
    if (plan.qt == 2) k = hd == 128 ? kvq_attn_kernel<T, 128, 2> : kvq_attn_kernel<T, 64, 2>;
  }
  // (the profiler's events: start of this kernel, end of the last one)
  hipEvent_t ea, eb;
  attn_take_events(&ea, &eb);
  const bool merge = plan.n_split > 1;
  hipExtLaunchKernelGGL(k, grid, dim3(kWaves * 64), 0, st, ea, merge ? nullptr : eb,
                        0, q, r, kv, H, Hkv, plan.n_split, plan.split_tokens,
                        scale, o_part, ml, out);
  if (merge)
    hipExtLaunchKernelGGL(kvq_merge_kernel<T>,
                          dim3(cdiv(H * hd, 1024), r.rows_per_seq, r.n_seqs),
                          dim3(256), 0, st, nullptr, eb, 0, r, kv, H, hd,
                          plan.n_split, plan.split_tokens, o_part, ml, out);
}

template void launch_kvq_attn<float>(const float*, const QRows&, const QView&,
                                     int, int, int, const QPlan&, float*,
                                     float*, float*, hipStream_t);
template void launch_kvq_attn<bf16_t>(const bf16_t*, const QRows&, const QView&,
                                      int, int, int, const QPlan&, float*,
                                      float*, bf16_t*, hipStream_t);

}  // namespace sb
