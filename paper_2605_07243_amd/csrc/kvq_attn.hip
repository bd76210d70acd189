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
// to bf16 for the bf16 product (at most 2^-8 relative each, averaged over the keys);
// its sum is taken before the rounding, in fp32.
//
// What bounds it.  Single tokens: the codes' way from HBM (64 sequences of 4096
// to 32768 entries: 2.4 GB in 413-460 us, 5.3 to 5.9 TB/s; a streaming read
// reaches 6.8).  Trees: every 32 query vectors read all of their KV head's codes from
// L2 and convert them; 500 rows over 8192 entries take 89-95 us (630 TFLOP/s; 49
// for the products alone at a large bf16 product's rate), in which a SIMD's vector
// instructions take 62% of the cycles and its matrix instructions 35%.
// Short prefixes: launch and the chain row bounds -> page table -> codes (a row
// over 1024 entries 9.4 us, of which an empty launch is 5).
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

__device__ __forceinline__ void store4(bf16_t* p, float4 v) {
  *reinterpret_cast<uint2*>(p) =
      make_uint2(pack_bf16x2(v.x, v.y), pack_bf16x2(v.z, v.w));
}
__device__ __forceinline__ void store4(float* p, float4 v) {
  *reinterpret_cast<float4*>(p) = v;
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
// Keys first .. first + 15 that a row sees, a bit each: below T, and below the
// sinks or from lo on.
__device__ __forceinline__ uint32_t page_bits(int first, int T, int sinks, int lo) {
  auto below = [&](int x) { return (1u << min(max(x - first, 0), 16)) - 1u; };
  return below(T) & (below(sinks) | ~below(lo));
}
// Segment slots 32 t .. 32 t + 31 that a row sees, of L > 32 t.
__device__ __forceinline__ uint32_t slot_bits(uint32_t word, int t, int L) {
  return L - 32 * t >= 32 ? word : word & ((1u << (L - 32 * t)) - 1u);
}
__device__ __forceinline__ int wave_max_i(int v) { return -wave_min_i(-v); }

// What a workgroup works on.  The dispatcher deals workgroups out round-robin
// over the 8 XCDs; (sequence, KV head, split) items go round with it, so that
// ragged sequences spread over the chip, and the query groups of an item, which
// read the same pages, follow each other on one XCD.
struct Item {
  int qg, s, kh, z;
};
__device__ __forceinline__ Item item_of(int groups, int n_seqs, int Hkv) {
  const unsigned b = blockIdx.x, y = b >> 3;
  Item i;
  i.qg = (int)(y % (unsigned)groups);
  const unsigned n = y / (unsigned)groups * 8 + (b & 7);
  i.kh = (int)(n % (unsigned)Hkv);
  const unsigned t = n / (unsigned)Hkv;
  i.s = (int)(t % (unsigned)n_seqs);
  i.z = (int)(t / (unsigned)n_seqs);
  return i;
}

// A workgroup: 16 query vectors of one KV head, one split of the prefix; the
// last split also takes the segment.  Each of its NW waves holds all of the
// queries and takes every NW-th tile of 32 keys (no barrier in the loop), one
// tile of loads ahead; their (O, m, l) meet in LDS at the end.
template <typename T, int HD>
__global__ __launch_bounds__(256, 2) void kvq_attn_kernel(
    const T* __restrict__ q, QRows r, QView kv, int groups, int H, int Hkv,
    int n_split, int split_tokens, float scale, float* __restrict__ o_part,
    float* __restrict__ ml, T* __restrict__ out) {
  constexpr int NW = 4;                // waves of a workgroup
  constexpr int NK = HD / 32;          // contraction steps of a score
  constexpr int NC = HD / 16;          // output column blocks
  constexpr int W4 = HD / 64;          // 16-byte loads per page half
  constexpr int LDO = HD + 4;
  __shared__ __attribute__((aligned(16))) float osh[NW][16][LDO];
  __shared__ float msh[NW][16], lsh[NW][16];
  const Item it = item_of(groups, r.n_seqs, Hkv);
  const int s = it.s, kh = it.kh, bz = it.z, G = H / Hkv;
  if (bz >= n_split) return;
  int row0, n_rows;
  rows_of(r, s, row0, n_rows);
  const int nq = n_rows * G, q0 = it.qg * 16;
  if (q0 >= nq) return;
  const int Tp = prefix_of(r, kv, s);
  const int ns = splits_of(r, Tp, n_split, split_tokens);
  if (bz >= ns) return;
  const int tid = threadIdx.x, lane = tid & 63;
  const int wave = __builtin_amdgcn_readfirstlane(tid >> 6);
  const int c16 = lane & 15, g = lane >> 4;
  Frag8<T> qf[NK];
  int row, lo = 0;                     // lo: first entry of the row's window
  {
    const int qv = q0 + c16;
    const bool valid = qv < nq;
    const int rq = valid ? div_small(qv, G) : 0;
    row = row0 + rq;
    const int head = kh * G + (valid ? qv - rq * G : 0);
#pragma unroll
    for (int i = 0; i < NK; ++i) {
      qf[i].load(q + ((size_t)row * H + head) * HD + g * (HD / 4) + 8 * i);
      if (!valid) qf[i].zero();
    }
  }
  int lo_min = 0, lo_max = 0;
  if (r.window > 0) {
    lo = (int)max(0LL, min((long long)r.pos[row] - (r.window - 1), (long long)Tp));
    lo_min = __builtin_amdgcn_readfirstlane(wave_min_i(lo));
    lo_max = __builtin_amdgcn_readfirstlane(wave_max_i(lo));
    // (the sinks reach into every window)
    if (lo_max <= r.sinks) lo = lo_min = lo_max = 0;
  }
  const Span sp = make_span(Tp, r.sinks, lo_min, lo_max);
  const int* ptab = kv.page_table + (size_t)s * kv.max_pages;
  const int tiles = (sp.n + 1) >> 1, per = (tiles + ns - 1) / ns;
  const int t0 = bz * per, t1 = max(t0, min(tiles, t0 + per));
  // this split's whole tiles, and what is left before and after them
  const int f0 = min(max(sp.full0, t0), t1), f1 = max(f0, min(sp.full1, t1));
  scale *= kLog2e;

  float m = kLow, l = 0.f;
  f32x4_t acc[NC];
#pragma unroll
  for (int c = 0; c < NC; ++c) acc[c] = f32x4_t{0.f, 0.f, 0.f, 0.f};

  // softmax step: raw scores of the two halves times k0, k1 (> 0) ->
  // probabilities, packed
  auto soften = [&](f32x4_t (&sc)[2], float k0, float k1, Frag8<T>& pf) {
    // (compared with the raw scores: a maximum of matrix results costs two
    // instructions each; the border need not be exact)
    const float b0 = (m + 8.f) * __builtin_amdgcn_rcpf(k0);
    const float b1 = (m + 8.f) * __builtin_amdgcn_rcpf(k1);
    bool up = false;
#pragma unroll
    for (int e = 0; e < 4; ++e) up |= (sc[0][e] > b0) | (sc[1][e] > b1);
    if (__ballot(up) != 0) {
      const float mx = fmaxf(
          k0 * fmaxf(fmaxf(sc[0][0], sc[0][1]), fmaxf(sc[0][2], sc[0][3])),
          k1 * fmaxf(fmaxf(sc[1][0], sc[1][1]), fmaxf(sc[1][2], sc[1][3])));
      const float m2 = fmaxf(m, max_x32(max_x16(mx)));
      const float a = __builtin_amdgcn_exp2f(m - m2);
      m = m2;
      l *= a;
#pragma unroll
      for (int c = 0; c < NC; ++c) acc[c] *= a;
    }
    float p[8];
#pragma unroll
    for (int e = 0; e < 8; ++e) {
      p[e] = __builtin_amdgcn_exp2f(
          __builtin_fmaf(sc[e >> 2][e & 3], e < 4 ? k0 : k1, -m));
      l += p[e];
    }
    pack8(pf, p);
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
  for (int n0 = 0; f0 + wave + NW * n0 < f1; n0 += 32) {
    const int cnt = min(32, (f1 - f0 - wave + NW - 1) / NW - n0);
    const int v_l = min(2 * (f0 + wave + NW * (n0 + (lane >> 1))) + (lane & 1),
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
      f32x4_t sc[2];
#pragma unroll
      for (int h = 0; h < 2; ++h) {
        sc[h] = f32x4_t{0.f, 0.f, 0.f, 0.f};
        const uint32_t* w = reinterpret_cast<const uint32_t*>(&kd[h][0]);
#pragma unroll
        for (int i = 0; i < NK; ++i) {
          Frag8<T> kf;
          cvt8(kf, w[2 * i], 1.f, w[2 * i + 1], 1.f);
          sc[h] = mma_16x16x32(kf, qf[i], sc[h]);
        }
      }
      Frag8<T> pf;
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
        acc[c] = mma_16x16x32(vf, pf, acc[c]);
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
  for (int i = (wave + NW - (f1 - f0) % NW) % NW; i < n_gen; i += NW) {
    // which keys of the tile the row sees
    uint32_t keys;
    const int v0 = 2 * (i < n_left ? t0 + i : f1 + i - n_left), t = i - n_pre;
    if (i < n_pre) {
      keys = page_bits(sp.page(v0) * 16, Tp, r.sinks, lo);
      if (v0 + 1 < sp.n) keys |= page_bits(sp.page(v0 + 1) * 16, Tp, r.sinks, lo) << 16;
    } else {
      keys = slot_bits(r.vis[(size_t)row * r.vis_words + t], t, L);
    }
    if (__ballot(keys != 0) == 0) continue;
    keys >>= 4 * g;
    const uint32_t seen = (keys & 15) | ((keys >> 12) & 0xF0);   // bit e: key of score e
    Frag8<T> vf[NC];
    f32x4_t sc[2];
    float ks[2];
    sc[0] = sc[1] = f32x4_t{0.f, 0.f, 0.f, 0.f};
    if (i < n_pre) {
      uint4 kd[2][W4], vd[2][W4];
      float vs[2];
#pragma unroll
      for (int h = 0; h < 2; ++h) {
        const int ap = sp.page(min(v0 + h, sp.n - 1));
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
          sc[h] = mma_16x16x32(kf, qf[c], sc[h]);
        }
      }
      const uint32_t* w0 = reinterpret_cast<const uint32_t*>(&vd[0][0]);
      const uint32_t* w1 = reinterpret_cast<const uint32_t*>(&vd[1][0]);
#pragma unroll
      for (int c = 0; c < NC; ++c) cvt8(vf[c], w0[c], vs[0], w1[c], vs[1]);
    } else {
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
          sc[h] = mma_16x16x32(kf, qf[c], sc[h]);
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
    }
#pragma unroll
    for (int h = 0; h < 2; ++h)
#pragma unroll
      for (int e = 0; e < 4; ++e)
        sc[h][e] = (seen >> (4 * h + e)) & 1u ? sc[h][e] : -__builtin_inff();
    Frag8<T> pf;
    soften(sc, ks[0], ks[1], pf);
    uint32_t bad = 0;
#pragma unroll
    for (int c = 0; c < NC; ++c) bad |= bad_bits(vf[c]);
    if (__ballot(bad != 0) != 0) {
#pragma unroll
      for (int c = 0; c < NC; ++c) {
        acc[c] = add_bad(take_bad(vf[c]), seen, acc[c]);
        __builtin_amdgcn_sched_barrier(0);   // (one column block at a time)
      }
    }
#pragma unroll
    for (int c = 0; c < NC; ++c)
      acc[c] = mma_16x16x32(vf[c], pf, acc[c]);
  }

  // the waves' shares
  l = sum_x32(sum_x16(l));
  if (g == 0) {
    msh[wave][c16] = m;
    lsh[wave][c16] = l;
  }
#pragma unroll
  for (int c = 0; c < NC; ++c)
    *reinterpret_cast<float4*>(&osh[wave][c16][16 * c + 4 * g]) =
        make_float4(acc[c][0], acc[c][1], acc[c][2], acc[c][3]);
  __syncthreads();
  constexpr int TPQ = NW * 64 / 16;     // threads of one query vector
  const int qj = tid / TPQ, part = tid % TPQ, qv = q0 + qj;
  if (qv >= nq) return;
  float M = kLow, Lsum = 0.f, wt[NW];
#pragma unroll
  for (int w = 0; w < NW; ++w) M = fmaxf(M, msh[w][qj]);
#pragma unroll
  for (int w = 0; w < NW; ++w) {
    wt[w] = __builtin_amdgcn_exp2f(msh[w][qj] - M);
    Lsum += wt[w] * lsh[w][qj];
  }
  const int rq = div_small(qv, G);
  const float inv = Lsum == 0.f ? 0.f : 1.0f / Lsum;
  const size_t at = (size_t)(row0 + rq) * H + kh * G + qv - rq * G;
#pragma unroll
  for (int col = part * 4; col < HD; col += 4 * TPQ) {
    float4 o = make_float4(0.f, 0.f, 0.f, 0.f);
#pragma unroll
    for (int w = 0; w < NW; ++w) {
      const float4 x = *reinterpret_cast<const float4*>(&osh[w][qj][col]);
      o.x += wt[w] * x.x;
      o.y += wt[w] * x.y;
      o.z += wt[w] * x.z;
      o.w += wt[w] * x.w;
    }
    if (ns > 1)
      *reinterpret_cast<float4*>(
          o_part + ((size_t)bz * r.n_rows * H + at) * HD + col) = o;
    else
      store4(out + at * HD + col, make_float4(o.x * inv, o.y * inv, o.z * inv, o.w * inv));
  }
  if (ns > 1 && part == 0)
    *reinterpret_cast<float2*>(ml + ((size_t)bz * r.n_rows * H + at) * 2) =
        make_float2(M, Lsum);
}

// ---- bf16: 32 query vectors a wave ------------------------------------------
//
// v_mfma_f32_32x32x16_bf16 with 32 keys (two pages) as rows and 32 query vectors
// as columns.  Its 32 cycles leave room for seven vector instructions, which
// the 16x16 form's 16 cycles do not (measured, cycles per SIMD: 8 of the large
// product with 64 FMAs 338, 16 of the small one with 64 FMAs 400, products or
// FMAs alone 274 to 330): conversions and softmax run beside the products.
//
// Lane (r = lane % 32, h = lane / 32) holds half h of key r's K row (hd / 2
// consecutive bytes), and of S^T the scores of query r for keys 4 h .. 4 h + 3
// and 8 + 4 h .. of each page, the B operand of O^T += V^T P^T.  A operand: the
// codes of those keys for columns 32 b + r, i.e. groups a = h and 2 + h of the
// V page; lanes r and r + 16 each load half of the 16 columns' run and swap the
// words that the other needs (v_permlane16_swap).  K is loaded a KiB at a time and
// turned to rows in LDS, each wave its own tiles: with the lanes 64 bytes apart, as
// the operand has them, the loads of K alone took 73 of 90 us (500 rows over 8192
// entries; V's 32).
//
// A workgroup: 32 query vectors of one KV head, one split; its NW waves take
// every NW-th tile, as above.  Two waves a SIMD (the accumulators, the queries
// and two tiles of loads fill the registers).  Bound inside the CU: the same 500
// rows took 90 us, 48 with the loads alone and 70 without them.  Measured while K
// came straight into the operand's registers (93 us then): 64 query vectors a wave 94
// to 108, four waves of other queries on the same tiles 104 to 120, tiles converted
// once for four such waves and shared in LDS 101.
typedef float f32x16_t __attribute__((ext_vector_type(16)));
typedef uint32_t u32x4 __attribute__((ext_vector_type(4)));

__device__ __forceinline__ f32x16_t mma_32x32x16(const Frag8<bf16_t>& a,
                                                 const Frag8<bf16_t>& b,
                                                 f32x16_t acc) {
  return __builtin_amdgcn_mfma_f32_32x32x16_bf16(
      __builtin_bit_cast(bf16x8_t, a.v), __builtin_bit_cast(bf16x8_t, b.v), acc,
      0, 0, 0);
}
__device__ __forceinline__ f32x16_t zero16() {
  f32x16_t z;
#pragma unroll
  for (int i = 0; i < 16; ++i) z[i] = 0.f;
  return z;
}
__device__ __forceinline__ f32x16_t add_bad32(const BadParts<bf16_t>& b,
                                              uint32_t seen8, f32x16_t acc) {
  float one[8];
#pragma unroll
  for (int e = 0; e < 8; ++e) one[e] = (seen8 >> e) & 1u ? 1.f : 0.f;
  Frag8<bf16_t> fs;
  pack8(fs, one);
  const f32x16_t nu = mma_32x32x16(b.up, fs, zero16());
  const f32x16_t nd = mma_32x32x16(b.dn, fs, zero16());
#pragma unroll
  for (int i = 0; i < 16; ++i) {
    if (nu[i] > 0.f) acc[i] += __builtin_inff();
    if (nd[i] > 0.f) acc[i] -= __builtin_inff();
  }
  return acc;
}

template <int HD, int NW>
__global__ __launch_bounds__(NW * 64, 2) void kvq_attn32_kernel(
    const bf16_t* __restrict__ q, QRows r, QView kv, int groups, int H, int Hkv,
    int n_split, int split_tokens, float scale, float* __restrict__ o_part,
    float* __restrict__ ml, bf16_t* __restrict__ out) {
  constexpr int NK = HD / 16;          // contraction steps of a score
  constexpr int NB = HD / 32;          // output column blocks
  constexpr int LDO = HD + 4;
  typedef Frag8<bf16_t> Frag;
  typedef uint32_t vword __attribute__((ext_vector_type(HD / 32)));
  __shared__ __attribute__((aligned(16))) float osh[NW][32][LDO];
  __shared__ float msh[NW][32], lsh[NW][32];
  const Item it = item_of(groups, r.n_seqs, Hkv);
  const int s = it.s, kh = it.kh, bz = it.z, G = H / Hkv;
  if (bz >= n_split) return;
  int row0, n_rows;
  rows_of(r, s, row0, n_rows);
  const int nq = n_rows * G, q0 = it.qg * 32;
  if (q0 >= nq) return;
  const int Tp = prefix_of(r, kv, s);
  const int ns = splits_of(r, Tp, n_split, split_tokens);
  if (bz >= ns) return;
  const int tid = threadIdx.x, lane = tid & 63;
  const int wave = __builtin_amdgcn_readfirstlane(tid >> 6);
  const int c32 = lane & 31, h = lane >> 5;
  Frag qf[NK];
  int row, lo = 0;                     // lo: first entry of the row's window
  {
    const int qv = q0 + c32;
    const bool valid = qv < nq;
    const int rq = valid ? div_small(qv, G) : 0;
    row = row0 + rq;
    const int head = kh * G + (valid ? qv - rq * G : 0);
    const bf16_t* qp = q + ((size_t)row * H + head) * HD + h * (HD / 2);
#pragma unroll
    for (int i = 0; i < NK; ++i) {
      qf[i].load(qp + 8 * i);
      if (!valid) qf[i].zero();
    }
  }
  int lo_min = 0, lo_max = 0;
  if (r.window > 0) {
    lo = (int)max(0LL, min((long long)r.pos[row] - (r.window - 1), (long long)Tp));
    lo_min = __builtin_amdgcn_readfirstlane(wave_min_i(lo));
    lo_max = __builtin_amdgcn_readfirstlane(wave_max_i(lo));
    // (the sinks reach into every window)
    if (lo_max <= r.sinks) lo = lo_min = lo_max = 0;
  }
  const Span sp = make_span(Tp, r.sinks, lo_min, lo_max);
  const int* ptab = kv.page_table + (size_t)s * kv.max_pages;
  const int tiles = (sp.n + 1) >> 1, per = (tiles + ns - 1) / ns;
  const int t0 = bz * per, t1 = max(t0, min(tiles, t0 + per));
  // this split's whole tiles, and what is left before and after them
  const int f0 = min(max(sp.full0, t0), t1), f1 = max(f0, min(sp.full1, t1));
  scale *= kLog2e;

  float m = 0.f, l = 0.f, lim = -__builtin_inff();
  f32x16_t acc[NB];
#pragma unroll
  for (int b = 0; b < NB; ++b) acc[b] = zero16();

  // raw scores of two pages -> score k - m, where the reference m moves when
  // that exceeds `lim` somewhere (k0, k1 > 0: the pages' scales): 8, or anything
  // a row sees while it has no reference yet
  auto refer = [&](f32x16_t& sc, float k0, float k1) {
#pragma unroll
    for (int i = 0; i < 16; ++i) sc[i] = __builtin_fmaf(sc[i], i < 8 ? k0 : k1, -m);
    float top = fmaxf(sc[0], sc[1]);
#pragma unroll
    for (int i = 2; i < 16; i += 2) top = fmaxf(fmaxf(top, sc[i]), sc[i + 1]);
    if (__ballot(top > lim) != 0) {
      const float x = max_x32(top);
      const bool move = x > lim, none = lim < 0.f;
      const float d = move ? (none ? x : fmaxf(x, 0.f)) : 0.f;
      const float a = none ? 1.f : __builtin_amdgcn_exp2f(-d);
      lim = move ? 8.f : lim;
      m += d;
      l *= a;
#pragma unroll
      for (int i = 0; i < 16; ++i) sc[i] -= d;
#pragma unroll
      for (int b = 0; b < NB; ++b) acc[b] *= a;
    }
  };
  // two probabilities, packed
  auto weigh = [&](float x, float y) {
    const float p = __builtin_amdgcn_exp2f(x), q = __builtin_amdgcn_exp2f(y);
    l += p;
    l += q;
    return pack_bf16x2(p, q);
  };
  auto put = [](Frag (&pf)[2], int c, uint32_t w) {   // pair c of 8
    Frag& f = pf[c / 4];
    if (c % 4 == 0) f.v.x = w;
    if (c % 4 == 1) f.v.y = w;
    if (c % 4 == 2) f.v.z = w;
    if (c % 4 == 3) f.v.w = w;
  };

  // a lane's codes: of K 16 bytes of every KiB of the tile (or, after LDS, half
  // a row), of each page of V half the words of groups h and 2 + h
  typedef u32x4 KRaw[HD / 32];
  typedef vword VRaw[2][2];
  const size_t page_bytes = (size_t)Hkv * 16 * HD;
  const uint8_t* kbase = kv.k + (size_t)kh * 16 * HD;
  const uint8_t* vbase = kv.v + (size_t)kh * 16 * HD;
  const uint32_t vlane = (h * 16 + (c32 & 15)) * (HD / 4) + (c32 >> 4) * (HD / 8);
  constexpr int NKL = HD / 32, NVL = 4;   // loads of a K tile, of a V tile
  auto load_k1 = [&](int p0, int p1, int j, KRaw& kq) {
    constexpr int N = HD / 64;         // 1 KiB runs of a page
    kq[j] = *reinterpret_cast<const u32x4*>(
        kbase + (size_t)(j < N ? p0 : p1) * page_bytes + (j % N * 1024 + lane * 16));
  };
  auto load_k = [&](int p0, int p1, KRaw& kq) {
#pragma unroll
    for (int j = 0; j < NKL; ++j) load_k1(p0, p1, j, kq);
  };
  // a K tile goes through LDS to the lanes that need its rows (the wave's own
  // 8 KiB, two tiles): 16-byte chunk c of row r at chunk c ^ r % NC of the row,
  // eight lanes on different banks both ways
  constexpr int NC = HD / 16;          // chunks of a row
  uint8_t* ring = reinterpret_cast<uint8_t*>(&osh[wave][0][0]);
  const int pr = lane / NC, put_at = pr * HD + ((lane % NC) ^ (pr % NC)) * 16;
  const int get_at = c32 * HD + ((h * (NC / 2)) ^ (c32 % NC)) * 16;
  auto put_k = [&](const KRaw& kq, int slot) {
#pragma unroll
    for (int j = 0; j < HD / 32; ++j)
      *reinterpret_cast<u32x4*>(ring + slot * 32 * HD + j * 1024 + put_at) = kq[j];
    wave_lds_sync();
  };
  auto get_k = [&](int slot, KRaw& kq) {
#pragma unroll
    for (int j = 0; j < HD / 32; ++j)
      kq[j] = *reinterpret_cast<const u32x4*>(ring + slot * 32 * HD + (get_at ^ (16 * j)));
  };
  auto load_v1 = [&](int p0, int p1, int j, VRaw& vq) {
    const uint8_t* vp = vbase + (size_t)(j / 2 ? p1 : p0) * page_bytes;
    vq[j / 2][j % 2] = *reinterpret_cast<const vword*>(vp + (vlane + j % 2 * 8 * HD));
  };
  auto load_v = [&](int p0, int p1, VRaw& vq) {
#pragma unroll
    for (int j = 0; j < NVL; ++j) load_v1(p0, p1, j, vq);
  };
  auto k_frag = [&](const KRaw& kq, int i, Frag& f) {
    cvt8(f, kq[i / 2][2 * (i % 2)], 1.f, kq[i / 2][2 * (i % 2) + 1], 1.f);
  };
  auto scores = [&](const KRaw& kq) {
    f32x16_t sc = zero16();
#pragma unroll
    for (int i = 0; i < NK; ++i) {
      Frag kf;
      k_frag(kq, i, kf);
      sc = mma_32x32x16(kf, qf[i], sc);
    }
    return sc;
  };
  // words of the V^T operands of page p: w[b][a], column block b, group h + 2 a
  auto v_words = [&](const VRaw& vq, int p, uint32_t (&w)[NB][2]) {
#pragma unroll
    for (int a = 0; a < 2; ++a) {
      vword v = vq[p][a];
      // (taken apart here and not where a loop begins, which would wait for it)
      __asm__ volatile("" : "+v"(v));
#pragma unroll
      for (int j = 0; j < NB / 2; ++j) {
        const auto x = __builtin_amdgcn_permlane16_swap(v[2 * j], v[2 * j + 1],
                                                        false, false);
        w[j][a] = x[0];
        w[NB / 2 + j][a] = x[1];
      }
    }
  };

  // whole tiles, 64 of this wave's at a time: lane n holds the pages and the
  // four scale bytes of tile n.  The scores of tile n + 1 are formed beside the
  // softmax of tile n; K of tile n + 2 goes to LDS, K of tile n + 4 and V of
  // tile n + 1 are loaded into free registers, a load beside each product.
  KRaw kq[2];
  VRaw vq[2];
  for (int n0 = 0; f0 + wave + NW * n0 < f1; n0 += 64) {
    const int cnt = min(64, (f1 - f0 - wave + NW - 1) / NW - n0);
    int id0, id1;
    uint32_t ex;
    {
      const int v = 2 * (f0 + wave + NW * (n0 + min(lane, cnt - 1)));
      id0 = checked_index(ptab[sp.page(v)], kv.n_pages, kv.err, kDevPage);
      id1 = checked_index(ptab[sp.page(v + 1)], kv.n_pages, kv.err, kDevPage);
      const size_t a0 = (size_t)id0 * Hkv + kh, a1 = (size_t)id1 * Hkv + kh;
      ex = kv.k_exp[a0] | kv.k_exp[a1] << 8 | kv.v_exp[a0] << 16 | (uint32_t)kv.v_exp[a1] << 24;
    }
    // (past the last tile: the last one again)
    auto fetch_k = [&](int n, KRaw& d) {
      n = min(n, cnt - 1);
      load_k(__builtin_amdgcn_readlane(id0, n), __builtin_amdgcn_readlane(id1, n), d);
    };
    fetch_k(0, kq[0]);
    fetch_k(1, kq[1]);
    load_v(__builtin_amdgcn_readlane(id0, 0), __builtin_amdgcn_readlane(id1, 0), vq[0]);
    put_k(kq[0], 0);
    fetch_k(2, kq[0]);
    KRaw kf;
    get_k(0, kf);
    f32x16_t sc = scores(kf);
    put_k(kq[1], 1);
    fetch_k(3, kq[1]);
    // one tile: kn holds K of tile n + 2, vn V of tile n, vo is free, the other
    // slot of LDS holds K of tile n + 1
    auto step = [&](int n, int slot, KRaw& kn, VRaw& vn, VRaw& vo) {
      get_k(slot ^ 1, kf);
      put_k(kn, slot);
      const int nk = min(n + 4, cnt - 1), nv = min(n + 1, cnt - 1);
      const int k0 = __builtin_amdgcn_readlane(id0, nk), k1 = __builtin_amdgcn_readlane(id1, nk);
      const int v2 = __builtin_amdgcn_readlane(id0, nv), v3 = __builtin_amdgcn_readlane(id1, nv);
      const uint32_t e = __builtin_amdgcn_readlane(ex, n);
      refer(sc, byte_scale(e & 255) * scale, byte_scale((e >> 8) & 255) * scale);
      f32x16_t next = zero16();
      Frag pf[2], f;
      k_frag(kf, 0, f);
#pragma unroll
      for (int i = 0; i < NK; ++i) {
        next = mma_32x32x16(f, qf[i], next);
        if (i + 1 < NK) k_frag(kf, i + 1, f);
#pragma unroll
        for (int c = i * (8 / NK); c < (i + 1) * (8 / NK); ++c)
          put(pf, c, weigh(sc[2 * c], sc[2 * c + 1]));
#pragma unroll
        for (int c = i * (NKL + NVL) / NK; c < (i + 1) * (NKL + NVL) / NK; ++c) {
          if (c < NKL) load_k1(k0, k1, c, kn);
          else load_v1(v2, v3, c - NKL, vo);
        }
      }
      sc = next;
      uint32_t w[2][NB][2];
      v_words(vn, 0, w[0]);
      const float v0 = byte_scale((e >> 16) & 255), v1 = byte_scale(e >> 24);
      cvt8(f, w[0][0][0], v0, w[0][0][1], v0);
      __builtin_amdgcn_sched_barrier(0);   // (first the softmax, then V's conversions)
#pragma unroll
      for (int c = 0; c < 2 * NB; ++c) {
        acc[c % NB] = mma_32x32x16(f, pf[c / NB], acc[c % NB]);
        if (c == 0) v_words(vn, 1, w[1]);
        if (c + 1 < 2 * NB) {
          const int p = (c + 1) / NB, b = (c + 1) % NB;
          cvt8(f, w[p][b][0], p ? v1 : v0, w[p][b][1], p ? v1 : v0);
        }
      }
    };
    // (a way out between the two steps would meet the loop's head, as the
    // compiler lays it out, and make that wait for every load under way)
    int n = 0;
    for (; n + 1 < cnt; n += 2) {
      step(n, 0, kq[0], vq[0], vq[1]);
      step(n + 1, 1, kq[1], vq[1], vq[0]);
    }
    if (n < cnt) step(n, 0, kq[0], vq[0], vq[1]);
  }

  // the other tiles: those that some row does not see whole, and, after the
  // last split's share of the prefix, the segment
  const int n_left = f0 - t0, n_pre = n_left + t1 - f1;
  int L = 0;
  if (bz == ns - 1 && kv.seg_pages > 0 && r.vis_words > 0)
    L = max(0, min(min(r.seg_len[s], kv.seg_pages * 16), r.vis_words * 32));
  const int n_gen = n_pre + ((L + 31) >> 5);
  for (int i = (wave + NW - (f1 - f0) % NW) % NW; i < n_gen; i += NW) {
    // which keys of the tile the row sees
    uint32_t keys;
    const int v0 = 2 * (i < n_left ? t0 + i : f1 + i - n_left), t = i - n_pre;
    if (i < n_pre) {
      keys = page_bits(sp.page(v0) * 16, Tp, r.sinks, lo);
      if (v0 + 1 < sp.n) keys |= page_bits(sp.page(v0 + 1) * 16, Tp, r.sinks, lo) << 16;
    } else {
      keys = slot_bits(r.vis[(size_t)row * r.vis_words + t], t, L);
    }
    if (__ballot(keys != 0) == 0) continue;
    keys >>= 4 * h;
    // bit e: key of score e
    const uint32_t seen = (keys & 15) | ((keys >> 4) & 0xF0) | ((keys >> 8) & 0xF00) |
                          ((keys >> 12) & 0xF000);
    f32x16_t sc;
    Frag vf[2][NB];
    float ks[2];
    if (i < n_pre) {
      int pg[2];
      float vs[2];
#pragma unroll
      for (int p = 0; p < 2; ++p) {
        const int ap = sp.page(min(v0 + p, sp.n - 1));
        pg[p] = checked_index(ptab[ap], kv.n_pages, kv.err, kDevPage);
        ks[p] = byte_scale(kv.k_exp[(size_t)pg[p] * Hkv + kh]) * scale;
        vs[p] = byte_scale(kv.v_exp[(size_t)pg[p] * Hkv + kh]);
      }
      load_k(pg[0], pg[1], kq[0]);
      load_v(pg[0], pg[1], vq[0]);
      put_k(kq[0], 0);
      get_k(0, kq[1]);
      sc = scores(kq[1]);
#pragma unroll
      for (int p = 0; p < 2; ++p) {
        uint32_t w[NB][2];
        v_words(vq[0], p, w);
#pragma unroll
        for (int b = 0; b < NB; ++b) cvt8(vf[p][b], w[b][0], vs[p], w[b][1], vs[p]);
      }
    } else {
      ks[0] = ks[1] = scale;
      const int pk = min(2 * t + (c32 >> 4), kv.seg_pages - 1);
      const bf16_t* kp = static_cast<const bf16_t*>(kv.seg_k) +
                         (((size_t)s * kv.seg_pages + pk) * Hkv + kh) * 16 * HD +
                         (c32 & 15) * HD + h * (HD / 2);
      sc = zero16();
#pragma unroll
      for (int c = 0; c < NK; ++c) {
        Frag kf;
        kf.load(kp + 8 * c);
        sc = mma_32x32x16(kf, qf[c], sc);
      }
#pragma unroll
      for (int p = 0; p < 2; ++p) {
        const int pv = min(2 * t + p, kv.seg_pages - 1);
        const bf16_t* vp = static_cast<const bf16_t*>(kv.seg_v) +
                           (((size_t)s * kv.seg_pages + pv) * Hkv + kh) * 16 * HD +
                           c32 * 16 + 4 * h;
#pragma unroll
        for (int b = 0; b < NB; ++b) {
          const uint2 x = *reinterpret_cast<const uint2*>(vp + 512 * b);
          const uint2 y = *reinterpret_cast<const uint2*>(vp + 512 * b + 8);
          vf[p][b].v = make_uint4(x.x, x.y, y.x, y.y);
        }
      }
    }
#pragma unroll
    for (int e = 0; e < 16; ++e) sc[e] = (seen >> e) & 1u ? sc[e] : -__builtin_inff();
    refer(sc, ks[0], ks[1]);
    Frag pf[2];
#pragma unroll
    for (int c = 0; c < 8; ++c) put(pf, c, weigh(sc[2 * c], sc[2 * c + 1]));
    uint32_t bad = 0;
#pragma unroll
    for (int p = 0; p < 2; ++p)
#pragma unroll
      for (int b = 0; b < NB; ++b) bad |= bad_bits(vf[p][b]);
    if (__ballot(bad != 0) != 0) {
#pragma unroll
      for (int p = 0; p < 2; ++p)
#pragma unroll
        for (int b = 0; b < NB; ++b) {
          acc[b] = add_bad32(take_bad(vf[p][b]), (seen >> (8 * p)) & 0xFFu, acc[b]);
          __builtin_amdgcn_sched_barrier(0);   // (one operand at a time)
        }
    }
#pragma unroll
    for (int p = 0; p < 2; ++p)
#pragma unroll
      for (int b = 0; b < NB; ++b) acc[b] = mma_32x32x16(vf[p][b], pf[p], acc[b]);
  }

  // the waves' shares
  l = sum_x32(l);
  if (h == 0) {
    msh[wave][c32] = lim < 0.f ? kLow : m;
    lsh[wave][c32] = l;
  }
#pragma unroll
  for (int b = 0; b < NB; ++b)
#pragma unroll
    for (int g = 0; g < 4; ++g)
      *reinterpret_cast<float4*>(&osh[wave][c32][32 * b + 8 * g + 4 * h]) = make_float4(
          acc[b][4 * g], acc[b][4 * g + 1], acc[b][4 * g + 2], acc[b][4 * g + 3]);
  __syncthreads();
  constexpr int TPQ = NW * 64 / 32;     // threads of one query vector
  const int qj = tid / TPQ, part = tid % TPQ, qv = q0 + qj;
  if (qv >= nq) return;
  float M = kLow, Lsum = 0.f, wt[NW];
#pragma unroll
  for (int w = 0; w < NW; ++w) M = fmaxf(M, msh[w][qj]);
#pragma unroll
  for (int w = 0; w < NW; ++w) {
    wt[w] = __builtin_amdgcn_exp2f(msh[w][qj] - M);
    Lsum += wt[w] * lsh[w][qj];
  }
  const int rq = div_small(qv, G);
  const float inv = Lsum == 0.f ? 0.f : 1.0f / Lsum;
  const size_t at = (size_t)(row0 + rq) * H + kh * G + qv - rq * G;
#pragma unroll
  for (int col = part * 4; col < HD; col += 4 * TPQ) {
    float4 o = make_float4(0.f, 0.f, 0.f, 0.f);
#pragma unroll
    for (int w = 0; w < NW; ++w) {
      const float4 x = *reinterpret_cast<const float4*>(&osh[w][qj][col]);
      o.x += wt[w] * x.x;
      o.y += wt[w] * x.y;
      o.z += wt[w] * x.z;
      o.w += wt[w] * x.w;
    }
    if (ns > 1)
      *reinterpret_cast<float4*>(
          o_part + ((size_t)bz * r.n_rows * H + at) * HD + col) = o;
    else
      store4(out + at * HD + col, make_float4(o.x * inv, o.y * inv, o.z * inv, o.w * inv));
  }
  if (ns > 1 && part == 0)
    *reinterpret_cast<float2*>(ml + ((size_t)bz * r.n_rows * H + at) * 2) =
        make_float2(M, Lsum);
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
  store4(out + row * H * hd + 4 * c,
         make_float4(o.x * inv, o.y * inv, o.z * inv, o.w * inv));
}

int cdiv(long a, long b) { return (int)((a + b - 1) / b); }

}  // namespace

// 32 query vectors a workgroup where there are more than 16 of a KV head (16
// trees of up to 64 nodes 71 us with 16, 46 with 32; fp32 has 16 throughout).
// No split below 1280 entries, where the merge costs what it saves (a row over
// 512: 7.5 us, in two 10.0; 60 nodes over 1024: 12.0, in four 13.2; over 1536:
// 14.3, in four 13.7).  Beyond that as many as give a workgroup on every CU and
// keep 256 entries each, of more than eight 512 (a row over 8192: 13.0 us in 16,
// 15.3 in 32): what a second one on a CU gains the merge costs (500 rows over
// 8192: 94 us, in two 105; 8 windows of 4096, 33 rows each: 29.6, in two 34.5).
// Longer prefixes are cut to 8192 entries so that ragged batches end together.
// The bound stands in for the lengths, which only the device knows: 60 rows over
// 8192 take 23 us with a bound of 8192, 43 with 32768, 50 with 262144.
// Eight waves a workgroup where there is at most one on a CU and it has 1024
// entries (8 windows of 4096: 29.6 us, with four 32.1; 60 nodes over 16384: 31.9
// and 33.4; with splits of 256 or 512 entries four are 1 to 4% faster, with two
// workgroups on a CU 20%).
QPlan kvq_attn_plan(int n_seqs, int rows_per_seq, int max_prefix, int window,
                    int sinks, int H, int Hkv, int es, int max_split) {
  long eff = max_prefix;
  if (window > 0) eff = std::min(eff, (long)window + sinks + 32);
  const long nq = (long)rows_per_seq * (H / Hkv);
  const int width = es == 4 || nq <= 16 ? 16 : 32;
  const long items = (long)cdiv(nq, width) * n_seqs * Hkv;
  long nz = 1;
  if (eff >= 1280)
    nz = std::min(std::max(1L, 256 / items), std::min(eff / 256, std::max(8L, eff / 512)));
  nz = std::max<long>(nz, cdiv(eff, 8192));
  // (the last bound: a launch holds fewer than 2^32 threads)
  nz = std::max(1L, std::min<long>({nz, max_split, kMaxSplit, (1L << 23) / items}));
  const int tokens = std::max(32, cdiv(cdiv(eff, nz), 32) * 32);
  const int n_waves = width == 32 && items * nz <= 256 && tokens >= 1024 ? 8 : 4;
  return QPlan{(int)nz, tokens, width, n_waves};
}

template <typename T>
void launch_kvq_attn(const T* q, const QRows& r, const QView& kv, int H,
                     int Hkv, int hd, const QPlan& plan, float* o_part,
                     float* ml, T* out, hipStream_t st) {
  const float scale = 1.0f / sqrtf((float)hd);
  const int groups = cdiv((long)r.rows_per_seq * (H / Hkv), plan.width);
  const int items = cdiv((long)r.n_seqs * Hkv * plan.n_split, 8) * 8;
  const dim3 grid(groups * items);
  // (the profiler's events: start of this kernel, end of the last one)
  hipEvent_t ea, eb;
  attn_take_events(&ea, &eb);
  const bool merge = plan.n_split > 1;
#define SB_RUN(K_, N_)                                                         \
  hipExtLaunchKernelGGL(K_, grid, dim3(N_), 0, st, ea, merge ? nullptr : eb, 0, \
                        q, r, kv, groups, H, Hkv, plan.n_split,                \
                        plan.split_tokens, scale, o_part, ml, out)
  const bool wide = plan.width == 32, eight = plan.n_waves == 8;
  if constexpr (sizeof(T) == 2) {
    if (wide && eight) {
      auto k = hd == 128 ? kvq_attn32_kernel<128, 8> : kvq_attn32_kernel<64, 8>;
      SB_RUN(k, 512);
    } else if (wide) {
      auto k = hd == 128 ? kvq_attn32_kernel<128, 4> : kvq_attn32_kernel<64, 4>;
      SB_RUN(k, 256);
    }
  }
  if (!wide) {
    auto k = hd == 128 ? kvq_attn_kernel<T, 128> : kvq_attn_kernel<T, 64>;
    SB_RUN(k, 256);
  }
#undef SB_RUN
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
