// Internal launch interface of the 8-bit K/V cache: storing into it, attention
// over it, and the page pool.
#pragma once
#include <hip/hip_runtime.h>
#include <stddef.h>
#include <stdint.h>

#include "specblock.h"

namespace sb {

// One layer of an 8-bit paged cache (codes [page][Hkv][16 hd], scale bytes
// [page][Hkv]) and the rows' own keys in the elem page layout.
struct QView {
  const uint8_t* k;
  const uint8_t* v;
  const uint8_t* k_exp;
  const uint8_t* v_exp;
  const int* page_table;     // [n_seqs][max_pages]
  int max_pages;
  int n_pages;
  const void* seg_k;         // [n_seqs][seg_pages][Hkv][16][hd]
  const void* seg_v;         // [n_seqs][seg_pages][Hkv][hd][16]
  int seg_pages;
  int* err;                  // debug status word (out-of-range pages), or null
};

// Rows of one attention call, sequence-major.
struct QRows {
  const int* row_off;        // [n_seqs + 1]
  const int* pos;            // [n_rows]
  const int* prefix_len;     // [n_seqs]
  const int* seg_len;        // [n_seqs]
  const uint32_t* vis;       // [n_rows][vis_words]
  int vis_words;
  int n_seqs;
  int n_rows;                // rows that the buffers hold
  int rows_per_seq;          // host bound of one sequence's rows
  int max_prefix;            // host bound of the prefixes
  int window;                // 0: everything is seen
  int sinks;
};

// Prefix splits of a call (host plan): n_split workgroups per query group, KV
// head and sequence at most, split_tokens entries each.
struct QPlan {
  int n_split;
  int split_tokens;
  int width;                 // query vectors per workgroup: 16 or 32
  int n_waves;               // waves of a workgroup
};
QPlan kvq_attn_plan(int n_seqs, int rows_per_seq, int max_prefix, int window,
                    int sinks, int H, int Hkv, int es, int max_split);
// o_part [n_split][n_rows][H][hd], ml [n_split][n_rows][H][2] (fp32; unused
// with one split).
template <typename T>
void launch_kvq_attn(const T* q, const QRows& r, const QView& kv, int H,
                     int Hkv, int hd, const QPlan& plan, float* o_part,
                     float* ml, T* out, hipStream_t st);

// Entries first[s] .. last[s] - 1 of n_seqs sequences and n_layers layers from
// an elem cache into an 8-bit one (at most max_entries of them).
template <typename T>
void launch_kvq_store(const T* src_k, const T* src_v, const int* src_table,
                      int src_pages, const sb_kvq& dst, int max_pages,
                      int n_seqs, const int* first, const int* last,
                      int max_entries, int Hkv, int hd, hipStream_t st);
// Commit into an 8-bit cache: segment slots 0 and path[0 .. a-1] of sequence s
// become entries T .. T + a.
template <typename T>
void launch_kvq_commit(const T* seg_k, const T* seg_v, int seg_pages,
                       int pool_seqs, const sb_kvq& dst, int max_pages,
                       int n_seqs, const int* T_old, const int* a,
                       const int* path, int path_cap, int Hkv, int hd, int* err,
                       hipStream_t st);

// Page pool (see specblock.h).
struct PoolList {            // sequences of a call, by value
  int n;
  unsigned char a[64];
  unsigned char b[64];
};
struct PoolRegion {          // one cache: k, v [n_layers][n_pages][page_bytes]
  char* k;
  char* v;
  uint8_t* k_exp;            // [n_layers][n_pages][exp_bytes], if any
  uint8_t* v_exp;
  int page_bytes;            // of 16 tokens of K or V, a multiple of 16
  int exp_bytes;
  int n_layers;
};
struct PoolRegions {
  int n;
  PoolRegion r[2];
};
void launch_pool_reset(const sb_pool& p, int max_seqs, int max_pages,
                       hipStream_t st);
void launch_pool_grow(const sb_pool& p, int n_seqs, const int* len, int extra,
                      int max_pages, hipStream_t st);
void launch_pool_release(const sb_pool& p, const PoolList& l, bool children,
                         int max_pages, hipStream_t st);
void launch_pool_fork(const sb_pool& p, const PoolList& l, const int* len,
                      const PoolRegions& rg, int max_pages, hipStream_t st);
void launch_pool_compact(const sb_pool& p, const PoolRegions& rg, int max_seqs,
                         int max_pages, hipStream_t st);

// Records a failure of a call without a context (sb_last_error(NULL)).
int fail_global(int code, const char* msg) noexcept;

}  // namespace sb
