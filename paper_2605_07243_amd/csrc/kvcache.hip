// C-ABI entry points of the 8-bit K/V cache and the page pool: argument
// checks, workspace layout and launches.  No context is involved; failures are
// described by sb_last_error(NULL).
#include <hip/hip_runtime.h>

#include <algorithm>
#include <cstdio>

#include "kernels.h"
#include "kvq.h"
#include "specblock.h"

using namespace sb;

namespace {

bool bad(const void* p, size_t align) {
  return p == nullptr || reinterpret_cast<uintptr_t>(p) % align != 0;
}

int fail2(int code, const char* call, const char* what) {
  char buf[192];
  snprintf(buf, sizeof buf, "%s: %s", call, what);
  return fail_global(code, buf);
}

int launched(const char* call) {
  const hipError_t e = hipGetLastError();
  return e == hipSuccess ? SB_OK : fail2(SB_EHIP, call, hipGetErrorString(e));
}

int check_shape(const sb_cache_shape* s, const char* call) {
  if (!s) return fail2(SB_EINVAL, call, "shape is NULL");
  if (s->dtype != SB_F32 && s->dtype != SB_BF16)
    return fail2(SB_EDTYPE, call, "dtype must be SB_F32 or SB_BF16");
  if (s->head_dim != 64 && s->head_dim != 128)
    return fail2(SB_ESHAPE, call, "head_dim must be 64 or 128");
  if (s->n_kv_heads < 1 || s->n_heads < 1 || s->n_heads > 64 ||
      s->n_heads % s->n_kv_heads)
    return fail2(SB_ESHAPE, call, "n_heads must be a multiple of n_kv_heads and <= 64");
  if (s->max_seqs < 1 || s->max_seqs > SB_MAX_SEQS)
    return fail2(SB_ESHAPE, call, "max_seqs must be in 1..64");
  if (s->max_pages < 1 || s->max_pages > 16384)
    return fail2(SB_ESHAPE, call, "max_pages must be in 1..16384");
  return SB_OK;
}

int check_kvq(const sb_kvq* kv, const char* call) {
  if (!kv) return fail2(SB_EINVAL, call, "the 8-bit cache is NULL");
  if (bad(kv->k, 16) || bad(kv->v, 16) || bad(kv->k_exp, 1) || bad(kv->v_exp, 1) ||
      bad(kv->page_table, 4))
    return fail2(SB_EINVAL, call, "8-bit cache pointer NULL or misaligned");
  if (kv->n_layers < 1 || kv->n_layers > 65535)
    return fail2(SB_ESHAPE, call, "n_layers must be in 1..65535");
  if (kv->n_pages < 1) return fail2(SB_EINVAL, call, "the 8-bit cache has no pages");
  return SB_OK;
}

int check_elem_kv(const sb_kv* kv, const char* call) {
  if (!kv) return fail2(SB_EINVAL, call, "the cache is NULL");
  if (bad(kv->k, 16) || bad(kv->v, 16) || bad(kv->page_table, 4))
    return fail2(SB_EINVAL, call, "cache pointer NULL or misaligned");
  if (kv->n_layers < 1 || kv->n_layers > 65535)
    return fail2(SB_ESHAPE, call, "n_layers must be in 1..65535");
  if (kv->n_pages < 1) return fail2(SB_EINVAL, call, "the cache has no pages");
  return SB_OK;
}

// Host values of a row description.
int check_rows(const sb_cache_shape* s, const sb_attn_rows* r, int window,
               int sinks, const char* call) {
  if (!r) return fail2(SB_EINVAL, call, "rows is NULL");
  if (r->n_seqs < 1 || r->n_seqs > s->max_seqs)
    return fail2(SB_ESHAPE, call, "n_seqs must be in 1..max_seqs");
  if (r->n_rows < 1 || r->n_rows > (1 << 22))
    return fail2(SB_ESHAPE, call, "n_rows must be in 1..2^22");
  if (r->rows_per_seq < 1 || r->rows_per_seq > 16384)
    return fail2(SB_ESHAPE, call, "rows_per_seq must be in 1..16384");
  if (r->max_prefix < 0) return fail2(SB_EINVAL, call, "max_prefix is negative");
  if (r->vis_words < 0 || r->vis_words > 16)
    return fail2(SB_ESHAPE, call, "vis_words must be in 0..16");
  if (r->seg_pages < 0 || r->seg_pages > 32)
    return fail2(SB_ESHAPE, call, "seg_pages must be in 0..32");
  if (window < 0 || sinks < 0)
    return fail2(SB_EINVAL, call, "window and sinks must not be negative");
  return SB_OK;
}

int prefix_bound(const sb_cache_shape* s, const sb_attn_rows* r) {
  const int cap = s->max_pages * 16;
  return r->max_prefix > 0 ? std::min(r->max_prefix, cap) : cap;
}

// No sequence has more rows than there are.
int most_rows(const sb_attn_rows* r) { return std::min(r->rows_per_seq, r->n_rows); }

QPlan plan_of(const sb_cache_shape* s, const sb_attn_rows* r, int window, int sinks) {
  return kvq_attn_plan(r->n_seqs, most_rows(r), prefix_bound(s, r), window, sinks,
                       s->n_heads, s->n_kv_heads, s->dtype == SB_BF16 ? 2 : 4, 64);
}

size_t align_up(size_t x) { return (x + 255) / 256 * 256; }

size_t part_bytes(const sb_cache_shape* s, const sb_attn_rows* r, const QPlan& p) {
  if (p.n_split == 1) return 0;
  return align_up((size_t)p.n_split * r->n_rows * s->n_heads * s->head_dim * 4);
}

size_t need_bytes(const sb_cache_shape* s, const sb_attn_rows* r, const QPlan& p) {
  const size_t ml =
      p.n_split == 1 ? 0 : align_up((size_t)p.n_split * r->n_rows * s->n_heads * 8);
  return std::max<size_t>(256, part_bytes(s, r, p) + ml);
}

bool overlap(const void* a, const void* b, size_t bytes) {
  const uintptr_t x = reinterpret_cast<uintptr_t>(a), y = reinterpret_cast<uintptr_t>(b);
  return x < y + bytes && y < x + bytes;
}

int check_pool(const sb_cache_shape* s, const sb_pool* p, const char* call) {
  const int rc = check_shape(s, call);
  if (rc) return rc;
  if (!p) return fail2(SB_EINVAL, call, "pool is NULL");
  if (bad(p->page_table, 4) || bad(p->held, 4) || bad(p->refs, 4) ||
      bad(p->refused, 4) || bad(p->scratch, 4))
    return fail2(SB_EINVAL, call, "pool pointer NULL or misaligned");
  if (p->n_pages < 1 || p->n_pages > (1 << 20))
    return fail2(SB_ESHAPE, call, "n_pages must be in 1..2^20");
  return SB_OK;
}

// The memory of the caches that go with a pool.
int regions(const sb_cache_shape* s, const sb_pool* p, const sb_kv* kv,
            const sb_kvq* kvq, PoolRegions* out, const char* call) {
  out->n = 0;
  const int elems = s->n_kv_heads * 16 * s->head_dim;
  if (kv) {
    const int rc = check_elem_kv(kv, call);
    if (rc) return rc;
    if (kv->n_pages != p->n_pages || kv->page_table != p->page_table)
      return fail2(SB_EINVAL, call, "the cache has another page table or page count");
    out->r[out->n++] = PoolRegion{static_cast<char*>(kv->k), static_cast<char*>(kv->v),
                                  nullptr, nullptr,
                                  elems * (s->dtype == SB_BF16 ? 2 : 4), 0,
                                  kv->n_layers};
  }
  if (kvq) {
    const int rc = check_kvq(kvq, call);
    if (rc) return rc;
    if (kvq->n_pages != p->n_pages || kvq->page_table != p->page_table)
      return fail2(SB_EINVAL, call, "the 8-bit cache has another page table or page count");
    out->r[out->n++] = PoolRegion{reinterpret_cast<char*>(kvq->k),
                                  reinterpret_cast<char*>(kvq->v), kvq->k_exp,
                                  kvq->v_exp, elems, s->n_kv_heads, kvq->n_layers};
  }
  return SB_OK;
}

int check_list(const sb_cache_shape* s, int n, const int32_t* list, const char* call) {
  if (n < 1 || n > s->max_seqs)
    return fail2(SB_ESHAPE, call, "the list must name 1..max_seqs sequences");
  if (!list) return fail2(SB_EINVAL, call, "the list is NULL");
  for (int i = 0; i < n; ++i)
    if (list[i] < 0 || list[i] >= s->max_seqs)
      return fail2(SB_EINVAL, call, "sequence out of range");
  return SB_OK;
}

bool distinct(int n, const int32_t* list) {
  uint64_t seen = 0;
  for (int i = 0; i < n; ++i) {
    if ((seen >> list[i]) & 1) return false;
    seen |= 1ull << list[i];
  }
  return true;
}

hipStream_t S_(void* s) { return static_cast<hipStream_t>(s); }

}  // namespace

extern "C" {

int sb_kvq_store(const sb_cache_shape* shape, int32_t n_seqs, const sb_kv* src,
                 const int32_t* first, const int32_t* last,
                 int32_t max_entries, sb_kvq* dst, void* stream) {
  const char* me = "sb_kvq_store";
  int rc = check_shape(shape, me);
  if (rc || (rc = check_elem_kv(src, me)) || (rc = check_kvq(dst, me))) return rc;
  if (n_seqs < 1 || n_seqs > shape->max_seqs)
    return fail2(SB_ESHAPE, me, "n_seqs must be in 1..max_seqs");
  if (src->n_layers != dst->n_layers)
    return fail2(SB_ESHAPE, me, "the caches differ in their layers");
  if (bad(first, 4) || bad(last, 4))
    return fail2(SB_EINVAL, me, "first or last NULL or misaligned");
  if (max_entries < 1) return fail2(SB_EINVAL, me, "max_entries must be >= 1");
  (void)hipGetLastError();
  if (shape->dtype == SB_BF16)
    launch_kvq_store<bf16_t>(static_cast<const bf16_t*>(src->k),
                             static_cast<const bf16_t*>(src->v), src->page_table,
                             src->n_pages, *dst, shape->max_pages, n_seqs, first,
                             last, max_entries, shape->n_kv_heads, shape->head_dim,
                             S_(stream));
  else
    launch_kvq_store<float>(static_cast<const float*>(src->k),
                            static_cast<const float*>(src->v), src->page_table,
                            src->n_pages, *dst, shape->max_pages, n_seqs, first,
                            last, max_entries, shape->n_kv_heads, shape->head_dim,
                            S_(stream));
  return launched(me);
}

size_t sb_kvq_attend_workspace(const sb_cache_shape* shape,
                               const sb_attn_rows* rows, int32_t window,
                               int32_t sinks) {
  const char* me = "sb_kvq_attend_workspace";
  if (check_shape(shape, me) || check_rows(shape, rows, window, sinks, me)) return 0;
  return need_bytes(shape, rows, plan_of(shape, rows, window, sinks));
}

int sb_kvq_attend(const sb_cache_shape* shape, const sb_kvq* kv, int32_t layer,
                  const sb_attn_rows* rows, const void* q, int32_t window,
                  int32_t sinks, void* out, void* workspace,
                  size_t workspace_bytes, void* stream) {
  const char* me = "sb_kvq_attend";
  int rc = check_shape(shape, me);
  if (rc || (rc = check_kvq(kv, me)) ||
      (rc = check_rows(shape, rows, window, sinks, me)))
    return rc;
  if (layer < 0 || layer >= kv->n_layers)
    return fail2(SB_EINVAL, me, "layer must be in 0..n_layers-1");
  if (bad(rows->row_off, 4) || bad(rows->prefix_len, 4) ||
      (window > 0 && bad(rows->pos, 4)))
    return fail2(SB_EINVAL, me, "rows pointer NULL or misaligned");
  const bool seg = rows->seg_pages > 0;
  if (seg && (rows->vis_words < 1 || bad(rows->seg_len, 4) || bad(rows->vis, 4) ||
              bad(rows->seg_k, 16) || bad(rows->seg_v, 16)))
    return fail2(SB_EINVAL, me, "a segment needs seg_len, vis, seg_k and seg_v");
  if (bad(q, 16) || bad(out, 16))
    return fail2(SB_EINVAL, me, "q or out NULL or not 16-byte aligned");
  const size_t bytes = (size_t)rows->n_rows * shape->n_heads * shape->head_dim *
                       (shape->dtype == SB_BF16 ? 2 : 4);
  if (overlap(q, out, bytes)) return fail2(SB_EINVAL, me, "q and out overlap");
  const QPlan plan = plan_of(shape, rows, window, sinks);
  if (bad(workspace, 256))
    return fail2(SB_EINVAL, me, "workspace NULL or not 256-byte aligned");
  if (workspace_bytes < need_bytes(shape, rows, plan))
    return fail2(SB_EBUDGET, me, "workspace too small (sb_kvq_attend_workspace)");
  const size_t page = (size_t)shape->n_kv_heads * 16 * shape->head_dim;
  const size_t at = (size_t)layer * kv->n_pages;
  const QView v{kv->k + at * page, kv->v + at * page,
                kv->k_exp + at * shape->n_kv_heads, kv->v_exp + at * shape->n_kv_heads,
                kv->page_table, shape->max_pages, kv->n_pages,
                rows->seg_k, rows->seg_v, rows->seg_pages, nullptr};
  const QRows r{rows->row_off, rows->pos, rows->prefix_len, rows->seg_len, rows->vis,
                seg ? rows->vis_words : 0, rows->n_seqs, rows->n_rows,
                most_rows(rows), prefix_bound(shape, rows), window, sinks};
  float* o_part = static_cast<float*>(workspace);
  float* ml = reinterpret_cast<float*>(static_cast<char*>(workspace) +
                                       part_bytes(shape, rows, plan));
  (void)hipGetLastError();
  if (shape->dtype == SB_BF16)
    launch_kvq_attn<bf16_t>(static_cast<const bf16_t*>(q), r, v, shape->n_heads,
                            shape->n_kv_heads, shape->head_dim, plan, o_part, ml,
                            static_cast<bf16_t*>(out), S_(stream));
  else
    launch_kvq_attn<float>(static_cast<const float*>(q), r, v, shape->n_heads,
                           shape->n_kv_heads, shape->head_dim, plan, o_part, ml,
                           static_cast<float*>(out), S_(stream));
  return launched(me);
}

int sb_pool_reset(const sb_cache_shape* shape, const sb_pool* pool, void* stream) {
  const char* me = "sb_pool_reset";
  const int rc = check_pool(shape, pool, me);
  if (rc) return rc;
  (void)hipGetLastError();
  launch_pool_reset(*pool, shape->max_seqs, shape->max_pages, S_(stream));
  return launched(me);
}

int sb_pool_grow(const sb_cache_shape* shape, const sb_pool* pool,
                 int32_t n_seqs, const int32_t* len, int32_t extra,
                 void* stream) {
  const char* me = "sb_pool_grow";
  const int rc = check_pool(shape, pool, me);
  if (rc) return rc;
  if (n_seqs < 1 || n_seqs > shape->max_seqs)
    return fail2(SB_ESHAPE, me, "n_seqs must be in 1..max_seqs");
  if (bad(len, 4)) return fail2(SB_EINVAL, me, "len NULL or misaligned");
  if (extra < 0) return fail2(SB_EINVAL, me, "extra must not be negative");
  (void)hipGetLastError();
  launch_pool_grow(*pool, n_seqs, len, extra, shape->max_pages, S_(stream));
  return launched(me);
}

int sb_pool_release(const sb_cache_shape* shape, const sb_pool* pool, int32_t n,
                    const int32_t* seqs, void* stream) {
  const char* me = "sb_pool_release";
  int rc = check_pool(shape, pool, me);
  if (rc || (rc = check_list(shape, n, seqs, me))) return rc;
  if (!distinct(n, seqs)) return fail2(SB_EINVAL, me, "the sequences are not distinct");
  PoolList l{};
  l.n = n;
  for (int i = 0; i < n; ++i) l.a[i] = (unsigned char)seqs[i];
  (void)hipGetLastError();
  launch_pool_release(*pool, l, false, shape->max_pages, S_(stream));
  return launched(me);
}

int sb_pool_fork(const sb_cache_shape* shape, const sb_pool* pool, int32_t n,
                 const int32_t* parent, const int32_t* child,
                 const int32_t* len, const sb_kv* kv, const sb_kvq* kvq,
                 void* stream) {
  const char* me = "sb_pool_fork";
  int rc = check_pool(shape, pool, me);
  if (rc || (rc = check_list(shape, n, parent, me)) ||
      (rc = check_list(shape, n, child, me)))
    return rc;
  if (!distinct(n, child)) return fail2(SB_EINVAL, me, "the children are not distinct");
  for (int i = 0; i < n; ++i)
    for (int j = 0; j < n; ++j)
      if (parent[i] == child[j]) return fail2(SB_EINVAL, me, "a child is a parent");
  if (bad(len, 4)) return fail2(SB_EINVAL, me, "len NULL or misaligned");
  PoolRegions rg;
  if ((rc = regions(shape, pool, kv, kvq, &rg, me))) return rc;
  PoolList l{};
  l.n = n;
  for (int i = 0; i < n; ++i) {
    l.a[i] = (unsigned char)parent[i];
    l.b[i] = (unsigned char)child[i];
  }
  (void)hipGetLastError();
  launch_pool_fork(*pool, l, len, rg, shape->max_pages, S_(stream));
  return launched(me);
}

int sb_pool_compact(const sb_cache_shape* shape, const sb_pool* pool,
                    const sb_kv* kv, const sb_kvq* kvq, void* stream) {
  const char* me = "sb_pool_compact";
  int rc = check_pool(shape, pool, me);
  if (rc) return rc;
  PoolRegions rg;
  if ((rc = regions(shape, pool, kv, kvq, &rg, me))) return rc;
  (void)hipGetLastError();
  launch_pool_compact(*pool, rg, shape->max_seqs, shape->max_pages, S_(stream));
  return launched(me);
}

}  // extern "C"
