// Paged key-value cache: what its kernels share (paged_append.hip, paged_attn.hip).
#pragma once
#include "af_internal.h"

// A cache and a batch as the kernels see them (af_paged_cache, af_paged_batch).
struct PagedView {
  half_t *k, *v;              // [n_pages][n_kv][page][head_dim], pages page_stride elements apart
  long long page_stride;
  const int32_t* table;       // [n_seqs][table_stride]
  const int32_t* kv_len;      // [n_seqs]
  const int32_t* q_start;     // [n_seqs + 1], or null: row b is sequence b's
  int table_stride, n_pages, page_shift, n_kv;
  int n_seqs, n_rows, max_q_len;
  int* tickets;               // of the workspace; the device error word lies behind them
};

// Host side of every paged entry point: the checks of cache and batch and the view, then (behind the entry
// point's own checks) those of the context.
int af_paged_view(const af_paged_cache* cache, const af_paged_batch* batch, int n_heads, PagedView* v);
int af_paged_ready(const af_ctx* ctx, PagedView* v);
bool af_paged_rows_ok(const void* p, long long stride, long long width);

#ifdef __HIPCC__
#define PAGED_HD __host__ __device__ __forceinline__

// One sequence of the batch: its rows [row0, row0 + q_len) of the token tensors and its len cached tokens, of
// which the rows are the last q_len.
struct PagedSeq {
  int row0, q_len, len;
};
// Numbers that cannot be right give no rows and no tokens (and false), so that no access ever follows them.
PAGED_HD bool paged_seq_check(const PagedView& v, int row0, int row1, int len, PagedSeq* s) {
  bool ok = len >= 0 && len <= (v.table_stride << v.page_shift);
  if (v.q_start) ok = ok && row0 >= 0 && row1 >= row0 && row1 <= v.n_rows && row1 - row0 <= v.max_q_len && row1 - row0 <= len;
  *s = PagedSeq{row0, ok ? row1 - row0 : 0, ok ? len : 0};
  return ok;
}
PAGED_HD bool paged_page_ok(const PagedView& v, int page) { return (unsigned)page < (unsigned)v.n_pages; }
// Element offset of token j's row of key head h inside the cache.
PAGED_HD size_t paged_offset(const PagedView& v, int page, int h, int j, int head_dim) {
  const int slot = j & ((1 << v.page_shift) - 1);
  return (size_t)page * (size_t)v.page_stride + (((size_t)h << v.page_shift) + slot) * head_dim;
}
// The keys that rows at the places p0 .. p1 of a sequence can see, in tiles of TK: tile i starts at key i TK for the
// first tokens (i < sinks), at lo + (i - sinks) TK behind them.  Tiles do not overlap; their ends may hold keys
// that a row does not see.  lo is a multiple of 16, so 16 keys from a tile's start on never lie in two pages.
struct PagedTiles {
  int sinks, lo, n;
};
template <int TK>
PAGED_HD PagedTiles paged_tiles(int p0, int p1, int window, int n_sink) {
  if (p1 < 0) return PagedTiles{0, 0, 0};
  const int first = window > 0 && p0 - window + 1 > 0 ? p0 - window + 1 : 0;
  int lo = first & ~15, sinks = ((n_sink < first ? n_sink : first) + TK - 1) / TK;
  if (sinks * TK >= lo) sinks = lo = 0;
  return PagedTiles{sinks, lo, sinks + (p1 - lo) / TK + 1};
}
template <int TK>
PAGED_HD int paged_tile_start(const PagedTiles& t, int i) {
  return i < t.sinks ? i * TK : t.lo + (i - t.sinks) * TK;
}
PAGED_HD bool paged_seen(int key, int place, int window, int n_sink) {
  return key <= place && (window <= 0 || key > place - window || key < n_sink);
}
// Whether a row at one of the places p0 .. p1 sees one of the 16 keys from `key` on.
PAGED_HD bool paged_span_seen(int key, int p0, int p1, int window, int n_sink) {
  return key <= p1 && (window <= 0 || key + 15 > p0 - window || key < n_sink);
}

__device__ __forceinline__ void paged_report(const PagedView& v) {
  __hip_atomic_fetch_or(v.tickets + AF_TICKET_ERR, (int)AF_DEVERR_PAGED, __ATOMIC_RELAXED, __HIP_MEMORY_SCOPE_AGENT);
}
__device__ __forceinline__ PagedSeq paged_seq_of(const PagedView& v, int row0, int row1, int len) {
  PagedSeq s;
  if (!paged_seq_check(v, row0, row1, len, &s)) paged_report(v);
  return s;
}
__device__ __forceinline__ PagedSeq paged_seq(const PagedView& v, int b) {
  return paged_seq_of(v, v.q_start ? v.q_start[b] : b, v.q_start ? v.q_start[b + 1] : b + 1, v.kv_len[b]);
}
// Page of token j of sequence b (j < len): -1 and a report if the table holds none.
__device__ __forceinline__ int paged_page(const PagedView& v, int b, int j) {
  const int id = v.table[(size_t)b * v.table_stride + (j >> v.page_shift)];
  if (paged_page_ok(v, id)) return id;
  paged_report(v);
  return -1;
}
#endif
