// A cache of keys and values in pages: what kernels take of it, and its checks on the host.
//
// Token p of a sequence is row p % page of the page that entry p / page of the sequence's row of the table names; page sizes are powers of two.  In E4M3 an
// element stands for itself times the scale of its page and key head, a power of two, so that whatever is made of the two in bf16 is exact.
#pragma once
#include "view.h"

namespace dfs {

struct PageArgs {
  View k, v;                                         // [pages, heads_kv, page, d]
  float *k_scale, *v_scale;                          // [pages, heads_kv]
  const int32_t* table;                              // [seqs, row]
  int32_t pages, heads_kv, row, bits;                // a page has 1 << bits rows
};

// The entry for page i of sequence s; -1 for those that the table has no room for or that name no page.
__device__ __forceinline__ int page_of(const PageArgs& a, int s, int i) {
  if (i < 0 || i >= a.row) return -1;
  const int id = a.table[int64_t(s) * a.row + i];
  return id >= 0 && id < a.pages ? id : -1;
}

// `dtype`: of the queries that go with it.
inline int check_pages(const char* call, const dfs_pages* p, int dtype, int seqs, int heads_kv, int d, bool output, PageArgs* a) {
  if (!p) return fail(DFS_EINVAL, "%s: pages is NULL", call);
  const bool bytes = p->dtype == DFS_E4M3 && dtype == DFS_BF16;
  if (p->dtype != dtype && !bytes) return fail(DFS_EDTYPE, "%s: pages of dtype %d do not go with tensors of dtype %d", call, p->dtype, dtype);
  if (p->page != 16 && p->page != 32 && p->page != 64 && p->page != 128) return fail(DFS_ESHAPE, "%s: page=%d must be 16, 32, 64 or 128", call, p->page);
  if (p->pages < 0 || p->table_row < 0 || int64_t(p->table_row) * p->page > 1 << 28)
    return fail(DFS_ESHAPE, "%s: pages=%d and table_row=%d must not be negative, table_row x page be at most 2^28", call, p->pages, p->table_row);
  if (misaligned(4, {p->table, p->k_scale, p->v_scale})) return fail(DFS_EINVAL, "%s: table and scales must be 4-byte aligned", call);
  const bool some = p->pages > 0 && seqs > 0 && p->table_row > 0;
  if (some && !p->table) return fail(DFS_EINVAL, "%s: table is NULL", call);
  if (bytes ? some && (!p->k_scale || !p->v_scale) : p->k_scale || p->v_scale)
    return fail(DFS_EINVAL, "%s: pages have scales if they are of DFS_E4M3, and only then", call);
  if (bytes && some && output) {                     // both are written, each by the values of its own
    const uintptr_t x = uintptr_t(p->k_scale), y = uintptr_t(p->v_scale);
    if ((x < y ? y - x : x - y) / sizeof(float) < uint64_t(p->pages) * heads_kv) return fail(DFS_EINVAL, "%s: k_scale and v_scale share memory", call);
  }
  int rc;
  if ((rc = check_view(call, "pages.k", &p->k, p->dtype, p->pages, heads_kv, p->page, d, output, &a->k))) return rc;
  if ((rc = check_view(call, "pages.v", &p->v, p->dtype, p->pages, heads_kv, p->page, d, output, &a->v))) return rc;
  for (const View* v : {&a->k, &a->v})
    if (v->row > (int64_t(1) << 24)) return fail(DFS_ESHAPE, "%s: rows of a page are more than 2^24 bytes apart", call);
  a->k_scale = p->k_scale;
  a->v_scale = p->v_scale;
  a->table = p->table;
  a->pages = p->pages;
  a->heads_kv = heads_kv;
  a->row = some ? p->table_row : 0;
  for (a->bits = 4; 1 << a->bits < p->page;) ++a->bits;
  return DFS_OK;
}

}  // namespace dfs
