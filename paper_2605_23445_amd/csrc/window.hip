// Attention over a window around each query's position and a few first keys: checks and launches.
#include <math.h>

#include "window_fwd.h"

namespace dfs {

// First keys that count: none where every window reaches back to them.
static int first_keys(const dfs_window* w) {
  if (w->left < 0 || w->left >= w->n_k) return 0;
  return w->sinks < w->n_k ? w->sinks : w->n_k;
}

static int check_window(const char* call, const dfs_window* w, int dtype) {
  if (!w) return fail(DFS_EINVAL, "%s: window pointer is NULL", call);
  if (dtype != DFS_F32 && dtype != DFS_BF16) return fail(DFS_EDTYPE, "%s: dtype %d is not DFS_F32 or DFS_BF16", call, dtype);
  if (w->batch < 0 || w->n_q < 0 || w->n_k < 0 || w->n_q > 1 << 28 || w->n_k > 1 << 28)
    return fail(DFS_ESHAPE, "%s: batch=%d must not be negative, n_q=%d and n_k=%d be in [0, 2^28]", call, w->batch, w->n_q, w->n_k);
  if (w->heads < 1 || w->heads_kv < 1 || w->heads > 65535 || w->heads % w->heads_kv)
    return fail(DFS_ESHAPE, "%s: heads=%d must be in [1, 65535] and a multiple of heads_kv=%d", call, w->heads, w->heads_kv);
  if (w->d != 64 && w->d != 128) return fail(DFS_ESHAPE, "%s: d=%d: head dimension must be 64 or 128", call, w->d);
  if (w->sinks < 0) return fail(DFS_ESHAPE, "%s: sinks=%d is negative", call, w->sinks);
  // A sequence's rows, which blocks of 128 may pass, are counted in 31 bits; a grid has fewer than 2^32 threads, 256 for a block of 128 rows or keys or
  // for 32 first keys.
  const int64_t rows = int64_t(w->heads / w->heads_kv) * w->n_q, most = rows > w->n_k ? rows : w->n_k, tiles = first_keys(w) / 32;
  const int64_t groups = (most / 128 > tiles ? most / 128 : tiles) + 1, seqs = int64_t(w->batch) * w->heads_kv;
  if (rows > int64_t(1) << 30 || seqs >= 1 << 24 || groups * seqs >= 1 << 24)
    return fail(DFS_ESHAPE, "%s: batch=%d x heads_kv=%d x rows of q or k too large", call, w->batch, w->heads_kv);
  return DFS_OK;
}

// Scratch of the backward pass: two sums of every row, then parts of gradients.  The queries of 32 first keys go to as many work-groups as make 256 in all, one a
// CU, of which each of four waves has two tiles of 32 at least.  Where blocks of 128 keys, or rows, are fewer than CUs, work-groups share one's queries,
// or keys, four tiles each at least: 4 000 fp32 rows of one key head would else have 32 work-groups, for milliseconds.
struct BwdLayout { size_t first, keys, rows, total; int tiles, splits, key_splits, row_splits; };
static BwdLayout bwd_layout(const dfs_window* w) {
  BwdLayout L;
  const int64_t seqs = int64_t(w->batch) * w->heads_kv, group = w->heads / w->heads_kv, rows = group * w->n_q;
  const int64_t reach = w->left < 0 || w->right < 0 ? int64_t(1) << 40 : int64_t(w->left) + w->right + 128;
  const int64_t key_blocks = (int64_t(w->n_k) + 127) / 128 * seqs, row_blocks = (rows + 127) / 128 * seqs, part = 64 * w->d * sizeof(float);
  L.tiles = (first_keys(w) + 31) / 32;
  L.splits = share(seqs * L.tiles, rows / 64);
  L.key_splits = share(key_blocks, ((reach < w->n_q ? reach : w->n_q) + 31) / 32 * group);
  L.row_splits = share(row_blocks, ((reach < w->n_k ? reach : w->n_k) + 63) / 64);
  L.first = align256(size_t(w->batch) * w->heads * w->n_q * sizeof(float2));
  L.keys = L.first + size_t(seqs) * L.tiles * L.splits * part;
  L.rows = L.keys + (L.key_splits > 1 ? size_t(key_blocks) * 4 * L.key_splits : size_t(seqs) * L.tiles) * part;
  L.total = L.rows + (L.row_splits > 1 ? size_t(row_blocks) * 4 * L.row_splits * (part / 2 + 64 * sizeof(float)) : 0);
  return L;
}

// The forward pass over few rows: into how many work-groups the keys of 32 rows are split; 0: not split, blocks of 128 rows.  Scratch: a row of fp32
// sums, its maximum and sum for each split.
struct FwdLayout { size_t sums, total; int64_t blocks; int splits; bool once; };
static FwdLayout fwd_layout(const dfs_window* w, int dtype) {
  const int64_t seqs = int64_t(w->batch) * w->heads_kv, group = w->heads / w->heads_kv, rows = group * w->n_q;
  FwdLayout L = {0, 0, (rows + 31) / 32 * seqs, 0, false};
  // Blocks of 128 rows need enough of them: 32 rows a work-group run four times as many, each in a quarter of the time, for as long as all run at once
  // (us, blocks of 128 against split: 2 048 tokens x 8 heads, d = 64, 20.5 / 11.4; 1 024 x 16 heads of 4 key heads, d = 128, 14.5 / 18.3; 30 000 x 1, d = 128,
  // 95 / 154; fp32, 1 000 x 12, d = 64, 47 / 31).
  if (rows > 32 && (rows + 127) / 128 * seqs > (w->d == 64 ? 128 : 64)) return L;
  const int waves = dtype == DFS_F32 && w->d == 128 ? 2 : 4;
  // keys that 32 rows see, at most
  int64_t keys = w->n_k, reach = int64_t(w->left) + w->right + 32 / group + 1;
  if (w->left >= 0 && w->right >= 0 && reach < keys) keys = reach + first_keys(w) < keys ? reach + first_keys(w) : keys;
  const int64_t tiles = (keys + 31) / 32 + (first_keys(w) > 0);
  // What is more than the memory-side cache holds from one step to the next passes it by (48 x 8 key heads over 4 100 keys, 0.8 GB: 156 -> 141 us).
  L.once = rows <= 32 && tiles * 32 * seqs * w->d * 2 * elem_size(dtype) > int64_t(256) << 20;
  // 128 work-groups draw all that memory gives (one token of 16 x 8 key heads over 4 100 keys: 6.2 TB/s); more of them cost each its start and its part, some
  // 5 us, which only long lists are worth, where they even out lengths (4 x 8 key heads over 32 768 to 65 536 keys: 128 take 187 us, 512 131).
  const int64_t some = 128 / (L.blocks ? L.blocks : 1), all = 512 / (L.blocks ? L.blocks : 1), own = tiles / (waves * 32);
  int64_t splits = some < (tiles + waves - 1) / waves ? some : (tiles + waves - 1) / waves;
  if (splits < all && splits < own) splits = all < own ? all : own;
  L.splits = splits < 1 ? 1 : int(splits);
  if (L.splits > 1) {
    L.sums = align256(size_t(L.blocks) * L.splits * 32 * w->d * sizeof(float));
    L.total = L.sums + size_t(L.blocks) * L.splits * 32 * sizeof(float2);
  }
  return L;
}

static int fill_window(const char* call, const dfs_window* w, int dtype, const dfs_view* q, const dfs_view* k, const dfs_view* v, const dfs_view* o, bool o_out,
                       const float* lse, const int32_t* q_len, const int32_t* k_len, float scale, WindowArgs* a) {
  int rc = check_window(call, w, dtype);
  if (rc) return rc;
  if (!(scale > 0.f) || !isfinite(scale)) return fail(DFS_EINVAL, "%s: scale must be positive and finite", call);
  if (misaligned(4, {lse, q_len, k_len})) return fail(DFS_EINVAL, "%s: lse and lengths must be 4-byte aligned", call);
  if ((rc = check_view(call, "q", q, dtype, w->batch, w->heads, w->n_q, w->d, false, &a->q))) return rc;
  if ((rc = check_view(call, "k", k, dtype, w->batch, w->heads_kv, w->n_k, w->d, false, &a->k))) return rc;
  if ((rc = check_view(call, "v", v, dtype, w->batch, w->heads_kv, w->n_k, w->d, false, &a->v))) return rc;
  if ((rc = check_view(call, "o", o, dtype, w->batch, w->heads, w->n_q, w->d, o_out, &a->o))) return rc;
  if ((rc = check_tiles(call, "k", a->k)) || (rc = check_tiles(call, "v", a->v))) return rc;
  a->lse = const_cast<float*>(lse);
  a->q_len = q_len;
  a->k_len = k_len;
  a->batch = w->batch;
  a->heads = w->heads;
  a->heads_kv = w->heads_kv;
  a->group = w->heads / w->heads_kv;
  a->seqs = w->batch * w->heads_kv;
  a->by_kv = Div(uint32_t(w->heads_kv));
  a->by_group = Div(uint32_t(a->group));
  a->n_q = w->n_q;
  a->n_k = w->n_k;
  a->left = w->left < 0 || w->left > NO_LIMIT ? NO_LIMIT : w->left;
  a->right = w->right < 0 || w->right > NO_LIMIT ? NO_LIMIT : w->right;
  a->sinks = first_keys(w);
  a->scale = scale;
  return DFS_OK;
}

}  // namespace dfs

using namespace dfs;

extern "C" {

size_t dfs_window_workspace_bytes(const dfs_window* w, int dtype, int backward) {
  if (check_window("dfs_window_workspace_bytes", w, dtype) != DFS_OK) return 0;
  return backward ? bwd_layout(w).total : fwd_layout(w, dtype).total;
}

int dfs_window_attn_fwd(const dfs_window* w, int dtype, const dfs_view* q, const dfs_view* k, const dfs_view* v, const int32_t* q_len,
                        const int32_t* k_len, float scale, const dfs_view* o, float* lse, void* ws, size_t ws_bytes, void* stream) {
  const char* call = "dfs_window_attn_fwd";
  WindowArgs a = {};
  int rc = fill_window(call, w, dtype, q, k, v, o, true, lse, q_len, k_len, scale, &a);
  if (rc) return rc;
  if (w->batch == 0 || w->n_q == 0) return DFS_OK;
  if ((rc = check_apart(call, {{"o", &a.o}}, {{"q", &a.q}, {"k", &a.k}, {"v", &a.v}}))) return rc;
  const FwdLayout L = fwd_layout(w, dtype);
  const hipStream_t st = as_stream(stream);
  if (L.total && (!ws || (uintptr_t(ws) & 255) || ws_bytes < L.total))
    return fail(DFS_EWORKSPACE, "%s: workspace of %zu bytes needed (256-byte aligned), got %zu", call, L.total, ws_bytes);
  auto by_type = [&](auto f) {
    auto d = [&](auto t) { w->d == 64 ? f(t, std::integral_constant<int, 64>{}) : f(t, std::integral_constant<int, 128>{}); };
    dtype == DFS_BF16 ? d(uint16_t{}) : d(float{});
  };
  if (L.splits) {
    a.set_blocks((int64_t(a.group) * a.n_q + 31) / 32);
    a.splits = L.splits;
    a.by_splits = Div(uint32_t(L.splits));
    a.part = static_cast<float*>(ws);
    a.part_sums = reinterpret_cast<float2*>(static_cast<char*>(ws) + L.sums);
    by_type([&](auto t, auto d) {
      using T = decltype(t);
      constexpr int D = decltype(d)::value;
      const unsigned grid = unsigned(L.blocks * L.splits);
      if (L.once) window_split_kernel<T, D, true, false><<<grid, 64 * split_waves<T, D>(), 0, st>>>(a);
      else window_split_kernel<T, D, false, false><<<grid, 64 * split_waves<T, D>(), 0, st>>>(a);
    });
    if (L.splits == 1) return launch_status(call);
    if ((rc = launch_status(call))) return rc;
    by_type([&](auto t, auto d) {
      constexpr int D = decltype(d)::value;
      window_join_kernel<decltype(t), D, false><<<unsigned(L.blocks * (D / 32)), 256, 0, st>>>(a);
    });
    return launch_status(call);
  }
  a.set_blocks((int64_t(a.group) * a.n_q + 127) / 128);
  const unsigned grid = unsigned(int64_t(a.blocks) * a.batch * a.heads_kv);
  if (dtype == DFS_BF16)
    w->d == 64 ? window_pipe_kernel<64, false><<<grid, 256, 0, st>>>(a) : window_pipe_kernel<128, false><<<grid, 256, 0, st>>>(a);
  else
    w->d == 64 ? window_f32_kernel<64, false><<<grid, 256, 0, st>>>(a) : window_f32_kernel<128, false><<<grid, 256, 0, st>>>(a);
  return launch_status(call);
}

int dfs_window_attn_bwd(const dfs_window* w, int dtype, const dfs_view* q, const dfs_view* k, const dfs_view* v, const dfs_view* o,
                        const float* lse, const dfs_view* d_o, const int32_t* q_len, const int32_t* k_len, float scale, const dfs_view* dq,
                        const dfs_view* dk, const dfs_view* dv, void* ws, size_t ws_bytes, void* stream) {
  const char* call = "dfs_window_attn_bwd";
  WindowArgs a = {};
  int rc = fill_window(call, w, dtype, q, k, v, o, false, lse, q_len, k_len, scale, &a);
  if (rc) return rc;
  if ((rc = check_view(call, "d_o", d_o, dtype, w->batch, w->heads, w->n_q, w->d, false, &a.d_o))) return rc;
  if ((rc = check_view(call, "dq", dq, dtype, w->batch, w->heads, w->n_q, w->d, true, &a.dq))) return rc;
  if ((rc = check_view(call, "dk", dk, dtype, w->batch, w->heads_kv, w->n_k, w->d, true, &a.dk))) return rc;
  if ((rc = check_view(call, "dv", dv, dtype, w->batch, w->heads_kv, w->n_k, w->d, true, &a.dv))) return rc;
  if ((rc = check_tiles(call, "q", a.q)) || (rc = check_tiles(call, "d_o", a.d_o))) return rc;
  if (!lse && w->batch && w->n_q) return fail(DFS_EINVAL, "%s: lse is NULL", call);
  const size_t need = dfs_window_workspace_bytes(w, dtype, 1);
  if (need && (!ws || (uintptr_t(ws) & 255) || ws_bytes < need))
    return fail(DFS_EWORKSPACE, "%s: workspace of %zu bytes needed (256-byte aligned), got %zu", call, need, ws_bytes);
  if (w->batch == 0) return DFS_OK;
  if ((rc = check_apart(call, {{"dq", &a.dq}, {"dk", &a.dk}, {"dv", &a.dv}}, {{"q", &a.q}, {"k", &a.k}, {"v", &a.v}, {"o", &a.o}, {"d_o", &a.d_o}}))) return rc;
  const BwdLayout L = bwd_layout(w);
  a.sums = static_cast<float2*>(ws);
  a.part = reinterpret_cast<float*>(static_cast<char*>(ws) + L.first);
  a.key_part = reinterpret_cast<float*>(static_cast<char*>(ws) + L.keys);
  a.row_part = reinterpret_cast<float*>(static_cast<char*>(ws) + L.rows);
  a.first_tiles = L.tiles;
  a.first_splits = L.splits;
  a.key_splits = L.key_splits;
  a.row_splits = L.row_splits;
  a.key_tiles = L.key_splits > 1 ? (a.n_k + 127) / 128 * 4 : L.tiles;
  return run_window_bwd(a, w->d, dtype, as_stream(stream));
}

}  // extern "C"
