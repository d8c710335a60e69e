// Attention within packed sequences, of different lengths one behind the other: checks and launches.  The kernels are those of windowed attention, whose blocks
// of rows find their sequence on the device.
//
// Bound as these are.  Times of calls differ with the clock that a card grants, cycles do not.  Six causal prompts of 16 384 tokens, 32 heads of 8, d = 128: 402 to 421 us, 0.96 to
// 1.0 PFLOP/s, 0.77 million cycles of which the matrix cores are busy 52 %; three clips of 24 815 x 30, d = 64, both ways: 1 850 to 1 930 us, 880 to 920 TFLOP/s, 3.5 million, 48 %.
// Forward and backward of nine causal texts, 8 192 tokens x 32 heads of 8, d = 128: 437 to 471 us, of which under the profiler forward 95 to 99, dq 177 to 184 (39 %), dk and dv 199 to
// 203 (34 %): blocks meet 1 to 21 tiles of keys, 455 keys a row on average; the search for a block's sequence, the ends of blocks and the diagonal are a part of that.
//
// fp32: 701 tokens of five sequences x 4 heads of 2, d = 64: 11.1 us, a launch and two pieces of keys one after the other; forward and backward of 1 000 tokens of three x 12 of 4: 114
// us in five launches.  The forward one, 30 us, has 384 work-groups of 128 KB of LDS, one a CU: two rounds (of the same longest text beside shorter ones, 256 work-groups, 17 us; 384,
// 26.5).  dq, 39 us, is shared by two only, as a work-group's share is four tiles of keys at least; dk and dv take 35.
#include <math.h>

#include "window_fwd.h"

namespace dfs {

static int check_packed(const char* call, const dfs_packed* w, int dtype) {
  if (!w) return fail(DFS_EINVAL, "%s: geometry pointer is NULL", call);
  if (dtype != DFS_F32 && dtype != DFS_BF16) return fail(DFS_EDTYPE, "%s: dtype %d is not DFS_F32 or DFS_BF16", call, dtype);
  if (w->seqs < 0 || w->n_q < 0 || w->n_k < 0 || w->n_q > 1 << 28 || w->n_k > 1 << 28)
    return fail(DFS_ESHAPE, "%s: seqs=%d must not be negative, n_q=%d and n_k=%d be in [0, 2^28]", call, w->seqs, w->n_q, w->n_k);
  if (w->heads < 1 || w->heads_kv < 1 || w->heads > 65535 || w->heads % w->heads_kv)
    return fail(DFS_ESHAPE, "%s: heads=%d must be in [1, 65535] and a multiple of heads_kv=%d", call, w->heads, w->heads_kv);
  if (w->d != 64 && w->d != 128) return fail(DFS_ESHAPE, "%s: d=%d: head dimension must be 64 or 128", call, w->d);
  // rows are counted in 31 bits; a grid has fewer than 2^32 threads, 256 for a block of 128 rows or keys, of which each sequence may have one that is not full
  const int64_t rows = int64_t(w->heads / w->heads_kv) * w->n_q, most = rows > w->n_k ? rows : w->n_k;
  if (rows > int64_t(1) << 30 || w->seqs >= 1 << 24 || (most / 128 + w->seqs + 1) * w->heads_kv >= 1 << 24)
    return fail(DFS_ESHAPE, "%s: heads_kv=%d x rows of q or k, or seqs=%d, too large", call, w->heads_kv, w->seqs);
  return DFS_OK;
}

// What the host knows of the lengths, which are on the device: a sequence has the mean of all, and hardly more than twice that.
static int64_t likely(int64_t n, const dfs_packed* w) {
  const int64_t twice = w->seqs ? 2 * ((n + w->seqs - 1) / w->seqs) : 0;
  return twice < n ? twice : n;
}

// As for sequences of one length: work-groups share the queries of a block of keys, or the keys of a block of rows, where these are few.
struct PackedBwd { size_t keys, rows, total; int key_splits, row_splits, query_groups; int64_t key_tiles; };
static PackedBwd bwd_layout(const dfs_packed* w, int dtype) {
  PackedBwd L;
  const int64_t group = w->heads / w->heads_kv, rows = group * w->n_q, part = 64 * w->d * sizeof(float);
  const int64_t reach = w->left < 0 || w->right < 0 ? int64_t(1) << 40 : int64_t(w->left) + w->right + 128;
  const int64_t key_blocks = (w->n_k / 128 + w->seqs) * int64_t(w->heads_kv), row_blocks = (rows / 128 + w->seqs) * int64_t(w->heads_kv);
  const int64_t q = likely(w->n_q, w), k = likely(w->n_k, w);
  // Twice as many as where all blocks have the same work: under a causal mask half of them have little (1 000 fp32 tokens of three sequences x 12 heads of 4: 122 -> 106 us).  For the same
  // reason up to 340 blocks of keys, a little more than run at once, are shared by three (us, 1 / 3 work-groups: 4 000 causal tokens of three x 32 heads of 8, d = 128, 272 blocks, 360 / 298,
  // fp32 3 833 / 2 520; 9 000 of six x 32 of 4, d = 64, 304, 480 / 397; 5 000 of two that see all of theirs, 328, 1 284 / 1 154), and in fp32, where a CU has one work-group, up to 512
  // by two (2 000 of five x 24, d = 64, 480 blocks: bf16 70 / 80, fp32 342 / 323; 6 000 of four x 32 of 8 with a window of 300, 400: 152 / 156, 1 017 / 888).  In bf16 a block has to have the
  // work for it: 96 tiles of 32 queries (3 000 of two x 12 with a window of 200, 10 tiles, 90 / 106; 3 000 of eight x 16 of 8, 48, 63 / 64; 2 500 of four x 24 of 8, 117, 131 / 122).
  const int64_t tiles = ((reach < q ? reach : q) + 31) / 32 * group;
  const int64_t even = dtype == DFS_F32 ? (key_blocks <= 340 ? 3 : key_blocks <= 512 ? 2 : 1) : key_blocks <= 340 && tiles >= 96 ? 3 : 1;
  L.key_splits = share(key_blocks, tiles, even * key_blocks > 512 ? even * key_blocks : 512);
  L.row_splits = share(row_blocks, ((reach < k ? reach : k) + 63) / 64, 512);
  // Under a causal mask the blocks of the first keys have several times the work of others; where all blocks run at once, or nearly so, the longest one is what the call waits for (us, two
  // groups of waves against one, d = 128, 32 heads of 8: 12 000 tokens of five texts, 800 blocks, 1 356 / 1 385; 16 000, 1 040, 2 335 / 2 239; 9 000 tokens of two x 12 that see all of
  // theirs 1 560 / 1 470).
  L.query_groups = w->left < 0 && w->right >= 0 && L.key_splits == 1 && key_blocks <= 900 ? 2 : 1;
  L.key_tiles = L.key_splits > 1 ? (int64_t(w->n_k) / 128 + w->seqs) * 4 : 0;
  L.keys = align256(size_t(w->heads) * w->n_q * sizeof(float2));
  L.rows = L.keys + (L.key_splits > 1 ? size_t(key_blocks) * 4 * L.key_splits * part : 0);
  L.total = L.rows + (L.row_splits > 1 ? size_t(row_blocks) * 4 * L.row_splits * (part / 2 + 64 * sizeof(float)) : 0);
  return L;
}

// The forward pass: into how many work-groups the keys of 32 rows are split; 0: not split, blocks of 128 rows.
struct PackedFwd { size_t sums, total; int64_t blocks; int splits; };
static PackedFwd fwd_layout(const dfs_packed* w, int dtype) {
  const int64_t group = w->heads / w->heads_kv, rows = group * w->n_q, some_seqs = w->seqs < w->n_q ? w->seqs : w->n_q;
  PackedFwd L = {0, 0, (rows / 32 + w->seqs) * w->heads_kv, 0};
  // Blocks of 128 rows need enough of them (us, blocks of 128 against split; causal: 1 431 tokens of two sequences x 5 heads, d = 128, 65 blocks, 20.6 / 13.5; 1 500 x 8,
  // 96, 29.4 / 29.1; 1 000 of four x 16 heads of 4, 140, 12.2 / 16.8; d = 64: 1 770 of three x 9 of 3, 132, 15.1 / 11.0; 1 500 x 16, 192, 24.0 / 24.4; 2 000 of
  // six x 12, 252, 11.9 / 15.2; fp32, d = 64: 2 000 x 16 of 4, 252, 181 / 142; 1 000 of four x 32 of 8, 280, 43 / 49).
  if (rows > 32 && (rows / 128 + some_seqs) * w->heads_kv > (w->d == 128 ? 96 : dtype == DFS_F32 ? 256 : 192)) return L;
  // Sequences without rows have room for a block as well: so many of them that blocks of 32 rows pass a grid's 2^32 threads leave those of 128, which the checks have counted.
  if (L.blocks >= 1 << 24) return L;
  const int waves = dtype == DFS_F32 && w->d == 128 ? 2 : 4;
  int64_t keys = likely(w->n_k, w);
  const int64_t reach = int64_t(w->left) + w->right + 32 / group + 1;
  if (w->left >= 0 && w->right >= 0 && reach < keys) keys = reach;
  const int64_t tiles = (keys + 31) / 32, by_waves = (tiles + waves - 1) / waves, some = L.blocks ? 128 / L.blocks : 1;
  const int64_t splits = some < by_waves ? some : by_waves;
  L.splits = splits < 1 ? 1 : int(splits);
  if (L.splits > 1) {
    L.sums = align256(size_t(L.blocks) * L.splits * 32 * w->d * sizeof(float));
    L.total = L.sums + size_t(L.blocks) * L.splits * 32 * sizeof(float2);
  }
  return L;
}

static int fill_packed(const char* call, const dfs_packed* w, int dtype, const dfs_view* q, const dfs_view* k, const dfs_view* v, const dfs_view* o, bool o_out,
                       const float* lse, const int32_t* q_start, const int32_t* k_start, float scale, WindowArgs* a) {
  int rc = check_packed(call, w, dtype);
  if (rc) return rc;
  if (!(scale > 0.f) || !isfinite(scale)) return fail(DFS_EINVAL, "%s: scale must be positive and finite", call);
  if (misaligned(4, {lse, q_start, k_start})) return fail(DFS_EINVAL, "%s: lse and starts must be 4-byte aligned", call);
  if (!q_start && w->seqs) return fail(DFS_EINVAL, "%s: q_start is NULL", call);
  if (!k_start && w->n_k != w->n_q) return fail(DFS_ESHAPE, "%s: n_k=%d and n_q=%d must be the same where k_start is NULL", call, w->n_k, w->n_q);
  if ((rc = check_view(call, "q", q, dtype, 1, w->heads, w->n_q, w->d, false, &a->q))) return rc;
  if ((rc = check_view(call, "k", k, dtype, 1, w->heads_kv, w->n_k, w->d, false, &a->k))) return rc;
  if ((rc = check_view(call, "v", v, dtype, 1, w->heads_kv, w->n_k, w->d, false, &a->v))) return rc;
  if ((rc = check_view(call, "o", o, dtype, 1, w->heads, w->n_q, w->d, o_out, &a->o))) return rc;
  if ((rc = check_tiles(call, "k", a->k)) || (rc = check_tiles(call, "v", a->v))) return rc;
  a->lse = const_cast<float*>(lse);
  a->q_start = q_start;
  a->k_start = k_start ? k_start : q_start;
  a->packed = w->seqs;
  a->batch = 1;
  a->heads = w->heads;
  a->heads_kv = w->heads_kv;
  a->group = w->heads / w->heads_kv;
  a->seqs = w->heads_kv;
  a->by_kv = Div(uint32_t(w->heads_kv));
  a->by_group = Div(uint32_t(a->group));
  a->n_q = w->n_q;
  a->n_k = w->n_k;
  a->left = w->left < 0 || w->left > NO_LIMIT ? NO_LIMIT : w->left;
  a->right = w->right < 0 || w->right > NO_LIMIT ? NO_LIMIT : w->right;
  a->scale = scale;
  return DFS_OK;
}

static int check_scratch(const char* call, size_t need, const void* ws, size_t ws_bytes) {
  if (need && (!ws || (uintptr_t(ws) & 255) || ws_bytes < need))
    return fail(DFS_EWORKSPACE, "%s: workspace of %zu bytes needed (256-byte aligned), got %zu", call, need, ws_bytes);
  return DFS_OK;
}

}  // namespace dfs

using namespace dfs;

extern "C" {

size_t dfs_packed_workspace_bytes(const dfs_packed* w, int dtype, int backward) {
  if (check_packed("dfs_packed_workspace_bytes", w, dtype) != DFS_OK) return 0;
  return backward ? bwd_layout(w, dtype).total : fwd_layout(w, dtype).total;
}

int dfs_packed_attn_fwd(const dfs_packed* w, int dtype, const dfs_view* q, const dfs_view* k, const dfs_view* v, const int32_t* q_start,
                        const int32_t* k_start, float scale, const dfs_view* o, float* lse, void* ws, size_t ws_bytes, void* stream) {
  const char* call = "dfs_packed_attn_fwd";
  WindowArgs a = {};
  int rc = fill_packed(call, w, dtype, q, k, v, o, true, lse, q_start, k_start, scale, &a);
  if (rc) return rc;
  const PackedFwd L = fwd_layout(w, dtype);
  if ((rc = check_scratch(call, L.total, ws, ws_bytes))) return rc;
  if (w->seqs == 0 || w->n_q == 0) return DFS_OK;
  if ((rc = check_apart(call, {{"o", &a.o}}, {{"q", &a.q}, {"k", &a.k}, {"v", &a.v}}))) return rc;
  const hipStream_t st = as_stream(stream);
  if (!L.splits) {
    a.set_blocks(int64_t(a.group) * a.n_q / 128 + a.packed);
    const unsigned grid = unsigned(int64_t(a.blocks) * a.heads_kv);
    if (dtype == DFS_BF16)
      w->d == 64 ? window_pipe_kernel<64, true><<<grid, 256, 0, st>>>(a) : window_pipe_kernel<128, true><<<grid, 256, 0, st>>>(a);
    else
      w->d == 64 ? window_f32_kernel<64, true><<<grid, 256, 0, st>>>(a) : window_f32_kernel<128, true><<<grid, 256, 0, st>>>(a);
    return launch_status(call);
  }
  auto by_type = [&](auto f) {
    auto d = [&](auto t) { w->d == 64 ? f(t, std::integral_constant<int, 64>{}) : f(t, std::integral_constant<int, 128>{}); };
    dtype == DFS_BF16 ? d(uint16_t{}) : d(float{});
  };
  a.set_blocks(int64_t(a.group) * a.n_q / 32 + a.packed);
  a.splits = L.splits;
  a.by_splits = Div(uint32_t(L.splits));
  a.part = static_cast<float*>(ws);
  a.part_sums = reinterpret_cast<float2*>(static_cast<char*>(ws) + L.sums);
  by_type([&](auto t, auto d) {
    using T = decltype(t);
    constexpr int D = decltype(d)::value;
    window_split_kernel<T, D, false, true><<<unsigned(L.blocks * L.splits), 64 * split_waves<T, D>(), 0, st>>>(a);
  });
  if ((rc = launch_status(call)) || L.splits == 1) return rc;
  by_type([&](auto t, auto d) {
    constexpr int D = decltype(d)::value;
    window_join_kernel<decltype(t), D, true><<<unsigned(L.blocks * (D / 32)), 256, 0, st>>>(a);
  });
  return launch_status(call);
}

int dfs_packed_attn_bwd(const dfs_packed* w, int dtype, const dfs_view* q, const dfs_view* k, const dfs_view* v, const dfs_view* o, const float* lse,
                        const dfs_view* d_o, const int32_t* q_start, const int32_t* k_start, float scale, const dfs_view* dq, const dfs_view* dk,
                        const dfs_view* dv, void* ws, size_t ws_bytes, void* stream) {
  const char* call = "dfs_packed_attn_bwd";
  WindowArgs a = {};
  int rc = fill_packed(call, w, dtype, q, k, v, o, false, lse, q_start, k_start, scale, &a);
  if (rc) return rc;
  if ((rc = check_view(call, "d_o", d_o, dtype, 1, w->heads, w->n_q, w->d, false, &a.d_o))) return rc;
  if ((rc = check_view(call, "dq", dq, dtype, 1, w->heads, w->n_q, w->d, true, &a.dq))) return rc;
  if ((rc = check_view(call, "dk", dk, dtype, 1, w->heads_kv, w->n_k, w->d, true, &a.dk))) return rc;
  if ((rc = check_view(call, "dv", dv, dtype, 1, w->heads_kv, w->n_k, w->d, true, &a.dv))) return rc;
  if ((rc = check_tiles(call, "q", a.q)) || (rc = check_tiles(call, "d_o", a.d_o))) return rc;
  if (!lse && w->seqs && w->n_q) return fail(DFS_EINVAL, "%s: lse is NULL", call);
  const PackedBwd L = bwd_layout(w, dtype);
  if ((rc = check_scratch(call, L.total, ws, ws_bytes))) return rc;
  if (w->seqs == 0) return DFS_OK;
  if ((rc = check_apart(call, {{"dq", &a.dq}, {"dk", &a.dk}, {"dv", &a.dv}}, {{"q", &a.q}, {"k", &a.k}, {"v", &a.v}, {"o", &a.o}, {"d_o", &a.d_o}}))) return rc;
  a.sums = static_cast<float2*>(ws);
  a.key_part = reinterpret_cast<float*>(static_cast<char*>(ws) + L.keys);
  a.row_part = reinterpret_cast<float*>(static_cast<char*>(ws) + L.rows);
  a.first_splits = 1;
  a.key_splits = L.key_splits;
  a.query_groups = L.query_groups;
  a.row_splits = L.row_splits;
  a.key_tiles = int32_t(L.key_tiles);
  return run_packed_bwd(a, w->d, dtype, as_stream(stream));
}

}  // extern "C"
