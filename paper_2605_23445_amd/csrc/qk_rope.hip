// Norm of queries and keys for each head and their rotation by position, forward and backward.
//
// A row x of d channels becomes y = x r w with r = 1 / sqrt(mean(x^2) + eps), and every pair (a, b) of channels of y turns by an angle t =
// position * theta^(-2i/n): (a cos t - b sin t, a sin t + b cos t).  With g the gradient of the result turned back by t,
// dx = r (g w - x r^2 mean(g w x)) and dw = sum of g x r.  Everything is read once and written once: the kernels are bound by memory, and
// what they have to do is to keep enough rows in flight and the arithmetic out of the way.
//
// A lane owns 16 bytes of a row at one token and walks over heads: the angles depend on the token alone, so that their sines and cosines stay in
// registers and are worked out once for all heads.  The lanes of a row sit side by side and sum by lane exchanges.  Angles are
// counted in 2^-64 revolutions: whole ones fall out of an integer product of position and frequency, which is off by 2^-34 of one at the farthest.
// (An fp64 product of a frequency that is good to 2^-53 left sines and cosines of far positions off by up to 4.5 x 2^-24.)
#include "rope.h"

namespace dfs {

struct RopeRows {
  View in[3], out[3];                                // q, k, v; backward: rows of q and k
  View grad[3];                                      // backward: gradients of the results
  const int32_t* positions;
  int64_t pos_batch;
  const float* w[2];
  const int32_t* kv_start;
  int32_t batch, tokens, heads, heads_kv, rows_kv;   // rows_kv: rows of k's and v's output
  int32_t per;                                       // rows of all heads' that a work-group's y index takes
  int32_t copy_v;
  float* part;                                       // backward: sums of g x r of each work-group [groups][2][d]
};
struct RopeArgs : RopeRows, Turns {};

// What a lane keeps of its token: where the token is, and its turn.
template <typename T, int D, bool PAIRS> struct Token : Turn<T, D, PAIRS> {
  int b, t;
  bool real;
  __device__ __forceinline__ Token(const RopeArgs& a, int64_t slot, int lane) {
    const int64_t n = int64_t(a.batch) * a.tokens;
    real = slot < n;
    const uint32_t s = uint32_t(real ? slot : n - 1);
    b = int(s / uint32_t(a.tokens));
    t = int(s - uint32_t(b) * uint32_t(a.tokens));
    const int32_t* pos = a.positions + b * a.pos_batch + int64_t(t) * a.axes;
    const int32_t p0 = pos[0], p1 = a.axes > 1 ? pos[1] : 0, p2 = a.axes > 2 ? pos[2] : 0;
    this->set(a, lane, p0, p1, p2);
  }
};

// Forward.  Bound by memory: 75 600 tokens x 40 heads of q, k and v, bf16, d = 128: 833 us, 5.6 TB/s (a plain copy: 4.9); 2 642 tokens x 12, fp32, d = 64:
// 9.9 us, 4.9 TB/s; one token of 4 sequences, 32 + 8 heads, into a cache: 4.1 to 4.9 us, a launch.
template <typename T, int D, bool PAIRS, bool ONCE>
__global__ void __launch_bounds__(256) rope_kernel(RopeArgs a) {
  using Tok = Token<T, D, PAIRS>;
  constexpr int N = Tok::N, L = Tok::L, U = 2;       // U: rows in flight
  const int lane = threadIdx.x & 63;
  const Tok tok(a, (int64_t(blockIdx.x) * blockDim.x + threadIdx.x) / L, lane);
  const int h0 = blockIdx.y * a.per, h1 = h0 + a.per;
  const int64_t at = a.kv_start && tok.real ? int64_t(a.kv_start[tok.b]) + tok.t : tok.t;
  const bool in_room = tok.real && at >= 0 && at < a.rows_kv;
  float w[N];
  // Rows [from, to) of tensor `which`, whose rows begin at `base` of the walk over all heads.
  auto walk = [&](auto which, int base, int heads) __attribute__((always_inline)) {
    constexpr int X = decltype(which)::value;
    const int from = h0 > base ? h0 - base : 0, to = h1 - base < heads ? h1 - base : heads;
    if (from >= to) return;
    if constexpr (X < 2) weights<N>(a.w[X], tok.c, w);
    const char* src = a.in[X].at(tok.b, 0, tok.t) + tok.c * 16;
    char* dst = a.out[X].at(tok.b, 0, X ? (in_room ? at : 0) : tok.t) + tok.c * 16;
    const bool store = X ? in_room : tok.real;
    for (int h = from; h < to; h += U) {
      u32x4 raw[U];
#pragma unroll
      for (int u = 0; u < U; ++u) raw[u] = load_chunk<ONCE>(src + (h + u < to ? h + u : h) * a.in[X].head);
#pragma unroll
      for (int u = 0; u < U; ++u) {
        if (X < 2) {
          float x[N], sq = 0.f;
          Chunk<T>::open(raw[u], x);
#pragma unroll
          for (int i = 0; i < N; ++i) sq = fmaf(x[i], x[i], sq);
          const float r = rsqrtf(row_sum<L>(sq) * (1.f / D) + a.eps);
#pragma unroll
          for (int i = 0; i < N; ++i) x[i] = x[i] * r * w[i];
          tok.template rotate<false>(x);
          raw[u] = Chunk<T>::close(x);
        }
        if (store && h + u < to) __builtin_nontemporal_store(raw[u], reinterpret_cast<u32x4*>(dst + (h + u) * a.out[X].head));
      }
    }
  };
  walk(std::integral_constant<int, 0>{}, 0, a.heads);
  walk(std::integral_constant<int, 1>{}, a.heads, a.heads_kv);
  if (a.copy_v) walk(std::integral_constant<int, 2>{}, a.heads + a.heads_kv, a.heads_kv);
}

// Backward.  A work-group takes several groups of tokens, so that the sums for the weights leave it once; `part` holds a row of both for each
// work-group, which rope_sum_kernel adds up in a fixed order.  Bound by memory: 17 550 tokens x 40 heads, bf16, d = 128: 290 us with the sums' 6, 5.0 TB/s.
// Small calls do not fill this: 666 tokens x (12 + 2 x 4), fp32, d = 64, 16 us (12.3 in a graph), of which 11 are this kernel's, in runs of one row where the loop
// takes two, behind the angles, and 4.4 the sums'.
template <typename T, int D, bool PAIRS>
__global__ void __launch_bounds__(256) rope_bwd_kernel(RopeArgs a) {
  using Tok = Token<T, D, PAIRS>;
  constexpr int N = Tok::N, L = Tok::L, U = 2, SLOTS = 256 / L;
  const int lane = threadIdx.x & 63;
  const int h0 = blockIdx.y * a.per, h1 = h0 + a.per;
  const int64_t n = int64_t(a.batch) * a.tokens;
  float w[2][N], dw[2][N] = {};
  weights<N>(a.w[0], lane % L, w[0]);
  weights<N>(a.w[1], lane % L, w[1]);
  for (int64_t first = int64_t(blockIdx.x) * SLOTS; first < n; first += int64_t(gridDim.x) * SLOTS) {
    const Tok tok(a, first + threadIdx.x / L, lane);
    auto walk = [&](auto which, int base, int heads) __attribute__((always_inline)) {
      constexpr int X = decltype(which)::value;
      const int from = h0 > base ? h0 - base : 0, to = h1 - base < heads ? h1 - base : heads;
      const char* src = a.in[X].at(tok.b, 0, tok.t) + tok.c * 16;
      const char* up = a.grad[X].at(tok.b, 0, tok.t) + tok.c * 16;
      char* dst = a.out[X].at(tok.b, 0, tok.t) + tok.c * 16;
      for (int h = from; h < to; h += U) {
        u32x4 raw[U], graw[U];
#pragma unroll
        for (int u = 0; u < U; ++u) {
          const int hh = h + u < to ? h + u : h;
          if (X < 2) raw[u] = __builtin_nontemporal_load(reinterpret_cast<const u32x4*>(src + hh * a.in[X].head));
          graw[u] = __builtin_nontemporal_load(reinterpret_cast<const u32x4*>(up + hh * a.grad[X].head));
        }
#pragma unroll
        for (int u = 0; u < U; ++u) {
          const bool mine = tok.real && h + u < to;
          if (X < 2) {
            float x[N], g[N], sq = 0.f, gx = 0.f;
            Chunk<T>::open(raw[u], x);
            Chunk<T>::open(graw[u], g);
            tok.template rotate<true>(g);
#pragma unroll
            for (int i = 0; i < N; ++i) {
              sq = fmaf(x[i], x[i], sq);
              gx = fmaf(g[i] * w[X % 2][i], x[i], gx);
            }
            const float r = rsqrtf(row_sum<L>(sq) * (1.f / D) + a.eps);
            const float m = row_sum<L>(gx) * (1.f / D) * r * r;
#pragma unroll
            for (int i = 0; i < N; ++i) {
              if (mine) dw[X % 2][i] = fmaf(g[i], x[i] * r, dw[X % 2][i]);
              x[i] = r * (g[i] * w[X % 2][i] - x[i] * m);
            }
            graw[u] = Chunk<T>::close(x);
          }
          if (mine) __builtin_nontemporal_store(graw[u], reinterpret_cast<u32x4*>(dst + (h + u) * a.out[X].head));
        }
      }
    };
    walk(std::integral_constant<int, 0>{}, 0, a.heads);
    walk(std::integral_constant<int, 1>{}, a.heads, a.heads_kv);
    if (a.copy_v) walk(std::integral_constant<int, 2>{}, a.heads + a.heads_kv, a.heads_kv);
  }
  if (!a.part) return;
  __shared__ float sums[4][2][D];
#pragma unroll
  for (int X = 0; X < 2; ++X)
#pragma unroll
    for (int i = 0; i < N; ++i) {
      float s = dw[X][i];
#pragma unroll
      for (int m = L; m < 64; m *= 2) s += __shfl_xor(s, m);
      if (lane < L) sums[threadIdx.x >> 6][X][lane * N + i] = s;
    }
  __syncthreads();
  float* mine = a.part + (int64_t(blockIdx.y) * gridDim.x + blockIdx.x) * 2 * D;
  for (int i = threadIdx.x; i < 2 * D; i += 256)
    mine[i] = (sums[0][i / D][i % D] + sums[1][i / D][i % D]) + (sums[2][i / D][i % D] + sums[3][i / D][i % D]);
}

// dw[x][c] = sum of part[.][x][c]: 16 columns a work-group, 64 threads a column that take rows in turn.
__global__ void __launch_bounds__(1024) rope_sum_kernel(const float* __restrict__ part, int rows, int d, float* dw_q, float* dw_k) {
  __shared__ float sums[64][17];
  const int c = threadIdx.x & 15, t = threadIdx.x >> 4, col = blockIdx.x * 16 + c;
  float s = 0.f;
#pragma unroll 8
  for (int i = t; i < rows; i += 64) s += part[int64_t(i) * 2 * d + col];
  sums[t][c] = s;
  for (int m = 32; m > 0; m /= 2) {
    __syncthreads();
    if (t < m) sums[t][c] += sums[t + m][c];
  }
  float* out = col < d ? dw_q : dw_k;
  if (t == 0 && out) out[col % d] = sums[0][c];
}

// Rows of all heads' that a work-group walks over, at most: all tokens go through one run of heads before the next begins, so that memory is written in few
// streams (75 600 tokens x 40 heads of q, k and v: 10 rows 840 us, 5.5 TB/s, all 120 900).  Fewer cost the angles again, and more for shared key heads
// (4 x 16 384 tokens, 32 + 2 x 8 rows: 8 339, 10 315, 14 312).
constexpr int RUN = 10;
constexpr int BWD_GROUPS = 1024;                     // at most, of rope_bwd_kernel: rows that rope_sum_kernel adds up

// What both directions take of the geometry.
static int fill_qk(const char* call, const dfs_qk_geom* g, int dtype, const int32_t* positions, int64_t pos_batch, const float* w_q, const float* w_k,
                   RopeArgs* a) {
  if (dtype != DFS_F32 && dtype != DFS_BF16) return fail(DFS_EDTYPE, "%s: dtype %d is not DFS_F32 or DFS_BF16", call, dtype);
  if (misaligned(4, {positions, w_q, w_k})) return fail(DFS_EINVAL, "%s: positions and weights must be 4-byte aligned", call);
  if (!positions && g->batch && g->tokens) return fail(DFS_EINVAL, "%s: positions is NULL", call);
  if (pos_batch < 0 || pos_batch > (int64_t(1) << 40)) return fail(DFS_EINVAL, "%s: pos_batch=%lld", call, (long long)pos_batch);
  a->positions = positions;
  a->pos_batch = pos_batch;
  a->w[0] = w_q;
  a->w[1] = w_k;
  a->batch = g->batch;
  a->tokens = g->tokens;
  a->heads = g->heads;
  a->heads_kv = g->heads_kv;
  fill_turns(g, a);
  return DFS_OK;
}

template <typename F> static void by_type(const dfs_qk_geom* g, int dtype, F f) {
  auto d = [&](auto t) {
    auto p = [&](auto n) { g->interleaved ? f(t, n, std::true_type{}) : f(t, n, std::false_type{}); };
    g->d == 64 ? p(std::integral_constant<int, 64>{}) : p(std::integral_constant<int, 128>{});
  };
  dtype == DFS_BF16 ? d(uint16_t{}) : d(float{});
}

// Groups of tokens of the backward pass, and into how many runs the heads are split.
struct BwdGrid { int64_t x; int y, per; };
static BwdGrid bwd_grid(const dfs_qk_geom* g, int e) {
  const int slots = 256 / (g->d * e / 16), all = g->heads + 2 * g->heads_kv;
  BwdGrid r;
  r.x = (int64_t(g->batch) * g->tokens + slots - 1) / slots;
  int64_t y = r.x ? BWD_GROUPS / r.x : 1, runs = (all + RUN - 1) / RUN;
  if (y < runs) y = runs < BWD_GROUPS ? runs : BWD_GROUPS;
  if (y > all) y = all;
  r.per = int((all + y - 1) / y);
  r.y = (all + r.per - 1) / r.per;
  const int64_t most = BWD_GROUPS / r.y > 1 ? BWD_GROUPS / r.y : 1;
  if (r.x > most) r.x = most;
  return r;
}

}  // namespace dfs

using namespace dfs;

extern "C" {

int dfs_qk_norm_rope(const dfs_qk_geom* g, int dtype, const dfs_view* q, const dfs_view* k, const dfs_view* v, const int32_t* positions,
                     int64_t pos_batch, const float* w_q, const float* w_k, const dfs_view* q_out, const dfs_view* k_out,
                     const dfs_view* v_out, const int32_t* kv_start, int32_t kv_rows, void* stream) {
  const char* call = "dfs_qk_norm_rope";
  int rc = check_qk(call, g);
  if (rc) return rc;
  RopeArgs a = {};
  if ((rc = fill_qk(call, g, dtype, positions, pos_batch, w_q, w_k, &a))) return rc;
  if (!v != !v_out) return fail(DFS_EINVAL, "%s: v and v_out go together", call);
  if (misaligned(4, {kv_start})) return fail(DFS_EINVAL, "%s: kv_start must be 4-byte aligned", call);
  if (kv_start && kv_rows < 0) return fail(DFS_ESHAPE, "%s: kv_rows=%d is negative", call, kv_rows);
  a.kv_start = kv_start;
  a.rows_kv = kv_start ? kv_rows : g->tokens;
  a.copy_v = v != nullptr;
  const dfs_view *in[3] = {q, k, v}, *out[3] = {q_out, k_out, v_out};
  const char *in_name[3] = {"q", "k", "v"}, *out_name[3] = {"q_out", "k_out", "v_out"};
  for (int i = 0; i < 2 + a.copy_v; ++i) {
    const int heads = i ? g->heads_kv : g->heads;
    if ((rc = check_view(call, in_name[i], in[i], dtype, g->batch, heads, g->tokens, g->d, false, &a.in[i]))) return rc;
    if ((rc = check_view(call, out_name[i], out[i], dtype, g->batch, heads, i ? a.rows_kv : g->tokens, g->d, true, &a.out[i]))) return rc;
  }
  const int64_t n = int64_t(g->batch) * g->tokens;
  if (n == 0) return DFS_OK;
  for (int i = 0; i < 2 + a.copy_v; ++i)
    if (moved(a.in[i], a.out[i]) || (i && kv_start && a.in[i].data == a.out[i].data))
      return fail(DFS_EINVAL, "%s: %s is %s with rows elsewhere", call, out_name[i], in_name[i]);
  if ((rc = check_apart(call, {{"q_out", &a.out[0]}, {"k_out", &a.out[1]}, {"v_out", &a.out[2]}}, {})) ||
      (rc = check_apart(call, {{"q_out", &a.out[0]}}, {{"k", &a.in[1]}, {"v", &a.in[2]}})) ||
      (rc = check_apart(call, {{"k_out", &a.out[1]}}, {{"q", &a.in[0]}, {"v", &a.in[2]}})) ||
      (rc = check_apart(call, {{"v_out", &a.out[2]}}, {{"q", &a.in[0]}, {"k", &a.in[1]}})))
    return rc;
  const int L = g->d * elem_size(dtype) / 16, all = g->heads + (1 + a.copy_v) * g->heads_kv;
  // Work-groups of one wave and runs of heads until there are eight waves a SIMD, or a row a lane.
  const int64_t waves = (n * L + 63) / 64, bytes = n * all * L * 16;
  const int threads = waves * 4 >= 8192 ? 256 : 64;
  const bool once = bytes > int64_t(256) << 20;
  int64_t y = (8192 + waves - 1) / waves, runs = (all + RUN - 1) / RUN;
  if (y < runs) y = runs;
  if (y > all) y = all;
  a.per = int((all + y - 1) / y);
  const dim3 grid(unsigned((n * L + threads - 1) / threads), unsigned((all + a.per - 1) / a.per));
  by_type(g, dtype, [&](auto t, auto d, auto p) {
    using T = decltype(t);
    constexpr int D = decltype(d)::value;
    constexpr bool PAIRS = decltype(p)::value;
    if (once) rope_kernel<T, D, PAIRS, true><<<grid, threads, 0, as_stream(stream)>>>(a);
    else rope_kernel<T, D, PAIRS, false><<<grid, threads, 0, as_stream(stream)>>>(a);
  });
  return launch_status(call);
}

size_t dfs_qk_workspace_bytes(const dfs_qk_geom* g) {
  if (check_qk("dfs_qk_workspace_bytes", g) != DFS_OK) return 0;
  return align256(size_t(BWD_GROUPS) * 2 * g->d * sizeof(float));
}

int dfs_qk_norm_rope_bwd(const dfs_qk_geom* g, int dtype, const dfs_view* q, const dfs_view* k, const int32_t* positions, int64_t pos_batch,
                         const float* w_q, const float* w_k, const dfs_view* dq_out, const dfs_view* dk_out, const dfs_view* dv_out,
                         const dfs_view* dq, const dfs_view* dk, const dfs_view* dv, float* dw_q, float* dw_k, void* ws, size_t ws_bytes,
                         void* stream) {
  const char* call = "dfs_qk_norm_rope_bwd";
  int rc = check_qk(call, g);
  if (rc) return rc;
  RopeArgs a = {};
  if ((rc = fill_qk(call, g, dtype, positions, pos_batch, w_q, w_k, &a))) return rc;
  if (!dv != !dv_out) return fail(DFS_EINVAL, "%s: dv_out and dv go together", call);
  if (misaligned(4, {dw_q, dw_k})) return fail(DFS_EINVAL, "%s: dw_q and dw_k must be 4-byte aligned", call);
  a.copy_v = dv != nullptr;
  const dfs_view *in[2] = {q, k}, *up[3] = {dq_out, dk_out, dv_out}, *out[3] = {dq, dk, dv};
  const char *in_name[2] = {"q", "k"}, *up_name[3] = {"dq_out", "dk_out", "dv_out"}, *out_name[3] = {"dq", "dk", "dv"};
  for (int i = 0; i < 2 + a.copy_v; ++i) {
    const int heads = i ? g->heads_kv : g->heads;
    if (i < 2 && (rc = check_view(call, in_name[i], in[i], dtype, g->batch, heads, g->tokens, g->d, false, &a.in[i]))) return rc;
    if ((rc = check_view(call, up_name[i], up[i], dtype, g->batch, heads, g->tokens, g->d, false, &a.grad[i]))) return rc;
    if ((rc = check_view(call, out_name[i], out[i], dtype, g->batch, heads, g->tokens, g->d, true, &a.out[i]))) return rc;
  }
  for (int i = 0; i < 2 + a.copy_v; ++i)
    if (moved(a.grad[i], a.out[i])) return fail(DFS_EINVAL, "%s: %s is %s with rows elsewhere", call, out_name[i], up_name[i]);
  if (g->batch && g->tokens &&
      ((rc = check_apart(call, {{"dq", &a.out[0]}, {"dk", &a.out[1]}, {"dv", &a.out[2]}}, {{"q", &a.in[0]}, {"k", &a.in[1]}})) ||
       (rc = check_apart(call, {{"dq", &a.out[0]}}, {{"dk_out", &a.grad[1]}, {"dv_out", &a.grad[2]}})) ||
       (rc = check_apart(call, {{"dk", &a.out[1]}}, {{"dq_out", &a.grad[0]}, {"dv_out", &a.grad[2]}})) ||
       (rc = check_apart(call, {{"dv", &a.out[2]}}, {{"dq_out", &a.grad[0]}, {"dk_out", &a.grad[1]}}))))
    return rc;
  if (dw_q && dw_q == dw_k) return fail(DFS_EINVAL, "%s: dw_q and dw_k are the same memory", call);
  const bool sums = dw_q || dw_k;
  if (sums && (!ws || (uintptr_t(ws) & 255) || ws_bytes < dfs_qk_workspace_bytes(g)))
    return fail(DFS_EWORKSPACE, "%s: workspace of %zu bytes needed (256-byte aligned), got %zu", call, dfs_qk_workspace_bytes(g), ws_bytes);
  const BwdGrid grid = bwd_grid(g, elem_size(dtype));
  a.per = grid.per;
  a.part = sums ? static_cast<float*>(ws) : nullptr;
  const hipStream_t st = as_stream(stream);
  if (grid.x > 0) {
    by_type(g, dtype, [&](auto t, auto d, auto p) {
      rope_bwd_kernel<decltype(t), decltype(d)::value, decltype(p)::value><<<dim3(unsigned(grid.x), unsigned(grid.y)), 256, 0, st>>>(a);
    });
    if ((rc = launch_status(call))) return rc;
  }
  if (sums) rope_sum_kernel<<<2 * g->d / 16, 1024, 0, st>>>(a.part, int(grid.x * grid.y), g->d, dw_q, dw_k);
  return launch_status(call);
}

}  // extern "C"
