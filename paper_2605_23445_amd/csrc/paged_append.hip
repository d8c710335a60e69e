// New tokens on their way into a cache in pages: queries and keys normed and turned by their position, keys and values put into the pages of their sequence.
//
// The arithmetic of a row is that of qk_rope.hip.  Queries are worked on as there: a lane owns 16 bytes of a row at one token and walks over heads.  Keys and values
// are worked on page by page: a work-group takes the new rows of one page and key head, or, where they are few, a wave.  In 8 bits (e4m3, largest value 448) a page's rows share one power of two c,
// the smallest with which the largest of them is at most 448 c: it is known when all of a page's new rows are, which therefore stay in registers, and
// where there are rows from before it is not less than it was; if it grows they are divided by the quotient, which is exact but for what falls below e4m3's smallest.
// Bound by memory: 16 384 tokens of five prompts, 32 + 2 x 8 heads, d = 128, into e4m3 pages of 64 rows: 91 us, 4.05 TB/s (69 where the inputs are in the memory-side cache; a plain
// copy: 4.9); 5 130 x 3 x 12, d = 64, into bf16 pages of 16: 12 us, 3.9 TB/s.  The smallest calls are bound by the launch and a chain of loads (starts, lengths and rows, table,
// scale): one token of 32 sequences 6.2 us, of 128 7.4, of 512 18.5 (15.5 with seven waves a SIMD in place of the four that a whole page's rows in registers leave).
#include <float.h>

#include "pages.h"
#include "rope.h"
#include "seqs.h"

namespace dfs {

struct AppendArgs : Turns {
  View in[3], q_out;
  PageArgs pages;
  const int32_t *q_start, *k_len, *positions;
  const float* w[2];
  int32_t seqs, tokens, heads, heads_kv, norm;
  int32_t fours;                                     // work-groups of four pages
  int32_t q_groups, per;                             // work-groups of all tokens; heads that one walks over
  uint32_t page_share;                               // work-groups of pages in 8 bits out of all, in 2^-32, rounded up
};

// A sequence's new tokens: its first row, how many there are, and the position of the first.
struct Piece {
  int q0, n, begin;
  __device__ __forceinline__ Piece(const AppendArgs& a, int from, int to, int k_len) {
    q0 = from;
    n = max_of(0, to - from);
    begin = max_of(0, min_of(k_len, a.pages.row << a.pages.bits)) - n;
  }
  __device__ __forceinline__ Piece(const AppendArgs& a, int s) : Piece(a, start_of(a.q_start, s, a.tokens), start_of(a.q_start, s + 1, a.tokens), a.k_len[s]) {}
};

// Up to 64 sequences, one a lane.
struct Lanes {
  int from, to, k_len;
  __device__ __forceinline__ Lanes(const AppendArgs& a) {
    const int lane = threadIdx.x & 63, s = min_of(lane, a.seqs - 1);
    from = lane < a.seqs ? start_of(a.q_start, s, a.tokens) : a.tokens;
    to = start_of(a.q_start, s + 1, a.tokens);
    k_len = a.k_len[s];
  }
};

template <class Tok> __device__ __forceinline__ void set_turn(const AppendArgs& a, Tok& t, int lane, int row, int p) {
  if (a.positions) {
    const int32_t* pos = a.positions + int64_t(row) * a.axes;
    t.set(a, lane, pos[0], a.axes > 1 ? pos[1] : 0, a.axes > 2 ? pos[2] : 0);
  } else {
    t.set(a, lane, p, 0, 0);
  }
}

// Norm and turn of a chunk of a row.
template <typename T, int D, bool PAIRS>
__device__ __forceinline__ void norm_and_turn(const AppendArgs& a, const Turn<T, D, PAIRS, true>& t, const float (&w)[Chunk<T>::N], float (&x)[Chunk<T>::N]) {
  constexpr int N = Chunk<T>::N;
  if (a.norm) {
    float sq = 0.f;
#pragma unroll
    for (int i = 0; i < N; ++i) sq = fmaf(x[i], x[i], sq);
    const float r = rsqrtf(row_sum<D / N>(sq) * (1.f / D) + a.eps);
#pragma unroll
    for (int i = 0; i < N; ++i) x[i] = x[i] * r * w[i];
  }
  t.template rotate<false>(x);
}

// Rows of tokens, those of all heads in turn: queries and, where they are stored as they are (KV), keys and values.
template <typename T, int D, bool PAIRS, bool KV>
__device__ __forceinline__ void append_tokens(const AppendArgs& a, int id) {
  using Tok = Turn<T, D, PAIRS, true>;
  constexpr int N = Tok::N, L = Tok::L, U = 2;
  const int lane = threadIdx.x & 63, y = id / a.q_groups, x = id - y * a.q_groups, t = x * (256 / L) + threadIdx.x / L;
  const int row = min_of(t, a.tokens - 1), c16 = lane % L * 16, h0 = y * a.per, h1 = min_of(h0 + a.per, a.heads + (KV ? 2 * a.heads_kv : 0));
  const char* src[3];
#pragma unroll
  for (int i = 0; i < 3; ++i) src[i] = a.in[i].at(0, 0, row) + c16;
  auto which = [&](int h) { return !KV || h < a.heads ? 0 : h < a.heads + a.heads_kv ? 1 : 2; };
  int64_t step[3] = {a.in[0].head, a.in[1].head, a.in[2].head}, to_step[3] = {a.q_out.head, a.pages.k.head, a.pages.v.head};
#pragma unroll
  for (int i = 0; i < 3; ++i) asm volatile("" : "+s"(step[i]), "+s"(to_step[i]));         // or the compiler selects addresses of arguments, which it then copies to scratch
  auto load = [&](int h_) {
    const int h = min_of(h_, h1 - 1);
    const int i = which(h);
    return load_chunk<false>(i == 0 ? src[0] + h * step[0] : i == 1 ? src[1] + (h - a.heads) * step[1] : src[2] + (h - a.heads - a.heads_kv) * step[2]);
  };
  u32x4 next[U];                                     // asked for in front of everything that takes a trip to memory
#pragma unroll
  for (int u = 0; u < U; ++u) next[u] = load(h0 + u);
  float w[2][N];
  weights<N>(a.w[0], lane % L, w[0]);
  if (KV) weights<N>(a.w[1], lane % L, w[1]);
  // the last sequence that begins at or in front of this token
  int s = -1;
  if (a.seqs <= 64) {
    const Lanes all(a);
    const int first = __builtin_amdgcn_readfirstlane(row);
#pragma unroll
    for (int j = 0; j < 64 / L; ++j) {
      const int n = __builtin_popcountll(__builtin_amdgcn_ballot_w64(lane < a.seqs && all.from <= min_of(first + j, a.tokens - 1)));
      if (lane / L == j) s = n - 1;
    }
  } else {
    for (int lo = 0, hi = a.seqs; lo < hi;) {
      const int mid = (lo + hi) / 2;
      if (start_of(a.q_start, mid, a.tokens) <= row) {
        s = mid;
        lo = mid + 1;
      } else {
        hi = mid;
      }
    }
  }
  const Piece piece(a, max_of(s, 0));
  const bool real = t < a.tokens && s >= 0 && row - piece.q0 < piece.n && row >= piece.q0;
  const int p = piece.begin + row - piece.q0;
  Tok tok;
  set_turn(a, tok, lane, row, p);
  char* dst[3] = {a.q_out.at(0, 0, row) + c16, nullptr, nullptr};
  bool stored = false;                               // whether keys and values have a place
  if (KV) {
    const int page = real ? page_of(a.pages, max_of(s, 0), p >> a.pages.bits) : -1, in = p & ((1 << a.pages.bits) - 1);
    stored = page >= 0;
    dst[1] = a.pages.k.at(max_of(page, 0), 0, in) + c16;
    dst[2] = a.pages.v.at(max_of(page, 0), 0, in) + c16;
  }
  for (int h = h0; h < h1; h += U) {
    u32x4 raw[U];
#pragma unroll
    for (int u = 0; u < U; ++u) raw[u] = next[u];
    if (h + U < h1) {
#pragma unroll
      for (int u = 0; u < U; ++u) next[u] = load(h + U + u);
    }
#pragma unroll
    for (int u = 0; u < U; ++u) {
      if (h + u >= h1) break;
      const int i = which(h + u);
      if (i < 2) {
        float v[N];
        Chunk<T>::open(raw[u], v);
        if (i == 0) norm_and_turn<T, D, PAIRS>(a, tok, w[0], v);
        else norm_and_turn<T, D, PAIRS>(a, tok, w[1], v);
        raw[u] = Chunk<T>::close(v);
      }
      char* to = i == 0 ? dst[0] + (h + u) * to_step[0] : i == 1 ? dst[1] + (h + u - a.heads) * to_step[1] : dst[2] + (h + u - a.heads - a.heads_kv) * to_step[2];
      if (i == 0 ? real : stored) __builtin_nontemporal_store(raw[u], reinterpret_cast<u32x4*>(to));
    }
  }
}

// The new rows of a page: which sequence, page and key head, and the rows [r0, r1) of the page, row r at tensor row `row0` + r.
struct Fresh {
  bool real = false;                                 // (whether there is such a page is not known yet)
  int page, kvh, r0, r1, row0, p0;                   // p0: position of the page's row 0
  __device__ __forceinline__ Fresh(const AppendArgs& a, int id) {
    // A sequence has room for as many pages as whole ones lie between its start and the next one's, and two more.
    const int slot = id / a.heads_kv, bits = a.pages.bits;
    kvh = id - slot * a.heads_kv;
    int s;
    Piece piece(a, 0, 0, 0);
    if (a.seqs <= 64) {
      const Lanes all(a);
      const int lane = threadIdx.x & 63;
      s = __builtin_popcountll(__builtin_amdgcn_ballot_w64(lane < a.seqs && (all.from >> bits) + 2 * lane <= slot)) - 1;
      if (s < 0) return;
      piece = Piece(a, __builtin_amdgcn_readlane(all.from, s), __builtin_amdgcn_readlane(all.to, s), __builtin_amdgcn_readlane(all.k_len, s));
    } else {
      s = run_of(a.seqs, slot, [&](int x) { return (start_of(a.q_start, x, a.tokens) >> bits) + 2 * x; });
      if (s < 0) return;
      piece = Piece(a, s);
    }
    const int begin = max_of(piece.begin, 0), i = (begin >> bits) + slot - (piece.q0 >> bits) - 2 * s, end = piece.begin + piece.n;
    p0 = i << bits;
    if (i < begin >> bits || p0 >= end || end <= begin) return;          // (in front: where starts fall)
    page = page_of(a.pages, s, i);
    r0 = max_of(begin - p0, 0);
    r1 = min_of(end - p0, 1 << bits);
    row0 = piece.q0 + p0 - piece.begin;
    real = r0 < r1;
  }
};

// Exponent, as fp32 has it, of the smallest power of two c >= 2^-120 with m <= 448 c.
__device__ __forceinline__ int scale_exponent(float m) {
  const uint32_t b = __float_as_uint(m);
  return max_of(int(b >> 23) - 8 + ((b & 0x7FFFFFu) > 0x600000u), 7);
}
// The scale of rows from before, as reading takes it: of a number that is no power of two the exponent alone counts.
__device__ __forceinline__ float scale_of(float was) { return __uint_as_float(__float_as_uint(was) & 0x7F800000u); }
// Whether it stays where new rows take `scale`.  One that is not finite does not: its rows become NaN.
__device__ __forceinline__ bool stays(float was, float scale) { return was >= scale && was <= FLT_MAX; }
// Infinities and NaN do not count for a scale.
__device__ __forceinline__ float size_of(float x) { return fabsf(x) <= FLT_MAX ? fabsf(x) : 0.f; }
__device__ __forceinline__ uint32_t four_bytes(float a, float b, float c, float d) {
  return uint32_t(__builtin_amdgcn_cvt_pk_fp8_f32(c, d, __builtin_amdgcn_cvt_pk_fp8_f32(a, b, 0, false), true));
}

// Rows [0, n) of a page in 8 bits, times f, by `threads` of which this is number t.
template <int D> __device__ __forceinline__ void shrink(const View& v, int page, int kvh, int n, float f, int t, int threads) {
  for (int i = t; i < n * (D / 16); i += threads) {
    u32x4* p = reinterpret_cast<u32x4*>(v.at(page, kvh, i / (D / 16)) + i % (D / 16) * 16);
    u32x4 x = *p;
#pragma unroll
    for (int j = 0; j < 4; ++j) {
      const auto lo = __builtin_amdgcn_cvt_pk_f32_fp8(int(x[j]), false), hi = __builtin_amdgcn_cvt_pk_f32_fp8(int(x[j]), true);
      x[j] = four_bytes(lo[0] * f, lo[1] * f, hi[0] * f, hi[1] * f);
    }
    *p = x;
  }
}

// Rows in 8 bits; PASSES of 256 / L rows are a page.
template <int D, bool PAIRS, int PASSES>
__device__ __forceinline__ void append_bytes(const AppendArgs& a, int id) {
  using Tok = Turn<uint16_t, D, PAIRS, true>;
  constexpr int N = Tok::N, L = Tok::L, R = 256 / L;
  __shared__ float most[2][4];
  const Fresh f(a, id);
  if (!f.real) return;
  const int lane = threadIdx.x & 63, c = lane % L, mine = f.r0 + threadIdx.x / L;
  float w[N], y[PASSES][N], top[2] = {};
  u32x4 raw[PASSES], v[PASSES];
#pragma unroll
  for (int u = 0; u < PASSES; ++u) {
    if (f.r0 + u * R >= f.r1) continue;
    const int row = f.row0 + min_of(mine + u * R, f.r1 - 1);
    raw[u] = load_chunk<false>(a.in[1].at(0, f.kvh, row) + c * 16);
    v[u] = load_chunk<false>(a.in[2].at(0, f.kvh, row) + c * 16);
  }
  weights<N>(a.w[1], c, w);
  if (f.page < 0) return;
  const int scale_at = f.page * a.heads_kv + f.kvh;
  const float was[2] = {scale_of(a.pages.k_scale[scale_at]), scale_of(a.pages.v_scale[scale_at])};
#pragma unroll
  for (int u = 0; u < PASSES; ++u) {
    if (f.r0 + u * R >= f.r1) continue;
    const int at = min_of(mine + u * R, f.r1 - 1);   // past the last row that once more, which changes no maximum
    Tok tok;
    set_turn(a, tok, lane, f.row0 + at, f.p0 + at);
    Chunk<uint16_t>::open(raw[u], y[u]);
    norm_and_turn<uint16_t, D, PAIRS>(a, tok, w, y[u]);
    float z[N];
    Chunk<uint16_t>::open(v[u], z);
#pragma unroll
    for (int i = 0; i < N; ++i) {
      top[0] = fmaxf(top[0], size_of(y[u][i]));
      top[1] = fmaxf(top[1], size_of(z[i]));
    }
  }
#pragma unroll
  for (int x = 0; x < 2; ++x) {
#pragma unroll
    for (int m = 1; m < 64; m *= 2) top[x] = fmaxf(top[x], __shfl_xor(top[x], m));
    if (lane == 0) most[x][threadIdx.x >> 6] = top[x];
  }
  __syncthreads();
  float back[2];                                     // 1 / c
#pragma unroll
  for (int x = 0; x < 2; ++x) {
    const int e = scale_exponent(fmaxf(fmaxf(most[x][0], most[x][1]), fmaxf(most[x][2], most[x][3])));
    float scale = __uint_as_float(uint32_t(e) << 23);
    if (f.r0 > 0) {
      if (stays(was[x], scale)) scale = was[x];
      else shrink<D>(x ? a.pages.v : a.pages.k, f.page, f.kvh, f.r0, was[x] / scale, threadIdx.x, 256);
    }
    back[x] = 1.f / scale;
    if (threadIdx.x == 0) (x ? a.pages.v_scale : a.pages.k_scale)[scale_at] = scale;
  }
#pragma unroll
  for (int u = 0; u < PASSES; ++u) {
    const int r = mine + u * R;
    if (r >= f.r1) continue;
    float z[N];
    Chunk<uint16_t>::open(v[u], z);
#pragma unroll
    for (int i = 0; i < N; ++i) {
      y[u][i] *= back[0];
      z[i] *= back[1];
    }
    *reinterpret_cast<uint2*>(a.pages.k.at(f.page, f.kvh, r) + c * 8) =
        make_uint2(four_bytes(y[u][0], y[u][1], y[u][2], y[u][3]), four_bytes(y[u][4], y[u][5], y[u][6], y[u][7]));
    *reinterpret_cast<uint2*>(a.pages.v.at(f.page, f.kvh, r) + c * 8) = make_uint2(four_bytes(z[0], z[1], z[2], z[3]), four_bytes(z[4], z[5], z[6], z[7]));
  }
}

// The same by a wave, where a page's new rows are as many as a wave has at once; false: they are more, and nothing is done.
template <int D, bool PAIRS> __device__ __forceinline__ bool append_few_bytes(const AppendArgs& a, int id) {
  using Tok = Turn<uint16_t, D, PAIRS, true>;
  constexpr int N = Tok::N, L = Tok::L, R = 64 / L;
  const Fresh f(a, id);
  if (!f.real) return true;
  if (f.r1 - f.r0 > R) return false;
  const int lane = threadIdx.x & 63, c = lane % L, r = f.r0 + lane / L, at = min_of(r, f.r1 - 1);        // past the last row that once more
  float w[N], y[N], z[N], top[2] = {};
  const u32x4 raw = load_chunk<false>(a.in[1].at(0, f.kvh, f.row0 + at) + c * 16), v = load_chunk<false>(a.in[2].at(0, f.kvh, f.row0 + at) + c * 16);
  weights<N>(a.w[1], c, w);
  if (f.page < 0) return true;
  const int scale_at = f.page * a.heads_kv + f.kvh;
  const float was[2] = {scale_of(a.pages.k_scale[scale_at]), scale_of(a.pages.v_scale[scale_at])};
  Tok tok;
  set_turn(a, tok, lane, f.row0 + at, f.p0 + at);
  Chunk<uint16_t>::open(raw, y);
  norm_and_turn<uint16_t, D, PAIRS>(a, tok, w, y);
  Chunk<uint16_t>::open(v, z);
#pragma unroll
  for (int i = 0; i < N; ++i) {
    top[0] = fmaxf(top[0], size_of(y[i]));
    top[1] = fmaxf(top[1], size_of(z[i]));
  }
  float back[2];                                     // 1 / c
#pragma unroll
  for (int x = 0; x < 2; ++x) {
#pragma unroll
    for (int m = 1; m < 64; m *= 2) top[x] = fmaxf(top[x], __shfl_xor(top[x], m));
    float scale = __uint_as_float(uint32_t(scale_exponent(top[x])) << 23);
    if (f.r0 > 0) {
      if (stays(was[x], scale)) scale = was[x];
      else shrink<D>(x ? a.pages.v : a.pages.k, f.page, f.kvh, f.r0, was[x] / scale, lane, 64);
    }
    back[x] = 1.f / scale;
    if (lane == 0) (x ? a.pages.v_scale : a.pages.k_scale)[scale_at] = scale;
  }
  if (r >= f.r1) return true;
#pragma unroll
  for (int i = 0; i < N; ++i) {
    y[i] *= back[0];
    z[i] *= back[1];
  }
  *reinterpret_cast<uint2*>(a.pages.k.at(f.page, f.kvh, r) + c * 8) = make_uint2(four_bytes(y[0], y[1], y[2], y[3]), four_bytes(y[4], y[5], y[6], y[7]));
  *reinterpret_cast<uint2*>(a.pages.v.at(f.page, f.kvh, r) + c * 8) = make_uint2(four_bytes(z[0], z[1], z[2], z[3]), four_bytes(z[4], z[5], z[6], z[7]));
  return true;
}

// Four pages to a work-group, a wave for each; those with more rows one after the other by all of it.  The four are far apart, so that a prompt's pages among single tokens are
// many work-groups'.  (Past the last page there is no sequence's.)
template <int D, bool PAIRS, int PASSES>
__device__ __forceinline__ void append_four(const AppendArgs& a, int id) {
  __shared__ int more[4];
  const int wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
  const bool done = append_few_bytes<D, PAIRS>(a, wave * a.fours + id);
  more[wave] = 0;
  if (!done) more[wave] = 1;
  __syncthreads();
  for (int i = 0; i < 4; ++i)
    if (__builtin_amdgcn_readfirstlane(more[i])) {
      append_bytes<D, PAIRS, PASSES>(a, i * a.fours + id);
      __syncthreads();                               // what its waves told one another has been read
    }
}

// PASSES 0: pages of T; FOURS: in 8 bits, few new rows each.  The work-groups of pages, which compute more, are spread evenly among those of tokens, which move more.
template <typename T, int D, bool PAIRS, int PASSES, bool FOURS>
__global__ void __launch_bounds__(256) paged_append_kernel(AppendArgs a) {
  const int id = blockIdx.x;
  if constexpr (PASSES > 0) {
    const int pages = int(__umulhi(uint32_t(id), a.page_share));         // of the work-groups in front of this one
    if (int(__umulhi(uint32_t(id) + 1, a.page_share)) <= pages) append_tokens<T, D, PAIRS, false>(a, id - pages);
    else if constexpr (FOURS) append_four<D, PAIRS, PASSES>(a, pages);
    else append_bytes<D, PAIRS, PASSES>(a, pages);
  } else {
    append_tokens<T, D, PAIRS, true>(a, id);
  }
}

constexpr int RUN = 10;                              // rows that a work-group's lanes walk over, at most

}  // namespace dfs

using namespace dfs;

extern "C" {

int dfs_paged_append(const dfs_qk_geom* g, int dtype, const dfs_view* q, const dfs_view* k, const dfs_view* v, const int32_t* q_start, const int32_t* k_len,
                     const int32_t* positions, const float* w_q, const float* w_k, const dfs_view* q_out, const dfs_pages* pages, int norm, void* stream) {
  const char* call = "dfs_paged_append";
  if (!g) return fail(DFS_EINVAL, "%s: geometry pointer is NULL", call);
  if (g->batch < 0 || g->batch >= 1 << 24) return fail(DFS_ESHAPE, "%s: batch=%d sequences must be in [0, 2^24)", call, g->batch);
  dfs_qk_geom one = *g;
  one.batch = 1;
  int rc = check_qk(call, &one);
  if (rc) return rc;
  if (dtype != DFS_F32 && dtype != DFS_BF16) return fail(DFS_EDTYPE, "%s: dtype %d is not DFS_F32 or DFS_BF16", call, dtype);
  AppendArgs a = {};
  if (misaligned(4, {positions, w_q, w_k, q_start, k_len})) return fail(DFS_EINVAL, "%s: starts, lengths, positions and weights must be 4-byte aligned", call);
  if (g->batch && g->tokens && (!q_start || !k_len)) return fail(DFS_EINVAL, "%s: q_start or k_len is NULL", call);
  if (!positions && g->axes > 1) return fail(DFS_EINVAL, "%s: positions is NULL, which takes axes=1", call);
  if (!norm && (w_q || w_k)) return fail(DFS_EINVAL, "%s: weights without a norm", call);
  const dfs_view* in[3] = {q, k, v};
  const char* in_name[3] = {"q", "k", "v"};
  for (int i = 0; i < 3; ++i)
    if ((rc = check_view(call, in_name[i], in[i], dtype, 1, i ? g->heads_kv : g->heads, g->tokens, g->d, false, &a.in[i]))) return rc;
  if ((rc = check_view(call, "q_out", q_out, dtype, 1, g->heads, g->tokens, g->d, true, &a.q_out))) return rc;
  if ((rc = check_pages(call, pages, dtype, g->batch, g->heads_kv, g->d, true, &a.pages))) return rc;
  if (int64_t(a.pages.pages) * g->heads_kv >= int64_t(1) << 31) return fail(DFS_ESHAPE, "%s: pages=%d x heads_kv=%d too many", call, a.pages.pages, g->heads_kv);
  const int L = g->d * elem_size(dtype) / 16;
  const int64_t n = g->tokens, waves = (n * L + 63) / 64, slots = (n >> a.pages.bits) + 2 * int64_t(g->batch);
  if (slots * g->heads_kv >= 1 << 23) return fail(DFS_ESHAPE, "%s: tokens=%d, batch=%d x heads_kv=%d too large", call, g->tokens, g->batch, g->heads_kv);
  if (n == 0 || g->batch == 0) return DFS_OK;
  if (moved(a.in[0], a.q_out)) return fail(DFS_EINVAL, "%s: q_out is q with rows elsewhere", call);
  if ((rc = check_apart(call, {{"pages.k", &a.pages.k}, {"pages.v", &a.pages.v}}, {{"q", &a.in[0]}, {"k", &a.in[1]}, {"v", &a.in[2]}, {"q_out", &a.q_out}})) ||
      (rc = check_apart(call, {{"q_out", &a.q_out}}, {{"k", &a.in[1]}, {"v", &a.in[2]}})))
    return rc;
  fill_turns(g, &a);
  a.q_start = q_start;
  a.k_len = k_len;
  a.positions = positions;
  a.w[0] = w_q;
  a.w[1] = w_k;
  a.seqs = g->batch;
  a.tokens = g->tokens;
  a.heads = g->heads;
  a.heads_kv = g->heads_kv;
  a.norm = norm != 0;
  // runs of heads until there are eight waves a SIMD, or a row a lane
  const bool bytes = pages->dtype == DFS_E4M3;
  const int all = g->heads + (bytes ? 0 : 2 * g->heads_kv);
  int64_t y = (8192 + waves - 1) / waves, runs = (all + RUN - 1) / RUN;
  if (y < runs) y = runs;
  if (y > all) y = all;
  a.per = int((all + y - 1) / y);
  a.q_groups = int((n * L + 255) / 256);
  // A wave for a page where a sequence has no more rows on average than a wave has at once, else a work-group (us, wave against work-group, 8 key heads, d = 128, pages of 64 rows: one token
  // of 32 streams 6.2 / 6.7, of 128 7.4 / 12.3, of 512 18.5 / 35.8; four of 128 11.3 / 15.9, eight 29.4 / 19.5; d = 64, eight of 128 10.8 / 13.5, sixteen 27.2 / 17.5; one token of 127 and a
  // piece of 380 19.1 / 19.6).
  const bool few = bytes && n <= int64_t(g->batch) * (64 / L);
  const int64_t all_pages = bytes && a.pages.row ? slots * g->heads_kv : 0, page_blocks = few ? (all_pages + 3) / 4 : all_pages;
  a.fours = int(page_blocks);
  const int64_t blocks = int64_t(a.q_groups) * ((all + a.per - 1) / a.per) + page_blocks;
  if (blocks >= 1 << 24) return fail(DFS_ESHAPE, "%s: tokens=%d x heads=%d too large", call, g->tokens, g->heads);
  a.page_share = uint32_t(((uint64_t(page_blocks) << 32) + blocks - 1) / blocks);
  const int passes = !bytes ? 0 : pages->page * L / 256 > 1 ? pages->page * L / 256 : 1;
  const hipStream_t st = as_stream(stream);
  auto run = [&](auto t, auto d, auto p, auto s) {
    using T = decltype(t);
    constexpr int D = decltype(d)::value, PASSES = decltype(s)::value;
    constexpr bool PAIRS = decltype(p)::value;
    if constexpr (PASSES > 0)
      if (few) return paged_append_kernel<T, D, PAIRS, PASSES, true><<<unsigned(blocks), 256, 0, st>>>(a);
    paged_append_kernel<T, D, PAIRS, PASSES, false><<<unsigned(blocks), 256, 0, st>>>(a);
  };
  auto by_passes = [&](auto t, auto d, auto p) {
    if (!passes) run(t, d, p, std::integral_constant<int, 0>{});
    if constexpr (sizeof(t) == 2) {
      if (passes == 1) run(t, d, p, std::integral_constant<int, 1>{});
      if (passes == 2) run(t, d, p, std::integral_constant<int, 2>{});
      if (passes == 4) run(t, d, p, std::integral_constant<int, 4>{});
      if constexpr (decltype(d)::value == 128)
        if (passes == 8) run(t, d, p, std::integral_constant<int, 8>{});
    }
  };
  auto by_dim = [&](auto t) {
    auto p = [&](auto d) { g->interleaved ? by_passes(t, d, std::true_type{}) : by_passes(t, d, std::false_type{}); };
    g->d == 64 ? p(std::integral_constant<int, 64>{}) : p(std::integral_constant<int, 128>{});
  };
  dtype == DFS_BF16 ? by_dim(uint16_t{}) : by_dim(float{});
  return launch_status(call);
}

}  // extern "C"
