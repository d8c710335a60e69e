// Kernels of attention over a window around each query's position and a few first keys, of sequences of one length, of packed ones, or of
// packed rows over a cache in pages (KIND).
//
// The rows of a work-group are queries of ALL heads that share a key head, query by query (row r is head r % group of query r / group): a tile of
// keys and values is brought in once for the group, and a block of rows spans fewer positions, so that it meets fewer tiles of which it
// sees only a part.  Keys come in pieces of 32 rows: first those of the first keys that lie in front of the block's window, then the window's, from its
// first key on.
#pragma once
#include <float.h>
#include <math.h>

#include "window.h"

namespace dfs {

constexpr int KN = 64;                               // keys of a tile

// How tiles of 64 keys and values come to LDS: rows of tensors, straight.
template <typename T, int D> struct RowFeed {
  static constexpr int STEP = 1;                     // what a window's first piece begins at a multiple of
  static constexpr bool STRAIGHT = true;
  using KLoader = typename Tile<T, D, KN, 4, false>::Loader;
  using VLoader = typename Tile<T, D, KN, 4, true>::Loader;
  const char *kh, *vh;
  int64_t k_row, v_row;
  KLoader k_load;
  VLoader v_load;
  template <class P, class S> __device__ __forceinline__ RowFeed(const WindowArgs& a, const P& at, const S& seq, const Span&, int wave, int lane)
      : kh(a.k.at(at.b, at.kvh, seq.k0)), vh(a.v.at(at.b, at.kvh, seq.k0)), k_row(a.k.row), v_row(a.v.row), k_load(a.k.row, wave, lane), v_load(a.v.row, wave, lane) {}
  __device__ __forceinline__ typename KLoader::Pair keys(const Span& span, int t) { return k_load.of(span, kh, k_row, t); }
  __device__ __forceinline__ typename VLoader::Pair values(const Span& span, int t) { return v_load.of(span, vh, v_row, t); }
  __device__ __forceinline__ void ask_keys(const typename KLoader::Pair& p, uint32_t to, int j) const { k_load.issue_one(p, to, j); }
  __device__ __forceinline__ void ask_values(const typename VLoader::Pair& p, uint32_t to, int j) const { v_load.issue_one(p, to, j); }
};

// f32: one step per tile of 64 keys, bound by the fp32 matrix instructions and by what their waves wait for in between, one thing after the other in two
// work-groups a CU at d = 64 and in one, which fills the LDS, at d = 128: 4 000 tokens x 16 heads, 1 000 keys each way, d = 64: 323 to 340 us, 85 to 89 TFLOP/s,
// matrix cores busy 60 % of the cycles; d = 128: 755 us, 76 TFLOP/s, 52 % (a large fp32 product of a library: 154).
template <int D, int KIND, class Feed = RowFeed<float, D>, class Args = WindowArgs>
__global__ void __launch_bounds__(256) window_f32_kernel(Args a) {
  using T = float;
  constexpr int NW = 4, BM = 32 * NW;
  using KTile = Tile<T, D, KN, NW, false>;
  using VTile = Tile<T, D, KN, NW, true>;
  constexpr int STEPS = KTile::STEPS;
  __shared__ __attribute__((aligned(1024))) char tiles[4 * KTile::BYTES];
  const uint32_t lds = uint32_t(reinterpret_cast<uintptr_t>((LDS_PTR(void))(tiles)));
  const int lane = threadIdx.x & 63, wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);

  const PlaceOf<KIND> at(a, blockIdx.x);
  const auto seq = Seq<KIND>::template of<BM, false>(a, at.b, at.blk, true);
  if (!seq.real) return;
  const Lengths& len = seq.len;
  const int r0 = seq.blk * BM, rows = rows_of(a, len, r0, BM);
  if (rows <= 0) return;
  const Row row(a, at, len, r0, rows, wave * 32 + (lane & 31), lane);
  const Span span(a, row.i0 + len.shift, row.i1 + len.shift, len.k, Feed::STEP);
  const int n_tiles = (span.n + 1) / 2;
  typename Mat<T>::Frag qf[STEPS];
  {
    const char* qp = a.q.at(at.b, row.qh, seq.q0 + row.qi);
#pragma unroll
    for (int s = 0; s < STEPS; ++s) qf[s] = *reinterpret_cast<const typename Mat<T>::Frag*>(qp + (2 * s + row.h) * 16);
  }
  Feed feed(a, at, seq, span, wave, lane);
  const typename KTile::RowReader k_read(lane);
  const typename VTile::ColumnReader v_read(lane);
  const uint32_t to = __builtin_amdgcn_readfirstlane(lds + uint32_t(wave) * 1024);
  auto issue = [&](int t) {
    const uint32_t buf = to + uint32_t((t & 1) * 2 * KTile::BYTES);
    const auto ks = feed.keys(span, t);
    const auto vs = feed.values(span, t);
#pragma unroll
    for (int j = 0; j < KTile::LOADS; ++j) feed.ask_keys(ks, buf, j);
#pragma unroll
    for (int j = 0; j < KTile::LOADS; ++j) feed.ask_values(vs, buf + KTile::BYTES, j);
  };

  f32x16 acc[D / 32];
  clear(acc);
  float m = -INFINITY, l = 0.f;                      // row maximum in the base-2 exponent's units, this lane's share of the row sum
  const float c2 = a.scale * LOG2E;
  if (n_tiles > 0) issue(0);
  for (int t = 0; t < n_tiles; ++t) {
    wait_loads();
    __syncthreads();                                 // tile t is there, and the buffers of tile t - 1 are free
    if (t + 1 < n_tiles) issue(t + 1);
    const uint32_t buf = lds + uint32_t((t & 1) * 2 * KTile::BYTES);
    f32x16 s[2];
    clear(s);
#pragma unroll
    for (int half = 0; half < 2; ++half) {
#pragma unroll
      for (int st = 0; st < STEPS; ++st) s[half] = Mat<T>::mma(k_read.get(buf, half, st), qf[st], s[half]);
      if (!span.whole(2 * t + half)) span.mask(a, 2 * t + half, row.p, row.h, s[half], -INFINITY);
    }
    float mx = s[0][0];
#pragma unroll
    for (int i = 0; i < 16; ++i) mx = fmaxf(mx, fmaxf(s[0][i], s[1][i]));
    const auto sw = __builtin_amdgcn_permlane32_swap(__float_as_uint(mx), __float_as_uint(mx), false, false);
    mx = fmaxf(__uint_as_float(sw[0]), __uint_as_float(sw[1])) * c2;
    const float m_new = fmaxf(m, mx), ref = m_new == -INFINITY ? 0.f : m_new;
    if (__builtin_amdgcn_ballot_w64(m_new > m)) {
      const float alpha = __builtin_amdgcn_exp2f(m - ref);
      m = m_new;
      l *= alpha;
#pragma unroll
      for (int c = 0; c < D / 32; ++c)
#pragma unroll
        for (int i = 0; i < 16; ++i) acc[c][i] *= alpha;
    }
#pragma unroll
    for (int half = 0; half < 2; ++half) {
#pragma unroll
      for (int i = 0; i < 16; ++i) {
        s[half][i] = __builtin_amdgcn_exp2f(fmaf(s[half][i], c2, -ref));
        l += s[half][i];
      }
      Weights<T> w;
      w.set(s[half]);
      v_read.mma(buf + KTile::BYTES, half, w, acc);
    }
  }
  const auto sw = __builtin_amdgcn_permlane32_swap(__float_as_uint(l), __float_as_uint(l), false, false);
  l = __uint_as_float(sw[0]) + __uint_as_float(sw[1]);
  store_row<T>(row.real, a.o.at(at.b, row.qh, seq.q0 + row.qi), acc, l == 0.f ? 0.f : 1.f / l, row.h);
  if (row.real && a.lse && row.h == 0) a.lse[(int64_t(at.b) * a.heads + row.qh) * a.n_q + seq.q0 + row.qi] = l == 0.f ? -INFINITY : (m + __builtin_amdgcn_logf(l)) * (1.f / LOG2E);
}

// bf16: a pipeline over pieces of 32 keys, two to a tile.  In one stage the matrix cores form the logits of the piece two ahead and the product of the previous
// one's weights with its values, while the vector units turn the logits of the piece between them into weights; scheduling fences keep matrix and vector
// instructions side by side.  K(t + 2) and V(t + 1) are asked for in tile t's first stage and have a whole tile to come.
//
// A row's weights are taken against a reference that is its largest logit's so far to start with and moves where weights have become large: the sums of a
// lane's weights, which are needed anyway, tell at the cost of a comparison.
//
// Weights are rounded to one bf16 term for the product with the values, which leaves o 2.2e-3 from 64 bits in 2-norm where rounding the result alone costs
// 1.65e-3; their sum is of the unrounded ones.  A second term would be half as many matrix instructions again in a kernel that these bound.
//
// Bound by the matrix cores and the vector port beside them.  d = 128: 75 600 tokens x 40 heads, 3 600 keys each way: 9.6 ms, 1 133 TFLOP/s, matrix cores
// busy 65 % of the cycles at 1.67 GHz; 2 x 8 192 x 32 heads of 8 key heads, 1 024 keys back: 298 us, 868 TFLOP/s, 45 %: a block meets 17 tiles, and its start,
// the first tiles' way and the end are a part of its time.  d = 64: 17 550 x 30, 1 350 each way: 433 us, 813 TFLOP/s, 43 %.
template <int D, int KIND, class Feed = RowFeed<uint16_t, D>, class Args = WindowArgs>
__global__ void __launch_bounds__(256, 2) window_pipe_kernel(Args a) {
  constexpr int NW = 4, BM = 32 * NW;
  using KTile = Tile<uint16_t, D, KN, NW, false>;
  using VTile = Tile<uint16_t, D, KN, NW, true>;
  constexpr int STEPS = KTile::STEPS, CS = D / 32, LOADS = KTile::LOADS, BYTES = KTile::BYTES;
  constexpr float SUM_LIMIT = 64.f;                  // of the sixteen weights of a piece that a lane works out
  // K of even tiles, of odd ones, V of even ones, of odd ones
  __shared__ __attribute__((aligned(1024))) char tiles[4 * BYTES];
  const uint32_t lds = uint32_t(reinterpret_cast<uintptr_t>((LDS_PTR(void))(tiles)));
  const int lane = threadIdx.x & 63, wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);

  const PlaceOf<KIND> at(a, blockIdx.x);
  const auto seq = Seq<KIND>::template of<BM, false>(a, at.b, at.blk, true);
  if (!seq.real) return;
  const Lengths& len = seq.len;
  const int r0 = seq.blk * BM, rows = rows_of(a, len, r0, BM);
  if (rows <= 0) return;
  const Row row(a, at, len, r0, rows, wave * 32 + (lane & 31), lane);
  const Span span(a, row.i0 + len.shift, row.i1 + len.shift, len.k, Feed::STEP);
  const int n_tiles = (span.n + 1) / 2;

  Feed feed(a, at, seq, span, wave, lane);
  const uint32_t to = __builtin_amdgcn_readfirstlane(lds + uint32_t(wave) * 1024);
  if constexpr (Feed::STRAIGHT) {
    if (n_tiles > 0) {
      const auto k0 = feed.keys(span, 0);
      const auto v0 = feed.values(span, 0);
      const auto k1 = feed.keys(span, 1);
#pragma unroll
      for (int j = 0; j < LOADS; ++j) feed.ask_keys(k0, to, j);
#pragma unroll
      for (int j = 0; j < LOADS; ++j) feed.ask_values(v0, to + 2 * BYTES, j);
#pragma unroll
      for (int j = 0; j < LOADS; ++j) feed.ask_keys(k1, to + BYTES, j);
    }
  } else if (n_tiles > 0) {                          // through registers: two tiles of keys and one of values put, the next ones on their way
    feed.ask_keys(span, 0);
    feed.ask_values(span, 0);
    feed.put_keys(lds);
    feed.put_values(lds + 2 * BYTES);
    feed.ask_keys(span, 1);
    feed.ask_values(span, 1);
    feed.put_keys(lds + BYTES);
    feed.ask_keys(span, 2);                          // (the values of a tile are asked for behind its keys and in front of the next tile's)
  }
  bf16x8 qf[STEPS];
  {
    const char* qp = a.q.at(at.b, row.qh, seq.q0 + row.qi);
#pragma unroll
    for (int s = 0; s < STEPS; ++s) qf[s] = *reinterpret_cast<const bf16x8*>(qp + (2 * s + row.h) * 16);
  }
  // LDS addresses of the operand reads, in the buffers of this tile's keys and values; the half tile is in the instructions' offsets
  const typename KTile::RowReader k_read(lane);
  typename VTile::ColumnReader v_read(lane);
  uint32_t k_at[STEPS];
#pragma unroll
  for (int s = 0; s < STEPS; ++s) k_at[s] = lds + k_read.at + ((uint32_t(2 * s + row.h) ^ k_read.sw) * 16);
#pragma unroll
  for (int c = 0; c < CS; ++c)
#pragma unroll
    for (int i = 0; i < 2; ++i) v_read.at[c][i] += lds + 2 * BYTES;
  auto k_frag = [&](int half, int s) {
    return __builtin_bit_cast(bf16x8, *reinterpret_cast<LDS_PTR(const u32x4)>(k_at[s] + uint32_t(half * 32 * KTile::RB)));
  };

  f32x16 acc[CS], s0, s1;
  Weights<uint16_t> w0 = {}, w1 = {};
  clear(acc);
  float ref = -FLT_MAX, l = 0.f;                     // reference in the base-2 exponent's units, this lane's share of the row sum
  const float c2 = a.scale * LOG2E;
  auto mask = [&](int i, f32x16& s) __attribute__((always_inline)) {
    if (__builtin_expect(span.whole(i), 1)) return;
    asm volatile("");                                // keeps this a branch
    span.mask(a, i, row.p, row.h, s, -INFINITY);
  };
  // The weights of logits s as they are packed, `from` .. `to_` of a lane's 16, and their sum.
  auto weigh = [&](float (&e)[16], Weights<uint16_t>& w, float& sum, int from, int to_) __attribute__((always_inline)) {
#pragma unroll
    for (int i = from; i < to_; ++i) {
      sum += e[i];
      if (i % 2 == 1) {
        const bf16x2 b2 = {(__bf16)e[i - 1], (__bf16)e[i]};
        w.p[i / 8][i % 8 / 2] = __builtin_bit_cast(uint32_t, b2);
      }
    }
  };
  auto all_weights = [&](const f32x16& s, Weights<uint16_t>& w, float& sum) __attribute__((always_inline)) {
    float e[16];
    sum = 0.f;
#pragma unroll
    for (int i = 0; i < 16; ++i) e[i] = __builtin_amdgcn_exp2f(fmaf(s[i], c2, -ref));
    weigh(e, w, sum, 0, 16);
  };
  // Behind the weights `w` of logits s, whose sum is `sum`: where a lane's are too large, rows that have grown raise their reference and the weights are
  // worked out again.  (A NaN does not pass the comparison.)
  auto settle = [&](const f32x16& s, Weights<uint16_t>& w, float sum) __attribute__((always_inline)) {
    if (__builtin_expect(__builtin_amdgcn_ballot_w64(!(sum <= SUM_LIMIT)) != 0, 0)) {
      float mx = s[0];
#pragma unroll
      for (int i = 1; i < 16; ++i) mx = fmaxf(mx, s[i]);
      const auto sw = __builtin_amdgcn_permlane32_swap(__float_as_uint(mx), __float_as_uint(mx), false, false);
      mx = fmaxf(__uint_as_float(sw[0]), __uint_as_float(sw[1])) * c2;
      const float top = mx > ref ? mx : ref;         // not fmaxf: a NaN leaves the reference where it is
      float f = __builtin_amdgcn_exp2f(ref - top);
      // The accumulators are scaled in place, by statements of their own, so that they keep one home across the branch.  The compiler does not see
      // what these read: the waits for matrix instructions in flight (19 states at most) stand in front.
      asm volatile("s_nop 15\n\ts_nop 3" : "+v"(f));
      ref = top;
      l *= f;
#pragma unroll
      for (int c = 0; c < CS; ++c)
#pragma unroll
        for (int i = 0; i < 16; ++i) {
          float y = acc[c][i];
          asm volatile("v_mul_f32 %0, %1, %0" : "+v"(y) : "v"(f));
          acc[c][i] = y;
        }
      all_weights(s, w, sum);
    }
    l += sum;
  };
  // One stage, in issue order: products of `pw` with half `half` of V, logits `sn` of half `half` of K, weights `w` of logits `s`.
  auto stage = [&](auto half_, const Weights<uint16_t>& pw, f32x16& sn, const f32x16& s, Weights<uint16_t>& w, float& sum, auto mem) __attribute__((always_inline)) {
    constexpr int half = decltype(half_)::value, v_half = half;
    constexpr int NF = 2 * STEPS, AHEAD = 3;         // operands: logits' and products' in turn
    bf16x8 frag[NF];
    auto load = [&](int f) { frag[f] = f % 2 == 0 ? k_frag(half, f / 2) : v_read.get(0, v_half, f / 2 / CS, f / 2 % CS); };
#pragma unroll
    for (int i = 0; i < 16; ++i) sn[i] = 0.f;
    float e[16];
    sum = 0.f;
#pragma unroll
    for (int f = 0; f < AHEAD; ++f) load(f);
    __builtin_amdgcn_sched_barrier(0);
#pragma unroll
    for (int f = 0; f < NF; ++f) {
      if (f + AHEAD < NF) load(f + AHEAD);
      mem(f);
      if (f % 2 == 0) sn = __builtin_amdgcn_mfma_f32_32x32x16_bf16(frag[f], qf[f / 2], sn, 0, 0, 0);
      else acc[f / 2 % CS] = __builtin_amdgcn_mfma_f32_32x32x16_bf16(frag[f], __builtin_bit_cast(bf16x8, pw.p[f / 2 / CS]), acc[f / 2 % CS], 0, 0, 0);
#pragma unroll
      for (int i = f * 16 / NF; i < (f + 1) * 16 / NF; ++i) {
        e[i] = __builtin_amdgcn_exp2f(fmaf(s[i], c2, -ref));
        asm volatile("" : "+v"(e[i]));
      }
      if (f > 0) weigh(e, w, sum, (f - 1) * 16 / NF, f * 16 / NF);
      if (f == NF - 1) weigh(e, w, sum, f * 16 / NF, 16);
      __builtin_amdgcn_sched_barrier(0);
    }
  };
  int k_step = BYTES, v_step = BYTES;                // to the other buffer of keys, of values
  if (n_tiles > 0) {
    // the logits of tile 0 and the weights of its first half
    if constexpr (Feed::STRAIGHT) wait_loads();
    __syncthreads();
#pragma unroll
    for (int i = 0; i < 16; ++i) s0[i] = s1[i] = 0.f;
#pragma unroll
    for (int s = 0; s < STEPS; ++s) {
      s0 = __builtin_amdgcn_mfma_f32_32x32x16_bf16(k_frag(0, s), qf[s], s0, 0, 0, 0);
      s1 = __builtin_amdgcn_mfma_f32_32x32x16_bf16(k_frag(1, s), qf[s], s1, 0, 0, 0);
    }
    mask(0, s0);
    mask(1, s1);
    float sum;
    all_weights(s0, w0, sum);
    settle(s0, w0, sum);
  }
  if constexpr (!Feed::STRAIGHT) {                   // the queries are waited for here, or the compiler does it in every tile and for all loads
#pragma unroll
    for (int s = 0; s < STEPS; ++s) asm volatile("" : "+v"(qf[s]));
  }
  // Tile t's values and tile t + 1's keys: s1 holds the logits of tile t's second half, w0 the weights of its first.
  for (int t = 0; t + 1 < n_tiles; ++t) {
    if constexpr (Feed::STRAIGHT) wait_loads();      // this wave's parts of K(t + 1) and V(t) are there
    __syncthreads();                                 // all parts are, and every wave has left K(t) and V(t - 1)
    const int t2 = t + 2 < n_tiles ? t + 2 : t + 1;  // behind the last tile that once more, into a buffer that nothing reads
    const uint32_t k_to = t & 1 ? BYTES : 0, v_to = (t & 1 ? 2 : 3) * BYTES;
    const auto vs = [&] { if constexpr (Feed::STRAIGHT) return feed.values(span, t + 1); else return 0; }();
    const auto ks = [&] { if constexpr (Feed::STRAIGHT) return feed.keys(span, t2); else return 0; }();
#pragma unroll
    for (int s = 0; s < STEPS; ++s) k_at[s] += k_step;
    k_step = -k_step;
    float sum;
    stage(std::integral_constant<int, 0>{}, w0, s0, s1, w1, sum, [&](int f) {
      if constexpr (Feed::STRAIGHT) {
        constexpr int NF = 2 * STEPS;
#pragma unroll
        for (int j = f * 2 * LOADS / NF; j < (f + 1) * 2 * LOADS / NF; ++j) {
          if (j < LOADS) feed.ask_values(vs, to + v_to, j);
          else feed.ask_keys(ks, to + k_to, j - LOADS);
        }
      }
    });
    settle(s1, w1, sum);
    mask(2 * t + 2, s0);
    stage(std::integral_constant<int, 1>{}, w1, s1, s0, w0, sum, [&](int f) {
      if constexpr (!Feed::STRAIGHT) feed.step(f, span, t, lds + v_to, lds + k_to);          // V(t + 1) and K(t + 2) to LDS, V(t + 2) and K(t + 3) asked for
    });
    settle(s0, w0, sum);
    mask(2 * t + 3, s1);
#pragma unroll
    for (int c = 0; c < CS; ++c)
#pragma unroll
      for (int i = 0; i < 2; ++i) v_read.at[c][i] += v_step;
    v_step = -v_step;
  }
  if (n_tiles > 0) {
    if constexpr (Feed::STRAIGHT) wait_loads();
    __syncthreads();
    v_read.mma(0, 0, w0, acc);
    float sum;
    all_weights(s1, w1, sum);
    settle(s1, w1, sum);
    v_read.mma(0, 1, w1, acc);
  }
  const auto sw = __builtin_amdgcn_permlane32_swap(__float_as_uint(l), __float_as_uint(l), false, false);
  l = __uint_as_float(sw[0]) + __uint_as_float(sw[1]);
  store_row<uint16_t>(row.real, a.o.at(at.b, row.qh, seq.q0 + row.qi), acc, l == 0.f ? 0.f : 1.f / l, row.h);
  if (row.real && a.lse && row.h == 0) a.lse[(int64_t(at.b) * a.heads + row.qh) * a.n_q + seq.q0 + row.qi] = l == 0.f ? -INFINITY : (ref + __builtin_amdgcn_logf(l)) * (1.f / LOG2E);
}

// Few queries: the keys of 32 rows are split over the waves of a work-group and over `splits` work-groups, and what they find is joined.  A wave's tiles of 32
// keys are its own, so that none waits for another before the end, and but for the keys or values
// that are worked on the LDS is full of loads on their way.  Bound by memory: 48 sequences of 8 key heads, 4 100 keys, bf16, d = 128: 139 us, 5.8 TB/s read; one
// sequence: 13.5 us with the join (11.9 in a graph), of which the keys' way is 2.4: a launch each, a chain of loads, the waves' join and the splits'.  Weights are one
// bf16 term here as well, and o 2.0e-3 to 2.2e-3 from 64 bits: two make that 1.65e-3 and cost 0.5 % of the time of these 48 sequences, 3 % of the one's and 12 % of a
// prompt's of 2 048 tokens x 8 heads, d = 64.
template <typename T, int D> constexpr int split_waves() { return sizeof(T) == 4 && D == 128 ? 2 : 4; }
template <typename T, int D, bool ONCE, bool PACKED>
__global__ void __launch_bounds__((64 * split_waves<T, D>()), 1) window_split_kernel(WindowArgs a) {
  constexpr int NW = split_waves<T, D>(), SN = 32, REGS = D / 2;
  using KTile = Tile<T, D, SN, 1, false>;
  using VTile = Tile<T, D, SN, 1, true>;
  constexpr int STEPS = KTile::STEPS;
  static_assert(REGS * 64 * 4 <= 4 * KTile::BYTES, "a wave's sums fit where its tiles were");
  __shared__ __attribute__((aligned(1024))) char tiles[NW * 4 * KTile::BYTES];
  __shared__ float s_m[NW][32], s_l[NW][32];
  const int lane = threadIdx.x & 63, wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6), n = lane & 31, h = lane >> 5;
  const uint32_t lds = uint32_t(reinterpret_cast<uintptr_t>((LDS_PTR(void))(tiles))) + uint32_t(wave * 4 * KTile::BYTES);

  const int at = a.by_splits(blockIdx.x), split = blockIdx.x - at * a.splits, bh = a.by_blocks(at), blk = at - bh * a.blocks, b = PACKED ? 0 : a.by_kv(bh), kvh = bh - b * a.heads_kv;
  const auto seq = Seq<PACKED>::template of<32, false>(a, b, blk, false);
  if (!seq.real) return;
  const Lengths& len = seq.len;
  const int r0 = seq.blk * 32, rows = rows_of(a, len, r0, 32);
  if (rows <= 0) return;
  const int i0 = query_of(a, r0), i1 = query_of(a, r0 + rows - 1);
  const Span span(a, i0 + len.shift, i1 + len.shift, len.k);
  const int per = a.by_splits(span.n + a.splits - 1), t_end = min_of(span.n, (split + 1) * per);

  const bool real = n < rows;
  const int qi = real ? query_of(a, r0 + n) : i0, qh = kvh * a.group + (real ? r0 + n - qi * a.group : 0), p = qi + len.shift;
  const char *kh = a.k.at(b, kvh, seq.k0), *vh = a.v.at(b, kvh, seq.k0);
  const typename KTile::Loader k_load(a.k.row, 0, lane);
  const typename VTile::Loader v_load(a.v.row, 0, lane);
  typename Mat<T>::Frag qf[STEPS];
  {
    const char* qp = a.q.at(b, qh, seq.q0 + qi);
#pragma unroll
    for (int s = 0; s < STEPS; ++s) qf[s] = *reinterpret_cast<const typename Mat<T>::Frag*>(qp + (2 * s + h) * 16);
  }
  // Two tiles' keys and values are on their way but for what is being read.  Behind the last tile nothing is asked for, by as many loads, so that the
  // waits count the same.
  auto ask_keys = [&](int t, int buf) {
    const int begin = span.begin(t), rest = t < t_end ? span.end(t) - begin : 0;
    k_load.template issue<ONCE>(kh + int64_t(begin) * a.k.row, rest, a.k.row, lds + uint32_t(buf * 2 * KTile::BYTES), 0);
  };
  auto ask_values = [&](int t, int buf) {
    const int begin = span.begin(t), rest = t < t_end ? span.end(t) - begin : 0;
    v_load.template issue<ONCE>(vh + int64_t(begin) * a.v.row, rest, a.v.row, lds + uint32_t(buf * 2 * KTile::BYTES + KTile::BYTES), 0);
  };
  int t = split * per + wave, parity = 0;
  if (t < t_end) {
    ask_keys(t, 0);
    ask_values(t, 0);
    ask_keys(t + NW, 1);
    ask_values(t + NW, 1);
  }
  // The queries are waited for here, with what was asked for behind them, or the compiler does it in every tile and for all loads.
#pragma unroll
  for (int s = 0; s < STEPS; ++s) asm volatile("" : "+v"(qf[s]));
  const typename KTile::RowReader k_read(lane);
  const typename VTile::ColumnReader v_read(lane);
  f32x16 acc[D / 32];
  clear(acc);
  float m = -INFINITY, l = 0.f;
  const float c2 = a.scale * LOG2E;
  for (; t < t_end; t += NW, parity ^= 1) {
    const uint32_t buf = lds + uint32_t(parity * 2 * KTile::BYTES);
    wait_loads_but<3 * KTile::LOADS>();
    f32x16 s;
#pragma unroll
    for (int i = 0; i < 16; ++i) s[i] = 0.f;
#pragma unroll
    for (int st = 0; st < STEPS; ++st) s = Mat<T>::mma(k_read.get(buf, 0, st), qf[st], s);
    wait_reads();
    ask_keys(t + 2 * NW, parity);
    if (!span.whole(t)) span.mask(a, t, p, h, s, -INFINITY);
    float mx = s[0];
#pragma unroll
    for (int i = 1; i < 16; ++i) mx = fmaxf(mx, s[i]);
    const auto sw = __builtin_amdgcn_permlane32_swap(__float_as_uint(mx), __float_as_uint(mx), false, false);
    const float m_new = fmaxf(m, fmaxf(__uint_as_float(sw[0]), __uint_as_float(sw[1])) * c2), ref = m_new == -INFINITY ? 0.f : m_new;
    if (__builtin_amdgcn_ballot_w64(m_new > m)) {
      const float alpha = __builtin_amdgcn_exp2f(m - ref);
      m = m_new;
      l *= alpha;
#pragma unroll
      for (int c = 0; c < D / 32; ++c)
#pragma unroll
        for (int i = 0; i < 16; ++i) acc[c][i] *= alpha;
    }
#pragma unroll
    for (int i = 0; i < 16; ++i) {
      s[i] = __builtin_amdgcn_exp2f(fmaf(s[i], c2, -ref));
      l += s[i];
    }
    Weights<T> w;
    w.set(s);
    wait_loads_but<3 * KTile::LOADS>();
    v_read.mma(buf + KTile::BYTES, 0, w, acc);
    wait_reads();
    ask_values(t + 2 * NW, parity);
  }
  wait_loads();                                      // the last ones, of nothing, still write zeros where the sums go
  const auto sw = __builtin_amdgcn_permlane32_swap(__float_as_uint(l), __float_as_uint(l), false, false);
  l = __uint_as_float(sw[0]) + __uint_as_float(sw[1]);
  // The waves' sums meet where the tiles were; each wave joins a share of the channels.
  float* all = reinterpret_cast<float*>(tiles);
  __syncthreads();
#pragma unroll
  for (int c = 0; c < D / 32; ++c)
#pragma unroll
    for (int i = 0; i < 16; ++i) all[(wave * REGS + c * 16 + i) * 64 + lane] = acc[c][i];
  if (h == 0) {
    s_m[wave][n] = m;
    s_l[wave][n] = l;
  }
  __syncthreads();
  float top = s_m[0][n], total = 0.f, share[NW];
#pragma unroll
  for (int w = 1; w < NW; ++w) top = fmaxf(top, s_m[w][n]);
  const float ref = top == -INFINITY ? 0.f : top;
#pragma unroll
  for (int w = 0; w < NW; ++w) {
    share[w] = __builtin_amdgcn_exp2f(s_m[w][n] - ref);
    total += share[w] * s_l[w][n];
  }
  if (!real) return;
  const bool alone = a.splits == 1;
  const float f = !alone ? 1.f : total == 0.f ? 0.f : 1.f / total;
  const int64_t slot = (int64_t(at) * a.splits + split) * 32 + n;
  char* out = alone ? a.o.at(b, qh, seq.q0 + qi) : reinterpret_cast<char*>(a.part + slot * D);
#pragma unroll
  for (int g = 0; g < REGS / NW; g += 4) {
    const int reg = wave * (REGS / NW) + g, ch = reg / 16 * 32 + reg % 16 * 2 + 4 * h;
    float x[4] = {};
#pragma unroll
    for (int w = 0; w < NW; ++w)
#pragma unroll
      for (int j = 0; j < 4; ++j) x[j] = fmaf(share[w], all[(w * REGS + reg + j) * 64 + lane], x[j]);
    if (alone) store_four<T>(out, ch, x, f);
    else store_four<float>(out, ch, x, f);
  }
  if (wave == 0 && h == 0) {
    if (!alone) a.part_sums[slot] = make_float2(top, total);
    else if (a.lse) a.lse[(int64_t(b) * a.heads + qh) * a.n_q + seq.q0 + qi] = total == 0.f ? -INFINITY : (top + __builtin_amdgcn_logf(total)) * (1.f / LOG2E);
  }
}

// Joins the splits of a row: a thread takes four channels.  Bound by a trip to memory, so eight splits' sums and rows are asked for at once (one token over
// 700 keys, 6 splits: 10.3 -> 8.7 us with the split kernel, over 4 100 keys, 16 splits, 12.5 -> 11.9; sixteen at once 9.4 and 11.9).
template <typename T, int D, bool PACKED>
__global__ void __launch_bounds__(256) window_join_kernel(WindowArgs a) {
  constexpr int TR = D / 4, RB = 256 / TR, U = 8;    // threads of a row, rows of a work-group, splits asked for at once
  const int at = blockIdx.x / (32 / RB), n = blockIdx.x % (32 / RB) * RB + threadIdx.x / TR, ch = threadIdx.x % TR * 4;
  const int bh = a.by_blocks(at), blk = at - bh * a.blocks, b = PACKED ? 0 : a.by_kv(bh), kvh = bh - b * a.heads_kv;
  const auto seq = Seq<PACKED>::template of<32, false>(a, b, blk, false);
  if (!seq.real) return;
  const int r = seq.blk * 32 + n;
  if (r >= seq.len.q * a.group) return;
  const int qi = query_of(a, r), qh = kvh * a.group + r - qi * a.group;
  const int64_t slot = int64_t(at) * a.splits * 32 + n;
  float top = -INFINITY, total = 0.f, x[4] = {};
  for (int s = 0; s < a.splits; s += U) {
    float2 ml[U];
    float4 y[U];
#pragma unroll
    for (int u = 0; u < U; ++u) {                    // behind the last split that once more, with a weight of zero
      const int64_t i = slot + (s + u < a.splits ? s + u : a.splits - 1) * 32;
      ml[u] = a.part_sums[i];
      y[u] = *reinterpret_cast<const float4*>(a.part + i * D + ch);
    }
    const float before = top;
#pragma unroll
    for (int u = 0; u < U; ++u) {
      if (s + u >= a.splits) ml[u].x = -INFINITY;
      top = fmaxf(top, ml[u].x);
    }
    const float ref = top == -INFINITY ? 0.f : top, f = __builtin_amdgcn_exp2f(before - ref);
    total *= f;
#pragma unroll
    for (int j = 0; j < 4; ++j) x[j] *= f;
#pragma unroll
    for (int u = 0; u < U; ++u) {
      const float share = __builtin_amdgcn_exp2f(ml[u].x - ref);
      total = fmaf(share, ml[u].y, total);
      x[0] = fmaf(share, y[u].x, x[0]);
      x[1] = fmaf(share, y[u].y, x[1]);
      x[2] = fmaf(share, y[u].z, x[2]);
      x[3] = fmaf(share, y[u].w, x[3]);
    }
  }
  store_four<T>(a.o.at(b, qh, seq.q0 + qi), ch, x, total == 0.f ? 0.f : 1.f / total);
  if (ch == 0 && a.lse) a.lse[(int64_t(b) * a.heads + qh) * a.n_q + seq.q0 + qi] = total == 0.f ? -INFINITY : (top + __builtin_amdgcn_logf(total)) * (1.f / LOG2E);
}

}  // namespace dfs
