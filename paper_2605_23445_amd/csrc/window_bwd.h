// Kernels of the backward pass of attention over a window and a few first keys, of sequences of one length (PACKED false) or packed ones: the queries' gradient, then those of keys and values.
//
// The first kernel goes over keys for a block of queries, as the forward pass does, and leaves <do, o> of every row beside its log-sum-exp; the second goes
// over queries for a block of keys, head by head of those that share it.  Both work the weights out anew from the log-sum-exp.  A block is one work-group's
// or, where blocks are few, shared by several, whose parts another kernel adds up in a fixed order: there are no atomics.  The second takes the pairs of the
// windows alone: the first keys, which every query sees, would keep a work-group for as long as all others take together.  Their other pairs are dealt to
// work-groups of a third kernel, and a fourth adds the parts up.
#pragma once
#include <float.h>
#include <math.h>

#include "window.h"

namespace dfs {

// Parts, as a wave holds them.  Of dk and dv of the 32 first keys of `tile`, from the queries that see them as first ones:
__device__ __forceinline__ float* first_part(const WindowArgs& a, int d, int bh, int tile, int split) {
  return a.part + ((int64_t(bh) * a.first_tiles + tile) * a.first_splits + split) * 64 * d;
}
// of dk and dv of the 32 keys of `tile`, from their windows: of all tiles where blocks of keys are shared, else of those of first keys;
__device__ __forceinline__ float* key_part(const WindowArgs& a, int d, int bh, int tile, int split) {
  return a.key_part + ((int64_t(bh) * a.key_tiles + tile) * a.key_splits + split) * 64 * d;
}
// of dq of the 32 rows of `tile`, and behind it (bf16) of the rows' sums of dS and of weights.
__device__ __forceinline__ float* row_part(const WindowArgs& a, int d, int64_t tile, int split) { return a.row_part + (tile * a.row_splits + split) * 32 * (d + 2); }

// Whether a row's weights, with this sum, are all that its log-sum-exp (here `ref`, in base 2) counts: not where that was joined with other keys'.  Then the sum
// of dS is zero but for rounding.  The sum is off from 1 by what fp32 rounds the weights' exponents by, below 2^-21 |ref|, and by the sums' own rounding; other
// keys of less weight than that are left out of a joined row's <do, o>.
__device__ __forceinline__ bool own_sum(float x, float ref) { return fabsf(x - 1.f) <= 0x1p-12f + 0x1p-20f * fabsf(ref); }

// Sum of what the two lanes that share a row hold.
__device__ __forceinline__ float both_halves(float x) {
  const auto sw = __builtin_amdgcn_permlane32_swap(__float_as_uint(x), __float_as_uint(x), false, false);
  return __uint_as_float(sw[0]) + __uint_as_float(sw[1]);
}

// f32: one step per tile of 64 keys, bound by the fp32 matrix instructions and by what their waves wait for in between, as in the forward pass: two work-groups a CU
// at d = 64, one at d = 128 (4 000 tokens x 16 heads, 1 000 keys each way: 473 and 1 030 us, matrix cores busy 62 and 54 % of the cycles; forward and backward 1.53
// and 3.37 ms, 43 and 39 % of a large product's rate).
template <int D, bool PACKED>
__global__ void __launch_bounds__(256, 1) window_dq_f32_kernel(WindowArgs a) {
  typedef float T;
  constexpr int NW = 4, BM = 32 * NW, KN = 64;
  using KTile = Tile<T, D, KN, NW, false>;
  constexpr int STEPS = KTile::STEPS;
  __shared__ __attribute__((aligned(1024))) char tiles[4 * KTile::BYTES];
  const uint32_t lds = uint32_t(reinterpret_cast<uintptr_t>((LDS_PTR(void))(tiles)));
  const int lane = threadIdx.x & 63, wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);

  const PlaceOf<PACKED> at(a, blockIdx.x);
  const int i = a.by_splits(at.blk), split = at.blk - i * a.row_splits;
  const auto seq = Seq<PACKED>::template of<BM, false>(a, at.b, i, true);
  if (!seq.real) return;
  const Lengths& len = seq.len;
  const int r0 = seq.blk * BM, rows = rows_of(a, len, r0, BM);
  if (rows <= 0) return;
  const Row row(a, at, len, r0, rows, wave * 32 + (lane & 31), lane);
  const Span span(a, row.i0 + len.shift, row.i1 + len.shift, len.k);
  const int all_tiles = (span.n + 1) / 2, per = a.by_splits(all_tiles + a.row_splits - 1), t0 = split * per, n_tiles = min_of(all_tiles, t0 + per);
  // this wave's positions
  const int first = min_of(wave * 32, rows - 1), last = min_of(wave * 32 + 31, rows - 1);
  const int q0 = query_of(a, r0 + first) + len.shift, q1 = query_of(a, r0 + last) + len.shift;

  Mat<T>::Frag qf[STEPS], gf[STEPS];
  const int64_t sums = (int64_t(at.b) * a.heads + row.qh) * a.n_q + seq.q0 + row.qi;
  float delta = 0.f;
  {
    const char *qp = a.q.at(at.b, row.qh, seq.q0 + row.qi), *gp = a.d_o.at(at.b, row.qh, seq.q0 + row.qi), *op = a.o.at(at.b, row.qh, seq.q0 + row.qi);
#pragma unroll
    for (int s = 0; s < STEPS; ++s) {
      qf[s] = *reinterpret_cast<const Mat<T>::Frag*>(qp + (2 * s + row.h) * 16);
      gf[s] = *reinterpret_cast<const Mat<T>::Frag*>(gp + (2 * s + row.h) * 16);
      const auto of = *reinterpret_cast<const Mat<T>::Frag*>(op + (2 * s + row.h) * 16);
#pragma unroll
      for (int i = 0; i < int(16 / sizeof(T)); ++i) delta = fmaf(float(gf[s][i]), float(of[i]), delta);
    }
    delta = both_halves(delta);
  }
  const float lse = a.lse[sums], ref = lse == -INFINITY ? INFINITY : lse * LOG2E;      // a row that sees nothing has weights of zero
  if (row.real && row.h == 0 && split == 0) a.sums[sums] = make_float2(ref, delta);
  const char *kh = a.k.at(at.b, at.kvh, seq.k0), *vh = a.v.at(at.b, at.kvh, seq.k0);
  const typename KTile::Loader k_load(a.k.row, wave, lane), v_load(a.v.row, wave, lane);
  const typename KTile::RowReader read(lane);
  const typename KTile::ColumnReader k_cols(lane);
  const uint32_t to = __builtin_amdgcn_readfirstlane(lds + uint32_t(wave) * 1024);
  auto issue = [&](int t) {
    const uint32_t buf = to + uint32_t((t & 1) * 2 * KTile::BYTES);
    const auto ks = k_load.of(span, kh, a.k.row, t);
    const auto vs = v_load.of(span, vh, a.v.row, t);
#pragma unroll
    for (int j = 0; j < KTile::LOADS; ++j) k_load.issue_one(ks, buf, j);
#pragma unroll
    for (int j = 0; j < KTile::LOADS; ++j) v_load.issue_one(vs, buf + KTile::BYTES, j);
  };
  f32x16 acc[D / 32];
  clear(acc);
  const float c2 = a.scale * LOG2E;
  if (t0 < n_tiles) issue(t0);
  for (int t = t0; t < n_tiles; ++t) {
    wait_loads();
    __syncthreads();
    if (t + 1 < n_tiles) issue(t + 1);
    const uint32_t buf = lds + uint32_t((t & 1) * 2 * KTile::BYTES);
#pragma unroll
    for (int half = 0; half < 2; ++half) {
      if (span.unseen(a, 2 * t + half, q0, q1)) continue;
      f32x16 s[1], g[1];
      clear(s);
      clear(g);
#pragma unroll
      for (int st = 0; st < STEPS; ++st) {
        s[0] = Mat<T>::mma(read.get(buf, half, st), qf[st], s[0]);
        g[0] = Mat<T>::mma(read.get(buf + KTile::BYTES, half, st), gf[st], g[0]);
      }
#pragma unroll
      for (int i = 0; i < 16; ++i) {
        const float w = __builtin_amdgcn_exp2f(fmaf(s[0][i], c2, -ref));
        s[0][i] = w * (g[0][i] - delta);
      }
      if (!span.whole(2 * t + half)) span.mask(a, 2 * t + half, row.p, row.h, s[0], 0.f);
      Weights<T> w;
      w.set(s[0]);
      k_cols.mma(buf, half, w, acc);
    }
  }
  if (a.row_splits > 1) {
    float* mine = row_part(a, D, (int64_t(at.bh) * (a.blocks / a.row_splits) + seq.slot) * NW + wave, split) + lane;
#pragma unroll
    for (int c = 0; c < D / 32; ++c)
#pragma unroll
      for (int i = 0; i < 16; ++i) mine[(c * 16 + i) * 64] = acc[c][i];
  } else {
    store_row<T>(row.real, a.dq.at(at.b, row.qh, seq.q0 + row.qi), acc, a.scale, row.h);
  }
}

// bf16: per piece of 32 keys three runs of products, <do, v>, the next piece's logits and dS k, with the weights worked out beside the first and dS beside the
// second; operands are asked for AHEAD of their instruction, scheduling fences keep it so.  The logits that a piece starts with are the piece's before.  Keys
// have three buffers, as the next tile's are read while this one's still are; two work-groups fill the LDS of a CU.
//
// dS goes into its product as two bf16 terms, and the rows' sums of dS, which are zero but for what rounding o has cost <do, o>, are added to that: dk
// is worked out with the corrected one.  (Where o and log-sum-exp were joined with other keys' they are not zero, and nothing is corrected.)  In one term and
// without it dq and dk were 1.6 to 2 times as far from 64 bits as rounding them alone (relative 2-norm 2.5e-3 to 3.3e-3; now 1.8e-3 to 2.4e-3).  Where a block
// of rows sees four tiles of keys at most, the error of <do, o> is most of dq's, so it is worked out from the keys beforehand.
//
// Bound by the matrix cores and the vector port beside them: 17 550 tokens x 30 heads, d = 64, 1 350 keys each way: 830 us, 848 TFLOP/s with the second term's,
// matrix cores busy 45 % of the cycles (790 and 48 % without the sum of weights); 2 x 4 001 (ragged) x 32 heads of 8 key heads, d = 128, 512 keys back: 118 us,
// 744 TFLOP/s, 38 %.
template <int D, bool PACKED>
__global__ void __launch_bounds__(256, D == 64 ? 3 : 2) window_dq_kernel(WindowArgs a) {
  typedef uint16_t T;
  constexpr int NW = 4, BM = 32 * NW, KN = 64;
  using KTile = Tile<T, D, KN, NW, false>;
  constexpr int STEPS = KTile::STEPS, CS = D / 32, LOADS = KTile::LOADS, BYTES = KTile::BYTES, RB = KTile::RB;
  __shared__ __attribute__((aligned(1024))) char tiles[5 * BYTES];                    // three of keys, two of values
  const uint32_t lds = uint32_t(reinterpret_cast<uintptr_t>((LDS_PTR(void))(tiles)));
  const int lane = threadIdx.x & 63, wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);

  const PlaceOf<PACKED> at(a, blockIdx.x);
  const int i = a.by_splits(at.blk), split = at.blk - i * a.row_splits;
  const auto seq = Seq<PACKED>::template of<BM, false>(a, at.b, i, true);
  if (!seq.real) return;
  const Lengths& len = seq.len;
  const int r0 = seq.blk * BM, rows = rows_of(a, len, r0, BM);
  if (rows <= 0) return;
  const Row row(a, at, len, r0, rows, wave * 32 + (lane & 31), lane);
  const Span span(a, row.i0 + len.shift, row.i1 + len.shift, len.k);
  const int all_tiles = (span.n + 1) / 2, per = a.by_splits(all_tiles + a.row_splits - 1), t0 = split * per, n_tiles = min_of(all_tiles, t0 + per);
  const char *kh = a.k.at(at.b, at.kvh, seq.k0), *vh = a.v.at(at.b, at.kvh, seq.k0);
  const typename KTile::Loader k_load(a.k.row, wave, lane), v_load(a.v.row, wave, lane);
  const uint32_t to = __builtin_amdgcn_readfirstlane(lds + uint32_t(wave) * 1024);
  auto issue = [&](int t, uint32_t k_buf, uint32_t v_buf) {
    // behind the last tile pieces without rows, or another's tile, which nothing reads
    const auto ks = k_load.of(span, kh, a.k.row, t);
    const auto vs = v_load.of(span, vh, a.v.row, t);
#pragma unroll
    for (int j = 0; j < LOADS; ++j) k_load.issue_one(ks, to + k_buf, j);
#pragma unroll
    for (int j = 0; j < LOADS; ++j) v_load.issue_one(vs, to + v_buf, j);
  };
  const bool few = all_tiles <= 4;                   // keys of which <do, o> is worked out beforehand, by every work-group that shares them
  if (t0 < n_tiles) issue(few ? 0 : t0, 0, 3 * BYTES);

  bf16x8 qf[STEPS], gf[STEPS];
  const int64_t sums = (int64_t(at.b) * a.heads + row.qh) * a.n_q + seq.q0 + row.qi;
  float delta = 0.f;
  {
    const char *qp = a.q.at(at.b, row.qh, seq.q0 + row.qi), *gp = a.d_o.at(at.b, row.qh, seq.q0 + row.qi), *op = a.o.at(at.b, row.qh, seq.q0 + row.qi);
#pragma unroll
    for (int s = 0; s < STEPS; ++s) {
      qf[s] = *reinterpret_cast<const bf16x8*>(qp + (2 * s + row.h) * 16);
      gf[s] = *reinterpret_cast<const bf16x8*>(gp + (2 * s + row.h) * 16);
      const auto of = *reinterpret_cast<const bf16x8*>(op + (2 * s + row.h) * 16);
#pragma unroll
      for (int i = 0; i < 8; ++i) delta = fmaf(float(gf[s][i]), float(of[i]), delta);
    }
    delta = both_halves(delta);
  }
  const float lse = a.lse[sums], ref = lse == -INFINITY ? INFINITY : lse * LOG2E;      // a row that sees nothing has weights of zero
  // LDS addresses of a lane's operands: this tile's keys by columns, by rows the keys whose logits come next and this tile's values; chunks by XOR
  const typename KTile::RowReader read(lane);
  const typename KTile::ColumnReader cols(lane);
  uint32_t next_at = lds + read.at + ((uint32_t(row.h) ^ read.sw) * 16), val_at = next_at + 3 * BYTES, col_at = lds + cols.at[0][0];
  auto by_rows = [](uint32_t x) { return __builtin_bit_cast(bf16x8, *reinterpret_cast<LDS_PTR(const u32x4)>(x)); };
  auto by_columns = [](uint32_t x, int s, int c) {
    constexpr uint32_t FAR = uint32_t(KTile::swizzle(8)) * 16;           // rows 8 further on: their chunks are swapped by this
    const s16x4 lo = __builtin_amdgcn_ds_read_tr16_b64_v4i16(reinterpret_cast<LDS_PTR(s16x4)>((x ^ uint32_t(64 * c)) + uint32_t(16 * s * RB)));
    const s16x4 hi = __builtin_amdgcn_ds_read_tr16_b64_v4i16(reinterpret_cast<LDS_PTR(s16x4)>((x ^ (uint32_t(64 * c) ^ FAR)) + uint32_t((16 * s + 8) * RB)));
    return __builtin_bit_cast(bf16x8, __builtin_shufflevector(lo, hi, 0, 1, 2, 3, 4, 5, 6, 7));
  };
  f32x16 acc[CS], s, s1;
  clear(acc);
  float off = 0.f, total = 0.f;                      // this lane's share of the sums of dS and of weights
  const float c2 = a.scale * LOG2E;
  auto mask = [&](int i, f32x16& s) __attribute__((always_inline)) {
    if (__builtin_expect(span.whole(i), 1)) return;
    asm volatile("");                                // keeps this a branch
    span.mask(a, i, row.p, row.h, s, -INFINITY);
  };
  // A piece, half `half` of this tile.  `between`: in front of the next piece's logits, which are those of half `next` at next_at.
  auto piece = [&](auto half_, f32x16& s, f32x16& sn, auto between) __attribute__((always_inline)) {
    constexpr int half = decltype(half_)::value, NF = 2 * STEPS + 4 * CS, AHEAD = 3;
    constexpr bool APART = half == 1;                // nothing is asked for across `between`
    bf16x8 frag[NF];
    f32x16 g;
    Weights<T> w, rest;
    // Slot j of the last run: contraction step, channels, and whether it is the product of dS's second term, which has its operand from the first's.
    auto step_of = [](int j) { return j / (2 * CS); };
    auto part_of = [](int j) { return j % CS; };
    auto second = [](int j) { return j % (2 * CS) >= CS; };
    auto load = [&](int f) {
      if (f < STEPS) frag[f] = by_rows((val_at ^ uint32_t(32 * f)) + uint32_t(half * 32 * RB));
      else if (f < 2 * STEPS) frag[f] = by_rows((next_at ^ uint32_t(32 * (f - STEPS))) + uint32_t((1 - half) * 32 * RB));
      else if (!second(f - 2 * STEPS)) frag[f] = by_columns(col_at + uint32_t(half * 32 * RB), step_of(f - 2 * STEPS), part_of(f - 2 * STEPS));
    };
#pragma unroll
    for (int i = 0; i < 16; ++i) g[i] = sn[i] = 0.f;
#pragma unroll
    for (int f = 0; f < AHEAD; ++f) load(f);
    __builtin_amdgcn_sched_barrier(0);
#pragma unroll
    for (int f = 0; f < NF; ++f) {
      if (f == STEPS) {
        between();
        if (APART) {
#pragma unroll
          for (int i = 0; i < AHEAD; ++i) load(f + i);
        }
        __builtin_amdgcn_sched_barrier(0);
      }
      if (f + AHEAD < NF && !(APART && f < STEPS && f + AHEAD >= STEPS)) load(f + AHEAD);
      const int j = f - 2 * STEPS;
      if (f < STEPS) g = __builtin_amdgcn_mfma_f32_32x32x16_bf16(frag[f], gf[f], g, 0, 0, 0);
      else if (f < 2 * STEPS) sn = __builtin_amdgcn_mfma_f32_32x32x16_bf16(frag[f], qf[f - STEPS], sn, 0, 0, 0);
      else if (!second(j))
        acc[part_of(j)] = __builtin_amdgcn_mfma_f32_32x32x16_bf16(frag[f], __builtin_bit_cast(bf16x8, w.p[step_of(j)]), acc[part_of(j)], 0, 0, 0);
      else
        acc[part_of(j)] = __builtin_amdgcn_mfma_f32_32x32x16_bf16(frag[f - CS], __builtin_bit_cast(bf16x8, rest.p[step_of(j)]), acc[part_of(j)], 0, 0, 0);
      constexpr int E = 16 / STEPS;
      if (f < STEPS) {
#pragma unroll
        for (int i = E * f; i < E * f + E; ++i) s[i] = __builtin_amdgcn_exp2f(fmaf(s[i], c2, -ref));
      } else if (f < 2 * STEPS) {
#pragma unroll
        for (int i = E * (f - STEPS); i < E * (f - STEPS) + E; ++i) {
          total += s[i];
          g[i] = s[i] * (g[i] - delta);
          off += g[i];
          asm volatile("" : "+v"(total), "+v"(off));   // here: put off, the sums kept 35 registers in scratch (1 990 -> 2 520 us, not 2 010)
          if (i % 2) {
            const bf16x2 pair = {(__bf16)g[i - 1], (__bf16)g[i]};
            const uint32_t p = w.p[i / 8][i % 8 / 2] = __builtin_bit_cast(uint32_t, pair);
            const bf16x2 left = {(__bf16)(g[i - 1] - __uint_as_float(p << 16)), (__bf16)(g[i] - __uint_as_float(p & 0xFFFF0000u))};
            rest.p[i / 8][i % 8 / 2] = __builtin_bit_cast(uint32_t, left);
          }
        }
      }
      __builtin_amdgcn_sched_barrier(0);
    }
  };
  if (few && t0 < n_tiles) {
    float sum = 0.f, weights = 0.f;
    for (int t = 0; t < all_tiles; ++t) {
      wait_loads();
      __syncthreads();
#pragma unroll 1
      for (int half = 0; half < 2; ++half) {
        const uint32_t k_at = next_at + uint32_t(half * 32 * RB), v_at = val_at + uint32_t(half * 32 * RB);
        f32x16 g;
#pragma unroll
        for (int i = 0; i < 16; ++i) s[i] = g[i] = 0.f;
#pragma unroll
        for (int f = 0; f < STEPS; ++f) {
          s = __builtin_amdgcn_mfma_f32_32x32x16_bf16(by_rows(k_at ^ uint32_t(32 * f)), qf[f], s, 0, 0, 0);
          g = __builtin_amdgcn_mfma_f32_32x32x16_bf16(by_rows(v_at ^ uint32_t(32 * f)), gf[f], g, 0, 0, 0);
          __builtin_amdgcn_sched_barrier(0);
        }
        mask(2 * t + half, s);
#pragma unroll
        for (int i = 0; i < 16; ++i) {
          const float x = __builtin_amdgcn_exp2f(fmaf(s[i], c2, -ref));
          weights += x;
          sum = fmaf(x, g[i], sum);
        }
      }
      __syncthreads();                               // every wave has left the tile
      issue(t + 1 < all_tiles ? t + 1 : t0, 0, 3 * BYTES);
    }
    if (own_sum(both_halves(weights), ref)) delta = both_halves(sum);
  }
  if (t0 < n_tiles) {
    wait_loads();
    __syncthreads();
    issue(t0 + 1, BYTES, 4 * BYTES);
#pragma unroll
    for (int i = 0; i < 16; ++i) s[i] = 0.f;
#pragma unroll
    for (int f = 0; f < STEPS; ++f) s = __builtin_amdgcn_mfma_f32_32x32x16_bf16(by_rows(next_at ^ uint32_t(32 * f)), qf[f], s, 0, 0, 0);
    mask(2 * t0, s);
  }
  int k_now = 0, v_step = BYTES;                     // buffer of this tile's keys; to the other buffer of values
  for (int t = t0; t < n_tiles; ++t) {
    asm volatile("" : "+v"(next_at), "+v"(val_at), "+v"(col_at));
    piece(std::integral_constant<int, 0>{}, s, s1, [] {});
    mask(2 * t + 1, s1);
    const int k_next = k_now == 2 * BYTES ? 0 : k_now + BYTES, k_far = k_next == 2 * BYTES ? 0 : k_next + BYTES;
    next_at += k_next - k_now;
    piece(std::integral_constant<int, 1>{}, s1, s, [&] {
      wait_loads();                                  // this wave's parts of the next tile are there
      __syncthreads();                               // all parts are, and every wave has left this tile's values and the keys of the tile before
      issue(t + 2, k_far, v_step > 0 ? 3 * BYTES : 4 * BYTES);
    });
    mask(2 * t + 2, s);
    col_at += k_next - k_now;
    val_at += v_step;
    k_now = k_next;
    v_step = -v_step;
  }
  off = both_halves(off);
  total = both_halves(total);
  if (row.real && row.h == 0 && split == 0) a.sums[sums] = make_float2(ref, a.row_splits == 1 && own_sum(total, ref) ? delta + off : delta);
  wait_loads();                                      // nothing of this work-group's is on its way when its LDS is another's
  if (a.row_splits > 1) {
    float* mine = row_part(a, D, (int64_t(at.bh) * (a.blocks / a.row_splits) + seq.slot) * NW + wave, split) + lane;
#pragma unroll
    for (int c = 0; c < CS; ++c)
#pragma unroll
      for (int i = 0; i < 16; ++i) mine[(c * 16 + i) * 64] = acc[c][i];
    if (row.h == 0) {
      mine[32 * D] = off;
      mine[32 * D + 32] = total;
    }
  } else {
    store_row<T>(row.real, a.dq.at(at.b, row.qh, seq.q0 + row.qi), acc, a.scale, row.h);
  }
}

// Four channels of what a lane holds of 32 rows: register i, row lane % 32.
__device__ __forceinline__ int channel_of(int i, int lane) { return i / 16 * 32 + i % 16 * 2 + lane / 32 * 4; }
__device__ __forceinline__ void add_four(float (&x)[4], const float* p) {
#pragma unroll
  for (int j = 0; j < 4; ++j) x[j] += p[j * 64];
}

// Adds up what the work-groups that share a block of rows left.  A thread takes four channels of a row.
template <typename T, int D, bool PACKED>
__global__ void __launch_bounds__(256) window_dq_sum_kernel(WindowArgs a) {
  const int tiles = a.blocks / a.row_splits * 4, tile = blockIdx.x % tiles, bh = blockIdx.x / tiles, b = bh / a.heads_kv, kvh = bh % a.heads_kv;
  const auto seq = Seq<PACKED>::template of<128, false>(a, b, tile / 4, false);
  if (!seq.real) return;
  const int at = blockIdx.y * 256 + threadIdx.x, lane = at % 64, i = at / 64 * 4, r = seq.blk * 128 + tile % 4 * 32 + lane % 32;
  if (r >= seq.len.q * a.group) return;
  const int qi = query_of(a, r), qh = kvh * a.group + r - qi * a.group;
  float x[4] = {};
#pragma unroll 8
  for (int s = 0; s < a.row_splits; ++s) add_four(x, row_part(a, D, blockIdx.x, s) + i * 64 + lane);
  store_four<T>(a.dq.at(b, qh, seq.q0 + qi), channel_of(i, lane), x, a.scale);
  if (sizeof(T) == 4 || at >= 32) return;
  float off = 0.f, total = 0.f;
  for (int s = 0; s < a.row_splits; ++s) {
    const float* p = row_part(a, D, blockIdx.x, s) + 32 * D + lane;
    off += p[0];
    total += p[32];
  }
  float2& sums = a.sums[(int64_t(b) * a.heads + qh) * a.n_q + seq.q0 + qi];
  if (own_sum(total, sums.x)) sums.y += off;
}

// Two sums of N query rows (32 or 64) to LDS, a row after the other; zeros for those behind `rows`.
template <int N> __device__ __forceinline__ void load_sums(const float2* from, int rows, uint32_t lds, int lane) {
  const uint64_t at = reinterpret_cast<uint64_t>(from);
  const u32x4 desc = {uint32_t(__builtin_amdgcn_readfirstlane(uint32_t(at))), uint32_t(__builtin_amdgcn_readfirstlane(uint32_t(at >> 32))) & 0xFFFFu,
                      uint32_t(__builtin_amdgcn_readfirstlane(min_of(rows, N) * 8)), 0x00020000u};
  const uint32_t to = __builtin_amdgcn_readfirstlane(lds);
#pragma unroll
  for (int j = 0; j < N / 32; ++j)
    asm volatile("s_add_u32 m0, %0, %3\n\ts_nop 0\n\tbuffer_load_dword %1, %2, 0 offen lds"
                 ::"s"(to), "v"(lane * 4 + j * 256), "s"(desc), "i"(j * 256) : "memory", "m0", "scc");
}

// Keys as columns: register i of a lane holds query row 8 (i / 4) + 4 h + i % 4 of a tile of 32, against the lane's key.  A lone wave a SIMD issues a vector
// instruction every eight to ten cycles and cannot keep the matrix cores busy, so in bf16 two work-groups share a CU: the keys' rows stay in registers and the
// values' come from LDS in every tile (at d = 128 the accumulators alone take 128 registers).  At the sizes above 770 to 800 us, 880 to 915 TFLOP/s, 47 %, and 148 us,
// 594 TFLOP/s, 31 %: of 512 places on the CUs the ragged lengths fill 368, and two work-groups a CU do not fill what one of them waits for.  P and dS are one bf16
// term each: dk and dv are 2.35e-3 from 64 bits in 2-norm where rounding the results alone costs 1.65e-3, and a second term would be half of this kernel's products
// again.  In fp32 one work-group a CU, whose 263 registers at d = 64 are seven more than two allow (4 000 tokens x 16 heads: 741 us, 54 %; d = 128: 1 490, 52 %).
//
// QG: groups of four waves that take the tiles of queries in turn, each with tiles of its own; what they find is added up in the end.  Two halve the time of the longest block,
// and a CU has as many waves as with two work-groups of one group.
template <typename T, int D, bool PACKED, int QG>
__global__ void __launch_bounds__(256 * QG, sizeof(T) == 2 ? 2 / QG : 1) window_dkv_kernel(WindowArgs a) {
  constexpr bool BF16 = sizeof(T) == 2, V_LDS = BF16;
  constexpr int NW = 4, BN = 32 * NW, QN = BF16 && D == 64 ? 64 : 32, HALVES = QN / 32;
  using QTile = Tile<T, D, QN, NW, false>;
  using VTile = Tile<T, D, BN, NW, false>;
  constexpr int STEPS = QTile::STEPS;
  __shared__ __attribute__((aligned(1024))) char tiles[QG * 4 * QTile::BYTES + (V_LDS ? VTile::BYTES : 0)];
  __shared__ __attribute__((aligned(1024))) float2 all_sums[QG][2][QN];
  const int lane = threadIdx.x & 63, all_waves = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6), qg = QG == 1 ? 0 : all_waves / NW, wave = all_waves - qg * NW;
  const int n = lane & 31, h = lane >> 5;
  float2 (&row_sums)[2][QN] = all_sums[qg];
  const uint32_t lds_tiles = uint32_t(reinterpret_cast<uintptr_t>((LDS_PTR(void))(tiles))), lds = lds_tiles + uint32_t(qg * 4 * QTile::BYTES);
  const uint32_t lds_v = lds_tiles + QG * 4 * QTile::BYTES;
  const uint32_t lds_sums = uint32_t(reinterpret_cast<uintptr_t>((LDS_PTR(void))(row_sums)));

  const PlaceOf<PACKED> at(a, blockIdx.x);
  const int i = a.by_splits(at.blk), split = at.blk - i * a.key_splits, bh = at.bh, b = at.b, kvh = at.kvh;
  const auto seq = Seq<PACKED>::template of<BN, true>(a, b, i, true);
  if (!seq.real) return;
  const Lengths& len = seq.len;
  const int blk = seq.slot, j0 = seq.blk * BN, keys = min_of(len.k - j0, BN);
  if (keys <= 0) return;
  const int key = j0 + wave * 32 + n;
  const bool real = wave * 32 + n < keys;
  // queries [lo, hi) see a key of this block in their window
  const int lo = max_of(0, j0 - a.right - len.shift), hi = min_of(len.q, max_of(0, j0 + keys + a.left - len.shift));
  // this work-group's run of their tiles, head by head
  const int per_head = hi > lo ? (hi - lo + QN - 1) / QN : 0, per = a.by_splits(per_head * a.group + a.key_splits - 1);
  const int tiles_n = max_of(0, min_of(per, per_head * a.group - split * per)), head = split && per_head ? split * per / per_head : 0;
  const int start = lo + (split * per - head * per_head) * QN;
  const typename QTile::Loader q_load(a.q.row, wave, lane), g_load(a.d_o.row, wave, lane);
  const typename QTile::RowReader read(lane);
  const typename QTile::ColumnReader cols(lane);
  // The tile to ask for next, with its rows' sums.
  int begin = start;
  const char *q_at = a.q.at(b, kvh * a.group + head, seq.q0 + start), *g_at = a.d_o.at(b, kvh * a.group + head, seq.q0 + start);
  const int64_t q_step = QN * a.q.row, g_step = QN * a.d_o.row, q_back = a.q.head - per_head * q_step, g_back = a.d_o.head - per_head * g_step;
  const float2* sums_at = a.sums + (int64_t(b) * a.heads + kvh * a.group + head) * a.n_q + seq.q0 + start;
  auto pass = [&] {
    begin += QN;
    q_at += q_step;
    g_at += g_step;
    sums_at += QN;
    if (begin >= hi) {                               // the next head's first
      begin = lo;
      q_at += q_back;
      g_at += g_back;
      sums_at += a.n_q - per_head * QN;
    }
  };
  auto issue = [&](int buf) {
    const uint32_t to = lds + uint32_t(buf * 2 * QTile::BYTES);
    q_load.issue(q_at, hi - begin, a.q.row, to, wave);
    g_load.issue(g_at, hi - begin, a.d_o.row, to + QTile::BYTES, wave);
    if (wave == 0) load_sums<QN>(sums_at, hi - begin, lds_sums + uint32_t(buf * QN * 8), lane);
#pragma unroll
    for (int i = 0; i < QG; ++i) pass();
  };
  if (QG == 2 && qg) pass();
  if (tiles_n > 0) {
    if (V_LDS && qg == 0) {
      const typename VTile::Loader v_load(a.v.row, wave, lane);
      v_load.issue(a.v.at(b, kvh, seq.k0 + j0), keys, a.v.row, lds_v, wave);
    }
    if (qg < tiles_n) issue(0);
  }
  typename Mat<T>::Frag kf[STEPS], vf[V_LDS ? 1 : STEPS];
  {
    const char *kp = a.k.at(b, kvh, seq.k0 + (real ? key : j0)), *vp = a.v.at(b, kvh, seq.k0 + (real ? key : j0));
#pragma unroll
    for (int s = 0; s < STEPS; ++s) {
      kf[s] = *reinterpret_cast<const typename Mat<T>::Frag*>(kp + (2 * s + h) * 16);
      if (!V_LDS) vf[V_LDS ? 0 : s] = *reinterpret_cast<const typename Mat<T>::Frag*>(vp + (2 * s + h) * 16);
    }
  }
  f32x16 dk[D / 32], dv[D / 32];
  clear(dk);
  clear(dv);
  const float c2 = a.scale * LOG2E;
  int row0 = start;                                  // first query of this tile
  auto next_row0 = [&] {
    row0 += QN;
    if (row0 >= hi) row0 = lo;
  };
  if (QG == 2 && qg) next_row0();
  // bf16: LDS addresses of a lane's operands by rows and by columns in this tile's queries, by rows in the values; the others follow by XOR of the chunk, so that
  // three registers do for forty.
  uint32_t row_at = lds + read.at + ((uint32_t(h) ^ read.sw) * 16), col_at = lds + cols.at[0][0], val_at = lds_v + uint32_t(wave * 32 * QTile::RB) + read.at + ((uint32_t(h) ^ read.sw) * 16);
  int to_other = 2 * QTile::BYTES;
  for (int t = 0; t * QG < tiles_n; ++t) {
    wait_loads();
    __syncthreads();
    const uint32_t buf = lds + uint32_t((t & 1) * 2 * QTile::BYTES);
    if ((t + 1) * QG + qg < tiles_n) issue((t + 1) & 1);
    if (QG == 2 && t * QG + qg >= tiles_n) break;    // an odd number of tiles: the other group has the last one
    auto part = [&](auto half_) __attribute__((always_inline)) {
      constexpr int half = decltype(half_)::value;
      const int first = row0 + 32 * half, p0 = first + len.shift;          // first query of the 32
      const bool whole = first + 32 <= hi && keys == BN && j0 + BN - 1 <= p0 + a.right && j0 >= p0 + 31 - a.left;
      auto mask = [&](f32x16& s) __attribute__((always_inline)) {
        if (whole) return;
        asm volatile("");                              // keeps this a branch
        const int p = p0 + 4 * h;
        keep(s, key - a.right - p, min_of(key + a.left - p, hi - 1 - first - 4 * h), -INFINITY);
      };
      f32x16 s, g;
#pragma unroll
      for (int i = 0; i < 16; ++i) s[i] = g[i] = 0.f;
      if constexpr (sizeof(T) == 2) {
        // The four products in issue order, operands asked for AHEAD of their instruction, the weights worked out beside the second product and dS beside the
        // third; scheduling fences keep it so, and keep operands that are asked for early from driving the accumulators to scratch.
        constexpr uint32_t AT = half * 32 * QTile::RB;
        constexpr int CS2 = 2 * (D / 32), NF = 2 * STEPS + 2 * CS2, AHEAD = D == 64 ? 3 : 2;
        bf16x8 frag[NF], vfrag[STEPS];
        f32x4 sums4[16 / 2];
        Weights<T> w, ws;
        auto by_rows = [](uint32_t at) { return __builtin_bit_cast(bf16x8, *reinterpret_cast<LDS_PTR(const u32x4)>(at)); };
        auto by_columns = [&](uint32_t at, int s, int c) {
          constexpr uint32_t FAR = uint32_t(QTile::swizzle(8)) * 16;        // rows 8 further on: their chunks are swapped by this
          const uint32_t lo = (at ^ uint32_t(64 * c)) + uint32_t(16 * s * QTile::RB), hi = (at ^ (uint32_t(64 * c) ^ FAR)) + uint32_t((16 * s + 8) * QTile::RB);
          const s16x4 x = __builtin_amdgcn_ds_read_tr16_b64_v4i16(reinterpret_cast<LDS_PTR(s16x4)>(lo));
          const s16x4 y = __builtin_amdgcn_ds_read_tr16_b64_v4i16(reinterpret_cast<LDS_PTR(s16x4)>(hi));
          return __builtin_bit_cast(bf16x8, __builtin_shufflevector(x, y, 0, 1, 2, 3, 4, 5, 6, 7));
        };
        auto load = [&](int f) {
          constexpr int C = D / 32;
          if (f < STEPS) frag[f] = by_rows((row_at ^ uint32_t(32 * f)) + AT);
          else if (f < 2 * STEPS) {
            frag[f] = by_rows((row_at ^ uint32_t(32 * (f - STEPS))) + QTile::BYTES + AT);
            if (V_LDS) vfrag[f - STEPS] = by_rows(val_at ^ uint32_t(32 * (f - STEPS)));
          } else if (f < 2 * STEPS + CS2) frag[f] = by_columns(col_at + QTile::BYTES + AT, (f - 2 * STEPS) / C, (f - 2 * STEPS) % C);
          else frag[f] = by_columns(col_at + AT, (f - 2 * STEPS - CS2) / C, (f - 2 * STEPS - CS2) % C);
        };
        asm volatile("" : "+v"(row_at), "+v"(col_at), "+v"(val_at));
#pragma unroll
        for (int f = 0; f < AHEAD; ++f) load(f);
        __builtin_amdgcn_sched_barrier(0);
#pragma unroll
        for (int f = 0; f < NF; ++f) {
          if (f == STEPS) {
            mask(s);
            __builtin_amdgcn_sched_barrier(0);
          }
          if (f + AHEAD < NF) load(f + AHEAD);
#pragma unroll
          for (int i = 0; i < 8; ++i)                  // two rows' sums two slots ahead of theirs, for the weights and, without room for them, again for dS
            if (f == STEPS + i * STEPS / 8 - 2 || (D == 128 && f == 2 * STEPS + i * CS2 / 8 - 2))
              sums4[i] = *reinterpret_cast<const f32x4*>(&row_sums[t & 1][32 * half + 8 * (i / 2) + 4 * h + i % 2 * 2]);
          if (f < STEPS) s = Mat<T>::mma(frag[f], kf[f], s);
          else if (f < 2 * STEPS) g = Mat<T>::mma(frag[f], V_LDS ? vfrag[f - STEPS] : vf[V_LDS ? 0 : f - STEPS], g);
          else if (f < 2 * STEPS + CS2) {
            const int j = f - 2 * STEPS;
            dv[j % (D / 32)] = __builtin_amdgcn_mfma_f32_32x32x16_bf16(frag[f], __builtin_bit_cast(bf16x8, w.p[j / (D / 32)]), dv[j % (D / 32)], 0, 0, 0);
          } else {
            const int j = f - 2 * STEPS - CS2;
            dk[j % (D / 32)] = __builtin_amdgcn_mfma_f32_32x32x16_bf16(frag[f], __builtin_bit_cast(bf16x8, ws.p[j / (D / 32)]), dk[j % (D / 32)], 0, 0, 0);
          }
          if (f >= STEPS && f < 2 * STEPS) {           // 16 weights over STEPS slots
            constexpr int E = 16 / STEPS;
            const int j = f - STEPS;
#pragma unroll
            for (int i = E * j; i < E * j + E; ++i) {
              s[i] = __builtin_amdgcn_exp2f(fmaf(s[i], c2, -sums4[i / 2][i % 2 * 2]));
              if (i % 2) {
                const bf16x2 pair = {(__bf16)s[i - 1], (__bf16)s[i]};
                w.p[i / 8][i % 8 / 2] = __builtin_bit_cast(uint32_t, pair);
              }
            }
          }
          if (f >= 2 * STEPS && f < 2 * STEPS + CS2) {
            constexpr int E = 16 / CS2;
            const int j = f - 2 * STEPS;
#pragma unroll
            for (int i = E * j; i < E * j + E; ++i) {
              g[i] = s[i] * (g[i] - sums4[i / 2][i % 2 * 2 + 1]);
              if (i % 2) {
                const bf16x2 pair = {(__bf16)g[i - 1], (__bf16)g[i]};
                ws.p[i / 8][i % 8 / 2] = __builtin_bit_cast(uint32_t, pair);
              }
            }
          }
          __builtin_amdgcn_sched_barrier(0);
        }
      } else {
#pragma unroll
        for (int st = 0; st < STEPS; ++st) {
          s = Mat<T>::mma(read.get(buf, 0, st), kf[st], s);
          g = Mat<T>::mma(read.get(buf + QTile::BYTES, 0, st), vf[V_LDS ? 0 : st], g);
        }
        mask(s);
#pragma unroll
        for (int i = 0; i < 16; ++i) {
          const int row = 8 * (i / 4) + 4 * h + i % 4;
          s[i] = __builtin_amdgcn_exp2f(fmaf(s[i], c2, -row_sums[t & 1][row].x));
          g[i] = s[i] * (g[i] - row_sums[t & 1][row].y);
        }
        Weights<T> w;
        w.set(s);
        cols.mma(buf + QTile::BYTES, 0, w, dv);
        w.set(g);
        cols.mma(buf, 0, w, dk);
      }
    };
    part(std::integral_constant<int, 0>{});
    if constexpr (HALVES == 2) part(std::integral_constant<int, 1>{});
#pragma unroll
    for (int i = 0; i < QG; ++i) next_row0();
    row_at += to_other;
    col_at += to_other;
    to_other = -to_other;
  }
  if constexpr (QG == 2) {                           // the first group adds up keys' gradients, the second those of values
    static_assert(D / 2 * 64 * 4 * NW <= QG * 4 * QTile::BYTES, "four waves' sums fit where the tiles were");
    float* all = reinterpret_cast<float*>(tiles) + (wave * (D / 2) * 64 + lane);
    auto give = [&](const f32x16 (&x)[D / 32]) {
#pragma unroll
      for (int c = 0; c < D / 32; ++c)
#pragma unroll
        for (int i = 0; i < 16; ++i) all[(c * 16 + i) * 64] = x[c][i];
    };
    auto take = [&](f32x16 (&x)[D / 32]) {
#pragma unroll
      for (int c = 0; c < D / 32; ++c)
#pragma unroll
        for (int i = 0; i < 16; ++i) x[c][i] += all[(c * 16 + i) * 64];
    };
    __syncthreads();
    if (qg == 1) give(dk);
    __syncthreads();
    if (qg == 0) take(dk);
    __syncthreads();
    if (qg == 0) give(dv);
    __syncthreads();
    if (qg == 1) take(dv);
  }
  // A key that no window has in it may hold anything: its products may be too.
  if (!(key <= len.k - 1 + a.right && key >= len.shift - a.left)) {
    clear(dk);
    clear(dv);
  }
  if (a.key_splits > 1 || blk * NW + wave < a.first_tiles) {           // window_dkv_sum_kernel adds the parts
    float* mine = key_part(a, D, bh, blk * NW + wave, split) + lane;
#pragma unroll
    for (int c = 0; c < D / 32; ++c)
#pragma unroll
      for (int i = 0; i < 16; ++i) {
        if (qg == 0) mine[(c * 16 + i) * 64] = dk[c][i];
        if (QG == 1 || qg == 1) mine[(D / 2 + c * 16 + i) * 64] = dv[c][i];
      }
    return;
  }
  if (!real) return;
#pragma unroll
  for (int c = 0; c < D / 32; ++c)
#pragma unroll
    for (int i = 0; i < 16; i += 4) {
      const float x[4] = {dk[c][i], dk[c][i + 1], dk[c][i + 2], dk[c][i + 3]}, y[4] = {dv[c][i], dv[c][i + 1], dv[c][i + 2], dv[c][i + 3]};
      if (qg == 0) store_four<T>(a.dk.at(b, kvh, seq.k0 + key), 32 * c + 2 * i + 4 * h, x, a.scale);
      if (QG == 1 || qg == 1) store_four<T>(a.dv.at(b, kvh, seq.k0 + key), 32 * c + 2 * i + 4 * h, y, 1.f);
    }
}

// The first keys against the queries that see them only because they are first.  Every query is one, so the queries are split over work-groups, and
// the waves of one take tiles of 32 queries in turn against 32 keys; tiles are a wave's own, so that nothing waits for another wave.  Bound by the way of q and
// do: 17 550 x 30, d = 64, 16 first keys: 31 us, 4.3 TB/s; 2 x 4 001 x 32, d = 128, 4 first keys: 24 us.
template <typename T, int D> constexpr int first_waves() { return sizeof(T) == 4 && D == 128 ? 2 : 4; }
template <typename T, int D>
__global__ void __launch_bounds__((64 * first_waves<T, D>()), 1) window_first_kernel(WindowArgs a) {
  constexpr int NW = first_waves<T, D>(), QN = 32;
  using QTile = Tile<T, D, QN, 1, false>;
  constexpr int STEPS = QTile::STEPS, ACC = D / 2;   // ACC: accumulators of a lane for one of the two gradients
  static_assert(2 * ACC * 64 * 4 <= 4 * QTile::BYTES, "a wave's sums fit where its tiles were");
  __shared__ __attribute__((aligned(1024))) char tiles[NW * 4 * QTile::BYTES];
  __shared__ __attribute__((aligned(1024))) float2 row_sums[NW][2][QN];
  const int lane = threadIdx.x & 63, wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6), n = lane & 31, h = lane >> 5;
  const uint32_t lds = uint32_t(reinterpret_cast<uintptr_t>((LDS_PTR(void))(tiles))) + uint32_t(wave * 4 * QTile::BYTES);

  const int split = blockIdx.x % a.first_splits, tile = blockIdx.x / a.first_splits % a.first_tiles, bh = blockIdx.x / a.first_splits / a.first_tiles;
  const int b = bh / a.heads_kv, kvh = bh % a.heads_kv;
  const Lengths len(a, b);
  const int key = tile * 32 + n, last = min_of(a.sinks, len.k), at_key = key < last ? key : 0;
  const int lo = max_of(0, a.left + tile * 32 + 1 - len.shift), hi = len.q;            // queries of which the window is behind the tile's first key
  const int per_head = tile * 32 < last && hi > lo ? (hi - lo + QN - 1) / QN : 0, tiles_n = per_head * a.group;
  const typename QTile::Loader q_load(a.q.row, 0, lane), g_load(a.d_o.row, 0, lane);
  const typename QTile::RowReader read(lane);
  const typename QTile::ColumnReader cols(lane);
  auto issue = [&](int t, int buf) {
    const int head = kvh * a.group + t / per_head, begin = lo + t % per_head * QN;
    const uint32_t to = lds + uint32_t(buf * 2 * QTile::BYTES);
    q_load.issue(a.q.at(b, head, begin), hi - begin, a.q.row, to, 0);
    g_load.issue(a.d_o.at(b, head, begin), hi - begin, a.d_o.row, to + QTile::BYTES, 0);
    load_sums<QN>(a.sums + (int64_t(b) * a.heads + head) * a.n_q + begin, hi - begin,
                  uint32_t(reinterpret_cast<uintptr_t>((LDS_PTR(void))(row_sums))) + uint32_t((wave * 2 + buf) * QN * 8), lane);
  };
  f32x16 dk[D / 32], dv[D / 32];
  clear(dk);
  clear(dv);
  const int t0 = split * NW + wave, step = a.first_splits * NW;
  if (t0 < tiles_n) {
    issue(t0, 0);
    typename Mat<T>::Frag kf[STEPS], vf[STEPS];
    const char *kp = a.k.at(b, kvh, at_key), *vp = a.v.at(b, kvh, at_key);
#pragma unroll
    for (int s = 0; s < STEPS; ++s) {
      kf[s] = *reinterpret_cast<const typename Mat<T>::Frag*>(kp + (2 * s + h) * 16);
      vf[s] = *reinterpret_cast<const typename Mat<T>::Frag*>(vp + (2 * s + h) * 16);
    }
    const float c2 = a.scale * LOG2E;
    int parity = 0;
    for (int t = t0; t < tiles_n; t += step, parity ^= 1) {
      const int row0 = lo + t % per_head * QN, p0 = row0 + len.shift;
      wait_loads_but<0>();
      wait_reads();                                  // of the tile before, whose place the next one takes
      if (t + step < tiles_n) issue(t + step, parity ^ 1);
      const uint32_t buf = lds + uint32_t(parity * 2 * QTile::BYTES);
      f32x16 s, g;
#pragma unroll
      for (int i = 0; i < 16; ++i) s[i] = g[i] = 0.f;
#pragma unroll
      for (int st = 0; st < STEPS; ++st) {
        s = Mat<T>::mma(read.get(buf, 0, st), kf[st], s);
        g = Mat<T>::mma(read.get(buf + QTile::BYTES, 0, st), vf[st], g);
      }
#pragma unroll
      for (int i = 0; i < 16; ++i) {
        const int row = 8 * (i / 4) + 4 * h + i % 4;
        const bool see = (key < last) & (key < p0 + row - a.left) & (row0 + row < hi);
        const float2 sums = row_sums[wave][parity][row];
        const float x = __builtin_amdgcn_exp2f(fmaf(s[i], c2, -sums.x)), d = x * (g[i] - sums.y);
        s[i] = see ? x : 0.f;
        g[i] = see ? d : 0.f;
      }
      Weights<T> w;
      w.set(s);
      cols.mma(buf + QTile::BYTES, 0, w, dv);
      w.set(g);
      cols.mma(buf, 0, w, dk);
    }
  }
  __syncthreads();
  float* all = reinterpret_cast<float*>(tiles);
#pragma unroll
  for (int c = 0; c < D / 32; ++c)
#pragma unroll
    for (int i = 0; i < 16; ++i) {
      all[(wave * 2 * ACC + c * 16 + i) * 64 + lane] = dk[c][i];
      all[(wave * 2 * ACC + ACC + c * 16 + i) * 64 + lane] = dv[c][i];
    }
  __syncthreads();
  float* mine = first_part(a, D, bh, tile, split);
  for (int i = threadIdx.x; i < 2 * ACC * 64; i += 64 * NW) {
    float x = all[i];
#pragma unroll
    for (int w = 1; w < NW; ++w) x += all[w * 2 * ACC * 64 + i];
    mine[i] = x;
  }
}

// Adds up what the work-groups that share a block of keys left, and those of the first keys.  A thread takes four channels of a key.
template <typename T, int D, bool PACKED>
__global__ void __launch_bounds__(256) window_dkv_sum_kernel(WindowArgs a, int tiles) {
  const int tile = blockIdx.x % tiles, bh = blockIdx.x / tiles, b = bh / a.heads_kv, kvh = bh % a.heads_kv;
  const auto seq = Seq<PACKED>::template of<128, true>(a, b, tile / 4, false);
  if (!seq.real) return;
  const int at = blockIdx.y * 256 + threadIdx.x, lane = at % 64, j = at / 64 * 4, which = j / (D / 2), key = seq.blk * 128 + tile % 4 * 32 + lane % 32;
  if (key >= seq.len.k) return;
  float x[4] = {};
#pragma unroll 8
  for (int s = 0; s < a.key_splits; ++s) add_four(x, key_part(a, D, bh, tile, s) + j * 64 + lane);
  if (tile < a.first_tiles) {
#pragma unroll 8
    for (int s = 0; s < a.first_splits; ++s) add_four(x, first_part(a, D, bh, tile, s) + j * 64 + lane);
  }
  store_four<T>((which ? a.dv : a.dk).at(b, kvh, seq.k0 + key), channel_of(j % (D / 2), lane), x, which ? 1.f : a.scale);
}

// Blocks of a key head: of `rows` rows 128 at a time, with packed sequences one more for each.
template <bool PACKED> static int64_t blocks_of(const WindowArgs& a, int64_t rows) { return PACKED ? rows / 128 + a.packed : (rows + 127) / 128; }

template <typename T, int D, bool PACKED>
static int launch(const char* call, const WindowArgs& args, hipStream_t st) {
  WindowArgs a = args;
  const int64_t seqs = int64_t(a.batch) * a.heads_kv;
  if (a.n_q > 0) {
    a.by_splits = Div(uint32_t(a.row_splits));
    a.set_blocks(blocks_of<PACKED>(a, int64_t(a.group) * a.n_q) * a.row_splits);
    if constexpr (sizeof(T) == 2) window_dq_kernel<D, PACKED><<<unsigned(a.blocks * seqs), 256, 0, st>>>(a);
    else window_dq_f32_kernel<D, PACKED><<<unsigned(a.blocks * seqs), 256, 0, st>>>(a);
    if (int rc = launch_status(call)) return rc;
    if (a.row_splits > 1) {
      window_dq_sum_kernel<T, D, PACKED><<<dim3(unsigned(a.blocks / a.row_splits * 4 * seqs), D / 32), 256, 0, st>>>(a);
      if (int rc = launch_status(call)) return rc;
    }
  }
  if (a.n_k == 0) return DFS_OK;
  a.by_splits = Div(uint32_t(a.key_splits));
  a.set_blocks(blocks_of<PACKED>(a, a.n_k) * a.key_splits);
  bool two = false;
  if constexpr (PACKED && sizeof(T) == 2) two = a.query_groups == 2;
  if constexpr (PACKED && sizeof(T) == 2)
    if (two) window_dkv_kernel<T, D, PACKED, 2><<<unsigned(a.blocks * seqs), 512, 0, st>>>(a);
  if (!two) window_dkv_kernel<T, D, PACKED, 1><<<unsigned(a.blocks * seqs), 256, 0, st>>>(a);
  if (int rc = launch_status(call)) return rc;
  if constexpr (!PACKED)
    if (a.first_tiles > 0) {
      window_first_kernel<T, D><<<unsigned(seqs * a.first_tiles * a.first_splits), 64 * first_waves<T, D>(), 0, st>>>(a);
      if (int rc = launch_status(call)) return rc;
    }
  if (a.key_tiles > 0) window_dkv_sum_kernel<T, D, PACKED><<<dim3(unsigned(seqs * a.key_tiles), D / 16), 256, 0, st>>>(a, a.key_tiles);
  return launch_status(call);
}

template <bool PACKED> static int run_bwd(const char* call, const WindowArgs& a, int d, int dtype, hipStream_t st) {
  if (dtype == DFS_BF16) return d == 64 ? launch<uint16_t, 64, PACKED>(call, a, st) : launch<uint16_t, 128, PACKED>(call, a, st);
  return d == 64 ? launch<float, 64, PACKED>(call, a, st) : launch<float, 128, PACKED>(call, a, st);
}

}  // namespace dfs
