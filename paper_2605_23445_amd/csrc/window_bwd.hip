// Backward pass of attention over a window and a few first keys: the queries' gradient, then those of keys and values.
//
// The first kernel goes over keys for a block of queries, as the forward pass does, and leaves delta = <do, o> of every row; the second goes over queries
// for a block of keys, head by head of those that share it, so that every sum is one work-group's and no atomics are needed.  Both work the weights
// out anew from the log-sum-exp.
#include <float.h>
#include <math.h>

#include "window.h"

namespace dfs {

template <typename T, int D>
__global__ void __launch_bounds__(256, 1) window_dq_kernel(WindowArgs a) {
  constexpr int NW = 4, BM = 32 * NW, KN = 64;
  using KTile = Tile<T, D, KN, NW, false>;
  constexpr int STEPS = KTile::STEPS;
  __shared__ __attribute__((aligned(1024))) char tiles[4 * KTile::BYTES];
  const uint32_t lds = uint32_t(reinterpret_cast<uintptr_t>((LDS_PTR(void))(tiles)));
  const int lane = threadIdx.x & 63, wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6), n = lane & 31, h = lane >> 5;

  const int id = xcd_order(blockIdx.x, gridDim.x), blk = id % a.blocks, bh = id / a.blocks, b = bh / a.heads_kv, kvh = bh % a.heads_kv;
  const Lengths len(a, b);
  const int64_t r0 = int64_t(blk) * BM, left = int64_t(len.q) * a.group - r0;
  const int rows = left < BM ? int(left) : BM;
  if (rows <= 0) return;
  const int i0 = int(r0 / a.group), i1 = int((r0 + rows - 1) / a.group);
  const Span<KN> span(a, i0 + len.shift, i1 + len.shift, len.k);

  const int64_t r = r0 + wave * 32 + n;
  const bool real = wave * 32 + n < rows;
  const int qi = real ? int(r / a.group) : i0, qh = kvh * a.group + (real ? int(r % a.group) : 0), p = qi + len.shift;
  typename Mat<T>::Frag qf[STEPS], gf[STEPS];
  const int64_t at = (int64_t(b) * a.heads + qh) * a.n_q + qi;
  float delta = 0.f;
  {
    const char *qp = a.q.at(b, qh, qi), *gp = a.d_o.at(b, qh, qi), *op = a.o.at(b, qh, qi);
#pragma unroll
    for (int s = 0; s < STEPS; ++s) {
      qf[s] = *reinterpret_cast<const typename Mat<T>::Frag*>(qp + (2 * s + h) * 16);
      gf[s] = *reinterpret_cast<const typename Mat<T>::Frag*>(gp + (2 * s + h) * 16);
      const auto of = *reinterpret_cast<const typename Mat<T>::Frag*>(op + (2 * s + h) * 16);
#pragma unroll
      for (int i = 0; i < int(16 / sizeof(T)); ++i) delta = fmaf(float(gf[s][i]), float(of[i]), delta);
    }
    const auto sw = __builtin_amdgcn_permlane32_swap(__float_as_uint(delta), __float_as_uint(delta), false, false);
    delta = __uint_as_float(sw[0]) + __uint_as_float(sw[1]);
    if (real && h == 0) a.delta[at] = delta;
  }
  const float lse = a.lse[at], ref = lse == -INFINITY ? INFINITY : lse * LOG2E;        // a row that sees nothing has weights of zero
  const char *kh = a.k.at(b, kvh, 0), *vh = a.v.at(b, kvh, 0);
  const typename KTile::Loader k_load(a.k.row, wave, lane), v_load(a.v.row, wave, lane);
  const typename KTile::RowReader read(lane);
  const typename KTile::ColumnReader k_cols(lane);
  auto issue = [&](int t) {
    const int begin = span.begin(t), rest = span.end(t) - begin;
    const uint32_t buf = lds + uint32_t((t & 1) * 2 * KTile::BYTES);
    k_load.issue(kh + int64_t(begin) * a.k.row, rest, a.k.row, buf, wave);
    v_load.issue(vh + int64_t(begin) * a.v.row, rest, a.v.row, buf + KTile::BYTES, wave);
  };
  f32x16 acc[D / 32];
  clear(acc);
  const float c2 = a.scale * LOG2E;
  const int key_lo = p - a.left, key_hi = p + a.right;
  if (span.n > 0) issue(0);
  for (int t = 0; t < span.n; ++t) {
    wait_loads();
    __syncthreads();
    if (t + 1 < span.n) issue(t + 1);
    const uint32_t buf = lds + uint32_t((t & 1) * 2 * KTile::BYTES);
    const int begin = span.begin(t), end = span.end(t);
    const bool whole = begin + KN <= end && begin + KN - 1 <= i0 + len.shift + a.right && (t < span.n_first || begin >= i1 + len.shift - a.left);
#pragma unroll
    for (int half = 0; half < 2; ++half) {
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
      if (!whole) {
#pragma unroll
        for (int i = 0; i < 16; ++i) {
          const int key = begin + 32 * half + 8 * (i / 4) + 4 * h + i % 4;
          s[0][i] = sees(key, end, key_lo, key_hi, a.sinks) ? s[0][i] : 0.f;
        }
      }
      Weights<T> w;
      w.set(s[0]);
      k_cols.mma(buf, half, w, acc);
    }
  }
  if (real) store_row<T>(a.dq.at(b, qh, qi), acc, a.scale, h);
}

// Keys as columns: register i of a lane holds query row 8 (i / 4) + 4 h + i % 4 of a half tile, against the lane's key.
template <typename T, int D>
__global__ void __launch_bounds__(256, 1) window_dkv_kernel(WindowArgs a) {
  constexpr int NW = 4, BN = 32 * NW, QN = 64;
  using QTile = Tile<T, D, QN, NW, false>;
  constexpr int STEPS = QTile::STEPS;
  __shared__ __attribute__((aligned(1024))) char tiles[4 * QTile::BYTES];
  __shared__ __attribute__((aligned(16))) float row_ref[2][QN], row_delta[2][QN];
  const uint32_t lds = uint32_t(reinterpret_cast<uintptr_t>((LDS_PTR(void))(tiles)));
  const int lane = threadIdx.x & 63, wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6), n = lane & 31, h = lane >> 5;

  const int id = xcd_order(blockIdx.x, gridDim.x), blk = id % a.blocks, bh = id / a.blocks, b = bh / a.heads_kv, kvh = bh % a.heads_kv;
  const Lengths len(a, b);
  const int j0 = blk * BN, keys = min_of(len.k - j0, BN);
  if (keys <= 0) return;
  const int key = j0 + wave * 32 + n;
  const bool real = wave * 32 + n < keys;
  typename Mat<T>::Frag kf[STEPS], vf[STEPS];
  {
    const char *kp = a.k.at(b, kvh, real ? key : j0), *vp = a.v.at(b, kvh, real ? key : j0);
#pragma unroll
    for (int s = 0; s < STEPS; ++s) {
      kf[s] = *reinterpret_cast<const typename Mat<T>::Frag*>(kp + (2 * s + h) * 16);
      vf[s] = *reinterpret_cast<const typename Mat<T>::Frag*>(vp + (2 * s + h) * 16);
    }
  }
  // queries [lo, hi) see a key of this block
  const int lo = max_of(0, j0 - a.right - len.shift);
  const int hi = j0 < a.sinks ? len.q : int(min_of(len.q, max_of(0, j0 + keys - 1 + a.left - len.shift + 1)));
  const int per_head = hi > lo ? (hi - lo + QN - 1) / QN : 0, tiles_n = per_head * a.group;
  const typename QTile::Loader q_load(a.q.row, wave, lane), g_load(a.d_o.row, wave, lane);
  const typename QTile::RowReader read(lane);
  const typename QTile::ColumnReader cols(lane);
  auto issue = [&](int t) {
    const int head = kvh * a.group + t / per_head, begin = lo + t % per_head * QN, rest = hi - begin;
    const uint32_t buf = lds + uint32_t((t & 1) * 2 * QTile::BYTES);
    q_load.issue(a.q.at(b, head, begin), rest, a.q.row, buf, wave);
    g_load.issue(a.d_o.at(b, head, begin), rest, a.d_o.row, buf + QTile::BYTES, wave);
    if (threadIdx.x < QN) {
      const int64_t at = (int64_t(b) * a.heads + head) * a.n_q + begin + threadIdx.x;
      const bool there = int(threadIdx.x) < rest;
      const float lse = there ? a.lse[at] : -INFINITY;
      row_ref[t & 1][threadIdx.x] = lse == -INFINITY ? INFINITY : lse * LOG2E;
      row_delta[t & 1][threadIdx.x] = there ? a.delta[at] : 0.f;
    }
  };
  f32x16 dk[D / 32], dv[D / 32];
  clear(dk);
  clear(dv);
  const float c2 = a.scale * LOG2E;
  if (tiles_n > 0) issue(0);
  for (int t = 0; t < tiles_n; ++t) {
    wait_loads();
    __syncthreads();
    if (t + 1 < tiles_n) issue(t + 1);
    const uint32_t buf = lds + uint32_t((t & 1) * 2 * QTile::BYTES);
    const int begin = lo + t % per_head * QN, p0 = begin + len.shift;
    const bool whole = begin + QN <= hi && keys == BN && j0 + BN - 1 <= p0 + a.right && j0 >= p0 + QN - 1 - a.left;
#pragma unroll
    for (int half = 0; half < 2; ++half) {
      f32x16 s[1], g[1];
      clear(s);
      clear(g);
#pragma unroll
      for (int st = 0; st < STEPS; ++st) {
        s[0] = Mat<T>::mma(read.get(buf, half, st), kf[st], s[0]);
        g[0] = Mat<T>::mma(read.get(buf + QTile::BYTES, half, st), vf[st], g[0]);
      }
#pragma unroll
      for (int i = 0; i < 16; ++i) {
        const int row = 32 * half + 8 * (i / 4) + 4 * h + i % 4;
        float w = __builtin_amdgcn_exp2f(fmaf(s[0][i], c2, -row_ref[t & 1][row]));
        float d = w * (g[0][i] - row_delta[t & 1][row]);
        if (!whole) {
          const int p = p0 + row;
          const bool see = sees(key, begin + row < hi ? NO_LIMIT : 0, p - a.left, p + a.right, a.sinks);
          w = see ? w : 0.f;
          d = see ? d : 0.f;
        }
        s[0][i] = w;
        g[0][i] = d;
      }
      Weights<T> w;
      w.set(s[0]);
      cols.mma(buf + QTile::BYTES, half, w, dv);
      w.set(g[0]);
      cols.mma(buf, half, w, dk);
    }
  }
  if (!real) return;
  store_row<T>(a.dk.at(b, kvh, key), dk, a.scale, h);
  store_row<T>(a.dv.at(b, kvh, key), dv, 1.f, h);
}

template <typename T, int D>
static int launch(const WindowArgs& args, hipStream_t st) {
  WindowArgs a = args;
  const int64_t seqs = int64_t(a.batch) * a.heads_kv;
  if (a.n_q > 0) {
    a.blocks = int((int64_t(a.group) * a.n_q + 127) / 128);
    window_dq_kernel<T, D><<<unsigned(a.blocks * seqs), 256, 0, st>>>(a);
    if (int rc = launch_status("dfs_window_attn_bwd")) return rc;
  }
  if (a.n_k > 0) {
    a.blocks = (a.n_k + 127) / 128;
    window_dkv_kernel<T, D><<<unsigned(a.blocks * seqs), 256, 0, st>>>(a);
  }
  return launch_status("dfs_window_attn_bwd");
}

int run_window_bwd(const WindowArgs& a, int d, int dtype, hipStream_t st) {
  if (dtype == DFS_BF16) return d == 64 ? launch<uint16_t, 64>(a, st) : launch<uint16_t, 128>(a, st);
  return d == 64 ? launch<float, 64>(a, st) : launch<float, 128>(a, st);
}

}  // namespace dfs
