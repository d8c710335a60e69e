// Backward pass of attention over a window and a few first keys: the queries' gradient, then those of keys and values.
//
// The first kernel goes over keys for a block of queries, as the forward pass does, and leaves delta = <do, o> of every row; the second goes over queries
// for a block of keys, head by head of those that share it, so that every sum is one work-group's and no atomics are needed.  Both work the weights
// out anew from the log-sum-exp.  The second takes the pairs of the windows alone: the first keys, which every query sees, would keep a work-group
// for as long as all others take together.  Their other pairs are dealt to work-groups of a third kernel, and a fourth adds the parts up.
#include <float.h>
#include <math.h>

#include "window.h"

namespace dfs {

// Sums of dk and dv of the 32 first keys of `tile`, as a wave holds them: split `split`, the last one's place is the key blocks'.
__device__ __forceinline__ float* first_part(const WindowArgs& a, int d, int bh, int tile, int split) {
  return a.part + ((int64_t(bh) * a.first_tiles + tile) * (a.first_splits + 1) + split) * 64 * d;
}

template <typename T, int D>
__global__ void __launch_bounds__(256, sizeof(T) == 2 ? 2 : 1) window_dq_kernel(WindowArgs a) {
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
  const int pw0 = int((r0 + wave * 32) / a.group) + len.shift, pw1 = int((r0 + min_of(rows, wave * 32 + 32) - 1) / a.group) + len.shift;    // this wave's positions
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
      if (span.unseen(a, t, begin + 32 * half, end, pw0, pw1)) continue;
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

// Keys as columns: register i of a lane holds query row 8 (i / 4) + 4 h + i % 4 of a tile of 32, against the lane's key.  A lone wave a SIMD issues a vector
// instruction every eight to ten cycles and cannot keep the matrix cores busy, so two work-groups share a CU: in bf16 at d = 128, where the accumulators
// alone take 128 registers, the keys' rows stay in registers and the values' come from LDS in every tile.
template <typename T, int D>
__global__ void __launch_bounds__(256, sizeof(T) == 2 ? 2 : 1) window_dkv_kernel(WindowArgs a) {
  constexpr int NW = 4, BN = 32 * NW, QN = 32;
  constexpr bool V_LDS = sizeof(T) == 2 && D == 128;
  using QTile = Tile<T, D, QN, NW, false>;
  using VTile = Tile<T, D, BN, NW, false>;
  constexpr int STEPS = QTile::STEPS;
  __shared__ __attribute__((aligned(1024))) char tiles[4 * QTile::BYTES + (V_LDS ? VTile::BYTES : 0)];
  __shared__ __attribute__((aligned(16))) float row_ref[2][QN], row_delta[2][QN];
  const uint32_t lds = uint32_t(reinterpret_cast<uintptr_t>((LDS_PTR(void))(tiles))), lds_v = lds + 4 * QTile::BYTES;
  const int lane = threadIdx.x & 63, wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6), n = lane & 31, h = lane >> 5;

  const int id = xcd_order(blockIdx.x, gridDim.x), blk = id % a.blocks, bh = id / a.blocks, b = bh / a.heads_kv, kvh = bh % a.heads_kv;
  const Lengths len(a, b);
  const int j0 = blk * BN, keys = min_of(len.k - j0, BN);
  if (keys <= 0) return;
  const int key = j0 + wave * 32 + n;
  const bool real = wave * 32 + n < keys;
  // queries [lo, hi) see a key of this block in their window
  const int lo = max_of(0, j0 - a.right - len.shift), hi = min_of(len.q, max_of(0, j0 + keys + a.left - len.shift));
  const int per_head = hi > lo ? (hi - lo + QN - 1) / QN : 0, tiles_n = per_head * a.group;
  const typename QTile::Loader q_load(a.q.row, wave, lane), g_load(a.d_o.row, wave, lane);
  const typename QTile::RowReader read(lane);
  const typename QTile::ColumnReader cols(lane);
  // The tile to ask for next, and the sums of the one behind it: asked for in front of a tile's rows, which nothing waits for before the next barrier.
  int head = kvh * a.group, begin = lo, sum_head = head, sum_begin = lo;
  float ref = 0.f, delta = 0.f;
  auto issue = [&](int buf) {
    const uint32_t to = lds + uint32_t(buf * 2 * QTile::BYTES);
    q_load.issue(a.q.at(b, head, begin), hi - begin, a.q.row, to, wave);
    g_load.issue(a.d_o.at(b, head, begin), hi - begin, a.d_o.row, to + QTile::BYTES, wave);
    begin += QN;
    if (begin >= hi) { begin = lo; ++head; }
  };
  auto ask_sums = [&](bool more) {
    if (more && threadIdx.x < QN) {
      const int row = min_of(sum_begin + int(threadIdx.x), hi - 1);
      const int64_t at = (int64_t(b) * a.heads + sum_head) * a.n_q + row;
      ref = a.lse[at];
      delta = a.delta[at];
    }
    sum_begin += QN;
    if (sum_begin >= hi) { sum_begin = lo; ++sum_head; }
  };
  auto keep_sums = [&](int buf) {
    if (threadIdx.x < QN) {
      row_ref[buf][threadIdx.x] = ref == -INFINITY ? INFINITY : ref * LOG2E;            // a row that sees nothing has weights of zero
      row_delta[buf][threadIdx.x] = delta;
    }
  };
  if (tiles_n > 0) {
    ask_sums(true);
    if (V_LDS) {
      const typename VTile::Loader v_load(a.v.row, wave, lane);
      v_load.issue(a.v.at(b, kvh, j0), keys, a.v.row, lds_v, wave);
    }
    keep_sums(0);
    ask_sums(tiles_n > 1);
    issue(0);
  }
  typename Mat<T>::Frag kf[STEPS], vf[V_LDS ? 1 : STEPS];
  {
    const char *kp = a.k.at(b, kvh, real ? key : j0), *vp = a.v.at(b, kvh, real ? key : j0);
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
  int row0 = lo;                                     // first query of this tile
  for (int t = 0; t < tiles_n; ++t) {
    wait_loads();
    __syncthreads();
    const uint32_t buf = lds + uint32_t((t & 1) * 2 * QTile::BYTES);
    if (t + 1 < tiles_n) {
      keep_sums((t + 1) & 1);
      ask_sums(t + 2 < tiles_n);
      issue((t + 1) & 1);
    }
    const int p0 = row0 + len.shift;
    const bool whole = row0 + QN <= hi && keys == BN && j0 + BN - 1 <= p0 + a.right && j0 >= p0 + QN - 1 - a.left;
    f32x16 s, g;
#pragma unroll
    for (int i = 0; i < 16; ++i) s[i] = g[i] = 0.f;
#pragma unroll
    for (int st = 0; st < STEPS; ++st) s = Mat<T>::mma(read.get(buf, 0, st), kf[st], s);
    __builtin_amdgcn_sched_barrier(0);
#pragma unroll
    for (int i = 0; i < 16; ++i) s[i] = __builtin_amdgcn_exp2f(fmaf(s[i], c2, -row_ref[t & 1][8 * (i / 4) + 4 * h + i % 4]));
    if (!whole) {
#pragma unroll
      for (int i = 0; i < 16; ++i) {
        const int row = 8 * (i / 4) + 4 * h + i % 4, p = p0 + row;
        s[i] = sees(key, row0 + row < hi ? NO_LIMIT : 0, p - a.left, p + a.right, 0) ? s[i] : 0.f;
      }
    }
    Weights<T> w;
    w.set(s);
    __builtin_amdgcn_sched_barrier(0);
    cols.mma(buf + QTile::BYTES, 0, w, dv);
    // Phases that the compiler does not mix: with operands asked for across them 64 registers went to scratch.
    __builtin_amdgcn_sched_barrier(0);
#pragma unroll
    for (int st = 0; st < STEPS; ++st)
      g = Mat<T>::mma(read.get(buf + QTile::BYTES, 0, st), V_LDS ? read.get(lds_v, wave, st) : vf[V_LDS ? 0 : st], g);
    __builtin_amdgcn_sched_barrier(0);
#pragma unroll
    for (int i = 0; i < 16; ++i) {
      const float d = s[i] * (g[i] - row_delta[t & 1][8 * (i / 4) + 4 * h + i % 4]);
      g[i] = whole ? d : s[i] == 0.f ? 0.f : d;      // where nothing is seen <do, v> may be anything
    }
    w.set(g);
    __builtin_amdgcn_sched_barrier(0);
    cols.mma(buf, 0, w, dk);
    row0 += QN;
    if (row0 >= hi) row0 = lo;
  }
  if (blk * NW + wave < a.first_tiles) {             // the first keys' part is added by window_first_sum_kernel
    float* mine = first_part(a, D, bh, blk * NW + wave, a.first_splits) + lane;
#pragma unroll
    for (int c = 0; c < D / 32; ++c)
#pragma unroll
      for (int i = 0; i < 16; ++i) {
        mine[(c * 16 + i) * 64] = dk[c][i];
        mine[(D / 2 + c * 16 + i) * 64] = dv[c][i];
      }
    return;
  }
  if (!real) return;
  store_row<T>(a.dk.at(b, kvh, key), dk, a.scale, h);
  store_row<T>(a.dv.at(b, kvh, key), dv, 1.f, h);
}

// The first keys against the queries that see them only because they are first.  Every query is one, so the queries are split over work-groups, and
// the waves of one take tiles of 32 queries in turn against 32 keys; tiles are a wave's own, so that nothing waits for another wave.
template <typename T, int D> constexpr int first_waves() { return sizeof(T) == 4 && D == 128 ? 2 : 4; }
template <typename T, int D>
__global__ void __launch_bounds__((64 * first_waves<T, D>()), 1) window_first_kernel(WindowArgs a) {
  constexpr int NW = first_waves<T, D>(), QN = 32;
  using QTile = Tile<T, D, QN, 1, false>;
  constexpr int STEPS = QTile::STEPS, ACC = D / 2;   // ACC: accumulators of a lane for one of the two gradients
  static_assert(2 * ACC * 64 * 4 <= 4 * QTile::BYTES, "a wave's sums fit where its tiles were");
  __shared__ __attribute__((aligned(1024))) char tiles[NW * 4 * QTile::BYTES];
  __shared__ __attribute__((aligned(16))) float row_ref[NW][QN], row_delta[NW][QN];
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
      const int64_t at = (int64_t(b) * a.heads + kvh * a.group + t / per_head) * a.n_q + min_of(row0 + n, hi - 1);
      const float ref = a.lse[at], delta = a.delta[at];
      row_ref[wave][n] = ref == -INFINITY ? INFINITY : ref * LOG2E;
      row_delta[wave][n] = delta;
      wait_loads();
      __builtin_amdgcn_fence(__ATOMIC_ACQ_REL, "wavefront");
      __builtin_amdgcn_wave_barrier();
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
        const float x = __builtin_amdgcn_exp2f(fmaf(s[i], c2, -row_ref[wave][row])), d = x * (g[i] - row_delta[wave][row]);
        s[i] = see ? x : 0.f;
        g[i] = see ? d : 0.f;
      }
      Weights<T> w;
      w.set(s);
      cols.mma(buf + QTile::BYTES, 0, w, dv);
      w.set(g);
      cols.mma(buf, 0, w, dk);
      __builtin_amdgcn_fence(__ATOMIC_ACQ_REL, "wavefront");
      __builtin_amdgcn_wave_barrier();               // the next round's sums stay behind this one's reads
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

// Adds up what the blocks of keys and the splits left of the first keys' gradients.  A thread takes four channels of a key.
template <typename T, int D>
__global__ void __launch_bounds__(256) window_first_sum_kernel(WindowArgs a) {
  const int tile = blockIdx.x % a.first_tiles, bh = blockIdx.x / a.first_tiles, b = bh / a.heads_kv, kvh = bh % a.heads_kv;
  const Lengths len(a, b);
  const int at = blockIdx.y * 256 + threadIdx.x, lane = at % 64, i = at / 64 * 4 % (D / 2), which = at / 64 * 4 / (D / 2);
  const int key = tile * 32 + lane % 32, ch = i / 16 * 32 + i % 16 * 2 + lane / 32 * 4;
  if (key >= len.k) return;
  float x[4] = {};
  for (int s = 0; s <= a.first_splits; ++s) {
    const float* p = first_part(a, D, bh, tile, s) + (which * (D / 2) + i) * 64 + lane;
#pragma unroll
    for (int j = 0; j < 4; ++j) x[j] += p[j * 64];
  }
  store_four<T>((which ? a.dv : a.dk).at(b, kvh, key), ch, x, which ? 1.f : a.scale);
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
  if (a.n_k == 0) return DFS_OK;
  a.blocks = (a.n_k + 127) / 128;
  window_dkv_kernel<T, D><<<unsigned(a.blocks * seqs), 256, 0, st>>>(a);
  if (int rc = launch_status("dfs_window_attn_bwd")) return rc;
  if (a.first_tiles > 0) {
    window_first_kernel<T, D><<<unsigned(seqs * a.first_tiles * a.first_splits), 64 * first_waves<T, D>(), 0, st>>>(a);
    if (int rc = launch_status("dfs_window_attn_bwd")) return rc;
    window_first_sum_kernel<T, D><<<dim3(unsigned(seqs * a.first_tiles), D / 16), 256, 0, st>>>(a);
  }
  return launch_status("dfs_window_attn_bwd");
}

int run_window_bwd(const WindowArgs& a, int d, int dtype, hipStream_t st) {
  if (dtype == DFS_BF16) return d == 64 ? launch<uint16_t, 64>(a, st) : launch<uint16_t, 128>(a, st);
  return d == 64 ? launch<float, 64>(a, st) : launch<float, 128>(a, st);
}

}  // namespace dfs
