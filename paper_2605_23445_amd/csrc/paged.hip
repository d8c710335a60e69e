// Attention over a cache in pages: few rows of each sequence over long lists of keys.
//
// The rows of 32 queries (of all heads that share a key head) and the keys that they see, in pieces of 32, are an item.  How many pieces there are is known on the device
// alone, so the pieces of all items, put behind one another, are dealt out to the work-groups in equal runs: one may end an item, take whole ones and begin
// another.  An item that one work-group has whole is stored at once, parts of items go to the workspace, and a second kernel joins them.
//
// Within a work-group the waves take pieces in turn, each with tiles of its own, so that none waits for another before the end of a run of pieces; but for what is being
// worked on the LDS is full of loads on their way.  Pieces begin at multiples of 32, so that each lies on one page, or with pages of 16 rows on two.  In 8 bits a tile holds the
// bytes as they lie in memory; they become bf16, times their scale, on the way from LDS to the matrix cores, which is exact.
#include <float.h>
#include <math.h>

#include "paged.h"

namespace dfs {

constexpr int GROUPS = 256;                          // work-groups: one a CU

// A sequence's rows and keys, its blocks of 32 or 16 rows, and the units of each of these with each key head (the pieces of all its rows together, one at least).
struct PagedSeq {
  int q0, n, k, blocks, units;
  PagedSeq() = default;
  __device__ __forceinline__ PagedSeq(const PagedArgs& a, int s) : PagedSeq(a, start_of(a.q_start, s, a.n_q), start_of(a.q_start, s + 1, a.n_q), a.k_len[s]) {}
  __device__ __forceinline__ PagedSeq(const PagedArgs& a, int from, int to, int k_) {
    q0 = from;
    n = max_of(0, to - from);
    k = max_of(0, min_of(k_, a.n_k));
    blocks = (n * a.group + (1 << a.row_bits) - 1) >> a.row_bits;
    const Span all(a, k - n, k - 1, k, 32);
    units = max_of(1, (all.n + a.unit - 1) / a.unit);
  }
  __device__ __forceinline__ int work(const PagedArgs& a) const { return blocks * units * a.heads_kv; }
};

// Units of all sequences in front of each, as a work-group's threads work them out: thread t adds up `each` sequences from t * each on; with up to 64, lane t of every wave
// has sequence t.
template <int NT> struct Deal {
  int each, mine, before, total, per;                // a thread's sum, the sum in front of it, all, and a work-group's share
  PagedSeq last;                                     // a thread's last sequence, which is its only one where there are up to NT
  __device__ __forceinline__ Deal(const PagedArgs& a, int (&sums)[NT / 64]) {
    if (a.packed <= 64) {                            // every wave by itself: no barrier
      const int s = threadIdx.x & 63;
      each = 1;
      last = PagedSeq(a, min_of(s, a.packed - 1));
      mine = s < a.packed ? last.work(a) : 0;
      const int upto = wave_sums(mine);
      before = upto - mine;
      total = __builtin_amdgcn_readlane(upto, 63);
      per = max_of((total + GROUPS - 1) / GROUPS, 1);
      return;
    }
    each = (a.packed + NT - 1) / NT;
    mine = 0;
    for (int i = 0, s = threadIdx.x * each; i < each && s < a.packed; ++i, ++s) {
      last = PagedSeq(a, s);
      mine += last.work(a);
    }
    const int upto = wave_sums(mine), wave = threadIdx.x >> 6;
    if ((threadIdx.x & 63) == 63) sums[wave] = upto;
    __syncthreads();
    before = upto - mine;
    total = 0;
#pragma unroll
    for (int w = 0; w < NT / 64; ++w) {
      if (w < wave) before += sums[w];
      total += sums[w];
    }
    per = max_of((total + GROUPS - 1) / GROUPS, 1);
  }
};

// Tiles of 32 rows of a page's elements in LDS, chunks of 16 bytes swapped within a row so that what is read at once lies in different banks.
template <typename T, int D, bool E4M3, int ROWS = 32> struct PageTile {
  static constexpr int RB = E4M3 ? D : D * int(sizeof(T)), CH = RB / 16, BYTES = 32 * RB, LOADS = BYTES / 1024;
  using Rows = Tile<T, D, 32, 1, false>;
  using Columns = Tile<T, D, 32, 1, true>;
  template <bool COLUMNS> static __device__ __forceinline__ int swizzle(int row) {
    if constexpr (E4M3) return row * RB / 256 % CH;
    else if constexpr (COLUMNS && ROWS == 16 && sizeof(T) == 4) return row / 4 % 4 * 4;      // four rows 4 apart are read at once, 16 channels each
    else return COLUMNS ? Columns::swizzle(row) : Rows::swizzle(row);
  }
  // Byte offset of this lane's chunk of load j of 16 rows.
  template <bool COLUMNS> static __device__ __forceinline__ uint32_t offset(int j, int lane, int64_t stride) {
    const int p = j * 64 + lane, row = p / CH;
    return uint32_t(row) * uint32_t(stride) + uint32_t((p % CH ^ swizzle<COLUMNS>(row)) * 16);
  }
};

// Waves of a work-group: as many as have room in LDS for two tiles of keys and two of values each.
template <typename T, int D, bool E4M3> constexpr int paged_waves() { return 1024 / (D * (E4M3 ? 1 : int(sizeof(T)))) < 8 ? 1024 / (D * (E4M3 ? 1 : int(sizeof(T)))) : 8; }

// The arithmetic of a wave: 32 rows, or 16, against the 32 keys of a tile.  A lane holds, of the logits and of the sums, one row's (n): with 32 rows keys and channels 8 (i / 4) + 4 h +
// i % 4 of 32, h = lane / 32, with 16 rows 4 g + i of 16, g = lane / 16.  Bytes become operands on the way from LDS: of keys a lane reads 16 channels at once, for
// two products; of values the transposing read hands it eight keys of a channel.  H: scales of a tile, of 16 rows each or of all.
template <typename T, int D, bool E4M3, int H> struct Wave32 {
  using PT = PageTile<T, D, E4M3>;
  using Frag = typename Mat<T>::Frag;
  static constexpr int ROWS = 32, STEPS = D * int(sizeof(T)) / 32, REGS = D / 2;
  int lane, n, h;
  Frag qf[STEPS];
  f32x16 acc[D / 32], x;
  Weights<T> w;
  float m, l;
  __device__ __forceinline__ Wave32(int lane_) : lane(lane_), n(lane_ & 31), h(lane_ >> 5) {}
  __device__ __forceinline__ void start(const char* q) {
#pragma unroll
    for (int st = 0; st < STEPS; ++st) qf[st] = *reinterpret_cast<const Frag*>(q + (E4M3 ? st / 2 * 4 + 2 * h + st % 2 : 2 * st + h) * 16);
    clear(acc);
    m = -INFINITY;
    l = 0.f;
  }
  __device__ __forceinline__ void wait_queries() {
#pragma unroll
    for (int st = 0; st < STEPS; ++st) asm volatile("" : "+v"(qf[st]));
  }
  __device__ __forceinline__ void keys(uint32_t buf, const float (&scale)[H]) {
#pragma unroll
    for (int i = 0; i < 16; ++i) x[i] = 0.f;
    if constexpr (E4M3) {
      const float mine = n < 16 ? scale[0] : scale[H - 1];
      u32x4 raw[STEPS / 2];
#pragma unroll
      for (int st = 0; st < STEPS / 2; ++st)
        raw[st] = *reinterpret_cast<LDS_PTR(const u32x4)>(buf + uint32_t(n * PT::RB + ((2 * st + h) ^ PT::template swizzle<false>(n)) * 16));
      __builtin_amdgcn_sched_barrier(0);             // operands that are worked out early drive the accumulators to scratch
#pragma unroll
      for (int st = 0; st < STEPS / 2; ++st) {
        x = Mat<T>::mma(eight(raw[st][0], raw[st][1], mine), qf[2 * st], x);
        x = Mat<T>::mma(eight(raw[st][2], raw[st][3], mine), qf[2 * st + 1], x);
        __builtin_amdgcn_sched_barrier(0);
      }
    } else {
      const typename PT::Rows::RowReader read(lane);
#pragma unroll
      for (int st = 0; st < STEPS; ++st) x = Mat<T>::mma(read.get(buf, 0, st), qf[st], x);
    }
  }
  // Logits to weights; p: the row's position.
  __device__ __forceinline__ void weigh(const PagedArgs& a, const Span& span, int t, int p, float c2) {
    if (!span.whole(t)) span.mask(a, t, p, h, x, -INFINITY);
    float mx = x[0];
#pragma unroll
    for (int i = 1; i < 16; ++i) mx = fmaxf(mx, x[i]);
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
      x[i] = __builtin_amdgcn_exp2f(fmaf(x[i], c2, -ref));
      l += x[i];
    }
    w.set(x);
  }
  __device__ __forceinline__ void values(uint32_t buf, const float (&scale)[H]) {
    if constexpr (E4M3) {
      const int i = (lane & 15) >> 1, row = 4 * h + i + (i < 4 ? 0 : 4);                     // 8 rows of 16 channels from 16 lanes, 8 rows of one channel to each
      i32x2 raw[2][D / 32];
#pragma unroll
      for (int half = 0; half < 2; ++half)
#pragma unroll
        for (int c = 0; c < D / 32; ++c) {
          const uint32_t chunk = uint32_t((2 * c + ((lane >> 4) & 1)) ^ PT::template swizzle<true>(row));
          raw[half][c] = __builtin_amdgcn_ds_read_tr8_b64_v2i32(reinterpret_cast<LDS_PTR(i32x2)>(buf + uint32_t((16 * half + row) * PT::RB) + chunk * 16 + (lane & 1) * 8));
        }
      __builtin_amdgcn_sched_barrier(0);
#pragma unroll
      for (int half = 0; half < 2; ++half)
#pragma unroll
        for (int c = 0; c < D / 32; ++c) {
          acc[c] = __builtin_amdgcn_mfma_f32_32x32x16_bf16(eight(uint32_t(raw[half][c][0]), uint32_t(raw[half][c][1]), scale[half < H ? half : 0]),
                                                           __builtin_bit_cast(bf16x8, w.p[half]), acc[c], 0, 0, 0);
          __builtin_amdgcn_sched_barrier(0);
        }
    } else {
      const typename PT::Columns::ColumnReader read(lane);
      read.mma(buf, 0, w, acc);
    }
  }
  __device__ __forceinline__ void finish() {
    const auto sw = __builtin_amdgcn_permlane32_swap(__float_as_uint(l), __float_as_uint(l), false, false);
    l = __uint_as_float(sw[0]) + __uint_as_float(sw[1]);
  }
  __device__ __forceinline__ float sum(int reg) const { return acc[reg / 16][reg % 16]; }
  __device__ __forceinline__ int channel(int reg) const { return reg / 16 * 32 + reg % 16 * 2 + 4 * h; }         // of the first of four
  __device__ __forceinline__ bool first() const { return h == 0; }
};

template <typename T, int D, bool E4M3, int H> struct Wave16 {
  using PT = PageTile<T, D, E4M3, 16>;
  using Frag = typename Mat<T>::Frag;
  static constexpr int ROWS = 16, STEPS = D * int(sizeof(T)) / 64, REGS = D / 4;
  int lane, n, g;
  Frag qf[STEPS];
  f32x4 acc[D / 16], x[2];
  u32x4 w;                                           // weights in bf16; in fp32 they serve as they are
  float m, l;
  __device__ __forceinline__ Wave16(int lane_) : lane(lane_), n(lane_ & 15), g(lane_ >> 4) {}
  __device__ __forceinline__ void start(const char* q) {
#pragma unroll
    for (int st = 0; st < STEPS; ++st) qf[st] = *reinterpret_cast<const Frag*>(q + (E4M3 ? (st / 2 * 4 + g) * 2 + st % 2 : 4 * st + g) * 16);
#pragma unroll
    for (int c = 0; c < D / 16; ++c) acc[c] = f32x4{0.f, 0.f, 0.f, 0.f};
    m = -INFINITY;
    l = 0.f;
  }
  __device__ __forceinline__ void wait_queries() {
#pragma unroll
    for (int st = 0; st < STEPS; ++st) asm volatile("" : "+v"(qf[st]));
  }
  __device__ __forceinline__ void keys(uint32_t buf, const float (&scale)[H]) {
    x[0] = x[1] = f32x4{0.f, 0.f, 0.f, 0.f};
    auto chunk = [&](int half, int st) {
      const int row = 16 * half + n;
      return *reinterpret_cast<LDS_PTR(const u32x4)>(buf + uint32_t(row * PT::RB + ((4 * st + g) ^ PT::template swizzle<false>(row)) * 16));
    };
    if constexpr (sizeof(T) == 4) {
#pragma unroll
      for (int st = 0; st < STEPS; ++st) {
        const f32x4 k0 = __builtin_bit_cast(f32x4, chunk(0, st)), k1 = __builtin_bit_cast(f32x4, chunk(1, st));
#pragma unroll
        for (int i = 0; i < 4; ++i) {
          x[0] = __builtin_amdgcn_mfma_f32_16x16x4f32(k0[i], qf[st][i], x[0], 0, 0, 0);
          x[1] = __builtin_amdgcn_mfma_f32_16x16x4f32(k1[i], qf[st][i], x[1], 0, 0, 0);
        }
      }
    } else {
      constexpr int READS = E4M3 ? D / 64 : STEPS;
      u32x4 raw[2][READS];
#pragma unroll
      for (int half = 0; half < 2; ++half)
#pragma unroll
        for (int st = 0; st < READS; ++st) raw[half][st] = chunk(half, st);
#pragma unroll
      for (int st = 0; st < READS; ++st)
#pragma unroll
        for (int half = 0; half < 2; ++half) {
          const u32x4 r = raw[half][st];
          if constexpr (E4M3) {
            x[half] = __builtin_amdgcn_mfma_f32_16x16x32_bf16(eight(r[0], r[1], scale[half < H ? half : 0]), qf[2 * st], x[half], 0, 0, 0);
            x[half] = __builtin_amdgcn_mfma_f32_16x16x32_bf16(eight(r[2], r[3], scale[half < H ? half : 0]), qf[2 * st + 1], x[half], 0, 0, 0);
          } else {
            x[half] = __builtin_amdgcn_mfma_f32_16x16x32_bf16(__builtin_bit_cast(bf16x8, r), qf[st], x[half], 0, 0, 0);
          }
        }
    }
  }
  static __device__ __forceinline__ float across(float v, bool add) {    // largest or sum over the four lanes of a row
    const auto a = __builtin_amdgcn_permlane16_swap(__float_as_uint(v), __float_as_uint(v), false, false);
    v = add ? __uint_as_float(a[0]) + __uint_as_float(a[1]) : fmaxf(__uint_as_float(a[0]), __uint_as_float(a[1]));
    const auto b = __builtin_amdgcn_permlane32_swap(__float_as_uint(v), __float_as_uint(v), false, false);
    return add ? __uint_as_float(b[0]) + __uint_as_float(b[1]) : fmaxf(__uint_as_float(b[0]), __uint_as_float(b[1]));
  }
  __device__ __forceinline__ void weigh(const PagedArgs& a, const Span& span, int t, int p, float c2) {
    if (!span.whole(t)) {
      const int key = span.begin(t) + 4 * g, top = min_of(span.end(t) - 1, p), low = t < span.n_first ? 0 : p - a.left, more = t < span.n_first ? 0 : a.sinks;
#pragma unroll
      for (int half = 0; half < 2; ++half)
#pragma unroll
        for (int i = 0; i < 4; ++i) {
          const int j = key + 16 * half + i;
          x[half][i] = ((j <= top) & ((j >= low) | (j < more))) ? x[half][i] : -INFINITY;
        }
    }
    float mx = fmaxf(x[0][0], x[1][0]);
#pragma unroll
    for (int i = 1; i < 4; ++i) mx = fmaxf(mx, fmaxf(x[0][i], x[1][i]));
    const float m_new = fmaxf(m, across(mx, false) * c2), ref = m_new == -INFINITY ? 0.f : m_new;
    if (__builtin_amdgcn_ballot_w64(m_new > m)) {
      const float alpha = __builtin_amdgcn_exp2f(m - ref);
      m = m_new;
      l *= alpha;
#pragma unroll
      for (int c = 0; c < D / 16; ++c)
#pragma unroll
        for (int i = 0; i < 4; ++i) acc[c][i] *= alpha;
    }
#pragma unroll
    for (int half = 0; half < 2; ++half)
#pragma unroll
      for (int i = 0; i < 4; ++i) {
        x[half][i] = __builtin_amdgcn_exp2f(fmaf(x[half][i], c2, -ref));
        l += x[half][i];
        if (sizeof(T) == 2 && i % 2) {
          const bf16x2 pair = {(__bf16)x[half][i - 1], (__bf16)x[half][i]};
          w[2 * half + i / 2] = __builtin_bit_cast(uint32_t, pair);
        }
      }
  }
  __device__ __forceinline__ void values(uint32_t buf, const float (&scale)[H]) {
    if constexpr (sizeof(T) == 4) {
#pragma unroll
      for (int half = 0; half < 2; ++half)
#pragma unroll
        for (int i = 0; i < 4; ++i) {
          const int row = 16 * half + 4 * g + i;
          const uint32_t from = buf + uint32_t(row * PT::RB), sw = uint32_t(PT::template swizzle<true>(row));
#pragma unroll
          for (int c = 0; c < D / 16; ++c) {
            const float v = *reinterpret_cast<LDS_PTR(const float)>(from + ((uint32_t(4 * c + n / 4)) ^ sw) * 16 + uint32_t(n % 4) * 4);
            acc[c] = __builtin_amdgcn_mfma_f32_16x16x4f32(v, x[half][i], acc[c], 0, 0, 0);
          }
        }
    } else if constexpr (E4M3) {
      const int i = (lane & 15) >> 1, row = 4 * g + i + (i < 4 ? 0 : 12);                    // keys 4 g .. 4 g + 3 of both halves
      i32x2 raw[D / 16];
#pragma unroll
      for (int c = 0; c < D / 16; ++c)
        raw[c] = __builtin_amdgcn_ds_read_tr8_b64_v2i32(
            reinterpret_cast<LDS_PTR(i32x2)>(buf + uint32_t(row * PT::RB) + uint32_t(c ^ PT::template swizzle<true>(row)) * 16 + (lane & 1) * 8));
#pragma unroll
      for (int c = 0; c < D / 16; ++c) {
        const bf16x8 v = eight(uint32_t(raw[c][0]), uint32_t(raw[c][1]), scale[0], scale[H - 1]);
        acc[c] = __builtin_amdgcn_mfma_f32_16x16x32_bf16(v, __builtin_bit_cast(bf16x8, w), acc[c], 0, 0, 0);
      }
    } else {
      const int row = 4 * g + ((lane & 15) >> 2), byte = (lane & 1) * 8;
#pragma unroll
      for (int c = 0; c < D / 16; ++c) {
        const int chunk = 2 * c + ((lane & 3) >> 1);
        const s16x4 lo = __builtin_amdgcn_ds_read_tr16_b64_v4i16(reinterpret_cast<LDS_PTR(s16x4)>(buf + uint32_t(row * PT::RB + (chunk ^ PT::template swizzle<true>(row)) * 16 + byte)));
        const s16x4 hi = __builtin_amdgcn_ds_read_tr16_b64_v4i16(
            reinterpret_cast<LDS_PTR(s16x4)>(buf + uint32_t((row + 16) * PT::RB + (chunk ^ PT::template swizzle<true>(row + 16)) * 16 + byte)));
        acc[c] = __builtin_amdgcn_mfma_f32_16x16x32_bf16(__builtin_bit_cast(bf16x8, __builtin_shufflevector(lo, hi, 0, 1, 2, 3, 4, 5, 6, 7)), __builtin_bit_cast(bf16x8, w), acc[c], 0, 0, 0);
      }
    }
  }
  __device__ __forceinline__ void finish() { l = across(l, true); }
  __device__ __forceinline__ float sum(int reg) const { return acc[reg / 4][reg % 4]; }
  __device__ __forceinline__ int channel(int reg) const { return reg / 4 * 16 + 4 * g; }
  __device__ __forceinline__ bool first() const { return g == 0; }
};

template <int ROWS, typename T, int D, bool E4M3, int H> struct WaveOf { using type = Wave32<T, D, E4M3, H>; };
template <typename T, int D, bool E4M3, int H> struct WaveOf<16, T, D, E4M3, H> { using type = Wave16<T, D, E4M3, H>; };

// Bound by memory and by what stands around it: 48 sequences of up to 16 384 keys, 8 key heads, d = 128, e4m3: 209 to 214 us of 218, 5.7 TB/s (as fast without the arithmetic; bare loads of
// this shape: 6.9); one sequence of 80 900 keys: 31 of 42, 5.4 TB/s.  The rest is the join and the way from one launch to the next.  16 sequences that see 1 024 keys each of
// bf16 pages of 16 rows, d = 64: 10.3 us, a chain of trips to memory (lengths, table, keys, values) and the waves' join.  Matrix cores busy 7 % of the cycles at most.
template <int ROWS, typename T, int D, bool E4M3, bool SMALL>
__global__ void __launch_bounds__((64 * paged_waves<T, D, E4M3>()), 1) paged_split_kernel(PagedArgs a) {
  constexpr int NW = paged_waves<T, D, E4M3>(), NT = 64 * NW, H = SMALL ? 2 : 1, RPH = 32 / H;        // H: pages of a piece
  using Wave = typename WaveOf<ROWS, T, D, E4M3, H>::type;
  using PT = typename Wave::PT;
  constexpr int LOADS = PT::LOADS, BYTES = PT::BYTES, REGS = Wave::REGS;
  static_assert(REGS * 64 * 4 <= 4 * BYTES, "a wave's sums fit where its tiles were");
  __shared__ __attribute__((aligned(1024))) char tiles[NW * 4 * BYTES];
  __shared__ float s_m[NW][ROWS], s_l[NW][ROWS];
  __shared__ int s_sums[NW], s_first[5];
  const int lane = threadIdx.x & 63, wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
  Wave wv(lane);
  const int n = wv.n;
  const uint32_t lds = uint32_t(reinterpret_cast<uintptr_t>((LDS_PTR(void))(tiles))) + uint32_t(wave * 4 * BYTES);

  const Deal<NT> deal(a, s_sums);
  int at = blockIdx.x * deal.per;
  const int end = min_of(deal.total, at + deal.per), start = at;
  if (at >= end) return;
  int s = a.packed, off = 0;                         // nobody's: where starts fall so far that the units of all pass 31 bits
  PagedSeq seq;
  const bool holds = deal.before <= at && at < deal.before + deal.mine;
  if (a.packed <= 64) {
    const uint64_t who = __builtin_amdgcn_ballot_w64(holds);
    if (who) {
      s = __builtin_ctzll(who);
      off = at - __builtin_amdgcn_readlane(deal.before, s);
      const int q0 = __builtin_amdgcn_readlane(deal.last.q0, s);
      seq = PagedSeq(a, q0, q0 + __builtin_amdgcn_readlane(deal.last.n, s), __builtin_amdgcn_readlane(deal.last.k, s));
    }
  } else {
    if (threadIdx.x == 0) s_first[0] = a.packed;
    __syncthreads();
    if (holds) {
      int i = threadIdx.x * deal.each, rest = at - deal.before;
      PagedSeq x = deal.last;
      if (deal.each > 1)
        for (; i < a.packed; ++i) {
          x = PagedSeq(a, i);
          const int w = x.work(a);
          if (rest < w) break;
          rest -= w;
        }
      s_first[0] = i;
      s_first[1] = rest;
      s_first[2] = x.q0;
      s_first[3] = x.n;
      s_first[4] = x.k;
    }
    __syncthreads();
    auto first = [&](int i) { return __builtin_amdgcn_readfirstlane(s_first[i]); };
    s = first(0);
    off = first(1);
    // (where starts fall so far that the units of all pass 31 bits, several threads may have written these: no row outside the tensors comes of it)
    seq = PagedSeq(a, first(2), first(2) + min_of(first(3), a.n_q - first(2)), first(4));
  }
  if (s >= a.packed) return;

  uint32_t k_off[LOADS], v_off[LOADS];
#pragma unroll
  for (int j = 0; j < LOADS; ++j) {
    k_off[j] = PT::template offset<false>(j, lane, a.pages.k.row);
    v_off[j] = PT::template offset<true>(j, lane, a.pages.v.row);
  }
  const float c2 = a.scale * LOG2E;
  while (at < end) {
    if (off >= seq.work(a)) {
      if (++s >= a.packed) return;
      off = 0;
      seq = PagedSeq(a, s);
      continue;
    }
    const int item = off / seq.units, u0 = off - item * seq.units, u1 = min_of(seq.units, u0 + end - at), blk = item / a.heads_kv, kvh = item - blk * a.heads_kv;
    const int r0 = blk * ROWS, rows = min_of(seq.n * a.group - r0, ROWS), shift = seq.k - seq.n;
    const int i0 = query_of(a, r0), i1 = query_of(a, r0 + rows - 1);
    const Span span(a, i0 + shift, i1 + shift, seq.k, 32);
    const int t_end = min_of(span.n, u1 * a.unit), lo = max_of(0, i0 + shift - a.left);        // lo: first key of the window
    const bool real = n < rows;
    const int qi = real ? query_of(a, r0 + n) : i0, qh = kvh * a.group + (real ? r0 + n - qi * a.group : 0), p = qi + shift;

    Entries<E4M3> entries(a, s);
    // Where a piece lies: on one page, or with pages of 16 rows on two.
    uint64_t k_at[H], v_at[H];
    int there[H], key = 0;
    float k_scale[2][H], v_scale[2][H];              // of the two pieces that are on their way
    auto locate = [&](int t, int parity) __attribute__((always_inline)) {
      key = span.begin(t);
      const int last = t < t_end ? span.end(t) : 0;
#pragma unroll
      for (int half = 0; half < H; ++half) {
        const int k0 = key + RPH * half, in = k0 & ((1 << a.pages.bits) - 1);
        there[half] = min_of(last - k0, RPH);
        const int l = there[half] > 0 ? entries.lane_of(a, k0 >> a.pages.bits, kvh) : 0;
        k_at[half] = entries.of(entries.k, l) + uint32_t(in) * uint32_t(a.pages.k.row);
        v_at[half] = entries.of(entries.v, l) + uint32_t(in) * uint32_t(a.pages.v.row);
        if constexpr (E4M3) {
          k_scale[parity][half] = entries.of(entries.ks, l);
          v_scale[parity][half] = entries.of(entries.vs, l);
        }
      }
    };
    // Asks for the keys or values of the piece that was located.  Behind the last piece nothing is asked for, by as many loads, so that the waits count the same.
    auto ask = [&](const uint64_t (&from)[H], int64_t stride, const uint32_t (&offs)[LOADS], int parity, bool values) __attribute__((always_inline)) {
      const bool front = values && key >= span.first && key < lo;         // values that no row sees must not be read: they may be anything, and their scale
#pragma unroll
      for (int half = 0; half < H; ++half) {
        const uint32_t bytes = there[half] > 0 ? uint32_t(there[half] - 1) * uint32_t(stride) + PT::RB : 0;
        const u32x4 desc = {uint32_t(from[half]), uint32_t(from[half] >> 32) & 0xFFFFu, bytes, 0x00020000u};
        const uint32_t to = __builtin_amdgcn_readfirstlane(lds + uint32_t((parity * 2 + values) * BYTES + half * (BYTES / 2)));
#pragma unroll
        for (int j = 0; j < LOADS / H; ++j) {
          uint32_t o = offs[j];
          if (front) {
            const int k = key + RPH * half + (j * 64 + lane) / PT::CH;
            if (k < lo && k >= a.sinks) o = 0x80000000u;
          }
          asm volatile("s_add_u32 m0, %0, %3\n\ts_nop 0\n\tbuffer_load_dwordx4 %1, %2, 0 offen lds" ::"s"(to), "v"(o), "s"(desc), "i"(j * 1024) : "memory", "m0", "scc");
        }
        if constexpr (E4M3)
          if (values && (there[half] <= 0 || (front && key + RPH * half + RPH - 1 < lo && key + RPH * half >= a.sinks))) v_scale[parity][half] = 1.f;
      }
    };
    auto ask_keys = [&](int t, int parity) __attribute__((always_inline)) {
      locate(t, parity);
      ask(k_at, a.pages.k.row, k_off, parity, false);
    };
    auto ask_values = [&](int parity) __attribute__((always_inline)) { ask(v_at, a.pages.v.row, v_off, parity, true); };
    int t = u0 * a.unit + wave;
    wv.start(a.q.at(0, qh, seq.q0 + qi));
    if (t < t_end) {
      ask_keys(t, 0);
      ask_values(0);
      ask_keys(t + NW, 1);
      ask_values(1);
    }
    // The queries are waited for here, with what was asked for behind them, or the compiler does it in every piece and for all loads.
    wv.wait_queries();
    auto piece = [&](auto parity_) __attribute__((always_inline)) {
      constexpr int parity = decltype(parity_)::value;
      const uint32_t buf = lds + uint32_t(parity * 2 * BYTES);
      float v_now[H];                                // the next piece's comes where it was
#pragma unroll
      for (int i = 0; i < H; ++i) v_now[i] = v_scale[parity][i];
      wait_loads_but<3 * LOADS>();
      wv.keys(buf, k_scale[parity]);
      wait_reads();
      ask_keys(t + 2 * NW, parity);
      wv.weigh(a, span, t, p, c2);
      wait_loads_but<3 * LOADS>();
      wv.values(buf + BYTES, v_now);
      wait_reads();
      ask_values(parity);
    };
    for (; t < t_end; t += NW) {
      piece(std::integral_constant<int, 0>{});
      t += NW;
      if (t >= t_end) break;
      piece(std::integral_constant<int, 1>{});
    }
    wait_loads();                                    // the last ones, of nothing, still write zeros where the sums go
    wv.finish();
    // The waves' sums meet where the tiles were; each wave joins a share of the channels.
    float* all = reinterpret_cast<float*>(tiles);
    __syncthreads();
#pragma unroll
    for (int i = 0; i < REGS; ++i) all[(wave * REGS + i) * 64 + lane] = wv.sum(i);
    if (wv.first()) {
      s_m[wave][n] = wv.m;
      s_l[wave][n] = wv.l;
    }
    __syncthreads();
    float top = s_m[0][n], total = 0.f, share_[NW];
#pragma unroll
    for (int w = 1; w < NW; ++w) top = fmaxf(top, s_m[w][n]);
    const float ref = top == -INFINITY ? 0.f : top;
#pragma unroll
    for (int w = 0; w < NW; ++w) {
      share_[w] = __builtin_amdgcn_exp2f(s_m[w][n] - ref);
      total += share_[w] * s_l[w][n];
    }
    const bool whole = u0 == 0 && u1 == seq.units;
    const float f = !whole ? 1.f : total == 0.f ? 0.f : 1.f / total;
    const int64_t slot = (int64_t(blockIdx.x) * 2 + (at != start)) * ROWS + n;                 // a run has two ends: parts of two items at most
    if (real) {
      char* out = whole ? a.o.at(0, qh, seq.q0 + qi) : reinterpret_cast<char*>(a.part + slot * D);
#pragma unroll
      for (int i = 0; i < (REGS / 4 + NW - 1) / NW; ++i) {
        const int reg = 4 * (i * NW + wave), ch = wv.channel(reg);
        if (reg >= REGS) break;
        float x[4] = {};
#pragma unroll
        for (int w = 0; w < NW; ++w)
#pragma unroll
          for (int j = 0; j < 4; ++j) x[j] = fmaf(share_[w], all[(w * REGS + reg + j) * 64 + lane], x[j]);
        if (whole) store_four<T>(out, ch, x, f);
        else store_four<float>(out, ch, x, f);
      }
      if (wave == 0 && wv.first()) {
        if (!whole) a.part_sums[slot] = make_float2(top, total);
        else if (a.lse) a.lse[int64_t(qh) * a.n_q + seq.q0 + qi] = total == 0.f ? -INFINITY : (top + __builtin_amdgcn_logf(total)) * (1.f / LOG2E);
      }
    }
    at += u1 - u0;
    off += u1 - u0;
    __syncthreads();                                 // the sums have been read: the next item's tiles may come
  }
}

// Joins the parts of an item: four rows a work-group, a thread takes four channels of a row and every so-manieth part; items in the order of blocks of rows, as packed
// sequences have them, and key heads.  Bound by a chain of trips to memory:
// lengths, the parts, the row: 5 to 6 us.
template <typename T, int D>
__global__ void __launch_bounds__(256) paged_join_kernel(PagedArgs a, int row_groups) {
  constexpr int TR = D / 4, RB = 4, SETS = 256 / TR / RB, U = 8;         // threads of a row, rows, sets of parts, parts that a thread asks for at once
  __shared__ int s_sums[4], s_owner, s_item[5];
  __shared__ float2 s_ml[SETS][RB];
  __shared__ float4 s_x[SETS][RB][TR];
  const int id = blockIdx.x / row_groups, in = threadIdx.x / TR % RB, set = threadIdx.x / TR / RB, ch = threadIdx.x % TR;
  const int slot = id / a.heads_kv, kvh = id - slot * a.heads_kv;
  const Deal<256> deal(a, s_sums);
  // The sequence that this block is of, and the units in front of its item.
  int base = 0, blk = 0;
  PagedSeq seq;
  if (a.packed <= 64) {
    const int lane = threadIdx.x & 63, mine = slot - int(uint32_t(deal.last.q0 * a.group) >> a.row_bits) - lane;
    const uint64_t who = __builtin_amdgcn_ballot_w64(lane < a.packed && mine >= 0 && mine < deal.last.blocks);
    if (!who) return;
    const int s = __builtin_ctzll(who), q0 = __builtin_amdgcn_readlane(deal.last.q0, s);     // (one of them where starts fall)
    seq = PagedSeq(a, q0, q0 + __builtin_amdgcn_readlane(deal.last.n, s), __builtin_amdgcn_readlane(deal.last.k, s));
    blk = __builtin_amdgcn_readlane(mine, s);
    base = __builtin_amdgcn_readlane(deal.before, s) + (blk * a.heads_kv + kvh) * seq.units;
  } else {
    if (threadIdx.x == 0) s_owner = -1;
    __syncthreads();
    int s = threadIdx.x * deal.each;
    bool mine = false;
    base = deal.before;
    seq = deal.last;
    for (int i = 0; i < deal.each && s < a.packed; ++i, ++s) {
      if (deal.each > 1) seq = PagedSeq(a, s);
      blk = slot - int(uint32_t(seq.q0 * a.group) >> a.row_bits) - s;
      mine = blk >= 0 && blk < seq.blocks;
      if (mine) break;
      base += seq.work(a);
    }
    if (mine) s_owner = threadIdx.x;
    __syncthreads();
    if (s_owner < 0) return;
    if (s_owner == int(threadIdx.x)) {               // one thread's numbers, also where starts fall and several have some
      s_item[0] = seq.q0;
      s_item[1] = seq.n;
      s_item[2] = seq.k;
      s_item[3] = base + (blk * a.heads_kv + kvh) * seq.units;
      s_item[4] = blk;
    }
    __syncthreads();
    seq = PagedSeq(a, s_item[0], s_item[0] + s_item[1], s_item[2]);
    base = s_item[3];
    blk = s_item[4];
  }
  const int first = blk << a.row_bits;
  const int g0 = base / deal.per, g1 = (base + seq.units - 1) / deal.per;
  if (g0 == g1 || g0 < 0 || g1 >= GROUPS) return;    // one work-group had it whole; (past the runs: where starts fall so far that 31 bits do not count all)
  for (int n = (blockIdx.x - id * row_groups) * RB + in; first + n - in < min_of(first + (1 << a.row_bits), seq.n * a.group); n += row_groups * RB) {
    const int r = min_of(first + n, seq.n * a.group - 1), row = r - first;
    float top = -INFINITY, total = 0.f, x[4] = {};
    for (int g = g0 + set; g <= g1; g += U * SETS) {
      float2 ml[U];
      float4 y[U];
#pragma unroll
      for (int u = 0; u < U; ++u) {                    // behind the last part that once more, with a weight of zero
        const int w = min_of(g + u * SETS, g1);
        const int64_t i = ((int64_t(w) * 2 + (w == g0 && base != w * deal.per)) << a.row_bits) + row;
        ml[u] = a.part_sums[i];
        y[u] = reinterpret_cast<const float4*>(a.part + i * D)[ch];
      }
      const float before = top;
#pragma unroll
      for (int u = 0; u < U; ++u) {
        if (g + u * SETS > g1) ml[u].x = -INFINITY;
        top = fmaxf(top, ml[u].x);
      }
      const float ref = top == -INFINITY ? 0.f : top, f = __builtin_amdgcn_exp2f(before - ref);
      total *= f;
#pragma unroll
      for (int j = 0; j < 4; ++j) x[j] *= f;
#pragma unroll
      for (int u = 0; u < U; ++u) {
        const float part = __builtin_amdgcn_exp2f(ml[u].x - ref);
        total = fmaf(part, ml[u].y, total);
        x[0] = fmaf(part, y[u].x, x[0]);
        x[1] = fmaf(part, y[u].y, x[1]);
        x[2] = fmaf(part, y[u].z, x[2]);
        x[3] = fmaf(part, y[u].w, x[3]);
      }
    }
    s_x[set][in][ch] = make_float4(x[0], x[1], x[2], x[3]);
    if (ch == 0) s_ml[set][in] = make_float2(top, total);
    __syncthreads();
    if (set == 0 && first + n < seq.n * a.group) {
#pragma unroll
      for (int i = 1; i < SETS; ++i) top = fmaxf(top, s_ml[i][in].x);
      const float ref = top == -INFINITY ? 0.f : top;
      total = x[0] = x[1] = x[2] = x[3] = 0.f;
#pragma unroll
      for (int i = 0; i < SETS; ++i) {
        const float part = __builtin_amdgcn_exp2f(s_ml[i][in].x - ref);
        const float4 y = s_x[i][in][ch];
        total = fmaf(part, s_ml[i][in].y, total);
        x[0] = fmaf(part, y.x, x[0]);
        x[1] = fmaf(part, y.y, x[1]);
        x[2] = fmaf(part, y.z, x[2]);
        x[3] = fmaf(part, y.w, x[3]);
      }
      const int qi = query_of(a, r), qh = kvh * a.group + r - qi * a.group;
      store_four<T>(a.o.at(0, qh, seq.q0 + qi), ch * 4, x, total == 0.f ? 0.f : 1.f / total);
      if (ch == 0 && a.lse) a.lse[int64_t(qh) * a.n_q + seq.q0 + qi] = total == 0.f ? -INFINITY : (top + __builtin_amdgcn_logf(total)) * (1.f / LOG2E);
    }
    __syncthreads();                                   // the sets' sums have been read
  }
}

static int check_paged(const char* call, const dfs_paged* w, int dtype) {
  if (!w) return fail(DFS_EINVAL, "%s: geometry pointer is NULL", call);
  if (dtype != DFS_F32 && dtype != DFS_BF16) return fail(DFS_EDTYPE, "%s: dtype %d is not DFS_F32 or DFS_BF16", call, dtype);
  if (w->seqs < 0 || w->n_q < 0 || w->n_q > 1 << 28) return fail(DFS_ESHAPE, "%s: seqs=%d must not be negative, n_q=%d be in [0, 2^28]", call, w->seqs, w->n_q);
  if (w->heads < 1 || w->heads_kv < 1 || w->heads > 65535 || w->heads % w->heads_kv)
    return fail(DFS_ESHAPE, "%s: heads=%d must be in [1, 65535] and a multiple of heads_kv=%d", call, w->heads, w->heads_kv);
  if (w->d != 64 && w->d != 128) return fail(DFS_ESHAPE, "%s: d=%d: head dimension must be 64 or 128", call, w->d);
  if (w->sinks < 0) return fail(DFS_ESHAPE, "%s: sinks=%d is negative", call, w->sinks);
  const int64_t rows = int64_t(w->heads / w->heads_kv) * w->n_q;
  if (rows > int64_t(1) << 30 || w->seqs >= 1 << 20 || (rows / 32 + w->seqs) * w->heads_kv >= 1 << 22)
    return fail(DFS_ESHAPE, "%s: heads_kv=%d x rows of q, or seqs=%d, too large", call, w->heads_kv, w->seqs);
  return DFS_OK;
}

// The parts of GROUPS runs, two each, and their sums.
static size_t part_bytes(const dfs_paged* w) { return size_t(GROUPS) * 2 * 32 * w->d * sizeof(float); }

}  // namespace dfs

using namespace dfs;

extern "C" {

size_t dfs_paged_workspace_bytes(const dfs_paged* w, int dtype, const dfs_pages* pages) {
  const char* call = "dfs_paged_workspace_bytes";
  PageArgs p;
  if (check_paged(call, w, dtype) != DFS_OK || check_pages(call, pages, dtype, w->seqs, w->heads_kv, w->d, false, &p) != DFS_OK) return 0;
  if (w->seqs == 0 || w->n_q == 0 || paged_is_long(w, dtype)) return 0;
  return part_bytes(w) + size_t(GROUPS) * 2 * 32 * sizeof(float2);
}

int dfs_paged_attn_fwd(const dfs_paged* w, int dtype, const dfs_view* q, const dfs_pages* pages, const int32_t* q_start, const int32_t* k_len, float scale,
                       const dfs_view* o, float* lse, void* ws, size_t ws_bytes, void* stream) {
  const char* call = "dfs_paged_attn_fwd";
  PagedArgs a = {};
  int rc = check_paged(call, w, dtype);
  if (rc) return rc;
  if (!(scale > 0.f) || !isfinite(scale)) return fail(DFS_EINVAL, "%s: scale must be positive and finite", call);
  if (misaligned(4, {lse, q_start, k_len})) return fail(DFS_EINVAL, "%s: lse, starts and lengths must be 4-byte aligned", call);
  if (w->seqs && (!q_start || !k_len)) return fail(DFS_EINVAL, "%s: q_start or k_len is NULL", call);
  if ((rc = check_view(call, "q", q, dtype, 1, w->heads, w->n_q, w->d, false, &a.q))) return rc;
  if ((rc = check_view(call, "o", o, dtype, 1, w->heads, w->n_q, w->d, true, &a.o))) return rc;
  if ((rc = check_pages(call, pages, dtype, w->seqs, w->heads_kv, w->d, false, &a.pages))) return rc;
  if (w->seqs == 0 || w->n_q == 0) return DFS_OK;
  const size_t need = paged_is_long(w, dtype) ? 0 : part_bytes(w) + size_t(GROUPS) * 2 * 32 * sizeof(float2);
  if (need && (!ws || (uintptr_t(ws) & 255) || ws_bytes < need))
    return fail(DFS_EWORKSPACE, "%s: workspace of %zu bytes needed (256-byte aligned), got %zu", call, need, ws_bytes);
  if ((rc = check_apart(call, {{"o", &a.o}}, {{"q", &a.q}, {"pages.k", &a.pages.k}, {"pages.v", &a.pages.v}}))) return rc;
  a.lse = lse;
  a.q_start = q_start;
  a.k_len = k_len;
  a.packed = w->seqs;
  a.batch = 1;
  a.heads = w->heads;
  a.heads_kv = w->heads_kv;
  a.group = w->heads / w->heads_kv;
  a.seqs = w->heads_kv;
  a.by_kv = Div(uint32_t(w->heads_kv));
  a.by_group = Div(uint32_t(a.group));
  a.n_q = w->n_q;
  a.n_k = a.pages.row << a.pages.bits;
  a.left = w->left < 0 || w->left > NO_LIMIT ? NO_LIMIT : w->left;
  a.right = 0;
  a.sinks = a.left == NO_LIMIT ? 0 : w->sinks < a.n_k ? w->sinks : a.n_k;
  a.scale = scale;
  a.part = static_cast<float*>(ws);
  a.part_sums = reinterpret_cast<float2*>(static_cast<char*>(ws) + part_bytes(w));
  // 16 rows where the sequences have no more on average: half of the matrix instructions and of the weights (one token over 80 900 keys, 4 heads a key head, 45 -> 43 us, 16 streams
  // with a window of 1 024 keys 11.5 -> 10.5; fp32, d = 128, 48 streams x 8 key heads over up to 4 000 keys 457 -> 296, 8 x 8 over up to 207 31.6 -> 21.6)
  const int64_t mean = (int64_t(a.group) * a.n_q + w->seqs - 1) / w->seqs;
  a.row_bits = mean <= 16 ? 4 : 5;
  const int64_t items = ((int64_t(a.group) * a.n_q >> a.row_bits) + w->seqs) * w->heads_kv, pieces = a.n_k / 32 + 2;
  const bool bytes = pages->dtype == DFS_E4M3;
  const int row_bytes = w->d * (bytes ? 1 : elem_size(dtype));
  a.unit = 1024 / row_bytes < 8 ? 1024 / row_bytes : 8;                  // a piece for each wave
  while (items * ((pieces + a.unit - 1) / a.unit) >= int64_t(1) << 30) a.unit *= 2;          // units are counted in 31 bits, and the last work-group's run may end behind them
  // Where no row sees many pieces an item is one unit: no parts, no second launch (us, whole against parts; one token of two streams x 2 key heads, d = 128, e4m3, 8 waves:
  // 1 024 keys 9.8 / 10.9, 2 048 12.9 / 10.8; bf16, 4 waves: 512 keys 10.0 / 10.4, 1 024 13.0 / 10.5; of 16 streams x 8, which fill the chip by themselves: e4m3
  // 2 048 keys 16.8 / 20.9, bf16 23.9 / 25.4.  fp32, where the matrix instructions of a piece take 2 us: 8 streams x 8, d = 128, 2 waves: 64 keys 10.1 / 12.1, 130 14.4 / 13.6;
  // d = 64, 4 waves: 250 keys 9.5 / 11.1, 500 13.1 / 11.4, 16 x 8 1 000 keys 22.1 / 22.2, 2 000 36.2 / 28.8).
  const int64_t reach = a.left == NO_LIMIT ? pieces : (int64_t(a.left) + a.n_q) / 32 + 2 + (a.sinks + 31) / 32, longest = reach < pieces ? reach : pieces;
  const bool fills = int64_t(w->seqs) * w->heads_kv >= 128;
  const bool whole = longest <= (dtype == DFS_F32 ? (fills && w->d == 64 ? 8 : 3) * a.unit : fills ? 72 : 5 * a.unit + 1);
  if (whole) a.unit = int(longest);
  const hipStream_t st = as_stream(stream);
  // work-groups of an item's join, four rows a turn, by the rows that a sequence has on average
  const int row_groups = mean < 1 << a.row_bits ? int(mean + 3) / 4 : 1 << a.row_bits >> 2;
  const unsigned joins = unsigned(items * row_groups);
  auto run = [&](auto t, auto d, auto b) {
    using T = decltype(t);
    constexpr int D = decltype(d)::value;
    constexpr bool E4M3 = decltype(b)::value;
    constexpr int NT = 64 * paged_waves<T, D, E4M3>();
    auto of = [&](auto rows) {
      if (a.pages.bits == 4) paged_split_kernel<decltype(rows)::value, T, D, E4M3, true><<<GROUPS, NT, 0, st>>>(a);
      else paged_split_kernel<decltype(rows)::value, T, D, E4M3, false><<<GROUPS, NT, 0, st>>>(a);
    };
    if (a.row_bits == 4) return of(std::integral_constant<int, 16>{});
    of(std::integral_constant<int, 32>{});
  };
  auto join = [&](auto t, auto d) { paged_join_kernel<decltype(t), decltype(d)::value><<<joins, 256, 0, st>>>(a, row_groups); };
  auto by_dim = [&](auto f) { w->d == 64 ? f(std::integral_constant<int, 64>{}) : f(std::integral_constant<int, 128>{}); };
  if (paged_is_long(w, dtype)) return run_paged_long(a, w->d, dtype, bytes, st);
  by_dim([&](auto d) {
    if (dtype == DFS_F32) run(float{}, d, std::false_type{});
    else if (bytes) run(uint16_t{}, d, std::true_type{});
    else run(uint16_t{}, d, std::false_type{});
  });
  if ((rc = launch_status(call)) || whole) return rc;
  by_dim([&](auto d) { dtype == DFS_F32 ? join(float{}, d) : join(uint16_t{}, d); });
  return launch_status(call);
}

}  // extern "C"
