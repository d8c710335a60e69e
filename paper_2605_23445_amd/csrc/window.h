// What the kernels of windowed attention share: their arguments, the tiles of rows in LDS and the operands of the matrix cores.
//
// All kernels work on tiles of rows of d channels.  A tile is loaded from global memory straight into LDS; rows behind its last real one are
// zeros.  An operand "by rows" (rows of the tile are rows of the matrix, contracted over channels) is a 16-byte chunk per lane; an operand "by columns"
// (channels are rows of the matrix, contracted over the tile's rows) comes through the transposing LDS read in bf16 and element by element in fp32.
// With 32x32 products a lane holds, of the result, column lane % 32 and rows 8 (i / 4) + 4 (lane / 32) + i % 4 in register i: as B operand of a product
// contracted over those rows the registers serve as they are.
#pragma once
#include "view.h"

namespace dfs {

typedef unsigned int u32x4 __attribute__((ext_vector_type(4)));
typedef float f32x4 __attribute__((ext_vector_type(4)));
typedef float f32x16 __attribute__((ext_vector_type(16)));
typedef __bf16 bf16x8 __attribute__((ext_vector_type(8)));
typedef __bf16 bf16x2 __attribute__((ext_vector_type(2)));
typedef short s16x4 __attribute__((ext_vector_type(4)));
#define LDS_PTR(T) __attribute__((address_space(3))) T*

constexpr int NO_LIMIT = 1 << 29;                    // of left and right: further than any two positions are apart
constexpr float LOG2E = 1.4426950408889634f;

// Division of x < 2^31 by a number that the host knows: a work-group makes half a dozen before it can ask for anything, and the compiler's take 40
// instructions each.  With l the bits of d - 1 and m = floor(2^(31 + l) / d) + 1, (x m) >> (31 + l) is x / d.
struct Div {
  uint32_t m = 0, l = 0;
  Div() = default;
  explicit Div(uint32_t d) {
    while ((uint64_t(1) << l) < d) ++l;
    m = uint32_t((uint64_t(1) << (31 + l)) / d + 1);
  }
  __device__ __forceinline__ int operator()(int x) const { return int(__umulhi(uint32_t(x) * 2, m) >> l); }
};

struct WindowArgs {
  View q, k, v, o, d_o, dq, dk, dv;
  float* lse;                                        // [batch, heads, n_q]
  float2* sums;                                      // backward, alike: a row's log-sum-exp in base 2 and <do, o>
  float* part;                                       // sums of a part: of the first keys' gradients, or of a row's output
  float *key_part, *row_part;                        // backward: sums of a split's part of 32 keys' gradients, of 32 rows'
  float2* part_sums;                                 // maximum and sum of a row's part
  const int32_t *q_len, *k_len;
  int32_t batch, heads, heads_kv, group, n_q, n_k, left, right, sinks;
  int32_t blocks, seqs;                              // work-groups of a sequence's key head; key heads of all sequences
  Div by_blocks, by_kv, by_group, by_splits;         // by_splits: by the work-groups that share a block
  int32_t first_tiles, first_splits;                 // backward: tiles of 32 first keys, and work-groups that share one's queries
  int32_t key_splits, row_splits;                    // backward: work-groups that share a block of keys, a block of rows
  int32_t splits;                                    // forward: work-groups that share the keys of 32 rows
  float scale;
  void set_blocks(int64_t n) {
    blocks = int32_t(n);
    by_blocks = Div(uint32_t(n));
  }
};

// A sequence's lengths, and the position of its first query.
struct Lengths {
  int q, k, shift;
  __device__ __forceinline__ Lengths(const WindowArgs& a, int b) {
    q = a.q_len ? a.q_len[b] : a.n_q;
    k = a.k_len ? a.k_len[b] : a.n_k;
    q = q < 0 ? 0 : q > a.n_q ? a.n_q : q;
    k = k < 0 ? 0 : k > a.n_k ? a.n_k : k;
    shift = k - q;
  }
};

__device__ __forceinline__ int min_of(int a, int b) { return a < b ? a : b; }
__device__ __forceinline__ int max_of(int a, int b) { return a > b ? a : b; }

// Puts `none` where register i of a lane's 32 x 32 result stands for a row outside [lo, hi] (and at or behind `more`) of those from 4 (lane / 32) on.  By
// selects and whole conditions: written with && and an assignment under `if`, the compiler (ROCm 7.2) made branches of it and lost the assignment to
// the first register of an accumulator in one of them.
__device__ __forceinline__ void keep(f32x16& x, int lo, int hi, float none) {
#pragma unroll
  for (int i = 0; i < 16; ++i) x[i] = ((8 * (i / 4) + i % 4 >= lo) & (8 * (i / 4) + i % 4 <= hi)) ? x[i] : none;
}
__device__ __forceinline__ void keep(f32x16& x, int lo, int hi, int more, float none) {
#pragma unroll
  for (int i = 0; i < 16; ++i)
    x[i] = ((8 * (i / 4) + i % 4 <= hi) & ((8 * (i / 4) + i % 4 >= lo) | (8 * (i / 4) + i % 4 < more))) ? x[i] : none;
}

// The keys that a run of queries needs, in pieces of 32: the first keys that lie in front of the run's window, then the window from its first key on.
struct Span {
  int p0, p1, lo, hi, first, n_first, n;             // positions; window [lo, hi); first keys [0, first) in front of it; pieces of these, and of all
  int first_whole, w0, w1;                           // pieces that every query sees whole: of first keys those in front of first_whole, [w0, w1)
  __device__ __forceinline__ Span(const WindowArgs& a, int p0_, int p1_, int k_len) : p0(p0_), p1(p1_) {
    lo = max_of(0, p0 - a.left);
    hi = min_of(k_len, p1 + a.right + 1);
    if (hi < 0) hi = 0;
    first = min_of(min_of(a.sinks, lo), hi);
    if (lo > hi) lo = hi;
    n_first = (first + 31) / 32;
    n = n_first + (hi - lo + 31) / 32;
    const int ahead = p0 + a.right + 1;              // keys in front of it are not too far ahead of any
    first_whole = max_of(0, min_of(first, ahead)) / 32;
    w0 = n_first + max_of(0, p1 - a.left - lo + 31) / 32;
    w1 = n_first + max_of(0, min_of(hi, ahead) - lo) / 32;
  }
  __device__ __forceinline__ int begin(int i) const { return i < n_first ? i * 32 : lo + (i - n_first) * 32; }
  __device__ __forceinline__ int end(int i) const { return i < n_first ? first : hi; }
  // Whether every query of the run sees all 32 keys of piece i.
  __device__ __forceinline__ bool whole(int i) const { return (i >= w0 && i < w1) || i < first_whole; }
  // Whether queries at positions q0 .. q1 see none of piece i's keys.
  __device__ __forceinline__ bool unseen(const WindowArgs& a, int i, int q0, int q1) const {
    const int key = begin(i);
    return key >= end(i) || key > q1 + a.right || (i >= n_first && key >= a.sinks && key + 31 < q0 - a.left);
  }
  // Puts `none` where the query at position p of this lane (half h of the wave) does not see a key of piece i; x holds keys as rows.
  __device__ __forceinline__ void mask(const WindowArgs& a, int i, int p, int h, f32x16& x, float none) const {
    const int key = begin(i) + 4 * h, top = min_of(end(i) - 1, p + a.right) - key;
    if (i >= n_first && key < a.sinks) keep(x, p - a.left - key, top, a.sinks - key, none);          // the window reaches back to first keys
    else keep(x, i < n_first ? 0 : p - a.left - key, top, none);
  }
};

// Which sequence's key head and which of its `blocks` work-groups a work-group is.  Consecutive work-groups go to the eight XCDs in turn: each XCD takes
// key heads of its own, whole ones, so that those who read the same rows share an L2; with a multiple of eight the XCDs take them in turn, so that sequences
// of different lengths spread over all.
struct Place {
  int blk, bh, b, kvh;
  __device__ __forceinline__ Place(const WindowArgs& a, int id) {
    const int xcd = id % 8, slot = id / 8;
    if (a.seqs % 8 == 0) {
      const int round = a.by_blocks(slot);
      blk = slot - round * a.blocks;
      bh = round * 8 + xcd;
    } else {
      const int n = a.seqs * a.blocks, per = n / 8, more = n % 8, at = xcd * per + (xcd < more ? xcd : more) + slot;
      bh = a.by_blocks(at);
      blk = at - bh * a.blocks;
    }
    b = a.by_kv(bh);
    kvh = bh - b * a.heads_kv;
  }
};

// Query of row r of a sequence's key head.  Rows are counted in 31 bits.
__device__ __forceinline__ int query_of(const WindowArgs& a, int r) { return a.by_group(r); }
// Rows of a block of `most` from r0 on that are there.
__device__ __forceinline__ int rows_of(const WindowArgs& a, const Lengths& len, int r0, int most) { return min_of(len.q * a.group - r0, most); }

// What a lane of a block of rows knows of its row.
struct Row {
  int n, h, i0, i1, qi, qh, p;                       // column and half of the wave; first and last query of the block; query, head, position
  bool real;
  __device__ __forceinline__ Row(const WindowArgs& a, const Place& at, const Lengths& len, int r0, int rows, int mine, int lane) {
    n = lane & 31;
    h = lane >> 5;
    i0 = query_of(a, r0);
    i1 = query_of(a, r0 + rows - 1);
    real = mine < rows;
    qi = real ? query_of(a, r0 + mine) : i0;
    qh = at.kvh * a.group + (real ? r0 + mine - qi * a.group : 0);
    p = qi + len.shift;
  }
};

template <typename T> struct Mat;
template <> struct Mat<uint16_t> {
  typedef bf16x8 Frag;
  // 16 bytes of every row: 16 channels in all
  static __device__ __forceinline__ f32x16 mma(Frag a, Frag b, f32x16 c) { return __builtin_amdgcn_mfma_f32_32x32x16_bf16(a, b, c, 0, 0, 0); }
};
template <> struct Mat<float> {
  typedef f32x4 Frag;
  // 8 channels in all
  static __device__ __forceinline__ f32x16 mma(Frag a, Frag b, f32x16 c) {
#pragma unroll
    for (int i = 0; i < 4; ++i) c = __builtin_amdgcn_mfma_f32_32x32x2f32(a[i], b[i], c, 0, 0, 0);
    return c;
  }
};

// A result of 32 x 32 as B operand of a product contracted over its rows; in bf16 rounded to one term, which the kernels' comments weigh.
template <typename T> struct Weights;
template <> struct Weights<uint16_t> {
  u32x4 p[2];
  __device__ __forceinline__ void set(const f32x16& x) {
#pragma unroll
    for (int i = 0; i < 16; i += 2) {
      const bf16x2 b = {(__bf16)x[i], (__bf16)x[i + 1]};
      p[i / 8][(i % 8) / 2] = __builtin_bit_cast(uint32_t, b);
    }
  }
};
template <> struct Weights<float> {
  f32x16 p;
  __device__ __forceinline__ void set(const f32x16& x) { p = x; }
};

// Tiles of ROWS rows of D elements, loaded by NW waves.  COLUMNS: the swizzle that suits reads by columns alone.
template <typename T, int D, int ROWS, int NW, bool COLUMNS>
struct Tile {
  static constexpr int RB = D * int(sizeof(T)), CH = RB / 16, BYTES = ROWS * RB, STEPS = CH / 2;   // STEPS: products of a contraction over channels
  static constexpr int LOADS = ROWS * CH / (64 * NW);
  static constexpr int FOLD = CH < 16 ? 16 / CH : 1;
  static_assert(ROWS * CH % (64 * NW) == 0, "a load fills 64 chunks");
  // XOR of the 16-byte chunks of a row, so that what a wave reads at once lies in different banks: one chunk of 16 rows or, by columns, four chunks of 4
  // rows.  A bf16 tile's does for both (with row % 16, which is good for rows alone, a fifth of the gradients' cycles at d = 128 were conflicts), and rows 8
  // further on differ in one bit of those that channels 32 further on count by, so that both take the same addresses.  An fp32 one's is for rows or,
  // COLUMNS, for columns, where it is known when compiled.
  static constexpr __host__ __device__ __forceinline__ int swizzle(int row) {
    if (sizeof(T) == 4) return COLUMNS ? 4 * (row % 4) : row % 16;
    const int near = row / FOLD & 1, far = row >> 3 & 1;
    return (CH == 16 ? (row >> 1 & 1) * 8 : 0) + (near ^ far) * 4 + near * 2 + (row >> 2 & 1);
  }
  // Loads: byte offset of this lane's chunk of load j in a tensor whose rows are `stride` bytes apart.
  struct Loader {
    uint32_t off[LOADS];
    __device__ __forceinline__ Loader(int64_t stride, int wave, int lane) {
#pragma unroll
      for (int j = 0; j < LOADS; ++j) {
        const int p = (j * NW + wave) * 64 + lane, row = p / CH, pc = p % CH;
        off[j] = uint32_t(row) * uint32_t(stride) + uint32_t((pc ^ swizzle(row)) * 16);
      }
    }
    // `rows` real rows from `src` on, as a descriptor that gives zeros behind them.
    static __device__ __forceinline__ u32x4 source(const char* src, int rows, int64_t stride) {
      const uint64_t at = reinterpret_cast<uint64_t>(src);
      const uint32_t bytes = rows > 0 ? uint32_t((rows < ROWS ? rows : ROWS) - 1) * uint32_t(stride) + RB : 0;
      return u32x4{uint32_t(__builtin_amdgcn_readfirstlane(uint32_t(at))), uint32_t(__builtin_amdgcn_readfirstlane(uint32_t(at >> 32))) & 0xFFFFu,
                   uint32_t(__builtin_amdgcn_readfirstlane(bytes)), 0x00020000u};
    }
    // Load j of a tile to `to`, where this wave's first chunk goes; ONCE: of rows that nothing else reads.  Asm, so that the compiler does not wait for it in
    // front of every LDS read; wait_loads() below does, in front of a barrier.
    template <bool ONCE = false> __device__ __forceinline__ void issue_one(u32x4 desc, uint32_t to, int j) const {
      if (ONCE)
        asm volatile("s_add_u32 m0, %0, %3\n\ts_nop 0\n\tbuffer_load_dwordx4 %1, %2, 0 offen nt lds"
                     ::"s"(to), "v"(off[j]), "s"(desc), "i"(j * NW * 1024) : "memory", "m0", "scc");
      else
        asm volatile("s_add_u32 m0, %0, %3\n\ts_nop 0\n\tbuffer_load_dwordx4 %1, %2, 0 offen lds"
                     ::"s"(to), "v"(off[j]), "s"(desc), "i"(j * NW * 1024) : "memory", "m0", "scc");
    }
    // Asks for a tile of two pieces of 32 rows, from src0 and src1 on.
    struct Pair { u32x4 desc[2]; };
    static __device__ __forceinline__ Pair pair(const char* src0, int rows0, const char* src1, int rows1, int64_t stride) {
      return Pair{{source(src0, rows0 < 32 ? rows0 : 32, stride), source(src1 - 32 * stride, rows1 > 0 ? (rows1 < 32 ? rows1 : 32) + 32 : 0, stride)}};
    }
    // Tile t of a span: pieces 2 t and 2 t + 1.  Most are 64 rows in one, which cost a tenth of the scalar work.
    template <class S> static __device__ __forceinline__ Pair of(const S& span, const char* base, int64_t stride, int t) {
      const int x = span.begin(2 * t);
      if (2 * t >= span.n_first && 2 * t + 2 < span.n) {
        const u32x4 all = source(base + x * stride, 64, stride);
        return Pair{{all, all}};
      }
      const int y = span.begin(2 * t + 1);
      return pair(base + x * stride, span.end(2 * t) - x, base + y * stride, span.end(2 * t + 1) - y, stride);
    }
    __device__ __forceinline__ void issue_one(const Pair& p, uint32_t to, int j) const { issue_one(p.desc[j * 2 / LOADS], to, j); }
    // Asks for the tile whose first row is at `src`; `rows` of it are real.  lds: byte address of the tile.
    template <bool ONCE = false> __device__ __forceinline__ void issue(const char* src, int rows, int64_t stride, uint32_t lds, int wave) const {
      const u32x4 desc = source(src, rows, stride);
      const uint32_t to = __builtin_amdgcn_readfirstlane(lds + uint32_t(wave) * 1024);
#pragma unroll
      for (int j = 0; j < LOADS; ++j) issue_one<ONCE>(desc, to, j);
    }
  };
  // Operand by rows: chunk 2 step + h of row 32 half + n.
  struct RowReader {
    uint32_t at, sw;
    int h;
    __device__ __forceinline__ RowReader(int lane) : at(uint32_t((lane & 31) * RB)), sw(uint32_t(swizzle(lane & 31))), h(lane >> 5) {}
    __device__ __forceinline__ typename Mat<T>::Frag get(uint32_t lds, int half, int step) const {
      return __builtin_bit_cast(typename Mat<T>::Frag,
                                *reinterpret_cast<LDS_PTR(const u32x4)>(lds + at + uint32_t(half * 32 * RB) + ((uint32_t(2 * step + h) ^ sw) * 16)));
    }
  };
  // acc[c] += (32 channels from 32 c on) x (rows of half `half`, contracted with w)
  struct ColumnReader {
    uint32_t at[D / 32][2];
    __device__ __forceinline__ ColumnReader(int lane) {
      const int h = lane >> 5;
      if constexpr (sizeof(T) == 2) {
        // the 16 lanes of a group hand in four rows of 16 channels and get four rows of one channel each
        const int row = 4 * h + ((lane & 15) >> 2), chunk = 2 * ((lane >> 4) & 1) + ((lane & 3) >> 1), byte = (lane & 1) * 8;
#pragma unroll
        for (int c = 0; c < D / 32; ++c) {
          at[c][0] = uint32_t(row * RB + ((4 * c + chunk) ^ swizzle(row)) * 16 + byte);
          at[c][1] = uint32_t((row + 8) * RB + ((4 * c + chunk) ^ swizzle(row + 8)) * 16 + byte);
        }
      } else {
        at[0][0] = uint32_t(lane & 31);
        at[0][1] = uint32_t(h);
      }
    }
    // bf16: rows 16 s .. 16 s + 15 of half `half`, channels 32 c .. 32 c + 31
    __device__ __forceinline__ bf16x8 get(uint32_t lds, int half, int s, int c) const {
      const uint32_t p = lds + uint32_t((half * 32 + s * 16) * RB);
      const s16x4 lo = __builtin_amdgcn_ds_read_tr16_b64_v4i16(reinterpret_cast<LDS_PTR(s16x4)>(p + at[c][0]));
      const s16x4 hi = __builtin_amdgcn_ds_read_tr16_b64_v4i16(reinterpret_cast<LDS_PTR(s16x4)>(p + at[c][1]));
      return __builtin_bit_cast(bf16x8, __builtin_shufflevector(lo, hi, 0, 1, 2, 3, 4, 5, 6, 7));
    }
    __device__ __forceinline__ void mma(uint32_t lds, int half, const Weights<T>& w, f32x16 (&acc)[D / 32]) const {
      if constexpr (sizeof(T) == 2) {
#pragma unroll
        for (int s = 0; s < 2; ++s)
#pragma unroll
          for (int c = 0; c < D / 32; ++c)
            acc[c] = __builtin_amdgcn_mfma_f32_32x32x16_bf16(get(lds, half, s, c), __builtin_bit_cast(bf16x8, w.p[s]), acc[c], 0, 0, 0);
      } else {
#pragma unroll
        for (int i = 0; i < 16; ++i) {
          const int row = half * 32 + 8 * (i / 4) + 4 * int(at[0][1]) + i % 4;
          const uint32_t p = lds + uint32_t(row * RB), sw = uint32_t(swizzle(row));
#pragma unroll
          for (int c = 0; c < D / 32; ++c) {
            const uint32_t ch = uint32_t(32 * c) + at[0][0];
            const float a = *reinterpret_cast<LDS_PTR(const float)>(p + ((ch / 4) ^ sw) * 16 + (ch % 4) * 4);
            acc[c] = __builtin_amdgcn_mfma_f32_32x32x2f32(a, w.p[i], acc[c], 0, 0, 0);
          }
        }
      }
    }
  };
};

__device__ __forceinline__ void wait_loads() { __builtin_amdgcn_s_waitcnt(0x0F70); }          // vmcnt(0)
// Until at most N of this wave's loads are on their way (they come in order), in front of reads of what the others brought.
template <int N> __device__ __forceinline__ void wait_loads_but() {
  __builtin_amdgcn_s_waitcnt(0x0F70 | (N & 15) | (N >> 4) << 14);
  __builtin_amdgcn_fence(__ATOMIC_ACQ_REL, "wavefront");
  __builtin_amdgcn_wave_barrier();
}
// Until this wave's LDS reads are done, in front of loads that overwrite what they read.
__device__ __forceinline__ void wait_reads() {
  __builtin_amdgcn_s_waitcnt(0xC07F);                // lgkmcnt(0)
  __builtin_amdgcn_fence(__ATOMIC_ACQ_REL, "wavefront");
  __builtin_amdgcn_wave_barrier();
}

template <int N> __device__ __forceinline__ void clear(f32x16 (&x)[N]) {
#pragma unroll
  for (int c = 0; c < N; ++c)
#pragma unroll
    for (int i = 0; i < 16; ++i) x[c][i] = 0.f;
}

// Four channels of a row from `ch` on, times f.
template <typename T> __device__ __forceinline__ void store_four(char* row, int ch, const float (&x)[4], float f) {
  if constexpr (sizeof(T) == 2) {
    const bf16x2 a = {(__bf16)(x[0] * f), (__bf16)(x[1] * f)}, b = {(__bf16)(x[2] * f), (__bf16)(x[3] * f)};
    *reinterpret_cast<uint2*>(row + ch * 2) = make_uint2(__builtin_bit_cast(uint32_t, a), __builtin_bit_cast(uint32_t, b));
  } else {
    *reinterpret_cast<float4*>(row + ch * 4) = make_float4(x[0] * f, x[1] * f, x[2] * f, x[3] * f);
  }
}

// Row `row` of accumulators by columns (column = lane % 32 of the row's 32 channels per c), times f, to a row of T: 16 bytes a lane, in bf16 after the lanes that
// hold a row's other halves have exchanged four channels of eight.
template <typename T, int N> __device__ __forceinline__ void store_row(bool real, char* row, const f32x16 (&x)[N], float f, int h) {
#pragma unroll
  for (int c = 0; c < N; ++c)
    if constexpr (sizeof(T) == 2) {
#pragma unroll
      for (int i = 0; i < 16; i += 8) {
        uint32_t p[4];
#pragma unroll
        for (int j = 0; j < 4; ++j) {
          const bf16x2 b = {(__bf16)(x[c][i + 2 * j] * f), (__bf16)(x[c][i + 2 * j + 1] * f)};
          p[j] = __builtin_bit_cast(uint32_t, b);
        }
        const auto lo = __builtin_amdgcn_permlane32_swap(p[0], p[2], false, false), hi = __builtin_amdgcn_permlane32_swap(p[1], p[3], false, false);
        if (real) *reinterpret_cast<u32x4*>(row + (32 * c + 2 * i + 8 * h) * 2) = u32x4{lo[0], hi[0], lo[1], hi[1]};
      }
    } else {
#pragma unroll
      for (int i = 0; i < 16; i += 4) {
        const float four[4] = {x[c][i], x[c][i + 1], x[c][i + 2], x[c][i + 3]};
        if (real) store_four<T>(row, 32 * c + 2 * i + 4 * h, four, f);
      }
    }
}

int run_window_bwd(const WindowArgs& a, int d, int dtype, hipStream_t st);

}  // namespace dfs
