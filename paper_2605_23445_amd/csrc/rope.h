// What the kernels that norm and turn rows share: chunks of 16 bytes of a row as fp32, sums over a row's lanes, sines and cosines of positions, and what the
// host makes of a geometry.
#pragma once
#include <math.h>

#include "view.h"

namespace dfs {

typedef unsigned int u32x4 __attribute__((ext_vector_type(4)));
typedef __bf16 bf16x2 __attribute__((ext_vector_type(2)));

// How rows turn, the same for all of a call's.
struct Turns {
  int32_t axes;
  int32_t rot[3];
  float eps;
  uint64_t freq[64];                                 // 2^-64 revolutions per unit of position, pair by pair
};

template <typename T> struct Chunk {};
template <> struct Chunk<uint16_t> {
  static constexpr int N = 8;
  static __device__ __forceinline__ void open(u32x4 p, float (&x)[8]) {
#pragma unroll
    for (int i = 0; i < 4; ++i) {
      x[2 * i] = __uint_as_float(p[i] << 16);
      x[2 * i + 1] = __uint_as_float(p[i] & 0xFFFF0000u);
    }
  }
  static __device__ __forceinline__ u32x4 close(const float (&x)[8]) {
    u32x4 p;
#pragma unroll
    for (int i = 0; i < 4; ++i) {
      const bf16x2 b = {(__bf16)x[2 * i], (__bf16)x[2 * i + 1]};
      p[i] = __builtin_bit_cast(uint32_t, b);
    }
    return p;
  }
};
template <> struct Chunk<float> {
  static constexpr int N = 4;
  static __device__ __forceinline__ void open(u32x4 p, float (&x)[4]) {
#pragma unroll
    for (int i = 0; i < 4; ++i) x[i] = __uint_as_float(p[i]);
  }
  static __device__ __forceinline__ u32x4 close(const float (&x)[4]) {
    return u32x4{__float_as_uint(x[0]), __float_as_uint(x[1]), __float_as_uint(x[2]), __float_as_uint(x[3])};
  }
};

// Sum over L lanes side by side (8, 16 or 32), the same bits in all of them.
template <int L> __device__ __forceinline__ float row_sum(float x) {
  auto dpp = [](float y, auto ctrl) { return __int_as_float(__builtin_amdgcn_mov_dpp(__float_as_int(y), decltype(ctrl)::value, 0xF, 0xF, true)); };
  x += dpp(x, std::integral_constant<int, 0xB1>{});  // within a quad: 1 0 3 2
  x += dpp(x, std::integral_constant<int, 0x4E>{});  // 2 3 0 1
  x += dpp(x, std::integral_constant<int, 0x141>{}); // mirrored within 8
  if (L > 8) x += dpp(x, std::integral_constant<int, 0x140>{});   // within 16
  if (L > 16) x += __shfl_xor(x, 16);
  return x;
}

// The turn of a token at position (p0, p1, p2): a lane keeps the cosines and sines of its channels.  SHARE: the two lanes of a pair's channels work out half of their angles
// each and exchange them, which is less work and a longer way.
template <typename T, int D, bool PAIRS, bool SHARE = false> struct Turn {
  static constexpr int N = Chunk<T>::N, L = D / N, C = PAIRS ? N / 2 : N;
  int c;
  int partner;                                       // halves: the lane that holds the other channels of this one's pairs
  float cs[C], sn[C];                                // halves: the sine with the sign that this lane's half takes

  template <class A> __device__ __forceinline__ void set(const A& a, int lane, int32_t p0, int32_t p1, int32_t p2) {
    c = lane % L;
    partner = lane;
    const int end0 = a.rot[0], end1 = end0 + a.rot[1], end2 = end1 + a.rot[2];
    if (PAIRS) {
#pragma unroll
      for (int i = 0; i < C; ++i) {
        const int ch = c * N + 2 * i;
        turn(ch < end0 ? p0 : ch < end1 ? p1 : p2, ch < end2 ? a.freq[ch / 2] : 0, cs[i], sn[i]);
      }
    } else {
      const int ch = c * N, axis = ch < end0 ? 0 : ch < end1 ? 1 : 2, begin = axis == 0 ? 0 : axis == 1 ? end0 : end1;
      const int half = (axis == 0 ? a.rot[0] : axis == 1 ? a.rot[1] : a.rot[2]) / 2, first = (ch - begin) < half;
      const bool turned = ch < end2;
      if (turned) partner = first ? lane + half / N : lane - half / N;
      const int base = begin / 2 + (ch - begin) - (first ? 0 : half);
      if constexpr (SHARE) {
        const int mine = first ? 0 : C / 2;
#pragma unroll
        for (int i = 0; i < C / 2; ++i) {
          float c0, s0;
          turn(axis == 0 ? p0 : axis == 1 ? p1 : p2, turned ? a.freq[base + mine + i] : 0, c0, s0);
          const float c1 = __shfl(c0, partner), s1 = __shfl(s0, partner);
          cs[i] = first ? c0 : c1;
          cs[i + C / 2] = first ? c1 : c0;
          sn[i] = first ? -s0 : s1;
          sn[i + C / 2] = first ? -s1 : s0;
        }
      } else {
#pragma unroll
        for (int i = 0; i < C; ++i) {
          turn(axis == 0 ? p0 : axis == 1 ? p1 : p2, turned ? a.freq[base + i] : 0, cs[i], sn[i]);
          if (first) sn[i] = -sn[i];
        }
      }
    }
  }
  static __device__ __forceinline__ void turn(int32_t p, uint64_t f, float& cos_, float& sin_) {
    const uint64_t t = uint64_t(int64_t(p)) * f;
    sincospif(fmaf(float(uint32_t(t)), 0x1p-63f, float(int32_t(t >> 32)) * 0x1p-31f), &sin_, &cos_);
  }
  // Turns a row; BACK: by the opposite angle.
  template <bool BACK> __device__ __forceinline__ void rotate(float (&y)[N]) const {
    if (PAIRS) {
#pragma unroll
      for (int i = 0; i < C; ++i) {
        const float p = y[2 * i], q = y[2 * i + 1], s = BACK ? -sn[i % C] : sn[i % C];
        y[2 * i] = p * cs[i] - q * s;
        y[2 * i + 1] = p * s + q * cs[i];
      }
    } else {
#pragma unroll
      for (int i = 0; i < N; ++i) {
        const float other = __shfl(y[i], partner);
        y[i] = y[i] * cs[i % C] + other * (BACK ? -sn[i % C] : sn[i % C]);
      }
    }
  }
};

// ONCE: past the memory-side cache, which cannot hold what is read.
template <bool ONCE> __device__ __forceinline__ u32x4 load_chunk(const char* p) {
  const u32x4* q = reinterpret_cast<const u32x4*>(p);
  return ONCE ? __builtin_nontemporal_load(q) : *q;
}

template <int N> __device__ __forceinline__ void weights(const float* w, int c, float (&x)[N]) {
#pragma unroll
  for (int i = 0; i < N; ++i) x[i] = w ? w[c * N + i] : 1.f;
}

inline int check_qk(const char* call, const dfs_qk_geom* g) {
  if (!g) return fail(DFS_EINVAL, "%s: geometry pointer is NULL", call);
  // a token has 32 lanes at most, and a grid fewer than 2^32 in whole work-groups of 256
  if (g->batch < 0 || g->tokens < 0 || int64_t(g->batch) * g->tokens > (int64_t(1) << 27) - 8)
    return fail(DFS_ESHAPE, "%s: batch=%d x tokens=%d must be in [0, 2^27 - 8]", call, g->batch, g->tokens);
  if (g->heads < 1 || g->heads_kv < 1 || g->heads > 65535 || g->heads_kv > 65535)
    return fail(DFS_ESHAPE, "%s: heads=%d, heads_kv=%d must be in [1, 65535]", call, g->heads, g->heads_kv);
  if (g->d != 64 && g->d != 128) return fail(DFS_ESHAPE, "%s: d=%d: head dimension must be 64 or 128", call, g->d);
  if (g->axes < 1 || g->axes > 3) return fail(DFS_ESHAPE, "%s: axes=%d must be 1 to 3", call, g->axes);
  int64_t sum = 0;
  for (int i = 0; i < g->axes; ++i) {
    if (g->rot[i] < 1 || g->rot[i] % (g->interleaved ? 2 : 16))
      return fail(DFS_ESHAPE, "%s: rot[%d]=%d must be a positive multiple of %d", call, i, g->rot[i], g->interleaved ? 2 : 16);
    sum += g->rot[i];
  }
  if (sum > g->d) return fail(DFS_ESHAPE, "%s: %lld channels to turn, d=%d", call, (long long)sum, g->d);
  if (!(g->theta > 0.0) || !isfinite(g->theta)) return fail(DFS_EINVAL, "%s: theta must be positive and finite", call);
  if (!(g->eps >= 0.f) || !isfinite(g->eps)) return fail(DFS_EINVAL, "%s: eps must be finite and not negative", call);
  return DFS_OK;
}

// A frequency in 2^-64 revolutions, whole ones left out.  By way of two doubles: a conversion of a long double costs 50 ns, and a call makes up to 64.
inline uint64_t revolutions(long double f) {
  const long double x = f < 0.25L ? f : f - floorl(f);
  const double half = double(x * 0.5L), rest = double(x * 0.5L - (long double)half);         // half a revolution, by rounding, is a whole one twice
  return (half < 0.5 ? uint64_t(int64_t(half * 0x1p64)) * 2 : 0) + uint64_t(int64_t(rest * 0x1p65));
}

inline void fill_turns(const dfs_qk_geom* g, Turns* a) {
  a->axes = g->axes;
  a->eps = g->eps;
  int pair = 0;
  for (int i = 0; i < 3; ++i) {
    a->rot[i] = i < g->axes ? g->rot[i] : 0;
    if (!a->rot[i]) continue;
    // in extended precision a frequency is good to 2^-57 after up to 64 products; positions are whole, so whole revolutions of it do not matter
    const long double step = powl((long double)g->theta, -2.0L / a->rot[i]);
    long double f = 1.0L / 6.283185307179586476925286766559L;
    for (int j = 0; j < a->rot[i] / 2; ++j, f *= step) a->freq[pair++] = revolutions(f);
  }
}

}  // namespace dfs
