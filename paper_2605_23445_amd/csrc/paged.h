// What the kernels of attention over a cache in pages share: their arguments, and how a wave finds pages.
#pragma once
#include "pages.h"
#include "window.h"

namespace dfs {

typedef int i32x2 __attribute__((ext_vector_type(2)));

struct PagedArgs : WindowArgs {                      // n_k: what the table has room for
  PageArgs pages;
  int32_t unit;                                      // pieces that are dealt out together
  int32_t row_bits;                                  // a block has 1 << row_bits rows
};

// Eight bytes of e4m3 times a power of two, exactly.
__device__ __forceinline__ bf16x8 eight(uint32_t a, uint32_t b, float scale_a, float scale_b) {
  const bf16x2 p = __builtin_amdgcn_cvt_scalef32_pk_bf16_fp8(a, scale_a, false), q = __builtin_amdgcn_cvt_scalef32_pk_bf16_fp8(a, scale_a, true);
  const bf16x2 r = __builtin_amdgcn_cvt_scalef32_pk_bf16_fp8(b, scale_b, false), s = __builtin_amdgcn_cvt_scalef32_pk_bf16_fp8(b, scale_b, true);
  return bf16x8{p[0], p[1], q[0], q[1], r[0], r[1], s[0], s[1]};
}
__device__ __forceinline__ bf16x8 eight(uint32_t a, uint32_t b, float scale) { return eight(a, b, scale, scale); }

// The pages of a sequence, 64 entries of the table at a time, one a lane: where a page's keys and values of a key head begin, and their scales.
template <bool E4M3> struct Entries {
  int first;
  uint64_t k, v;
  float ks, vs;
  const int32_t* row;
  __device__ __forceinline__ Entries(const PagedArgs& a, int s) : first(-(1 << 30)), k(0), v(0), ks(0.f), vs(0.f), row(a.pages.table + int64_t(s) * a.pages.row) {}
  // Lane that holds entry i.
  __device__ __forceinline__ int lane_of(const PagedArgs& a, int i, int kvh) {
    if (uint32_t(i - first) >= 64u) {
      first = i;
      int id = row[min_of(i + int(threadIdx.x & 63), a.pages.row - 1)];
      if (uint32_t(id) >= uint32_t(a.pages.pages)) id = 0;
      k = reinterpret_cast<uint64_t>(a.pages.k.at(id, kvh, 0));
      v = reinterpret_cast<uint64_t>(a.pages.v.at(id, kvh, 0));
      if constexpr (E4M3) {
        const int64_t at = int64_t(id) * a.pages.heads_kv + kvh;
        ks = a.pages.k_scale[at];
        vs = a.pages.v_scale[at];
        asm volatile("" : "+v"(ks), "+v"(vs));       // waited for here, or the compiler does it wherever they are used, and for all loads
      }
    }
    return i - first;
  }
  // What a lane holds, for the whole wave.
  static __device__ __forceinline__ uint64_t of(uint64_t x, int lane) {
    return uint64_t(uint32_t(__builtin_amdgcn_readlane(int(uint32_t(x >> 32)), lane))) << 32 | uint32_t(__builtin_amdgcn_readlane(int(uint32_t(x)), lane));
  }
  static __device__ __forceinline__ float of(float x, int lane) { return __int_as_float(__builtin_amdgcn_readlane(__float_as_int(x), lane)); }
};

// Whether the rows are so many that blocks of 128 of them, each over all its keys, are the faster way, and the launch of these.
bool paged_is_long(const dfs_paged* w, int dtype);
int run_paged_long(const PagedArgs& a, int d, int dtype, bool bytes, hipStream_t st);

}  // namespace dfs
