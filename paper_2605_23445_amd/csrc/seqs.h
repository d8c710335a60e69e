// How a wave finds its sequence among those that lie behind one another: their lengths are known on the device alone.
#pragma once
#include "common.h"

namespace dfs {

__device__ __forceinline__ int min_of(int a, int b) { return a < b ? a : b; }
__device__ __forceinline__ int max_of(int a, int b) { return a > b ? a : b; }

// Sum over a wave, the same in all lanes.
__device__ __forceinline__ int wave_sum(int x) {
  x += __builtin_amdgcn_mov_dpp(x, 0xB1, 0xF, 0xF, true);              // within a quad: 1 0 3 2
  x += __builtin_amdgcn_mov_dpp(x, 0x4E, 0xF, 0xF, true);              // 2 3 0 1
  x += __builtin_amdgcn_mov_dpp(x, 0x141, 0xF, 0xF, true);             // mirrored within 8
  x += __builtin_amdgcn_mov_dpp(x, 0x140, 0xF, 0xF, true);             // within 16
  const auto half = __builtin_amdgcn_permlane16_swap(uint32_t(x), uint32_t(x), false, false);
  x = int(half[0] + half[1]);
  const auto all = __builtin_amdgcn_permlane32_swap(uint32_t(x), uint32_t(x), false, false);
  return __builtin_amdgcn_readfirstlane(int(all[0] + all[1]));
}

// Sums over the lanes up to each one.
__device__ __forceinline__ int wave_sums(int x) {
  x += __builtin_amdgcn_update_dpp(0, x, 0x111, 0xF, 0xF, false);      // from 1, 2, 4 and 8 lanes in front, of the same 16
  x += __builtin_amdgcn_update_dpp(0, x, 0x112, 0xF, 0xF, false);
  x += __builtin_amdgcn_update_dpp(0, x, 0x114, 0xF, 0xF, false);
  x += __builtin_amdgcn_update_dpp(0, x, 0x118, 0xF, 0xF, false);
  x += __builtin_amdgcn_update_dpp(0, x, 0x142, 0xA, 0xF, false);      // the last of 16 to the next 16: rows 1 and 3
  x += __builtin_amdgcn_update_dpp(0, x, 0x143, 0xC, 0xF, false);      // of 32 to the next 32
  return x;
}

// Where sequence s begins; past the last one, where that ends.  Cut to the n rows that there are.
__device__ __forceinline__ int start_of(const int32_t* starts, int s, int n) { return max_of(0, min_of(starts[s], n)); }

// The last of n runs that begins at or in front of i, or -1; begin(s) does not fall.  A wave's lanes look at 64 at once.
template <class F> __device__ __forceinline__ int run_of(int n, int i, F begin) {
  const int lane = threadIdx.x & 63;
  int s = 0;
  while (n > 0) {
    const int step = (n + 63) / 64, at = lane * step;
    const bool begun = at < n && begin(s + min_of(at, n - 1)) <= i;
    const int c = __builtin_popcountll(__builtin_amdgcn_ballot_w64(begun));
    if (c == 0) return -1;
    s += (c - 1) * step;
    n = min_of(step, n - (c - 1) * step);
    if (step == 1) break;
  }
  return n > 0 ? __builtin_amdgcn_readfirstlane(s) : -1;
}

}  // namespace dfs
