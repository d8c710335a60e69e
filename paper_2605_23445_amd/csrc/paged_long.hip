// Attention over a cache in pages: many rows, in blocks of 128 that each go over all their keys.  The kernels are those of windowed attention; this file brings the tiles
// of 64 keys, which lie on one to four pages each.
#include "paged.h"
#include "window_fwd.h"

namespace dfs {

// Where a tile's 16 rows number g lie (16 rows are on one page): their address, how many of them there are, and on which lane of the entries their scales.
struct Sixteen {
  uint64_t at;
  int rows, lane;
  template <bool E4M3>
  __device__ __forceinline__ Sixteen(const PagedArgs& a, Entries<E4M3>& entries, const View& v, const Span& span, int kvh, int t, int g, bool values) {
    const int piece = 2 * t + g / 2, key = span.begin(piece) + 16 * (g % 2), lo = max_of(0, span.p0 - a.left);
    rows = piece < span.n ? max_of(0, min_of(span.end(piece) - key, 16)) : 0;
    if (values && piece >= span.n_first && key + 15 < lo && key >= a.sinks) rows = 0;        // in front of every window
    lane = rows > 0 ? entries.lane_of(a, key >> a.pages.bits, kvh) : 0;
    at = Entries<E4M3>::of(values ? entries.v : entries.k, lane) + uint32_t(key & ((1 << a.pages.bits) - 1)) * uint32_t(v.row);
  }
};

// Rows [from, to) of tile t that no query of the block sees although some behind them are seen: their values, which may be anything, are left out.
struct Unseen {
  int from, to;
  __device__ __forceinline__ Unseen(const PagedArgs& a, const Span& span, int t) : from(0), to(0) {
    const int piece = span.n_first, lo = max_of(0, span.p0 - a.left);
    if (piece / 2 != t) return;
    const int key = span.begin(piece), row = piece % 2 * 32;
    from = row + max_of(0, a.sinks - key);
    to = row + min_of(lo - key, 32);
  }
};

// Rows of pages as they are, straight to LDS.
template <typename T, int D> struct PageFeed {
  static constexpr int STEP = 32, NW = 4;
  static constexpr bool STRAIGHT = true;
  using KTile = Tile<T, D, KN, NW, false>;
  using VTile = Tile<T, D, KN, NW, true>;
  static constexpr int LOADS = KTile::LOADS, CH = KTile::CH, RB = KTile::RB;
  const PagedArgs& a;
  int kvh, wave, lane;
  Entries<false> entries;
  typename KTile::Loader k_load;
  typename VTile::Loader v_load;
  struct Want {
    u32x4 desc[LOADS];
    int from, to;
  };
  template <class P, class S> __device__ __forceinline__ PageFeed(const PagedArgs& a_, const P& at, const S& seq, int wave_, int lane_)
      : a(a_), kvh(at.kvh), wave(wave_), lane(lane_), entries(a_, seq.seq), k_load(a_.pages.k.row, wave_, lane_), v_load(a_.pages.v.row, wave_, lane_) {}
  __device__ __forceinline__ Want tile(const View& v, const Span& span, int t, bool values) {
    Want w;
#pragma unroll
    for (int j = 0; j < LOADS; ++j) {
      const int g = (j * NW + wave) * 4 / CH;
      const Sixteen x(a, entries, v, span, kvh, t, g, values);
      const uint64_t at = x.at - uint64_t(16 * g) * uint64_t(v.row);
      const uint32_t bytes = x.rows > 0 ? uint32_t(16 * g + x.rows - 1) * uint32_t(v.row) + RB : 0;
      w.desc[j] = u32x4{uint32_t(__builtin_amdgcn_readfirstlane(uint32_t(at))), uint32_t(__builtin_amdgcn_readfirstlane(uint32_t(at >> 32))) & 0xFFFFu,
                        uint32_t(__builtin_amdgcn_readfirstlane(bytes)), 0x00020000u};
    }
    const Unseen u(a, span, t);
    w.from = values ? u.from : 0;
    w.to = values ? u.to : 0;
    return w;
  }
  __device__ __forceinline__ Want keys(const Span& span, int t) { return tile(a.pages.k, span, t, false); }
  __device__ __forceinline__ Want values(const Span& span, int t) { return tile(a.pages.v, span, t, true); }
  __device__ __forceinline__ void ask_keys(const Want& w, uint32_t to, int j) const { k_load.issue_one(w.desc[j], to, j); }
  __device__ __forceinline__ void ask_values(const Want& w, uint32_t to, int j) const {
    const int row = ((j * NW + wave) * 64 + lane) / CH;
    typename VTile::Loader load = v_load;
    if (row >= w.from && row < w.to) load.off[j] = 0x80000000u;          // zeros
    load.issue_one(w.desc[j], to, j);
  }
};

// Rows in 8 bits: through registers, where they become bf16.  A thread takes 16 bytes of a row.
template <int D> struct ByteFeed {
  static constexpr int STEP = 32, NW = 4;
  static constexpr bool STRAIGHT = false;
  using KTile = Tile<uint16_t, D, KN, NW, false>;
  using VTile = Tile<uint16_t, D, KN, NW, true>;
  static constexpr int SHARES = D / 64, CH = D / 16;                     // loads of a thread for a tile; chunks of a row
  const PagedArgs& a;
  int kvh, wave, row[SHARES], c;
  Entries<true> entries;
  u32x4 k[SHARES], v[SHARES];
  float k_scale[SHARES], v_scale[SHARES];
  template <class P, class S> __device__ __forceinline__ ByteFeed(const PagedArgs& a_, const P& at, const S& seq, int wave_, int lane)
      : a(a_), kvh(at.kvh), wave(wave_), c(lane % CH), entries(a_, seq.seq) {
#pragma unroll
    for (int j = 0; j < SHARES; ++j) row[j] = ((j * NW + wave) * 64 + lane) / CH;
  }
  __device__ __forceinline__ u32x4 load(const View& view, const Sixteen& x, int r) const {
    const auto from = __builtin_amdgcn_make_buffer_rsrc(reinterpret_cast<void*>(x.at), 0, x.rows > 0 ? uint32_t(x.rows - 1) * uint32_t(view.row) + D : 0, 0x00020000);
    return __builtin_bit_cast(u32x4, __builtin_amdgcn_raw_buffer_load_b128(from, r < 0 ? int(0x80000000u) : int(uint32_t(r % 16) * uint32_t(view.row)) + c * 16, 0, 0));
  }
  __device__ __forceinline__ void ask_keys(const Span& span, int t) {
#pragma unroll
    for (int j = 0; j < SHARES; ++j) {
      const Sixteen x(a, entries, a.pages.k, span, kvh, t, (j * NW + wave) * 4 / CH, false);
      k[j] = load(a.pages.k, x, row[j]);
      k_scale[j] = x.rows > 0 ? entries.of(entries.ks, x.lane) : 1.f;
    }
  }
  __device__ __forceinline__ void ask_values(const Span& span, int t) {
    const Unseen u(a, span, t);
#pragma unroll
    for (int j = 0; j < SHARES; ++j) {
      const Sixteen x(a, entries, a.pages.v, span, kvh, t, (j * NW + wave) * 4 / CH, true);
      v[j] = load(a.pages.v, x, row[j] >= u.from && row[j] < u.to ? -1 : row[j]);
      v_scale[j] = x.rows > 0 ? entries.of(entries.vs, x.lane) : 1.f;
    }
  }
  template <class TileT> __device__ __forceinline__ void put(const u32x4& x, float scale, uint32_t lds, int r) const {
    const uint32_t at = lds + uint32_t(r * TileT::RB) + (uint32_t(2 * c) ^ uint32_t(TileT::swizzle(r))) * 16;
    const bf16x8 lo = eight(x[0], x[1], scale), hi = eight(x[2], x[3], scale);
    *reinterpret_cast<LDS_PTR(u32x4)>(at) = __builtin_bit_cast(u32x4, lo);
    *reinterpret_cast<LDS_PTR(u32x4)>(at ^ 16) = __builtin_bit_cast(u32x4, hi);
  }
  __device__ __forceinline__ void put_keys(uint32_t lds, int j) const { put<KTile>(k[j], k_scale[j], lds, row[j]); }
  __device__ __forceinline__ void put_values(uint32_t lds, int j) const { put<VTile>(v[j], v_scale[j], lds, row[j]); }
  __device__ __forceinline__ void put_keys(uint32_t lds) const {
#pragma unroll
    for (int j = 0; j < SHARES; ++j) put_keys(lds, j);
  }
  __device__ __forceinline__ void put_values(uint32_t lds) const {
#pragma unroll
    for (int j = 0; j < SHARES; ++j) put_values(lds, j);
  }
};

bool paged_is_long(const dfs_paged* w) {
  const int64_t rows = int64_t(w->heads / w->heads_kv) * w->n_q, some = w->seqs < w->n_q ? w->seqs : w->n_q;
  return rows > 32 * int64_t(w->seqs) && (rows / 128 + some) * w->heads_kv > (w->d == 64 ? 128 : 64);
}

int run_paged_long(const PagedArgs& args, int d, int dtype, bool bytes, hipStream_t st) {
  PagedArgs a = args;
  a.set_blocks(int64_t(a.group) * a.n_q / 128 + a.packed);
  const unsigned grid = unsigned(int64_t(a.blocks) * a.heads_kv);
  auto run = [&](auto dim) {
    constexpr int D = decltype(dim)::value;
    if (dtype == DFS_F32) window_f32_kernel<D, IN_PAGES, PageFeed<float, D>, PagedArgs><<<grid, 256, 0, st>>>(a);
    else if (bytes) window_pipe_kernel<D, IN_PAGES, ByteFeed<D>, PagedArgs><<<grid, 256, 0, st>>>(a);
    else window_pipe_kernel<D, IN_PAGES, PageFeed<uint16_t, D>, PagedArgs><<<grid, 256, 0, st>>>(a);
  };
  d == 64 ? run(std::integral_constant<int, 64>{}) : run(std::integral_constant<int, 128>{});
  return launch_status("dfs_paged_attn_fwd");
}

}  // namespace dfs
