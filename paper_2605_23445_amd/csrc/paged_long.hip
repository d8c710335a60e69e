// Attention over a cache in pages: many rows, in blocks of 128 that each go over all their keys.  The kernels are those of windowed attention; this file brings the tiles
// of 64 keys, which lie on one to four pages each.
#include "paged.h"
#include "window_fwd.h"

namespace dfs {

// Where 16 rows of a tile lie, which are on one page: their keys and values, how many there are, and on which lane of the entries the page is.  (The entries may be other
// ones when the values are asked for.)
struct Sixteen {
  uint64_t k, v;
  int lane, rows;
  // Number g of tile t.
  template <bool E4M3> __device__ __forceinline__ void find(const PagedArgs& a, Entries<E4M3>& entries, const Span& span, int kvh, int t, int g) {
    const int piece = 2 * t + g / 2, key = span.begin(piece) + 16 * (g % 2);
    const uint32_t in = uint32_t(key) & ((1u << a.pages.bits) - 1);
    rows = max_of(0, min_of(span.end(piece) - key, 16));                 // (behind the last piece `key` is past the end)
    lane = rows > 0 ? entries.lane_of(a, key >> a.pages.bits, kvh) : 0;
    k = entries.of(entries.k, lane) + in * uint32_t(a.pages.k.row);
    v = entries.of(entries.v, lane) + in * uint32_t(a.pages.v.row);
  }
};

// The first tile with rows of the window, and its rows [from, to) that no query of the block sees although some behind them are seen: their values, and what scales them, may be
// anything, and are left out.
struct Unseen {
  int tile, from, to;
  __device__ __forceinline__ Unseen(const PagedArgs& a, const Span& span) {
    const int piece = span.n_first, key = span.begin(piece), row = piece % 2 * 32;
    tile = piece / 2;
    from = row + max_of(0, a.sinks - key);
    to = row + min_of(max_of(0, span.p0 - a.left) - key, 32);
  }
};

// Rows of pages as they are, straight to LDS.  Values are asked for behind the same tile's keys.
template <typename T, int D> struct PageFeed {
  static constexpr int STEP = 32, NW = 4;
  static constexpr bool STRAIGHT = true;
  using KTile = Tile<T, D, KN, NW, false>;
  using VTile = Tile<T, D, KN, NW, true>;
  static constexpr int LOADS = KTile::LOADS, CH = KTile::CH;
  const PagedArgs& a;
  int kvh, wave, lane;
  Entries<false> entries;
  typename KTile::Loader k_load;
  typename VTile::Loader v_load;
  Sixteen place[LOADS];                              // of the keys asked for last
  Unseen unseen;
  struct Want {
    u32x4 desc[LOADS];
    int from, to;
  };
  template <class P, class S> __device__ __forceinline__ PageFeed(const PagedArgs& a_, const P& at, const S& seq, const Span& span, int wave_, int lane_)
      : a(a_), kvh(at.kvh), wave(wave_), lane(lane_), entries(a_, seq.seq), k_load(a_.pages.k.row, wave_, lane_), v_load(a_.pages.v.row, wave_, lane_), unseen(a_, span) {}
  __device__ __forceinline__ int group(int j) const { return (j * NW + wave) * 4 / CH; }
  __device__ __forceinline__ u32x4 desc(int j, uint64_t from, const View& v) const {
    const uint32_t front = uint32_t(16 * group(j)) * uint32_t(v.row);     // offsets count from the tile's first row
    const uint64_t at = from - front;
    const uint32_t bytes = place[j].rows > 0 ? front + uint32_t(place[j].rows - 1) * uint32_t(v.row) + KTile::RB : 0;
    return u32x4{uint32_t(__builtin_amdgcn_readfirstlane(uint32_t(at))), uint32_t(__builtin_amdgcn_readfirstlane(uint32_t(at >> 32))) & 0xFFFFu,
                 uint32_t(__builtin_amdgcn_readfirstlane(bytes)), 0x00020000u};
  }
  __device__ __forceinline__ Want keys(const Span& span, int t) {
    Want w;
#pragma unroll
    for (int j = 0; j < LOADS; ++j) {
      if (j > 0 && CH >= 16 && group(j) == group(j - 1)) place[j] = place[j - 1];
      else place[j].find(a, entries, span, kvh, t, group(j));
      w.desc[j] = desc(j, place[j].k, a.pages.k);
    }
    w.from = w.to = 0;
    return w;
  }
  __device__ __forceinline__ Want values(const Span& span, int t) {
    Want w;
#pragma unroll
    for (int j = 0; j < LOADS; ++j) w.desc[j] = desc(j, place[j].v, a.pages.v);
    w.from = t == unseen.tile ? unseen.from : 0;
    w.to = t == unseen.tile ? unseen.to : 0;
    return w;
  }
  __device__ __forceinline__ void ask_keys(const Want& w, uint32_t to, int j) const { k_load.issue_one(w.desc[j], to, j); }
  __device__ __forceinline__ void ask_values(const Want& w, uint32_t to, int j) const {
    const int row = ((j * NW + wave) * 64 + lane) / CH;
    typename VTile::Loader load = v_load;
    if (row >= w.from && row < w.to) load.off[j] = 0x80000000u;          // zeros
    load.issue_one(w.desc[j], to, j);
  }
};

// Rows in 8 bits: through registers, where they become bf16.  A thread takes 16 bytes of a row.  Bound by the vector port and the matrix cores beside it: 4 096 tokens of four prompts
// over up to 9 200 keys, 32 heads of 8, d = 128: 536 to 574 us as the clock has it (593 to 602 under the profiler, which lowers it), 830 to 890 TFLOP/s, 1.21 million cycles of which the matrix cores
// are busy 39 %.  Where it took 550, making bf16 of the bytes cost 80 of them (467 without it, 397 without the loads as well: 1.2 PFLOP/s); blocks of 256 rows, which halve it, take as long, as eight waves then wait for one another.  The writes' bank conflicts
// (an eighth of the LDS's time; none with the halves of every second four lanes swapped, which costs selects) are not what it waits for.
template <int D> struct ByteFeed {
  static constexpr int STEP = 32, NW = 4;
  static constexpr bool STRAIGHT = false;
  using KTile = Tile<uint16_t, D, KN, NW, false>;
  using VTile = Tile<uint16_t, D, KN, NW, true>;
  static constexpr int SHARES = D / 64, CH = D / 16;                     // loads of a thread for a tile; chunks of a row
  const PagedArgs& a;
  int kvh, wave, c, row[SHARES];
  uint32_t k_off[SHARES], v_off[SHARES], put_at[SHARES];                 // in a page's 16 rows; in a tile in LDS
  Entries<true> entries;
  Sixteen place[SHARES];                             // of the keys asked for last
  Unseen unseen;
  u32x4 k[SHARES], v[SHARES];
  float k_scale[SHARES], v_scale[SHARES], next_scale[SHARES];            // next: of the values that lie beside the keys asked for last
  template <class P, class S> __device__ __forceinline__ ByteFeed(const PagedArgs& a_, const P& at, const S& seq, const Span& span, int wave_, int lane)
      : a(a_), kvh(at.kvh), wave(wave_), c(lane % CH), entries(a_, seq.seq), unseen(a_, span) {
    static_assert(KTile::swizzle(5) == VTile::swizzle(5) && KTile::swizzle(13) == VTile::swizzle(13), "keys and values lie alike");
#pragma unroll
    for (int j = 0; j < SHARES; ++j) {
      row[j] = ((j * NW + wave) * 64 + lane) / CH;
      k_off[j] = uint32_t(row[j] % 16) * uint32_t(a.pages.k.row) + c * 16;
      v_off[j] = uint32_t(row[j] % 16) * uint32_t(a.pages.v.row) + c * 16;
      put_at[j] = uint32_t(row[j] * KTile::RB) + (uint32_t(2 * c) ^ uint32_t(KTile::swizzle(row[j]))) * 16;
    }
  }
  static __device__ __forceinline__ u32x4 load(uint64_t at_, int rows, const View& view, uint32_t off) {
    // (without these the descriptor is taken for one that differs from lane to lane, and the load becomes a loop)
    const uint64_t at = uint64_t(uint32_t(__builtin_amdgcn_readfirstlane(int(at_ >> 32)))) << 32 | uint32_t(__builtin_amdgcn_readfirstlane(int(uint32_t(at_))));
    const int n = __builtin_amdgcn_readfirstlane(rows);
    const uint32_t bytes = n > 0 ? uint32_t(n - 1) * uint32_t(view.row) + D : 0;
    return __builtin_bit_cast(u32x4, __builtin_amdgcn_raw_buffer_load_b128(__builtin_amdgcn_make_buffer_rsrc(reinterpret_cast<void*>(at), 0, bytes, 0x00020000), off, 0, 0));
  }
  __device__ __forceinline__ void ask_keys(const Span& span, int t) {
#pragma unroll
    for (int j = 0; j < SHARES; ++j) {
      place[j].find(a, entries, span, kvh, t, (j * NW + wave) * 4 / CH);
      k[j] = load(place[j].k, place[j].rows, a.pages.k, k_off[j]);
      k_scale[j] = entries.of(entries.ks, place[j].lane);
      next_scale[j] = place[j].rows > 0 ? entries.of(entries.vs, place[j].lane) : 1.f;
    }
  }
  // Behind the same tile's keys.
  __device__ __forceinline__ void ask_values(const Span& span, int t) {
#pragma unroll
    for (int j = 0; j < SHARES; ++j) {
      uint32_t off = v_off[j];
      v_scale[j] = next_scale[j];
      if (t == unseen.tile) {
        if (row[j] >= unseen.from && row[j] < unseen.to) off = 0x80000000u;                  // zeros
        const int first = (j * NW + wave) * 4 / CH * 16;
        if (first >= unseen.from && first + 16 <= unseen.to) v_scale[j] = 1.f;
      }
      v[j] = load(place[j].v, place[j].rows, a.pages.v, off);
    }
  }
  // Half `h` of a thread's chunk to a tile.
  __device__ __forceinline__ void put(const u32x4& x, float scale, uint32_t to, int h) const {
    *reinterpret_cast<LDS_PTR(u32x4)>(to ^ uint32_t(16 * h)) = __builtin_bit_cast(u32x4, h ? eight(x[2], x[3], scale) : eight(x[0], x[1], scale));
  }
  __device__ __forceinline__ void put_keys(uint32_t lds) const {
#pragma unroll
    for (int i = 0; i < 2 * SHARES; ++i) put(k[i / 2], k_scale[i / 2], lds + put_at[i / 2], i % 2);
  }
  __device__ __forceinline__ void put_values(uint32_t lds) const {
#pragma unroll
    for (int i = 0; i < 2 * SHARES; ++i) put(v[i / 2], v_scale[i / 2], lds + put_at[i / 2], i % 2);
  }
  // Slot f of a stage of tile t, of which there are 4 SHARES + 2 at least: the values of tile t + 1 and the keys of tile t + 2 go to LDS, and the next ones of both are
  // asked for, a little in every slot, so that matrix instructions go out between.
  __device__ __forceinline__ void step(int f, const Span& span, int t, uint32_t v_to, uint32_t k_to) {
    constexpr int U = 2 * SHARES;
    if (f < U) put(v[f / 2], v_scale[f / 2], v_to + put_at[f / 2], f % 2);
    else if (f == U) ask_values(span, t + 2);
    else if (f <= 2 * U) put(k[(f - U - 1) / 2], k_scale[(f - U - 1) / 2], k_to + put_at[(f - U - 1) / 2], (f - U - 1) % 2);
    else if (f == 2 * U + 1) ask_keys(span, t + 3);
  }
};

// Blocks of 128 rows, if they were all full, need to be 128 (us, blocks of 128 against keys dealt out; e4m3, d = 128, 8 key heads of 4: 200 tokens of two prompts over 4 000 keys, 50 blocks,
// 77 / 38; 500, 125, 81 / 70; 256 of sixteen, 64, 86 / 51; bf16, 8 of 8: 256 of 32, 128, 120 / 138; d = 64, 4 of 4: 600 of four over 3 000 keys, 75, 44 / 34;
// 1 600 over 1 000, 200, 28 / 40; fp32, d = 128, 32 of 8: 600 of four over 2 600, 150, 400 / 461), in fp32 at d = 64, where the others leave fewer rows empty, 256 (600 of four over 2 600, 150,
// 206 / 124; 5 000 of one x 8, 312, 533 / 529; 2 000 of four over 1 500, 500, 223 / 302).  That the rows lie in many sequences, a few in each, is not looked at: one token of each of 511
// streams over 1 024 to 8 192 keys, e4m3, 32 heads of 8, takes 853 us, of 512 streams, whose blocks have four rows each, 1 461; and a block's keys are one work-group's, so that a token over
// 100 000 keys beside a prompt of 2 048 and 126 streams makes a call of 2 408 us, of which the prompt alone takes 56 and the tokens alone 278.
bool paged_is_long(const dfs_paged* w, int dtype) { return int64_t(w->heads) * w->n_q >= (w->d == 64 && dtype == DFS_F32 ? 256 * 128 : 128 * 128); }

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
