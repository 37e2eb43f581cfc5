// Which kernels an attention over packed prompts or pages takes, and how large its grids and its workspace are: host arithmetic on the
// bounds of a batch, without any HIP, so that a host compiler can build it alone.
#pragma once
#include <stddef.h>

#include "../../include/samkv.h"

namespace samkv {

// Sizes of a launch that follow from the bounds alone.
struct PagedAttnPlan {
  int kg;     // which wide tiles there are: see paged_attn.hpp
  bool once;  // every sequence is one tile of 32 rows
  int target_log2, ragged_log2, min_chunk, max_items, max_slots, tile_rows;
  bool joins;  // whether any sequence can have more than one chunk
  size_t part_lse, bytes;  // workspace: part_o, then part_lse
};

// Tiles have 32 rows (KG = 0); or, in launches that have wide ones, sequences of at most 32 rows per KV head are one tile of 32 and
// the others are cut into wide tiles: KG = 1, 256 rows, KG = 2, 128 rows whose keys two groups of waves share.  So there are no
// more items than whole tiles in the batch's rows and sequences, and the grid has few workgroups without an item.
constexpr int kFewRows = 32;
template <int KG>
constexpr int wide_rows() { return KG == 2 ? 128 : 256; }
template <int KG>
constexpr int wide_cost() { return KG == 2 ? 3 : 5; }  // time of a wide tile over a number of keys, in tiles of 32 rows


// What the device makes of a batch's lengths (Items in paged_attn.hpp).  Keys of a chunk: the cost of all tiles and heads, `total` keys
// of tiles of 32 rows, is shared out over 2^log2 workgroups; a wide tile's chunk has fewer keys by what the tile costs more.
// Wide tiles fill a compute unit and spend the time of 500 keys on their start and end: no more of them than there are units, so a
// sequence's chunks are rounded to the nearest, down up to 3/4 (2 x 300 tokens over 1500 keys, 32 heads, 160 tiles: 59 us with
// chunks rounded up, 44 to the nearest, 39 uncut; 500 over 8000, 128 tiles: 108 either way, 151 uncut).
struct ChunkKeys {
  int few, wide;
};
template <int KG>
constexpr ChunkKeys chunk_keys(unsigned long long total, int hkv, int log2, int min_chunk) {
  const unsigned long long share = (total * hkv + (1ull << log2) - 1) >> log2, of_wide = share / wide_cost<KG>(), longest = 1ull << 30;
  const int few = (int)((share < longest ? share : longest) + 63) / 64 * 64, wide = (int)(of_wide < longest ? of_wide : longest);
  return {few > min_chunk ? few : min_chunk, wide > 2 * min_chunk ? wide : 2 * min_chunk};
}
constexpr int chunks_of(bool wide, int len, ChunkKeys c) {
  const int n = wide ? (len + c.wide / 4) / c.wide : (len + c.few - 1) / c.few;
  return n > 1 ? n : 1;
}

// Which tiles a batch takes (KG). Times of a workgroup in steps of 256 rows x 64 keys (about 2.8 us, 2 where the chip is not full),
// with what it spends on its start and end: four steps for the wide kernels, which fill a compute unit each (five for the smaller),
// one and a half for tiles of 32 rows, of which two share one.
// Prompts: the larger of the longest workgroup and the mean one times the rounds that there are. Measured, prompts of one length,
// tiles of 32 / 128 / 256 rows, us: d = 128, 32 heads over 8: 1 x 200 tokens 10 / 14 / 16, 1 x 1000 35 / 31 / 42, 1 x 2048 95 / 65
// / 81, 1 x 4096 314 / 226 / 207, 4 x 512 49 / 37 / 31, 32 x 64 29 / 22 / 15, 20 x 300 101 / 81 / 57; d = 64, 8 heads: 1 x 1000 12
// / 19 / 28, 1 x 2048 19 / 31 / 49, 1 x 4096 51 / 56 / 91, 10 x 700 31 / 31 / 24.
// How the rows are spread over the sequences is known to the device alone: anything from evenly over all of them to prompts of
// max_len beside sequences of padding (a captured batch with room for many), so the tiles are taken whose loss is smallest where it
// is largest. 32 heads over 8, d = 128, 32 / 128 / 256 rows, us: 1 x 4000 tokens beside 70 x 30 348 / 253 / 222, 1 x 8192 and 511
// sequences without rows 1060 / 814 / 753, 4 x 1024 and 60 without 110 / 79 / 78; 8 heads over 2: 80 / 80 / 122, 268 / 210 / 263,
// 36 / 28 / 40.
inline int prompt_shape(long long rows, long long n_rows, long long n_seq, int max_len) {
  struct Times { double few, wide, mid; };
  auto times = [&](double mean_len) {
    const double longest = max_len / 64.0, mean = mean_len / 128;
    auto time = [&](double tile, double resident, double of_longest, double of_mean, double ends) {
      const double a = of_longest * longest + ends, b = rows / tile / resident * (of_mean * mean + ends);
      return a > b ? a : b;
    };
    const Times t = {time(32, 512, 0.45, 0.8, 1.5), time(256, 256, 1, 1, 4), time(128, 256, 0.5, 0.7, 5)};
    const double some = t.wide < t.mid ? t.wide : t.mid, best = t.few < some ? t.few : some;
    return Times{t.few / best, t.wide / best, t.mid / best};
  };
  const Times even = times(n_rows < n_seq ? 1 : n_rows / n_seq), packed = times(max_len < n_rows ? max_len : n_rows);
  auto larger = [](double x, double y) { return x > y ? x : y; };
  const double few = larger(even.few, packed.few), wide = larger(even.wide, packed.wide), mid = larger(even.mid, packed.mid);
  return few <= wide && few <= mid ? 0 : wide <= mid ? 1 : 2;
}
// New tokens over a cache: tiles of 32 rows where they are few (`tiles`, of all heads) and have few keys to see, since two of them
// share a compute unit and start and end in half the time; else 128 rows, or 256 where there are many. Measured, 32 / 128 / 256
// rows, us, 32 heads over 8, d = 128: 1 x 256 tokens over 600 keys 16 / 21 / 29, 4 x 128 21 / 22 / 30, 16 x 64 38 / 26 / 33, 64 x
// 40 83 / 93 / 68; over 2000: 1 x 64 19 / 27 / 33, 4 x 128 43 / 46 / 50, 4 x 400 120 / 90 / 80; over 6000: 1 x 64 31 / 37 / 46, 1 x
// 256 84 / 53 / 57; 8 heads over 2, d = 64: 4 x 400 over 2000 27 / 34 / 34, 16 x 64 24 / 33 / 34, 16 x 200 51 / 38 / 58, over 6000:
// 4 x 400 70 / 58 / 57. Sequences of at most two tiles of 32 have less to gain from sharing keys, 32 heads over 8, d = 128: 64 x 16
// over 600 41 / 50 / 51, over 2000 120 / 123 / 122, over 6000 306 / 304 / 306, 16 x 16 over 6000 90 / 94 / 95.
inline int paged_shape(long long most, long long rows, int max_len, int d) {
  const double tiles = rows / 32.0, keys = tiles * max_len;
  if (most <= 64 ? keys <= 2.6e6 : tiles <= 512 && keys * d <= 8e5 * 128) return 0;
  return rows <= 49152 ? 2 : 1;
}

// Whether the keys of a batch over pages may be cut: where the longest sequence can take `passes` steps of a tile's keys, `share`
// of the compute units have a tile without that, and the join (4 us; 6 to 10 for the results of wide tiles) costs less than the
// other units save. Where they all have one, only sequences of very different lengths gain, which the host does not see, and long
// ones are cut so that none takes the time of many. Measured, uncut / cut, us: single tokens, d = 128, 32 heads over 8: 4 sequences
// of 380 keys 14.3 / 14.7, 500 15.5 / 14.7, 16 of 760 20.6 / 21.2, 1000 24.4 / 22.3, 24 of 2000 42 / 47, 64 of 250 to 2000 59 / 61,
// 375 to 3000 83 / 82, 500 to 4000 111 / 106; wide tiles: 2 x 300 tokens over 1500 37 / 42, 8 x 200 over 3000 119 / 121, 1 x 500
// over 2000 44 / 44, 3000 61 / 54, 8000 143 / 108, 16 x 64 over 400 to 3000 66 / 68, 750 to 6000 117 / 111; 32 x 100, one over
// 30000 keys and the others over 600: 917 / 161.
inline bool cuts(int kg, double share, double passes) {
  if (kg > 0) return passes > (share <= 0.5 ? 8 / (1 - share) : 32);
  return passes > (share < 1 && 3 / (1 - share) < 16 ? 3 / (1 - share) : 16);
}

// Tiles of `tile` rows that there can be: sequences have at most `most` rows per KV head and `rows` together.
inline long long tiles_of(long long n_seq, long long n_rows, long long rows, long long most, long long tile) {
  const long long with_rows = n_seq < n_rows ? n_seq : n_rows;  // sequences with rows
  const long long each = with_rows * ((most + tile - 1) / tile), packed = rows / tile + with_rows;
  return each < packed ? each : packed;
}
inline long long shares_of(int log2, int hkv) { return ((1 << log2) + hkv - 1) / hkv; }
// Only tiles of more than one chunk have partial results, and those have less than twice their share of chunks.
inline long long slots_of(long long tiles, long long shares, long long tile) {
  return (tiles + shares < 2 * shares ? tiles + shares : 2 * shares) * (tile / 32);
}
constexpr int kUneven = 10;  // ragged_log2 of tiles of 32 rows
inline size_t up256(size_t x) { return (x + 255) / 256 * 256; }

inline PagedAttnPlan paged_attn_plan(int dtype, int d, int hq, int hkv, int n_seq, int n_rows, int max_new, int max_len, bool paged) {
  PagedAttnPlan p;
  const long long group = hq / hkv, rows = n_rows * group, most = max_new * group, n = n_seq;
  p.kg = dtype != SAMKV_BF16 || most <= 32 ? 0 : paged ? paged_shape(most, rows * hkv, max_len, d) : prompt_shape(rows * hkv, n_rows, n, max_len);
  p.once = most <= 32;
  p.target_log2 = p.kg > 0 ? 8 : 9;  // workgroups: as many as are resident at once
  p.min_chunk = p.kg > 0 || (dtype == SAMKV_BF16 && d == 64) ? 256 : 128;  // four waves with a tile of keys each
  // Items: the tiles that there can be, and the chunks that Items cuts (one holds at least 2^-ragged_log2 of the keys that
  // the tiles of all heads see).
  const long long tile = p.kg == 2 ? 128 : p.kg == 1 ? 256 : 32, tiles = tiles_of(n, n_rows, rows, most, tile);
  p.joins = paged && cuts(p.kg, tiles * hkv / 256.0, (double)max_len / (p.kg > 0 ? 128 : p.min_chunk));
  p.ragged_log2 = p.kg == 0 && n > 1 && tiles * hkv >= 128 ? kUneven : p.target_log2;  // fewer have many chunks each
  const long long shares = shares_of(p.ragged_log2, hkv);
  p.max_items = (int)(tiles + (p.joins ? shares : 0));
  p.max_slots = (int)(p.joins ? slots_of(tiles, shares, tile) : 0);
  p.tile_rows = (int)(most < 32 ? most : 32);
  const size_t part_rows = (size_t)p.max_slots * hkv * p.tile_rows;
  p.part_lse = up256(part_rows * d * 4);
  p.bytes = p.part_lse + up256(part_rows * 4);
  return p;
}

// Workspace of an attention over pages: enough for every batch of the same heads whose counts and bounds are no larger, one of which may
// be cut where this one is not (64 single tokens over 2048 keys are not, 4 are), or take smaller tiles.  The slots of either
// kind of tiles grow with the bounds; a batch of one tile is the first to be cut.
inline size_t paged_attn_workspace(int dtype, int d, int hq, int hkv, int n_seq, int n_rows, int max_new, int max_len) {
  const PagedAttnPlan p = paged_attn_plan(dtype, d, hq, hkv, n_seq, n_rows, max_new, max_len, true);
  const long long group = hq / hkv, rows = n_rows * group, most = max_new * group;
  auto bytes = [&](int kg, int min_step, long long tile, int log2) -> size_t {
    if (!cuts(kg, hkv / 256.0, (double)max_len / min_step)) return 0;
    const size_t part_rows = (size_t)slots_of(tiles_of(n_seq, n_rows, rows, most, tile), shares_of(log2, hkv), tile) * hkv * (most < 32 ? most : 32);
    return up256(part_rows * d * 4) + up256(part_rows * 4);
  };
  const bool even = n_seq == 1 || tiles_of(n_seq, n_rows, rows, most, 32) * hkv < 128;
  const size_t few = bytes(0, dtype == SAMKV_BF16 && d == 64 ? 256 : 128, 32, even ? 9 : kUneven);
  const size_t wide = p.kg > 0 ? bytes(p.kg, 128, p.kg == 2 ? 128 : 256, 8) : 0;  // a smaller batch takes no wider tiles
  return few > wide ? few : wide;
}

}  // namespace samkv
