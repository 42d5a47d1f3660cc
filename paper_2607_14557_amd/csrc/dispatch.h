// Which form a launch takes, from the sizes that the host knows.  Plain C++: no
// device code, so that the rules can be held to measured times on any machine.
#pragma once

#include <stddef.h>

namespace seer {

// ---- bf16 attention ---------------------------------------------------------

// The most tiles of `qt` rows that `rows` rows in `batch` sequences can make.
inline int max_row_tiles(int rows, int batch, int qt) {
  return rows >= batch ? (rows - batch) / qt + batch : rows;
}

// Queries of a workgroup of the split-key form.
constexpr int kFewQueries = 32;

// Whether the attention splits the keys over the waves of 32-query workgroups
// (attn_few_bf16_kernel) instead of walking them in 128-query ones.  Its
// workgroups hold 128 KiB of LDS, one a CU, and load K and V four times as often:
// it pays while one round holds them all, whatever the lengths (8 heads, 3700
// cached keys: 49 against 78 us at 1024 rows in two sequences; 64 against 56 at
// 2048, where they need two rounds), and while there are keys to split (4
// sequences of 64 rows and 100 cached keys, 32 heads: 12.0 against 10.2).
inline bool few_attention(int rows_ub, int batch, int heads, int kv_rows_ub, int cus) {
  const long long groups = (long long)max_row_tiles(rows_ub, batch, kFewQueries) * heads;
  const long long keys = ((long long)rows_ub + kv_rows_ub) / batch;     // of a sequence, on average
  return groups <= cus && keys >= 320;
}

// ---- bf16 GEMM of few tiles -------------------------------------------------

// The forms of a launch whose 256x256 tiles (of the rows bound) fill at most one
// round of the CUs:
//   FEW_NARROW, FEW_WIDE  128x64 and 128x128 tiles, K split over the waves of a
//                         workgroup and over few_k_splits workgroups (few_tile)
//   FEW_PARTS             256x256 tiles, K split over workgroups that leave fp32
//                         sums, added by a second launch
//   FEW_WHOLE             256x256 tiles and halves
enum FewShape { FEW_WHOLE, FEW_NARROW, FEW_WIDE, FEW_PARTS };

// The tiles that run whole in full rounds; the others are the last round's, K split.
constexpr int few_full(int units, int tiles) { return tiles > units ? tiles / units * units : 0; }

// K splits of a tile so that `tiles` tiles of 64-wide K tiles fill one round.
constexpr int few_k_splits(int units, int tiles, int ktiles) {
  if (tiles == 0) return 1;
  int s = units / tiles;
  s = s < ktiles / 8 ? s : ktiles / 8;
  return s < 1 ? 1 : (s > 16 ? 16 : s);
}

// The form by the number of 128-row tiles, which the kernel reads on the device:
// up to the first run's end its shape, and so on, FEW_WHOLE past the last.  A run
// is one word, so that the kernel has the rule with one scalar load.
constexpr int kFewRuns = 8;
struct FewRuns {
  unsigned run[kFewRuns];            // end << 16 | k_split << 12 | parts << 4 | shape
};
constexpr int few_end(unsigned run) { return (int)(run >> 16); }
constexpr int few_form(unsigned run) { return (int)(run & 15); }
constexpr int few_run_parts(unsigned run) { return (int)(run >> 4 & 255); }     // FEW_PARTS: K splits of a tile
constexpr bool few_run_splits(unsigned run) { return (run >> 12 & 1) != 0; }    // whether few_k_splits applies

struct FewRule {
  FewRuns runs;
  int n_runs;
  int grid;              // the most workgroups that any row count up to the bound has
  int parts_rows;        // rows that the second launch has to cover, 0 for none
};

struct FewLaunch {
  int m_ub, N, K;
  int units;             // workgroups that run at once
  bool k_split;          // scratch and counters for few_k_splits
  bool parts;            // the epilogue has a second launch
  size_t scratch;        // bytes for its sums
};

// K splits of FEW_PARTS: the most whose units fit one round and their sums (of
// whole 128-row tiles) the scratch, each of an even number of 64-wide K tiles
// (the loop's unroll); 0 for fewer than three, where two gain nothing over halves,
// and for a K below 8192, where the second launch costs more than the parts save
// (K = 5632, N = 2048, 1280 rows: 48.9 against 41.9 us in 128x128 tiles; K = 12288,
// N = 4096, 640 rows: 84.5 against 101).
inline int few_parts(const FewLaunch& g, int row_tiles) {
  if (!g.parts || g.K < 8192) return 0;
  const int ktiles = g.K / 64;
  int s = g.units / ((row_tiles + 1) / 2 * (g.N / 256));
  s = s < 16 ? s : 16;
  while (s > 2 && (ktiles % (2 * s) != 0 || (size_t)s * row_tiles * 128 * g.N * 4 > g.scratch)) --s;
  return s > 2 ? s : 0;
}

// Expected us of a form at `row_tiles` row tiles, below 0 where it doesn't apply:
// fits to the measured times of each form alone, 97 to 12,000 rows, d_model 512 to
// 4096 (rms 10, 11, 16 and 6%).  128x64 tiles are left to one round and 128x128
// ones to two: more never paid (2048 rows at N = K = 2048: 28 us in one round of
// 128x128 tiles, 32 in two of 128x64 ones, 29 whole).
inline double few_us(const FewLaunch& g, int shape, int row_tiles) {
  const double k = g.K / 4096.0, weights = 2.0 * g.N * g.K;
  if (shape == FEW_NARROW || shape == FEW_WIDE) {
    const bool wide = shape == FEW_WIDE;
    const int tiles = row_tiles * (g.N / (wide ? 128 : 64));
    // the 128x128 loop takes two K tiles a wave
    if (tiles > (wide ? 2 : 1) * g.units || (wide && g.K % 512 != 0)) return -1.0;
    const int full = few_full(g.units, tiles), rem = tiles - full;
    const int s = g.k_split ? few_k_splits(g.units, rem, g.K / 64) : 1;
    const double round = (wide ? 29.3 : 20.8) * k;
    double us = rem > 0 ? round : 0.0;
    if (rem > 0 && s > 1) us = round / s + (wide ? 9.9 + 0.66 * s : 5.2 + 0.16 * s);
    if (full > 0) us = 1.1 * (us + round * (full / g.units));
    return (wide ? 9.4 : 6.0) + (us > weights / 5.0e6 ? us : weights / 5.0e6);
  }
  if (shape == FEW_PARTS) {
    const int s = few_parts(g, row_tiles);
    if (s == 0) return -1.0;
    return 10.0 + 88.6 * k / s + 0.16 * s * (128.0 * row_tiles) * g.N * 8e-6;
  }
  const int tn = g.N / 256;
  const int full = row_tiles / 2 * tn, half = row_tiles % 2 ? tn : 0;   // tiles; half tiles of a short last row
  const bool halves = 2 * full + half <= g.units;
  const double us = halves ? 47.3 * k : 89.1 * k * ((full + g.units - 1) / g.units);
  return 5.8 + (us > weights / 4.0e6 ? us : weights / 4.0e6);
}

inline FewRule few_rule(const FewLaunch& g) {
  FewRule r{};
  const int tn = g.N / 256;
  const int last = (g.m_ub + 127) / 128;
  // past two rounds of 128x128 tiles only whole tiles are left
  int lim = g.units / tn + 1;
  lim = lim < last ? lim : last;
  auto best = [&](int t, bool parts) {
    int shape = FEW_WHOLE;
    double us = few_us(g, FEW_WHOLE, t);
    for (int f = FEW_NARROW; f <= FEW_PARTS; ++f) {
      const double v = f == FEW_PARTS && !parts ? -1.0 : few_us(g, f, t);
      if (v >= 0.0 && v < us) { us = v; shape = f; }
    }
    return shape;
  };
  // Every row count waits for the second launch, in vain where its form has none
  // (5 us), so parts are for a bound that takes them itself and row counts within
  // two row tiles of it.
  const bool parts = best(last, true) == FEW_PARTS;
  // whole tiles: tiles of 128 rows while they fit as halves, else of 256
  const int whole = (last + 1) / 2 * tn;
  int most = last * tn <= g.units ? last * tn : (g.units / tn) * tn;
  most = most > whole ? most : whole;
  int used = 0, prev = -1;
  for (int t = 1; t <= lim; ++t) {
    const int shape = best(t, parts && t >= last - 1);
    int p = 0, u = 0;
    if (shape == FEW_PARTS) {
      p = few_parts(g, t);
      u = (t + 1) / 2 * tn * p;
      r.parts_rows = 128 * t;
    } else if (shape != FEW_WHOLE) {
      const int tiles = t * (g.N / (shape == FEW_WIDE ? 128 : 64)), full = few_full(g.units, tiles);
      u = full + (tiles - full) * (g.k_split ? few_k_splits(g.units, tiles - full, g.K / 64) : 1);
    }
    const int key = p << 4 | shape;
    if (key != prev) {
      if (used == kFewRuns) break;                   // the rest runs whole
      ++used;
      prev = key;
    }
    r.runs.run[used - 1] = (unsigned)t << 16 | (g.k_split ? 1u : 0u) << 12 | (unsigned)key;
    if (shape != FEW_WHOLE) r.n_runs = used;         // whole runs at the end need no word
    most = u > most ? u : most;
  }
  // Asking on the device costs whole tiles 1 to 1.5 us (1068 rows, d 4096, QKV: 93.8
  // against 95.4): not where only rows below a quarter of the bound gain by it.
  if (r.n_runs > 0 && last > 4 * few_end(r.runs.run[r.n_runs - 1])) r.n_runs = 0;
  for (int i = r.n_runs; i < kFewRuns; ++i) r.runs.run[i] = 0;
  r.grid = most;
  return r;
}

// ---- attention with grouped heads ---------------------------------------------

// Rows (token, head of the group) of a workgroup: 128 that walk the keys together,
// 32 whose keys are split over the workgroup's waves, 16 likewise (fp32).
constexpr int kGqaTile = 128, kGqaFew = 32, kGqaF32 = 16;

struct GqaRule {
  int rt;                // rows of a tile
  bool cut;              // whether the tiles' keys are cut, over `grid` workgroups
  int grid;
  bool sort;             // several rounds of 128-row tiles: the longest requests first (up to 64)
};

struct GqaLaunch {
  bool bf16;
  int heads, n_kv, dim;
  int rows, batch;       // bounds of the call
  long long keys;        // bound on the keys of a request
  bool half;             // a causal prompt: its tiles see half the keys on average
};

// x / d for x below 2^31 is (mulhi(x, mul) + x) >> shift.
struct GqaDivisor {
  unsigned mul;
  int shift;
};
inline GqaDivisor gqa_divisor(int d) {
  GqaDivisor r{0, 0};
  while ((1ll << r.shift) < d) ++r.shift;
  r.mul = (unsigned)((((1ull << r.shift) - d) << 32) / d + 1);
  return r;
}

// The most tiles, over all key/value heads.
inline long long gqa_tiles(const GqaLaunch& g, int rt) {
  const long long pairs = (long long)g.rows * (g.heads / g.n_kv);
  return (pairs >= g.batch ? (pairs - g.batch) / rt + g.batch : pairs) * g.n_kv;
}

// Workgroups that a cut launch has: as many as run at once, but on average at most 32
// parts a tile (the joining of 128 parts took 20 us), nor more than there are blocks.
inline int gqa_cut_grid(const GqaLaunch& g, int rt) {
  const int wgs = rt == kGqaFew && g.dim <= 64 ? 1024 : 512;
  const long long blocks = (g.keys + 63) / 64 > 0 ? (g.keys + 63) / 64 : 1;
  const long long most = gqa_tiles(g, rt) * (blocks < 32 ? blocks : 32);
  return (int)(most < wgs ? most : wgs);
}

// Expected us of a form, the call's host time included where it is the longer: fits
// to the measured times of each form alone (bf16: 420 calls of 1 to 256 requests, 1 to
// 4000 rows and 15 to 40,000 keys each, rms 5 to 11% uncut, 20 to 22% cut; fp32: 201 calls,
// rms 16 to 24%).  Uncut, a tile's keys are one walk, and the tiles run in rounds; cut,
// all workgroups share the blocks, and a second launch joins.
inline double gqa_us(const GqaLaunch& g, int rt, bool cut) {
  struct Uncut { double base, first, step, round, round_step; int slots, keys; };
  struct Cut { double base, block, tile; };
  static constexpr Uncut kUncut[3][2] = {             // [form][head_dim > 64]
      {{7.4, 0.0, 0.94, 1.5, 1.29, 512, 64}, {7.6, 0.7, 1.27, 5.1, 1.79, 512, 64}},
      {{5.1, 2.3, 0.95, 4.8, 1.18, 512, 128}, {5.3, 3.0, 1.32, 6.3, 1.20, 256, 128}},
      {{5.8, 1.2, 1.34, 2.8, 1.54, 512, 64}, {4.1, 3.3, 2.93, 7.1, 3.31, 512, 64}}};
  static constexpr Cut kCut[3][2] = {
      {{13.4, 1.26, 2.5}, {14.7, 1.92, 5.0}},
      {{13.7, 1.21, 3.1}, {14.2, 1.34, 3.3}},
      {{11.3, 1.59, 0.0}, {11.1, 3.02, 4.2}}};
  const int form = rt == kGqaTile ? 0 : (rt == kGqaFew ? 1 : 2), big = g.dim > 64;
  const double tiles = (double)gqa_tiles(g, rt);
  // of packed rows the host knows the sum alone: no request is taken for longer than twice the average
  double keys = (double)g.keys;
  if (g.half && keys > 2.0 * g.rows / g.batch) keys = 2.0 * g.rows / g.batch;
  // what all tiles see together, by the bound: a causal prompt's half; the pages that a table has
  // room for are seldom all in use (64 requests of 500 to 16,000 keys: 115 us cut, 192 uncut)
  const double some = g.half ? 0.5 : 0.6;
  if (!cut) {
    const Uncut& c = kUncut[form][big];
    const double steps = keys / c.keys, one = c.first + c.step * steps;
    const double all = tiles / c.slots * (c.round + c.round_step * steps * some);
    return c.base + (one > all ? one : all);
  }
  const Cut& c = kCut[form][big];
  const double slots = rt == kGqaFew && !big ? 1024 : 512, share = tiles * keys / 64 / slots * (g.half ? 1.0 : some);
  return c.base + c.block * (share > 1.0 ? share : 1.0) + c.tile * tiles / slots;
}

inline GqaRule gqa_rule(const GqaLaunch& g) {
  GqaRule best{};
  double least = 0.0;
  const int forms[2] = {g.bf16 ? kGqaFew : kGqaF32, kGqaTile};
  for (int f = 0; f < (g.bf16 ? 2 : 1); ++f) {
    const int rt = forms[f];
    const long long tiles = gqa_tiles(g, rt), blocks = (g.keys + 63) / 64;
    for (int cut = 0; cut < 2; ++cut) {
      // the places of the line are counted in 31 bits; 128-row parts are for more than 32 rows a request
      if (cut && (blocks > 0x7fffffff / tiles ||
                  (rt == kGqaTile && (long long)g.rows * (g.heads / g.n_kv) <= 32ll * g.batch)))
        continue;
      const double us = gqa_us(g, rt, cut);
      if (best.rt == 0 || us < least) {
        best.rt = rt;
        best.cut = cut;
        best.grid = cut ? gqa_cut_grid(g, rt) : (int)tiles;
        best.sort = !cut && rt == kGqaTile && g.batch > 1 && g.batch <= 64 && tiles > 512;
        least = us;
      }
    }
  }
  return best;
}

// The keys of a request over pages: no more than its row of the table has, and at most
// 2^31 - 1024, so that a place up to four tiles behind the last key fits an int.
constexpr int kGqaMostKeys = 0x7fffffff - 1023;
constexpr int gqa_keys(int kv_len, int width, int shift) {
  const long long room = (long long)width << shift, most = room < kGqaMostKeys ? room : kGqaMostKeys;
  return kv_len < 0 ? 0 : (kv_len > most ? (int)most : kv_len);
}

// Whether the line of `all` blocks is cut in runs of one length (GqaCut): more blocks than
// workgroups, and room for two runs a tile.  `tiles` goes up to 2^31 - 1.
constexpr bool gqa_in_runs(int all, int most, int tiles) { return all > most && tiles > 1 && tiles <= most / 2; }

// The shortest run that leaves room for each tile's odd one.
constexpr int gqa_run_room(int blocks, int most, int tiles) {
  return (int)(((unsigned)blocks + most - tiles - 1) / (unsigned)(most - tiles));
}

// Bytes of the parts of a cut launch: their records, then two results a workgroup (the
// sums of each row, its maximum and its divisor).
inline size_t gqa_record_bytes(int grid) { return ((size_t)grid * 32 + 255) / 256 * 256; }
inline size_t gqa_part_bytes(int grid, int rt, int dim) {
  return gqa_record_bytes(grid) + (size_t)2 * grid * rt * ((dim > 64 ? 128 : 64) + 2) * 4;
}

// The most that any launch with up to these rows and requests needs, whatever its keys and mask.
inline size_t gqa_workspace(GqaLaunch g) {
  g.keys = 1 << 20;
  const int few = g.bf16 ? kGqaFew : kGqaF32;
  size_t most = gqa_part_bytes(gqa_cut_grid(g, few), few, g.dim);
  // 128-row parts are for more than 32 rows a request, so the most requests of a call that has them
  const long long tiled = ((long long)g.rows * (g.heads / g.n_kv) - 1) / 32;
  if (g.bf16 && tiled > 0) {
    g.batch = tiled < g.batch ? (int)tiled : g.batch;
    const size_t tile = gqa_part_bytes(gqa_cut_grid(g, kGqaTile), kGqaTile, g.dim);
    most = tile > most ? tile : most;
  }
  return most;
}

// ---- attention weight of cached tokens --------------------------------------------

// Rows (token, head of the group) of a workgroup that makes their statistics.
inline int weights_tile(bool bf16) { return bf16 ? 128 : 16; }

// Parts that a request's keys are cut in for the rows' statistics: what gives each of 1024
// workgroups about two tiles (bf16) or one (fp32).  The second launch joins them for each of its
// tiles, so no more than 8 up to 8192 places.  bf16, us with at most 4, 8 and 12 parts: 64
// rows of each of 7 prompts of 1500 to 8192 74, 64 and 68; 4 requests of 64 rows over 4064
// keys, 16 heads on 1, 40, 34 and 36; 2 of 12 to 20 rows over up to 11,600 keys 59, 38 and 33, with
// 22 28.  Parts of 256 keys or more: with at least 64, 256 and 1024 100 rows over 2000 keys, 28
// heads on 4, take 31, 28 and 38 us, 4 requests of 64 rows over 964 keys 25, 22 and 30.  fp32, with
// at most 4, 8 and 16 parts: trees over 1198 keys 20.5, 18.7 and 21.4 us; 800 rows over 4800
// keys, 8 heads on 2, 119 with up to 4 parts, 126 with 8, which 1024 tiles cut to 2.
inline int weights_want(bool bf16) { return bf16 ? 2048 : 1024; }
constexpr int kWeightsParts = 32, kWeightsPart = 256;
inline int weights_parts(long long rows, int batch, int heads, int n_kv, long long places, bool bf16, bool few) {
  const int tile = few ? 32 : weights_tile(bf16);
  const long long tiles = ((rows * (heads / n_kv) + tile - 1) / tile + batch - 1) * n_kv;
  const long long parts = (few ? 4096 : weights_want(bf16)) / tiles;
  long long most = few ? kWeightsParts : 8;
  if (bf16 && !few) {
    if (places > 8192) most = places / 512 < kWeightsParts ? places / 512 : kWeightsParts;
    if (places / kWeightsPart < most) most = places / kWeightsPart;
  }
  return parts < 1 || most < 1 ? 1 : (int)(parts > most ? most : parts);
}

// The most (row, head, part) that any call with up to so many rows has: as tiles are at
// least rows * heads / tile, there are at most want * tile of them where the keys are cut at all.
inline long long weights_stats(long long rows, int heads, bool bf16) {
  const long long all = rows * heads, most = (long long)weights_want(bf16) * weights_tile(bf16);
  const long long cut = all > most ? all : most;
  return cut < all * kWeightsParts ? cut : all * kWeightsParts;
}

// Whether the scores of the statistics' launch are kept for the sums (bf16): 8 bytes a row,
// head and key, written and read, instead of the head's key again, 2 * head_dim; not for more
// than 16 rows of a head on average, nor for more scores than this in all.  Tiles and kept
// scores, us: 64 requests over 4000 keys, 32 heads on 8, of 1 row 227 and 132, 4 rows (16 of a
// head) 234 and 165, 8 rows 240 and 239; 16 requests over 1000 keys, 32 heads, of 16 rows 62
// and 67, 32 rows 61 and 84; 64 requests over 2000 keys, 8 heads of 64, of 8 rows 71 and 53, 32
// rows 72 and 93.
constexpr long long kWeightsScores = 1 << 26, kWeightsFew = 16;
inline bool weights_few(long long rows, int batch, int heads, int n_kv, long long places, bool bf16) {
  return bf16 && rows * (heads / n_kv) <= kWeightsFew * batch && rows * heads <= kWeightsScores / places;
}
// The most that a call with up to so many rows and requests keeps.
inline long long weights_scores(long long rows, int batch, int heads, int n_kv, long long places, bool bf16) {
  const long long few = kWeightsFew * batch / (heads / n_kv);          // rows of that many requests
  const long long most = (rows < few ? rows : few) * heads;
  return bf16 ? (most < kWeightsScores / places ? most : kWeightsScores / places) * places : 0;
}

// Parts that a request's rows are cut in for the sums (bf16, tiles): where the tiles of keys are
// few and the rows many, as with one or two key/value heads; 4 tiles of 64 rows each if one
// request has twice what all have on average.  Uncut and cut, us, without a mask: 256 rows over
// 1056 keys, 32 heads on 8, 32 and 25; 512 rows over 1312 keys 53 and 33; 64 rows over 4064 keys, 16
// heads on 1, 36 and 27; 8 requests of 150 rows over 450 keys, 14 heads on 2 of 64, 32 and 25; 5 of up
// to 400 rows over up to 900 keys, 14 heads on 2, causal, 70 and 31; 8 of 64 rows over 564 keys, 32 heads
// on 8, 21.5 and 25 (not cut by this).  All by the bounds of a call: 512 rows over 1312 keys in a
// table of 32,768 places are not cut and take 67.
constexpr int kWeightsSums = 16, kWeightsSumTiles = 1024;
inline int weights_sums(long long rows, int batch, int heads, int n_kv, long long places) {
  const long long tiles = (places + 127) / 128 * batch * n_kv;
  long long parts = 2 * rows * (heads / n_kv) / (64 * 4 * (batch + 1ll));
  parts = parts < kWeightsSumTiles / tiles ? parts : kWeightsSumTiles / tiles;
  return parts < 2 ? 1 : (parts > kWeightsSums ? kWeightsSums : (int)parts);
}
// The most floats of them: parts * tiles * 128.
constexpr long long kWeightsPartial = kWeightsSumTiles * 128;

// ---- eviction ---------------------------------------------------------------------

// Lists of up to 2048 places move their own rows, longer ones leave that to a second launch
// of many workgroups; in tables of up to 8192 places 1024 threads a list where there are fewer than
// two lists a CU, 256 or 512 otherwise, in wider ones always 1024.  us, lists of 1500 places in a launch of their own with 1024 and 256 threads, then
// in two: one token over, 32 lists 12.1 and 11.2, 15.4 and 15.6; 384 lists 12.6 and 11.3, 16.2
// and 15.6; 528 lists 16.0 and 12.3, 19.9 and 16.9; cut to 700, 32 lists 16 and 32, 15 and 17;
// 384 lists 37 and 50, 42 and 41; 528 lists 65 and 72, 65 and 62.  Lists of 6000 cut to 1024 in
// one launch and two: 32 lists 33 and 21, 288 lists 102 and 79, 528 lists 179 and 145 (one
// token over 5000, 32 lists: 13 and 17).
struct EvictRule {
  int places;            // the most of a list that a workgroup keeps in registers; 0: any number, read again
  bool few;              // few lists: more threads each
  bool fused;            // whether it moves the list's rows too, instead of a second launch
  int parts;             // workgroups of a list in that
};
inline EvictRule evict_rule(int lists, bool shared, long long places) {
  EvictRule r{};
  r.places = places <= 2048 ? 2048 : (places <= 8192 ? 8192 : (places <= 16384 ? 16384 : 0));
  r.few = lists < 512;
  r.fused = !shared && r.places == 2048;
  r.parts = lists >= 4096 ? 1 : (4096 / lists > 128 ? 128 : 4096 / lists);
  return r;
}

// Moves that a list has room for: half its places, in whole 64.
inline size_t evict_room(long long places) { return (size_t)(places / 2 + 63) / 64 * 64; }
// Bytes of a list: slots from and to, and a bit of each place.
inline size_t evict_list_bytes(long long places) { return evict_room(places) * 8 + evict_room(places) / 32 * 8; }

}  // namespace seer
