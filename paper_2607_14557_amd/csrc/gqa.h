// What the kernels of the attention with grouped heads share: how a launch is
// cut into units, where keys lie, which of them a row sees.
#pragma once

#include <limits.h>
#include <math.h>

#include "common.h"
#include "dispatch.h"
#include "kernels.h"

namespace seer {

// Keys are cut at multiples of this.
constexpr int kGqaBlock = 128;

// Rows of a key/value head are (token, query head of its group) pairs, the head
// fastest: row i is token i / G, head i % G.  A tile is RT such rows, so K and V
// are read once for all the query heads that share them, whatever G is.

// A request of the call.
struct GqaSeq {
  int s0, len, used;       // first row, rows, real rows
  int nk, past;            // keys; the position of the first row (may be negative)
  int rows, tiles;         // len * G and the tiles of it
};

template <int RT>
__device__ __forceinline__ GqaSeq gqa_seq(const GqaParams& p, int b) {
  GqaSeq s;
  s.s0 = p.cu[b];
  int len = p.cu[b + 1] - s.s0;
  if (s.s0 < 0 || s.s0 >= p.rows_ub || len < 0) len = 0;
  s.len = len > p.rows_ub - s.s0 ? p.rows_ub - s.s0 : len;    // never touch rows past the bound
  int used = p.used ? p.used[b] : s.len;
  s.used = used < 0 ? 0 : (used > s.len ? s.len : used);
  if (p.table) {
    const long long most = (long long)p.width << p.shift;
    const int nk = p.kv_len[b];
    s.nk = nk < 0 ? 0 : (nk > most ? (int)most : nk);
  } else {
    s.nk = s.used;
  }
  s.past = s.nk - s.used;
  s.rows = s.len * p.group;
  s.tiles = (s.rows + RT - 1) / RT;
  return s;
}

__device__ __forceinline__ int gqa_blocks(int nk) { return nk > kGqaBlock ? (nk - 1) / kGqaBlock + 1 : 1; }

// One workgroup's share: tile t of request b for key/value head hk, keys
// [lo, hi); part `part` of the `parts` that the tile's keys are cut into, whose
// results lie from slot on (slot + part is this one's).
struct GqaUnit {
  int b, t, hk, lo, hi, part, parts, slot;
  GqaSeq s;
};

// The keys that any row of tile t sees end here.
template <int RT>
__device__ __forceinline__ int gqa_tile_end(const GqaParams& p, const GqaSeq& s, int t) {
  if (s.used == 0) return 0;
  if (p.mask != kMaskCausal) return s.nk;
  int last = ((t + 1) * RT - 1) / p.group;                 // last token of the tile
  last = last < s.used ? last : s.used - 1;
  const int end = s.past + last + 1;
  return end < 0 ? 0 : (end < s.nk ? end : s.nk);
}

// Finds unit bid of the launch; false past the last one.  Called by all 256
// threads: each sums its share of the requests, then one scan over the
// workgroup locates the unit.  p.target > 0: the tiles' keys are cut so that
// about p.target units come out over all heads, every part the same number of
// blocks, whatever the requests' lengths.  TILES: bid counts tiles instead (for
// the joining of their parts).
template <int RT, bool TILES>
__device__ __forceinline__ bool gqa_find(const GqaParams& p, int bid, GqaUnit& u) {
  __shared__ long long wave_sum[4];
  __shared__ int found[4];
  const int tid = threadIdx.x, lane = tid & (kWave - 1), wave = tid >> 6;
  const int per = (p.B + 255) / 256;
  const int b0 = tid * per < p.B ? tid * per : p.B;
  const int b1 = b0 + per < p.B ? b0 + per : p.B;
  int chunk = INT_MAX;
  if (p.target > 0) {
    long long n = 0;
    for (int b = b0; b < b1; ++b) {
      const GqaSeq s = gqa_seq<RT>(p, b);
      n += (long long)s.tiles * gqa_blocks(s.nk);
    }
#pragma unroll
    for (int off = 32; off > 0; off >>= 1) n += __shfl_xor(n, off, kWave);
    if (lane == 0) wave_sum[wave] = n;
    __syncthreads();
    n = (wave_sum[0] + wave_sum[1] + wave_sum[2] + wave_sum[3]) * p.n_kv;
    __syncthreads();
    const long long c = (n + p.target - 1) / p.target;
    chunk = c < p.min_chunk ? p.min_chunk : (c < INT_MAX ? (int)c : INT_MAX);
  }
  int units = 0, tiles = 0;
  for (int b = b0; b < b1; ++b) {
    const GqaSeq s = gqa_seq<RT>(p, b);
    units += s.tiles * ((gqa_blocks(s.nk) - 1) / chunk + 1);
    tiles += s.tiles;
  }
  // both sums in one scan
  long long inc = (long long)tiles << 32 | (unsigned)units;
  const long long own = inc;
#pragma unroll
  for (int off = 1; off < kWave; off <<= 1) {
    const long long v = __shfl_up(inc, off, kWave);
    if (lane >= off) inc += v;
  }
  if (lane == kWave - 1) wave_sum[wave] = inc;
  __syncthreads();
  long long all = 0, before = inc - own;
#pragma unroll
  for (int w = 0; w < 4; ++w) {
    if (w < wave) before += wave_sum[w];
    all += wave_sum[w];
  }
  const int n = TILES ? (int)(all >> 32) : (int)all;         // of one head
  if (bid >= n * p.n_kv || (long long)(unsigned)all * p.n_kv > p.max_units) return false;
  // each XCD takes a contiguous range of units, heads slowest: the tiles of one
  // request and head find their keys in its L2
  const int w = xcd_remap(bid, n * p.n_kv);
  u.hk = w / n;
  const int j = w - u.hk * n;
  int first = TILES ? (int)(before >> 32) : (int)before, unit0 = (int)before;
  if (j >= first && j < first + (TILES ? tiles : units)) {
    int b = b0;
    for (;; ++b) {
      const GqaSeq s = gqa_seq<RT>(p, b);
      const int parts = (gqa_blocks(s.nk) - 1) / chunk + 1, m = TILES ? s.tiles : s.tiles * parts;
      if (j < first + m) break;
      first += m;
      unit0 += s.tiles * parts;
    }
    found[0] = b;
    found[1] = j - first;
    found[2] = unit0;
  }
  __syncthreads();
  u.b = __builtin_amdgcn_readfirstlane(found[0]);
  const int rem = __builtin_amdgcn_readfirstlane(found[1]);
  const int base = __builtin_amdgcn_readfirstlane(found[2]);
  u.s = gqa_seq<RT>(p, u.b);
  const int most = (gqa_blocks(u.s.nk) - 1) / chunk + 1;       // parts that the request's tiles have room for
  u.part = TILES ? 0 : rem % most;
  // the tiles of a causal prompt from the last, which has the most keys, to the first
  u.t = u.s.tiles - 1 - (TILES ? rem : rem / most);
  const int end = gqa_tile_end<RT>(p, u.s, u.t);
  u.parts = (gqa_blocks(end) - 1) / chunk + 1;
  u.slot = u.hk * (int)all + base + (u.s.tiles - 1 - u.t) * most;
  const long long lo = (long long)u.part * chunk * kGqaBlock, hi = lo + (long long)chunk * kGqaBlock;
  u.lo = lo < end ? (int)lo : end;
  u.hi = hi < end ? (int)hi : end;
  return true;
}

// A read that the scalar unit makes where the address is the same for the whole wave.
__device__ __forceinline__ int scalar_load(const int* p, size_t i) {
  return reinterpret_cast<const __attribute__((address_space(4))) int*>(reinterpret_cast<uintptr_t>(p))[i];
}

// Which of keys [k0, k0 + 64) row `row` of the call (position pos, own rows from
// `past`) sees, of the keys before hi; bit i for key k0 + i.
__device__ __forceinline__ unsigned long long gqa_seen(const GqaParams& p, int k0, int hi, int pos, int past,
                                                       size_t row) {
  unsigned long long m = ~0ull;
  if (hi - k0 < 64) m = hi > k0 ? (1ull << (hi - k0)) - 1 : 0;
  if (p.mask == kMaskCausal) {
    const int d = pos - k0;
    if (d < 63) m &= d < 0 ? 0 : (2ull << d) - 1;
  } else if (p.mask == kMaskTree) {
    const int j = k0 - past;                       // the row of the call that key k0 is
    if (j > -64) {
      auto word = [&](int w) { return w < p.words ? p.bits[row * p.words + w] : 0ull; };
      if (j < 0) {
        m &= word(0) << -j | ((1ull << -j) - 1);
      } else {
        const int w = j >> 6, sh = j & 63;
        unsigned long long x = word(w) >> sh;
        if (sh) x |= word(w + 1) << (64 - sh);
        m &= x;
      }
    }
  }
  return m;
}

// The first key from which on gqa_seen may hide some from a row at position pos
// or later.
__device__ __forceinline__ int gqa_open_end(const GqaParams& p, int hi, int pos, int past) {
  if (p.mask == kMaskCausal) return pos + 1 < hi ? pos + 1 : hi;
  if (p.mask == kMaskTree) return past < hi ? past : hi;
  return hi;
}

}  // namespace seer
