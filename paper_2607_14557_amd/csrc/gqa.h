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

// What the joining of a tile's parts has to know, left by the unit of its first
// part (parts < 2: nothing to join), one per slot.
struct GqaRecord {
  int parts, s0, used, rows, t, hk, pad[2];
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

// Finds the workgroup's unit; false where there is none.  Called by all NT
// threads: each sums its share of the requests, then one scan over the workgroup
// locates the unit.  p.target > 0: the tiles' keys are cut so that about p.target
// units come out over all heads, every part the same number of blocks, whatever
// the requests' lengths; the workgroup leaves its slot's record.
template <int RT, int NT>
__device__ __forceinline__ bool gqa_find(const GqaParams& p, GqaUnit& u) {
  constexpr int NW = NT / kWave;
  __shared__ long long wave_sum[2][NW];
  __shared__ int found[10];
  const int tid = threadIdx.x, lane = tid & (kWave - 1), wave = tid >> 6;
  const int per = (p.B + NT - 1) / NT;
  const int b0 = tid * per < p.B ? tid * per : p.B;
  const int b1 = b0 + per < p.B ? b0 + per : p.B;
  // with at most one request a thread its lengths are read once
  GqaSeq mine{};
  if (per == 1 && b0 < b1) mine = gqa_seq<RT>(p, b0);
  auto seq = [&](int b) { return per == 1 ? mine : gqa_seq<RT>(p, b); };
  int chunk = INT_MAX;
  if (p.target > 0) {
    long long n = 0;
    for (int b = b0; b < b1; ++b) {
      const GqaSeq s = seq(b);
      n += (long long)s.tiles * gqa_blocks(s.nk);
    }
#pragma unroll
    for (int off = 32; off > 0; off >>= 1) n += __shfl_xor(n, off, kWave);
    if (lane == 0) wave_sum[0][wave] = n;
    __syncthreads();
    n = 0;
#pragma unroll
    for (int w = 0; w < NW; ++w) n += wave_sum[0][w];
    const long long c = (n * p.n_kv + p.target - 1) / p.target;
    chunk = c < 1 ? 1 : (c < INT_MAX ? (int)c : INT_MAX);
  }
  int units = 0;
  for (int b = b0; b < b1; ++b) {
    const GqaSeq s = seq(b);
    units += s.tiles * ((gqa_blocks(s.nk) - 1) / chunk + 1);
  }
  int inc = units;
#pragma unroll
  for (int off = 1; off < kWave; off <<= 1) {
    const int v = __shfl_up(inc, off, kWave);
    if (lane >= off) inc += v;
  }
  if (lane == kWave - 1) wave_sum[1][wave] = inc;
  __syncthreads();
  int n = 0, first = inc - units;
#pragma unroll
  for (int w = 0; w < NW; ++w) {
    if (w < wave) first += (int)wave_sum[1][w];
    n += (int)wave_sum[1][w];
  }
  GqaRecord* records = reinterpret_cast<GqaRecord*>(p.records);
  const int bid = blockIdx.x;
  if (bid >= (long long)n * p.n_kv || (long long)n * p.n_kv > p.max_units) {
    if (p.target > 0 && tid == 0) records[bid].parts = 0;
    return false;
  }
  // each XCD takes a contiguous range of units, heads slowest: the tiles of one
  // request and head find their keys in its L2
  const int w = xcd_remap(bid, n * p.n_kv);
  u.hk = w / n;
  const int j = w - u.hk * n;
  if (j >= first && j < first + units) {
    int b = b0;
    GqaSeq s;
    int m;
    for (;; ++b) {
      s = seq(b);
      m = s.tiles * ((gqa_blocks(s.nk) - 1) / chunk + 1);
      if (j < first + m) break;
      first += m;
    }
    found[0] = b; found[1] = j - first; found[2] = first;
    found[3] = s.s0; found[4] = s.len; found[5] = s.used; found[6] = s.nk; found[7] = s.past; found[8] = s.rows;
    found[9] = s.tiles;
  }
  __syncthreads();
  auto get = [&](int i) { return __builtin_amdgcn_readfirstlane(found[i]); };
  u.b = get(0);
  const int rem = get(1), base = get(2);
  u.s.s0 = get(3); u.s.len = get(4); u.s.used = get(5); u.s.nk = get(6); u.s.past = get(7); u.s.rows = get(8);
  u.s.tiles = get(9);
  const int most = (gqa_blocks(u.s.nk) - 1) / chunk + 1;       // parts that the request's tiles have room for
  u.part = rem % most;
  // the tiles of a causal prompt from the last, which has the most keys, to the first
  u.t = u.s.tiles - 1 - rem / most;
  const int end = gqa_tile_end<RT>(p, u.s, u.t);
  u.parts = (gqa_blocks(end) - 1) / chunk + 1;
  u.slot = u.hk * n + base + (u.s.tiles - 1 - u.t) * most;
  const long long lo = (long long)u.part * chunk * kGqaBlock, hi = lo + (long long)chunk * kGqaBlock;
  u.lo = lo < end ? (int)lo : end;
  u.hi = hi < end ? (int)hi : end;
  if (p.target > 0 && tid == 0)
    records[u.slot + u.part] = GqaRecord{u.part == 0 ? u.parts : 0, u.s.s0, u.s.used, u.s.rows, u.t, u.hk, {0, 0}};
  return u.part < u.parts;
}

// A read that the scalar unit makes where the address is the same for the whole wave.
__device__ __forceinline__ int scalar_load(const int* p, size_t i) {
  return reinterpret_cast<const __attribute__((address_space(4))) int*>(reinterpret_cast<uintptr_t>(p))[i];
}

// What a row sees: the keys before `lim`, and of those from `past` on (the rows of
// the call), with SEER_MASK_TREE, the ones whose bits are set.
template <bool PAGED>
struct GqaSight {
  int lim, past;
  const unsigned long long* bits;      // null but for SEER_MASK_TREE
  int words;

  __device__ __forceinline__ GqaSight(const GqaParams& p, const GqaUnit& u, int tok) {
    past = u.s.past;
    lim = u.hi;
    if (p.mask == kMaskCausal && past + tok + 1 < lim) lim = past + tok + 1;
    words = p.words;
    bits = PAGED && p.mask == kMaskTree ? p.bits + (size_t)(u.s.s0 + tok) * p.words : nullptr;
  }
  // bit i: key k0 + i, i < 64
  __device__ __forceinline__ unsigned long long seen(int k0) const {
    const int n = lim - k0;
    unsigned long long m = n >= 64 ? ~0ull : (n > 0 ? (1ull << n) - 1 : 0);
    if (PAGED && bits) {
      const int j = k0 - past;                       // the row of the call that key k0 is
      if (j > -64) {
        auto word = [&](int w) { return w < words ? bits[w] : 0ull; };
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
};

// The first key from which on some row of the unit at token `tok` or later may be
// blind to one.
__device__ __forceinline__ int gqa_open_end(const GqaParams& p, const GqaUnit& u, int tok) {
  const int end = p.mask == kMaskCausal ? u.s.past + tok + 1 : (p.mask == kMaskTree ? u.s.past : u.hi);
  return end < u.hi ? end : u.hi;
}

}  // namespace seer
