// What the kernels of the attention with grouped heads share: how the work of a
// launch is cut, and which keys a row sees.
#pragma once

#include <limits.h>
#include <math.h>

#include "common.h"
#include "dispatch.h"
#include "kernels.h"

namespace seer {

// Keys are cut at multiples of this.
constexpr int kGqaBlock = 64;

// Rows of a key/value head are (token, query head of its group) pairs, the head
// fastest: row i is token i / G, head i % G.  A tile is RT such rows, so K and V
// are read once for all the query heads that share them, whatever G is.

// x / group without a division (gqa_divisor).
__device__ __forceinline__ int gqa_token(const GqaParams& p, int x) {
  return (int)((__umulhi((unsigned)x, p.group_mul) + (unsigned)x) >> p.group_shift);
}

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
    s.nk = gqa_keys(p.kv_len[b], p.width, p.shift);
  } else {
    s.nk = s.used;
  }
  s.past = s.nk - s.used;
  s.rows = s.len * p.group;
  s.tiles = (s.rows + RT - 1) / RT;
  return s;
}

__device__ __forceinline__ int gqa_blocks(int nk) { return nk > kGqaBlock ? (nk - 1) / kGqaBlock + 1 : 1; }

// The keys that any row of tile t sees end here.
template <int RT>
__device__ __forceinline__ int gqa_tile_end(const GqaParams& p, const GqaSeq& s, int t) {
  if (s.used == 0) return 0;
  if (p.mask != kMaskCausal) return s.nk;
  int last = gqa_token(p, (t + 1) * RT - 1);               // last token of the tile
  last = last < s.used ? last : s.used - 1;
  const int end = s.past + last + 1;
  return end < 0 ? 0 : (end < s.nk ? end : s.nk);
}

// A piece of work: keys [lo, hi) for tile t of request b and key/value head hk;
// all that the tile's rows see (whole), or a part whose result goes to `slot`.
struct GqaUnit {
  int b, t, hk, lo, hi, slot;
  bool whole;
  GqaSeq s;
};

// What the joining of a tile's parts has to know: the first part lies in slot
// `first`, the others in the even slots of the workgroups after it.  One for each
// workgroup, by the one that has the tile's first key (parts < 2: nothing to join).
struct GqaRecord {
  int parts, first, s0, used, rows, t, hk, pad;
};

// How the work of a launch is cut.
//   p.cut:     every tile's keys count as blocks of 64, the blocks of all heads,
//              requests and tiles stand in one line, and each of the p.wgs workgroups
//              takes an equal stretch of it, whatever the requests' lengths: no
//              workgroup waits for another, and none starts after the others.  A tile
//              that lies in several stretches is joined by a second launch.  With few
//              tiles the places of the line are runs of several blocks (below).
//   otherwise: a workgroup for each tile, request after request (p.sort: the ones with
//              the most keys first, so that no long walk starts at the end: sixteen
//              prompts of 200 to 1300 rows 142 -> 135 us), in each all heads, in each the
//              tiles from the last, which sees the most, to the first.  An XCD has heads
//              of its own where their number allows it, so that a head's keys are in one L2.
// Every workgroup sums the requests' lengths for itself (each thread its share of
// the requests, then a scan); with at most one request a thread they are read once.
template <int RT, int NT>
struct GqaCut {
  static constexpr int NW = NT / kWave;
  struct Shared {
    int sums[NW];
    int first[NT + 1];           // of each thread's stretch of a head's line
    GqaSeq seq[NT];              // of each thread's only request, and its index
    int id[NT];
  };
  Shared& sh;
  int run;                       // cut: blocks of a place of the line
  int n, all;                    // length of a head's line, and of the whole
  int wgs, each, more;           // workgroups with work: `more` of them take each + 1, the others each
  int x, x0, x1;                 // the next place, and the workgroup's stretch
  int wg;
  int heads, head0;              // uncut: the heads of this workgroup's XCD

  // places of a tile of request s
  __device__ __forceinline__ int places(const GqaParams& p, const GqaSeq& s) const {
    if (!p.cut) return 1;
    const int nb = gqa_blocks(s.nk);
    return run == 1 ? nb : (int)((unsigned)(nb + run - 1) / (unsigned)run);
  }
  __device__ __forceinline__ int weight(const GqaParams& p, const GqaSeq& s) const { return s.tiles * places(p, s); }
  __device__ __forceinline__ int start(int i) const { return i * each + (i < more ? i : more); }
  // the workgroup that has place y
  __device__ __forceinline__ int holder(int y) const {
    const int head = more * (each + 1);
    return y < head ? (int)((unsigned)y / (unsigned)(each + 1)) : more + (int)((unsigned)(y - head) / (unsigned)each);
  }

  // How many workgroups share a line of `all` blocks.  Each of them costs its start,
  // the reads of its queries and up to two parts (66 KB each of 128 rows by 128) written
  // and joined, so a short line goes to one workgroup a CU instead of all that run at
  // once: 128 rows at 1280 blocks 29.7 -> 21.7 us, at 1736 33.1 -> 30.1, at 2720 38.1 ->
  // 35.9, at 3392 40.7 -> 46.4; 32 rows at 600 blocks 21.0 -> 15.2, at 1280 25.3 -> 21.5,
  // at 2008 26.0 -> 30.2; 32 rows 64 wide with 512 for 1024 at 2576 blocks 26.4 -> 22.5,
  // at 5672 25.0 -> 28.9.
  __device__ __forceinline__ static int workgroups(int most, int all) {
    if (RT == kGqaF32) return most;
    if (all < (RT == kGqaTile ? 2800 : 1300)) return most < 256 ? most : 256;
    return all < 5000 && most > 512 ? 512 : most;
  }

  // The line: the sums of the threads' places before each of them, and of all.
  __device__ __forceinline__ void scan(const GqaParams& p, int own) {
    const int tid = threadIdx.x, lane = tid & (kWave - 1), wave = tid >> 6;
    int inc = own;
#pragma unroll
    for (int off = 1; off < kWave; off <<= 1) {
      const int v = __shfl_up(inc, off, kWave);
      if (lane >= off) inc += v;
    }
    if (lane == kWave - 1) sh.sums[wave] = inc;
    __syncthreads();
    int first = inc - own;
    n = 0;
#pragma unroll
    for (int w = 0; w < NW; ++w) {
      if (w < wave) first += sh.sums[w];
      n += sh.sums[w];
    }
    n = __builtin_amdgcn_readfirstlane(n);
    sh.first[tid] = first;
    if (tid == NT - 1) sh.first[NT] = n;
    all = n * p.n_kv;
  }

  __device__ __forceinline__ GqaCut(const GqaParams& p, Shared& shared) : sh(shared), run(1) {
    const int tid = threadIdx.x, lane = tid & (kWave - 1), wave = tid >> 6;
    const int per = (p.B + NT - 1) / NT;
    const int b0 = tid * per < p.B ? tid * per : p.B;
    const int b1 = b0 + per < p.B ? b0 + per : p.B;
    int own = 0;
    if (per == 1) {
      GqaSeq s{};
      if (tid < p.B) s = gqa_seq<RT>(p, tid);
      own = weight(p, s);
      int at = tid;
      if (p.sort && wave == 0) {
        // the request's rank by its keys
        int rank = 0;
        for (int k = 0; k < p.B; ++k) {
          const int nk = __builtin_amdgcn_readlane(s.nk, k);
          rank += nk > s.nk || (nk == s.nk && k < lane);
        }
        if (tid < p.B) at = rank;
        own = __builtin_amdgcn_ds_permute(at * 4, own);
      }
      sh.seq[at] = s;
      sh.id[at] = tid;
    } else {
      for (int b = b0; b < b1; ++b) own += weight(p, gqa_seq<RT>(p, b));
    }
    scan(p, own);
    const int most = p.cut ? workgroups(p.wgs, all) : all;
    // Few tiles: an equal stretch that crosses from one tile to the next makes two
    // pieces, one after the other, and the launch waits for it (5 us, what 2 blocks take
    // in fp32 and 3 to 4 in bf16).  So a tile's blocks are taken in runs of one length,
    // a run a workgroup: the least that is not below an equal stretch, or, if those are
    // more runs than workgroups, the length that leaves room for each tile's odd one,
    // while it is not too much above an equal stretch.  One token, 32 heads on 8: 3000
    // keys 26.3 -> 19.7 us, 6000 26.6 -> 22.2; 4 tokens of 16 heads on 1 at 4000 keys 26.0 ->
    // 19.2; fp32, 4 tokens of 8 heads on 2 at 4000 keys 28.9 -> 21.7.  Runs twice the equal
    // stretch: 8 tokens of 32 heads on 32 at 4000 keys 64.9 -> 77.6.
    if (p.cut && gqa_in_runs(all, most, p.tiles)) {
      const int blocks = all, fair = ((unsigned)blocks + most - 1) / (unsigned)most;
      auto lay = [&](int r) {
        run = r;
        own = 0;
        if (per == 1) own = weight(p, sh.seq[tid]);
        else
          for (int b = b0; b < b1; ++b) own += weight(p, gqa_seq<RT>(p, b));
        __syncthreads();
        scan(p, own);
      };
      lay(fair);
      if (all > most) {
        const int room = gqa_run_room(blocks, most, p.tiles);
        lay(room <= fair + (RT == kGqaF32 ? 1 : 2) ? room : 1);
      }
    }
    const int bid = blockIdx.x;
    wg = 0;
    wgs = all;
    each = 1;
    more = 0;
    if (all > most) {
      wgs = most;
      each = (unsigned)all / (unsigned)wgs;
      more = all - each * wgs;
    }
    x0 = x1 = 0;
    heads = p.n_kv;
    head0 = 0;
    if (!p.cut) {
      int i = bid;
      if (p.n_kv % 8 == 0) {
        heads = p.n_kv / 8;
        head0 = (bid & 7) * heads;
        i = bid >> 3;
      }
      x0 = i;
      x1 = i < n * heads ? i + 1 : i;
    } else if (bid < wgs) {
      // each XCD takes a contiguous part of the line: the tiles of one request and
      // head find their keys in its L2
      wg = xcd_remap(bid, wgs);
      x0 = start(wg);
      x1 = start(wg + 1);
    } else if (tid == 0) {
      static_cast<GqaRecord*>(p.records)[bid].parts = 0;
    }
    x = x0;
  }

  // The next piece of the workgroup's stretch; false at its end.  Every wave looks
  // for itself.
  __device__ __forceinline__ bool next(const GqaParams& p, GqaUnit& u) {
    if (x >= x1) return false;
    const int lane = threadIdx.x & (kWave - 1);
    const int per = (p.B + NT - 1) / NT;
    // cut: head after head; otherwise: the requests' tiles times the heads
    const int q = (unsigned)x / (unsigned)(p.cut ? n : heads);
    const int j = p.cut ? x - q * n : q;
    __syncthreads();               // the line is written, and the last piece's reads of LDS are done
    int f = 0;                     // the thread whose stretch has place j
#pragma unroll
    for (int c = 0; c < NT; c += kWave) {
      const unsigned long long hit = __ballot(j >= sh.first[c + lane] && j < sh.first[c + lane + 1]);
      if (hit) f = c + __builtin_ctzll(hit);
    }
    int at = sh.first[f];
    u.b = f;
    GqaSeq s;
    if (per == 1) {
      s = sh.seq[f];
      u.b = sh.id[f];
    } else {
      // the thread's requests, one a lane
      for (int i0 = 0; i0 < per; i0 += kWave) {
        const int b = f * per + i0 + lane;
        GqaSeq mine{};
        if (i0 + lane < per && b < p.B) mine = gqa_seq<RT>(p, b);
        const int m = weight(p, mine);
        int inc = m;
#pragma unroll
        for (int off = 1; off < kWave; off <<= 1) {
          const int v = __shfl_up(inc, off, kWave);
          if (lane >= off) inc += v;
        }
        const unsigned long long hit = __ballot(j >= at + inc - m && j < at + inc);
        if (hit) {
          const int l = __builtin_ctzll(hit);
          auto of = [&](int v) { return __builtin_amdgcn_readlane(v, l); };
          u.b = f * per + i0 + l;
          at += of(inc - m);
          s.s0 = of(mine.s0); s.len = of(mine.len); s.used = of(mine.used); s.nk = of(mine.nk); s.past = of(mine.past);
          s.rows = of(mine.rows); s.tiles = of(mine.tiles);
          break;
        }
        at += __builtin_amdgcn_readlane(inc, kWave - 1);
      }
    }
    auto uni = [](int v) { return __builtin_amdgcn_readfirstlane(v); };
    u.b = uni(u.b);
    const int rem = uni(p.cut ? j - at : x - at * heads);
    u.s.tiles = uni(s.tiles); u.s.s0 = uni(s.s0); u.s.len = uni(s.len); u.s.used = uni(s.used); u.s.nk = uni(s.nk);
    u.s.past = uni(s.past); u.s.rows = uni(s.rows);
    const int nb = places(p, u.s), line = p.cut ? nb : u.s.tiles;
    const int quot = (unsigned)rem / (unsigned)line, left = rem - quot * line;
    u.hk = p.cut ? q : head0 + quot;
    const int tile = p.cut ? quot : left, block = p.cut ? left : 0;
    // the tiles of a causal prompt from the last, which has the most keys, to the first
    u.t = u.s.tiles - 1 - tile;
    const int end = gqa_tile_end<RT>(p, u.s, u.t);
    u.whole = true;
    u.lo = 0;
    u.hi = end;
    u.slot = 0;
    int take = 1;
    if (p.cut) {
      take = nb - block < x1 - x ? nb - block : x1 - x;
      u.whole = take == nb;
      const long long lo = (long long)block * run * kGqaBlock, hi = lo + (long long)take * run * kGqaBlock;
      u.lo = lo < end ? (int)lo : end;
      u.hi = hi < end ? (int)hi : end;
      u.slot = 2 * wg + (x == x0 ? 0 : 1);
      if (threadIdx.x == 0 && x + take >= x1) {
        // the last piece: where it opens a tile that goes on, the tile's record
        GqaRecord r{};
        if (block == 0 && take < nb)
          r = GqaRecord{holder(x + nb - 1) - wg + 1, u.slot, u.s.s0, u.s.used, u.s.rows, u.t, u.hk, 0};
        static_cast<GqaRecord*>(p.records)[wg] = r;
      }
    }
    x += take;
    return true;
  }
};

// The slot of part i of a record of workgroup wg.
__device__ __forceinline__ int gqa_slot(const GqaRecord& r, int wg, int i) { return i == 0 ? r.first : 2 * (wg + i); }

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
