// Eviction from the cache by accumulated attention weight.  Of the L places of a
// request, N are kept: protected tokens before the others, of either kind those with
// the larger weight, of equal ones those in lower places.  The places below N that
// are given up are filled with the kept tokens from N on, the i-th with the i-th, so
// that no more rows move than have to; where they come from and where they go never
// overlap, so all move at once.
//
// A list is what one head keeps of a request, or all of them together.  A workgroup
// reads a list's marks once, into registers, finds the order of the last token that
// stays by histograms of 11, 11 and 10 bits, and ranks what moves by ballots.
//
// Bound by the latency of one list's steps where little moves, by bytes where much does.
// Measured (MI355X, us): 96 requests, 8 heads, 700 to 1500 tokens, one of each evicted 12.5
// (a launch is 5); 24 prompts of 1500 to 16,000 tokens, 4 heads, cut to 1024 41, of which the
// choice 21 and the move of 78 MB 15 (5.2 TB/s); 16 prefixes of 32 heads, shared choice, 44, of
// which the choice 9 and the move of 105 MB 25 (4.2 TB/s).  Of the 21 us, by the
// clocks of a list of 16,000, its marks take about 5, the histograms 4.5, what stays 1.5.
// Where all weights are equal, as in a cache that was never weighed, every place falls in one bin: 96
// lists of 1400 then take 10.5 instead of 7 of a choice that moves nothing, longer ones no more than others.
#include "common.h"
#include "dispatch.h"
#include "kernels.h"

namespace seer {

namespace {

// Whole numbers in the order of the weights: -inf lowest, the two zeros equal, NaN above all.
__device__ __forceinline__ uint32_t order_of(float w) {
  if (!(w == w)) return 0xffffffffu;
  const uint32_t u = __float_as_uint(w + 0.0f);        // -0 + 0 is +0
  return u & 0x80000000u ? ~u : u | 0x80000000u;
}

struct Request {
  int L, N, seen;
  int kept;              // N, or -1 - N where other layers keep another number
  bool refused;          // the plan was: no tokens then, and kept stays
  const int* table;
};

__device__ __forceinline__ Request request(const EvictParams& p, int b) {
  Request r;
  const long long most = (long long)p.width << p.shift;
  const int L = p.kv_len[b];
  r.seen = p.seen[b];                            // on its way with the others
  const int others = p.alike ? p.kept[b] : 0, least = others < 0 ? -1 - others : others;
  const int N = p.budget ? p.budget[b] : least;
  r.refused = p.status && *p.status != 0;
  r.L = L < 0 || r.refused ? 0 : (L > most ? (int)most : L);
  r.N = r.kept = N < 0 ? 0 : (N < r.L ? N : r.L);
  if (p.alike) {
    // (who reads what another workgroup of the request has written already finds the same N)
    r.N = r.N < least ? r.N : least;
    r.kept = r.kept == others ? others : -1 - r.N;
  }
  r.table = p.table + (size_t)b * p.width;
  return r;
}

// The slot of place j in the pool; -1 on a page that is none of it.
__device__ __forceinline__ int slot_of(const EvictParams& p, const Request& r, int j) {
  const int id = r.table[j >> p.shift];
  return id < 0 || id >= p.n_pages ? -1 : (id << p.shift) + (j & ((1 << p.shift) - 1));
}
// Where a slot's marks for head h are.
__device__ __forceinline__ long long mark_of(const EvictParams& p, int slot, int h) {
  // (pages times heads stay below 2^31)
  return ((long long)((slot >> p.shift) * p.n_kv + h) << p.shift) + (slot & ((1 << p.shift) - 1));
}

struct Mark {
  float w;               // the head's weight, or the heads' sum
  int number, slot;
};

__device__ __forceinline__ Mark look(const EvictParams& p, const Request& r, int h, int j) {
  Mark m{0.0f, 0, slot_of(p, r, j)};
  if (m.slot < 0) return m;
  const long long at = mark_of(p, m.slot, h);
  if (p.shared) {
    double sum = 0.0;
    int i = 0;
    for (; i + 8 <= p.n_kv; i += 8) {
      float w[8];                                // on their way together
#pragma unroll
      for (int e = 0; e < 8; ++e) w[e] = p.weight[at + ((long long)(i + e) << p.shift)];
#pragma unroll
      for (int e = 0; e < 8; ++e) sum += (double)w[e];
    }
    for (; i < p.n_kv; ++i) sum += (double)p.weight[at + ((long long)i << p.shift)];
    m.w = (float)sum;
  } else {
    m.w = p.weight[at];
  }
  m.number = p.number[at];
  return m;
}

// Order and kind of a place: without a page lighter than any weight, and not protected.
__device__ __forceinline__ uint32_t order_of(const Mark& m) { return m.slot < 0 ? 0u : order_of(m.w); }
__device__ __forceinline__ bool guarded(const EvictParams& p, const Mark& m, int seen) {
  return m.slot >= 0 && (m.number < p.first || (long long)m.number >= (long long)seen - p.recent);
}

template <int NT>
struct Shared {
  static constexpr int NW = NT / kWave;
  uint32_t hist[3][2048];
  int part[NW];
  int guarded, digit, left, moving;
};

// The `left` largest members of a kind stay: those above the order that is returned, and
// the first `left` (now) of those with exactly it; -1: all of those, or of those that share
// the bits that were looked at.  each(f) calls f(order) for the thread's members.
template <int NT, typename Each>
__device__ __forceinline__ uint32_t threshold(Shared<NT>& sh, int& left, Each each) {
  constexpr int PER = 2048 / NT, NW = NT / kWave;
  const int tid = threadIdx.x, lane = tid & (kWave - 1), wave = tid >> 6;
  uint32_t prefix = 0, mask = 0;
#pragma unroll 1
  for (int pass = 0; pass < 3; ++pass) {
    const int shift = pass == 0 ? 21 : (pass == 1 ? 10 : 0), bins = pass == 2 ? 1024 : 2048;
    uint32_t* hist = sh.hist[pass];
    each([&](uint32_t key) {
      // the largest first
      if ((key & mask) == prefix) atomicAdd(&hist[bins - 1 - (key >> shift & (bins - 1))], 1u);
    });
    __syncthreads();
    int n[PER], own = 0;
#pragma unroll
    for (int i = 0; i < PER; ++i) {
      n[i] = hist[tid * PER + i];
      own += n[i];
    }
    const int inc = wave_scan(own);
    if (lane == kWave - 1) sh.part[wave] = inc;
    __syncthreads();
    int before = inc - own;
#pragma unroll
    for (int w = 0; w < NW; ++w)
      if (w < wave) before += sh.part[w];
    if (before < left && left <= before + own) {
      int need = left - before, d = 0;
#pragma unroll
      for (int i = 0; i < PER - 1; ++i)
        if (d == i && need > n[i]) { need -= n[i]; d = i + 1; }
      int same = n[0];
#pragma unroll
      for (int i = 1; i < PER; ++i) same = d == i ? n[i] : same;
      sh.digit = bins - 1 - (tid * PER + d);
      sh.left = need == same ? -1 : need;
    }
    __syncthreads();
    prefix |= (uint32_t)sh.digit << shift;
    mask |= (uint32_t)(bins - 1) << shift;
    left = sh.left;
    if (left < 0) break;                         // the whole bin stays
  }
  return prefix;
}

// A move's K and V rows and marks: pieces [i, end) of those of n moves of `heads` heads
// from h0 on, 16 bytes each, in steps.
__device__ __forceinline__ void move_rows(const EvictParams& p, const int* from, const int* to, int n, int h0, int heads,
                                          long long first, long long step) {
  const int pieces = 2 * p.head_pieces;
  const size_t row = (size_t)p.head_pieces * 16;
  const long long page = (long long)p.n_kv << p.shift;
  for (long long i = first; i < (long long)n * heads * pieces; i += step) {
    const int mh = (int)(i / pieces), c = (int)(i - (long long)mh * pieces);
    const int m = mh / heads, h = h0 + mh - m * heads;
    const int src = from[m], dst = to[m];
    if (src < 0 || dst < 0) continue;
    const long long s = mark_of(p, src, h), d = mark_of(p, dst, h);
    // K of a page lies before its V
    const int v = c >= p.head_pieces, piece = v ? c - p.head_pieces : c;
    const long long sr = s + (src >> p.shift) * page + v * page, dr = d + (dst >> p.shift) * page + v * page;
    *reinterpret_cast<u32x4_t*>(p.pool + dr * row + piece * 16) =
        *reinterpret_cast<const u32x4_t*>(p.pool + sr * row + piece * 16);
    if (c == 0) {
      const float w = p.weight[s];
      const int number = p.number[s];
      p.weight_out[d] = w;
      p.number_out[d] = number;
    }
  }
}

}  // namespace

// Lanes whose place, `first` and the lane's number, lies before `end`.
__device__ __forceinline__ unsigned long long before(int end, int first) {
  const int n = end - first;
  return n <= 0 ? 0ull : (n >= kWave ? ~0ull : (1ull << n) - 1);
}

// A list of at most NT * K places, place k * NT + tid a thread's k-th.  p.fused: the workgroup
// moves its list's rows too; otherwise it leaves the slots of what moves, and of shared lists
// which places below N are given up, for evict_move_kernel.  All reads are on their way
// together (one after the other they took 8 of 23 us of a list of 16 per thread); what stays
// and moves is held as a bit a place, 64 places in two scalar registers.
// counts [K][NT / 64]: of what moves, per 64 places, then their sums before; from [NT * K]:
// slots of what moves, and in its second half those where it goes.
template <int NT, int K>
__device__ __forceinline__ void evict_list(const EvictParams& p, const Request& r, int b, int h, Shared<NT>& sh, int* counts,
                                           int* from) {
  constexpr int NW = NT / kWave, MOST = NT * K / 2;
  typedef unsigned long long bits_t;
  const int tid = threadIdx.x, lane = tid & (kWave - 1), wave = __builtin_amdgcn_readfirstlane(tid >> 6);
  const int seen = r.seen;
  const auto start = [&](int k) { return k * NT + wave * kWave; };         // the wave's first place of the k-th
  int slot[K];
#pragma unroll
  for (int k = 0; k < K; ++k) slot[k] = slot_of(p, r, k * NT + tid < r.L ? k * NT + tid : 0);
  for (int i = tid; i < 3 * 2048; i += NT) (&sh.hist[0][0])[i] = 0;
  if (tid == 0) sh.guarded = 0;
  uint32_t order[K];
  uint32_t kinds = 0;                            // bit k: the k-th place is protected
  {
    // of a place without a page the first slot's marks, which are not looked at
    auto at = [&](int k) { return mark_of(p, slot[k] < 0 ? 0 : slot[k], h); };
    auto take = [&](int k, float w, int number) {
      const Mark m{w, number, slot[k]};
      order[k] = order_of(m);
      kinds |= (uint32_t)(k * NT + tid < r.L && guarded(p, m, seen)) << k;
    };
    constexpr int A = K <= 8 ? K : 8;            // places on their way together
    if (!p.shared) {
#pragma unroll
      for (int k0 = 0; k0 < K; k0 += A) {
        float w[A];
        int number[A];
#pragma unroll
        for (int k = 0; k < A; ++k) {
          const long long mark = at(k0 + k);
          w[k] = p.weight[mark];
          number[k] = p.number[mark];
        }
#pragma unroll
        for (int k = 0; k < A; ++k) take(k0 + k, w[k], number[k]);
      }
    } else {
      constexpr int G = 16 / A;                  // and heads of each
#pragma unroll
      for (int k0 = 0; k0 < K; k0 += A) {
        double sum[A];
        long long mark[A];
        int number[A];
#pragma unroll
        for (int k = 0; k < A; ++k) {
          mark[k] = at(k0 + k);
          number[k] = p.number[mark[k]];
          sum[k] = 0.0;
        }
        int i = 0;
        for (; i + G <= p.n_kv; i += G) {
          float x[A][G];
#pragma unroll
          for (int k = 0; k < A; ++k)
#pragma unroll
            for (int e = 0; e < G; ++e) x[k][e] = p.weight[mark[k] + ((long long)(i + e) << p.shift)];
#pragma unroll
          for (int k = 0; k < A; ++k)
#pragma unroll
            for (int e = 0; e < G; ++e) sum[k] += (double)x[k][e];
        }
        for (; i < p.n_kv; ++i)
#pragma unroll
          for (int k = 0; k < A; ++k) sum[k] += (double)p.weight[mark[k] + ((long long)i << p.shift)];
#pragma unroll
        for (int k = 0; k < A; ++k) take(k0 + k, (float)sum[k], number[k]);
      }
    }
  }
  __syncthreads();
  int mine = 0;
#pragma unroll
  for (int k = 0; k < K; ++k) mine += __popcll(__ballot(kinds >> k & 1));
  if (lane == 0 && mine) atomicAdd(&sh.guarded, mine);
  __syncthreads();
  // the kind of which some stay, and how many of them
  const int guarded_all = sh.guarded;
  const bool of_guarded = guarded_all >= r.N;
  const int members = of_guarded ? guarded_all : r.L - guarded_all;
  int left = of_guarded ? r.N : r.N - guarded_all;
  const bool some = left > 0 && left < members;
  // members above the least order stay, and with `equal` those with exactly it
  uint32_t least = left > 0 ? 0u : 0xffffffffu;
  bool equal = left > 0;
  if (some) {
    least = threshold<NT>(sh, left, [&](auto f) {
#pragma unroll
      for (int k = 0; k < K; ++k)
        if (k * NT + tid < r.L && (kinds >> k & 1) == of_guarded) f(order[k]);
    });
    equal = left < 0;
  }
  // which stay
  bits_t stays[K];
#pragma unroll
  for (int k = 0; k < K; ++k) {
    const bits_t in = before(r.L, start(k)), kind = __ballot(kinds >> k & 1);
    const bits_t member = of_guarded ? kind : in & ~kind;
    const bits_t above = __ballot(order[k] > least) | (equal ? __ballot(order[k] == least) : 0ull);
    stays[k] = (member & above) | (of_guarded ? 0ull : kind);
  }
  // ranks in the order of the places: counts of each 64, their sums, and the bits before
  auto rank = [&](auto set, auto use) {
    int own = 0;
#pragma unroll
    for (int k = 0; k < K; ++k) {
      const int n = __popcll(set(k));            // (all lanes' ballots, before one lane takes it)
      own = lane == k ? n : own;
    }
    __syncthreads();
    if (lane < K) counts[lane * NW + wave] = own;
    __syncthreads();
    if (wave == 0) {
      int* c = counts;
      int base = 0;
#pragma unroll
      for (int i = 0; i < K * NW; i += kWave) {
        const int n = i + lane < K * NW ? c[i + lane] : 0;
        const int inc = wave_scan(n);
        if (i + lane < K * NW) c[i + lane] = base + inc - n;
        base += __builtin_amdgcn_readlane(inc, kWave - 1);
      }
      if (lane == 0) sh.moving = base;
    }
    __syncthreads();
    const int first = counts[(lane < K ? lane : 0) * NW + wave], all = sh.moving;
#pragma unroll
    for (int k = 0; k < K; ++k) {
      const bits_t bits = set(k);
      if (bits)
        use(k, bits >> lane & 1, __builtin_amdgcn_mbcnt_hi((uint32_t)(bits >> 32), __builtin_amdgcn_mbcnt_lo(
                                     (uint32_t)bits, __builtin_amdgcn_readlane(first, k))), all);
    }
  };
  if (some && left > 0) {
    // of the places with exactly the least order, the first `left`
    auto ties = [&](int k) {
      const bits_t kind = __ballot(kinds >> k & 1);
      return __ballot(order[k] == least) & (of_guarded ? kind : before(r.L, start(k)) & ~kind);
    };
    rank(ties, [&](int k, bool is, int at, int) { stays[k] |= __ballot(is && at < left); });
  }
  // places below N that are given up, and kept ones from N on: as many of either
  auto moves = [&](int k) { return (stays[k] ^ before(r.N, start(k))) & before(r.L, start(k)); };
  // the first half of the ranks are those of places below N
  rank(moves, [&](int k, bool is, int at, int all) {
    if (is) from[at < all / 2 ? MOST + at : at - all / 2] = slot[k];
  });
  const int n = sh.moving / 2;
  if (p.weight_out != p.weight) {
    if (!p.shared) {
      // marks that stay where they are, in another pool (read again: held, they would cost registers)
#pragma unroll
      for (int k = 0; k < K; ++k)
        if ((stays[k] & before(r.N, start(k))) >> lane & 1 && slot[k] >= 0) {
          const long long at = mark_of(p, slot[k], h);
          p.weight_out[at] = p.weight[at];
          p.number_out[at] = p.number[at];
        }
    } else {
      unsigned long long* gone_bits = p.bits + (size_t)blockIdx.x * (p.room / 32);
#pragma unroll
      for (int k = 0; k < K; ++k)
        if (lane == 0 && start(k) < r.N) gone_bits[(k * NT >> 6) + wave] = ~stays[k];
    }
  }
  if (tid == 0) {
    if (h == 0 && !r.refused) p.kept[b] = r.kept;
    if (!p.fused) p.counts[blockIdx.x] = n;
  }
  __syncthreads();
  if (p.fused) {
    if (n > 0) move_rows(p, from, from + MOST, n, h, 1, tid, NT);
  } else {
    int* moves = p.moves + (size_t)blockIdx.x * 2 * p.room;
    for (int i = tid; i < n; i += NT) {
      moves[i] = from[i];
      moves[p.room + i] = from[MOST + i];
    }
  }
}

// Lists of at most NT * K places; short ones among them, as in a table that is wider than the
// requests are long, take the steps of theirs.
template <int NT, int K>
__global__ __launch_bounds__(NT) void evict_kernel(EvictParams p) {
  __shared__ Shared<NT> sh;
  __shared__ int counts[K * NT / kWave], from[NT * K];
  const int b = blockIdx.x / p.lists, h = blockIdx.x % p.lists;
  const Request r = request(p, b);
  constexpr int SHORT = 2048 / NT;
  if constexpr (K > SHORT) {
    if (r.L <= NT * SHORT) {
      evict_list<NT, SHORT>(p, r, b, h, sh, counts, from);
      return;
    }
  }
  evict_list<NT, K>(p, r, b, h, sh, counts, from);
}

// Lists of any length; the marks of those of more than 8192 places are read again for each
// histogram.
__global__ __launch_bounds__(1024) void evict_long_kernel(EvictParams p) {
  constexpr int NT = 1024, NW = NT / kWave, K = 8;
  __shared__ Shared<NT> sh;
  __shared__ int part[3][NW];
  __shared__ int counts[K * NW], from_lds[NT * K];
  const int tid = threadIdx.x, lane = tid & (kWave - 1), wave = tid >> 6;
  const int b = blockIdx.x / p.lists, h = blockIdx.x % p.lists;
  const Request r = request(p, b);
  if (r.L <= 2 * NT) {
    evict_list<NT, 2>(p, r, b, h, sh, counts, from_lds);
    return;
  }
  if (r.L <= K * NT) {
    evict_list<NT, K>(p, r, b, h, sh, counts, from_lds);
    return;
  }
  const int seen = r.seen;
  for (int i = tid; i < 3 * 2048; i += NT) (&sh.hist[0][0])[i] = 0;
  if (tid == 0) sh.guarded = 0;
  __syncthreads();
  int mine = 0;
  for (int j = tid; j < r.L; j += NT) mine += guarded(p, look(p, r, h, j), seen);
  if (mine) atomicAdd(&sh.guarded, mine);
  __syncthreads();
  const int guarded_all = sh.guarded;
  const bool of_guarded = guarded_all >= r.N;
  const int members = of_guarded ? guarded_all : r.L - guarded_all;
  int left = of_guarded ? r.N : r.N - guarded_all;
  const bool some = left > 0 && left < members;
  uint32_t least = 0;
  if (some)
    least = threshold<NT>(sh, left, [&](auto f) {
      for (int j = tid; j < r.L; j += NT) {
        const Mark m = look(p, r, h, j);
        if (guarded(p, m, seen) == of_guarded) f(order_of(m));
      }
    });
  int* from = p.moves + (size_t)blockIdx.x * 2 * p.room;
  int* to = from + p.room;
  unsigned long long* gone_bits = p.bits + (size_t)blockIdx.x * (p.room / 32);
  int ties = 0, holes = 0, sources = 0;          // before this stretch of places
  for (int j0 = 0; j0 < r.L; j0 += NT) {
    const int j = j0 + tid;
    Mark m{0.0f, 0, -1};
    bool tie = false, stays = false;
    if (j < r.L) {
      m = look(p, r, h, j);
      if (guarded(p, m, seen) != of_guarded) stays = !of_guarded;
      else if (!some) stays = left > 0;
      else {
        const uint32_t order = order_of(m);
        tie = left > 0 && order == least;
        stays = order > least || (left < 0 && order == least);
      }
    }
    auto rank = [&](bool is, int k, int& total) {
      const unsigned long long set = __ballot(is);
      if (lane == 0) part[k][wave] = __popcll(set);
      __syncthreads();
      int before = 0;
      total = 0;
      for (int w = 0; w < NW; ++w) {
        const int n = part[k][w];
        if (w < wave) before += n;
        total += n;
      }
      return before + __popcll(set & ((1ull << lane) - 1));
    };
    int all;
    const int tie_at = ties + rank(tie, 0, all);
    ties += all;
    if (tie) stays = tie_at < left;
    const bool hole = j < r.N && !stays, source = j >= r.N && stays;
    const int hole_at = holes + rank(hole, 1, all);
    holes += all;
    const int source_at = sources + rank(source, 2, all);
    sources += all;
    if (hole) to[hole_at] = m.slot;
    if (source) from[source_at] = m.slot;
    if (p.weight_out != p.weight) {
      if (!p.shared) {
        if (j < r.N && stays && m.slot >= 0) {
          const long long at = mark_of(p, m.slot, h);
          p.weight_out[at] = m.w;
          p.number_out[at] = m.number;
        }
      } else {
        const unsigned long long set = __ballot(!stays);
        if (lane == 0 && j < r.N) gone_bits[j >> 6] = set;
      }
    }
    __syncthreads();
  }
  if (tid == 0) {
    p.counts[blockIdx.x] = sources;
    if (h == 0) p.kept[b] = r.kept;              // (a refused plan's lists are short ones)
  }
}

// The moves of all lists, p.parts workgroups each, and of shared lists the marks that
// stay where they are, in another pool.
__global__ __launch_bounds__(256) void evict_move_kernel(EvictParams p) {
  const int list = blockIdx.x / p.parts, part = blockIdx.x % p.parts;
  const int h0 = p.shared ? 0 : list % p.lists, heads = p.shared ? p.n_kv : 1;
  const int* from = p.moves + (size_t)list * 2 * p.room;
  const long long first = (long long)part * 256 + threadIdx.x, step = 256ll * p.parts;
  move_rows(p, from, from + p.room, p.counts[list], h0, heads, first, step);
  if (!p.shared || p.weight_out == p.weight) return;
  const Request r = request(p, list);
  const unsigned long long* gone = p.bits + (size_t)list * (p.room / 32);
  for (long long i = first; i < (long long)r.N * heads; i += step) {
    const int h = (int)(i / r.N), j = (int)(i - (long long)h * r.N);
    const int slot = slot_of(p, r, j);
    if (slot < 0 || (gone[j >> 6] >> (j & 63) & 1)) continue;
    const long long at = mark_of(p, slot, h);
    p.weight_out[at] = p.weight[at];
    p.number_out[at] = p.number[at];
  }
}

int launch_evict(const EvictParams& p, const EvictRule& r, hipStream_t s) {
  const dim3 grid(p.B * p.lists);
  if (r.places == 2048 && r.few) hipLaunchKernelGGL((evict_kernel<1024, 2>), grid, dim3(1024), 0, s, p);
  else if (r.places == 2048) hipLaunchKernelGGL((evict_kernel<256, 8>), grid, dim3(256), 0, s, p);
  else if (r.places == 8192 && r.few) hipLaunchKernelGGL((evict_kernel<1024, 8>), grid, dim3(1024), 0, s, p);
  else if (r.places == 8192) hipLaunchKernelGGL((evict_kernel<512, 16>), grid, dim3(512), 0, s, p);
  else if (r.places == 16384) hipLaunchKernelGGL((evict_kernel<1024, 16>), grid, dim3(1024), 0, s, p);
  else hipLaunchKernelGGL(evict_long_kernel, grid, dim3(1024), 0, s, p);
  if (!p.fused) hipLaunchKernelGGL(evict_move_kernel, dim3(p.B * p.lists * p.parts), dim3(256), 0, s, p);
  return hipGetLastError() == hipSuccess ? 0 : -1;
}

}  // namespace seer
