// Eviction from the cache by accumulated attention weight.  Of the L places of a
// request, N are kept: protected tokens before the others, of either kind those with
// the larger weight, of equal ones those in lower places.  The places below N that
// are given up are filled with the kept tokens from N on, the i-th with the i-th, so
// that no more rows move than have to; where they come from and where they go never
// overlap, so all move at once.
#include "common.h"
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
  int L, N;
  const int* table;
};

__device__ __forceinline__ Request request(const EvictParams& p, int b) {
  Request r;
  const long long most = (long long)p.width << p.shift;
  const int L = p.kv_len[b], N = p.budget[b];
  r.L = L < 0 ? 0 : (L > most ? (int)most : L);
  r.N = N < 0 ? 0 : (N < r.L ? N : r.L);
  r.table = p.table + (size_t)b * p.width;
  return r;
}

// Index of head 0 of place j in the marks; -1 on a page that is none of the pool's.
__device__ __forceinline__ long long mark_of(const EvictParams& p, const Request& r, int j) {
  const int id = r.table[j >> p.shift];
  if (id < 0 || id >= p.n_pages) return -1;
  return (((long long)id * p.n_kv) << p.shift) + (j & ((1 << p.shift) - 1));
}

}  // namespace

constexpr int NT = 1024, NW = NT / kWave;

// What a request keeps, for one head or for all: a workgroup finds the weight of the
// last token that stays, eight bits of it at a time by their histogram, and lists the
// moves in the order of the places.
__global__ __launch_bounds__(NT) void evict_select_kernel(EvictParams p) {
  __shared__ uint32_t hist[256];
  __shared__ int part[4][NW];
  __shared__ uint32_t digit_lds;
  __shared__ int left_lds, guarded_lds;
  const int tid = threadIdx.x, lane = tid & (kWave - 1), wave = tid >> 6;
  const int b = blockIdx.x / p.lists, h = blockIdx.x % p.lists;
  const Request r = request(p, b);
  const int seen = p.seen[b];
  if (tid == 0) guarded_lds = 0;
  __syncthreads();

  // order and kind of place j
  auto look = [&](int j, uint32_t& key, bool& guarded) {
    const long long at = mark_of(p, r, j);
    key = 0;
    guarded = false;
    if (at < 0) return;
    const long long head = at + ((long long)h << p.shift);
    float w;
    if (p.shared) {
      double sum = 0.0;
      for (int i = 0; i < p.n_kv; ++i) sum += (double)p.weight[at + ((long long)i << p.shift)];
      w = (float)sum;
    } else {
      w = p.weight[head];
    }
    const int number = p.number[head];
    key = order_of(w);
    guarded = number < p.first || (long long)number >= (long long)seen - p.recent;
  };
  int mine = 0;
  for (int j = tid; j < r.L; j += NT) {
    uint32_t key;
    bool guarded;
    look(j, key, guarded);
    mine += guarded;
  }
  if (mine) atomicAdd(&guarded_lds, mine);
  __syncthreads();
  // the kind of which some stay, and how many of them
  const int guarded_all = guarded_lds;
  const bool of_guarded = guarded_all >= r.N;
  int left = of_guarded ? r.N : r.N - guarded_all;
  uint32_t prefix = 0, mask = 0;
  if (left > 0) {
    for (int shift = 24; shift >= 0; shift -= 8) {
      if (tid < 256) hist[tid] = 0;
      __syncthreads();
      for (int j = tid; j < r.L; j += NT) {
        uint32_t key;
        bool guarded;
        look(j, key, guarded);
        if (guarded == of_guarded && (key & mask) == prefix) atomicAdd(&hist[key >> shift & 255], 1u);
      }
      __syncthreads();
      if (tid == 0) {
        int n = left, d = 255;
        for (; d > 0 && (int)hist[d] < n; --d) n -= hist[d];
        digit_lds = d;
        left_lds = n;
      }
      __syncthreads();
      prefix |= digit_lds << shift;
      mask |= 255u << shift;
      left = left_lds;
      __syncthreads();
    }
  }
  // `left` of the places with exactly this order stay (none at all where left is 0)
  int* from = p.moves + (size_t)blockIdx.x * 2 * p.room;
  int* to = from + p.room;
  int ties = 0, holes = 0, sources = 0;          // before this stretch of places
  for (int j0 = 0; j0 < r.L; j0 += NT) {
    const int j = j0 + tid;
    uint32_t key = 0;
    bool guarded = false, tie = false, stays = false;
    if (j < r.L) {
      look(j, key, guarded);
      if (guarded != of_guarded) stays = guarded;
      else if (left > 0) {
        tie = key == prefix;
        stays = key > prefix;
      }
    }
    auto rank = [&](bool is, int k, int& total) {
      const unsigned long long m = __ballot(is);
      if (lane == 0) part[k][wave] = __popcll(m);
      __syncthreads();
      int before = 0;
      total = 0;
      for (int w = 0; w < NW; ++w) {
        const int n = part[k][w];
        if (w < wave) before += n;
        total += n;
      }
      return before + __popcll(m & ((1ull << lane) - 1));
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
    if (hole) to[hole_at] = j;
    if (source) from[source_at] = j;
    if (j < r.N && stays && p.weight_out != p.weight) {
      // marks that stay where they are, in another pool
      const long long at = mark_of(p, r, j);
      if (at >= 0)
        for (int i = 0; i < (p.shared ? p.n_kv : 1); ++i) {
          const long long m = at + ((long long)(p.shared ? i : h) << p.shift);
          p.weight_out[m] = p.weight[m];
          p.number_out[m] = p.number[m];
        }
    }
    __syncthreads();
  }
  if (tid == 0) {
    p.counts[blockIdx.x] = sources;
    if (h == 0) p.kept[b] = r.N;
  }
}

// The moves: a wave takes a token and head, its K, V and marks.
__global__ __launch_bounds__(256) void evict_move_kernel(EvictParams p) {
  const int lane = threadIdx.x & (kWave - 1), wave = threadIdx.x >> 6;
  const int list = blockIdx.x / p.parts, part = blockIdx.x % p.parts;
  const int b = list / p.lists, h0 = p.shared ? 0 : list % p.lists, heads = p.shared ? p.n_kv : 1;
  const Request r = request(p, b);
  const int n = p.counts[list];
  const int* from = p.moves + (size_t)list * 2 * p.room;
  const int* to = from + p.room;
  const size_t row = (size_t)p.head_pieces * 16;
  for (long long i = (long long)part * 4 + wave; i < (long long)n * heads; i += 4ll * p.parts) {
    const int m = (int)(i / heads), h = h0 + (int)(i - (long long)m * heads);
    const long long src = mark_of(p, r, from[m]), dst = mark_of(p, r, to[m]);
    if (src < 0 || dst < 0) continue;
    const long long s = src + ((long long)h << p.shift), d = dst + ((long long)h << p.shift);
    if (lane == 0) {
      const float w = p.weight[s];
      const int number = p.number[s];
      p.weight_out[d] = w;
      p.number_out[d] = number;
    }
    // K of a page lies before its V
    const long long page = (long long)p.n_kv << p.shift;
    const size_t sk = (size_t)(src / page * page + s), dk = (size_t)(dst / page * page + d);
    for (int c = lane; c < 2 * p.head_pieces; c += kWave) {
      const int v = c >= p.head_pieces, piece = v ? c - p.head_pieces : c;
      *reinterpret_cast<u32x4_t*>(p.pool + (dk + v * page) * row + piece * 16) =
          *reinterpret_cast<const u32x4_t*>(p.pool + (sk + v * page) * row + piece * 16);
    }
  }
}

int launch_evict(const EvictParams& p, hipStream_t s) {
  hipLaunchKernelGGL(evict_select_kernel, dim3(p.B * p.lists), dim3(NT), 0, s, p);
  hipLaunchKernelGGL(evict_move_kernel, dim3(p.B * p.lists * p.parts), dim3(256), 0, s, p);
  return hipGetLastError() == hipSuccess ? 0 : -1;
}

}  // namespace seer
