// The plan of a step: which pages it takes and gives back, and the slot of each new row.
#pragma once
#include <limits.h>

#include <type_traits>

#include "common.h"
#include "kernels.h"

namespace seer {

// For request b, H = ceil(held / page) pages are held and
// N = ceil((keep + rows) / page) needed; max(H - N, 0) are given back and
// max(N - H, 0) taken.  With the inclusive sums of both over the requests, the
// e-th page given back and the k-th page taken are known without a word
// between workgroups: the stack is free_pages[0 .. in) with the given pages on
// top, and the k-th page taken is k below its top.  So every workgroup makes
// the sums for itself (at most 16 requests a thread) and then works on its
// share of the rows, of the taken entries and of the given ones.  Nothing that
// one workgroup writes is read by another: table entries are written from H on
// and read below H, free_pages is written from `in` on and read below it, and
// the counts and lengths have two buffers.
// Bound by latency: one launch, the loads of the lengths, a block-wide sum, a
// search in LDS, the read of a page and its use: 6.0 us for the 240 tokens of 256
// requests, 5.2 us for 39,936 rows of 48 (a call from the host takes 5.6 us).
namespace {
constexpr int PLAN_T = 256;

struct Lens {
  int held, keep, real;      // tokens held and kept, real rows of the call
  bool bad;
};

__device__ __forceinline__ Lens lens_of(const PagePlanParams& p, int b) {
  Lens l;
  l.held = p.held[b];
  l.keep = p.keep[b];
  int n = p.cu[b + 1] - p.cu[b];
  n = n < 0 ? 0 : n;
  if (p.used) {
    const int u = p.used[b];
    n = u < n ? (u < 0 ? 0 : u) : n;
  }
  l.real = n;
  l.bad = l.held < 0 || l.keep < 0 || l.keep > l.held ||
          ((long long)l.held + (1 << p.shift) - 1) >> p.shift > p.width;
  return l;
}

__device__ __forceinline__ int pages_of(long long tokens, int shift) {
  return (int)((tokens + (1 << shift) - 1) >> shift);
}

// First index in [0, n) whose value in the non-decreasing v exceeds x.
__device__ __forceinline__ int first_above(const int* v, int n, int x) {
  int lo = 0, hi = n - 1;
  while (lo < hi) {
    const int mid = (lo + hi) >> 1;
    if (v[mid] > x) hi = mid;
    else lo = mid + 1;
  }
  return lo;
}
}  // namespace

// A plan where p.kept bounds what stays.  A kernel of its own with arguments of its own: the look at it,
// and arguments that pass 128 bytes, cost every plan 0.2 us.
struct KeptParams : PagePlanParams {
  const int* kept;       // [B] tokens that an eviction has left
};

template <typename P>
__global__ __launch_bounds__(PLAN_T) void page_plan_kernel(P p) {
  extern __shared__ int lds[];
  int* give_end = lds;               // [B] inclusive sums of the pages given back
  int* take_end = lds + p.B;         // [B] and of the pages taken
  int* row_end = lds + 2 * p.B;      // [B] cu[b + 1]
  __shared__ long long wave_give[PLAN_T / kWave], wave_take[PLAN_T / kWave];
  __shared__ int err;
  const int tid = threadIdx.x, lane = tid & (kWave - 1), wave = tid >> 6;
  const int in = *p.free_in;         // used after the sums: under way with the lengths
  if (tid == 0) err = 0;
  __syncthreads();

  const int per = (p.B + PLAN_T - 1) / PLAN_T;
  const int b0 = tid * per < p.B ? tid * per : p.B;
  const int b1 = b0 + per < p.B ? b0 + per : p.B;
  long long give = 0, take = 0;
  int bad = 0;
  Lens first_l{};                    // of b0, read once
  for (int b = b0; b < b1; ++b) {
    const Lens l = lens_of(p, b);
    if (b == b0) first_l = l;
    const int H = pages_of(l.held, p.shift), N = pages_of((long long)l.keep + l.real, p.shift);
    if (l.bad) bad |= kPagesInvalid;
    if constexpr (std::is_same_v<P, KeptParams>) {
      const int kept = p.kept[b];
      if (l.keep > (kept < 0 ? -1 - kept : kept)) bad |= kPagesInvalid;
    }
    if ((long long)l.keep + l.real > (long long)p.width << p.shift || (long long)l.keep + l.real > INT_MAX)
      bad |= kPagesWidth;
    give += H > N ? H - N : 0;
    take += N > H ? N - H : 0;
  }
  long long ig = give, it = take;
#pragma unroll
  for (int off = 1; off < kWave; off <<= 1) {
    const long long a = __shfl_up(ig, off, kWave), c = __shfl_up(it, off, kWave);
    if (lane >= off) { ig += a; it += c; }
  }
  if (lane == kWave - 1) { wave_give[wave] = ig; wave_take[wave] = it; }
  if (bad) atomicOr(&err, bad);
  __syncthreads();
  long long og = ig - give, ot = it - take, gave = 0, took = 0;
#pragma unroll
  for (int w = 0; w < PLAN_T / kWave; ++w) {
    if (w < wave) { og += wave_give[w]; ot += wave_take[w]; }
    gave += wave_give[w];
    took += wave_take[w];
  }
  int e = err | (in < 0 || in > p.n_pages ? kPagesInvalid : 0);
  if (e == 0 && in + gave > p.n_pages) e = kPagesInvalid;
  if (e == 0 && took > in + gave) e = kPagesExhausted;
  const int stride = gridDim.x * PLAN_T, first = blockIdx.x * PLAN_T + tid;
  const unsigned rows = p.rows_ub;   // up to 2^31 - 1: a row's index plus the stride passes an int
  if (first == 0) {
    *p.status = e;
    if (e && p.refused) *p.refused |= e;
    *p.free_out = e ? in : (int)(in + gave - took);
  }
  if (e) {
    for (unsigned r = first; r < rows; r += stride) p.slots[r] = -1;
    for (int b = first; b < p.B; b += stride) p.kv_len[b] = p.held[b];
    return;
  }
  for (int b = b0; b < b1; ++b) {
    const Lens l = b == b0 ? first_l : lens_of(p, b);
    const int H = pages_of(l.held, p.shift), N = pages_of((long long)l.keep + l.real, p.shift);
    og += H > N ? H - N : 0;
    ot += N > H ? N - H : 0;
    give_end[b] = (int)og;
    take_end[b] = (int)ot;
    row_end[b] = p.cu[b + 1];
    if (blockIdx.x == 0) p.kv_len[b] = l.keep + l.real;
  }
  __syncthreads();

  // the e-th page given back
  auto given = [&](int i) {
    const int b = first_above(give_end, p.B, i);
    const Lens l = lens_of(p, b);
    const int N = pages_of((long long)l.keep + l.real, p.shift);
    return p.table[(size_t)b * p.width + N + i - (b > 0 ? give_end[b - 1] : 0)];
  };
  // the k-th page taken
  const int top = in + (int)gave - 1;
  auto taken = [&](int k) {
    const int s = top - k;
    return s < in ? p.free_pages[s] : given(s - in);
  };
  for (unsigned at = first; at < rows; at += stride) {
    const int r = at;
    int slot = -1;
    if (r < row_end[p.B - 1]) {
      const int b = first_above(row_end, p.B, r);
      const Lens l = lens_of(p, b);
      const int i = r - p.cu[b];
      if (i >= 0 && i < l.real) {
        const int pos = l.keep + i, H = pages_of(l.held, p.shift), pi = pos >> p.shift;
        const int id = pi < H ? p.table[(size_t)b * p.width + pi] : taken((b > 0 ? take_end[b - 1] : 0) + pi - H);
        if (id >= 0 && id < p.n_pages) slot = (id << p.shift) + (pos & ((1 << p.shift) - 1));
      }
    }
    p.slots[r] = slot;
  }
  for (int k = first; k < (int)took; k += stride) {
    const int b = first_above(take_end, p.B, k);
    const int H = pages_of(p.held[b], p.shift);
    p.table[(size_t)b * p.width + H + k - (b > 0 ? take_end[b - 1] : 0)] = taken(k);
  }
  for (int i = first; i < (int)(gave - took); i += stride) p.free_pages[in + i] = given(i);
}

template <typename P>
int launch_plan(const P& p, hipStream_t s) {
  const int n = p.rows_ub > p.B ? p.rows_ub : p.B;
  const int blocks = n > 256 * PLAN_T ? 256 : (n + PLAN_T - 1) / PLAN_T;
  hipLaunchKernelGGL(page_plan_kernel<P>, dim3(blocks), dim3(PLAN_T), 3 * (size_t)p.B * sizeof(int), s, p);
  return hipGetLastError() == hipSuccess ? 0 : -1;
}

}  // namespace seer
