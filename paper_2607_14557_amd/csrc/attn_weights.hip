// The attention weight that the rows of a call give to each cached token:
//
//   w_j = decay prev_j + sum over rows i and heads h of the group of p_ihj,
//   p_ihj = exp(s_ihj - lse_ih),  s = scale q . k,  lse_ih = log sum_j exp(s_ihj) over the keys that row i sees
//
// per key/value head.  A row's sum is known when all its keys have been seen, so the
// scores are made twice: by weights_stats_kernel, transposed (S^T = K Q^T), where a
// lane owns a row and its maximum and sum, for a part of the keys; and, after
// weights_lse_kernel has joined the parts, by weights_sum_kernel (S = Q K^T), where a
// lane owns a key and adds up its rows in registers.  Both operands of a tile come in
// the same layout, so either may stand first.  Each weight is written once, by one wave
// that adds in one order: no atomics, the same bits every time.
#include <limits.h>

#include "common.h"
#include "dispatch.h"
#include "kernels.h"

namespace seer {

namespace {

constexpr int NT = 256, WAVES = NT / kWave;

// 32 x 32 products of bf16 rows: fragment ks of a row is dims 16 ks + 8 (lane / 32) + e.
template <int DH>
struct TileBf16 {
  static constexpr int T = 32, ACC = 16, F = DH / 16;
  typedef f32x16_t acc_t;
  struct Frag { bf16x8_t f[F]; };
  __device__ __forceinline__ static int row(int lane) { return lane & 31; }
  // index along the first operand's rows of element r
  __device__ __forceinline__ static int of(int lane, int r) { return 8 * (r >> 2) + 4 * (lane >> 5) + (r & 3); }
  __device__ __forceinline__ static void load(Frag& f, const void* base, long long at, int, int lane) {
    const uint16_t* p = static_cast<const uint16_t*>(base) + at + 8 * (lane >> 5);
#pragma unroll
    for (int i = 0; i < F; ++i) f.f[i] = __builtin_bit_cast(bf16x8_t, *reinterpret_cast<const u32x4_t*>(p + 16 * i));
  }
  __device__ __forceinline__ static void mul(acc_t& c, const Frag& a, const Frag& b) {
#pragma unroll
    for (int r = 0; r < 16; ++r) c[r] = 0.0f;
#pragma unroll
    for (int i = 0; i < F; ++i) c = __builtin_amdgcn_mfma_f32_32x32x16_bf16(a.f[i], b.f[i], c, 0, 0, 0);
  }
  // over the lanes that share a second operand's row
  __device__ __forceinline__ static float max(float v) { return fmaxf(v, __shfl_xor(v, 32, kWave)); }
  __device__ __forceinline__ static float sum(float v) { return v + __shfl_xor(v, 32, kWave); }
};

// 16 x 16 products of fp32 rows: fragment i of a row is dims 16 i + 4 (lane / 16) + e, zero past the head.
template <int HALVES>
struct TileF32 {
  static constexpr int T = 16, ACC = 4, F = 4 * HALVES;
  typedef f32x4_t acc_t;
  struct Frag { f32x4_t f[F]; };
  __device__ __forceinline__ static int row(int lane) { return lane & 15; }
  __device__ __forceinline__ static int of(int lane, int r) { return 4 * (lane >> 4) + r; }
  __device__ __forceinline__ static void load(Frag& f, const void* base, long long at, int dim, int lane) {
    const float* p = static_cast<const float*>(base) + at;
#pragma unroll
    for (int i = 0; i < F; ++i) {
      const int d = 16 * i + 4 * (lane >> 4);
      f.f[i] = *reinterpret_cast<const f32x4_t*>(p + (d < dim ? d : 0));
      if (d >= dim) f.f[i] = f32x4_t{0.0f, 0.0f, 0.0f, 0.0f};
    }
  }
  __device__ __forceinline__ static void mul(acc_t& c, const Frag& a, const Frag& b) {
    // two chains, so that one product does not wait for the one before
    f32x4_t c0 = {0.0f, 0.0f, 0.0f, 0.0f}, c1 = c0;
#pragma unroll
    for (int i = 0; i < F; ++i)
#pragma unroll
      for (int e = 0; e < 4; e += 2) {
        c0 = __builtin_amdgcn_mfma_f32_16x16x4f32(a.f[i][e], b.f[i][e], c0, 0, 0, 0);
        c1 = __builtin_amdgcn_mfma_f32_16x16x4f32(a.f[i][e + 1], b.f[i][e + 1], c1, 0, 0, 0);
      }
    c = c0 + c1;
  }
  __device__ __forceinline__ static float max(float v) {
    v = fmaxf(v, __shfl_xor(v, 16, kWave));
    return fmaxf(v, __shfl_xor(v, 32, kWave));
  }
  __device__ __forceinline__ static float sum(float v) {
    v += __shfl_xor(v, 16, kWave);
    return v + __shfl_xor(v, 32, kWave);
  }
};

// A request of the call: the rows that count, and its keys.
struct Seq {
  int row0, rows;        // first row that counts, and how many (token, head of a group) pairs do
  int index0;            // that row's index among the request's rows of the call
  int used;              // rows that count
  int nk, past;          // keys; those before the request's first row of the call
};

__device__ __forceinline__ Seq seq_of(const WeightsParams& p, int b) {
  Seq s;
  const int s0 = p.cu[b];
  int len = p.cu[b + 1] - s0;
  if (s0 < 0 || s0 >= p.rows_ub || len < 0) len = 0;
  len = len > p.rows_ub - s0 ? p.rows_ub - s0 : len;
  int n = p.used ? p.used[b] : len;
  n = n < 0 ? 0 : (n > len ? len : n);
  s.index0 = p.last > 0 && n > p.last ? n - p.last : 0;
  s.used = n - s.index0;
  s.row0 = s0 + s.index0;
  s.rows = s.used * p.group;
  s.nk = gqa_keys(p.kv_len[b], p.width, p.shift);
  s.past = s.nk - n;
  return s;
}

// Keys of a part: the parts of a request are equal, whole tiles of 64 keys.
__device__ __forceinline__ int part_keys(const WeightsParams& p, int nk) {
  const int blocks = (nk + 63) / 64;
  return ((blocks + p.parts - 1) / p.parts) * 64;
}

// The units of a launch: those of request after request in one line, whose ends each
// workgroup finds for itself.
struct Line {
  int* end;              // [B] inclusive sums of the requests' units
  int* rows;             // [B] and of their rows that count
  int all;
};

template <typename Units>
__device__ __forceinline__ Line line_of(const WeightsParams& p, int* lds, Units units) {
  __shared__ int sums[2][WAVES];
  Line l{lds, lds + p.B, 0};
  const int tid = threadIdx.x, lane = tid & (kWave - 1), wave = tid >> 6;
  const int per = (p.B + NT - 1) / NT;
  const int b0 = tid * per < p.B ? tid * per : p.B;
  const int b1 = b0 + per < p.B ? b0 + per : p.B;
  int n = 0, m = 0;
  for (int b = b0; b < b1; ++b) {
    const Seq s = seq_of(p, b);
    n += units(s);
    m += s.used;
  }
  int in = n, im = m;
#pragma unroll
  for (int off = 1; off < kWave; off <<= 1) {
    const int a = __shfl_up(in, off, kWave), c = __shfl_up(im, off, kWave);
    if (lane >= off) { in += a; im += c; }
  }
  if (lane == kWave - 1) { sums[0][wave] = in; sums[1][wave] = im; }
  __syncthreads();
  int on = in - n, om = im - m;
#pragma unroll
  for (int w = 0; w < WAVES; ++w) {
    if (w < wave) { on += sums[0][w]; om += sums[1][w]; }
    l.all += sums[0][w];
  }
  for (int b = b0; b < b1; ++b) {
    const Seq s = seq_of(p, b);
    on += units(s);
    om += s.used;
    l.end[b] = on;
    l.rows[b] = om;
  }
  __syncthreads();
  return l;
}

// The request of unit u, and the unit's place there.
__device__ __forceinline__ int request_of(const Line& l, int B, int u, int& at) {
  int lo = 0, hi = B - 1;
  while (lo < hi) {
    const int mid = (lo + hi) >> 1;
    if (l.end[mid] > u) hi = mid;
    else lo = mid + 1;
  }
  at = u - (lo > 0 ? l.end[lo - 1] : 0);
  return lo;
}

// The row of a key of the pool, in elements; the first page's where its page is none of the pool's (held false).
__device__ __forceinline__ long long key_row(const WeightsParams& p, const int* table, int hk, int key, bool& held) {
  const int id = table[key >> p.shift];
  held = id >= 0 && id < p.n_pages;
  const long long half = (long long)p.n_kv << p.shift;
  return ((held ? id : 0) * 2 * half + ((long long)hk << p.shift) + (key & ((1 << p.shift) - 1))) * p.head_dim;
}

// Whether the row with this index among its request's rows of the call sees a key.
__device__ __forceinline__ bool sees(const WeightsParams& p, const Seq& s, int b_row, int index, int key) {
  if (key >= s.nk) return false;
  if (p.mask == kMaskCausal) return key <= s.past + index;
  if (p.mask == kMaskTree) {
    const int j = key - s.past;
    if (j < 0) return true;
    return j >> 6 < p.words && (p.bits[(size_t)b_row * p.words + (j >> 6)] >> (j & 63) & 1);
  }
  return true;
}

__device__ __forceinline__ int token_of(const WeightsParams& p, int x) {
  return (int)((__umulhi((unsigned)x, p.group_mul) + (unsigned)x) >> p.group_shift);
}

}  // namespace

// Maximum and sum of the rows of a tile over a part of the keys: a wave a unit.
template <typename Tile>
__global__ __launch_bounds__(NT) void weights_stats_kernel(WeightsParams p) {
  extern __shared__ int lds[];
  constexpr int T = Tile::T;
  auto units = [&](const Seq& s) { return s.nk > 0 ? (s.rows + T - 1) / T * p.n_kv * p.parts : 0; };
  const Line line = line_of(p, lds, units);
  const int lane = threadIdx.x & (kWave - 1), wave = threadIdx.x >> 6;
  const float c = p.scale * 1.4426950408889634f;
  for (int u = blockIdx.x * WAVES + wave; u < line.all; u += gridDim.x * WAVES) {
    int at;
    const int b = request_of(line, p.B, u, at);
    const Seq s = seq_of(p, b);
    const int tiles = (s.rows + T - 1) / T;
    const int t = at % tiles, part = at / tiles % p.parts, hk = at / tiles / p.parts;
    const int row = t * T + Tile::row(lane), src = row < s.rows ? row : s.rows - 1;
    const int tok = token_of(p, src), head = hk * p.group + src - tok * p.group;
    typename Tile::Frag q, k;
    Tile::load(q, p.q, (long long)(s.row0 + tok) * p.q_stride + (long long)head * p.head_dim, p.head_dim, lane);
    const int keys = part_keys(p, s.nk);
    const long long begin = (long long)part * keys, end = begin + keys;
    const int lo = begin < s.nk ? (int)begin : s.nk, hi = end < s.nk ? (int)end : s.nk;
    const int* table = p.table + (size_t)b * p.width;
    float m = -INFINITY, l = 0.0f;
    for (int k0 = lo; k0 < hi; k0 += T) {
      const int key = k0 + Tile::row(lane) < s.nk ? k0 + Tile::row(lane) : s.nk - 1;
      bool held;
      Tile::load(k, p.pool, key_row(p, table, hk, key, held), p.head_dim, lane);
      const unsigned long long lost = ~__ballot(held);
      typename Tile::acc_t a;
      Tile::mul(a, k, q);
      float x[Tile::ACC], top = -INFINITY;
#pragma unroll
      for (int r = 0; r < Tile::ACC; ++r) {
        const int i = Tile::of(lane, r);
        const bool see = sees(p, s, s.row0 + tok, s.index0 + tok, k0 + i) && !(lost >> i & 1);
        x[r] = see ? a[r] * c : -INFINITY;
        top = fmaxf(top, x[r]);
      }
      const float to = fmaxf(m, top), ref = to == -INFINITY ? 0.0f : to;
      float sum = 0.0f;
#pragma unroll
      for (int r = 0; r < Tile::ACC; ++r) sum += __builtin_amdgcn_exp2f(x[r] - ref);
      l = l * __builtin_amdgcn_exp2f(m - ref) + sum;
      m = to;
    }
    const float top = Tile::max(m), ref = top == -INFINITY ? 0.0f : top;
    l = Tile::sum(l * __builtin_amdgcn_exp2f(m - ref));
    if (row < s.rows && lane < T) {
      const long long r = (line.rows[b] - s.used + tok) * (long long)p.n_heads + head;
      p.stats[r * p.parts + part] = f32x2_t{top, l};
    }
  }
}

// log2 of each row's sum, from its parts: a thread a row and head.
__global__ __launch_bounds__(NT) void weights_lse_kernel(WeightsParams p) {
  extern __shared__ int lds[];
  const Line line = line_of(p, lds, [&](const Seq& s) { return s.nk > 0 ? s.used : 0; });
  const long long all = (long long)line.rows[p.B - 1] * p.n_heads;
  for (long long r = (long long)blockIdx.x * NT + threadIdx.x; r < all; r += (long long)gridDim.x * NT) {
    const f32x2_t* from = p.stats + r * p.parts;
    float top = -INFINITY, sum = 0.0f;
    for (int i = 0; i < p.parts; ++i) top = fmaxf(top, from[i][0]);
    const float ref = top == -INFINITY ? 0.0f : top;
    for (int i = 0; i < p.parts; ++i) sum += from[i][1] * __builtin_amdgcn_exp2f(from[i][0] - ref);
    p.lse[r] = top + __builtin_amdgcn_logf(sum);
  }
}

// The weights of a tile of keys: a wave a unit.
template <typename Tile>
__global__ __launch_bounds__(NT) void weights_sum_kernel(WeightsParams p) {
  extern __shared__ int lds[];
  constexpr int T = Tile::T;
  auto units = [&](const Seq& s) { return s.used > 0 ? (s.nk + T - 1) / T * p.n_kv : 0; };
  const Line line = line_of(p, lds, units);
  const int lane = threadIdx.x & (kWave - 1), wave = threadIdx.x >> 6;
  const float c = p.scale * 1.4426950408889634f;
  for (int u = blockIdx.x * WAVES + wave; u < line.all; u += gridDim.x * WAVES) {
    int at;
    const int b = request_of(line, p.B, u, at);
    const Seq s = seq_of(p, b);
    const int tiles = (s.nk + T - 1) / T;
    const int hk = at / tiles, k0 = (at - hk * tiles) * T;
    const int* table = p.table + (size_t)b * p.width;
    const int key = k0 + Tile::row(lane), src = key < s.nk ? key : s.nk - 1;
    bool held;
    typename Tile::Frag k, q;
    const long long krow = key_row(p, table, hk, src, held);
    Tile::load(k, p.pool, krow, p.head_dim, lane);
    const float* lse = p.lse + (long long)(line.rows[b] - s.used) * p.n_heads + hk * p.group;
    float sum = 0.0f;
    for (int r0 = 0; r0 < s.rows; r0 += T) {
      const int row = r0 + Tile::row(lane) < s.rows ? r0 + Tile::row(lane) : s.rows - 1;
      const int tok = token_of(p, row), head = row - tok * p.group;
      Tile::load(q, p.q, (long long)(s.row0 + tok) * p.q_stride + (long long)(hk * p.group + head) * p.head_dim, p.head_dim,
                 lane);
      typename Tile::acc_t a;
      Tile::mul(a, q, k);
#pragma unroll
      for (int r = 0; r < Tile::ACC; ++r) {
        const int i = r0 + Tile::of(lane, r);
        if (i >= s.rows) continue;
        const int it = token_of(p, i), ih = i - it * p.group;
        if (!sees(p, s, s.row0 + it, s.index0 + it, key)) continue;
        sum += __builtin_amdgcn_exp2f(a[r] * c - lse[(long long)it * p.n_heads + ih]);
      }
    }
    sum = Tile::sum(sum);
    if (lane < T && key < s.nk && held) {
      const long long id = table[key >> p.shift];
      const long long mark = (((id * p.n_kv) + hk) << p.shift) + (key & ((1 << p.shift) - 1));
      p.weight[mark] = p.prev ? __builtin_fmaf(p.decay, p.prev[mark], sum) : sum;
    }
  }
}

int launch_weights(const WeightsParams& p, hipStream_t s) {
  const size_t lds = 2 * (size_t)p.B * sizeof(int);
  auto go = [&](auto tile) {
    using Tile = decltype(tile);
    hipLaunchKernelGGL((weights_stats_kernel<Tile>), dim3(2048), dim3(NT), lds, s, p);
    hipLaunchKernelGGL(weights_lse_kernel, dim3(256), dim3(NT), lds, s, p);
    hipLaunchKernelGGL((weights_sum_kernel<Tile>), dim3(2048), dim3(NT), lds, s, p);
  };
  if (p.bf16) {
    if (p.head_dim == 128) go(TileBf16<128>{});
    else go(TileBf16<64>{});
  } else {
    if (p.head_dim > 64) go(TileF32<2>{});
    else go(TileF32<1>{});
  }
  return hipGetLastError() == hipSuccess ? 0 : -1;
}

}  // namespace seer
