// Rotary positions of packed query and key rows, alone or on the way into pages,
// and the positions of a step's rows.
//
//   x'_a = m (x_a cos t - x_b sin t),  x'_b = m (x_b cos t + x_a sin t),  t = position * f_j
//
// for the pairs (a, b) = (j, j + R/2) or (2j, 2j + 1), j < R/2; dims from R on are
// copied.  The frequencies come as turns a position in fp64: the product with a
// position and what is left of it after whole turns are taken in fp64, since an
// angle of 10^6 radians in fp32 is off by 0.06.  Sine and cosine of the rest, at most
// half a turn, and the products are fp32; the result is rounded once, to the row's
// type.
#include "common.h"
#include "kernels.h"

namespace seer {

namespace {

constexpr int NT = 256, WAVES = NT / kWave;

// Elements of a 16-byte piece.
template <int ES>
struct Piece {
  static constexpr int N = 16 / ES;
  float x[N];
  __device__ __forceinline__ void from(u32x4_t v) {
#pragma unroll
    for (int e = 0; e < 4; ++e) {
      if constexpr (ES == 2) {
        x[2 * e] = __uint_as_float(v[e] << 16);
        x[2 * e + 1] = __uint_as_float(v[e] & 0xffff0000u);
      } else {
        x[e] = __uint_as_float(v[e]);
      }
    }
  }
  __device__ __forceinline__ u32x4_t bits() const {
    u32x4_t v;
#pragma unroll
    for (int e = 0; e < 4; ++e) {
      if constexpr (ES == 2) v[e] = pack_bf2(x[2 * e], x[2 * e + 1]);
      else v[e] = __float_as_uint(x[e]);
    }
    return v;
  }
};

template <int ES>
__device__ __forceinline__ float load1(const uint8_t* p) {
  if constexpr (ES == 2) return bf2f(*reinterpret_cast<const uint16_t*>(p));
  else return *reinterpret_cast<const float*>(p);
}
template <int ES>
__device__ __forceinline__ void store1(uint8_t* p, float x) {
  if constexpr (ES == 2) *reinterpret_cast<uint16_t*>(p) = f2bf(x);
  else *reinterpret_cast<float*>(p) = x;
}

__device__ __forceinline__ u32x4_t load16(const uint8_t* p) { return *reinterpret_cast<const u32x4_t*>(p); }
__device__ __forceinline__ void store16(uint8_t* p, u32x4_t v) { *reinterpret_cast<u32x4_t*>(p) = v; }

// The heads of a row: head h of the source at src + h * from, of the result at dst + h * to (bytes).
struct Heads {
  const uint8_t* src;
  uint8_t* dst;
  size_t from, to;
  int n;
};

// Turns a row's heads; the whole wave works on it.  cs: cosine and sine of each pair (LDS).
template <int ES>
__device__ __forceinline__ void turn_heads(const RopeParams& p, const Heads& r, const f32x2_t* cs, int lane) {
  constexpr int N = Piece<ES>::N;
  const int R = p.rot, half = R / 2, pieces = p.dim / N;
  if (p.pairs) {
    // a piece holds its pairs whole
    for (int i = lane; i < r.n * pieces; i += kWave) {
      const int h = i / pieces, d = (i - h * pieces) * N;
      Piece<ES> x;
      x.from(load16(r.src + h * r.from + (size_t)d * ES));
#pragma unroll
      for (int e = 0; e < N; e += 2) {
        if (d + e < R) {
          const f32x2_t t = cs[(d + e) / 2];
          const float u = x.x[e], v = x.x[e + 1];
          x.x[e] = u * t[0] - v * t[1];
          x.x[e + 1] = v * t[0] + u * t[1];
        }
      }
      store16(r.dst + h * r.to + (size_t)d * ES, x.bits());
    }
    return;
  }
  if (half % N == 0) {
    // two pieces half the turned dims apart, then the dims behind them
    const int hp = half / N;
    for (int i = lane; i < r.n * hp; i += kWave) {
      const int h = i / hp, d = (i - h * hp) * N;
      const uint8_t* s = r.src + h * r.from + (size_t)d * ES;
      Piece<ES> x, y;
      x.from(load16(s));
      y.from(load16(s + (size_t)half * ES));
#pragma unroll
      for (int e = 0; e < N; ++e) {
        const f32x2_t t = cs[d + e];
        const float u = x.x[e], v = y.x[e];
        x.x[e] = u * t[0] - v * t[1];
        y.x[e] = v * t[0] + u * t[1];
      }
      uint8_t* o = r.dst + h * r.to + (size_t)d * ES;
      store16(o, x.bits());
      store16(o + (size_t)half * ES, y.bits());
    }
  } else {
    for (int i = lane; i < r.n * half; i += kWave) {
      const int h = i / half, j = i - h * half;
      const uint8_t* s = r.src + h * r.from + (size_t)j * ES;
      const float u = load1<ES>(s), v = load1<ES>(s + (size_t)half * ES);
      const f32x2_t t = cs[j];
      uint8_t* o = r.dst + h * r.to + (size_t)j * ES;
      store1<ES>(o, u * t[0] - v * t[1]);
      store1<ES>(o + (size_t)half * ES, v * t[0] + u * t[1]);
    }
  }
  if (r.src == r.dst) return;                  // in place: the rest is where it belongs
  const int lo = (R + N - 1) / N * N, odd = lo - R, tail = (p.dim - lo) / N;
  for (int i = lane; i < r.n * odd; i += kWave) {
    const int h = i / odd, d = R + i - h * odd;
    store1<ES>(r.dst + h * r.to + (size_t)d * ES, load1<ES>(r.src + h * r.from + (size_t)d * ES));
  }
  for (int i = lane; i < r.n * tail; i += kWave) {
    const int h = i / tail, d = lo + (i - h * tail) * N;
    store16(r.dst + h * r.to + (size_t)d * ES, load16(r.src + h * r.from + (size_t)d * ES));
  }
}

}  // namespace

// A wave a row: its angles (a pair a lane), then its heads in 16-byte pieces.  Bound by
// bytes: 19,048 rows of q and k in and out, 390 MB, take 78 us (5.0 TB/s, a copy's rate); 20,118
// rows of q, k and v of 32 heads on their way into pages, 994 MB, 199 us (5.0 TB/s); 256 rows 6.
template <int ES, bool STORE>
__global__ __launch_bounds__(NT) void rope_kernel(RopeParams p) {
  __shared__ f32x2_t cs_lds[WAVES][64];
  const int lane = threadIdx.x & (kWave - 1), wave = threadIdx.x >> 6;
  f32x2_t* cs = cs_lds[wave];
  for (long long r = (long long)blockIdx.x * WAVES + wave; r < p.rows_ub; r += (long long)gridDim.x * WAVES) {
    const int pos = p.positions[r];
    const int slot = STORE ? p.slots[r] : 0;
    if (pos < 0 || slot < 0 || (STORE && (slot >> p.shift) >= p.n_pages)) continue;
    if (lane < p.rot / 2) {
      double t = (double)pos * p.turns[lane];
      t -= __builtin_rint(t);
      float s, c;
      sincospif(2.0f * (float)t, &s, &c);
      cs[lane] = f32x2_t{p.magnitude * c, p.magnitude * (p.inverse ? -s : s)};
    }
    __builtin_amdgcn_fence(__ATOMIC_ACQ_REL, "wavefront");      // the wave's own LDS
    __builtin_amdgcn_wave_barrier();
    const size_t head = (size_t)p.dim * ES;
    if (p.q)
      turn_heads<ES>(p, Heads{p.q + (size_t)r * p.q_stride, p.q_out + (size_t)r * p.q_out_stride, head, head, p.n_heads},
                     cs, lane);
    if constexpr (STORE) {
      const size_t rows = (size_t)p.n_kv << p.shift;            // head rows of K (or V) in a page
      const int off = slot & ((1 << p.shift) - 1);
      const size_t page = (size_t)(slot >> p.shift) * 2 * rows;
      uint8_t* to = p.pool + (page + off) * head;
      const size_t step = head << p.shift;
      turn_heads<ES>(p, Heads{p.k + (size_t)r * p.k_stride, to, head, step, p.n_kv}, cs, lane);
      const uint8_t* v = p.v + (size_t)r * p.v_stride;
      const int pieces = p.dim * ES / 16;
      for (int i = lane; i < p.n_kv * pieces; i += kWave) {
        const int h = i / pieces, c = i - h * pieces;
        store16(to + rows * head + h * step + (size_t)c * 16, load16(v + (size_t)i * 16));
      }
      if (p.weight)
        for (int h = lane; h < p.n_kv; h += kWave) {
          const size_t at = page / 2 + ((size_t)h << p.shift) + off;
          p.weight[at] = 0.0f;
          p.number[at] = pos;
        }
    } else if (p.k) {
      turn_heads<ES>(p, Heads{p.k + (size_t)r * p.k_stride, p.k_out + (size_t)r * p.k_out_stride, head, head, p.n_kv},
                     cs, lane);
    }
    __builtin_amdgcn_fence(__ATOMIC_ACQ_REL, "wavefront");
    __builtin_amdgcn_wave_barrier();
  }
}

int launch_rope(const RopeParams& p, hipStream_t s) {
  const int blocks = p.rows_ub / WAVES + (p.rows_ub % WAVES != 0);
  const dim3 grid(blocks < 1 << 22 ? blocks : 1 << 22), block(NT);
  if (p.pool) {
    if (p.es == 2) hipLaunchKernelGGL((rope_kernel<2, true>), grid, block, 0, s, p);
    else hipLaunchKernelGGL((rope_kernel<4, true>), grid, block, 0, s, p);
  } else {
    if (p.es == 2) hipLaunchKernelGGL((rope_kernel<2, false>), grid, block, 0, s, p);
    else hipLaunchKernelGGL((rope_kernel<4, false>), grid, block, 0, s, p);
  }
  return hipGetLastError() == hipSuccess ? 0 : -1;
}

// ---------------------------------------------------------------------------
// The positions of a step's rows: a thread a row finds its request in cu.  Bound by
// latency, the search's dependent reads: a call of 64 to 39,936 rows takes 5.7 us, a launch.
__global__ __launch_bounds__(NT) void row_positions_kernel(RowPositionsParams p) {
  const long long first = (long long)blockIdx.x * NT + threadIdx.x, step = (long long)gridDim.x * NT;
  auto real = [&](int b) {
    int n = p.cu[b + 1] - p.cu[b];
    n = n < 0 ? 0 : n;
    if (p.used) {
      const int u = p.used[b];
      n = u < n ? (u < 0 ? 0 : u) : n;
    }
    return n;
  };
  const bool refused = p.status && *p.status != 0;
  const int* base = p.base ? p.base : p.seen;
  for (long long r = first; r < p.rows_ub; r += step) {
    int at = -1;
    if (!refused && r < p.cu[p.B]) {
      int lo = 0, hi = p.B - 1;                  // the first request that ends behind the row
      while (lo < hi) {
        const int mid = (lo + hi) >> 1;
        if (p.cu[mid + 1] > r) hi = mid;
        else lo = mid + 1;
      }
      const int i = (int)r - p.cu[lo];
      if (i >= 0 && i < real(lo)) at = (base ? base[lo] : 0) + i;
    }
    p.positions[r] = at;
  }
  if (p.next)
    for (long long b = first; b < p.B; b += step)
      p.next[b] = refused ? (p.seen ? p.seen[b] : 0) : (base ? base[b] : 0) + real((int)b);
  if (p.kept && !refused)
    for (long long b = first; b < p.B; b += step) p.kept[b] = p.kv_len[b];
}

int launch_row_positions(const RowPositionsParams& p, hipStream_t s) {
  const int n = p.rows_ub > p.B ? p.rows_ub : p.B;
  const int blocks = n / NT + (n % NT != 0);
  hipLaunchKernelGGL(row_positions_kernel, dim3(blocks < 4096 ? blocks : 4096), dim3(NT), 0, s, p);
  return hipGetLastError() == hipSuccess ? 0 : -1;
}

}  // namespace seer
