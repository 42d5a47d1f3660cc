// Attention with grouped heads over packed prompts and over pages, fp32 (any
// head_dim <= 128 that is a multiple of 4), on the fp32 matrix instruction.
//
// A workgroup takes 16 rows; its four waves take 16 keys of every 64 each and
// join at the end.  Scores are computed transposed (S^T = K Q^T, 16x16x4), so
// that a lane holds four keys of one row and its probabilities are the B operand
// of O^T += V^T P^T as they are: instruction i of four takes keys 4 g + i, g the
// lane's group of 16.  K and V go from memory to the operand registers in
// 16-byte loads; the order of the head's dims in the products is the one that
// those loads give.  Bound by latency where it is used for checks and small models:
// 97 rows of 4 heads by 64, 8.2 us.
#include <type_traits>

#include "gqa.h"

namespace seer {

namespace {
constexpr int NT = 256;

// A part's result: sums [H][e] of 64 lanes x 16 bytes, maxima and sums of 16 rows.
template <int H>
struct Parts {
  static constexpr size_t FLOATS = 16 * (64 * H + 2);
  float* base;
  __device__ __forceinline__ Parts(const GqaParams& p, int slot) : base(p.partial + (size_t)slot * FLOATS) {}
  __device__ __forceinline__ f32x4_t* sum(int t, int lane) const { return reinterpret_cast<f32x4_t*>(base) + t * 64 + lane; }
  __device__ __forceinline__ float* max(int row) const { return base + 16 * 64 * H + row; }
  __device__ __forceinline__ float* div(int row) const { return base + 16 * 64 * H + 16 + row; }
};

__device__ __forceinline__ float inverse(float l) { return l == 0.0f ? 0.0f : 1.0f / l; }
}  // namespace

// H: halves of 64 dims.
template <int H, bool PAGED>
__global__ __launch_bounds__(NT) void gqa_f32_kernel(GqaParams p) {
  constexpr int C = 4 * H;                                     // 16-dim pieces
  __shared__ f32x4_t o_part[4][4 * H][64];
  __shared__ float m_part[4][16], l_part[4][16];
  __shared__ int odd_part[4];
  __shared__ typename GqaCut<kGqaF32, NT>::Shared cut_lds;
  GqaCut<kGqaF32, NT> cut(p, cut_lds);
  GqaUnit u;
  while (cut.next(p, u)) {
  const int lane = threadIdx.x & 63;
  const int wv = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
  const int fr = lane & 15, g = lane >> 4;
  const int D = p.head_dim;
  const int row = u.t * kGqaF32 + fr;
  const int src = row < u.s.rows ? row : u.s.rows - 1;
  const int tok = gqa_token(p, src), head = src - tok * p.group;
  const GqaSight<PAGED> sight(p, u, tok);
  const int open = gqa_open_end(p, u, gqa_token(p, u.t * kGqaF32));
  const float c = p.scale * 1.4426950408889634f;
  const f32x4_t zero = {0.0f, 0.0f, 0.0f, 0.0f};

  f32x4_t qf[C];
  {
    const float* q = static_cast<const float*>(p.q) + (size_t)(u.s.s0 + tok) * p.q_stride + (size_t)(u.hk * p.group + head) * D;
#pragma unroll
    for (int i = 0; i < C; ++i) {
      const int d = 16 * i + 4 * g;
      qf[i] = *reinterpret_cast<const f32x4_t*>(q + (d < D ? d : 0));
      if (d >= D) qf[i] = zero;
    }
  }
  const float* kp = static_cast<const float*>(p.k);
  const float* vp = static_cast<const float*>(p.v);
  const int* table = PAGED ? p.table + (size_t)u.b * p.width : nullptr;
  const size_t half = PAGED ? ((size_t)p.n_kv << p.shift) * D : 0;
  if (!PAGED) {
    kp += (size_t)u.s.s0 * p.k_stride + (size_t)u.hk * D;
    vp += (size_t)u.s.s0 * p.v_stride + (size_t)u.hk * D;
  }
  f32x4_t o[4 * H];
#pragma unroll
  for (int i = 0; i < 4 * H; ++i) o[i] = zero;
  float m = -INFINITY, l = 0.0f;

  // where the group of keys from k0 on lies (k0 a multiple of 16); false: its page is none of the pool's
  auto place = [&](int k0, const float*& ks, const float*& vs, size_t& step_k, size_t& step_v) {
    if (PAGED) {
      const int id = scalar_load(table, k0 >> p.shift);
      const bool held = id >= 0 && id < p.n_pages;
      ks = kp + (size_t)(held ? id : 0) * 2 * half + (((size_t)u.hk << p.shift) + (k0 & ((1 << p.shift) - 1))) * D;
      vs = ks + half;
      step_k = step_v = D;
      return held;
    }
    ks = kp + (size_t)k0 * p.k_stride;
    vs = vp + (size_t)k0 * p.v_stride;
    step_k = p.k_stride;
    step_v = p.v_stride;
    return true;
  };
  int odd_from = INT_MAX;
  for (int k0 = u.lo + 16 * wv; k0 < u.hi; k0 += 64) {
    const int last = u.hi - 1 - k0 < 15 ? u.hi - 1 - k0 : 15;   // the group's last key: those past it are it again
    const float *ks, *vs;
    size_t step_k, step_v;
    const bool held = place(k0, ks, vs, step_k, step_v);
    const float* kr = ks + (fr < last ? fr : last) * step_k;
    f32x4_t kf[C], vf[4][H];
#pragma unroll
    for (int i = 0; i < C; ++i) {
      const int d = 16 * i + 4 * g;
      kf[i] = *reinterpret_cast<const f32x4_t*>(kr + (d < D ? d : 0));
    }
#pragma unroll
    for (int i = 0; i < 4; ++i) {
      const int r = 4 * g + i;
      const float* vr = vs + (r < last ? r : last) * step_v;
#pragma unroll
      for (int h = 0; h < H; ++h) {
        const int d = 64 * h + 4 * fr;
        vf[i][h] = *reinterpret_cast<const f32x4_t*>(vr + (d < D ? d : 0));
      }
    }
    // two chains, so that one product does not wait for the one before
    f32x4_t s0 = zero, s1 = zero;
#pragma unroll
    for (int i = 0; i < C; ++i) {
      if (16 * i >= D) break;
      const f32x4_t k = 16 * i + 4 * g < D ? kf[i] : zero;
#pragma unroll
      for (int e = 0; e < 4; e += 2) {
        s0 = __builtin_amdgcn_mfma_f32_16x16x4f32(k[e], qf[i][e], s0, 0, 0, 0);
        s1 = __builtin_amdgcn_mfma_f32_16x16x4f32(k[e + 1], qf[i][e + 1], s1, 0, 0, 0);
      }
    }
    f32x4_t s = s0 + s1;                                      // key k0 + 4 g + e
    const bool masked = k0 + 16 > open || !held;
    if (masked) {
      const uint32_t mine = held ? (uint32_t)(sight.seen(k0) >> (4 * g)) : 0;
#pragma unroll
      for (int e = 0; e < 4; ++e)
        if (!(mine >> e & 1)) s[e] = -INFINITY;
      // values that are no numbers would reach the rows that do not see their keys as
      // 0 * value: zeros here, and added to the rows that see them at the end
      bool odd = false;
#pragma unroll
      for (int i = 0; i < 4; ++i)
#pragma unroll
        for (int h = 0; h < H; ++h)
#pragma unroll
          for (int e = 0; e < 4; ++e)
            if (!(fabsf(vf[i][h][e]) < INFINITY)) {
              vf[i][h][e] = 0.0f;
              odd = true;
            }
      if (__any(odd)) odd_from = k0 < odd_from ? k0 : odd_from;
    }
    float mt = fmaxf(fmaxf(s[0], s[1]), fmaxf(s[2], s[3]));
    mt = fmaxf(mt, __shfl_xor(mt, 16, kWave));
    mt = fmaxf(mt, __shfl_xor(mt, 32, kWave));
    if (__any(mt > m)) {
      const float m_new = fmaxf(m, mt);
      const float alpha = m == -INFINITY ? 1.0f : __builtin_amdgcn_exp2f((m - m_new) * c);
      m = m_new;
      l *= alpha;
#pragma unroll
      for (int i = 0; i < 4 * H; ++i) o[i] *= alpha;
    }
    const float mc = m == -INFINITY ? 0.0f : m * c;
    f32x4_t w;
#pragma unroll
    for (int e = 0; e < 4; ++e) w[e] = __builtin_amdgcn_exp2f(s[e] * c - mc);
    l += (w[0] + w[1]) + (w[2] + w[3]);
#pragma unroll
    for (int i = 0; i < 4; ++i)
#pragma unroll
      for (int h = 0; h < H; ++h)
#pragma unroll
        for (int e = 0; e < 4; ++e)
          o[4 * h + e] = __builtin_amdgcn_mfma_f32_16x16x4f32(vf[i][h][e], w[i], o[4 * h + e], 0, 0, 0);
  }

  // join the waves: wave w takes sums w, w + 4
  l += __shfl_xor(l, 16, kWave);
  l += __shfl_xor(l, 32, kWave);
#pragma unroll
  for (int i = 0; i < 4 * H; ++i) o_part[wv][i][lane] = o[i];
  if (g == 0) {
    m_part[wv][fr] = m;
    l_part[wv][fr] = l;
  }
  if (lane == 0) odd_part[wv] = odd_from;
  __syncthreads();
  m = fmaxf(fmaxf(m_part[0][fr], m_part[1][fr]), fmaxf(m_part[2][fr], m_part[3][fr]));
  const float ref = m == -INFINITY ? 0.0f : m;
  l = 0.0f;
  f32x4_t sum[H];
#pragma unroll
  for (int h = 0; h < H; ++h) sum[h] = zero;
#pragma unroll
  for (int v = 0; v < 4; ++v) {
    const float mv = m_part[v][fr], lv = l_part[v][fr];
    if (mv == -INFINITY && lv == 0.0f) continue;              // a wave whose keys the row does not see
    const float a = __builtin_amdgcn_exp2f((mv - ref) * c);
    l += lv * a;
#pragma unroll
    for (int h = 0; h < H; ++h) sum[h] += a * o_part[v][4 * h + wv][lane];
  }
  // sum[h][i] is dim 64 h + 16 g + 4 i + wv
  odd_from = min(min(odd_part[0], odd_part[1]), min(odd_part[2], odd_part[3]));
  odd_from = __builtin_amdgcn_readfirstlane(odd_from);
  if (odd_from < u.hi) {
    // the values that were left out, for the keys that the row sees (again for those
    // of other groups, which changes nothing)
    for (int k0 = odd_from; k0 < u.hi; k0 += 16) {
      const float *ks, *vs;
      size_t step_k, step_v;
      if (!place(k0, ks, vs, step_k, step_v)) continue;
      const uint32_t seen = (uint32_t)sight.seen(k0);
      for (int j = 0; j < 16 && k0 + j < u.hi; ++j)
#pragma unroll
        for (int h = 0; h < H; ++h)
#pragma unroll
          for (int i = 0; i < 4; ++i) {
            const int d = 64 * h + 16 * g + 4 * i + wv;
            const float x = vs[j * step_v + (d < D ? d : 0)];
            if ((seen >> j & 1) && !(fabsf(x) < INFINITY)) sum[h][i] += x;
          }
    }
  }
  if (row >= u.s.rows) continue;
  if (!u.whole) {
    const Parts<H> to(p, u.slot);
#pragma unroll
    for (int h = 0; h < H; ++h) *to.sum(4 * h + wv, lane) = sum[h];
    if (wv == 0 && g == 0) {
      *to.max(fr) = m;
      *to.div(fr) = l;
    }
    continue;
  }
  const bool real = tok < u.s.used;
  const float inv = inverse(l);
  float* out = static_cast<float*>(p.out) + (size_t)(u.s.s0 + tok) * p.o_stride + (size_t)(u.hk * p.group + head) * D;
#pragma unroll
  for (int h = 0; h < H; ++h)
#pragma unroll
    for (int i = 0; i < 4; ++i) {
      const int d = 64 * h + 16 * g + 4 * i + wv;
      if (d < D) out[d] = real ? sum[h][i] * inv : 0.0f;
    }
  }
}

// Adds the parts of each tile whose keys were cut; wave w as in the kernel above.
template <int H>
__global__ __launch_bounds__(NT) void gqa_f32_join_kernel(GqaParams p) {
  const int wg = blockIdx.x;
  const GqaRecord r = static_cast<const GqaRecord*>(p.records)[wg];
  if (r.parts < 2) return;
  const int lane = threadIdx.x & 63, wv = threadIdx.x >> 6, fr = lane & 15, g = lane >> 4, D = p.head_dim;
  const int row = r.t * kGqaF32 + fr;
  if (row >= r.rows) return;
  const float c = p.scale * 1.4426950408889634f;
  // the loads of several parts under way together
  float m = -INFINITY, l = 0.0f;
  f32x4_t sum[H];
#pragma unroll
  for (int h = 0; h < H; ++h) sum[h] = f32x4_t{0.0f, 0.0f, 0.0f, 0.0f};
  auto add = [&](int i0, auto width) {
    constexpr int W = decltype(width)::value;
    float pm[W], pl[W];
    f32x4_t v[W][H];
#pragma unroll
    for (int k = 0; k < W; ++k) {
      const Parts<H> from(p, gqa_slot(r, wg, i0 + k < r.parts ? i0 + k : r.parts - 1));
      pm[k] = *from.max(fr);
      pl[k] = *from.div(fr);
#pragma unroll
      for (int h = 0; h < H; ++h) v[k][h] = *from.sum(4 * h + wv, lane);
    }
    float top = m;
#pragma unroll
    for (int k = 0; k < W; ++k) top = fmaxf(top, pm[k]);
    const float ref = top == -INFINITY ? 0.0f : top;
    const float keep = m == -INFINITY ? 1.0f : __builtin_amdgcn_exp2f((m - ref) * c);
    m = top;
    l *= keep;
#pragma unroll
    for (int h = 0; h < H; ++h) sum[h] *= keep;
#pragma unroll
    for (int k = 0; k < W; ++k) {
      const bool none = i0 + k >= r.parts || (pm[k] == -INFINITY && pl[k] == 0.0f);
      const float a = none ? 0.0f : __builtin_amdgcn_exp2f((pm[k] - ref) * c);
      l += none ? 0.0f : pl[k] * a;
#pragma unroll
      for (int h = 0; h < H; ++h) sum[h] += none ? f32x4_t{0, 0, 0, 0} : a * v[k][h];
    }
  };
  if (r.parts <= 4) add(0, std::integral_constant<int, 4>{});
  else if (r.parts <= 8) add(0, std::integral_constant<int, 8>{});
  else
    for (int i0 = 0; i0 < r.parts; i0 += 16) add(i0, std::integral_constant<int, 16>{});
  const int tok = gqa_token(p, row), head = row - tok * p.group;
  const bool real = tok < r.used;
  const float inv = inverse(l);
  float* out = static_cast<float*>(p.out) + (size_t)(r.s0 + tok) * p.o_stride + (size_t)(r.hk * p.group + head) * D;
#pragma unroll
  for (int h = 0; h < H; ++h)
#pragma unroll
    for (int i = 0; i < 4; ++i) {
      const int d = 64 * h + 16 * g + 4 * i + wv;
      if (d < D) out[d] = real ? sum[h][i] * inv : 0.0f;
    }
}

int launch_gqa_f32(const GqaParams& p, const GqaRule& r, hipStream_t s) {
  const dim3 grid(r.grid), block(NT);
  if (p.head_dim > 64) {
    if (p.table) hipLaunchKernelGGL((gqa_f32_kernel<2, true>), grid, block, 0, s, p);
    else hipLaunchKernelGGL((gqa_f32_kernel<2, false>), grid, block, 0, s, p);
    if (r.cut) hipLaunchKernelGGL(gqa_f32_join_kernel<2>, dim3(r.grid), block, 0, s, p);
  } else {
    if (p.table) hipLaunchKernelGGL((gqa_f32_kernel<1, true>), grid, block, 0, s, p);
    else hipLaunchKernelGGL((gqa_f32_kernel<1, false>), grid, block, 0, s, p);
    if (r.cut) hipLaunchKernelGGL(gqa_f32_join_kernel<1>, dim3(r.grid), block, 0, s, p);
  }
  return hipGetLastError() == hipSuccess ? 0 : -1;
}

}  // namespace seer
