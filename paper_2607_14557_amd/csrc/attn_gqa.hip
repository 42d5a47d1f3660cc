// Attention with grouped heads over packed rows or pages.
#include <math.h>

#include "common.h"
#include "kernels.h"

namespace seer {

namespace {
__device__ __forceinline__ float to_f(const float* p) { return *p; }
__device__ __forceinline__ float to_f(const __bf16* p) { return static_cast<float>(*p); }
__device__ __forceinline__ float to_f(const _Float16* p) { return static_cast<float>(*p); }
}  // namespace

// One wave per row and head: 64 keys at a time, a key to a lane for the scores,
// a dim to a lane for the sums.
template <typename T, typename VT, bool PAGED>
__global__ __launch_bounds__(256) void gqa_rows_kernel(GqaParams p) {
  const int lane = threadIdx.x & (kWave - 1);
  const long long idx = (long long)blockIdx.x * 4 + (threadIdx.x >> 6);
  const int r = (int)(idx / p.n_heads), h = (int)(idx % p.n_heads), hk = h / (p.n_heads / p.n_kv);
  if (r >= p.rows_ub || r >= p.cu[p.B]) return;
  int lo = 0, hi = p.B - 1;
  while (lo < hi) {
    const int mid = (lo + hi) >> 1;
    if (p.cu[mid + 1] > r) hi = mid;
    else lo = mid + 1;
  }
  const int b = lo, i = r - p.cu[b];
  if (i < 0) return;
  int len = p.cu[b + 1] - p.cu[b];
  int used = p.used ? p.used[b] : len;
  used = used < 0 ? 0 : (used > len ? len : used);
  T* out = static_cast<T*>(p.out) + (size_t)r * p.o_stride + (size_t)h * p.head_dim;
  const int D = p.head_dim;
  float o[2] = {0.0f, 0.0f}, m = -INFINITY, l = 0.0f;
  if (i < used) {
    const int ps = 1 << p.shift;
    int nk = used;
    if (PAGED) {
      const long long most = (long long)p.width << p.shift;
      nk = p.kv_len[b];
      nk = nk < 0 ? 0 : (nk > most ? (int)most : nk);
    }
    const int past = nk - used, pos = past + i;
    const T* q = static_cast<const T*>(p.q) + (size_t)r * p.q_stride + (size_t)h * D;
    auto k_row = [&](int key, int page) {
      return PAGED ? static_cast<const T*>(p.k) + ((((size_t)page * 2) * p.n_kv + hk) * ps + (key & (ps - 1))) * D
                   : static_cast<const T*>(p.k) + (size_t)(p.cu[b] + key) * p.k_stride + (size_t)hk * D;
    };
    auto v_row = [&](int key, int page) {
      return PAGED ? static_cast<const VT*>(p.v) + ((((size_t)page * 2 + 1) * p.n_kv + hk) * ps + (key & (ps - 1))) * D
                   : static_cast<const VT*>(p.v) + (size_t)(p.cu[b] + key) * p.v_stride + (size_t)hk * D;
    };
    for (int k0 = 0; k0 < nk; k0 += kWave) {
      const int key = k0 + lane;
      int page = 0;
      bool see = key < nk;
      if (see && PAGED) {
        page = p.table[(size_t)b * p.width + (key >> p.shift)];
        see = page >= 0 && page < p.n_pages;
      }
      if (see && p.mask == kMaskCausal) see = key <= pos;
      if (see && p.mask == kMaskTree && key >= past) {
        const int j = key - past;
        see = j < 64 * p.words && (p.bits[(size_t)r * p.words + (j >> 6)] >> (j & 63) & 1);
      }
      float s = -INFINITY;
      if (see) {
        const T* k = k_row(key, page);
        float acc = 0.0f;
        for (int d = 0; d < D; ++d) acc = fmaf(to_f(q + d), to_f(k + d), acc);
        s = acc * p.scale;
      }
      const float m_new = fmaxf(m, wave_max(s));
      const unsigned long long any = __ballot(see);
      if (any == 0) continue;
      const float w = see ? expf(s - m_new) : 0.0f;
      const float a = m == -INFINITY ? 0.0f : expf(m - m_new);
      m = m_new;
      l = l * a + wave_sum(w);
      o[0] *= a;
      o[1] *= a;
      for (int t = 0; t < kWave; ++t) {
        if (!(any >> t & 1)) continue;
        const float wt = __shfl(w, t, kWave);
        const VT* v = v_row(k0 + t, __shfl(page, t, kWave));
#pragma unroll
        for (int e = 0; e < 2; ++e)
          if (lane + 64 * e < D) o[e] = fmaf(wt, to_f(v + lane + 64 * e), o[e]);
      }
    }
  }
#pragma unroll
  for (int e = 0; e < 2; ++e)
    if (lane + 64 * e < D) out[lane + 64 * e] = static_cast<T>(l == 0.0f ? 0.0f : o[e] / l);
}

int launch_gqa(const GqaParams& p, hipStream_t s) {
  const long long waves = (long long)p.rows_ub * p.n_heads;
  const dim3 grid((unsigned)((waves + 3) / 4)), block(256);
  auto go = [&](auto t, auto v) {
    if (p.table) hipLaunchKernelGGL((gqa_rows_kernel<decltype(t), decltype(v), true>), grid, block, 0, s, p);
    else hipLaunchKernelGGL((gqa_rows_kernel<decltype(t), decltype(v), false>), grid, block, 0, s, p);
  };
  if (!p.bf16) go(float{}, float{});
  else if (p.v_f16) go(__bf16{}, _Float16{});
  else go(__bf16{}, __bf16{});
  return hipGetLastError() == hipSuccess ? 0 : -1;
}

}  // namespace seer
