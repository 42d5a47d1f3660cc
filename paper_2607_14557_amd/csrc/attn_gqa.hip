// Attention with grouped heads over packed prompts and over pages, bf16 on the
// gfx950 matrix cores (head_dim 64 and 128; V in bf16 or fp16).
//
//   out_i = sum_j p_ij v_j,   p_ij = softmax_j(scale q_i . k_j) over the keys that row i sees
//
// in one pass over the keys with a running maximum and sum.  Scores are
// computed transposed, S^T = K Q^T (32x32x16 MFMA): a lane owns one row of
// queries, its statistics are per-lane values, its mask is one 64-bit word, and
// the probabilities already sit in the B-operand layout of O^T += V^T P^T.  K
// and V come by direct-to-LDS loads, V's operand by the LDS transpose read.
// Two forms:
//   gqa_tile_kernel  128 rows a workgroup, 32 a wave, K and V tiles of 64 keys shared by the four waves
//   gqa_few_kernel   32 rows a workgroup, the keys split over its two or four waves
// both over all of a tile's keys or, where there are few tiles, over a part of
// them; gqa_join_kernel then adds the parts.
//
// What bounds them, on an MI355X whose large copies reach 4.9 TB/s (5.9 read only)
// and whose 8192^3 products reach 1225 TFLOP/s in bf16:
//   many keys a row (14,416 rows, 32 heads on 8, 1500 to 8192 a prompt): the chain
//     inside a tile, scores, exponentials, products, with the matrix pipe half busy:
//     651 us, 1027 TFLOP/s
//   single tokens (64 requests of 500 to 16,000 keys, 28 heads on 4): the read of the
//     cache, 115 us, 5.3 TB/s
//   short prompts and windows: half the time is that chain, half what each workgroup
//     does once (its place in the call, queries, first keys, results): 9937 rows of 16
//     prompts, 32 heads, 136 us, 496 TFLOP/s
//   a few tiles (one token over 794 keys): the latency of two launches, 14 us
// Tried and slower: the join by the last workgroup to arrive in the first launch (one
// token 16 -> 42 us: the waits for stores to reach the other XCDs), workgroups of 1024
// for the join, and a join of the records in use alone (their search costs what the
// empty workgroups do).  Without effect: raised wave priority around the products,
// the requests summed by lanes instead of through LDS.
#include <type_traits>

#include "gqa.h"

namespace seer {

namespace {

typedef short v4i16_t __attribute__((ext_vector_type(4)));
typedef __attribute__((address_space(3))) v4i16_t lds_v4i16_t;

constexpr int NT = 256;

// LDS tiles hold a key per row of DH * 2 bytes, in 16-byte pieces whose place is
// exchanged so that the reads of a fragment meet distinct banks: piece c of row r
// of K at c ^ swz_k(r), of V at c ^ swz_v(r).
template <int DH>
__device__ __forceinline__ int swz_k(int r) { return DH == 128 ? r & 15 : (r >> 1) & 7; }
template <int DH>
__device__ __forceinline__ int swz_v(int r) { return DH == 128 ? 4 * (r & 3) : 4 * ((r >> 1) & 1); }

// Where 16 consecutive keys (a multiple of 16 on) lie: a page holds them all.
struct KeyRows {
  const uint8_t* k;
  const uint8_t* v;
  size_t step_k, step_v;       // bytes from key to key
};

template <int DH, bool PAGED>
struct KeySource {
  const uint8_t* k;            // packed: the head's first key; paged: the pool
  const uint8_t* v;
  size_t step_k, step_v;
  const int* table;            // the request's row
  int shift, n_pages, hk, n_kv;

  __device__ __forceinline__ KeySource(const GqaParams& p, const GqaUnit& u) {
    if constexpr (PAGED) {
      k = static_cast<const uint8_t*>(p.k);
      v = k;
      step_k = step_v = DH * 2;
      table = p.table + (size_t)u.b * p.width;
      shift = p.shift;
      n_pages = p.n_pages;
      hk = u.hk;
      n_kv = p.n_kv;
    } else {
      step_k = (size_t)p.k_stride * 2;
      step_v = (size_t)p.v_stride * 2;
      k = static_cast<const uint8_t*>(p.k) + (size_t)u.s.s0 * step_k + u.hk * (DH * 2);
      v = static_cast<const uint8_t*>(p.v) + (size_t)u.s.s0 * step_v + u.hk * (DH * 2);
    }
  }
  // the page of key g (one below the request's end)
  __device__ __forceinline__ int page(int g) const { return PAGED ? scalar_load(table, g >> shift) : 0; }
  __device__ __forceinline__ bool held(int id) const { return !PAGED || (id >= 0 && id < n_pages); }
  __device__ __forceinline__ KeyRows rows(int g, int id) const {
    if constexpr (PAGED) {
      const size_t half = (size_t)n_kv << shift;
      const size_t r = (size_t)(held(id) ? id : 0) * 2 * half + ((size_t)hk << shift) + (g & ((1 << shift) - 1));
      return {k + r * (DH * 2), k + (r + half) * (DH * 2), DH * 2, DH * 2};
    } else {
      return {k + (size_t)g * step_k, v + (size_t)g * step_v, step_k, step_v};
    }
  }
};

// Loads of 16 keys of K and V into their rows of the LDS tiles.  The lane adds to a
// group's address its row of a load, and the piece of the row that the exchange
// puts at its place (the same for every load of V).
template <int DH>
struct KeyLoads {
  static constexpr int ROW = DH * 2, RPL = 1024 / ROW, LPR = ROW / 16;      // rows of a load, lanes of a row
  uint32_t at_k[16 / RPL], at_v;
  int lane;
  __device__ __forceinline__ KeyLoads(size_t step_k, size_t step_v, int lane_) : lane(lane_) {
    const int r = lane / LPR, c = lane % LPR;
#pragma unroll
    for (int q = 0; q < 16 / RPL; ++q)
      at_k[q] = (RPL * q + r) * (uint32_t)step_k + ((uint32_t)(c ^ swz_k<DH>(RPL * q + r)) << 4);
    at_v = r * (uint32_t)step_v + ((uint32_t)(c ^ swz_v<DH>(r)) << 4);
  }
  // keys past `last` are the last one again
  __device__ __forceinline__ void issue(const KeyRows& src, int last, uint8_t* kd, uint8_t* vd) const {
    const __amdgpu_buffer_rsrc_t rk = __builtin_amdgcn_make_buffer_rsrc(const_cast<uint8_t*>(src.k), 0, -1, 0x00020000);
    const __amdgpu_buffer_rsrc_t rv = __builtin_amdgcn_make_buffer_rsrc(const_cast<uint8_t*>(src.v), 0, -1, 0x00020000);
    const uint32_t sk = (uint32_t)src.step_k, sv = (uint32_t)src.step_v;
#pragma unroll
    for (int q = 0; q < 16 / RPL; ++q) {
      uint32_t ok = at_k[q], ov = at_v + RPL * q * sv;
      if (last < 15) {
        const int r = RPL * q + lane / LPR, less = r > last ? r - last : 0;
        ok -= less * sk;
        ov -= less * sv;
      }
      __builtin_amdgcn_raw_ptr_buffer_load_lds(rk, (lds_void_t*)(kd + RPL * q * ROW), 16, ok, 0, 0, 0);
      __builtin_amdgcn_raw_ptr_buffer_load_lds(rv, (lds_void_t*)(vd + RPL * q * ROW), 16, ov, 0, 0, 0);
    }
  }
};

// Values that are no numbers (NaN, infinities) under a mask: the product would
// carry them to rows that do not see their keys, as 0 * value.  So the tiles in
// which some row is blind to a key are swept before they are used (each wave the
// keys that it loaded itself): such values become zeros there, and after the last
// tile add_odd adds them to the rows that do see them.  Returns whether there were any.
template <bool VF16, int BYTES>
__device__ __forceinline__ bool sweep(uint8_t* tile, int lane) {
  constexpr uint32_t EXPO = VF16 ? 0x7c007c00u : 0x7f807f80u, LOW = VF16 ? 0x04000400u : 0x00800080u;
  bool odd = false;
#pragma unroll
  for (int i = 0; i < BYTES / 1024; ++i) {
    u32x4_t* at = reinterpret_cast<u32x4_t*>(tile + i * 1024 + lane * 16);
    u32x4_t v = *at;
    bool any = false;
#pragma unroll
    for (int e = 0; e < 4; ++e) {
      // an exponent of all ones carries into the bit above it
      const uint32_t full = ((v[e] & EXPO) + LOW) & 0x80008000u;
      any |= full != 0;
      v[e] &= ~((full >> 15) * 0xffffu);
    }
    if (any) *at = v;
    odd |= any;
  }
  return __any(odd);
}

// A wave's 32 rows against NI groups of 32 keys.  FINE: the probabilities as a sum
// of two bf16 values, for where the matrix instructions are not what bounds.
template <int DH, bool VF16, int NI, bool FINE>
struct Rows32 {
  static constexpr int ROW = DH * 2, KS = DH / 16, DT = DH / 32;
  using vfrag_t = typename std::conditional<VF16, f16x8_t, bf16x8_t>::type;
  bf16x8_t qf[KS];
  f32x16_t o[DT];
  float m, l;                  // reference maximum (of unscaled scores) and this lane's half of the sum
  float c;                     // scale * log2(e)

  __device__ __forceinline__ void init(const GqaParams& p, const uint16_t* q, int lane) {
#pragma unroll
    for (int ks = 0; ks < KS; ++ks)
      qf[ks] = __builtin_bit_cast(bf16x8_t, *reinterpret_cast<const u32x4_t*>(q + 16 * ks + 8 * (lane >> 5)));
#pragma unroll
    for (int i = 0; i < DT; ++i)
#pragma unroll
      for (int r = 0; r < 16; ++r) o[i][r] = 0.0f;
    m = -INFINITY;
    l = 0.0f;
    c = p.scale * 1.4426950408889634f;
  }

  __device__ __forceinline__ static f32x16_t mfma_v(vfrag_t a, u32x4_t b, f32x16_t acc) {
    if constexpr (VF16) return __builtin_amdgcn_mfma_f32_32x32x16_f16(a, __builtin_bit_cast(f16x8_t, b), acc, 0, 0, 0);
    else return __builtin_amdgcn_mfma_f32_32x32x16_bf16(a, __builtin_bit_cast(bf16x8_t, b), acc, 0, 0, 0);
  }

  // One tile: keys fr and 32 + fr at kl, V at vl.  `masked` (the same for the whole
  // wave): this lane's row sees the keys of `seen` only.
  __device__ __forceinline__ void step(const uint8_t* kl, const uint8_t* vl, int lane, bool masked,
                                       unsigned long long seen) {
    const int fr = lane & 31, fhalf = lane >> 5;
    f32x16_t s[NI];
#pragma unroll
    for (int i = 0; i < NI; ++i)
#pragma unroll
      for (int r = 0; r < 16; ++r) s[i][r] = 0.0f;
    {
      const uint8_t* krow = kl + fr * ROW;
      auto kread = [&](int ks, bf16x8_t* dst) {
        const int ch = (2 * ks + fhalf) ^ swz_k<DH>(fr);
#pragma unroll
        for (int i = 0; i < NI; ++i)
          dst[i] = __builtin_bit_cast(bf16x8_t, *reinterpret_cast<const u32x4_t*>(krow + i * 32 * ROW + ch * 16));
      };
      bf16x8_t kf[2][NI];
      __builtin_amdgcn_sched_barrier(0);
      kread(0, kf[0]);
      __builtin_amdgcn_sched_barrier(0);
#pragma unroll
      for (int ks = 0; ks < KS; ++ks) {
        if (ks + 1 < KS) kread(ks + 1, kf[(ks + 1) & 1]);
#pragma unroll
        for (int i = 0; i < NI; ++i)
          s[i] = __builtin_amdgcn_mfma_f32_32x32x16_bf16(kf[ks & 1][i], qf[ks], s[i], 0, 0, 0);
        if (ks + 1 < KS) __builtin_amdgcn_sched_group_barrier(0x100, NI, 0);
        __builtin_amdgcn_sched_group_barrier(0x008, NI, 0);
      }
      __builtin_amdgcn_sched_barrier(0);
    }
    // element r of s[i] is key 32 i + 8 (r / 4) + 4 fhalf + r % 4
    if (masked) {
      const unsigned long long mine = seen >> (4 * fhalf);
      const uint32_t half[2] = {(uint32_t)mine, (uint32_t)(mine >> 32)};
#pragma unroll
      for (int i = 0; i < NI; ++i)
#pragma unroll
        for (int r = 0; r < 16; ++r)
          if (!(half[i] >> (8 * (r >> 2) + (r & 3)) & 1)) s[i][r] = -INFINITY;
    }
    // Probabilities against the reference maximum, rounded to V's type (half a step:
    // bf16 2^-8, fp16 2^-11; the two bf16 values of FINE 2^-16) as the matrix
    // instruction takes them, and their sum in fp32, over the rounded values where
    // they are coarse, so that the weights add up to one.
    u32x4_t pf[2 * NI], pl[FINE ? 2 * NI : 1];
    float lsum;
    auto probs = [&](float ref) {
      // fp16: all 2^10 times as large, so that those down to 2^-24 of the reference are
      // normal numbers; bf16: 2^-16, so that none passes 1 before the reference moves (it
      // goes with the division by their sum)
      const float mc = VF16 ? ref * c - 10.0f : ref * c + 16.0f;
      lsum = 0.0f;
#pragma unroll
      for (int sl = 0; sl < 2 * NI; ++sl)
#pragma unroll
        for (int e = 0; e < 4; ++e) {
          const float p0 = __builtin_amdgcn_exp2f(s[sl >> 1][(sl & 1) * 8 + 2 * e] * c - mc);
          const float p1 = __builtin_amdgcn_exp2f(s[sl >> 1][(sl & 1) * 8 + 2 * e + 1] * c - mc);
          if constexpr (VF16) {
            const f16x2_t h = __builtin_convertvector(f32x2_t{p0, p1}, f16x2_t);
            lsum = __builtin_amdgcn_fdot2(h, f16x2_t{(_Float16)1.0f, (_Float16)1.0f}, lsum, false);
            pf[sl][e] = __builtin_bit_cast(uint32_t, h);
          } else if constexpr (FINE) {
            // the upper halves as they are, so that what is left is not negative; 2^-20 of
            // the whole keeps it above zero, as an infinite value times zero would be none
            const uint32_t b0 = __float_as_uint(p0), b1 = __float_as_uint(p1);
            lsum += p0 + p1;
            pf[sl][e] = __builtin_amdgcn_perm(b1, b0, 0x07060302u);
            pl[sl][e] = pack_bf2(__builtin_fmaf(p0, 1.0f + 0x1p-20f, -__uint_as_float(b0 & 0xffff0000u)),
                                 __builtin_fmaf(p1, 1.0f + 0x1p-20f, -__uint_as_float(b1 & 0xffff0000u)));
          } else {
            const bf16x2_t h = __builtin_convertvector(f32x2_t{p0, p1}, bf16x2_t);
            lsum = __builtin_amdgcn_fdot2_f32_bf16(h, bf16x2_t{(__bf16)1.0f, (__bf16)1.0f}, lsum, false);
            pf[sl][e] = __builtin_bit_cast(uint32_t, h);
          }
        }
    };
    // The reference is the maximum of the first tile in which the row sees a key, and
    // moves only where a later tile's probabilities pass fp16's range (2^6 of the
    // reference) or, with bf16, add up to 2^16 of it in a lane: any reference gives the
    // same softmax, and the common tile takes no maximum.  With bf16 the sums of large
    // values stay in fp32's range, as a lane's 16 or 32 keys of a tile count for less than 1
    // together (a limit of 2^6 without the factor did that too, and took 7% longer where
    // scores spread by 4).  While a row has seen no key its reference is -inf, and the NaN
    // or infinity that this gives (-inf + inf, x + inf) asks for the tile's maximum too.
    probs(m);
    if (__any(!(lsum < (VF16 ? INFINITY : 1.0f)))) {
      float mt = s[0][0];
#pragma unroll
      for (int i = 0; i < NI; ++i)
#pragma unroll
        for (int r = 0; r < 16; ++r) mt = fmaxf(mt, s[i][r]);
      // lanes l and l ^ 32 hold the two halves of a row's keys
      const u32x2_t sw = __builtin_amdgcn_permlane32_swap(__float_as_uint(mt), __float_as_uint(mt), false, false);
      mt = fmaxf(__uint_as_float(sw[0]), __uint_as_float(sw[1]));
      const float m_new = fmaxf(m, mt);
      const float alpha = m == -INFINITY ? 1.0f : __builtin_amdgcn_exp2f((m - m_new) * c);
      m = m_new;
      l *= alpha;
#pragma unroll
      for (int i = 0; i < DT; ++i)
#pragma unroll
        for (int r = 0; r < 16; ++r) o[i][r] *= alpha;
      probs(m == -INFINITY ? 0.0f : m);
    }
    l += lsum;

    // A operand of step n (16-key slice sl, 32-dim tile dt): lane l needs 8 keys of
    // dim 32 dt + l % 32, in the order of the P fragment.  In each group of 16 lanes
    // the transpose read hands lane j element j % 4 of lanes 4 e + j / 4, e < 4.
    const int il = lane & 15;
    const int vkey = 4 * fhalf + (il >> 2);
    const int vc8 = 4 * ((lane >> 4) & 1) + (il & 3);
    const uint8_t* vrow = vl + vkey * ROW;
    auto vread = [&](int n) {
      const int sl = n / DT, dt = n % DT;
      const uint8_t* a = vrow + 16 * sl * ROW + (((8 * dt + vc8) ^ (2 * swz_v<DH>(vkey))) << 3);
      const v4i16_t lo = __builtin_amdgcn_ds_read_tr16_b64_v4i16((lds_v4i16_t*)a);
      const v4i16_t hi = __builtin_amdgcn_ds_read_tr16_b64_v4i16((lds_v4i16_t*)(a + 8 * ROW));
      return __builtin_shufflevector(lo, hi, 0, 1, 2, 3, 4, 5, 6, 7);
    };
    constexpr int STEPS = 2 * NI * DT;
    vfrag_t vf[3];
    __builtin_amdgcn_sched_barrier(0);
    vf[0] = __builtin_bit_cast(vfrag_t, vread(0));
    vf[1] = __builtin_bit_cast(vfrag_t, vread(1));
    __builtin_amdgcn_sched_barrier(0);
#pragma unroll
    for (int n = 0; n < STEPS; ++n) {
      if (n + 2 < STEPS) vf[(n + 2) % 3] = __builtin_bit_cast(vfrag_t, vread(n + 2));
      o[n % DT] = mfma_v(vf[n % 3], pf[n / DT], o[n % DT]);
      if constexpr (FINE) o[n % DT] = mfma_v(vf[n % 3], pl[n / DT], o[n % DT]);
      if (n + 2 < STEPS) __builtin_amdgcn_sched_group_barrier(0x100, 2, 0);
      __builtin_amdgcn_sched_group_barrier(0x008, FINE ? 2 : 1, 0);
    }
    __builtin_amdgcn_sched_barrier(0);
  }
};

// 1 / l, and 0 for a row that saw no key (its sums are zero); a NaN stays one.
__device__ __forceinline__ float inverse(float l) { return l == 0.0f ? 0.0f : 1.0f / l; }

// v (four dims from `dim` on) with what the swept values do to a row: keys from
// `from` to the unit's end.  Those of tiles that were not swept have done it
// already; an infinity or a NaN added again changes nothing.
template <int DH, bool VF16, bool PAGED>
__device__ __forceinline__ f32x4_t add_odd(f32x4_t v, const KeySource<DH, PAGED>& keys, const GqaUnit& u,
                                           const GqaSight<PAGED>& sight, int from, int dim) {
  for (int k0 = from; k0 < u.hi; k0 += 16) {
    const int id = keys.page(k0);
    if (!keys.held(id)) continue;
    const KeyRows src = keys.rows(k0, id);
    const uint32_t seen = (uint32_t)sight.seen(k0) & 0xffffu;
    for (int i = 0; i < 16 && k0 + i < u.hi; ++i) {
      const uint16_t* at = reinterpret_cast<const uint16_t*>(src.v + i * src.step_v) + dim;
#pragma unroll
      for (int e = 0; e < 4; ++e) {
        const float x = VF16 ? (float)__builtin_bit_cast(_Float16, at[e]) : bf2f(at[e]);
        if ((seen >> i & 1) && !(fabsf(x) < INFINITY)) v[e] += x;
      }
    }
  }
  return v;
}

// Where unit (slot) leaves its result: per 32 rows and 32 dims 4 x 64 lanes x 16
// bytes as the lanes hold them, then the rows' maxima and sums.
template <int RT, int DH>
struct Parts {
  static constexpr size_t FLOATS = RT * (DH + 2);
  float* base;
  __device__ __forceinline__ Parts(const GqaParams& p, int slot) : base(p.partial + (size_t)slot * FLOATS) {}
  __device__ __forceinline__ f32x4_t* sum(int w, int dt, int g, int lane) const {
    return reinterpret_cast<f32x4_t*>(base) + (((w * (DH / 32) + dt) * 4 + g) * 64 + lane);
  }
  __device__ __forceinline__ float* max(int row) const { return base + RT * DH + row; }
  __device__ __forceinline__ float* div(int row) const { return base + RT * (DH + 1) + row; }
};

__device__ __forceinline__ uint16_t* out_row(const GqaParams& p, int row, int head, int dh) {
  return static_cast<uint16_t*>(p.out) + (size_t)row * p.o_stride + (size_t)head * dh;
}

__device__ __forceinline__ void store4(uint16_t* at, f32x4_t v) {
  uint2 w;
  w.x = pack_bf2(v[0], v[1]);
  w.y = pack_bf2(v[2], v[3]);
  *reinterpret_cast<uint2*>(at) = w;
}

}  // namespace

// 128 rows: K and V of 64 keys are in LDS twice (64 KB at head_dim 128), one tile
// under way while the other is used, two workgroups a CU.  A step of 64 keys takes
// 1.27 us alone and 1.84 us with both, 0.92 each, of which the matrix instructions
// are a half: the other workgroup fills the waits of the chain.  A third buffer
// would leave LDS for one workgroup only.
template <int DH, bool VF16, bool PAGED>
__global__ __launch_bounds__(NT, 2) void gqa_tile_kernel(GqaParams p) {
  constexpr int ROW = DH * 2, DT = DH / 32;
  __shared__ __attribute__((aligned(1024))) uint8_t k_lds0[64 * ROW];
  __shared__ __attribute__((aligned(1024))) uint8_t k_lds1[64 * ROW];
  __shared__ __attribute__((aligned(1024))) uint8_t v_lds0[64 * ROW];
  __shared__ __attribute__((aligned(1024))) uint8_t v_lds1[64 * ROW];
  __shared__ int odd_at[2];                  // the first tile that had values to sweep; pieces alternate
  __shared__ typename GqaCut<kGqaTile, NT>::Shared cut_lds;
  if (threadIdx.x < 2) odd_at[threadIdx.x] = INT_MAX;
  GqaCut<kGqaTile, NT> cut(p, cut_lds);
  GqaUnit u;
  for (int turn = 0; cut.next(p, u); turn ^= 1) {
  if (threadIdx.x == 0) odd_at[turn ^ 1] = INT_MAX;
  const int lane = threadIdx.x & 63;
  const int wv = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
  const int fr = lane & 31, fhalf = lane >> 5;
  const int row = u.t * kGqaTile + wv * 32 + fr;
  const int src = row < u.s.rows ? row : u.s.rows - 1;
  const int tok = gqa_token(p, src), head = src - tok * p.group;
  const GqaSight<PAGED> sight(p, u, tok);
  // where the workgroup's and the wave's rows begin to be blind to some keys, and
  // where the wave's last row sees no more
  const int open_all = gqa_open_end(p, u, gqa_token(p, u.t * kGqaTile));
  const int open = gqa_open_end(p, u, gqa_token(p, u.t * kGqaTile + wv * 32));
  int end = u.hi;
  if (p.mask == kMaskCausal) end = u.s.past + gqa_token(p, u.t * kGqaTile + wv * 32 + 31) + 1;

  Rows32<DH, VF16, 2, false> w;
  w.init(p, static_cast<const uint16_t*>(p.q) + (size_t)(u.s.s0 + tok) * p.q_stride +
                (size_t)(u.hk * p.group + head) * DH, lane);

  const KeySource<DH, PAGED> keys(p, u);
  const KeyLoads<DH> loads(keys.step_k, keys.step_v, lane);
  const int n = (u.hi - u.lo + 63) / 64;
  int id[4];                                 // pages of the four 16-key groups of the next tile
  auto pages = [&](int kbase) {
#pragma unroll
    for (int i = 0; i < 4; ++i) {
      const int g = kbase + 16 * i;
      id[i] = keys.page(g < u.hi ? g : u.hi - 1);
    }
  };
  auto load = [&](int kbase, auto buf) {
    constexpr int B = decltype(buf)::value;
    int g = kbase + 16 * wv;                 // a group past the end is the last one again
    g = g < u.hi ? g : (u.hi - 1) & ~15;
    const int page = wv == 0 ? id[0] : (wv == 1 ? id[1] : (wv == 2 ? id[2] : id[3]));
    loads.issue(keys.rows(g, page), u.hi - 1 - g < 15 ? u.hi - 1 - g : 15, (B ? k_lds1 : k_lds0) + 16 * wv * ROW,
                (B ? v_lds1 : v_lds0) + 16 * wv * ROW);
  };
  // bits of the keys whose pages are none of the pool's
  unsigned long long lost = 0, lost_next = 0;
  auto lost_of = [&]() {
    unsigned long long m = 0;
    if constexpr (PAGED) {
#pragma unroll
      for (int i = 0; i < 4; ++i)
        if (!keys.held(id[i])) m |= 0xffffull << (16 * i);
    }
    return m;
  };
  // after this wave's part of a tile has landed, before the barrier that publishes it
  auto check = [&](int kbase, auto buf, unsigned long long lost) {
    constexpr int B = decltype(buf)::value;
    if (kbase + 64 <= open_all && lost == 0) return;
    if (sweep<VF16, 16 * ROW>((B ? v_lds1 : v_lds0) + 16 * wv * ROW, lane) && lane == 0) atomicMin(&odd_at[turn], kbase);
  };
  if (n > 0) {
    pages(u.lo);
    load(u.lo, std::integral_constant<int, 0>{});
    lost = lost_of();
    pages(u.lo + 64 < u.hi ? u.lo + 64 : u.hi - 1);
  }
  // every load so far (Q and tile 0) lands before the loop, so that the waits in it
  // are for the next tile alone
  __builtin_amdgcn_sched_barrier(0);
  __builtin_amdgcn_s_waitcnt(0x0f70);       // vmcnt(0)
  __builtin_amdgcn_sched_barrier(0);
  if (n > 0) check(u.lo, std::integral_constant<int, 0>{}, lost);
  __syncthreads();
  auto step = [&](int kt, auto buf) {
    constexpr int B = decltype(buf)::value;
    const int kbase = u.lo + 64 * kt;
    if (kt + 1 < n) {
      load(kbase + 64, std::integral_constant<int, B ^ 1>{});
      lost_next = lost_of();
      if (kt + 2 < n) pages(kbase + 128);
    }
    if (kbase < end) {
      const bool masked = kbase + 64 > open || lost != 0;
      unsigned long long seen = 0;
      if (masked) seen = ~lost & sight.seen(kbase);
      w.step(B ? k_lds1 : k_lds0, B ? v_lds1 : v_lds0, lane, masked, seen);
    }
    lost = lost_next;
    // this wave's loads of the next tile have landed, then one barrier publishes it
    __builtin_amdgcn_s_waitcnt(0x0f70);
    if (kt + 1 < n) check(kbase + 64, std::integral_constant<int, B ^ 1>{}, lost);
    __syncthreads();
  };
  for (int kt = 0; kt < n; kt += 2) {
    step(kt, std::integral_constant<int, 0>{});
    if (kt + 1 < n) step(kt + 1, std::integral_constant<int, 1>{});
  }

  f32x4_t sum[DT * 4];
#pragma unroll
  for (int i = 0; i < DT * 4; ++i)
#pragma unroll
    for (int e = 0; e < 4; ++e) sum[i][e] = w.o[i >> 2][4 * (i & 3) + e];
  const int odd = __builtin_amdgcn_readfirstlane(odd_at[turn]);
  if (odd < u.hi) {
#pragma unroll 1
    for (int i = 0; i < DT * 4; ++i) {
      // one copy of the code: the quadruples take turns at the front
      const f32x4_t v = add_odd<DH, VF16, PAGED>(sum[0], keys, u, sight, odd, 32 * (i >> 2) + 8 * (i & 3) + 4 * fhalf);
#pragma unroll
      for (int k = 0; k + 1 < DT * 4; ++k) sum[k] = sum[k + 1];
      sum[DT * 4 - 1] = v;
    }
  }
  const float l = w.l + __shfl_xor(w.l, 32, kWave);
  if (row >= u.s.rows) continue;
  if (!u.whole) {
    const Parts<kGqaTile, DH> to(p, u.slot);
#pragma unroll
    for (int i = 0; i < DT * 4; ++i) *to.sum(wv, i >> 2, i & 3, lane) = sum[i];
    if (fhalf == 0) {
      *to.max(wv * 32 + fr) = w.m;
      *to.div(wv * 32 + fr) = l;
    }
    continue;
  }
  const bool real = tok < u.s.used;
  const float inv = inverse(l);
  uint16_t* to = out_row(p, u.s.s0 + tok, u.hk * p.group + head, DH) + fhalf * 4;
#pragma unroll
  for (int i = 0; i < DT * 4; ++i) store4(to + (i >> 2) * 32 + (i & 3) * 8, real ? sum[i] * inv : f32x4_t{0, 0, 0, 0});
  }
}

// 32 rows: each wave walks 32 of every 32 NW keys by itself, its tiles of its own in
// LDS, without a barrier until the waves are joined, so that its loads never wait for
// another wave.  Cut lines have two waves, for more independent walks a CU; whole
// tiles four, for the shorter walk.
template <int DH, bool VF16, bool PAGED, int NW>
__global__ __launch_bounds__(64 * NW, 1) void gqa_few_kernel(GqaParams p) {
  constexpr int ROW = DH * 2, DT = DH / 32, FT = 32 * ROW;      // bytes of a wave's K or V tile
  constexpr int PW = DT * 4 / NW;                               // 8-dim pieces that a wave joins
  __shared__ __attribute__((aligned(1024))) uint8_t k_lds0[NW * FT];
  __shared__ __attribute__((aligned(1024))) uint8_t k_lds1[NW * FT];
  __shared__ __attribute__((aligned(1024))) uint8_t v_lds0[NW * FT];
  __shared__ __attribute__((aligned(1024))) uint8_t v_lds1[NW * FT];
  __shared__ float m_part[NW][32], l_part[NW][32];
  __shared__ int odd_from[NW];
  __shared__ typename GqaCut<kGqaFew, 64 * NW>::Shared cut_lds;
  GqaCut<kGqaFew, 64 * NW> cut(p, cut_lds);
  GqaUnit u;
  while (cut.next(p, u)) {
  const int lane = threadIdx.x & 63;
  const int wv = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
  const int fr = lane & 31, fhalf = lane >> 5;
  const int row = u.t * kGqaFew + fr;
  const int src = row < u.s.rows ? row : u.s.rows - 1;
  const int tok = gqa_token(p, src), head = src - tok * p.group;
  const GqaSight<PAGED> sight(p, u, tok);
  const int open = gqa_open_end(p, u, gqa_token(p, u.t * kGqaFew));

  Rows32<DH, VF16, 1, !VF16> w;
  w.init(p, static_cast<const uint16_t*>(p.q) + (size_t)(u.s.s0 + tok) * p.q_stride +
                (size_t)(u.hk * p.group + head) * DH, lane);

  const KeySource<DH, PAGED> keys(p, u);
  const KeyLoads<DH> loads(keys.step_k, keys.step_v, lane);
  // this wave's tiles: 32 of every 32 NW keys
  constexpr int STEP = 32 * NW;
  const int k0 = u.lo + 32 * wv;
  const int n = u.hi > k0 ? (u.hi - k0 + STEP - 1) / STEP : 0;
  int id[2];
  auto pages = [&](int kbase) {
#pragma unroll
    for (int i = 0; i < 2; ++i) {
      const int g = kbase + 16 * i;
      id[i] = keys.page(g < u.hi ? g : u.hi - 1);
    }
  };
  auto load = [&](int kbase, auto buf) {
    constexpr int B = decltype(buf)::value;
#pragma unroll
    for (int i = 0; i < 2; ++i) {
      int g = kbase + 16 * i;
      g = g < u.hi ? g : (u.hi - 1) & ~15;
      loads.issue(keys.rows(g, id[i]), u.hi - 1 - g < 15 ? u.hi - 1 - g : 15, (B ? k_lds1 : k_lds0) + wv * FT + 16 * i * ROW,
                  (B ? v_lds1 : v_lds0) + wv * FT + 16 * i * ROW);
    }
  };
  uint32_t lost[2] = {0, 0};
  auto lost_of = [&]() {
    uint32_t m = 0;
    if constexpr (PAGED) {
      if (!keys.held(id[0])) m |= 0xffffu;
      if (!keys.held(id[1])) m |= 0xffff0000u;
    }
    return m;
  };
  int odd = INT_MAX;
  constexpr int LOADS = 2 * 32 * ROW / 1024;            // of a tile
  if (n > 0) {
    pages(k0);
    load(k0, std::integral_constant<int, 0>{});
    lost[0] = lost_of();
    if (n > 1) {
      pages(k0 + STEP);
      load(k0 + STEP, std::integral_constant<int, 1>{});
      lost[1] = lost_of();
    }
    pages(k0 + 2 * STEP < u.hi ? k0 + 2 * STEP : u.hi - 1);
  }
  // Both buffers are under way; a tile's buffer is filled again as soon as the tile
  // is done, so that one to two tiles are in flight all the time.
  auto step = [&](int kt, auto buf) {
    constexpr int B = decltype(buf)::value;
    const int kbase = k0 + STEP * kt;
    uint8_t* vl = (B ? v_lds1 : v_lds0) + wv * FT;
    __builtin_amdgcn_sched_barrier(0);
    if (kt + 1 < n) __builtin_amdgcn_s_waitcnt(0x0f70 | (LOADS & 15) | (LOADS >> 4) << 14);    // vmcnt(LOADS)
    else __builtin_amdgcn_s_waitcnt(0x0f70);                                                    // vmcnt(0)
    __builtin_amdgcn_wave_barrier();
    __builtin_amdgcn_sched_barrier(0);
    const bool masked = kbase + 32 > open || lost[B] != 0;
    unsigned long long seen = 0;
    if (masked) {
      seen = ~lost[B] & sight.seen(kbase);
      if (sweep<VF16, FT>(vl, lane)) odd = kbase < odd ? kbase : odd;
    }
    w.step((B ? k_lds1 : k_lds0) + wv * FT, vl, lane, masked, seen);
    if (kt + 2 < n) {
      // this tile's fragments have been read
      __builtin_amdgcn_sched_barrier(0);
      __builtin_amdgcn_s_waitcnt(0xc07f);     // lgkmcnt(0)
      __builtin_amdgcn_wave_barrier();
      __builtin_amdgcn_sched_barrier(0);
      load(kbase + 2 * STEP, buf);
      lost[B] = lost_of();
      if (kt + 3 < n) pages(kbase + 3 * STEP);
    }
  };
  for (int kt = 0; kt < n; kt += 2) {
    step(kt, std::integral_constant<int, 0>{});
    if (kt + 1 < n) step(kt + 1, std::integral_constant<int, 1>{});
  }

  // join the waves: each leaves its sums in its own K tiles and takes PW pieces
  const float l_own = w.l + __shfl_xor(w.l, 32, kWave);
  if (fhalf == 0) {
    m_part[wv][fr] = w.m;
    l_part[wv][fr] = l_own;
  }
  if (lane == 0) odd_from[wv] = odd;
  auto sums = [&](int v, int at) {          // piece `at` of DT * 4 blocks of 1 KiB; a buffer has FT / 1024 of them
    return reinterpret_cast<f32x4_t*>((at >= FT / 1024 ? k_lds1 : k_lds0) + v * FT + at % (FT / 1024) * 1024 + lane * 16);
  };
#pragma unroll
  for (int at = 0; at < DT * 4; ++at)
    *sums(wv, at) = f32x4_t{w.o[at >> 2][4 * (at & 3)], w.o[at >> 2][4 * (at & 3) + 1], w.o[at >> 2][4 * (at & 3) + 2],
                            w.o[at >> 2][4 * (at & 3) + 3]};
  __syncthreads();
  float m = -INFINITY;
#pragma unroll
  for (int v = 0; v < NW; ++v) m = fmaxf(m, m_part[v][fr]);
  const float ref = m == -INFINITY ? 0.0f : m;
  float l = 0.0f;
  f32x4_t sum[PW];
#pragma unroll
  for (int i = 0; i < PW; ++i) sum[i] = f32x4_t{0, 0, 0, 0};
#pragma unroll
  for (int v = 0; v < NW; ++v) {
    // a wave whose keys the row does not see has no part
    const bool none = m_part[v][fr] == -INFINITY && l_part[v][fr] == 0.0f;
    const float a = none ? 0.0f : __builtin_amdgcn_exp2f((m_part[v][fr] - ref) * w.c);
    l += l_part[v][fr] * a;
#pragma unroll
    for (int i = 0; i < PW; ++i) sum[i] += a * *sums(v, wv * PW + i);
  }
  odd = odd_from[0];
#pragma unroll
  for (int v = 1; v < NW; ++v) odd = odd_from[v] < odd ? odd_from[v] : odd;
  odd = __builtin_amdgcn_readfirstlane(odd);
  if (odd < u.hi) {
#pragma unroll 1
    for (int i = 0; i < PW; ++i) {
      // one copy of the code: the quadruples take turns at the front
      const int at = wv * PW + i;
      const f32x4_t v = add_odd<DH, VF16, PAGED>(sum[0], keys, u, sight, odd & ~15, 32 * (at >> 2) + 8 * (at & 3) + 4 * fhalf);
#pragma unroll
      for (int k = 0; k + 1 < PW; ++k) sum[k] = sum[k + 1];
      sum[PW - 1] = v;
    }
  }
  if (row >= u.s.rows) continue;
  if (!u.whole) {
    const Parts<kGqaFew, DH> to(p, u.slot);
#pragma unroll
    for (int i = 0; i < PW; ++i) *to.sum(0, (wv * PW + i) >> 2, (wv * PW + i) & 3, lane) = sum[i];
    if (wv == 0 && fhalf == 0) {
      *to.max(fr) = m;
      *to.div(fr) = l;
    }
    continue;
  }
  const bool real = tok < u.s.used;
  const float inv = inverse(l);
  uint16_t* to = out_row(p, u.s.s0 + tok, u.hk * p.group + head, DH) + fhalf * 4;
#pragma unroll
  for (int i = 0; i < PW; ++i) {
    const int at = wv * PW + i;
    store4(to + (at >> 2) * 32 + (at & 3) * 8, real ? sum[i] * inv : f32x4_t{0, 0, 0, 0});
  }
  }
}

// Adds the parts of each tile whose keys were cut, by the records that its first
// part left: a wave takes 32 rows x 8 dims (16 bytes a lane).  Bound by the latency
// of two dependent reads, a record and its parts (6 us), with many 128-row parts by
// their bytes (104 tiles in 256 parts: 7 us).  4, 8 or 16 parts are under way at once.
template <int RT, int DH>
__global__ __launch_bounds__(NT) void gqa_join_kernel(GqaParams p) {
  constexpr int DT = DH / 32, PIECES = RT / 32 * DT;       // workgroups of a tile
  const int wg = blockIdx.x / PIECES, piece = blockIdx.x % PIECES;
  const GqaRecord r = static_cast<const GqaRecord*>(p.records)[wg];
  if (r.parts < 2) return;
  const int lane = threadIdx.x & 63, g = threadIdx.x >> 6, fr = lane & 31, fhalf = lane >> 5;
  const int w = piece / DT, dt = piece % DT;
  const int row = r.t * RT + w * 32 + fr;
  if (row >= r.rows) return;
  const float c = p.scale * 1.4426950408889634f;
  // the loads of several parts under way together
  float m = -INFINITY, l = 0.0f;
  f32x4_t sum = {0.0f, 0.0f, 0.0f, 0.0f};
  auto add = [&](int i0, auto width) {
    constexpr int W = decltype(width)::value;
    float pm[W], pl[W];
    f32x4_t v[W];
#pragma unroll
    for (int k = 0; k < W; ++k) {
      const Parts<RT, DH> from(p, gqa_slot(r, wg, i0 + k < r.parts ? i0 + k : r.parts - 1));
      pm[k] = *from.max(w * 32 + fr);
      pl[k] = *from.div(w * 32 + fr);
      v[k] = *from.sum(w, dt, g, lane);
    }
    float top = m;
#pragma unroll
    for (int k = 0; k < W; ++k) top = fmaxf(top, pm[k]);
    const float ref = top == -INFINITY ? 0.0f : top;
    const float keep = m == -INFINITY ? 1.0f : __builtin_amdgcn_exp2f((m - ref) * c);
    m = top;
    l *= keep;
    sum *= keep;
#pragma unroll
    for (int k = 0; k < W; ++k) {
      const bool none = i0 + k >= r.parts || (pm[k] == -INFINITY && pl[k] == 0.0f);
      const float a = none ? 0.0f : __builtin_amdgcn_exp2f((pm[k] - ref) * c);
      l += none ? 0.0f : pl[k] * a;
      sum += none ? f32x4_t{0, 0, 0, 0} : a * v[k];
    }
  };
  if (r.parts <= 4) add(0, std::integral_constant<int, 4>{});
  else if (RT == kGqaFew && r.parts <= 8) add(0, std::integral_constant<int, 8>{});
  else if constexpr (RT == kGqaTile)
    for (int i0 = 0; i0 < r.parts; i0 += 8) add(i0, std::integral_constant<int, 8>{});
  else
    for (int i0 = 0; i0 < r.parts; i0 += 16) add(i0, std::integral_constant<int, 16>{});
  const int tok = gqa_token(p, row), head = row - tok * p.group;
  const float inv = inverse(l);
  store4(out_row(p, r.s0 + tok, r.hk * p.group + head, DH) + dt * 32 + g * 8 + fhalf * 4,
         tok < r.used ? sum * inv : f32x4_t{0, 0, 0, 0});
}

int launch_gqa_bf16(const GqaParams& p, const GqaRule& r, hipStream_t s) {
  auto go = [&](auto dh, auto vf16, auto paged) {
    constexpr int DH = decltype(dh)::value;
    constexpr bool V = decltype(vf16)::value, P = decltype(paged)::value;
    if (r.rt == kGqaTile) {
      hipLaunchKernelGGL((gqa_tile_kernel<DH, V, P>), dim3(r.grid), dim3(NT), 0, s, p);
      if (r.cut) hipLaunchKernelGGL((gqa_join_kernel<kGqaTile, DH>), dim3(r.grid * (4 * DH / 32)), dim3(NT), 0, s, p);
    } else if (r.cut) {
      hipLaunchKernelGGL((gqa_few_kernel<DH, V, P, 2>), dim3(r.grid), dim3(128), 0, s, p);
      hipLaunchKernelGGL((gqa_join_kernel<kGqaFew, DH>), dim3(r.grid * (DH / 32)), dim3(NT), 0, s, p);
    } else {
      hipLaunchKernelGGL((gqa_few_kernel<DH, V, P, 4>), dim3(r.grid), dim3(256), 0, s, p);
    }
  };
  auto with = [&](auto dh, auto vf16) {
    if (p.table) go(dh, vf16, std::true_type{});
    else go(dh, vf16, std::false_type{});
  };
  if (p.head_dim == 128) {
    if (p.v_f16) with(std::integral_constant<int, 128>{}, std::true_type{});
    else with(std::integral_constant<int, 128>{}, std::false_type{});
  } else {
    if (p.v_f16) with(std::integral_constant<int, 64>{}, std::true_type{});
    else with(std::integral_constant<int, 64>{}, std::false_type{});
  }
  return hipGetLastError() == hipSuccess ? 0 : -1;
}

}  // namespace seer
