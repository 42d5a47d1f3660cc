// The attention weight that the rows of a call give to each cached token:
//
//   w_j = decay prev_j + sum over rows i and heads h of the group of p_ihj,
//   p_ihj = exp(s_ihj - lse_ih),  s = scale q . k,  lse_ih = log sum_j exp(s_ihj) over the keys that row i sees
//
// per key/value head.  A row's sum is known when all its keys have been seen, so there are
// two passes; each weight is added up by one wave, or by one for each part of the rows and
// then part after part: no atomics, the same bits every time.  A lane adds a tile's rows up by
// themselves and then to its sum: thousands of equal terms, one after the other, end off by as many
// half steps to one side.  Three forms, by the call's bounds (dispatch.h):
//
//   bf16, many rows   weights_stats_tile_kernel: 128 rows stay in registers, keys pass by in
//                     LDS tiles of 64 (S^T = K Q^T, a lane owns a row); where the rows' tiles
//                     are few, each takes a part of the keys.  weights_sum_tile_kernel: the
//                     rows' parts joined, 128 keys stay, rows pass by (S = Q K^T, a lane owns
//                     a key and adds up its rows in a register); where those tiles are few,
//                     each takes a part of the rows and weights_join_kernel adds the parts.  The scores are
//                     made twice: 4 bytes a score, written and read, would take 170 us of the
//                     windows below where the second product takes 30.
//   bf16, few rows    weights_scores_kernel reads the keys once and keeps the scores, which are
//                     fewer bytes than the keys; weights_few_kernel makes the weights of them.
//   fp32              weights_stats_kernel and weights_sum_kernel, tiles of 16 x 16 a wave.
//
// Measured (MI355X, us a call among others; in brackets its kernels, medians of 30 passes in the
// profiler, together up to a tenth more): 3076 rows of 16 requests over 793 cached keys each and
// their own, 32 heads: 103 to 111 over machines (53 and 65, at least 50 and 60); 64 rows each of 7
// prompts of 1500 to 8192 tokens, 32 heads on 8: 58 (30 and 33); a token of 64 requests over 294,950
// keys, 28 heads on 4: 90 (68, which read the keys at 4.4 TB/s, and 14); one token over 794 keys: 12
// (7 and 6); trees of drafted tokens in fp32 over 1198 keys: 18.3 (7.5 and 11.6); all 32,267 rows of
// 7 prompts, 32 heads on 8, 1.5 TFLOP: 2140 (700 TFLOP/s).
#include <limits.h>

#include <type_traits>

#include "gqa.h"

namespace seer {

namespace {

constexpr int NT = 256, WAVES = NT / kWave;

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

// Maximum and sum over the 32 lanes of a half of the wave, in all of them.
template <typename Op>
__device__ __forceinline__ float half_reduce(float v, Op op) {
  auto turn = [&](auto ctrl) {                   // around the row of 16
    return __int_as_float(__builtin_amdgcn_update_dpp(0, __float_as_int(v), decltype(ctrl)::value, 0xf, 0xf, false));
  };
  v = op(v, turn(std::integral_constant<int, 0x128>{}));
  v = op(v, turn(std::integral_constant<int, 0x124>{}));
  v = op(v, turn(std::integral_constant<int, 0x122>{}));
  v = op(v, turn(std::integral_constant<int, 0x121>{}));
  return op(v, __shfl_xor(v, 16, kWave));
}

// Keys of a part: the parts of a request are equal, whole blocks of 64 keys, `least` or more.
__device__ __forceinline__ int part_keys(const WeightsParams& p, int nk, int least = 1) {
  const int blocks = ((nk + 63) / 64 + p.parts - 1) / p.parts;
  return (blocks > least ? blocks : least) * 64;
}

// The units of a launch: those of request after request in one line, whose ends each
// workgroup finds for itself.  Where there are few requests, what is known of each is kept
// with them.
constexpr int kKept = 128;
struct Line {
  int* end;              // [B] inclusive sums of the requests' units
  int* rows;             // [B] and of their rows that count
  Seq* kept;             // [B], B <= kKept
  int all;
  int chunk;             // blocks of 64 keys of a unit of the scores, at least
  __device__ __forceinline__ Seq seq(const WeightsParams& p, int b) const {
    Seq s;
    if (p.B <= kKept) s = kept[b];
    else s = seq_of(p, b);
    auto uni = [](int v) { return __builtin_amdgcn_readfirstlane(v); };
    return Seq{uni(s.row0), uni(s.rows), uni(s.index0), uni(s.used), uni(s.nk), uni(s.past)};
  }
};

// units(seq, chunk): units of a request.  CHUNK: whether all blocks of keys are counted
// first, so that units of `chunk` of them are about two for each workgroup that runs at once.
// Row offsets that fall are no call: there are no units then, as rows would be counted twice
// and the workspace has room for each once.
template <bool CHUNK, typename Units>
__device__ __forceinline__ Line line_of(const WeightsParams& p, int* lds, Units units) {
  __shared__ int sums[2][WAVES];
  __shared__ float blocks_lds[WAVES];
  Line l{lds, lds + p.B, reinterpret_cast<Seq*>(lds + 2 * p.B), 0, 2};
  const int tid = threadIdx.x, lane = tid & (kWave - 1), wave = tid >> 6;
  const int per = (p.B + NT - 1) / NT;
  const int b0 = tid * per < p.B ? tid * per : p.B;
  const int b1 = b0 + per < p.B ? b0 + per : p.B;
  Seq only{};                                    // of the thread's first request, read once
  float blocks = 0.0f;
  for (int b = b0; b < b1; ++b) {
    const Seq s = seq_of(p, b);
    if (b == b0) only = s;
    if (p.B <= kKept) l.kept[b] = s;
    blocks += (float)((s.rows + 31) / 32) * (float)((s.nk + 63) / 64);
  }
  if (CHUNK) {
    blocks = wave_sum(blocks);
    if (lane == 0) blocks_lds[wave] = blocks;
    __syncthreads();
    float all = 0.0f;
#pragma unroll
    for (int w = 0; w < WAVES; ++w) all += blocks_lds[w];
    const float want = all * p.n_kv * (1.0f / 2048.0f);
    if (want > 2.0f) l.chunk = __builtin_amdgcn_readfirstlane((int)want + 1);
  }
  int n = 0, m = 0;
  bool falls = false;
  for (int b = b0; b < b1; ++b) {
    const Seq s = b == b0 ? only : seq_of(p, b);
    n += units(s, l.chunk);
    m += s.used;
    falls |= p.cu[b + 1] < p.cu[b];
  }
  const bool none = __any(falls);
  const int in = wave_scan(n), im = wave_scan(m);
  if (lane == kWave - 1) { sums[0][wave] = in; sums[1][wave] = none ? -1 : im; }
  __syncthreads();
  int on = in - n, om = im - m, all = 0;
#pragma unroll
  for (int w = 0; w < WAVES; ++w) {
    if (w < wave) { on += sums[0][w]; om += sums[1][w]; }
    all += sums[0][w];
    falls |= sums[1][w] < 0;
  }
  l.all = falls ? 0 : all;
  for (int b = b0; b < b1; ++b) {
    const Seq s = b == b0 ? only : seq_of(p, b);
    on += units(s, l.chunk);
    om += s.used;
    l.end[b] = on;
    l.rows[b] = om;
  }
  __syncthreads();
  return l;
}

// The line of a launch on tiles: where the heads divide by the 8 XCDs, each XCD has heads
// of its own and a line of them, so that the units of a head, which read the same keys or
// rows, run side by side and find them in its L2; otherwise all workgroups share one line.
struct Share {
  int heads, head0, first, step;
  __device__ __forceinline__ Share(int n_kv) {
    const bool own = n_kv % 8 == 0;              // (the grid is a multiple of 8)
    heads = own ? n_kv / 8 : n_kv;
    head0 = own ? (blockIdx.x & 7) * heads : 0;
    first = own ? blockIdx.x >> 3 : blockIdx.x;
    step = own ? gridDim.x >> 3 : gridDim.x;
  }
};

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

__device__ __forceinline__ int token_of(const WeightsParams& p, int x) {
  return (int)((__umulhi((unsigned)x, p.group_mul) + (unsigned)x) >> p.group_shift);
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

// Which of the 32 keys from k0 on a row of the request (with its heads) sees, a lane a row, so
// that the tree's words of all rows are on their way together.
__device__ __forceinline__ uint32_t window(const WeightsParams& p, const Seq& s, int row, int k0) {
  const int tok = token_of(p, row < s.rows ? row : s.rows - 1);
  auto first = [](int n) { return n <= 0 ? 0u : (n >= 32 ? ~0u : (1u << n) - 1); };
  uint32_t x = first(s.nk - k0);
  if (p.mask == kMaskCausal) x &= first(s.past + s.index0 + tok + 1 - k0);
  if (p.mask == kMaskTree) {
    const int before = s.past - k0, at = before < 0 ? -before : 0, word = at >> 6, shift = at & 63;
    const unsigned long long* bits = p.bits + (size_t)(s.row0 + tok) * p.words;
    const unsigned long long b0 = word < p.words ? bits[word] : 0, b1 = word + 1 < p.words ? bits[word + 1] : 0;
    const uint32_t own = (uint32_t)(b0 >> shift | (shift ? b1 << (64 - shift) : 0));
    if (before < 32) x &= first(before) | (before > 0 ? own << before : own);
  }
  return x;
}

// What the place of a score that its row does not see holds among the kept ones.  No product of bf16
// rows gives these bits: a NaN of theirs has the upper 16 of an operand's, or the default ones.
constexpr uint32_t kUnseen = 0xffffffffu;

__device__ __forceinline__ float scale_of(const WeightsParams& p) { return p.scale * 1.4426950408889634f; }

// Where the statistics of a request's rows for a key/value head begin: request after request, in each head
// after head, in each row after row.
__device__ __forceinline__ long long stat_row(const WeightsParams& p, const Line& l, const Seq& s, int b, int hk) {
  return (long long)(l.rows[b] - s.used) * p.n_heads + (long long)hk * s.rows;
}

// log2 of a row's sum, from its parts, eight of which are on their way together.
struct Parts {
  f32x2_t x[8];
  __device__ __forceinline__ void load(const f32x2_t* from, int parts) {
#pragma unroll
    for (int k = 0; k < 8; ++k) x[k] = from[k < parts ? k : parts - 1];
  }
  __device__ __forceinline__ void add(int parts, float& top, float& sum) const {
    float to = top;
#pragma unroll
    for (int k = 0; k < 8; ++k) to = fmaxf(to, x[k][0]);
    const float ref = to == -INFINITY ? 0.0f : to;
    sum *= __builtin_amdgcn_exp2f(top - ref);
#pragma unroll
    for (int k = 0; k < 8; ++k) sum += k < parts ? x[k][1] * __builtin_amdgcn_exp2f(x[k][0] - ref) : 0.0f;
    top = to;
  }
};
__device__ __forceinline__ float join(const WeightsParams& p, long long r, int parts) {
  const f32x2_t* from = p.stats + r * p.parts;
  float top = -INFINITY, sum = 0.0f;
  for (int k = 0; k < parts; k += 8) {
    Parts x;
    x.load(from + k, parts - k);
    x.add(parts - k, top, sum);
  }
  return top + __builtin_amdgcn_logf(sum);
}

// ---- tiles of 64 in LDS, for requests of many rows (bf16) -------------------------
// Both launches keep one operand in registers and pass the other by it in tiles of 64
// rows, which the four waves share: two buffers in LDS, filled by direct loads.  Rows
// lie in 16-byte pieces whose place is exchanged so that the reads of a fragment meet
// distinct banks: piece c of row r at c ^ swz(r).
constexpr int TILE = 64;
template <int DH>
__device__ __forceinline__ int swz(int r) { return DH == 128 ? r & 15 : (r >> 1) & 7; }

template <int DH>
struct Stream {
  static constexpr int ROW = DH * 2, RPL = 1024 / ROW, LPR = ROW / 16, LOADS = 16 / RPL;
  // 16 rows from `base` on, the lane's row of load q at off(RPL * q + lane / LPR) bytes
  template <typename Off>
  __device__ __forceinline__ static void load(const void* base, uint8_t* to, int lane, Off off) {
    const __amdgpu_buffer_rsrc_t r = __builtin_amdgcn_make_buffer_rsrc(const_cast<void*>(base), 0, -1, 0x00020000);
#pragma unroll
    for (int q = 0; q < LOADS; ++q) {
      const int row = RPL * q + lane / LPR;
      __builtin_amdgcn_raw_ptr_buffer_load_lds(r, (lds_void_t*)(to + RPL * q * ROW), 16,
                                               off(row) + ((uint32_t)((lane % LPR) ^ swz<DH>(row)) << 4), 0, 0, 0);
    }
  }
  // products of 32 rows in registers with those of a tile
  __device__ __forceinline__ static void mul_by(f32x16_t& a, const uint8_t* tile, const bf16x8_t (&st)[DH / 16], int lane) {
    const int fr = lane & 31;
    bf16x8_t f[DH / 16];
#pragma unroll
    for (int ks = 0; ks < DH / 16; ++ks)
      f[ks] = __builtin_bit_cast(bf16x8_t, *reinterpret_cast<const u32x4_t*>(
                                               tile + fr * ROW + (((2 * ks + (lane >> 5)) ^ swz<DH>(fr & 15)) << 4)));
#pragma unroll
    for (int r = 0; r < 16; ++r) a[r] = 0.0f;
#pragma unroll
    for (int ks = 0; ks < DH / 16; ++ks) a = __builtin_amdgcn_mfma_f32_32x32x16_bf16(st[ks], f[ks], a, 0, 0, 0);
  }
  // products of the tile's rows 32 i .. 32 i + 31 with 32 rows in registers; the fragments
  // are read AHEAD products before they are used
  __device__ __forceinline__ static void mul(f32x16_t& a, const uint8_t* tile, int i, const bf16x8_t (&st)[DH / 16], int lane) {
    constexpr int KS = DH / 16, AHEAD = 3;
    const int fr = lane & 31;
    const uint8_t* row = tile + (32 * i + fr) * ROW;
    auto read = [&](int ks) {
      const int c = (2 * ks + (lane >> 5)) ^ swz<DH>(fr);
      return __builtin_bit_cast(bf16x8_t, *reinterpret_cast<const u32x4_t*>(row + c * 16));
    };
    bf16x8_t f[AHEAD + 1];
    __builtin_amdgcn_sched_barrier(0);
#pragma unroll
    for (int ks = 0; ks < AHEAD; ++ks) f[ks] = read(ks);
#pragma unroll
    for (int r = 0; r < 16; ++r) a[r] = 0.0f;
    __builtin_amdgcn_sched_barrier(0);
#pragma unroll
    for (int ks = 0; ks < KS; ++ks) {
      if (ks + AHEAD < KS) f[(ks + AHEAD) % (AHEAD + 1)] = read(ks + AHEAD);
      a = __builtin_amdgcn_mfma_f32_32x32x16_bf16(f[ks % (AHEAD + 1)], st[ks], a, 0, 0, 0);
      if (ks + AHEAD < KS) __builtin_amdgcn_sched_group_barrier(0x100, 1, 0);
      __builtin_amdgcn_sched_group_barrier(0x008, 1, 0);
    }
    __builtin_amdgcn_sched_barrier(0);
  }
};

template <int DH>
__device__ __forceinline__ void load_row(bf16x8_t (&f)[DH / 16], const uint16_t* at, int lane) {
#pragma unroll
  for (int ks = 0; ks < DH / 16; ++ks)
    f[ks] = __builtin_bit_cast(bf16x8_t, *reinterpret_cast<const u32x4_t*>(at + 16 * ks + 8 * (lane >> 5)));
}

}  // namespace

// Maximum and sum of 128 rows over a part of the keys, which pass by: a lane owns
// a row, half of each tile's keys, and needs no other lane before the end.  The
// reference of a row's exponentials is the maximum of the first tile in which it sees a
// key and moves only where a later tile adds up to 2^40 of it: any reference gives the
// same sum, and the common tile takes no maximum.  Four workgroups a CU (120 registers) hide
// each other's barriers: of 16 x 256 rows over 1024 keys of 32 heads, 34 GFLOP, one a CU takes
// 80 us, two 55, four 46 (750 TFLOP/s); without the exponentials it would be 41, with half the
// products 40.  Where requests fill their last 128 rows badly (1.34 times the products for the
// windows above), that is what is lost.
template <int DH>
__global__ __launch_bounds__(NT, 4) void weights_stats_tile_kernel(WeightsParams p) {
  extern __shared__ int lds[];
  __shared__ __attribute__((aligned(1024))) uint8_t tile0[TILE * DH * 2];
  __shared__ __attribute__((aligned(1024))) uint8_t tile1[TILE * DH * 2];
  constexpr int RT = 128;
  const Share share(p.n_kv);
  auto units = [&](const Seq& s, int) { return s.nk > 0 ? (s.rows + RT - 1) / RT * share.heads * p.parts : 0; };
  const Line line = line_of<false>(p, lds, units);
  const int lane = threadIdx.x & (kWave - 1), wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
  const float c = scale_of(p);
  const uint16_t* q = static_cast<const uint16_t*>(p.q);
  const uint8_t* pool = static_cast<const uint8_t*>(p.pool);
  for (int u = share.first; u < line.all; u += share.step) {
    int at;
    const int b = __builtin_amdgcn_readfirstlane(request_of(line, p.B, u, at));
    at = __builtin_amdgcn_readfirstlane(at);
    const Seq s = line.seq(p, b);
    const int tiles = (s.rows + RT - 1) / RT;
    const int t = at % tiles, part = at / tiles % p.parts, hk = share.head0 + at / tiles / p.parts;
    const int row0 = t * RT + 32 * wave;
    bf16x8_t st[DH / 16];
    float m = -INFINITY, l = 0.0f;
    const int row = row0 + (lane & 31), src = row < s.rows ? row : s.rows - 1;
    const int tok = token_of(p, src), head = hk * p.group + src - tok * p.group;
    load_row<DH>(st, q + (long long)(s.row0 + tok) * p.q_stride + (long long)head * DH, lane);
    const int index = s.index0 + tok;            // of the lane's row among the request's rows of the call
    const int keys = part_keys(p, s.nk);
    const long long begin = (long long)part * keys, end = begin + keys;
    const int lo = begin < s.nk ? (int)begin : s.nk;
    int hi = end < s.nk ? (int)end : s.nk;
    // where the tile's rows see no more, and where the first one begins to be blind
    const int last = token_of(p, t * RT + RT < s.rows ? t * RT + RT - 1 : s.rows - 1);
    if (p.mask == kMaskCausal) {
      const int stop = s.past + s.index0 + last + 1;
      hi = stop < hi ? (stop > lo ? stop : lo) : hi;
    }
    const int first = s.past + s.index0 + token_of(p, row0 < s.rows ? row0 : s.rows - 1) + 1;
    const int open = p.mask == kMaskCausal ? first : (p.mask == kMaskTree ? s.past : hi);
    const int* table = p.table + (size_t)b * p.width;
    const int n = (hi - lo + TILE - 1) / TILE;
    int id[4];
    auto pages = [&](int k0) {
#pragma unroll
      for (int i = 0; i < 4; ++i) {
        const int key = k0 + 16 * i;
        id[i] = scalar_load(table, (key < hi ? key : hi - 1) >> p.shift);
      }
    };
    auto held = [&](int i) { return i >= 0 && i < p.n_pages; };
    auto lost_of = [&]() {
      unsigned long long x = 0;
#pragma unroll
      for (int i = 0; i < 4; ++i)
        if (!held(id[i])) x |= 0xffffull << (16 * i);
      return x;
    };
    auto load = [&](int k0, uint8_t* to) {
      int key = k0 + 16 * wave;                  // a group past the end is the last one again, as are keys past it
      key = key < hi ? key : (hi - 1) & ~15;
      const int mine = wave == 0 ? id[0] : (wave == 1 ? id[1] : (wave == 2 ? id[2] : id[3]));
      const int most = hi - 1 - key < 15 ? hi - 1 - key : 15;
      const long long row = ((held(mine) ? (long long)mine : 0) * 2 * p.n_kv << p.shift) + ((long long)hk << p.shift) +
                            (key & ((1 << p.shift) - 1));
      Stream<DH>::load(pool + row * (DH * 2), to + 16 * wave * DH * 2, lane,
                       [&](int r) { return (uint32_t)((r < most ? r : most) * DH * 2); });
    };
    unsigned long long lost = 0, lost_next = 0;
    if (n > 0) {
      pages(lo);
      load(lo, tile0);
      lost = lost_of();
      if (n > 1) pages(lo + TILE);
    }
    __builtin_amdgcn_s_waitcnt(0x0f70);          // vmcnt(0)
    __syncthreads();
    auto step = [&](int kt, auto buf) {
      constexpr int B = decltype(buf)::value;
      const int k0 = lo + TILE * kt;
      if (kt + 1 < n) {
        load(k0 + TILE, B ? tile0 : tile1);
        lost_next = lost_of();
        if (kt + 2 < n) pages(k0 + 2 * TILE);
      }
      if (row0 < s.rows) {
        const bool masked = k0 + TILE > open || k0 + TILE > hi || lost != 0;
        float x[2][16];
#pragma unroll
        for (int i = 0; i < 2; ++i) {
          f32x16_t a;
          Stream<DH>::mul(a, B ? tile1 : tile0, i, st, lane);
#pragma unroll
          for (int r = 0; r < 16; ++r) x[i][r] = a[r];
        }
        if (masked) {
          int lim = hi;
          if (p.mask == kMaskCausal && s.past + index + 1 < lim) lim = s.past + index + 1;
          const GqaSight<true> sight(lim, s.past, p.mask == kMaskTree ? p.bits + (size_t)(s.row0 - s.index0 + index) * p.words
                                                                     : nullptr, p.words);
          const unsigned long long seen = (sight.seen(k0) & ~lost) >> (4 * (lane >> 5));
#pragma unroll
          for (int i = 0; i < 2; ++i) {
            const uint32_t half = (uint32_t)(seen >> (32 * i));
#pragma unroll
            for (int r = 0; r < 16; ++r)
              if (!(half >> (8 * (r >> 2) + (r & 3)) & 1)) x[i][r] = -INFINITY;
          }
        }
        float sum;
        auto add = [&](float ref) {
          float s0 = 0.0f, s1 = 0.0f;
          const float mc = ref * c;
#pragma unroll
          for (int r = 0; r < 16; ++r) {
            s0 += __builtin_amdgcn_exp2f(__builtin_fmaf(x[0][r], c, -mc));
            s1 += __builtin_amdgcn_exp2f(__builtin_fmaf(x[1][r], c, -mc));
          }
          sum = s0 + s1;
        };
        add(m);
        // (no key seen yet: the reference is -inf, and -inf + inf or x + inf ask for a maximum too)
        if (__any(!(sum < 0x1p40f))) {
          float top = m;
#pragma unroll
          for (int r = 0; r < 16; ++r) top = fmaxf(top, fmaxf(x[0][r], x[1][r]));
          l *= m == -INFINITY ? 1.0f : __builtin_amdgcn_exp2f((m - top) * c);
          m = top;
          add(top == -INFINITY ? 0.0f : top);
        }
        l += sum;
      }
      lost = lost_next;
      __builtin_amdgcn_s_waitcnt(0x0f70);
      __syncthreads();
    };
    for (int kt = 0; kt < n; kt += 2) {
      step(kt, std::integral_constant<int, 0>{});
      if (kt + 1 < n) step(kt + 1, std::integral_constant<int, 1>{});
    }
    const float top = fmaxf(m, __shfl_xor(m, 32, kWave)), ref = top == -INFINITY ? 0.0f : top;
    const float part_l = l * __builtin_amdgcn_exp2f((m - ref) * c);
    const float all = part_l + __shfl_xor(part_l, 32, kWave);
    if (row < s.rows && lane < 32) {
      const long long r = stat_row(p, line, s, b, hk) + row;
      if (p.parts == 1) p.lse[r] = top * c + __builtin_amdgcn_logf(all);
      else p.stats[r * p.parts + part] = f32x2_t{top * c, all};
    }
  }
}

// The weights of 128 keys, which stay, from all rows, which pass by.  A row that is blind to
// a lane's key stands before the lane's first row that sees it (causal), so one number of a
// key masks a tile; the tiles without a mask have a copy of the code of their own.
// The parts of the rows' sums are joined here, 1024 rows at a time, by all threads (in a launch
// of its own it took 5 us).
template <int DH>
__global__ __launch_bounds__(NT, 4) void weights_sum_tile_kernel(WeightsParams p) {
  extern __shared__ int lds[];
  __shared__ __attribute__((aligned(1024))) uint8_t tile0[TILE * DH * 2];
  __shared__ __attribute__((aligned(1024))) uint8_t tile1[TILE * DH * 2];
  constexpr int ROWS = 1024;                     // whose logarithms are held at a time
  __shared__ __attribute__((aligned(16))) float lse_lds[ROWS];
  constexpr int KT = 128;
  const Share share(p.n_kv);
  auto units = [&](const Seq& s, int) { return s.used > 0 ? (s.nk + KT - 1) / KT * share.heads * p.sums : 0; };
  const Line line = line_of<false>(p, lds, units);
  const int tid = threadIdx.x, lane = tid & (kWave - 1), wave = __builtin_amdgcn_readfirstlane(tid >> 6);
  const float c = scale_of(p);
  const uint8_t* q = static_cast<const uint8_t*>(p.q);
  const uint16_t* pool = static_cast<const uint16_t*>(p.pool);
  for (int u = share.first; u < line.all; u += share.step) {
    int at;
    const int b = __builtin_amdgcn_readfirstlane(request_of(line, p.B, u, at));
    at = __builtin_amdgcn_readfirstlane(at);
    const Seq s = line.seq(p, b);
    const int tiles = (s.nk + KT - 1) / KT;
    const int quot = at / tiles, key0 = (at - quot * tiles) * KT, k0 = key0 + 32 * wave;
    const int hk = share.head0 + quot / p.sums, part = quot % p.sums;
    const int* table = p.table + (size_t)b * p.width;
    bf16x8_t st[DH / 16];
    float sum = 0.0f;
    const int key = k0 + (lane & 31), src = key < s.nk ? key : s.nk - 1;
    bool held;
    load_row<DH>(st, pool + key_row(p, table, hk, src, held), lane);
    // rows that do not see the lane's key (causal): those before the first that does
    const int behind = key - s.past - s.index0;
    const int blind = behind > 0 ? (behind < s.used ? behind * p.group : s.rows) : 0;
    // the first row that sees a key of the workgroup's, in whole tiles
    int from = 0;
    if (p.mask == kMaskCausal) {
      const int token = key0 - s.past - s.index0;
      if (token > 0) from = token < s.used ? token * p.group / TILE * TILE : s.rows;
    }
    const long long stat = stat_row(p, line, s, b, hk);
    int n = (s.rows - from + TILE - 1) / TILE;
    if (p.sums > 1) {                            // an equal share of them
      const int per = (n + p.sums - 1) / p.sums, skip = part * per < n ? part * per : n;
      from += skip * TILE;
      n = n - skip < per ? n - skip : per;
    }
    // the logarithms of the sums of the rows of tile rt and those behind it
    auto hold = [&](int rt) {
      const int r0 = from + TILE * rt;
      for (int t = tid; t < ROWS && r0 + (t & ~63) < s.rows; t += NT) {
        float x = INFINITY;
        if (r0 + t < s.rows) x = p.parts > 1 ? join(p, stat + r0 + t, p.parts) : p.lse[stat + r0 + t];
        lse_lds[t] = x == -INFINITY ? INFINITY : x;          // a row that sees no key
      }
    };
    auto load = [&](int r0, uint8_t* to) {
      int row = r0 + 16 * wave;
      row = row < s.rows ? row : s.rows - 1;     // rows past the end are the last one again
      const int base = token_of(p, row);
      const uint8_t* at = q + ((long long)(s.row0 + base) * p.q_stride + (long long)hk * p.group * DH) * 2;
      const int most = s.rows - 1 - row < 15 ? s.rows - 1 - row : 15;
      Stream<DH>::load(at, to + 16 * wave * DH * 2, lane, [&](int r) {
        const int i = row + (r < most ? r : most), tok = token_of(p, i);
        return (uint32_t)(tok - base) * (uint32_t)(p.q_stride * 2) + (uint32_t)(i - tok * p.group) * (DH * 2);
      });
    };
    if (n > 0) {
      load(from, tile0);
      hold(0);
    }
    __builtin_amdgcn_s_waitcnt(0x0f70);
    __syncthreads();
    auto step = [&](int rt, auto buf) {
      constexpr int B = decltype(buf)::value;
      const int r0 = from + TILE * rt;
      if (rt + 1 < n) load(r0 + TILE, B ? tile0 : tile1);
      if (k0 < s.nk) {
        const int sure = p.mask == kMaskCausal ? s.past + s.index0 + token_of(p, r0) + 1
                                               : (p.mask == kMaskTree ? s.past : s.nk);
        const bool masked = p.mask != kMaskNone && k0 + 32 > sure;
        unsigned long long seen = 0;             // which rows see the lane's key, in the order of its elements
        if (masked && p.mask == kMaskCausal) {
          const int hidden = blind - r0;
          seen = hidden <= 0 ? ~0ull : (hidden >= TILE ? 0ull : ~0ull << hidden);
        } else if (masked) {
          const uint32_t keys = window(p, s, r0 + lane, k0);
#pragma unroll
          for (int r = 0; r < 32; ++r) {
            const uint32_t low = __builtin_amdgcn_readlane(keys, r) >> (lane & 31) & 1;
            const uint32_t high = __builtin_amdgcn_readlane(keys, r + 32) >> (lane & 31) & 1;
            seen |= low << r | (unsigned long long)(high << r) << 32;
          }
        }
        seen >>= 4 * (lane >> 5);
        const float* lse = &lse_lds[rt % (ROWS / TILE) * TILE + 4 * (lane >> 5)];
        // (two copies, so that a half's sums do not wait for the branch)
        float own = 0.0f;                        // of this tile's rows
        auto add = [&](auto blinded) {
#pragma unroll
          for (int i = 0; i < 2; ++i) {
            f32x16_t a;
            Stream<DH>::mul(a, B ? tile1 : tile0, i, st, lane);
            const uint32_t half = (uint32_t)(seen >> (32 * i));
#pragma unroll
            for (int g = 0; g < 4; ++g) {
              const f32x4_t x = *reinterpret_cast<const f32x4_t*>(lse + 32 * i + 8 * g);
#pragma unroll
              for (int r = 0; r < 4; ++r) {
                const float w = __builtin_amdgcn_exp2f(__builtin_fmaf(a[4 * g + r], c, -x[r]));
                own += !decltype(blinded)::value || (half >> (8 * g + r) & 1) ? w : 0.0f;
              }
            }
          }
        };
        if (masked) add(std::true_type{});
        else add(std::false_type{});
        sum += own;
      }
      __builtin_amdgcn_s_waitcnt(0x0f70);
      __syncthreads();
      if ((rt + 1) % (ROWS / TILE) == 0 && rt + 1 < n) {
        hold(rt + 1);
        __syncthreads();
      }
    };
    for (int rt = 0; rt < n; rt += 2) {
      step(rt, std::integral_constant<int, 0>{});
      if (rt + 1 < n) step(rt + 1, std::integral_constant<int, 1>{});
    }
    const float all = sum + __shfl_xor(sum, 32, kWave);
    if (p.sums > 1) {
      if (lane < 32 && key < s.nk) p.partial[(((long long)b * p.n_kv + hk) * p.places + key) * p.sums + part] = all;
      continue;
    }
    const long long id = key < s.nk ? table[key >> p.shift] : -1;
    if (lane < 32 && id >= 0 && id < p.n_pages) {
      const long long mark = ((id * p.n_kv + hk) << p.shift) + (key & ((1 << p.shift) - 1));
      p.weight[mark] = p.prev ? __builtin_fmaf(p.decay, p.prev[mark], all) : all;
    }
  }
}

// The weights from the sums of parts of the rows, in their order.
__global__ __launch_bounds__(NT) void weights_join_kernel(WeightsParams p) {
  extern __shared__ int lds[];
  const Line line = line_of<false>(p, lds, [&](const Seq& s, int) { return s.used > 0 ? (s.nk + NT - 1) / NT * p.n_kv : 0; });
  for (int u = blockIdx.x; u < line.all; u += gridDim.x) {
    int at;
    const int b = request_of(line, p.B, u, at);
    const Seq s = line.seq(p, b);
    const int tiles = (s.nk + NT - 1) / NT, hk = at / tiles, key = (at - hk * tiles) * NT + threadIdx.x;
    if (key >= s.nk) continue;
    const long long id = p.table[(size_t)b * p.width + (key >> p.shift)];
    if (id < 0 || id >= p.n_pages) continue;
    const float* from = p.partial + (((long long)b * p.n_kv + hk) * p.places + key) * p.sums;
    float sum = 0.0f;
    for (int i = 0; i < p.sums; ++i) sum += from[i];
    const long long mark = ((id * p.n_kv + hk) << p.shift) + (key & ((1 << p.shift) - 1));
    p.weight[mark] = p.prev ? __builtin_fmaf(p.decay, p.prev[mark], sum) : sum;
  }
}

// Requests of few rows (bf16): 32 of them against a part of the keys, whose scores are
// kept.  Each wave walks every fourth 32 keys by itself, its tiles of its own in LDS, two
// of them on their way, without a barrier before the end.  S = Q K^T: a lane owns a key,
// its registers are rows, 8 for each group of four, so that only the groups with rows are
// looked at and a row's scores go to memory 128 bytes at a time.  Bound by the read of the
// keys: 302 MB in 68 us for the 64 tokens above (4.4 TB/s; a copy's read reaches 5.9).
template <int DH>
__global__ __launch_bounds__(NT) void weights_scores_kernel(WeightsParams p) {
  extern __shared__ int lds[];
  constexpr int FT = 32 * DH * 2, LOADS = 2 * Stream<DH>::LOADS;
  __shared__ __attribute__((aligned(1024))) uint8_t tile0[WAVES * FT];
  __shared__ __attribute__((aligned(1024))) uint8_t tile1[WAVES * FT];
  __shared__ f32x2_t found[WAVES][32];
  const Line line = line_of<true>(p, lds, [&](const Seq& s, int chunk) {
    const int keys = part_keys(p, s.nk, chunk);
    return s.nk > 0 ? (s.rows + 31) / 32 * p.n_kv * ((s.nk + keys - 1) / keys) : 0;
  });
  const int lane = threadIdx.x & (kWave - 1), wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6), half = lane >> 5;
  const float c = scale_of(p);
  const uint8_t* pool = static_cast<const uint8_t*>(p.pool);
  for (int u = blockIdx.x; u < line.all; u += gridDim.x) {
    int at;
    const int b = __builtin_amdgcn_readfirstlane(request_of(line, p.B, u, at));
    at = __builtin_amdgcn_readfirstlane(at);
    const Seq s = line.seq(p, b);
    const int keys = part_keys(p, s.nk, line.chunk), tiles = (s.rows + 31) / 32, parts = (s.nk + keys - 1) / keys;
    const int quot = at / tiles, r0 = (at - quot * tiles) * 32, hk = quot / parts, part = quot - hk * parts;
    const int lo = part * keys, hi = s.nk - lo < keys ? s.nk : lo + keys;
    const int n = hi - lo > 32 * wave ? (hi - lo - 32 * wave + 127) / 128 : 0;       // the wave's tiles
    const int* table = p.table + (size_t)b * p.width;
    const long long stat = stat_row(p, line, s, b, hk) + r0;
    const int left = s.rows - r0 < 32 ? s.rows - r0 : 32;
    // the first key to which some row may be blind
    int open = hi;
    if (p.mask == kMaskCausal) open = s.past + s.index0 + token_of(p, r0) + 1;
    if (p.mask == kMaskTree) open = s.past;
    open = open < hi ? open : hi;

    // pages of the groups of 16 keys of 32 tiles, one a lane
    auto page = [&](int k) {
      const long long key = lo + (long long)(k + (lane >> 1)) * 128 + 32 * wave + 16 * (lane & 1);
      return table[(int)(key < hi ? key : hi - 1) >> p.shift];
    };
    int id = page(0);
    bf16x8_t st[DH / 16];
    {
      const int row = r0 + ((lane & 31) < left ? (lane & 31) : left - 1), tok = token_of(p, row);
      load_row<DH>(st, static_cast<const uint16_t*>(p.q) + (long long)(s.row0 + tok) * p.q_stride +
                           (long long)(hk * p.group + row - tok * p.group) * DH, lane);
    }
    bool lost[2] = {false, false};               // whether the lane's key of each buffer is on no page
    auto load = [&](int k, auto buf) {
      constexpr int B = decltype(buf)::value;
      if ((k & 31) == 0 && k > 0) {
        id = page(k);
        __builtin_amdgcn_s_waitcnt(0x0f70);      // here, and not before each step's use of it
      }
      const int key = lo + k * 128 + 32 * wave;
#pragma unroll
      for (int g = 0; g < 2; ++g) {
        const int mine = __builtin_amdgcn_readlane(id, 2 * (k & 31) + g);
        const bool held = mine >= 0 && mine < p.n_pages;
        int first = key + 16 * g;                // a group past the end is the last one again, as are keys past it
        first = first < hi ? first : (hi - 1) & ~15;
        const int most = hi - 1 - first;
        const long long row = (((held ? (long long)mine : 0) * 2 * p.n_kv + hk) << p.shift) + (first & ((1 << p.shift) - 1));
        Stream<DH>::load(pool + row * (DH * 2), (B ? tile1 : tile0) + wave * FT + 16 * g * DH * 2, lane,
                         [&](int r) { return (uint32_t)((r < most ? r : most) * DH * 2); });
        if ((lane >> 4 & 1) == g) lost[B] = !held;
      }
    };
    // NG groups of 8 rows
    auto walk = [&](auto groups) {
      constexpr int NG = decltype(groups)::value, NR = 4 * NG;
      float m[NR], l[NR];
#pragma unroll
      for (int r = 0; r < NR; ++r) {
        m[r] = -INFINITY;
        l[r] = 0.0f;
      }
      if (n > 0) load(0, std::integral_constant<int, 0>{});
      if (n > 1) load(1, std::integral_constant<int, 1>{});
      __builtin_amdgcn_s_waitcnt(0x0f70);        // vmcnt(0): the rows too
      auto step = [&](int k, auto buf) {
        constexpr int B = decltype(buf)::value;
        // newer than this tile's loads: the other buffer's, and what the tile before has stored
        // (rows past the last are the last again, so that the number of stores is known)
        constexpr int NEWER = LOADS + NR;
        __builtin_amdgcn_sched_barrier(0);
        if (k > 0 && k + 1 < n) __builtin_amdgcn_s_waitcnt(0x0f70 | (NEWER & 15) | (NEWER >> 4) << 14);
        else if (k + 1 < n) __builtin_amdgcn_s_waitcnt(0x0f70 | (LOADS & 15) | (LOADS >> 4) << 14);
        else __builtin_amdgcn_s_waitcnt(0x0f70);
        __builtin_amdgcn_wave_barrier();
        __builtin_amdgcn_sched_barrier(0);
        const int k0 = lo + k * 128 + 32 * wave, key = k0 + (lane & 31);
        f32x16_t a;
        Stream<DH>::mul_by(a, (B ? tile1 : tile0) + wave * FT, st, lane);
        uint32_t score[NR];
#pragma unroll
        for (int r = 0; r < NR; ++r) score[r] = __float_as_uint(a[r]);
        if (k0 + 32 > open || __any(lost[B])) {
          const uint32_t keys = window(p, s, r0 + (lane & 31), k0);
#pragma unroll
          for (int r = 0; r < NR; ++r) {
            const int row = 8 * (r >> 2) + (r & 3);
            const uint32_t low = __builtin_amdgcn_readlane(keys, row), high = __builtin_amdgcn_readlane(keys, row + 4);
            const bool see = ((half ? high : low) >> (lane & 31) & 1) && !lost[B];
            score[r] = see ? score[r] : kUnseen;
            a[r] = see ? a[r] : -INFINITY;
          }
        }
#pragma unroll
        for (int r = 0; r < NR; ++r) {
          const int row = 8 * (r >> 2) + 4 * half + (r & 3);
          // past the caches: 2 to 3% of a large launch
          __builtin_nontemporal_store(score[r], reinterpret_cast<uint32_t*>(p.scores) +
                                                    (stat + (row < left ? row : left - 1)) * p.places + key);
        }
        if (k + 2 < n) {
          // this tile's fragments have been read
          __builtin_amdgcn_sched_barrier(0);
          __builtin_amdgcn_s_waitcnt(0xc07f);    // lgkmcnt(0)
          __builtin_amdgcn_wave_barrier();
          __builtin_amdgcn_sched_barrier(0);
          load(k + 2, buf);
        }
#pragma unroll
        for (int r = 0; r < NR; ++r) {
          const float x = a[r] * c, to = fmaxf(m[r], x), ref = to == -INFINITY ? 0.0f : to;
          l[r] = l[r] * __builtin_amdgcn_exp2f(m[r] - ref) + __builtin_amdgcn_exp2f(x - ref);
          m[r] = to;
        }
      };
      for (int k = 0; k < n; k += 2) {
        step(k, std::integral_constant<int, 0>{});
        if (k + 1 < n) step(k + 1, std::integral_constant<int, 1>{});
      }
      // over the 32 keys of a half of the wave
#pragma unroll
      for (int r = 0; r < NR; ++r) {
        const float top = half_reduce(m[r], [](float a, float b) { return fmaxf(a, b); }), ref = top == -INFINITY ? 0.0f : top;
        const float sum = half_reduce(l[r] * __builtin_amdgcn_exp2f(m[r] - ref), [](float a, float b) { return a + b; });
        if ((lane & 31) == 0) found[wave][8 * (r >> 2) + 4 * half + (r & 3)] = f32x2_t{top, sum};
      }
    };
    if (left <= 8) walk(std::integral_constant<int, 1>{});
    else walk(std::integral_constant<int, 4>{});
    __syncthreads();
    if (threadIdx.x < (unsigned)left) {
      float top = -INFINITY, sum = 0.0f;
#pragma unroll
      for (int w = 0; w < WAVES; ++w) top = fmaxf(top, found[w][threadIdx.x][0]);
      const float ref = top == -INFINITY ? 0.0f : top;
#pragma unroll
      for (int w = 0; w < WAVES; ++w) sum += found[w][threadIdx.x][1] * __builtin_amdgcn_exp2f(found[w][threadIdx.x][0] - ref);
      p.stats[(stat + threadIdx.x) * p.parts + part] = f32x2_t{top, sum};
    }
    __syncthreads();
  }
}

// fp32.  Maximum and sum of the rows of a tile over a part of the keys, every fourth tile of
// keys a wave, the next one on its way.  Bound by latency: trees of 54 rows over 1198 keys.
template <typename Tile>
__global__ __launch_bounds__(NT) void weights_stats_kernel(WeightsParams p) {
  extern __shared__ int lds[];
  constexpr int T = Tile::T, STEP = WAVES * T;
  __shared__ f32x2_t found[WAVES][T];
  const Line line = line_of<false>(
      p, lds, [&](const Seq& s, int) { return s.nk > 0 ? (s.rows + T - 1) / T * p.n_kv * p.parts : 0; });
  const int lane = threadIdx.x & (kWave - 1), wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
  const float c = scale_of(p);
  for (int u = blockIdx.x; u < line.all; u += gridDim.x) {
    int at;
    const int b = __builtin_amdgcn_readfirstlane(request_of(line, p.B, u, at));
    at = __builtin_amdgcn_readfirstlane(at);
    const Seq s = line.seq(p, b);
    const int tiles = (s.rows + T - 1) / T;
    const int t = at % tiles, part = at / tiles % p.parts, hk = at / tiles / p.parts;
    const int row = t * T + Tile::row(lane), src = row < s.rows ? row : s.rows - 1;
    const int tok = token_of(p, src), head = hk * p.group + src - tok * p.group;
    typename Tile::Frag q, k[2];
    Tile::load(q, p.q, (long long)(s.row0 + tok) * p.q_stride + (long long)head * p.head_dim, p.head_dim, lane);
    const int keys = part_keys(p, s.nk);
    const long long begin = (long long)part * keys, end = begin + keys;
    const int lo = begin < s.nk ? (int)begin : s.nk;
    int hi = end < s.nk ? (int)end : s.nk;
    if (p.mask == kMaskCausal) {                 // where the tile's rows see no more
      const int stop = s.past + s.index0 + token_of(p, t * T + T < s.rows ? t * T + T - 1 : s.rows - 1) + 1;
      hi = stop < hi ? (stop > lo ? stop : lo) : hi;
    }
    const int open = p.mask == kMaskCausal ? s.past + s.index0 + token_of(p, t * T) + 1 : (p.mask == kMaskTree ? s.past : s.nk);
    const int* table = p.table + (size_t)b * p.width;
    float m = -INFINITY, l = 0.0f;
    bool held[2] = {true, true};
    auto load = [&](int k0, int i) {
      const int key = k0 + Tile::row(lane) < s.nk ? k0 + Tile::row(lane) : s.nk - 1;
      Tile::load(k[i], p.pool, key_row(p, table, hk, key, held[i]), p.head_dim, lane);
    };
    auto step = [&](int k0, int i) {
      if (k0 + STEP < hi) load(k0 + STEP, i ^ 1);
      const unsigned long long lost = ~__ballot(held[i]);
      typename Tile::acc_t a;
      Tile::mul(a, k[i], q);
      float x[Tile::ACC], top = m;
#pragma unroll
      for (int r = 0; r < Tile::ACC; ++r) x[r] = a[r] * c;
      if (k0 + T > open || k0 + T > s.nk || lost) {
#pragma unroll
        for (int r = 0; r < Tile::ACC; ++r) {
          const int j = Tile::of(lane, r);
          // (a choice of two values: with a branch around the assignment masked scores counted here, for a
          // cause that was not found)
          const bool see = sees(p, s, s.row0 + tok, s.index0 + tok, k0 + j) && !(lost >> j & 1);
          x[r] = see ? x[r] : -INFINITY;
        }
      }
#pragma unroll
      for (int r = 0; r < Tile::ACC; ++r) top = fmaxf(top, x[r]);
      const float ref = top == -INFINITY ? 0.0f : top;
      float sum = 0.0f;
#pragma unroll
      for (int r = 0; r < Tile::ACC; ++r) sum += __builtin_amdgcn_exp2f(x[r] - ref);
      l = l * __builtin_amdgcn_exp2f(m - ref) + sum;
      m = top;
    };
    if (lo + wave * T < hi) load(lo + wave * T, 0);
    for (int k0 = lo + wave * T; k0 < hi; k0 += 2 * STEP) {
      step(k0, 0);
      if (k0 + STEP < hi) step(k0 + STEP, 1);
    }
    const float top = Tile::max(m), ref = top == -INFINITY ? 0.0f : top;
    l = Tile::sum(l * __builtin_amdgcn_exp2f(m - ref));
    if (lane < T) found[wave][lane] = f32x2_t{top, l};
    __syncthreads();
    if (wave == 0 && lane < T && row < s.rows) {
      float all = -INFINITY, sum = 0.0f;
#pragma unroll
      for (int w = 0; w < WAVES; ++w) all = fmaxf(all, found[w][lane][0]);
      const float to = all == -INFINITY ? 0.0f : all;
#pragma unroll
      for (int w = 0; w < WAVES; ++w) sum += found[w][lane][1] * __builtin_amdgcn_exp2f(found[w][lane][0] - to);
      p.stats[(stat_row(p, line, s, b, hk) + row) * p.parts + part] = f32x2_t{all, sum};
    }
    __syncthreads();
  }
}

// The weights from scores that the statistics' launch has left: where a request has few
// rows, those are fewer bytes than its keys.  A workgroup takes 1024 keys of a head and
// all rows, whose logarithms it makes for itself: 14 us for the 33 MB of the 64 tokens.
__global__ __launch_bounds__(NT) void weights_few_kernel(WeightsParams p) {
  extern __shared__ int lds[];
  __shared__ float lse[NT];
  constexpr int KT = 4 * NT;
  const Line line = line_of<true>(p, lds, [&](const Seq& s, int) { return s.used > 0 ? (s.nk + KT - 1) / KT * p.n_kv : 0; });
  const int tid = threadIdx.x;
  for (int u = blockIdx.x; u < line.all; u += gridDim.x) {
    int at;
    const int b = request_of(line, p.B, u, at);
    const Seq s = line.seq(p, b);
    const int tiles = (s.nk + KT - 1) / KT, hk = at / tiles, key = (at - hk * tiles) * KT + 4 * tid;
    const long long first = stat_row(p, line, s, b, hk);
    const int keys = part_keys(p, s.nk, line.chunk), parts = (s.nk + keys - 1) / keys;
    f32x4_t sum = {0.0f, 0.0f, 0.0f, 0.0f};
    for (int r0 = 0; r0 < s.rows; r0 += NT) {
      const int n = s.rows - r0 < NT ? s.rows - r0 : NT;
      if (tid < n) {
        const float x = join(p, first + r0 + tid, parts);
        lse[tid] = x == -INFINITY ? INFINITY : x;          // a row that sees no key
      }
      __syncthreads();
      if (key < s.nk) {
        const float* from = p.scores + (first + r0) * p.places + key;
        for (int r = 0; r < n; r += 8) {
          f32x4_t x[8];                          // on their way together; rows past the last are the last again
#pragma unroll
          for (int i = 0; i < 8; ++i) x[i] = *reinterpret_cast<const f32x4_t*>(from + (r + i < n ? r + i : n - 1) * p.places);
          f32x4_t own = {0.0f, 0.0f, 0.0f, 0.0f};
#pragma unroll
          for (int i = 0; i < 8; ++i) {
            const float l = r + i < n ? lse[r + i] : INFINITY;
#pragma unroll
            for (int e = 0; e < 4; ++e) {
              // (by its bits: of a row whose logarithm is NaN, -inf would give NaN to keys that it does not see)
              const float w = __builtin_amdgcn_exp2f(x[i][e] * scale_of(p) - l);
              own[e] += __float_as_uint(x[i][e]) == kUnseen ? 0.0f : w;
            }
          }
#pragma unroll
          for (int e = 0; e < 4; ++e) sum[e] += own[e];
        }
      }
      __syncthreads();
    }
    if (key < s.nk) {
      // a page holds all four
      const int id = p.table[(size_t)b * p.width + (key >> p.shift)];
      if (id >= 0 && id < p.n_pages) {
        const long long mark = (((long long)id * p.n_kv + hk) << p.shift) + (key & ((1 << p.shift) - 1));
#pragma unroll
        for (int e = 0; e < 4; ++e)
          if (key + e < s.nk) p.weight[mark + e] = p.prev ? __builtin_fmaf(p.decay, p.prev[mark + e], sum[e]) : sum[e];
      }
    }
  }
}

// fp32.  The weights of a tile of keys, from every fourth tile of rows a wave, whose
// logarithms it makes from the parts, the next tile's rows on their way.
template <typename Tile>
__global__ __launch_bounds__(NT) void weights_sum_kernel(WeightsParams p) {
  extern __shared__ int lds[];
  __shared__ float sums[WAVES][Tile::T];
  constexpr int T = Tile::T;
  const Line line = line_of<false>(p, lds, [&](const Seq& s, int) { return s.used > 0 ? (s.nk + T - 1) / T * p.n_kv : 0; });
  const int lane = threadIdx.x & (kWave - 1), wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
  const float c = scale_of(p);
  for (int u = blockIdx.x; u < line.all; u += gridDim.x) {
    int at;
    const int b = __builtin_amdgcn_readfirstlane(request_of(line, p.B, u, at));
    at = __builtin_amdgcn_readfirstlane(at);
    const Seq s = line.seq(p, b);
    const int tiles = (s.nk + T - 1) / T;
    const int hk = at / tiles, k0 = (at - hk * tiles) * T;
    const int* table = p.table + (size_t)b * p.width;
    const int key = k0 + Tile::row(lane), src = key < s.nk ? key : s.nk - 1;
    bool held;
    typename Tile::Frag k, q[2];
    Parts part[2];                               // of the lane's row's sum, at most 8
    const long long krow = key_row(p, table, hk, src, held);
    Tile::load(k, p.pool, krow, p.head_dim, lane);
    const long long stat = stat_row(p, line, s, b, hk);
    auto load = [&](int r0, int i) {
      const int row = r0 + Tile::row(lane) < s.rows ? r0 + Tile::row(lane) : s.rows - 1;
      const int tok = token_of(p, row), head = row - tok * p.group;
      Tile::load(q[i], p.q, (long long)(s.row0 + tok) * p.q_stride + (long long)(hk * p.group + head) * p.head_dim, p.head_dim,
                 lane);
      part[i].load(p.stats + (stat + row) * p.parts, p.parts);
    };
    float sum = 0.0f;
    auto step = [&](int r0, int i) {
      if (r0 + WAVES * T < s.rows) load(r0 + WAVES * T, i ^ 1);
      typename Tile::acc_t a;
      Tile::mul(a, q[i], k);
      float top = -INFINITY, all = 0.0f;
      part[i].add(p.parts, top, all);
      const float lse = top + __builtin_amdgcn_logf(all);
      const int sure = p.mask == kMaskCausal ? s.past + s.index0 + token_of(p, r0) + 1 : (p.mask == kMaskTree ? s.past : s.nk);
      const bool masked = k0 + T > sure || r0 + T > s.rows;
      float own = 0.0f;
#pragma unroll
      for (int r = 0; r < Tile::ACC; ++r) {
        float w = __builtin_amdgcn_exp2f(a[r] * c - __shfl(lse, Tile::of(lane, r), kWave));
        if (masked) {
          const int j = r0 + Tile::of(lane, r), it = token_of(p, j < s.rows ? j : s.rows - 1);
          const bool see = j < s.rows && sees(p, s, s.row0 + it, s.index0 + it, key);
          w = see ? w : 0.0f;
        }
        own += w;
      }
      sum += own;
    };
    // the first row that sees a key of the tile, in whole tiles
    int from = wave * T;
    if (p.mask == kMaskCausal) {
      const int behind = k0 - s.past - s.index0;
      if (behind > 0) from += behind < s.used ? behind * p.group / T * T : s.rows;
    }
    if (from < s.rows) load(from, 0);
    for (int r0 = from; r0 < s.rows; r0 += 2 * WAVES * T) {
      step(r0, 0);
      if (r0 + WAVES * T < s.rows) step(r0 + WAVES * T, 1);
    }
    sum = Tile::sum(sum);
    if (lane < T) sums[wave][lane] = sum;
    __syncthreads();
    if (wave == 0 && lane < T && key < s.nk && held) {
#pragma unroll
      for (int w = 1; w < WAVES; ++w) sum += sums[w][lane];
      const long long id = table[key >> p.shift];
      const long long mark = (((id * p.n_kv) + hk) << p.shift) + (key & ((1 << p.shift) - 1));
      p.weight[mark] = p.prev ? __builtin_fmaf(p.decay, p.prev[mark], sum) : sum;
    }
    __syncthreads();
  }
}

int launch_weights(const WeightsParams& p, hipStream_t s) {
  const size_t lds = 2 * (size_t)p.B * sizeof(int) + (p.B <= kKept ? p.B * sizeof(Seq) : 0);
  // no more workgroups than there can be units, where a call is small (one token: 16 -> 12 us); a multiple of 8
  auto grid = [](long long units, int most) { return dim3(units < most ? (units + 7) / 8 * 8 : most); };
  auto tiles_of = [&](int rows) { return (p.rows * p.group / rows + p.B) * p.n_kv * p.parts; };
  auto keys_of = [&](int keys) { return ((p.places + keys - 1) / keys) * p.B * p.n_kv; };
  auto go = [&](auto tile) {
    using Tile = decltype(tile);
    hipLaunchKernelGGL((weights_stats_kernel<Tile>), grid(tiles_of(Tile::T), 2048), dim3(NT), lds, s, p);
    hipLaunchKernelGGL((weights_sum_kernel<Tile>), grid(keys_of(Tile::T), 2048), dim3(NT), lds, s, p);
  };
  auto tiles = [&](auto dh) {
    constexpr int DH = decltype(dh)::value;
    if (p.scores) {
      hipLaunchKernelGGL((weights_scores_kernel<DH>), grid(tiles_of(32), 2048), dim3(NT), lds, s, p);
      hipLaunchKernelGGL(weights_few_kernel, grid(keys_of(4 * NT), 2048), dim3(NT), lds, s, p);
      return;
    }
    hipLaunchKernelGGL((weights_stats_tile_kernel<DH>), grid(tiles_of(128), 1024), dim3(NT), lds, s, p);
    hipLaunchKernelGGL((weights_sum_tile_kernel<DH>), grid(keys_of(128) * p.sums, 1024), dim3(NT), lds, s, p);
    if (p.sums > 1) hipLaunchKernelGGL(weights_join_kernel, grid(keys_of(NT), 1024), dim3(NT), lds, s, p);
  };
  if (p.bf16) {
    if (p.head_dim == 128) tiles(std::integral_constant<int, 128>{});
    else tiles(std::integral_constant<int, 64>{});
  } else {
    if (p.head_dim > 64) go(TileF32<2>{});
    else go(TileF32<1>{});
  }
  return hipGetLastError() == hipSuccess ? 0 : -1;
}

}  // namespace seer
