// Pages of cached keys and values: which pages a step takes and gives back, the
// slot of each new row, and the copy of key and value rows into their slots.
#include "page_plan.h"

namespace seer {

int launch_page_plan(const PagePlanParams& p, hipStream_t s) { return launch_plan(p, s); }

// ---------------------------------------------------------------------------
// Rows into pages: a wave copies a row's K and V in 16-byte pieces, head after
// head; a head's piece of a row is contiguous in the page.  Bound by memory: 20,118
// rows of 32 heads by 128, 659 MB moved, 132 us, 5.0 TB/s, the rate of a large copy;
// 256 rows of 8 heads 3.5 us, the latency of a slot, a row and its store.
__global__ __launch_bounds__(256) void kv_store_kernel(KvStoreParams p) {
  const int lane = threadIdx.x & (kWave - 1);
  const size_t half = (size_t)p.n_kv << p.shift;           // head rows of K (or V) in a page
  const int n = p.n_kv * p.head_pieces;
  for (long long r = blockIdx.x * 4 + (threadIdx.x >> 6); r < p.rows_ub; r += 4ll * gridDim.x) {
    const int slot = p.slots[r];
    if (slot < 0 || (slot >> p.shift) >= p.n_pages) continue;
    const int off = slot & ((1 << p.shift) - 1);
    const size_t page = (size_t)(slot >> p.shift) * 2 * half;
    for (int c = lane; c < 2 * n; c += kWave) {
      const int v = c >= n, j = v ? c - n : c;
      const int h = j / p.head_pieces, piece = j - h * p.head_pieces;
      const uint8_t* src = v ? p.v + (size_t)r * p.v_stride : p.k + (size_t)r * p.k_stride;
      const size_t row = page + v * half + ((size_t)h << p.shift) + off;
      *reinterpret_cast<u32x4_t*>(p.pool + (row * p.head_pieces + piece) * 16) =
          *reinterpret_cast<const u32x4_t*>(src + (size_t)j * 16);
    }
  }
}

int launch_kv_store(const KvStoreParams& p, hipStream_t s) {
  // a row a wave, up to the threads that one launch may have
  const int blocks = p.rows_ub / 4 + (p.rows_ub % 4 != 0);
  hipLaunchKernelGGL(kv_store_kernel, dim3(blocks < 1 << 22 ? blocks : 1 << 22), dim3(256), 0, s, p);
  return hipGetLastError() == hipSuccess ? 0 : -1;
}

}  // namespace seer
