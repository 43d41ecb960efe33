// Forks of sequences on a paged cache: the child's row of the page table, and a copy of the parent's last page where it
// is not full, in every layer.  Pure data movement: 256-byte rows as 16-byte vectors, eight in flight per thread.
#include "cache_step.cuh"

namespace cc {

namespace {

// 64 children x 32 layers, half a page of 16 tokens x 8 heads each (132 MB of reads and writes), us: 256 threads and 85 registers 26.1,
// four vectors in flight at 48 registers 19.9, 128 threads and 80 registers 18.8.
constexpr int kThreads = 128;
constexpr int kUnroll = 8;

// grid: (parts of a page, layers, children)
__global__ void __launch_bounds__(kThreads, 6)
fork_kernel(const __grid_constant__ CacheSeqs cs, const CacheGeom g, const __grid_constant__ ForkArgs A,
            DeviceStatus* status) {
  pdl_launch_dependents();
  const int child = blockIdx.z, layer = blockIdx.y, s = A.parent[child];
  pdl_wait();
  const int n = cache_len(cs, g, s, status);
  const int full = n >> g.page_shift, rest = n & ((1 << g.page_shift) - 1);
  const int32_t* parent_row = g.table + (int64_t)s * g.table_stride;
  const int fresh = rest > 0 ? A.free_pages[child] : -1;
  const bool fresh_ok = fresh >= 0 && fresh < g.pool_pages;
  const int last = rest > 0 ? parent_row[full] : -1;
  const bool last_ok = last >= 0 && last < g.pool_pages;
  if (layer == 0 && A.write_table) {
    int32_t* row = A.child_table + (int64_t)child * A.child_stride;
    for (int i = blockIdx.x * kThreads + threadIdx.x; i < A.child_stride; i += gridDim.x * kThreads) {
      int page = -1;
      if (i < full) {
        page = parent_row[i];
        if (page < 0 || page >= g.pool_pages) {
          report_error(status, CC_ERR_DEVICE_FLAG, 611);
          page = -1;
        }
      } else if (i == full && rest > 0) {
        if (fresh_ok && last_ok) page = fresh;     // (a page that receives nothing holds what its last owner left)
        else if (!fresh_ok) report_error(status, CC_ERR_DEVICE_FLAG, 612);
      }
      row[i] = page;
    }
  }
  if (rest == 0) return;
  if (!last_ok) {
    if (threadIdx.x == 0) report_error(status, CC_ERR_DEVICE_FLAG, 613);
    return;
  }
  if (!fresh_ok) return;
  const int64_t from = ((int64_t)last << g.page_shift) * g.kv_tok, to = ((int64_t)fresh << g.page_shift) * g.kv_tok;
  const int chunks = rest * g.hkv * 32;          // 16-byte vectors of the rows, K and V by turns of a row
  uint16_t* const k = A.k[layer];
  uint16_t* const v = A.v[layer];
  for (int c0 = blockIdx.x * kThreads * kUnroll + threadIdx.x; c0 < chunks; c0 += gridDim.x * kThreads * kUnroll) {
    uint4 x[kUnroll];
    int64_t at[kUnroll];
#pragma unroll
    for (int i = 0; i < kUnroll; ++i) {
      const int c = c0 + i * kThreads;
      const int unit = c >> 5, t = unit / g.hkv, h = unit - t * g.hkv;
      at[i] = t * g.kv_tok + h * g.kv_head + (c & 15) * 8;
      if (c < chunks) x[i] = __ldcs(reinterpret_cast<const uint4*>((c & 16 ? v : k) + from + at[i]));
    }
#pragma unroll
    for (int i = 0; i < kUnroll; ++i) {
      const int c = c0 + i * kThreads;
      if (c < chunks) __stcs(reinterpret_cast<uint4*>((c & 16 ? v : k) + to + at[i]), x[i]);
    }
  }
}

}  // namespace

cudaError_t launch_fork(const Launch& L, const CacheSeqs& cs, const CacheGeom& g, const ForkArgs& a) {
  const int most = (32 * g.hkv) << g.page_shift;             // vectors of a whole page
  const int parts = (most + kThreads * kUnroll - 1) / (kThreads * kUnroll);
  const dim3 grid((unsigned)parts, (unsigned)a.n_layers, (unsigned)a.n_children);
  return launch_pdl(fork_kernel, grid, dim3(kThreads), 0, L.stream, 1, cs, g, a, L.status);
}

}  // namespace cc
