// Declarations shared by the kernels that work on a paged cache after the compression: rotation and append,
// attention of new tokens, forks.
#pragma once

#include "cc_internal.cuh"

namespace cc {

// The sequences of a call, by value in the kernels' parameters.
struct CacheSeqs {
  int num_seqs;
  int new_off[CC_MAX_SEQS + 1];   // first row of a sequence in [sum T_s] arrays
  int kv_len[CC_MAX_SEQS];        // n_s, or its upper bound with device lengths
};

struct CacheGeom {
  int hq, hkv, group;
  int page_shift;                 // page_size = 1 << page_shift
  int pool_pages, table_stride;
  const int32_t* table;
  const int32_t* dev_lens;        // or null
  int causal;
  float scale;
  int64_t qn_tok, qn_head, kvn_tok, kvn_head, q_tok, q_head, kv_tok, kv_head, out_tok, out_head;
};

// n_s as the call finds it.
__device__ __forceinline__ int cache_len(const CacheSeqs& cs, const CacheGeom& g, int s, DeviceStatus* st) {
  const int most = cs.kv_len[s];
  if (g.dev_lens == nullptr) return most;
  const int n = g.dev_lens[s];
  if (n >= 0 && n <= most) return n;
  report_error(st, CC_ERR_DEVICE_FLAG, 600);
  return n < 0 ? 0 : most;
}

// Sequence of row `tok` of a [sum T_s] array.
__device__ __forceinline__ int seq_of_new(const CacheSeqs& cs, int tok) {
  int lo = 0, hi = cs.num_seqs;                // new_off[lo] <= tok < new_off[hi]
  while (hi - lo > 1) {
    const int mid = (lo + hi) >> 1;
    if (cs.new_off[mid] <= tok) lo = mid;
    else hi = mid;
  }
  return lo;
}

struct RopeFreqs {
  int dims, interleaved;
  float scale;
  uint64_t turns[kHeadDim / 2];
};

cudaError_t launch_rope(const Launch& L, const CacheSeqs& cs, const CacheGeom& g, const RopeFreqs& f, const void* q_new,
                        const void* k_new, const void* v_new, const int32_t* positions, void* q, void* k, void* v);

constexpr int kForkLayers = 64;     // layers per launch
struct ForkArgs {
  int n_layers, n_children, child_stride;
  int write_table;
  const int32_t* free_pages;
  int32_t* child_table;
  uint8_t parent[CC_MAX_CHILDREN];
  uint16_t* k[kForkLayers];
  uint16_t* v[kForkLayers];
};
static_assert(CC_MAX_SEQS <= 256, "parents in a byte");
cudaError_t launch_fork(const Launch& L, const CacheSeqs& cs, const CacheGeom& g, const ForkArgs& a);

// Attention: bytes of workspace (0: more work than a call takes); launch (drv_err receives the code of a failed tensor map).
size_t attend_ws_bytes(const CacheSeqs& cs, const CacheGeom& g, int sm_count);
cudaError_t launch_attend(const Launch& L, const CacheSeqs& cs, const CacheGeom& g, const void* q, const void* k, const void* v,
                          void* out, float* lse, void* ws, void* encode_fn, int* drv_err);

}  // namespace cc
