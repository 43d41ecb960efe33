// Attention over a paged cache: which kernel takes which sequences, the tensor maps, the join of cut problems.
#include <cuda_bf16.h>

#include <algorithm>

#include "attend_plan.cuh"
#include "exp2_poly.cuh"
#include "tc_ptx.cuh"

namespace cc {

namespace {

constexpr int kJoinWarps = 8;

// Joins the parts of the problems that are cut: a block per (boundary between two shares, eight rows), idle unless the
// boundary is the first inside its problem.  A warp takes a row; the parts follow each other in the order of the CTAs.
//   out = sum_k 2^(m_k - M) o_k / sum_k 2^(m_k - M) l_k
__global__ void __launch_bounds__(kJoinWarps * 32)
attend_join_kernel(const __grid_constant__ CacheSeqs cs, const CacheGeom g, const __grid_constant__ AttendSeqs as,
                   const AttendWs ws, int grid, const AttendOut o, DeviceStatus* status) {
  pdl_launch_dependents();
  pdl_wait();
  const int lane = threadIdx.x & 31, r = blockIdx.y * kJoinWarps + (threadIdx.x >> 5);
  const int b = blockIdx.x + 1;                    // the share that begins at the boundary
  const Place p = ws.place[b], before = ws.place[b - 1];
  auto inside = [&](const Place& x) { return x.tile > 0 && x.h == p.h && x.i == p.i && x.b == p.b; };
  if (p.tile <= 0 || inside(before)) return;
  const int s = as.src[p.i], T = cs.new_off[s + 1] - cs.new_off[s];
  const int in_tile = (r & 127) / g.group, t = p.b * as.block_tokens + (r >> 7) * as.tile_tokens + in_tile;
  if (in_tile >= as.tile_tokens || t >= T) return;
  int last = b;                                    // the last share with a part of the problem
  while (last + 1 < grid && inside(ws.place[last + 1])) ++last;
  const int parts = last - b + 2;
  // part 0 is the end of share b - 1, part k the beginning of share b - 1 + k
  auto entry = [&](int k) { return (int64_t)(k == 0 ? 2 * (b - 1) + 1 : 2 * (b - 1 + k)) * as.rows + r; };
  float top = -INFINITY;
  for (int k = lane; k < parts; k += 32) top = fmaxf(top, ws.stat[entry(k)].x);
#pragma unroll
  for (int d = 16; d > 0; d >>= 1) top = fmaxf(top, __shfl_xor_sync(0xffffffffu, top, d));
  float total = 0.f;
  float4 v = make_float4(0.f, 0.f, 0.f, 0.f);
  for (int k0 = 0; k0 < parts; k0 += 32) {
    float f = 0.f;
    if (k0 + lane < parts) {
      const float2 st = ws.stat[entry(k0 + lane)];
      f = st.x == -INFINITY ? 0.f : ex2(st.x - top);
      total += f * st.y;
    }
    const int m = min(32, parts - k0);
#pragma unroll 4
    for (int k = 0; k < m; ++k) {
      const float w = __shfl_sync(0xffffffffu, f, k);
      const float4 x = __ldcg(reinterpret_cast<const float4*>(ws.out + entry(k0 + k) * kHeadDim) + lane);
      v.x = fmaf(w, x.x, v.x);
      v.y = fmaf(w, x.y, v.y);
      v.z = fmaf(w, x.z, v.z);
      v.w = fmaf(w, x.w, v.w);
    }
  }
#pragma unroll
  for (int d = 16; d > 0; d >>= 1) total += __shfl_xor_sync(0xffffffffu, total, d);
  const int n = cache_len(cs, g, s, status);
  const bool none = (g.causal ? n - T + t + 1 : n) <= 0;
  const float inv = none ? 0.f : 1.0f / total;
  const int64_t tok = cs.new_off[s] + t;
  const int h = p.h * g.group + (r & 127) - in_tile * g.group;
  const __nv_bfloat162 lo = __floats2bfloat162_rn(v.x * inv, v.y * inv), hi = __floats2bfloat162_rn(v.z * inv, v.w * inv);
  uint2 bits;
  bits.x = *reinterpret_cast<const uint32_t*>(&lo);
  bits.y = *reinterpret_cast<const uint32_t*>(&hi);
  *reinterpret_cast<uint2*>(o.out + tok * g.out_tok + h * g.out_head + lane * 4) = bits;
  if (o.lse && lane == 0) o.lse[tok * g.hq + h] = none ? -INFINITY : (top + log2f(total)) * 0.6931471805599453f;
}

// The launches of a call: sequences with at most 16 query rows per KV head go to the kernel for few rows, the others to the
// tensor-core kernel (which wants 17 rows and more).
struct AttendPlan {
  AttendSeqs as;
  int grid;
};
struct AttendPlans { AttendPlan rows, tc; };

AttendPlans plan_attend(const CacheSeqs& cs, const CacheGeom& g, int sm_count) {
  AttendPlans p = {};
  AttendSeqs& few = p.rows.as;
  few.tile_keys = kRowsTile;
  few.rows = kRowsMost;
  few.block_tokens = few.tile_tokens = std::max(1, kRowsMost / g.group);
  few.start_weight = 1;
  AttendSeqs& many = p.tc.as;
  many.tile_keys = kTcTile;
  many.rows = 2 * kTcTile;
  many.tile_tokens = kTcTile / g.group;
  many.block_tokens = 2 * many.tile_tokens;
  many.start_weight = 2;
  for (int s = 0; s < cs.num_seqs; ++s) {
    const int T = cs.new_off[s + 1] - cs.new_off[s];
    if (T == 0) continue;
    AttendSeqs& as = (int64_t)T * g.group <= kRowsMost ? few : many;
    as.src[as.num++] = (uint8_t)s;
  }
  for (AttendPlan* x : {&p.rows, &p.tc}) {
    const AttendSeqs& as = x->as;
    int64_t total = 0;                             // of the weights (attend_weigh), at the longest
    for (int i = 0; i < as.num; ++i) {
      const int s = as.src[i];
      const int64_t blocks = (cs.new_off[s + 1] - cs.new_off[s] + as.block_tokens - 1) / as.block_tokens;
      total += blocks * (as.start_weight + (cs.kv_len[s] + as.tile_keys - 1) / as.tile_keys) * g.hkv;
    }
    x->grid = (int)std::min<int64_t>(total, sm_count);
  }
  return p;
}

// A page (or as many of its tokens as a tile has), both halves of the channels, one head, in one copy: in shared memory
// groups of eight tokens of 2 KB each, the eight rows of channels 0-63 followed by those of channels 64-127.
CUresult encode_pool(EncodeTiledFn encode, const CacheGeom& g, const void* p, int tile_keys, CUtensorMap* map) {
  const cuuint32_t estr[5] = {1, 1, 1, 1, 1};
  const cuuint64_t rows = (cuuint64_t)g.pool_pages << g.page_shift;
  const cuuint64_t dims[5] = {64, 8, 2, rows / 8, (cuuint64_t)g.hkv};
  const cuuint64_t strides[4] = {(cuuint64_t)g.kv_tok * 2, 128, (cuuint64_t)g.kv_tok * 16, (cuuint64_t)g.kv_head * 2};
  const cuuint32_t box[5] = {64, 8, 2, (cuuint32_t)(std::min(1 << g.page_shift, tile_keys) / 8), 1};
  return encode(map, CU_TENSOR_MAP_DATA_TYPE_BFLOAT16, 5, const_cast<void*>(p), dims, strides, box, estr,
                CU_TENSOR_MAP_INTERLEAVE_NONE, CU_TENSOR_MAP_SWIZZLE_128B, CU_TENSOR_MAP_L2_PROMOTION_L2_256B,
                CU_TENSOR_MAP_FLOAT_OOB_FILL_NONE);
}

// The tokens of a tile, the heads of a group, half of the channels: rows token * group + head of 128 bytes.
CUresult encode_queries(EncodeTiledFn encode, const CacheSeqs& cs, const CacheGeom& g, const void* q, int tile_tokens, CUtensorMap* map) {
  const cuuint32_t estr[3] = {1, 1, 1};
  const cuuint64_t dims[3] = {(cuuint64_t)kHeadDim, (cuuint64_t)g.hq, (cuuint64_t)cs.new_off[cs.num_seqs]};
  const cuuint64_t strides[2] = {(cuuint64_t)g.q_head * 2, (cuuint64_t)g.q_tok * 2};
  const cuuint32_t box[3] = {64, (cuuint32_t)g.group, (cuuint32_t)tile_tokens};
  return encode(map, CU_TENSOR_MAP_DATA_TYPE_BFLOAT16, 3, const_cast<void*>(q), dims, strides, box, estr,
                CU_TENSOR_MAP_INTERLEAVE_NONE, CU_TENSOR_MAP_SWIZZLE_128B, CU_TENSOR_MAP_L2_PROMOTION_L2_256B,
                CU_TENSOR_MAP_FLOAT_OOB_FILL_NONE);
}

}  // namespace

cudaError_t launch_attend_join(const Launch& L, const CacheSeqs& cs, const CacheGeom& g, const AttendSeqs& as, const AttendWs& ws,
                               int grid, const AttendOut& o) {
  if (grid < 2) return cudaSuccess;
  return launch_pdl(attend_join_kernel, dim3((unsigned)(grid - 1), (unsigned)((as.rows + kJoinWarps - 1) / kJoinWarps)),
                    dim3(kJoinWarps * 32), 0, L.stream, 1, cs, g, as, ws, grid, o, L.status);
}

size_t attend_ws_bytes(const CacheSeqs& cs, const CacheGeom& g, int sm_count) {
  const AttendPlans p = plan_attend(cs, g, sm_count);          // one launch after the other uses it
  return std::max(attend_ws_size(p.rows.grid, p.rows.as.rows), attend_ws_size(p.tc.grid, p.tc.as.rows));
}

cudaError_t launch_attend(const Launch& L, const CacheSeqs& cs, const CacheGeom& g, const void* q, const void* k, const void* v,
                          void* out, float* lse, void* ws, void* encode_fn, int* drv_err) {
  *drv_err = 0;
  const EncodeTiledFn encode = (EncodeTiledFn)encode_fn;
  const AttendOut o = {(uint16_t*)out, lse};
  const AttendPlans p = plan_attend(cs, g, L.sm_count);
  CUtensorMap q_map, k_map, v_map;
  auto pools = [&](int tile_keys) {
    CUresult r = encode_pool(encode, g, k, tile_keys, &k_map);
    if (r == CUDA_SUCCESS) r = encode_pool(encode, g, v, tile_keys, &v_map);
    *drv_err = (int)r;
    return r == CUDA_SUCCESS;
  };
  cudaError_t e = cudaSuccess;
  if (p.tc.as.num > 0) {
    if (!pools(p.tc.as.tile_keys)) return cudaErrorUnknown;
    *drv_err = (int)encode_queries(encode, cs, g, q, p.tc.as.tile_tokens, &q_map);
    if (*drv_err != 0) return cudaErrorUnknown;
    const AttendWs w = attend_ws(ws, p.tc.grid, p.tc.as.rows);
    e = launch_attend_tc(L, cs, g, p.tc.as, w, p.tc.grid, o, q_map, k_map, v_map);
    if (e == cudaSuccess) e = launch_attend_join(L, cs, g, p.tc.as, w, p.tc.grid, o);
  }
  if (e == cudaSuccess && p.rows.as.num > 0) {
    if (!pools(p.rows.as.tile_keys)) return cudaErrorUnknown;
    const AttendWs w = attend_ws(ws, p.rows.grid, p.rows.as.rows);
    e = launch_attend_rows(L, cs, g, p.rows.as, w, p.rows.grid, o, q, k_map, v_map);
    if (e == cudaSuccess) e = launch_attend_join(L, cs, g, p.rows.as, w, p.rows.grid, o);
  }
  return e;
}

}  // namespace cc
