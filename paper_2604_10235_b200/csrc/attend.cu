// Attention over a paged cache: which kernel takes which sequences, the tensor maps, the join of cut problems.
#include <cuda_bf16.h>

#include <stdint.h>

#include <algorithm>

#include "attend_plan.cuh"
#include "exp2_poly.cuh"
#include "tc_ptx.cuh"

namespace cc {

namespace {

constexpr int kJoinWarps = 8;

// The join of the problems that are cut: blocks per (boundary between two shares, rows), idle unless the boundary is the first inside
// its problem.  The parts of a problem follow each other in the order of the CTAs.
//   out = sum_k 2^(m_k - M) o_k / sum_k 2^(m_k - M) l_k
// Bound by latency (what it reads is in L2).  FEW rows of many parts (the kernel for few rows): a warp takes a row, and its first eight
// outputs are asked for together with their statistics.  Many rows of a few parts: eight lanes take a row, all of them two
// parts at once, so that a warp does four rows in the time of one (a warp per row and four rows after one another: 15 us of
// the 90 of 517 tokens over 8709 keys).
template <bool FEW>
__global__ void __launch_bounds__(kJoinWarps * 32)
attend_join_kernel(const CacheGeom g, const __grid_constant__ AttendSeqs as, const AttendWs ws, int grid, const AttendOut o,
                   DeviceStatus* status) {
  constexpr int kLanes = FEW ? 32 : 8;             // per row
  constexpr int kVecs = 32 / kLanes;               // 16-byte vectors of a row's output per lane
  constexpr int kAhead = FEW ? 8 : 2;              // parts under way at once
  pdl_launch_dependents();
  pdl_wait();
  const int lane = threadIdx.x & 31;
  const int b = blockIdx.x + 1;                    // the share that begins at the boundary
  auto place = [&](int share) {
    const int4 x = share < grid ? __ldcg(reinterpret_cast<const int4*>(ws.place + share)) : make_int4(0, 0, 0, -1);
    return Place{x.x, x.y, x.z, x.w};
  };
  const Place near = place(b - 1 + lane);          // of shares b - 1, b, ...
  const Place p = {__shfl_sync(0xffffffffu, near.h, 1), __shfl_sync(0xffffffffu, near.i, 1), __shfl_sync(0xffffffffu, near.b, 1),
                   __shfl_sync(0xffffffffu, near.tile, 1)};
  auto inside = [&](const Place& x) { return x.tile > 0 && x.h == p.h && x.i == p.i && x.b == p.b; };
  unsigned in = __ballot_sync(0xffffffffu, inside(near));
  if (p.tile <= 0 || (in & 1u)) return;
  if (p.h >= g.hkv || p.i >= as.num || p.b >= as.seq[p.i].blocks) return;      // (another call wrote to this workspace)
  int parts = __ffs(~(in >> 1));                   // shares b, b + 1, ... that begin inside, and the one before
  if (in == 0xfffffffeu) {
    for (int s0 = b + 31;; s0 += 32) {
      in = __ballot_sync(0xffffffffu, inside(place(s0 + lane)));
      parts += in == 0xffffffffu ? 32 : __ffs(~in) - 1;
      if (in != 0xffffffffu) break;
    }
  }
  const AttendSeq q = as.seq[p.i];
  const int n = attend_len(as, g, p.i, status);
  const int l = lane % kLanes;                     // of the row
  for (int r0 = (blockIdx.y * kJoinWarps + (threadIdx.x >> 5)) * (32 / kLanes); r0 < as.rows; r0 += gridDim.y * kJoinWarps * (32 / kLanes)) {
    const int r = r0 + lane / kLanes;
    const int in_tile = (r & 127) / g.group, t = p.b * as.block_tokens + (r >> 7) * as.tile_tokens + in_tile;
    const bool real = in_tile < as.tile_tokens && t < q.T;
    if (!__any_sync(0xffffffffu, real)) continue;
    // part 0 is the end of share b - 1, part k the beginning of share b - 1 + k
    auto entry = [&](int k) { return (int64_t)((k == 0 ? 2 * (b - 1) + 1 : 2 * (b - 1 + k)) * as.rows + r); };
    auto output = [&](int k, int v) { return __ldcg(reinterpret_cast<const float4*>(ws.out + entry(k) * kHeadDim) + v * kLanes + l); };
    auto stat = [&](int k) { return real && k < parts ? __ldcg(ws.stat + entry(k)) : make_float2(-INFINITY, 0.f); };
    float4 x[kAhead][kVecs];
    auto load = [&](int k0) {
#pragma unroll
      for (int k = 0; k < kAhead; ++k)
#pragma unroll
        for (int v = 0; v < kVecs; ++v) x[k][v] = real && k0 + k < parts ? output(k0 + k, v) : make_float4(0.f, 0.f, 0.f, 0.f);
    };
    load(0);
    const float2 first = stat(l);
    float top = first.x;
    for (int k = kLanes + l; k < parts; k += kLanes) top = fmaxf(top, stat(k).x);
#pragma unroll
    for (int d = kLanes / 2; d > 0; d >>= 1) top = fmaxf(top, __shfl_xor_sync(0xffffffffu, top, d));
    float total = 0.f;
    float4 sum[kVecs];
#pragma unroll
    for (int v = 0; v < kVecs; ++v) sum[v] = make_float4(0.f, 0.f, 0.f, 0.f);
    float f = 0.f;                                 // weight of part k0 + l of every kLanes parts
    for (int k0 = 0; k0 < parts; k0 += kAhead) {
      if (k0 > 0) load(k0);
#pragma unroll
      for (int k = 0; k < kAhead; ++k) {
        if (k0 + k >= parts) break;
        if ((k0 + k) % kLanes == 0) {
          const float2 st = k0 + k == 0 ? first : stat(k0 + k + l);
          f = st.x == -INFINITY ? 0.f : ex2(st.x - top);
          total += f * st.y;
        }
        const float w = __shfl_sync(0xffffffffu, f, (k0 + k) % kLanes, kLanes);
#pragma unroll
        for (int v = 0; v < kVecs; ++v) {
          sum[v].x = fmaf(w, x[k][v].x, sum[v].x);
          sum[v].y = fmaf(w, x[k][v].y, sum[v].y);
          sum[v].z = fmaf(w, x[k][v].z, sum[v].z);
          sum[v].w = fmaf(w, x[k][v].w, sum[v].w);
        }
      }
    }
#pragma unroll
    for (int d = kLanes / 2; d > 0; d >>= 1) total += __shfl_xor_sync(0xffffffffu, total, d);
    if (!real) continue;
    const bool none = (g.causal ? n - q.T + t + 1 : n) <= 0;
    const float inv = none ? 0.f : 1.0f / total;
    const int64_t tok = q.row0 + t;
    const int h = p.h * g.group + (r & 127) - in_tile * g.group;
#pragma unroll
    for (int v = 0; v < kVecs; ++v) {
      const __nv_bfloat162 lo = __floats2bfloat162_rn(sum[v].x * inv, sum[v].y * inv), hi = __floats2bfloat162_rn(sum[v].z * inv, sum[v].w * inv);
      uint2 bits;
      bits.x = *reinterpret_cast<const uint32_t*>(&lo);
      bits.y = *reinterpret_cast<const uint32_t*>(&hi);
      *reinterpret_cast<uint2*>(o.out + tok * g.out_tok + h * g.out_head + (v * kLanes + l) * 4) = bits;
    }
    if (o.lse && l == 0) o.lse[tok * g.hq + h] = none ? -INFINITY : (top + log2f(total)) * 0.6931471805599453f;
  }
}

// The launches of a call: sequences with at most 16 query rows per KV head go to the kernel for few rows, the others to the
// tensor-core kernel (which wants 17 rows and more).
struct AttendPlan {
  AttendSeqs as;
  int grid;
};
constexpr int kSplit = 4;
constexpr int64_t kFewKeys = 400000;      // (keys x KV heads)
struct AttendPlans {
  AttendPlan rows, tc;
  bool too_much;                                   // 2^31 tiles and more
};

AttendPlans plan_attend(const CacheSeqs& cs, const CacheGeom& g, int sm_count) {
  AttendPlans p = {};
  AttendSeqs& few = p.rows.as;
  few.tile_shift = 6;
  static_assert(kRowsTile == 1 << 6 && kTcTile == 1 << 7, "tiles");
  few.rows = kRowsMost;
  few.block_tokens = few.tile_tokens = std::max(1, kRowsMost / g.group);
  few.start_weight = 1;
  AttendSeqs& many = p.tc.as;
  many.tile_shift = 7;
  many.rows = 2 * kTcTile;
  many.tile_tokens = kTcTile / g.group;
  many.block_tokens = 2 * many.tile_tokens;
  many.start_weight = 3;              // (2: ragged chunks 273 -> 254 us with 3; 4: 257)
  // A batch of both kinds goes to the tensor-core kernel as a whole unless the sequences with few rows have many keys: that kernel
  // takes a quarter longer over them (64 tokens over 245000 keys x 8 heads: 213 against 168 us) and a launch of their own costs
  // 10 us (16 sequences of 1 to 8 tokens, four of them with few rows: 58.6 against 48.7 us).
  int64_t few_keys = 0;
  bool mixed = false;
  auto is_few = [&](int T) { return (int64_t)T * g.group <= kRowsMost; };
  for (int s = 0; s < cs.num_seqs; ++s) {
    const int T = cs.new_off[s + 1] - cs.new_off[s];
    if (is_few(T)) few_keys += T > 0 ? cs.kv_len[s] : 0;
    else mixed = true;
  }
  const bool apart = !mixed || few_keys * g.hkv > kFewKeys;
  for (int s = 0; s < cs.num_seqs; ++s) {
    const int T = cs.new_off[s + 1] - cs.new_off[s];
    if (T == 0) continue;
    AttendSeqs& as = is_few(T) && apart ? few : many;
    as.seq[as.num] = AttendSeq{cs.new_off[s], T, cs.kv_len[s], (T + as.block_tokens - 1) / as.block_tokens};
    as.src[as.num++] = (uint8_t)s;
  }
  // Rows that a block can have (a short chunk has fewer than two tiles of them).
  int64_t longest = 0;
  for (int i = 0; i < many.num; ++i) longest = std::max<int64_t>(longest, many.seq[i].T);
  if (longest <= many.tile_tokens) many.rows = ((int)longest * g.group + 31) / 32 * 32;
  for (AttendPlan* x : {&p.rows, &p.tc}) {
    const AttendSeqs& as = x->as;
    int64_t total = 0;                             // of the weights (attend_weigh), at the longest
    for (int i = 0; i < as.num; ++i)
      total += (int64_t)as.seq[i].blocks * (as.start_weight + ((as.seq[i].n + (1 << as.tile_shift) - 1) >> as.tile_shift));
    total *= g.hkv;
    if (total >> 31) p.too_much = true;
    x->grid = (int)std::min<int64_t>(total, sm_count);
    // Fewer problems than SMs, and all alike: as many CTAs for each.  A CTA then has part of one problem instead of the end of one and
    // the beginning of another, which costs it a start and an end (kSplit tiles; 517 tokens over 8709 keys 96 -> 90 us).
    int64_t problems = 0, most = 0, least = INT64_MAX;
    for (int i = 0; i < as.num; ++i) {
      const int64_t n = as.seq[i].n, first = g.causal ? std::max<int64_t>(0, n - as.seq[i].T) : n;
      problems += (int64_t)as.seq[i].blocks * g.hkv;
      most = std::max(most, (n + (1 << as.tile_shift) - 1) >> as.tile_shift);
      least = std::min(least, first >> as.tile_shift);
    }
    if (x == &p.tc && problems > 0 && problems <= x->grid) {
      const int64_t each = x->grid / problems;
      if (least >= 2 * each && most / each < total / x->grid + kSplit) {
        x->as.each = (int)each;
        x->grid = (int)(each * problems);
      }
    }
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

cudaError_t launch_attend_join(const Launch& L, const CacheGeom& g, const AttendSeqs& as, const AttendWs& ws,
                               int grid, const AttendOut& o) {
  if (grid < 2) return cudaSuccess;
  const bool few = as.rows <= kRowsMost;
  const int rows = kJoinWarps * (few ? 1 : 4);     // of a block at a time
  auto kern = few ? attend_join_kernel<true> : attend_join_kernel<false>;
  return launch_pdl(kern, dim3((unsigned)(grid - 1), (unsigned)((as.rows + rows - 1) / rows)), dim3(kJoinWarps * 32), 0, L.stream, 1, g,
                    as, ws, grid, o, L.status);
}

size_t attend_ws_bytes(const CacheSeqs& cs, const CacheGeom& g, int sm_count) {
  const AttendPlans p = plan_attend(cs, g, sm_count);          // one launch after the other uses it
  if (p.too_much) return 0;
  return std::max<size_t>({256, attend_ws_size(p.rows.grid, p.rows.as.rows), attend_ws_size(p.tc.grid, p.tc.as.rows)});
}

cudaError_t launch_attend(const Launch& L, const CacheSeqs& cs, const CacheGeom& g, const void* q, const void* k, const void* v,
                          void* out, float* lse, void* ws, void* encode_fn, int* drv_err) {
  *drv_err = 0;
  const EncodeTiledFn encode = (EncodeTiledFn)encode_fn;
  const AttendOut o = {(uint16_t*)out, lse, (uintptr_t)out % 32 == 0 && g.out_tok % 16 == 0 && g.out_head % 16 == 0};
  const AttendPlans p = plan_attend(cs, g, L.sm_count);
  if (p.too_much) return cudaErrorInvalidConfiguration;
  CUtensorMap q_map, k_map, v_map;
  auto pools = [&](int tile_keys) {
    CUresult r = encode_pool(encode, g, k, tile_keys, &k_map);
    if (r == CUDA_SUCCESS) r = encode_pool(encode, g, v, tile_keys, &v_map);
    *drv_err = (int)r;
    return r == CUDA_SUCCESS;
  };
  cudaError_t e = cudaSuccess;
  if (p.tc.as.num > 0) {
    if (!pools(1 << p.tc.as.tile_shift)) return cudaErrorUnknown;
    *drv_err = (int)encode_queries(encode, cs, g, q, p.tc.as.tile_tokens, &q_map);
    if (*drv_err != 0) return cudaErrorUnknown;
    const AttendWs w = attend_ws(ws, p.tc.grid, p.tc.as.rows);
    e = launch_attend_tc(L, g, p.tc.as, w, p.tc.grid, o, v, q_map, k_map, v_map);
    if (e == cudaSuccess) e = launch_attend_join(L, g, p.tc.as, w, p.tc.grid, o);
  }
  if (e == cudaSuccess && p.rows.as.num > 0) {
    if (!pools(1 << p.rows.as.tile_shift)) return cudaErrorUnknown;
    const AttendWs w = attend_ws(ws, p.rows.grid, p.rows.as.rows);
    e = launch_attend_rows(L, g, p.rows.as, w, p.rows.grid, o, q, k_map, v_map);
    if (e == cudaSuccess) e = launch_attend_join(L, g, p.rows.as, w, p.rows.grid, o);
  }
  return e;
}

}  // namespace cc
