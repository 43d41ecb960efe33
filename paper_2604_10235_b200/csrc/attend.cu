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
constexpr int kManyParts = 5;            // CTAs per problem from which on its parts are spread over warps,
constexpr int kSpreadRows = 20;          // if its rows are no more than that per CTA of the attention

// The join of the problems that are cut: blocks per (boundary between two shares, rows), idle unless the boundary is the first inside
// its problem.  The parts of a problem follow each other in the order of the CTAs.
//   out = sum_k 2^(m_k - M) o_k / sum_k 2^(m_k - M) l_k
// Bound by latency (what it reads is in L2), so whatever a row needs is asked for at once.
struct CutProblem {
  Place p;
  int first, parts;                                // its first boundary, parts (0: the boundary is not one)
  // Part 0 is the end of share first - 1, part k the beginning of share first - 1 + k.
  __device__ __forceinline__ int64_t entry(const AttendSeqs& as, int k, int r) const {
    return (int64_t)(k == 0 ? 2 * (first - 1) + 1 : 2 * (first - 1 + k)) * as.rows + r;
  }
};
// One whole warp; the places of 31 shares in one load.
__device__ __forceinline__ CutProblem cut_problem(const CacheGeom& g, const AttendSeqs& as, const AttendWs& ws, int grid, int b) {
  const int lane = threadIdx.x & 31;
  auto place = [&](int share) {
    const int4 x = share < grid ? __ldcg(reinterpret_cast<const int4*>(ws.place + share)) : make_int4(0, 0, 0, -1);
    return Place{x.x, x.y, x.z, x.w};
  };
  const Place near = place(b - 1 + lane);          // of shares b - 1, b, ...
  CutProblem c;
  c.first = b;
  c.parts = 0;
  c.p = Place{__shfl_sync(0xffffffffu, near.h, 1), __shfl_sync(0xffffffffu, near.i, 1), __shfl_sync(0xffffffffu, near.b, 1),
              __shfl_sync(0xffffffffu, near.tile, 1)};
  auto inside = [&](const Place& x) { return x.tile > 0 && x.h == c.p.h && x.i == c.p.i && x.b == c.p.b; };
  unsigned in = __ballot_sync(0xffffffffu, inside(near));
  if (c.p.tile <= 0 || (in & 1u)) return c;
  if (c.p.h >= g.hkv || c.p.i >= as.num || c.p.b >= as.seq[c.p.i].blocks) return c;      // (another call wrote to this workspace)
  c.parts = __ffs(~(in >> 1));                     // shares b, b + 1, ... that begin inside, and the one before
  if (in == 0xfffffffeu) {
    for (int s0 = b + 31;; s0 += 32) {
      in = __ballot_sync(0xffffffffu, inside(place(s0 + lane)));
      c.parts += in == 0xffffffffu ? 32 : __ffs(~in) - 1;
      if (in != 0xffffffffu) break;
    }
  }
  return c;
}
// The problem with index `at` in the list (heads outermost), found among all places; one whole warp.
__device__ __forceinline__ CutProblem problem_at(const AttendSeqs& as, const AttendWs& ws, int grid, int at) {
  const int lane = threadIdx.x & 31;
  CutProblem c;
  c.p = Place{at / as.blocks, 0, at % as.blocks, 0};
  while (c.p.b >= as.seq[c.p.i].blocks) c.p.b -= as.seq[c.p.i++].blocks;
  c.first = 0;
  c.parts = 0;
  for (int s0 = 0; s0 < grid; s0 += 5 * 32) {      // (five loads under way: as many as there are SMs)
    int4 x[5];
#pragma unroll
    for (int k = 0; k < 5; ++k) {
      const int share = s0 + k * 32 + lane;
      x[k] = share < grid ? __ldcg(reinterpret_cast<const int4*>(ws.place + share)) : make_int4(0, 0, 0, -1);
    }
#pragma unroll
    for (int k = 0; k < 5; ++k) {
      const unsigned in = __ballot_sync(0xffffffffu, x[k].w > 0 && x[k].x == c.p.h && x[k].y == c.p.i && x[k].z == c.p.b);
      if (in && c.parts == 0) {
        c.first = s0 + k * 32 + __ffs(in) - 1;
        c.parts = 1;
      }
      c.parts += __popc(in);
    }
  }
  return c;
}
__device__ __forceinline__ void add_part(float4& v, float w, const float4& x) {
  v.x = fmaf(w, x.x, v.x);
  v.y = fmaf(w, x.y, v.y);
  v.z = fmaf(w, x.z, v.z);
  v.w = fmaf(w, x.w, v.w);
}
// Four channels of a row; lse with the first of them.
__device__ __forceinline__ void store_row(const CacheGeom& g, const AttendOut& o, int64_t tok, int h, int c, const float4& v, float top,
                                          float total, bool none) {
  const float inv = none ? 0.f : 1.0f / total;
  const __nv_bfloat162 lo = __floats2bfloat162_rn(v.x * inv, v.y * inv), hi = __floats2bfloat162_rn(v.z * inv, v.w * inv);
  uint2 bits;
  bits.x = *reinterpret_cast<const uint32_t*>(&lo);
  bits.y = *reinterpret_cast<const uint32_t*>(&hi);
  *reinterpret_cast<uint2*>(o.out + tok * g.out_tok + h * g.out_head + c) = bits;
  if (o.lse && c == 0) o.lse[tok * g.hq + h] = none ? -INFINITY : (top + log2f(total)) * 0.6931471805599453f;
}

// Few rows of many parts: a block takes a row, each of its warps every eighth part, four of them under way at once.
__global__ void __launch_bounds__(kJoinWarps * 32)
attend_join_few_kernel(const CacheGeom g, const __grid_constant__ AttendSeqs as, const AttendWs ws, int grid, const AttendOut o,
                       DeviceStatus* status) {
  constexpr int kAhead = 4;
  __shared__ float4 fold[kJoinWarps][32];
  pdl_launch_dependents();
  pdl_wait();
  const int lane = threadIdx.x & 31, warp = threadIdx.x >> 5, r = blockIdx.y;
  const CutProblem c = cut_problem(g, as, ws, grid, blockIdx.x + 1);
  if (c.parts == 0) return;
  const AttendSeq q = as.seq[c.p.i];
  const int in_block = r / g.group, t = c.p.b * as.block_tokens + in_block;
  if (in_block >= as.block_tokens || t >= q.T) return;
  auto output = [&](int k) { return __ldcg(reinterpret_cast<const float4*>(ws.out + c.entry(as, k, r) * kHeadDim) + lane); };
  float4 x[kAhead];
#pragma unroll
  for (int k = 0; k < kAhead; ++k) x[k] = warp + k * kJoinWarps < c.parts ? output(warp + k * kJoinWarps) : make_float4(0.f, 0.f, 0.f, 0.f);
  auto stat = [&](int k) { return k < c.parts ? __ldcg(ws.stat + c.entry(as, k, r)) : make_float2(-INFINITY, 0.f); };
  const float2 first = stat(lane);
  float top = first.x;
  for (int k = 32 + lane; k < c.parts; k += 32) top = fmaxf(top, stat(k).x);
#pragma unroll
  for (int d = 16; d > 0; d >>= 1) top = fmaxf(top, __shfl_xor_sync(0xffffffffu, top, d));
  float total = 0.f;
  float4 v = make_float4(0.f, 0.f, 0.f, 0.f);
  for (int k0 = 0; k0 < c.parts; k0 += 32) {
    const float2 st = k0 == 0 ? first : stat(k0 + lane);
    const float f = st.x == -INFINITY ? 0.f : ex2(st.x - top);
    total += f * st.y;
#pragma unroll
    for (int k = 0; k < kAhead; ++k) {             // (32 parts: four per warp)
      const int part = warp + k * kJoinWarps;
      const float w = __shfl_sync(0xffffffffu, f, part);
      if (k0 + part < c.parts) add_part(v, w, k0 == 0 ? x[k] : output(k0 + part));
    }
  }
#pragma unroll
  for (int d = 16; d > 0; d >>= 1) total += __shfl_xor_sync(0xffffffffu, total, d);
  fold[warp][lane] = v;
  __syncthreads();
  if (warp != 0) return;
#pragma unroll
  for (int k = 1; k < kJoinWarps; ++k) add_part(v, 1.f, fold[k][lane]);
  const int n = attend_len(as, g, c.p.i, status);
  const int slots = g.causal ? n - q.T + t + 1 : n;
  store_row(g, o, q.row0 + t, c.p.h * g.group + r - in_block * g.group, lane * 4, v, top, total,
            slots <= 0 || (total == 0.f && attend_no_slot(as, g, c.p.i, slots)));
}

// Many parts of few problems: a block takes four rows of a problem, eight lanes a row, each of its warps every eighth part (38 tokens
// over 18246 keys, 2 KV heads: 30.6 -> 19.9 us).  Every block looks through all places, so it loses where there are many of
// them: 219 tokens in two sequences, 28 problems of 256 rows in five parts, 26.7 -> 36.9 us.
__global__ void __launch_bounds__(kJoinWarps * 32)
attend_join_spread_kernel(const CacheGeom g, const __grid_constant__ AttendSeqs as, const AttendWs ws, int grid, const AttendOut o,
                          DeviceStatus* status) {
  constexpr int kLanes = 8, kVecs = 32 / kLanes, kAhead = 2;
  __shared__ float4 fold[kJoinWarps][4][32];
  __shared__ float2 stats[4];
  pdl_launch_dependents();
  pdl_wait();
  const int lane = threadIdx.x & 31, warp = threadIdx.x >> 5, l = lane % kLanes;
  const CutProblem c = problem_at(as, ws, grid, blockIdx.x);
  if (c.parts == 0) return;
  const AttendSeq q = as.seq[c.p.i];
  auto token = [&](int r) {                        // of the sequence, -1: the block of tokens has no such row
    const int in_tile = (r & 127) / g.group, t = c.p.b * as.block_tokens + (r >> 7) * as.tile_tokens + in_tile;
    return r < as.rows && in_tile < as.tile_tokens && t < q.T ? t : -1;
  };
  const int r = blockIdx.y * 4 + lane / kLanes;
  const bool real = token(r) >= 0;
  if (!__any_sync(0xffffffffu, real)) return;      // (the same four rows in all warps)
  auto output = [&](int k, int v) { return __ldcg(reinterpret_cast<const float4*>(ws.out + c.entry(as, k, r) * kHeadDim) + v * kLanes + l); };
  auto stat = [&](int k) { return real && k < c.parts ? __ldcg(ws.stat + c.entry(as, k, r)) : make_float2(-INFINITY, 0.f); };
  float4 x[kAhead][kVecs];
  auto load = [&](int k0) {
#pragma unroll
    for (int k = 0; k < kAhead; ++k)
#pragma unroll
      for (int v = 0; v < kVecs; ++v) {
        const int part = k0 + k * kJoinWarps;
        x[k][v] = real && part < c.parts ? output(part, v) : make_float4(0.f, 0.f, 0.f, 0.f);
      }
  };
  load(warp);
  float2 st[4];
#pragma unroll
  for (int k = 0; k < 4; ++k) st[k] = stat(l + k * kLanes);
  float top = fmaxf(fmaxf(st[0].x, st[1].x), fmaxf(st[2].x, st[3].x));
  for (int k = 32 + l; k < c.parts; k += kLanes) top = fmaxf(top, stat(k).x);
#pragma unroll
  for (int d = kLanes / 2; d > 0; d >>= 1) top = fmaxf(top, __shfl_xor_sync(0xffffffffu, top, d));
  float total = 0.f;
#pragma unroll
  for (int k = 0; k < 4; ++k) total += st[k].x == -INFINITY ? 0.f : st[k].y * ex2(st[k].x - top);
  for (int k = 32 + l; k < c.parts; k += kLanes) {
    const float2 y = stat(k);
    total += y.x == -INFINITY ? 0.f : y.y * ex2(y.x - top);
  }
#pragma unroll
  for (int d = kLanes / 2; d > 0; d >>= 1) total += __shfl_xor_sync(0xffffffffu, total, d);
  float4 sum[kVecs];
#pragma unroll
  for (int v = 0; v < kVecs; ++v) sum[v] = make_float4(0.f, 0.f, 0.f, 0.f);
  for (int k0 = warp; k0 < c.parts; k0 += kAhead * kJoinWarps) {
    float w[kAhead];
#pragma unroll
    for (int k = 0; k < kAhead; ++k) {
      const float m = stat(k0 + k * kJoinWarps).x;
      w[k] = m == -INFINITY ? 0.f : ex2(m - top);
    }
    if (k0 > warp) load(k0);
#pragma unroll
    for (int k = 0; k < kAhead; ++k)
#pragma unroll
      for (int v = 0; v < kVecs; ++v)
        if (k0 + k * kJoinWarps < c.parts) add_part(sum[v], w[k], x[k][v]);
  }
#pragma unroll
  for (int v = 0; v < kVecs; ++v) fold[warp][lane / kLanes][v * kLanes + l] = sum[v];
  if (warp == 0 && l == 0) stats[lane / kLanes] = make_float2(top, total);
  __syncthreads();
  if (warp >= 4) return;
  const int t = token(blockIdx.y * 4 + warp);      // a warp per row now
  if (t < 0) return;
  float4 v = fold[0][warp][lane];
#pragma unroll
  for (int k = 1; k < kJoinWarps; ++k) add_part(v, 1.f, fold[k][warp][lane]);
  const int row = blockIdx.y * 4 + warp, n = attend_len(as, g, c.p.i, status), slots = g.causal ? n - q.T + t + 1 : n;
  store_row(g, o, q.row0 + t, c.p.h * g.group + (row & 127) % g.group, lane * 4, v, stats[warp].x, stats[warp].y,
            slots <= 0 || (stats[warp].y == 0.f && attend_no_slot(as, g, c.p.i, slots)));
}

// Many rows of a few parts: eight lanes take a row, all of them two parts at once, so that a warp does four rows in the time of one (a
// warp per row and four rows after one another took 15 us for 517 tokens over 8709 keys, this takes about 7).
__global__ void __launch_bounds__(kJoinWarps * 32)
attend_join_kernel(const CacheGeom g, const __grid_constant__ AttendSeqs as, const AttendWs ws, int grid, const AttendOut o,
                   DeviceStatus* status) {
  constexpr int kLanes = 8, kVecs = 32 / kLanes;   // per row; 16-byte vectors of its output per lane
  constexpr int kAhead = 2;                        // parts under way at once
  static_assert(kLanes % kAhead == 0, "weights of kLanes parts at a time");
  pdl_launch_dependents();
  pdl_wait();
  const int lane = threadIdx.x & 31, l = lane % kLanes;
  const CutProblem c = cut_problem(g, as, ws, grid, blockIdx.x + 1);
  if (c.parts == 0) return;
  const AttendSeq q = as.seq[c.p.i];
  const int r = (blockIdx.y * kJoinWarps + (threadIdx.x >> 5)) * (32 / kLanes) + lane / kLanes;
  const int in_tile = (r & 127) / g.group, t = c.p.b * as.block_tokens + (r >> 7) * as.tile_tokens + in_tile;
  const bool real = r < as.rows && in_tile < as.tile_tokens && t < q.T;
  if (!__any_sync(0xffffffffu, real)) return;
  auto output = [&](int k, int v) { return __ldcg(reinterpret_cast<const float4*>(ws.out + c.entry(as, k, r) * kHeadDim) + v * kLanes + l); };
  auto stat = [&](int k) { return real && k < c.parts ? __ldcg(ws.stat + c.entry(as, k, r)) : make_float2(-INFINITY, 0.f); };
  float4 x[kAhead][kVecs];
  auto load = [&](int k0) {
#pragma unroll
    for (int k = 0; k < kAhead; ++k)
#pragma unroll
      for (int v = 0; v < kVecs; ++v) x[k][v] = real && k0 + k < c.parts ? output(k0 + k, v) : make_float4(0.f, 0.f, 0.f, 0.f);
  };
  load(0);
  const float2 first = stat(l);
  float top = first.x;
  for (int k = kLanes + l; k < c.parts; k += kLanes) top = fmaxf(top, stat(k).x);
#pragma unroll
  for (int d = kLanes / 2; d > 0; d >>= 1) top = fmaxf(top, __shfl_xor_sync(0xffffffffu, top, d));
  float total = 0.f;
  float4 sum[kVecs];
#pragma unroll
  for (int v = 0; v < kVecs; ++v) sum[v] = make_float4(0.f, 0.f, 0.f, 0.f);
  float f = 0.f;                                   // weight of part k0 + l of every kLanes parts
  for (int k0 = 0; k0 < c.parts; k0 += kAhead) {
    if (k0 > 0) load(k0);
    if (k0 % kLanes == 0) {
      const float2 st = k0 == 0 ? first : stat(k0 + l);
      f = st.x == -INFINITY ? 0.f : ex2(st.x - top);
      total += f * st.y;
    }
#pragma unroll
    for (int k = 0; k < kAhead; ++k) {
      const float w = __shfl_sync(0xffffffffu, f, (k0 + k) % kLanes, kLanes);
#pragma unroll
      for (int v = 0; v < kVecs; ++v)
        if (k0 + k < c.parts) add_part(sum[v], w, x[k][v]);
    }
  }
#pragma unroll
  for (int d = kLanes / 2; d > 0; d >>= 1) total += __shfl_xor_sync(0xffffffffu, total, d);
  if (!real) return;
  const int n = attend_len(as, g, c.p.i, status), slots = g.causal ? n - q.T + t + 1 : n;
  const bool none = slots <= 0 || (total == 0.f && attend_no_slot(as, g, c.p.i, slots));
#pragma unroll
  for (int v = 0; v < kVecs; ++v)
    store_row(g, o, q.row0 + t, c.p.h * g.group + (r & 127) - in_tile * g.group, (v * kLanes + l) * 4, sum[v], top, total, none);
}

// The launches of a call: sequences with at most 16 query rows per KV head go to the kernel for few rows, the others to the
// tensor-core kernel (which wants 17 rows and more).
struct AttendPlan {
  AttendSeqs as;
  int grid;
};
constexpr int64_t kFewKeys = 400000;      // (keys x KV heads)
struct AttendPlans {
  AttendPlan rows, tc;
  bool too_much;                                   // 2^31 tiles and more
};

// Fewer problems than SMs in the tensor-core kernel: the number of CTAs for each of them, or 0: shares by weight, which even out problems
// of different lengths but give a CTA the end of one and the beginning of another.  What a choice takes, in tenths of a us: the
// longest share's steps of 128 keys, a second start (shares by weight), the join and its parts; fitted to 90 random batches timed with
// every number: 1.4 % below shares by weight on average, with 1 each and no join 504 tokens in three sequences over 251 to
// 848 keys 24.2 -> 19.2 us, 4 % above at worst.
int ctas_each(const CacheGeom& g, const AttendSeqs& as, int64_t total, int* grid) {
  constexpr int64_t kStep = 17, kStart = 50, kJoin = 50, kJoinPart = 1;
  const int64_t problems = (int64_t)as.blocks * g.hkv;
  if (problems > *grid) return 0;
  int64_t most = 0;
  for (int i = 0; i < as.num; ++i) most = std::max<int64_t>(most, (as.seq[i].n + (1 << as.tile_shift) - 1) >> as.tile_shift);
  int best = 0;
  int64_t least = (total + *grid - 1) / *grid * kStep + kStart + *grid / problems * kJoinPart;
  for (int64_t each = 1; each * problems <= *grid && each <= std::max<int64_t>(1, most); ++each) {
    const int64_t time = (most + each - 1) / each * kStep + (each > 1 ? kJoin + each * kJoinPart : 0);
    if (time < least) {
      least = time;
      best = (int)each;
    }
  }
  if (best > 0) *grid = (int)(best * problems);
  return best;
}

AttendPlans plan_attend(const CacheSeqs& cs, const CacheGeom& g, int sm_count) {
  AttendPlans p = {};
  AttendSeqs& few = p.rows.as;
  few.tile_shift = 6;
  static_assert(kRowsTile == 1 << 6 && kTcTile == 1 << 7, "tiles");
  few.block_tokens = few.tile_tokens = std::max(1, kRowsMost / g.group);
  few.start_weight = 1;
  AttendSeqs& many = p.tc.as;
  many.tile_shift = 7;
  many.rows = 2 * kTcTile;
  many.tile_tokens = kTcTile / g.group;
  many.block_tokens = 2 * many.tile_tokens;
  many.start_weight = 3;              // (2: ragged chunks 273 -> 254 us with 3; 4: 257)
  // A batch of both kinds goes to the tensor-core kernel as a whole unless the sequences with few rows have many keys: that kernel
  // takes a quarter longer over them (64 tokens over 245000 keys x 8 heads: 201 against 163 us) and a launch of their own costs
  // 14 us (16 sequences of 1 to 8 tokens, four of them with few rows: 59.4 against 45.2 us).
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
  // Rows that a block can have.
  few.rows = 0;
  for (int i = 0; i < few.num; ++i) few.rows = std::max(few.rows, few.seq[i].T * g.group);
  int64_t longest = 0;
  for (int i = 0; i < many.num; ++i) longest = std::max<int64_t>(longest, many.seq[i].T);
  if (longest <= many.tile_tokens) {
    many.rows = ((int)longest * g.group + 31) / 32 * 32;
    many.start_weight = 1;            // (fewer rows to hand over: drafts 46.9 us with 3, 45.9 with 1)
  }
  for (AttendPlan* x : {&p.rows, &p.tc}) {
    const AttendSeqs& as = x->as;
    int64_t total = 0;                             // of the weights (attend_weigh), at the longest
    for (int i = 0; i < as.num; ++i)
      total += (int64_t)as.seq[i].blocks * (as.start_weight + ((as.seq[i].n + (1 << as.tile_shift) - 1) >> as.tile_shift));
    total *= g.hkv;
    if (total >> 31) p.too_much = true;
    x->grid = (int)std::min<int64_t>(total, sm_count);
    for (int i = 0; i < as.num; ++i) x->as.blocks += as.seq[i].blocks;
    if (x == &p.tc && as.num > 0) x->as.each = ctas_each(g, x->as, total, &x->grid);
  }
  return p;
}

// A page (or as many of its tokens as a tile has), both halves of the channels, one head, in one copy: in shared memory
// groups of eight tokens of 2 KB each, the eight rows of channels 0-63 followed by those of channels 64-127.
// `fill`: what a copy from behind the pool brings.
CUresult encode_pool(EncodeTiledFn encode, const CacheGeom& g, const void* p, int tile_keys, CUtensorMapFloatOOBfill fill, CUtensorMap* map) {
  const cuuint32_t estr[5] = {1, 1, 1, 1, 1};
  const cuuint64_t rows = (cuuint64_t)g.pool_pages << g.page_shift;
  const cuuint64_t dims[5] = {64, 8, 2, rows / 8, (cuuint64_t)g.hkv};
  const cuuint64_t strides[4] = {(cuuint64_t)g.kv_tok * 2, 128, (cuuint64_t)g.kv_tok * 16, (cuuint64_t)g.kv_head * 2};
  const cuuint32_t box[5] = {64, 8, 2, (cuuint32_t)(std::min(1 << g.page_shift, tile_keys) / 8), 1};
  return encode(map, CU_TENSOR_MAP_DATA_TYPE_BFLOAT16, 5, const_cast<void*>(p), dims, strides, box, estr,
                CU_TENSOR_MAP_INTERLEAVE_NONE, CU_TENSOR_MAP_SWIZZLE_128B, CU_TENSOR_MAP_L2_PROMOTION_L2_256B, fill);
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
  if (as.each == 1) return cudaSuccess;            // no problem is cut
  const dim3 threads(kJoinWarps * 32);
  if (as.rows <= kRowsMost)
    return launch_pdl(attend_join_few_kernel, dim3((unsigned)(grid - 1), (unsigned)as.rows), threads, 0, L.stream, 1, g, as, ws, grid, o,
                      L.status);
  const int64_t problems = (int64_t)as.blocks * g.hkv;
  if (problems * kManyParts <= grid && problems * as.rows <= (int64_t)kSpreadRows * grid)
    return launch_pdl(attend_join_spread_kernel, dim3((unsigned)problems, (unsigned)((as.rows + 3) / 4)), threads, 0, L.stream, 1, g, as, ws,
                      grid, o, L.status);
  const int rows = kJoinWarps * 4;
  return launch_pdl(attend_join_kernel, dim3((unsigned)(grid - 1), (unsigned)((as.rows + rows - 1) / rows)), threads, 0, L.stream, 1, g,
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
    CUresult r = encode_pool(encode, g, k, tile_keys, CU_TENSOR_MAP_FLOAT_OOB_FILL_NAN_REQUEST_ZERO_FMA, &k_map);
    if (r == CUDA_SUCCESS) r = encode_pool(encode, g, v, tile_keys, CU_TENSOR_MAP_FLOAT_OOB_FILL_NONE, &v_map);
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
