// How the two attention kernels share out their work, and the form of their partial results.
//
// A problem is (KV head, sequence, block of new tokens): the block's tokens x group query rows against the keys that
// any of them attends to, in tiles.  Problems lie one after the other, heads outermost, each with a weight of its
// tiles plus a constant for its start; every CTA takes an equal share of the total weight, so it has a stretch of
// (problem, tile) places that may begin and end inside a problem.  A problem that one CTA has whole is finished there;
// of one that is cut every CTA leaves its rows' (maximum, sum, unnormalised output) and a second launch joins them
// in the order of the CTAs.  The shares depend on the lengths alone: equal calls give equal bits.
//
// Lengths may be known only on the device, so the shares are computed there, by every CTA for itself.
#pragma once

#include "cache_step.cuh"

namespace cc {

struct AttendSeqs {            // the sequences of one launch
  int num;                     // sequences with new tokens that this kernel takes
  int block_tokens;            // new tokens per block
  int tile_tokens;             // of them in each 128 rows: row r of a block is row r % 128 of its tile r / 128, token
                               // (r % 128) / group of the tile
  int tile_keys;               // keys per tile
  int start_weight;            // weight of a problem's start, in tiles (at least 1)
  int rows;                    // rows of a block (and of a partial result)
  uint8_t src[CC_MAX_SEQS];    // index of the sequence in the call
};

// A place in the list of problems: `tile` is the first tile of the problem behind the place.
struct Place { int h, i, b, tile; };         // head, entry of AttendSeqs, block

struct AttendShare {           // shared memory
  long long weight[CC_MAX_SEQS + 1];         // of the sequences before, of one head
  int len[CC_MAX_SEQS];                      // n_s by entry
  Place from, to;
};

__device__ __forceinline__ int attend_limit(const CacheSeqs& cs, const CacheGeom& g, const AttendSeqs& as, int s, int n, int b) {
  if (!g.causal) return n;
  const int T = cs.new_off[s + 1] - cs.new_off[s];
  const int last = min(T, (b + 1) * as.block_tokens);
  return max(0, n - T + last);
}
// Tiles of a block: those that hold a key which one of its tokens attends to.
__device__ __forceinline__ int attend_tiles(const CacheSeqs& cs, const CacheGeom& g, const AttendSeqs& as, int s, int n, int b) {
  return (attend_limit(cs, g, as, s, n, b) + as.tile_keys - 1) / as.tile_keys;
}
__device__ __forceinline__ int attend_blocks(const CacheSeqs& cs, const AttendSeqs& as, int s) {
  return (cs.new_off[s + 1] - cs.new_off[s] + as.block_tokens - 1) / as.block_tokens;
}

// Fills sh->len and sh->weight; all threads of the block, which must synchronise afterwards (twice inside).
__device__ __forceinline__ void attend_weigh(const CacheSeqs& cs, const CacheGeom& g, const AttendSeqs& as, AttendShare* sh,
                                             DeviceStatus* st) {
  const int lane = threadIdx.x & 31, warp = threadIdx.x >> 5, warps = blockDim.x >> 5;
  for (int i = threadIdx.x; i < as.num; i += blockDim.x) {
    const int s = as.src[i], n = cache_len(cs, g, s, st);
    sh->len[i] = n;
    const int nb = attend_blocks(cs, as, s);
    if (nb == 1) sh->weight[i + 1] = as.start_weight + attend_tiles(cs, g, as, s, n, 0);
    else if (!g.causal) sh->weight[i + 1] = (long long)nb * (as.start_weight + attend_tiles(cs, g, as, s, n, 0));
  }
  __syncthreads();
  if (g.causal) {
    for (int i = warp; i < as.num; i += warps) {
      const int s = as.src[i], n = sh->len[i], nb = attend_blocks(cs, as, s);
      if (nb == 1) continue;
      long long sum = 0;
      for (int b = lane; b < nb; b += 32) sum += as.start_weight + attend_tiles(cs, g, as, s, n, b);
#pragma unroll
      for (int o = 16; o > 0; o >>= 1) sum += __shfl_xor_sync(0xffffffffu, sum, o);
      if (lane == 0) sh->weight[i + 1] = sum;
    }
    __syncthreads();
  }
  if (warp == 0) {                                 // running sums: two entries per lane
    static_assert(CC_MAX_SEQS == 64, "two entries per lane");
    const long long a = 2 * lane < as.num ? sh->weight[2 * lane + 1] : 0;
    const long long b = 2 * lane + 1 < as.num ? sh->weight[2 * lane + 2] : 0;
    long long run = a + b;
#pragma unroll
    for (int o = 1; o < 32; o <<= 1) {
      const long long up = __shfl_up_sync(0xffffffffu, run, o);
      if (lane >= o) run += up;
    }
    if (lane == 0) sh->weight[0] = 0;
    sh->weight[2 * lane + 1] = run - b;
    sh->weight[2 * lane + 2] = run;
  }
}

// CTAs that get a share.
__device__ __forceinline__ int attend_workers(const AttendSeqs& as, const AttendShare* sh, int hkv, int grid) {
  const long long total = sh->weight[as.num] * hkv;
  return total < grid ? (int)total : grid;
}

// The place at which the share of CTA `cta` of `workers` begins (cta == workers: behind everything); one whole warp.
__device__ __forceinline__ Place attend_place(const CacheSeqs& cs, const CacheGeom& g, const AttendSeqs& as,
                                              const AttendShare* sh, int cta, int workers) {
  const int lane = threadIdx.x & 31;
  const long long per_head = sh->weight[as.num], total = per_head * g.hkv;
  Place p = {g.hkv, 0, 0, 0};
  if (cta >= workers) return p;
  // total * cta fits: 2^31 tokens / 64 keys x 2^31 / 128 heads stay far below 2^53
  const long long at = total / workers * cta + total % workers * cta / workers;
  p.h = (int)(at / per_head);
  long long rest = at - per_head * p.h;
  const int e0 = 2 * lane, e1 = 2 * lane + 1;
  const bool in0 = e0 < as.num && sh->weight[e0] <= rest && rest < sh->weight[e0 + 1];
  const bool in1 = e1 < as.num && sh->weight[e1] <= rest && rest < sh->weight[e1 + 1];
  const unsigned m0 = __ballot_sync(0xffffffffu, in0), m1 = __ballot_sync(0xffffffffu, in1);
  p.i = m0 ? 2 * (__ffs(m0) - 1) : 2 * (__ffs(m1) - 1) + 1;
  rest -= sh->weight[p.i];
  const int s = as.src[p.i], n = sh->len[p.i], nb = attend_blocks(cs, as, s);
  for (int b0 = 0; b0 < nb; b0 += 32) {
    const int b = b0 + lane;
    const long long w = b < nb ? as.start_weight + attend_tiles(cs, g, as, s, n, b) : 0;
    long long run = w;
#pragma unroll
    for (int o = 1; o < 32; o <<= 1) {
      const long long up = __shfl_up_sync(0xffffffffu, run, o);
      if (lane >= o) run += up;
    }
    const unsigned m = __ballot_sync(0xffffffffu, b < nb && rest < run);
    if (m) {
      const int l = __ffs(m) - 1;
      const long long before = __shfl_sync(0xffffffffu, run - w, l);
      p.b = b0 + l;
      p.tile = (int)max(0LL, rest - before - as.start_weight);
      break;
    }
    rest -= __shfl_sync(0xffffffffu, run, 31);
  }
  return p;
}

// The problems of a share one after the other.
struct AttendWalk {
  Place at, to;
  int s, n, T, n_blocks, tiles;      // of the current problem
  int t0, t1;                        // tiles of it in this share
  __device__ __forceinline__ bool same(const Place& a, const Place& b) const { return a.h == b.h && a.i == b.i && a.b == b.b; }
  __device__ __forceinline__ void seq(const CacheSeqs& cs, const AttendSeqs& as, const AttendShare* sh) {
    s = as.src[at.i];
    n = sh->len[at.i];
    T = cs.new_off[s + 1] - cs.new_off[s];
    n_blocks = attend_blocks(cs, as, s);
  }
  __device__ __forceinline__ bool open(const CacheSeqs& cs, const CacheGeom& g, const AttendSeqs& as) {
    if (at.h >= g.hkv) return false;
    const bool last = same(at, to);
    if (last && to.tile == 0) return false;        // the problem belongs to the next share
    tiles = attend_tiles(cs, g, as, s, n, at.b);
    t0 = at.tile;
    t1 = last ? to.tile : tiles;
    return t0 < t1 || tiles == 0;
  }
  __device__ __forceinline__ bool first(const CacheSeqs& cs, const CacheGeom& g, const AttendSeqs& as, const AttendShare* sh) {
    at = sh->from;
    to = sh->to;
    if (at.h >= g.hkv) return false;
    seq(cs, as, sh);
    return open(cs, g, as);
  }
  __device__ __forceinline__ bool next(const CacheSeqs& cs, const CacheGeom& g, const AttendSeqs& as, const AttendShare* sh) {
    if (same(at, to)) return false;
    at.tile = 0;
    if (++at.b == n_blocks) {
      at.b = 0;
      if (++at.i == as.num) {
        at.i = 0;
        ++at.h;
      }
      if (at.h >= g.hkv) return false;
      seq(cs, as, sh);
    }
    return open(cs, g, as);
  }
  __device__ __forceinline__ bool whole() const { return t0 == 0 && t1 == tiles; }
  // The entry of the workspace for what this share has of a cut problem: a share begins inside one problem at most and
  // ends inside one at most.
  __device__ __forceinline__ int slot() const { return 2 * (int)blockIdx.x + (t0 == 0 ? 1 : 0); }
};

// Workspace of a launch: per CTA the place at which its share begins, then two partial results per CTA: outputs
// [rows][128], then (maximum in units of log2, sum) [rows].
struct AttendWs {
  Place* place;                      // [grid]; tile = -1: no share
  float* out;                        // [2 * grid][rows][128]
  float2* stat;                      // [2 * grid][rows]
};
inline size_t attend_ws_size(int grid, int rows) {
  return ((size_t)grid * sizeof(Place) + 255) / 256 * 256 + (size_t)2 * grid * rows * (kHeadDim * 4 + 8);
}
inline AttendWs attend_ws(void* ws, int grid, int rows) {
  AttendWs w;
  w.place = (Place*)ws;
  w.out = (float*)((char*)ws + ((size_t)grid * sizeof(Place) + 255) / 256 * 256);
  w.stat = (float2*)(w.out + (size_t)2 * grid * rows * kHeadDim);
  return w;
}

struct AttendOut {
  uint16_t* out;
  float* lse;                        // or null
};

// Launches the join of cut problems (attend.cu).
cudaError_t launch_attend_join(const Launch& L, const CacheSeqs& cs, const CacheGeom& g, const AttendSeqs& as, const AttendWs& ws,
                               int grid, const AttendOut& o);
// The kernel for up to 16 rows per block (attend_rows.cu) and the one for blocks of 256 (attend_tc.cu).
cudaError_t launch_attend_rows(const Launch& L, const CacheSeqs& cs, const CacheGeom& g, const AttendSeqs& as, const AttendWs& ws,
                               int grid, const AttendOut& o, const void* q, const CUtensorMap& k_map, const CUtensorMap& v_map);
cudaError_t launch_attend_tc(const Launch& L, const CacheSeqs& cs, const CacheGeom& g, const AttendSeqs& as, const AttendWs& ws,
                             int grid, const AttendOut& o, const CUtensorMap& q_map, const CUtensorMap& k_map,
                             const CUtensorMap& v_map);
constexpr int kTcTile = 128;         // keys per tile of attend_tc.cu, and query rows per tile (two tiles a block)
constexpr int kRowsTile = 64;        // keys per tile of attend_rows.cu
constexpr int kRowsMost = 16;        // query rows of its blocks

}  // namespace cc
