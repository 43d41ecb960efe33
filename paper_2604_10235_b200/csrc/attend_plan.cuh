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

// One sequence of a launch: first row of its new tokens, their number, n_s or its upper bound, blocks of new tokens.
struct __align__(16) AttendSeq { int row0, T, n, blocks; };

struct AttendSeqs {            // the sequences of one launch
  int num;                     // sequences with new tokens that this kernel takes
  int block_tokens;            // new tokens per block
  int tile_tokens;             // of them in each 128 rows: row r of a block is row r % 128 of its tile r / 128, token
                               // (r % 128) / group of the tile
  int tile_shift;              // keys per tile = 1 << tile_shift
  int start_weight;            // weight of a problem's start, in tiles (at least 1)
  int rows;                    // rows of a block (and of a partial result)
  int each;                    // > 0: no shares by weight, every problem has that many CTAs
  int blocks;                  // of all sequences
  AttendSeq seq[CC_MAX_SEQS];
  uint8_t src[CC_MAX_SEQS];    // index of the sequence in the call
};

// A place in the list of problems: `tile` is the first tile of the problem behind the place.
struct __align__(16) Place { int h, i, b, tile; };         // head, entry of AttendSeqs, block

struct AttendShare {           // shared memory
  AttendSeq seq[CC_MAX_SEQS];                // n as the call finds it
  unsigned weight[CC_MAX_SEQS + 1];          // of the sequences before, of one head (all heads together: below 2^31)
  Place from, to;
};

// n_s as the call finds it.
__device__ __forceinline__ int attend_len(const AttendSeqs& as, const CacheGeom& g, int i, DeviceStatus* st) {
  const int most = as.seq[i].n;
  if (g.dev_lens == nullptr) return most;
  const int n = g.dev_lens[as.src[i]];
  if (n >= 0 && n <= most) return n;
  report_error(st, CC_ERR_DEVICE_FLAG, 600);
  return n < 0 ? 0 : most;
}
// Keys that the block's last token attends to.
__device__ __forceinline__ int attend_limit(const AttendSeq& q, int block_tokens, int causal, int b) {
  return causal ? max(0, q.n - q.T + min(q.T, (b + 1) * block_tokens)) : q.n;
}
// Tiles of a block: those that hold a key which one of its tokens attends to.
__device__ __forceinline__ int attend_tiles(const AttendSeq& q, const AttendSeqs& as, int causal, int b) {
  return (attend_limit(q, as.block_tokens, causal, b) + (1 << as.tile_shift) - 1) >> as.tile_shift;
}

// Fills sh->seq and sh->weight; all threads of the block, which must synchronise afterwards.
__device__ __forceinline__ void attend_weigh(const CacheGeom& g, const AttendSeqs& as, AttendShare* sh, DeviceStatus* st) {
  const int lane = threadIdx.x & 31, warp = threadIdx.x >> 5, warps = blockDim.x >> 5;
  bool blocks = false;
  for (int i = threadIdx.x; i < as.num; i += blockDim.x) {
    AttendSeq q = as.seq[i];
    q.n = attend_len(as, g, i, st);
    sh->seq[i] = q;
    // (of a causal chunk of several blocks each block has a limit of its own: below)
    if (as.each) sh->weight[i + 1] = (unsigned)q.blocks;
    else if (q.blocks == 1 || !g.causal) sh->weight[i + 1] = (unsigned)q.blocks * (as.start_weight + attend_tiles(q, as, g.causal, 0));
    else blocks = true;
  }
  if (__syncthreads_or(blocks)) {
    for (int i = warp; i < as.num; i += warps) {
      const AttendSeq q = sh->seq[i];
      if (q.blocks == 1) continue;
      unsigned sum = 0;
      for (int b = lane; b < q.blocks; b += 32) sum += as.start_weight + attend_tiles(q, as, g.causal, b);
      sum = __reduce_add_sync(0xffffffffu, sum);
      if (lane == 0) sh->weight[i + 1] = sum;
    }
    __syncthreads();
  }
  if (warp == 0) {                                 // running sums: two entries per lane
    static_assert(CC_MAX_SEQS == 64, "two entries per lane");
    const unsigned a = 2 * lane < as.num ? sh->weight[2 * lane + 1] : 0;
    const unsigned b = 2 * lane + 1 < as.num ? sh->weight[2 * lane + 2] : 0;
    unsigned run = a + b;
#pragma unroll
    for (int o = 1; o < 32; o <<= 1) {
      const unsigned up = __shfl_up_sync(0xffffffffu, run, o);
      if (lane >= o) run += up;
    }
    if (lane == 0) sh->weight[0] = 0;
    sh->weight[2 * lane + 1] = run - b;
    sh->weight[2 * lane + 2] = run;
  }
}

// CTAs that get a share.
__device__ __forceinline__ int attend_workers(const AttendSeqs& as, const AttendShare* sh, int hkv, int grid) {
  return (int)min(sh->weight[as.num] * (unsigned)hkv * max(as.each, 1), (unsigned)grid);
}

// The place at which the share of CTA `cta` of `workers` begins (cta == workers: behind everything); one whole warp.
__device__ __forceinline__ Place attend_place(const CacheGeom& g, const AttendSeqs& as, const AttendShare* sh, int cta, int workers) {
  const int lane = threadIdx.x & 31;
  const unsigned per_head = sh->weight[as.num], total = per_head * (unsigned)g.hkv;
  Place p = {g.hkv, 0, 0, 0};
  if (cta >= workers) return p;
  const unsigned each = total / (unsigned)workers, extra = total - each * (unsigned)workers;
  const unsigned at = as.each ? (unsigned)(cta / as.each)
                              : each * (unsigned)cta + extra * (unsigned)cta / (unsigned)workers;    // floor(total * cta / workers)
  p.h = (int)(at / per_head);
  unsigned rest = at - per_head * (unsigned)p.h;
  const int e0 = 2 * lane, e1 = 2 * lane + 1;
  const bool in0 = e0 < as.num && sh->weight[e0] <= rest && rest < sh->weight[e0 + 1];
  const bool in1 = e1 < as.num && sh->weight[e1] <= rest && rest < sh->weight[e1 + 1];
  const unsigned m0 = __ballot_sync(0xffffffffu, in0), m1 = __ballot_sync(0xffffffffu, in1);
  p.i = m0 ? 2 * (__ffs(m0) - 1) : 2 * (__ffs(m1) - 1) + 1;
  rest -= sh->weight[p.i];
  const AttendSeq q = sh->seq[p.i];
  if (as.each) {
    p.b = (int)rest;
    const int tiles = attend_tiles(q, as, g.causal, p.b), part = cta % as.each;
    p.tile = part * ((tiles + as.each - 1) / as.each);
    if (part > 0 && p.tile >= tiles) {             // (fewer tiles than CTAs: the next problem's beginning)
      p.tile = 0;
      if (++p.b == q.blocks) {
        p.b = 0;
        if (++p.i == as.num) {
          p.i = 0;
          ++p.h;
        }
      }
    }
    return p;
  }
  if (q.blocks == 1) {
    p.tile = max(0, (int)rest - as.start_weight);
    return p;
  }
  for (int b0 = 0; b0 < q.blocks; b0 += 32) {
    const int b = b0 + lane;
    const unsigned w = b < q.blocks ? as.start_weight + attend_tiles(q, as, g.causal, b) : 0;
    unsigned run = w;
#pragma unroll
    for (int o = 1; o < 32; o <<= 1) {
      const unsigned up = __shfl_up_sync(0xffffffffu, run, o);
      if (lane >= o) run += up;
    }
    const unsigned m = __ballot_sync(0xffffffffu, b < q.blocks && rest < run);
    if (m) {
      const int l = __ffs(m) - 1;
      const unsigned before = __shfl_sync(0xffffffffu, run - w, l);
      p.b = b0 + l;
      p.tile = max(0, (int)(rest - before) - as.start_weight);
      break;
    }
    rest -= __shfl_sync(0xffffffffu, run, 31);
  }
  return p;
}

// The whole beginning of a kernel: sh->from and sh->to, and the workspace's entry.  Where the lengths are the call's own, all of it
// is arithmetic on the parameters and runs before the launch before this one has ended.
__device__ __forceinline__ void attend_share(const CacheGeom& g, const AttendSeqs& as, AttendShare* sh, Place* places,
                                             DeviceStatus* st) {
  const int warp = threadIdx.x >> 5;
  if (g.dev_lens) pdl_wait();
  attend_weigh(g, as, sh, st);
  __syncthreads();
  const int workers = attend_workers(as, sh, g.hkv, gridDim.x);
  Place p = {0, 0, 0, -1};
  if (warp < 2) {
    p = attend_place(g, as, sh, blockIdx.x + warp, workers);
    if ((threadIdx.x & 31) == 0) (warp == 0 ? sh->from : sh->to) = p;
  }
  pdl_wait();
  if (threadIdx.x == 0) places[blockIdx.x] = (int)blockIdx.x < workers ? p : Place{0, 0, 0, -1};
  __syncthreads();
}

// The problems of a share one after the other.
struct AttendWalk {
  Place at, to;
  AttendSeq q;                       // of the current problem
  int limit, tiles;                  // keys that any of its tokens attends to, tiles that hold them
  int t0, t1;                        // tiles of it in this share
  __device__ __forceinline__ bool same(const Place& a, const Place& b) const { return a.h == b.h && a.i == b.i && a.b == b.b; }
  __device__ __forceinline__ bool open(const CacheGeom& g, const AttendSeqs& as, const AttendShare* sh) {
    if (at.h >= g.hkv) return false;
    const bool last = same(at, to);
    if (last && to.tile == 0) return false;        // the problem belongs to the next share
    q = sh->seq[at.i];
    limit = attend_limit(q, as.block_tokens, g.causal, at.b);
    tiles = (limit + (1 << as.tile_shift) - 1) >> as.tile_shift;
    t0 = at.tile;
    t1 = last ? to.tile : tiles;
    return t0 < t1 || tiles == 0;
  }
  __device__ __forceinline__ bool first(const CacheGeom& g, const AttendSeqs& as, const AttendShare* sh) {
    at = sh->from;
    to = sh->to;
    return open(g, as, sh);
  }
  __device__ __forceinline__ bool next(const CacheGeom& g, const AttendSeqs& as, const AttendShare* sh) {
    if (same(at, to)) return false;
    at.tile = 0;
    if (++at.b == q.blocks) {
      at.b = 0;
      if (++at.i == as.num) {
        at.i = 0;
        ++at.h;
      }
    }
    return open(g, as, sh);
  }
  __device__ __forceinline__ bool whole() const { return t0 == 0 && t1 == tiles; }
  // The entry of the workspace for what this share has of a cut problem: a share begins inside one problem at most and
  // ends inside one at most.
  __device__ __forceinline__ int slot() const { return 2 * (int)blockIdx.x + (t0 == 0 ? 1 : 0); }
};

// Slots on a page that is not one of the pool take no part.  Their copies start behind the pool's last row, where the map of K gives no
// numbers and that of V zeros: logits that are no numbers are what the kernels look for anyway, so that only then a
// warp asks the page table.  (Over 57 batches of keys that are all there 0.5 % on average; 2.4 % with an entry per tile that says which keys
// are missing and that every warp reads.)
__device__ __forceinline__ int copy_group(const CacheGeom& g, bool good, int page, int in_page) {       // first group of eight rows
  return good ? (int)((((int64_t)page << g.page_shift) + in_page) >> 3) : (int)(((int64_t)g.pool_pages << g.page_shift) >> 3);
}
// Groups of eight keys of the sequence from key0 (a multiple of eight) on that are missing, a bit each; one whole warp.
__device__ __forceinline__ uint32_t missing_groups(const AttendSeqs& as, const CacheGeom& g, int i, int key0, int groups, int limit) {
  const int lane = threadIdx.x & 31, key = key0 + lane * 8;
  int page = 0;
  if (lane < groups && key < limit) page = g.table[(int64_t)as.src[i] * g.table_stride + (key >> g.page_shift)];
  return __ballot_sync(0xffffffffu, page < 0 || page >= g.pool_pages);
}
// Whether none of the first `lim` slots of a sequence lies on a page of the pool.  Asked where a row's sum is zero: a reference is a logit
// of its row and gives 1, so such a row had no slot, or logits of minus infinity alone (whose softmax is no number).
__device__ __forceinline__ bool attend_no_slot(const AttendSeqs& as, const CacheGeom& g, int i, int lim) {
  const int32_t* table = g.table + (int64_t)as.src[i] * g.table_stride;
#pragma unroll 1
  for (int p = 0; (p << g.page_shift) < lim; ++p) {
    const int page = table[p];
    if (page >= 0 && page < g.pool_pages) return false;
  }
  return true;
}

// Pairs of bf16: a mask of the finite ones, and whether any of eight is infinite or no number.
__device__ __forceinline__ uint32_t odd_halves(uint32_t two) { return ((two & 0x7f807f80u) + 0x00800080u) & 0x80008000u; }
__device__ __forceinline__ uint32_t finite_halves(uint32_t two) {
  const uint32_t odd = odd_halves(two);
  return (odd & 0x8000u ? 0u : 0xffffu) | (odd & 0x80000000u ? 0u : 0xffff0000u);
}
__device__ __forceinline__ bool any_odd(const uint4& x) {
  return (odd_halves(x.x) | odd_halves(x.y) | odd_halves(x.z) | odd_halves(x.w)) != 0;
}

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
  bool wide;                         // rows of out begin on 32-byte boundaries
};

// Launches the join of cut problems (attend.cu).
cudaError_t launch_attend_join(const Launch& L, const CacheGeom& g, const AttendSeqs& as, const AttendWs& ws,
                               int grid, const AttendOut& o);
// The kernel for up to 16 rows per block (attend_rows.cu) and the one for blocks of 256 (attend_tc.cu).
cudaError_t launch_attend_rows(const Launch& L, const CacheGeom& g, const AttendSeqs& as, const AttendWs& ws,
                               int grid, const AttendOut& o, const void* q, const CUtensorMap& k_map, const CUtensorMap& v_map);
cudaError_t launch_attend_tc(const Launch& L, const CacheGeom& g, const AttendSeqs& as, const AttendWs& ws,
                             int grid, const AttendOut& o, const void* v, const CUtensorMap& q_map, const CUtensorMap& k_map,
                             const CUtensorMap& v_map);
constexpr int kTcTile = 128;         // keys per tile of attend_tc.cu, and query rows per tile (two tiles a block)
constexpr int kRowsTile = 64;        // keys per tile of attend_rows.cu
constexpr int kRowsMost = 16;        // query rows of its blocks

}  // namespace cc
