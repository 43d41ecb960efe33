// Attention of few query rows (new tokens x group <= 16) over a paged cache: single tokens, drafted tokens.
//
//   o_r = sum_j p_rj v_j / sum_j p_rj,   p_rj = exp(scale q_r . k_j - reference_r)
//
// Every row of K and V is read once and 4 flops are done with each of its bytes per query row: bound by HBM (64 sequences, 245 k
// keys, 8 heads, 1.0 GB: 157 to 164 us, 6.1 to 6.4 TB/s), few keys by latency (2305 keys x 8 heads 9.8 to 10.3 us, of which the kernel 5).  The matrix
// instructions are mma.sync (m16n8k16): the 16 rows are their M side, against at least 64 of tcgen05.mma, and a tile's 32 per
// scheduler, some 500 clocks, fit well into the 1400 that its 32 KB take at this SM's share of the bandwidth.  The tensor-core
// kernel takes 201 us for the same.
//
// One CTA per SM.  A warp brings K and V tiles of 64 keys by TMA, one copy per page, through a ring of four stages of 32 KB,
// and the query rows of the next problem beside them; eight warps work on them in two groups that take tiles by turns, a
// warp on 16 keys of a tile.  Each warp has a running reference, sum and output of its own for all rows, so that
// tiles need no exchange between warps; they meet once per problem, each leaving its output in shared memory, where all threads
// add them up (one barrier; added by halves with three: 162 us).  A reference is replaced only when a logit, in units of
// log2, exceeds it by 8: outputs are sums in f32, and a probability of up to 2^8 rounds to bf16 like any other.
#include <cuda_bf16.h>

#include "attend_plan.cuh"
#include "exp2_poly.cuh"
#include "tc_ptx.cuh"

namespace cc {

namespace {

constexpr int kStages = 4;
constexpr int kGroups = 2;                       // groups of four warps
// A stage is always the same group's: a group that is a whole turn of the ring ahead would otherwise take the completed phase
// before the one that it waits for, which has the same parity.
static_assert(kStages % kGroups == 0, "stages by groups");
constexpr int kWorkers = 4 * kGroups;            // warps that compute
constexpr int kThreads = 32 * (1 + kWorkers);
constexpr uint32_t kTileBytes = kRowsTile * kHeadDim * 2;          // of K, or of V
constexpr int kQPitch = kHeadDim * 2 + 16;       // bytes of a query row in shared memory
constexpr int kFoldPitch = kHeadDim + 8;         // floats of an output row in shared memory
constexpr float kSlack = 8.0f;                   // log2 of how far a logit may lie above the reference

struct Shared {
  float fold[kWorkers][kRowsMost * kFoldPitch];  // outputs of the warps while they are joined
  uint8_t q[2][kRowsMost * kQPitch];
  float2 stat[kWorkers][kRowsMost];              // (reference, sum) of a problem's rows by warp
  AttendShare share;
  uint64_t full[kStages], empty[kStages], q_full[2], q_empty[2];
  int abort_flag;
};
constexpr size_t kSmem = 1024 + (size_t)kStages * 2 * kTileBytes + sizeof(Shared);
static_assert(kSmem <= kSmemPerCta, "shared memory of a CTA");

__device__ __forceinline__ void ldsm4(uint32_t addr, uint32_t (&r)[4]) {
  asm volatile("ldmatrix.sync.aligned.m8n8.x4.shared.b16 {%0,%1,%2,%3}, [%4];"
               : "=r"(r[0]), "=r"(r[1]), "=r"(r[2]), "=r"(r[3]) : "r"(addr) : "memory");
}
__device__ __forceinline__ void ldsm4_trans(uint32_t addr, uint32_t (&r)[4]) {
  asm volatile("ldmatrix.sync.aligned.m8n8.x4.trans.shared.b16 {%0,%1,%2,%3}, [%4];"
               : "=r"(r[0]), "=r"(r[1]), "=r"(r[2]), "=r"(r[3]) : "r"(addr) : "memory");
}
__device__ __forceinline__ void mma16816(float (&d)[4], const uint32_t (&a)[4], uint32_t b0, uint32_t b1) {
  asm volatile("mma.sync.aligned.m16n8k16.row.col.f32.bf16.bf16.f32 {%0,%1,%2,%3}, {%4,%5,%6,%7}, {%8,%9}, {%0,%1,%2,%3};"
               : "+f"(d[0]), "+f"(d[1]), "+f"(d[2]), "+f"(d[3])
               : "r"(a[0]), "r"(a[1]), "r"(a[2]), "r"(a[3]), "r"(b0), "r"(b1));
}
__device__ __forceinline__ float max_nan(float a, float b) {
  float d;
  asm("max.NaN.f32 %0, %1, %2;" : "=f"(d) : "f"(a), "f"(b));
  return d;
}
__device__ __forceinline__ uint32_t pack_bf16(float lo, float hi) {
  uint32_t r;
  asm("cvt.rn.bf16x2.f32 %0, %1, %2;" : "=r"(r) : "f"(hi), "f"(lo));
  return r;
}
__device__ __forceinline__ void worker_barrier() { asm volatile("bar.sync 1, %0;" ::"n"(kWorkers * 32) : "memory"); }

// Byte offset of 16-byte chunk `c` (of 16) of key `key` in a tile as the copies leave it: groups of eight keys, of each the
// channels 0-63 of the eight rows, then the channels 64-127, 128 bytes a row with its chunks swizzled by the row.
__device__ __forceinline__ uint32_t tile_at(int key, int c) {
  return (uint32_t)((key >> 3) * 2048 + (c >> 3) * 1024 + (key & 7) * 128 + (((c & 7) ^ (key & 7)) << 4));
}

__global__ void __launch_bounds__(kThreads, 1)
attend_rows_kernel(const CacheGeom g, const __grid_constant__ AttendSeqs as,
                   const __grid_constant__ CUtensorMap k_map, const __grid_constant__ CUtensorMap v_map,
                   const uint16_t* __restrict__ q, const AttendOut o, const AttendWs ws, DeviceStatus* status) {
  extern __shared__ uint8_t dyn[];
  uint8_t* ring = dyn + ((1024u - (smem_u32(dyn) & 1023u)) & 1023u);
  Shared* sh = reinterpret_cast<Shared*>(ring + (size_t)kStages * 2 * kTileBytes);
  const int warp = threadIdx.x >> 5, lane = threadIdx.x & 31;
  pdl_launch_dependents();
  if (warp == 1 && elect_one()) {
    prefetch_map(&k_map);
    prefetch_map(&v_map);
  }
  if (warp == 0) {
    if (lane < kStages) {
      mbar_init(smem_u32(&sh->full[lane]), 1);
      mbar_init(smem_u32(&sh->empty[lane]), 4);
    }
    if (lane < 2) {
      mbar_init(smem_u32(&sh->q_full[lane]), 1);
      mbar_init(smem_u32(&sh->q_empty[lane]), kWorkers);
    }
    if (lane == 0) sh->abort_flag = 0;
    fence_barrier_init();
  }
  for (int i = threadIdx.x; i < 2 * kRowsMost * kQPitch / 16; i += kThreads)     // rows that no problem has stay zero
    reinterpret_cast<uint4*>(sh->q)[i] = make_uint4(0u, 0u, 0u, 0u);
  fence_proxy_async();
  attend_share(g, as, &sh->share, ws.place, status);
  const BoundedWait pipe = {&sh->abort_flag, &status->code};

  if (warp == 0) {
    // ---------------------------------------------------------------- copies
    AttendWalk w;
    const int span = min(1 << g.page_shift, kRowsTile);        // keys per copy
    const int copies = kRowsTile / span;
    const uint32_t copy_bytes = (uint32_t)span * kHeadDim * 2;
    const bool elected = elect_one();
    // (No hint for L2: K and V of a sequence are read once, but sequences that a fork has made share pages.  Marked as the first to go,
    // 16 children each of 4 prompts of 16000 tokens, 8 heads, took 640 us instead of 554, 8 each of 8 of 4000 tokens 170 instead of 163;
    // sequences that share nothing 0.2 % less, one token over 131071 keys 0.9 %.)
    int stage = 0, seg = 0;
    uint32_t phase = 0;
    bool ok = true;
    for (bool more = w.first(g, as, &sh->share); more && ok; more = w.next(g, as, &sh->share), ++seg) {
      const int32_t* table = g.table + (int64_t)as.src[w.at.i] * g.table_stride;
      auto page_of = [&](int t) {                  // of this lane's copy, -1 where it has none
        const int key = t * kRowsTile + lane * span;
        return lane < copies && key < w.limit && t < w.t1 ? table[key >> g.page_shift] : -1;
      };
      int page = page_of(w.t0);                    // always one tile ahead
      const int buf = seg & 1;
      if (!bounded_wait(pipe, &sh->q_empty[buf], ((seg >> 1) & 1) ^ 1, CC_ERR_TIMEOUT, 70)) break;
      const int rows = min(as.block_tokens, w.q.T - w.at.b * as.block_tokens) * g.group;
      const uint32_t qb = smem_u32(&sh->q_full[buf]);
      if (elected) mbar_expect_tx(qb, (uint32_t)rows * kHeadDim * 2);
      __syncwarp();
      if (lane < rows) {
        const int t = lane / g.group, h = w.at.h * g.group + lane - t * g.group;
        const int64_t tok = w.q.row0 + w.at.b * as.block_tokens + t;
        bulk_load(smem_u32(sh->q[buf]) + lane * kQPitch, q + tok * g.q_tok + h * g.q_head, kHeadDim * 2, qb);
      }
      for (int t = w.t0; t < w.t1; ++t) {
        const int key = t * kRowsTile + lane * span;           // first key of this lane's copy
        const bool mine = lane < copies && key < w.limit;
        const int id = page;
        page = page_of(t + 1);
        if (!bounded_wait(pipe, &sh->empty[stage], phase ^ 1, CC_ERR_TIMEOUT, 71)) { ok = false; break; }
        const bool good = mine && id >= 0 && id < g.pool_pages;
        if (mine && !good) report_error(status, CC_ERR_DEVICE_FLAG, 620);
        const unsigned mask = __ballot_sync(0xffffffffu, mine);
        const int group8 = copy_group(g, good, id, key & ((1 << g.page_shift) - 1));
        const uint32_t fb = smem_u32(&sh->full[stage]);
        const uint32_t dst = smem_u32(ring) + (uint32_t)stage * 2 * kTileBytes;
        if (elected) mbar_expect_tx(fb, (uint32_t)__popc(mask) * 2u * copy_bytes);
        for (unsigned left = mask; left; left &= left - 1) {
          const int p = __ffs(left) - 1;
          const int at = __shfl_sync(0xffffffffu, group8, p);
          if (elected) {
            tma_load_5d(dst + p * copy_bytes, &k_map, fb, at, w.at.h);
            tma_load_5d(dst + kTileBytes + p * copy_bytes, &v_map, fb, at, w.at.h);
          }
        }
        if (++stage == kStages) { stage = 0; phase ^= 1; }
      }
    }
  } else {
    // ---------------------------------------------------------------- products
    const int me = warp - 1, group = me >> 2, quarter = me & 3;          // 16 keys of every second tile
    const int r0 = lane >> 2;                                            // rows r0 and r0 + 8
    const float c2 = g.scale * 1.4426950408889634f;
    // rows of the operands that this lane addresses for ldmatrix
    const int k_key = quarter * 16 + (lane & 7) + ((lane >> 4) << 3), k_chunk = (lane >> 3) & 1;
    const int v_key = quarter * 16 + (lane & 15), v_chunk = lane >> 4;
    AttendWalk w;
    int it = 0, seg = 0;             // tiles and problems of the share so far
    bool dead = false;
    for (bool more = w.first(g, as, &sh->share); more; more = w.next(g, as, &sh->share), ++seg) {
      const int buf = seg & 1;
      if (!dead) dead = !bounded_wait(pipe, &sh->q_full[buf], (seg >> 1) & 1, CC_ERR_TIMEOUT, 72);
      uint32_t qa[8][4];
      {
        const uint32_t base = smem_u32(sh->q[buf]) + (lane & 15) * kQPitch + (lane >> 4) * 16;
#pragma unroll
        for (int ks = 0; ks < 8; ++ks) ldsm4(base + ks * 32, qa[ks]);
        __syncwarp();
        if (lane == 0) mbar_arrive(smem_u32(&sh->q_empty[buf]));
      }
      const int tok0 = w.at.b * as.block_tokens;
      const int real = min(as.block_tokens, w.q.T - tok0) * g.group;       // rows of the problem
      int lim[2];                                                        // keys that rows r0 and r0 + 8 attend to
#pragma unroll
      for (int i = 0; i < 2; ++i) {
        const int r = r0 + 8 * i;
        lim[i] = r < real ? (g.causal ? max(0, w.q.n - w.q.T + tok0 + r / g.group + 1) : w.q.n) : 0;
      }
      const int most = w.limit;
      const int least = g.causal ? max(0, w.q.n - w.q.T + tok0 + 1) : w.q.n;
      float acc[16][4];
#pragma unroll
      for (int i = 0; i < 16; ++i)
#pragma unroll
        for (int e = 0; e < 4; ++e) acc[i][e] = 0.f;
      float ref[2] = {-INFINITY, -INFINITY}, sum[2] = {0.f, 0.f};
      for (int t = w.t0; t < w.t1; ++t, ++it) {
        if ((it & (kGroups - 1)) != group) continue;
        const int stage = it % kStages;
        if (!dead) dead = !bounded_wait(pipe, &sh->full[stage], (it / kStages) & 1, CC_ERR_TIMEOUT, 73);
        const uint32_t kt = smem_u32(ring) + (uint32_t)stage * 2 * kTileBytes, vt = kt + kTileBytes;
        const int key0 = t * kRowsTile + quarter * 16;
        if (!dead && key0 < most) {
          float sc[2][4] = {{0.f, 0.f, 0.f, 0.f}, {0.f, 0.f, 0.f, 0.f}};
#pragma unroll
          for (int ks = 0; ks < 8; ++ks) {
            uint32_t kb[4];
            ldsm4(kt + tile_at(k_key, 2 * ks + k_chunk), kb);
            mma16816(sc[0], qa[ks], kb[0], kb[1]);
            mma16816(sc[1], qa[ks], kb[2], kb[3]);
          }
          const bool edge = key0 + 16 > least;
          if (key0 + 16 > most) {        // rows of V that no row attends to may hold anything: 0 x NaN
            for (int i = (most - key0) * 16 + lane; i < 16 * 16; i += 32)
              *reinterpret_cast<uint4*>(ring + (size_t)stage * 2 * kTileBytes + kTileBytes +
                                        tile_at(quarter * 16 + (i >> 4), i & 15)) = make_uint4(0u, 0u, 0u, 0u);
            __syncwarp();
          }
          // Of the keys that some of the rows attend to and others do not, values of V that are infinite or no numbers would
          // reach them all (0 x inf): they count for the rows that attend to them here, and the product finds zeros.
          const bool shared_edge = edge && least < most;
          float x[2][4];                 // [row][key]: keys key0 + 2 (lane % 4) + {0, 1, 8, 9}
          float top[2];
#pragma unroll
          for (int i = 0; i < 2; ++i) {
#pragma unroll
            for (int e = 0; e < 4; ++e) {
              x[i][e] = sc[e >> 1][2 * i + (e & 1)] * c2;
              if (edge && key0 + 2 * (lane & 3) + (e & 1) + 8 * (e >> 1) >= lim[i]) x[i][e] = -INFINITY;
            }
            top[i] = max_nan(max_nan(x[i][0], x[i][1]), max_nan(x[i][2], x[i][3]));
            top[i] = max_nan(top[i], __shfl_xor_sync(0xffffffffu, top[i], 1));
            top[i] = max_nan(top[i], __shfl_xor_sync(0xffffffffu, top[i], 2));
          }
          if (__any_sync(0xffffffffu, !(top[0] <= ref[0] + kSlack && top[1] <= ref[1] + kSlack))) {
            if (__builtin_expect(__any_sync(0xffffffffu, top[0] != top[0] || top[1] != top[1]), 0)) {
              const uint32_t lost = missing_groups(as, g, w.at.i, key0, 2, most);
#pragma unroll
              for (int i = 0; i < 2; ++i) {
#pragma unroll
                for (int e = 0; e < 4; ++e)
                  if (lost >> (e >> 1) & 1u) x[i][e] = -INFINITY;
                // (a logit that is no number is not a reference)
                top[i] = fmaxf(fmaxf(x[i][0], x[i][1]), fmaxf(x[i][2], x[i][3]));
                top[i] = fmaxf(top[i], __shfl_xor_sync(0xffffffffu, top[i], 1));
                top[i] = fmaxf(top[i], __shfl_xor_sync(0xffffffffu, top[i], 2));
              }
            }
#pragma unroll
            for (int i = 0; i < 2; ++i) {
              const float up = fmaxf(ref[i], top[i]);
              const float f = ref[i] == -INFINITY ? 0.f : ex2(ref[i] - up);
              ref[i] = up;
              sum[i] *= f;
#pragma unroll
              for (int c = 0; c < 16; ++c) {
                acc[c][2 * i] *= f;
                acc[c][2 * i + 1] *= f;
              }
            }
          }
          if (shared_edge) {
            uint8_t* v_rows = ring + (size_t)stage * 2 * kTileBytes + kTileBytes;
            bool odd = false;
            for (int i = lane; i < 16 * 16; i += 32) odd |= any_odd(*reinterpret_cast<const uint4*>(v_rows + tile_at(quarter * 16 + (i >> 4), i & 15)));
            if (__any_sync(0xffffffffu, odd)) {
              for (int key = 0; key < 16; ++key) {
#pragma unroll
                for (int c = 0; c < 16; ++c) {
                  uint32_t* at = reinterpret_cast<uint32_t*>(v_rows + tile_at(quarter * 16 + key, c) + 4 * (lane & 3));
                  const uint32_t both = *at, keep = finite_halves(both);
                  const float bad[2] = {__uint_as_float((both & ~keep) << 16), __uint_as_float((both & ~keep) & 0xffff0000u)};
#pragma unroll
                  for (int i = 0; i < 2; ++i)
                    if (key0 + key < lim[i]) {
                      acc[c][2 * i] += bad[0];
                      acc[c][2 * i + 1] += bad[1];
                    }
                  __syncwarp();
                  *at = both & keep;
                }
              }
              __syncwarp();
            }
          }
          uint32_t pa[4];
#pragma unroll
          for (int i = 0; i < 2; ++i) {
            const float off = ref[i] == -INFINITY ? 0.f : ref[i];
            float p[4];
#pragma unroll
            for (int e = 0; e < 4; ++e) p[e] = ex2(x[i][e] - off);
            sum[i] += (p[0] + p[1]) + (p[2] + p[3]);
            pa[i] = pack_bf16(p[0], p[1]);
            pa[i + 2] = pack_bf16(p[2], p[3]);
          }
#pragma unroll
          for (int c = 0; c < 16; c += 2) {
            uint32_t vb[4];
            ldsm4_trans(vt + tile_at(v_key, c + v_chunk), vb);
            mma16816(acc[c], pa, vb[0], vb[1]);
            mma16816(acc[c + 1], pa, vb[2], vb[3]);
          }
          if (edge) fence_proxy_async();                   // this warp's stores before the copy that comes next
        }
        __syncwarp();
        if (lane == 0) mbar_arrive(smem_u32(&sh->empty[stage]));
      }

      // the warps' parts of the problem
#pragma unroll
      for (int i = 0; i < 2; ++i) {
        sum[i] += __shfl_xor_sync(0xffffffffu, sum[i], 1);
        sum[i] += __shfl_xor_sync(0xffffffffu, sum[i], 2);
      }
      if (seg > 0) worker_barrier();               // what the warps left of the problem before has been read
      if ((lane & 3) < 2) sh->stat[me][r0 + 8 * (lane & 1)] = make_float2(lane & 1 ? ref[1] : ref[0], lane & 1 ? sum[1] : sum[0]);
#pragma unroll
      for (int i = 0; i < 2; ++i) {
        if (8 * i >= real) break;
#pragma unroll
        for (int c = 0; c < 16; ++c)
          *reinterpret_cast<float2*>(sh->fold[me] + (r0 + 8 * i) * kFoldPitch + c * 8 + 2 * (lane & 3)) =
              make_float2(acc[c][2 * i], acc[c][2 * i + 1]);
      }
      worker_barrier();
      const bool whole = w.whole();
      for (int i = threadIdx.x - 32; i < real * 32; i += kWorkers * 32) {
        const int r = i >> 5, c = (i & 31) * 4;
        float2 st[kWorkers];
        float top = -INFINITY, total = 0.f;
#pragma unroll
        for (int k = 0; k < kWorkers; ++k) {
          st[k] = sh->stat[k][r];
          top = fmaxf(top, st[k].x);
        }
        float4 v = make_float4(0.f, 0.f, 0.f, 0.f);
#pragma unroll
        for (int k = 0; k < kWorkers; ++k) {
          const float f = st[k].x == -INFINITY ? 0.f : ex2(st[k].x - top);
          total = fmaf(st[k].y, f, total);
          const float4 part = *reinterpret_cast<const float4*>(sh->fold[k] + r * kFoldPitch + c);
          v.x = fmaf(part.x, f, v.x);
          v.y = fmaf(part.y, f, v.y);
          v.z = fmaf(part.z, f, v.z);
          v.w = fmaf(part.w, f, v.w);
        }
        if (whole) {
          const int t = r / g.group, h = w.at.h * g.group + r - t * g.group;
          const int64_t tok = w.q.row0 + tok0 + t;
          const int slots = g.causal ? w.q.n - w.q.T + tok0 + t + 1 : w.q.n;
          const bool none = slots <= 0 || (total == 0.f && attend_no_slot(as, g, w.at.i, slots));
          const float inv = none ? 0.f : 1.0f / total;
          *reinterpret_cast<uint2*>(o.out + tok * g.out_tok + h * g.out_head + c) =
              make_uint2(pack_bf16(v.x * inv, v.y * inv), pack_bf16(v.z * inv, v.w * inv));
          if (o.lse && c == 0) o.lse[tok * g.hq + h] = none ? -INFINITY : (top + log2f(total)) * 0.6931471805599453f;
        } else {
          const int64_t at = (int64_t)w.slot() * as.rows + r;
          *reinterpret_cast<float4*>(ws.out + at * kHeadDim + c) = v;
          if (c == 0) ws.stat[at] = make_float2(top, total);
        }
      }
    }
  }
  __syncthreads();
  if (sh->abort_flag) {
    // copies still in flight get time to land before shared memory is released
#pragma unroll 1
    for (int i = 0; i < 2000; ++i) __nanosleep(1000);
  }
}

}  // namespace

cudaError_t launch_attend_rows(const Launch& L, const CacheGeom& g, const AttendSeqs& as, const AttendWs& ws,
                               int grid, const AttendOut& o, const void* q, const CUtensorMap& k_map, const CUtensorMap& v_map) {
  const cudaError_t e = allow_smem(attend_rows_kernel);
  if (e != cudaSuccess) return e;
  return launch_pdl(attend_rows_kernel, dim3((unsigned)grid), dim3(kThreads), kSmem, L.stream, 1, g, as, k_map, v_map,
                    (const uint16_t*)q, o, ws, L.status);
}

}  // namespace cc
