// Attention of many query rows (chunks of new tokens) over a paged cache, on the tensor cores of sm_100a.
//
// A block has two tiles of 128 rows, row = token * group + head of the group, so that K and V of a KV head are read once for
// its whole group.  Per tile of 128 keys and of rows:
//
//   S = Q K^T           tcgen05.mma, both operands in shared memory, S in tensor memory (128 lanes x 128 columns)
//   P = 2^(S c - ref)   one thread per row: S to registers, maximum, exponentials, P as bf16 back over S
//   O += P V            tcgen05.mma, P from tensor memory, V as it lies in the cache (channels contiguous: MN-major)
//
// Tensor memory holds S and O of both tiles, all 512 columns.  While the four warps of one tile compute exponentials the tensor
// core works on the other tile, and P goes to it in two halves, so that the product with V starts when the first is there.
//
// The reference of a row's exponentials need not be its maximum, only near it: P up to 2^24 rounds to bf16 and sums in f32 like
// P up to 1.  So only tiles with masked keys look at their maximum beforehand, the others compute with the reference that there is
// (of a row's first keys); where the sum of a half tile shows that a logit is far above it (or no number), nothing has been
// handed over yet, the row's maximum becomes the reference, its O is scaled in tensor memory and the half is computed again.
// One pair of exponentials in eight is evaluated on the FMA pipe (exp2_poly.cuh, good to 7.8e-5, a fiftieth of what P loses as bf16): 517
// tokens over 8709 keys take 79.6 us with one pair in four, 77.7 with one in eight, 77.3 with one in sixteen; 2048 over 32768, at
// the power limit, 1042, 1058 and 1054, within what two runs differ by.
//
// Roles (320 threads, one CTA per SM): warps 0-3 and 4-7 the softmax of the two tiles, warp 8 the copies (Q once per
// problem, K and V by turns through a ring of five stages of 32 KB, a copy per page), warp 9 the products.
#include <cuda_bf16.h>

#include "attend_plan.cuh"
#include "exp2_poly.cuh"
#include "tc_ptx.cuh"

namespace cc {

namespace {

constexpr int kThreads = 320;
constexpr int kTmaWarp = 8, kMmaWarp = 9;
constexpr int kStages = 5;
constexpr uint32_t kTileBytes = kTcTile * kHeadDim * 2;        // of K, of V, or of one tile of Q
constexpr float kSlack = 8.0f;                                 // a maximum that far (log2) above the reference replaces it
constexpr float kMostSum = 16777216.0f;                        // of half a tile
constexpr float kMostPoly = 100.0f;                            // arguments up to here are computed on the FMA pipe
constexpr float kLog2e = 1.4426950408889634f, kLn2 = 0.6931471805599453f;

struct Shared {
  AttendShare share;
  uint64_t full[kStages], empty[kStages];
  uint64_t q_full, q_empty;
  uint64_t s_full[2], p_full[2][2], half_done[2], o_full[2], o_empty[2];       // per tile of the block (P: per half of it)
  uint32_t tmem_base;
  int abort_flag;
  int odd_values;                // V has had infinities or no numbers among keys that only some rows of a block attend to
};
constexpr size_t kSmem = 1024 + (size_t)(kStages + 2) * kTileBytes + sizeof(Shared);
static_assert(kSmem <= kSmemPerCta, "shared memory of a CTA");

__device__ __forceinline__ float max3_nan(float a, float b, float c) {
  float d;
  asm("max.NaN.f32 %0, %1, %2, %3;" : "=f"(d) : "f"(a), "f"(b), "f"(c));
  return d;
}
__device__ __forceinline__ void store32(void* p, const uint32_t* v) {      // 32 bytes, on a 32-byte boundary
  asm volatile("st.global.v8.b32 [%0], {%1, %2, %3, %4, %5, %6, %7, %8};"
               ::"l"(p), "r"(v[0]), "r"(v[1]), "r"(v[2]), "r"(v[3]), "r"(v[4]), "r"(v[5]), "r"(v[6]), "r"(v[7]) : "memory");
}
__device__ __forceinline__ uint32_t pack_bf16(float lo, float hi) {
  uint32_t r;
  asm("cvt.rn.bf16x2.f32 %0, %1, %2;" : "=r"(r) : "f"(hi), "f"(lo));
  return r;
}

// 2^(v c + off) of 32 values as bf16, added to `sum`; POLY: some on the FMA pipe, whose largest value goes into `reach`.
template <bool POLY>
__device__ __forceinline__ void exponentials(const uint32_t (&v)[32], uint64_t c2, uint64_t off2, uint32_t (&p)[16], uint64_t (&sum)[2],
                                             float& reach) {
#pragma unroll
  for (int e = 0; e < 16; ++e) {
    const float a = __uint_as_float(v[2 * e]), b = __uint_as_float(v[2 * e + 1]);
    const uint64_t x = fma2(pack2(a, b), c2, off2);
    const bool poly = POLY && e % 8 == 7;
    const uint64_t y = poly ? ex2_pair_fma(x) : ex2_pair_sfu(x);
    if (poly) reach = max3_nan(reach, a, b);
    sum[e & 1] = add2(sum[e & 1], y);
    float y0, y1;
    unpack2(y, y0, y1);
    p[e] = pack_bf16(y0, y1);
  }
}
__device__ __forceinline__ float total_of(const uint64_t (&sum)[2]) {
  float a, b;
  unpack2(add2(sum[0], sum[1]), a, b);
  return a + b;
}
__device__ __forceinline__ float max32_nan(const uint32_t (&v)[32]) {
  float m0 = __uint_as_float(v[0]), m1 = __uint_as_float(v[1]);
#pragma unroll
  for (int e = 2; e < 30; e += 4) {
    m0 = max3_nan(m0, __uint_as_float(v[e]), __uint_as_float(v[e + 1]));
    m1 = max3_nan(m1, __uint_as_float(v[e + 2]), __uint_as_float(v[e + 3]));
  }
  return max3_nan(max3_nan(m0, m1, __uint_as_float(v[30])), __uint_as_float(v[31]), __uint_as_float(v[31]));
}

__device__ __forceinline__ uint64_t offset_of(float ref) {
  const float off = ref == -INFINITY ? 0.f : -ref;
  return pack2(off, off);
}
// Whether a row of the warp has a logit far above its reference, or no number.
__device__ __forceinline__ bool out_of_range(bool real, const uint64_t (&part)[2], float reach, float c2, float ref) {
  return __any_sync(0xffffffffu, real && !(total_of(part) <= kMostSum && fmaf(reach, c2, -ref) <= kMostPoly));
}
// Makes `high` the row's reference where it is far above the one that there is, and scales what the row has: its sum and, with
// `scale_o`, its O in tensor memory (the products with V so far are complete).
__device__ __forceinline__ void raise(float high, bool real, float& ref, uint64_t (&sum)[2], bool scale_o, uint32_t o_addr) {
  if (!__any_sync(0xffffffffu, real && !(high <= ref + kSlack))) return;
  // a row of infinities or of values that are no numbers has no reference: everything becomes NaN
  float up = max3_nan(ref, high, high);
  if (up == INFINITY) up = NAN;
  const float f = ref == -INFINITY ? 0.f : ex2(ref - up);
  ref = up;
  const uint64_t f2 = pack2(f, f);
  sum[0] = mul2(sum[0], f2);
  sum[1] = mul2(sum[1], f2);
  if (scale_o) {
#pragma unroll 1
    for (int c = 0; c < 8; ++c) {
      uint32_t x[16];
      tmem_ld16(o_addr + c * 16, x);
      tmem_wait_ld();
#pragma unroll
      for (int e = 0; e < 16; ++e) x[e] = __float_as_uint(__uint_as_float(x[e]) * f);
      tmem_st16(o_addr + c * 16, x);
    }
  }
}
// Writes minus infinity over the logits of missing keys (groups of eight, a bit each), from chunk `from` of 32 keys on; the maximum of
// the chunks' first `last` keys.
__device__ __forceinline__ float mask_missing(uint32_t s_addr, int from, int last, uint32_t lost, uint32_t (&v)[32]) {
  float high = -INFINITY;
#pragma unroll 1
  for (int c = from; c < 4; ++c) {
    tmem_ld32(s_addr + c * 32, v);
    tmem_wait_ld();
#pragma unroll
    for (int e = 0; e < 32; ++e)
      if (c * 32 + e >= last || (lost >> (c * 4 + (e >> 3)) & 1u)) v[e] = 0xff800000u;
    tmem_st32(s_addr + c * 32, v);
    high = max3_nan(high, max32_nan(v), high);
  }
  tmem_wait_st();
  return high;
}
// Half of a tile of P is complete.
__device__ __forceinline__ void hand_over(uint32_t bar, int lane) {
  tmem_wait_st();
  tc_fence_before();
  __syncwarp();
  if (lane == 0) mbar_arrive(bar);
}

__global__ void __launch_bounds__(kThreads, 1)
attend_tc_kernel(const CacheGeom g, const __grid_constant__ AttendSeqs as,
                 const __grid_constant__ CUtensorMap q_map, const __grid_constant__ CUtensorMap k_map,
                 const __grid_constant__ CUtensorMap v_map, const uint16_t* __restrict__ v_pool, const AttendOut o, const AttendWs ws, DeviceStatus* status) {
  extern __shared__ uint8_t dyn[];
  uint8_t* q_smem = dyn + ((1024u - (smem_u32(dyn) & 1023u)) & 1023u);
  uint8_t* ring = q_smem + 2 * kTileBytes;
  Shared* sh = reinterpret_cast<Shared*>(ring + (size_t)kStages * kTileBytes);
  const int warp = threadIdx.x >> 5, lane = threadIdx.x & 31;
  pdl_launch_dependents();
  if (warp == kTmaWarp && elect_one()) {
    prefetch_map(&q_map);
    prefetch_map(&k_map);
    prefetch_map(&v_map);
  }
  if (warp == kMmaWarp) {
    if (lane < kStages) {
      mbar_init(smem_u32(&sh->full[lane]), 1);
      mbar_init(smem_u32(&sh->empty[lane]), 1);
    }
    if (lane < 2) {
      mbar_init(smem_u32(&sh->s_full[lane]), 1);
      mbar_init(smem_u32(&sh->p_full[lane][0]), 4);
      mbar_init(smem_u32(&sh->p_full[lane][1]), 4);
      mbar_init(smem_u32(&sh->half_done[lane]), 1);
      mbar_init(smem_u32(&sh->o_full[lane]), 1);
      mbar_init(smem_u32(&sh->o_empty[lane]), 4);
    }
    if (lane == 0) {
      mbar_init(smem_u32(&sh->q_full), 1);
      mbar_init(smem_u32(&sh->q_empty), 1);
      sh->abort_flag = 0;
      sh->odd_values = 0;
    }
    fence_barrier_init();
    __syncwarp();
    tmem_alloc(smem_u32(&sh->tmem_base), 512);
    tmem_relinquish();
  }
  tc_fence_before();
  attend_share(g, as, &sh->share, ws.place, status);         // (synchronises)
  tc_fence_after();
  const uint32_t tmem = __shfl_sync(0xffffffffu, sh->tmem_base, 0);
  const BoundedWait pipe = {&sh->abort_flag, &status->code};
  auto wait = [&](uint64_t* bar, uint32_t parity, int where) { return bounded_wait(pipe, bar, parity, CC_ERR_TIMEOUT, where); };
  AttendWalk w;

  if (warp == kTmaWarp) {
    // ---------------------------------------------------------------- copies
    const int span = 1 << g.page_shift, copies = kTcTile >> g.page_shift;
    const uint32_t copy_bytes = (uint32_t)span * kHeadDim * 2;
    const uint32_t q_bytes = (uint32_t)(as.tile_tokens * g.group) * 128u;        // of one half of the channels of a tile
    const bool elected = elect_one();
    int stage = 0;
    uint32_t phase = 0, q_phase = 0;
    bool ok = true;
    for (bool more = w.first(g, as, &sh->share); more && ok; more = w.next(g, as, &sh->share)) {
      const int limit = w.limit;
      const int32_t* table = g.table + (int64_t)as.src[w.at.i] * g.table_stride;
      const int tok0 = w.at.b * as.block_tokens;
      const bool second = w.q.T - tok0 > as.tile_tokens;
      for (int t = w.t0; t < w.t1 && ok; ++t) {
        const int key = t * kTcTile + lane * span;             // first key of this lane's copy
        const bool mine = lane < copies && key < limit;
        int page = -1;
        if (mine) page = table[key >> g.page_shift];
        const bool good = mine && page >= 0 && page < g.pool_pages;
        if (mine && !good) report_error(status, CC_ERR_DEVICE_FLAG, 621);
        const unsigned mask = __ballot_sync(0xffffffffu, mine);
        const int group8 = copy_group(g, good, page, 0);
#pragma unroll 1
        for (int kv = 0; kv < 2; ++kv) {
          if (!wait(&sh->empty[stage], phase ^ 1, 81)) { ok = false; break; }
          const uint32_t fb = smem_u32(&sh->full[stage]);
          const uint32_t dst = smem_u32(ring) + (uint32_t)stage * kTileBytes;
          if (elected) mbar_expect_tx(fb, (uint32_t)__popc(mask) * copy_bytes);
          for (unsigned left = mask; left; left &= left - 1) {
            const int p = __ffs(left) - 1;
            const int at = __shfl_sync(0xffffffffu, group8, p);
            if (elected) tma_load_5d(dst + p * copy_bytes, kv ? &v_map : &k_map, fb, at, w.at.h);
          }
          if (++stage == kStages) { stage = 0; phase ^= 1; }
          if (kv == 0 && t == w.t0) {
            if (!wait(&sh->q_empty, q_phase ^ 1, 80)) { ok = false; break; }
            q_phase ^= 1;
            if (elected) {
              const uint32_t qb = smem_u32(&sh->q_full);
              mbar_expect_tx(qb, q_bytes * (second ? 4u : 2u));
              for (int i = 0; i < (second ? 2 : 1); ++i) {
                const int tok = w.q.row0 + tok0 + i * as.tile_tokens;
                const uint32_t at = smem_u32(q_smem) + (uint32_t)i * kTileBytes;
                tma_load_3d(at, &q_map, qb, 0, w.at.h * g.group, tok);
                tma_load_3d(at + kTileBytes / 2, &q_map, qb, 64, w.at.h * g.group, tok);
              }
            }
          }
        }
      }
    }
  } else if (warp == kMmaWarp) {
    // ---------------------------------------------------------------- products
    // Descriptor words: low = start >> 4 | leading offset, high = stride offset >> 4, version 1, 128-byte swizzle.  Q: groups of
    // eight rows 1 KB apart, the second half of the channels 16 KB on.  K and V: groups of eight keys 2 KB apart, the second half of
    // the channels 1 KB on (for V that is the leading offset, between 64 channels and the next 64).
    const uint32_t q_lo = ((smem_u32(q_smem) & 0x3FFFFu) >> 4) | (1u << 16), q_hi = (1024u >> 4) | (1u << 14) | (2u << 29);
    const uint32_t r_lo = ((smem_u32(ring) & 0x3FFFFu) >> 4), r_hi = (2048u >> 4) | (1u << 14) | (2u << 29);
    const uint32_t idesc_s = instr_desc(128, 128) | (g.scale < 0.f ? 1u << 13 : 0u);       // of a negative scale -Q is multiplied
    const uint32_t idesc_o = instr_desc(128, 128) | (1u << 16);                            // V: MN-major
    const bool elected = elect_one();
    int stage = 0;
    uint32_t phase = 0, q_phase = 0, p_phases = 0, o_phases = 3;         // (of the barriers of both tiles: a bit each)
    auto next_stage = [&] { if (++stage == kStages) { stage = 0; phase ^= 1; } };
    auto scores = [&](int i, uint32_t k_lo) {
#pragma unroll
      for (int ks = 0; ks < kHeadDim / 16; ++ks) {
        const uint32_t a = q_lo + (uint32_t)i * (kTileBytes >> 4) + (ks >= 4 ? (kTileBytes / 2) >> 4 : 0u) + (ks & 3) * 2u;
        const uint32_t b = k_lo + (1u << 16) + (ks >= 4 ? 1024u >> 4 : 0u) + (ks & 3) * 2u;
        umma(tmem + i * 128, a | ((uint64_t)q_hi << 32), b | ((uint64_t)r_hi << 32), idesc_s, ks > 0);
      }
      umma_commit(smem_u32(&sh->s_full[i]));
    };
    auto outputs = [&](int i, int half, uint32_t v_lo, bool accumulate) {
#pragma unroll
      for (int s4 = 0; s4 < kTcTile / 32; ++s4) {
        const int ks = half * (kTcTile / 32) + s4;
        const uint32_t b = v_lo + ((1024u >> 4) << 16) + ks * (4096u >> 4);
        umma_tmem_a(tmem + 256 + i * 128, tmem + i * 128 + ks * 8, b | ((uint64_t)r_hi << 32), idesc_o, accumulate || ks > 0);
      }
    };
    bool ok = true;
    for (bool more = w.first(g, as, &sh->share); more && ok; more = w.next(g, as, &sh->share)) {
      if (w.t0 == w.t1) continue;
      const int tiles = w.q.T - w.at.b * as.block_tokens > as.tile_tokens ? 2 : 1;
      ok = wait(&sh->full[stage], phase, 82) && wait(&sh->q_full, q_phase, 83);
      if (!ok) break;
      q_phase ^= 1;
      tc_fence_after();
      if (elected) {
        for (int i = 0; i < tiles; ++i) scores(i, r_lo + (uint32_t)stage * (kTileBytes >> 4));
        umma_commit(smem_u32(&sh->empty[stage]));
        if (w.t0 + 1 == w.t1) umma_commit(smem_u32(&sh->q_empty));
      }
      next_stage();
      for (int t = w.t0; t < w.t1 && ok; ++t) {
        const bool more_keys = t + 1 < w.t1;
        const int v_stage = stage;
        ok = wait(&sh->full[stage], phase, 84);
        next_stage();
        const int k_stage = stage;
        if (ok && more_keys) ok = wait(&sh->full[stage], phase, 87);         // (here, not between the products)
        const uint32_t v_lo = r_lo + (uint32_t)v_stage * (kTileBytes >> 4), k_lo = r_lo + (uint32_t)k_stage * (kTileBytes >> 4);
#pragma unroll
        for (int i = 0; i < 2; ++i) {
          if (i >= tiles) break;
          if (t == w.t0) {
            ok = ok && wait(&sh->o_empty[i], (o_phases >> i) & 1, 85);
            o_phases ^= 1u << i;
          }
          ok = ok && wait(&sh->p_full[i][0], (p_phases >> i) & 1, 86);
          if (!ok) break;
          tc_fence_after();
          if (elected) {
            outputs(i, 0, v_lo, t > w.t0);
            umma_commit(smem_u32(&sh->half_done[i]));
          }
          ok = wait(&sh->p_full[i][1], (p_phases >> i) & 1, 79);
          p_phases ^= 1u << i;
          if (!ok) break;
          tc_fence_after();
          if (elected) {
            outputs(i, 1, v_lo, true);
            if (i == tiles - 1) umma_commit(smem_u32(&sh->empty[v_stage]));
            if (more_keys) {
              scores(i, k_lo);
              if (i == tiles - 1) {
                umma_commit(smem_u32(&sh->empty[k_stage]));
                if (t + 2 == w.t1) umma_commit(smem_u32(&sh->q_empty));
              }
            } else {
              umma_commit(smem_u32(&sh->o_full[i]));
            }
          }
        }
        if (more_keys) next_stage();
      }
    }
  } else {
    // ---------------------------------------------------------------- softmax
    const int i = warp >> 2;                       // tile of the block
    const int r = (warp & 3) * 32 + lane;          // row of the tile = lane of tensor memory
    const uint32_t s_addr = tmem + i * 128 + ((uint32_t)((warp & 3) * 32) << 16), o_addr = s_addr + 256;
    const float c2 = fabsf(g.scale) * kLog2e;
    const uint64_t c22 = pack2(c2, c2);
    const int in_tile = r / g.group;
    uint32_t s_phase = 0, of_phase = 0;
    uint32_t entry = 1;                            // of V of the next tile in the order of the ring
    bool dead = false;
    for (bool more = w.first(g, as, &sh->share); more; more = w.next(g, as, &sh->share)) {
      const int tok = w.at.b * as.block_tokens + i * as.tile_tokens + in_tile;       // of the sequence
      if (w.q.T - w.at.b * as.block_tokens <= i * as.tile_tokens) {                    // no such tile
        entry += 2u * (uint32_t)(w.t1 - w.t0);
        continue;
      }
      const bool real = in_tile < as.tile_tokens && tok < w.q.T;
      const int lim = real ? (g.causal ? max(0, w.q.n - w.q.T + tok + 1) : w.q.n) : 0;     // keys that the row attends to
      const bool idle = !__any_sync(0xffffffffu, real);
      const int least = __reduce_min_sync(0xffffffffu, real ? lim : 0x7fffffff);
      const int shared = g.causal ? max(0, w.q.n - w.q.T + w.at.b * as.block_tokens + 1) : w.q.n;       // keys from here on: not by all rows
      const int plain = min(least, w.limit) / kTcTile;         // tiles before this one have no masked keys
      float ref = -INFINITY;
      uint64_t sum[2] = {0ull, 0ull};
      for (int t = w.t0; t < w.t1; ++t, entry += 2) {
        if (!dead) dead = !wait(&sh->s_full[i], s_phase, 88 + i);
        s_phase ^= 1;
        const int key0 = t * kTcTile;
        if (i == 0 && key0 + kTcTile > shared && !dead) {
          // Rows of V that no row of the block attends to may hold anything, and infinities of rows that only some attend to
          // would reach all (0 x inf): the products find zeros, and the latter count at the end.  (Both products with V come behind this
          // tile's P.)
          const int stage = entry % kStages;
          dead = !wait(&sh->full[stage], (entry / kStages) & 1, 90);
          for (int e = max(0, shared - key0) * 16 + (int)threadIdx.x; e < kTcTile * 16; e += 128) {
            uint4* at = reinterpret_cast<uint4*>(ring + (size_t)stage * kTileBytes + (e >> 7) * 2048 + ((e >> 3) & 1) * 1024 +
                                                 ((e >> 4) & 7) * 128 + (e & 7) * 16);
            if (key0 + (e >> 4) >= w.limit) {
              *at = make_uint4(0u, 0u, 0u, 0u);
            } else {
              uint4 x = *at;
              if (any_odd(x)) {
                x.x &= finite_halves(x.x);
                x.y &= finite_halves(x.y);
                x.z &= finite_halves(x.z);
                x.w &= finite_halves(x.w);
                *at = x;
                sh->odd_values = 1;
              }
            }
          }
          fence_proxy_async();
        }
        if (!dead) tc_fence_after();
        if (!dead && !idle) {
          const uint32_t p_bar = smem_u32(&sh->p_full[i][0]);
          int from = 0;                            // first chunk of 32 keys that is not handed over yet
          if (t < plain) {
            // With the reference that there is, in the first tile the maximum of its first 32 keys.
            uint32_t v0[32], v1[32], p0[16], p1[16];
            float reach = -INFINITY;
            uint64_t part[2] = {0ull, 0ull};
            tmem_ld32(s_addr, v0);
            tmem_ld32(s_addr + 32, v1);
            tmem_wait_ld();
            if (t == w.t0) ref = max32_nan(v0) * c2;
            const uint64_t off2 = offset_of(ref);
            exponentials<true>(v0, c22, off2, p0, part, reach);
            exponentials<true>(v1, c22, off2, p1, part, reach);
            if (!out_of_range(real, part, reach, c2, ref)) {
              tmem_st16(s_addr, p0);
              tmem_st16(s_addr + 16, p1);
              tmem_ld32(s_addr + 64, v0);
              tmem_ld32(s_addr + 96, v1);
              hand_over(p_bar, lane);
              from = 2;
              sum[0] = add2(sum[0], part[0]);
              sum[1] = add2(sum[1], part[1]);
              part[0] = part[1] = 0ull;
              reach = -INFINITY;
              tmem_wait_ld();
              exponentials<true>(v0, c22, off2, p0, part, reach);
              exponentials<true>(v1, c22, off2, p1, part, reach);
              if (!out_of_range(real, part, reach, c2, ref)) {
                tmem_st16(s_addr + 32, p0);
                tmem_st16(s_addr + 48, p1);
                hand_over(p_bar + 8, lane);
                from = 4;
                sum[0] = add2(sum[0], part[0]);
                sum[1] = add2(sum[1], part[1]);
              } else {
                dead = !wait(&sh->half_done[i], s_phase ^ 1, 92);        // the product of the first half with V is under way
                tc_fence_after();
              }
            }
          }
          if (from < 4) {
            // The maximum first: tiles with masked keys, logits far above the reference or no numbers, missing keys among the latter.
            const int last = t >= plain ? lim - key0 : kTcTile;
            if (t == w.t0 && from == 0) ref = -INFINITY;
            float high = -INFINITY;
            uint32_t v[32];
#pragma unroll 1
            for (int c = from; c < 4; ++c) {
              tmem_ld32(s_addr + c * 32, v);
              tmem_wait_ld();
              if (last < kTcTile) {
#pragma unroll
                for (int e = 0; e < 32; ++e)
                  if (c * 32 + e >= last) v[e] = 0xff800000u;
              }
              high = max3_nan(high, max32_nan(v), high);
            }
            if (__builtin_expect(__any_sync(0xffffffffu, real && high != high), 0))
              high = mask_missing(s_addr, from, last, missing_groups(as, g, w.at.i, key0, kTcTile / 8, w.limit), v);
            raise(high * c2, real, ref, sum, t > w.t0 || from > 0, o_addr);
            const uint64_t off2 = offset_of(ref);
            float reach = 0.f;
#pragma unroll 1
            for (int c = from; c < 4; ++c) {
              tmem_ld32(s_addr + c * 32, v);
              tmem_wait_ld();
              if (last < kTcTile) {
#pragma unroll
                for (int e = 0; e < 32; ++e)
                  if (c * 32 + e >= last) v[e] = 0xff800000u;
              }
              uint32_t p[16];
              exponentials<false>(v, c22, off2, p, sum, reach);
              tmem_st16(s_addr + c * 16, p);
              if (c & 1) hand_over(p_bar + (c >> 1) * 8, lane);
            }
          }
        } else {
          tc_fence_before();
          __syncwarp();
          if (lane < 2) mbar_arrive(smem_u32(&sh->p_full[i][lane]));
        }
      }

      // the rows' outputs
      if (w.t0 < w.t1) {
        if (!dead) dead = !wait(&sh->o_full[i], of_phase, 91);
        of_phase ^= 1;
        tc_fence_after();
      }
      const float total = total_of(sum);
      const bool whole = w.whole();
      bool none = lim <= 0;
      if (__builtin_expect(__any_sync(0xffffffffu, whole && !none && total == 0.f), 0)) {
        if (total == 0.f) none = attend_no_slot(as, g, w.at.i, lim);
        __syncwarp();
      }
      const int h = w.at.h * g.group + r - in_tile * g.group;
      const int64_t row = w.q.row0 + tok, at = (int64_t)w.slot() * as.rows + i * 128 + r;
      if (!dead && !idle) {
        const float inv = none ? 0.f : 1.0f / total;
        if (real && whole && o.lse) o.lse[row * g.hq + h] = none ? -INFINITY : (ref + log2f(total)) * kLn2;
        if (real && !whole) ws.stat[at] = make_float2(ref, total);
#pragma unroll 1
        for (int c = 0; c < 4; ++c) {
          uint32_t x[32];
          if (w.t0 < w.t1) {
            tmem_ld32(o_addr + c * 32, x);
            tmem_wait_ld();
          } else {
#pragma unroll
            for (int e = 0; e < 32; ++e) x[e] = 0u;
          }
          if (real && *(volatile int*)&sh->odd_values) {
            const int32_t* table = g.table + (int64_t)as.src[w.at.i] * g.table_stride;
#pragma unroll 1
            for (int key = max(shared, w.t0 * kTcTile); key < min(lim, w.t1 * kTcTile); ++key) {
              const int page = table[key >> g.page_shift];
              if (page < 0 || page >= g.pool_pages) continue;
              const uint32_t* v_row = reinterpret_cast<const uint32_t*>(
                  v_pool + (((int64_t)page << g.page_shift) + (key & ((1 << g.page_shift) - 1))) * g.kv_tok + (int64_t)w.at.h * g.kv_head) + c * 16;
#pragma unroll
              for (int e = 0; e < 16; ++e) {
                const uint32_t two = v_row[e], bad = two & ~finite_halves(two);
                x[2 * e] = __float_as_uint(__uint_as_float(x[2 * e]) + __uint_as_float(bad << 16));
                x[2 * e + 1] = __float_as_uint(__uint_as_float(x[2 * e + 1]) + __uint_as_float(bad & 0xffff0000u));
              }
            }
          }
          if (real && whole) {
            uint16_t* dst = o.out + row * g.out_tok + h * g.out_head + c * 32;
            uint32_t y[16];
#pragma unroll
            for (int e = 0; e < 16; ++e)
              y[e] = none ? 0u : pack_bf16(__uint_as_float(x[2 * e]) * inv, __uint_as_float(x[2 * e + 1]) * inv);
            if (o.wide) {
              store32(dst, y);
              store32(dst + 16, y + 8);
            } else {
#pragma unroll
              for (int e = 0; e < 4; ++e) reinterpret_cast<uint4*>(dst)[e] = make_uint4(y[4 * e], y[4 * e + 1], y[4 * e + 2], y[4 * e + 3]);
            }
          } else if (real) {
            float* dst = ws.out + at * kHeadDim + c * 32;
#pragma unroll
            for (int e = 0; e < 4; ++e) store32(dst + 8 * e, x + 8 * e);
          }
          __syncwarp();
        }
      }
      if (w.t0 < w.t1) {
        tc_fence_before();
        __syncwarp();
        if (lane == 0) mbar_arrive(smem_u32(&sh->o_empty[i]));
      }
    }
  }

  if (*(volatile int*)&sh->abort_flag) {
    // copies and products still in flight get time to land before shared and tensor memory are released
#pragma unroll 1
    for (int k = 0; k < 2000; ++k) __nanosleep(1000);
  }
  tc_fence_before();
  __syncthreads();
  if (warp == kMmaWarp) {
    tc_fence_after();
    tmem_dealloc(tmem, 512);
  }
}

}  // namespace

cudaError_t launch_attend_tc(const Launch& L, const CacheGeom& g, const AttendSeqs& as, const AttendWs& ws,
                             int grid, const AttendOut& o, const void* v, const CUtensorMap& q_map, const CUtensorMap& k_map,
                             const CUtensorMap& v_map) {
  const cudaError_t e = allow_smem(attend_tc_kernel);
  if (e != cudaSuccess) return e;
  return launch_pdl(attend_tc_kernel, dim3((unsigned)grid), dim3(kThreads), kSmem, L.stream, 1, g, as, q_map, k_map, v_map,
                    (const uint16_t*)v, o, ws, L.status);
}

}  // namespace cc
