// Rotary positions of new tokens and the append of their keys and values to a paged cache, in one pass.
//
//   (x, y) -> scale * (x cos a - y sin a, x sin a + y cos a),  a = 2 pi * frac(p * turns_i)
//
// Angles.  turns_i = f_i / (2 pi) comes as a 64-bit fraction, so p * turns_i modulo 2^64 is the place on the circle
// exactly, wherever p lies; its upper 32 bits go to sincospi.  (In f32 an angle of 10^6 radians is off by 0.03.)
//
// A warp takes a token, or a part of its heads: eight lanes to a row of 256 bytes, two 16-byte chunks a lane, so that
// both sides of a pair are in one thread; the lanes of four rows share the work of the sines (two each) and keep all
// eight in registers for every head of the token.  Bound by HBM: every row is read once and written once (8132 tokens of 32 + 8 + 8
// heads, 200 MB: 35.1 us, 5.7 TB/s with the launch); few tokens by latency (64 tokens: 2.9 us from a graph).
#include <cuda_bf16.h>

#include "cache_step.cuh"

namespace cc {

namespace {

constexpr int kThreads = 128;
constexpr int kWarps = kThreads / 32;
// Rows in flight per lane and rows of a warp at most (half a token of 32 + 8 + 8 heads), 8 blocks per SM.  8132 tokens of 32 + 8 heads
// and 5003 of 28 + 4, us: four in flight, a token per warp, 256 threads (98 registers, 2 blocks) 38.3 and 23.6; 16 rows a warp and two in
// flight (64 registers) 35.7 and 19.5; blocks of 128 threads 35.2 and 18.6; 24 rows a warp 35.5 and 17.9, 48 rows 35.1 and 20.7.
// The first rows asked for before the sines: 38.8 and 18.5.
constexpr int kUnroll = 2;
constexpr int kWarpRows = 24;

struct RopePtrs {
  const uint16_t *q_new, *k_new, *v_new;
  const int32_t* positions;
  uint16_t *q, *k, *v;
};

__device__ __forceinline__ uint4 ld_once(const uint16_t* p) {
  uint4 v;
  asm volatile("ld.global.L1::no_allocate.v4.u32 {%0,%1,%2,%3}, [%4];"
               : "=r"(v.x), "=r"(v.y), "=r"(v.z), "=r"(v.w) : "l"(p) : "memory");
  return v;
}
__device__ __forceinline__ float lo_of(uint32_t w) { return __uint_as_float(w << 16); }
__device__ __forceinline__ float hi_of(uint32_t w) { return __uint_as_float(w & 0xffff0000u); }
__device__ __forceinline__ uint32_t two(float lo, float hi) {
  uint32_t r;
  asm("cvt.rn.bf16x2.f32 %0, %1, %2;" : "=r"(r) : "f"(hi), "f"(lo));
  return r;
}

// The rotation of two words that hold the first and the second channels of two pairs (halves), or of one word that
// holds a pair (interleaved).
__device__ __forceinline__ void rotate_halves(uint32_t& a, uint32_t& b, float c0, float s0, float c1, float s1) {
  const float x0 = lo_of(a), x1 = hi_of(a), y0 = lo_of(b), y1 = hi_of(b);
  a = two(fmaf(x0, c0, -(y0 * s0)), fmaf(x1, c1, -(y1 * s1)));
  b = two(fmaf(x0, s0, y0 * c0), fmaf(x1, s1, y1 * c1));
}
__device__ __forceinline__ void rotate_pair(uint32_t& a, float c, float s) {
  const float x = lo_of(a), y = hi_of(a);
  a = two(fmaf(x, c, -(y * s)), fmaf(x, s, y * c));
}

template <bool INTERLEAVED>
__global__ void __launch_bounds__(kThreads, 8)
rope_append_kernel(const __grid_constant__ CacheSeqs cs, const CacheGeom g, const __grid_constant__ RopeFreqs f,
                   const RopePtrs P, DeviceStatus* status) {
  __shared__ uint64_t turns[kHeadDim / 2];
  pdl_launch_dependents();
  if (threadIdx.x < kHeadDim / 2) turns[threadIdx.x] = f.turns[threadIdx.x];
  __syncthreads();
  const int lane = threadIdx.x & 31, sub = lane >> 3, l8 = lane & 7;
  const int tok = (int)blockIdx.x * kWarps + (threadIdx.x >> 5), part = blockIdx.y, parts = gridDim.y;
  pdl_wait();
  if (tok >= cs.new_off[cs.num_seqs]) return;

  const int s = seq_of_new(cs, tok);
  const int t = tok - cs.new_off[s], T = cs.new_off[s + 1] - cs.new_off[s];
  const int slot = cache_len(cs, g, s, status) - T + t;
  const int pos = P.positions ? P.positions[tok] : slot;
  const int nq = P.q_new ? g.hq : 0, nk = P.k_new ? g.hkv : 0;
  int64_t row = -1;                              // of the pool
  if (nk > 0) {
    int page = -1;
    if (slot >= 0) page = g.table[(int64_t)s * g.table_stride + (slot >> g.page_shift)];
    if (page >= 0 && page < g.pool_pages) row = ((int64_t)page << g.page_shift) + (slot & ((1 << g.page_shift) - 1));
    else report_error(status, CC_ERR_DEVICE_FLAG, 601);
  }

  // chunks of the row that this lane has; the first `turned` lanes hold the rotated channels
  const int turned = f.dims >> 4;
  const bool turns_mine = l8 < turned;
  const int c0 = turns_mine ? l8 : 2 * l8, c1 = turns_mine ? l8 + turned : 2 * l8 + 1;
  float cosv[8], sinv[8];
  {
    float cs2[2], sn2[2];
#pragma unroll
    for (int i = 0; i < 2; ++i) {
      const int e = 2 * sub + i;                 // the lane's pairs 2 sub and 2 sub + 1; all eight by exchange
      const int pair = INTERLEAVED ? (e < 4 ? 4 * l8 + e : 4 * (l8 + turned) + e - 4) : 8 * l8 + e;
      const uint64_t place = (uint64_t)(int64_t)pos * turns[turns_mine ? pair : 0];
      sincospif((float)(int32_t)(place >> 32) * (1.0f / 2147483648.0f), &sn2[i], &cs2[i]);
      cs2[i] *= f.scale;
      sn2[i] *= f.scale;
    }
#pragma unroll
    for (int e = 0; e < 8; ++e) {
      cosv[e] = __shfl_sync(0xffffffffu, cs2[e & 1], (e >> 1) * 8 + l8);
      sinv[e] = __shfl_sync(0xffffffffu, sn2[e & 1], (e >> 1) * 8 + l8);
    }
  }

  const int rows = nq + 2 * nk;                  // q heads, k heads, v heads
  const int per = (rows + 4 * parts - 1) / (4 * parts) * 4;
  const int end = min(rows, (part + 1) * per);
#pragma unroll 1
  for (int r0 = part * per + sub; r0 < end; r0 += 4 * kUnroll) {
    uint4 a[kUnroll], b[kUnroll];
    uint16_t* dst[kUnroll];
#pragma unroll
    for (int i = 0; i < kUnroll; ++i) {
      const int r = r0 + 4 * i;
      const uint16_t* src = nullptr;
      dst[i] = nullptr;
      if (r < end) {
        if (r < nq) {
          src = P.q_new + (int64_t)tok * g.qn_tok + (int64_t)r * g.qn_head;
          dst[i] = P.q + (int64_t)tok * g.q_tok + (int64_t)r * g.q_head;
        } else if (row >= 0) {
          const bool is_k = r < nq + nk;
          const int h = r - nq - (is_k ? 0 : nk);
          src = (is_k ? P.k_new : P.v_new) + (int64_t)tok * g.kvn_tok + (int64_t)h * g.kvn_head;
          dst[i] = (is_k ? P.k : P.v) + row * g.kv_tok + (int64_t)h * g.kv_head;
        }
      }
      if (dst[i]) {
        a[i] = ld_once(src + c0 * 8);
        b[i] = ld_once(src + c1 * 8);
      }
    }
#pragma unroll
    for (int i = 0; i < kUnroll; ++i) {
      if (!dst[i]) continue;
      if (turns_mine && r0 + 4 * i < nq + nk) {
        if (INTERLEAVED) {
          rotate_pair(a[i].x, cosv[0], sinv[0]);
          rotate_pair(a[i].y, cosv[1], sinv[1]);
          rotate_pair(a[i].z, cosv[2], sinv[2]);
          rotate_pair(a[i].w, cosv[3], sinv[3]);
          rotate_pair(b[i].x, cosv[4], sinv[4]);
          rotate_pair(b[i].y, cosv[5], sinv[5]);
          rotate_pair(b[i].z, cosv[6], sinv[6]);
          rotate_pair(b[i].w, cosv[7], sinv[7]);
        } else {
          rotate_halves(a[i].x, b[i].x, cosv[0], sinv[0], cosv[1], sinv[1]);
          rotate_halves(a[i].y, b[i].y, cosv[2], sinv[2], cosv[3], sinv[3]);
          rotate_halves(a[i].z, b[i].z, cosv[4], sinv[4], cosv[5], sinv[5]);
          rotate_halves(a[i].w, b[i].w, cosv[6], sinv[6], cosv[7], sinv[7]);
        }
      }
      *reinterpret_cast<uint4*>(dst[i] + c0 * 8) = a[i];
      *reinterpret_cast<uint4*>(dst[i] + c1 * 8) = b[i];
    }
  }
}

}  // namespace

cudaError_t launch_rope(const Launch& L, const CacheSeqs& cs, const CacheGeom& g, const RopeFreqs& f, const void* q_new,
                        const void* k_new, const void* v_new, const int32_t* positions, void* q, void* k, void* v) {
  const RopePtrs P = {(const uint16_t*)q_new, (const uint16_t*)k_new, (const uint16_t*)v_new, positions,
                      (uint16_t*)q, (uint16_t*)k, (uint16_t*)v};
  const int rows = (q_new ? g.hq : 0) + (k_new ? 2 * g.hkv : 0);
  const int64_t tokens = cs.new_off[cs.num_seqs];
  // Few tokens: the heads of a token are spread over more warps until every SM has sixteen.
  int parts = (rows + kWarpRows - 1) / kWarpRows;
  while (tokens * parts < (int64_t)L.sm_count * 16 && parts < (rows + 3) / 4) ++parts;
  const int64_t blocks = (tokens + kWarps - 1) / kWarps;
  auto kern = f.interleaved ? rope_append_kernel<true> : rope_append_kernel<false>;
  return launch_pdl(kern, dim3((unsigned)blocks, (unsigned)parts), dim3(kThreads), 0, L.stream, 1, cs, g, f, P, L.status);
}

}  // namespace cc
