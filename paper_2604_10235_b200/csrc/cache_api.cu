// C-ABI layer of the calls on a paged cache after the compression: argument checks, launches.
#include <math.h>
#include <string.h>

#include "cache_step.cuh"
#include "cc_context.cuh"

namespace {

using namespace cc;

// The context's device is the current one while this lives.
struct DeviceScope {
  int back = -1;
  cudaError_t error = cudaSuccess;
  explicit DeviceScope(int device) {
    int now = device;
    error = cudaGetDevice(&now);
    if (error != cudaSuccess || now == device) return;
    error = cudaSetDevice(device);
    if (error == cudaSuccess) back = now;
  }
  ~DeviceScope() {
    if (back >= 0) cudaSetDevice(back);
  }
};

// What the calls on a cache have in common.
int take_desc(cc_ctx* ctx, const cc_cache_desc* d, CacheSeqs* cs, CacheGeom* g) {
  if (!ctx) return CC_ERR_INVALID_ARG;
  if (!d) return fail(ctx, CC_ERR_INVALID_ARG, "descriptor is NULL");
  if (d->n_heads_q <= 0 || d->n_heads_kv <= 0 || d->n_heads_q % d->n_heads_kv != 0)
    return fail(ctx, CC_ERR_INVALID_ARG, "n_heads_q must be a positive multiple of n_heads_kv");
  if (d->n_heads_q / d->n_heads_kv > 128 || d->n_heads_q > 65536)
    return fail(ctx, CC_ERR_UNSUPPORTED, "at most 128 query heads per KV head and 65536 in all");
  if (d->head_dim != kHeadDim) return fail(ctx, CC_ERR_UNSUPPORTED, "head_dim must be 128");
  if (d->dtype != CC_BF16) return fail(ctx, CC_ERR_UNSUPPORTED, "dtype must be CC_BF16");
  if (d->num_seqs < 1 || d->num_seqs > CC_MAX_SEQS)
    return fail(ctx, CC_ERR_UNSUPPORTED, "num_seqs must be in [1, %d]", CC_MAX_SEQS);
  const int ps = d->page_size;
  if (!(ps == 8 || ps == 16 || ps == 32 || ps == 64 || ps == 128))
    return fail(ctx, CC_ERR_UNSUPPORTED, "page_size must be 8, 16, 32, 64 or 128");
  if (d->pool_pages <= 0 || d->page_table_stride <= 0 || !d->page_table || !d->kv_lens)
    return fail(ctx, CC_ERR_INVALID_ARG, "page_table, its stride, pool_pages and kv_lens are needed");
  if (((int64_t)d->pool_pages * ps) >> 31) return fail(ctx, CC_ERR_UNSUPPORTED, "a pool of 2^31 rows or more");
  const int64_t strides[10] = {d->q_new_stride_tok, d->q_new_stride_head, d->kv_new_stride_tok, d->kv_new_stride_head,
                               d->q_stride_tok, d->q_stride_head, d->kv_stride_tok, d->kv_stride_head,
                               d->out_stride_tok, d->out_stride_head};
  for (int64_t x : strides) {
    if (x % 8) return fail(ctx, CC_ERR_UNSUPPORTED, "strides must be multiples of 8 elements (16 bytes)");
    if (x != 0 && x < kHeadDim) return fail(ctx, CC_ERR_INVALID_ARG, "strides smaller than head_dim");
    if (x > ((int64_t)1 << 32)) return fail(ctx, CC_ERR_UNSUPPORTED, "strides of more than 2^32 elements");
  }
  cs->num_seqs = d->num_seqs;
  int64_t tok = 0;
  for (int s = 0; s < d->num_seqs; ++s) {
    const int n = d->kv_lens[s], t = d->new_lens ? d->new_lens[s] : 1;
    if (n < 0 || t < 0) return fail(ctx, CC_ERR_INVALID_ARG, "negative length (sequence %d)", s);
    if (((int64_t)n + ps - 1) / ps > d->page_table_stride)
      return fail(ctx, CC_ERR_INVALID_ARG, "page_table_stride too small for sequence %d", s);
    cs->new_off[s] = (int)tok;
    cs->kv_len[s] = n;
    tok += t;
    if (n > 1 << 30 || tok > 1 << 30) return fail(ctx, CC_ERR_UNSUPPORTED, "more than 2^30 tokens");
  }
  for (int s = d->num_seqs; s <= CC_MAX_SEQS; ++s) cs->new_off[s] = (int)tok;
  for (int s = d->num_seqs; s < CC_MAX_SEQS; ++s) cs->kv_len[s] = 0;
  memset(g, 0, sizeof(*g));
  g->hq = d->n_heads_q;
  g->hkv = d->n_heads_kv;
  g->group = g->hq / g->hkv;
  while ((1 << g->page_shift) < ps) ++g->page_shift;
  g->pool_pages = d->pool_pages;
  g->table_stride = d->page_table_stride;
  g->table = d->page_table;
  g->dev_lens = d->dev_kv_lens;
  g->causal = d->causal != 0;
  const int64_t q_row = (int64_t)g->hq * kHeadDim, kv_row = (int64_t)g->hkv * kHeadDim;
  auto or_dense = [](int64_t x, int64_t dense) { return x ? x : dense; };
  g->qn_tok = or_dense(d->q_new_stride_tok, q_row);
  g->qn_head = or_dense(d->q_new_stride_head, kHeadDim);
  g->kvn_tok = or_dense(d->kv_new_stride_tok, kv_row);
  g->kvn_head = or_dense(d->kv_new_stride_head, kHeadDim);
  g->q_tok = or_dense(d->q_stride_tok, q_row);
  g->q_head = or_dense(d->q_stride_head, kHeadDim);
  g->kv_tok = or_dense(d->kv_stride_tok, kv_row);
  g->kv_head = or_dense(d->kv_stride_head, kHeadDim);
  g->out_tok = or_dense(d->out_stride_tok, q_row);
  g->out_head = or_dense(d->out_stride_head, kHeadDim);
  return CC_OK;
}

bool aligned(std::initializer_list<const void*> ps) {
  for (const void* p : ps)
    if ((uintptr_t)p % 16) return false;
  return true;
}

}  // namespace

extern "C" {

int cc_rope_freqs(const cc_rope_params* p, uint64_t* freqs) {
  if (!p || !freqs) return CC_ERR_INVALID_ARG;
  if (p->dims < 16 || p->dims > kHeadDim || p->dims % 16) return CC_ERR_UNSUPPORTED;
  if (p->kind < CC_ROPE_PLAIN || p->kind > CC_ROPE_GIVEN) return CC_ERR_INVALID_ARG;
  const bool given = p->kind == CC_ROPE_GIVEN;
  if (given ? !p->inv_freq : !(p->base > 1.0 && isfinite(p->base))) return CC_ERR_INVALID_ARG;
  if (!given && p->kind != CC_ROPE_PLAIN && !(p->factor >= 1.0 && isfinite(p->factor))) return CC_ERR_INVALID_ARG;
  if (p->kind == CC_ROPE_BANDS &&
      !(p->low > 0.0 && p->high > p->low && isfinite(p->high) && p->original > 0.0 && isfinite(p->original)))
    return CC_ERR_INVALID_ARG;
  const long double two_pi = 6.283185307179586476925286766559005768L;
  long double base = p->base;
  if (p->kind == CC_ROPE_BASE) base *= powl(p->factor, (long double)p->dims / (p->dims - 2));
  for (int i = 0; i < p->dims / 2; ++i) {
    long double f;
    if (given) {
      if (!(p->inv_freq[i] >= 0.0 && isfinite(p->inv_freq[i]))) return CC_ERR_INVALID_ARG;
      f = p->inv_freq[i];
    } else {
      f = powl(base, -2.0L * i / p->dims);
    }
    if (p->kind == CC_ROPE_LINEAR) f /= p->factor;
    if (p->kind == CC_ROPE_BANDS) {
      const long double turns = p->original * f / two_pi;
      long double share = (turns - p->low) / (p->high - p->low);
      share = share < 0 ? 0 : share > 1 ? 1 : share;
      f = (1 - share) * f / p->factor + share * f;
    }
    long double turn = fmodl(f / two_pi, 1.0L);
    const long double word = roundl(ldexpl(turn, 64));
    freqs[i] = word >= 18446744073709551616.0L ? 0 : (uint64_t)word;
  }
  return CC_OK;
}

int cc_rope_append(cc_ctx* ctx, const cc_cache_desc* desc, const void* q_new, const void* k_new, const void* v_new,
                   const int32_t* positions, void* q, void* k, void* v, void* stream) {
  CacheSeqs cs;
  CacheGeom g;
  const int rc = take_desc(ctx, desc, &cs, &g);
  if (rc != CC_OK) return rc;
  if (desc->rope_dims != 0 && (desc->rope_dims < 16 || desc->rope_dims > kHeadDim || desc->rope_dims % 16))
    return fail(ctx, CC_ERR_UNSUPPORTED, "rope_dims must be 0 or a multiple of 16 up to 128");
  if (desc->rope_dims != 0 && !desc->rope_freqs) return fail(ctx, CC_ERR_INVALID_ARG, "rope_freqs is NULL");
  if (!isfinite(desc->rope_scale)) return fail(ctx, CC_ERR_INVALID_ARG, "rope_scale must be finite");
  if (cs.new_off[cs.num_seqs] == 0 || (!q_new && !k_new)) return CC_OK;
  if ((q_new && !q) || (k_new && (!v_new || !k || !v))) return fail(ctx, CC_ERR_INVALID_ARG, "NULL tensor pointer");
  if (!aligned({q_new, k_new, v_new, q, k, v}))
    return fail(ctx, CC_ERR_INVALID_ARG, "tensor pointers must be 16-byte aligned");
  if (q_new == q && q_new && (g.qn_tok != g.q_tok || g.qn_head != g.q_head))
    return fail(ctx, CC_ERR_INVALID_ARG, "rotation in place needs equal strides of q_new and q");
  for (int s = 0; k_new && s < cs.num_seqs; ++s)
    if (cs.kv_len[s] < cs.new_off[s + 1] - cs.new_off[s])
      return fail(ctx, CC_ERR_INVALID_ARG, "sequence %d has fewer slots than new tokens", s);
  RopeFreqs f;
  memset(&f, 0, sizeof(f));
  f.dims = desc->rope_dims;
  f.interleaved = desc->rope_interleaved != 0;
  f.scale = desc->rope_scale != 0.f ? desc->rope_scale : 1.f;
  if (f.dims) memcpy(f.turns, desc->rope_freqs, f.dims / 2 * sizeof(uint64_t));
  const DeviceScope scope(ctx->device);
  if (scope.error != cudaSuccess) return cuda_fail(ctx, scope.error, "context's device");
  const cudaError_t e = launch_rope(make_launch(ctx, stream), cs, g, f, q_new, k_new, v_new, positions, q, k, v);
  if (e != cudaSuccess) return cuda_fail(ctx, e, "rope + append launch");
  return CC_OK;
}

size_t cc_attention_workspace_bytes(const cc_ctx* ctx, const cc_cache_desc* desc) {
  CacheSeqs cs;
  CacheGeom g;
  if (take_desc(const_cast<cc_ctx*>(ctx), desc, &cs, &g) != CC_OK) return 0;
  if (cs.new_off[cs.num_seqs] == 0) return 256;
  const size_t n = align256(attend_ws_bytes(cs, g, ctx->sm_count));
  if (n == 0) fail(const_cast<cc_ctx*>(ctx), CC_ERR_UNSUPPORTED, "2^31 tiles of work and more in one call");
  return n;
}

int cc_paged_attention(cc_ctx* ctx, const cc_cache_desc* desc, const void* q, const void* k, const void* v, void* out,
                       float* lse, void* ws, size_t ws_bytes, void* stream) {
  CacheSeqs cs;
  CacheGeom g;
  int rc = take_desc(ctx, desc, &cs, &g);
  if (rc != CC_OK) return rc;
  if (!isfinite(desc->scale)) return fail(ctx, CC_ERR_INVALID_ARG, "scale must be finite");
  g.scale = desc->scale != 0.f ? desc->scale : 0.08838834764831845f;
  if (cs.new_off[cs.num_seqs] == 0) return CC_OK;
  if (!q || !k || !v || !out) return fail(ctx, CC_ERR_INVALID_ARG, "NULL tensor pointer");
  if (!aligned({q, k, v, out})) return fail(ctx, CC_ERR_INVALID_ARG, "tensor pointers must be 16-byte aligned");
  const size_t need = attend_ws_bytes(cs, g, ctx->sm_count);
  if (need == 0) return fail(ctx, CC_ERR_UNSUPPORTED, "2^31 tiles of work and more in one call");
  if ((rc = check_ws(ctx, need, ws, ws_bytes)) != CC_OK) return rc;
  const DeviceScope scope(ctx->device);
  if (scope.error != cudaSuccess) return cuda_fail(ctx, scope.error, "context's device");
  int drv = 0;
  const cudaError_t e = launch_attend(make_launch(ctx, stream), cs, g, q, k, v, out, lse, ws, ctx->encode_tiled, &drv);
  if (drv != 0) return fail(ctx, CC_ERR_CUDA, "cuTensorMapEncodeTiled failed with code %d", drv);
  if (e != cudaSuccess) return cuda_fail(ctx, e, "paged attention launch");
  return CC_OK;
}

int cc_fork_pages(cc_ctx* ctx, const cc_cache_desc* desc, int32_t n_layers, void* const* k, void* const* v,
                  const int32_t* parents, int32_t n_children, int32_t* child_table, int32_t child_table_stride,
                  const int32_t* free_pages, void* stream) {
  CacheSeqs cs;
  CacheGeom g;
  const int rc = take_desc(ctx, desc, &cs, &g);
  if (rc != CC_OK) return rc;
  if (n_layers < 0 || n_children < 0) return fail(ctx, CC_ERR_INVALID_ARG, "negative count");
  if (n_children > CC_MAX_CHILDREN) return fail(ctx, CC_ERR_UNSUPPORTED, "more than %d children", CC_MAX_CHILDREN);
  if (n_children == 0 || n_layers == 0) return CC_OK;
  if (!k || !v || !parents || !child_table || !free_pages) return fail(ctx, CC_ERR_INVALID_ARG, "NULL pointer");
  for (int l = 0; l < n_layers; ++l) {
    if (!k[l] || !v[l]) return fail(ctx, CC_ERR_INVALID_ARG, "NULL tensor pointer");
    if (!aligned({k[l], v[l]})) return fail(ctx, CC_ERR_INVALID_ARG, "tensor pointers must be 16-byte aligned");
  }
  ForkArgs a;
  memset(&a, 0, sizeof(a));
  const uintptr_t row = (uintptr_t)g.table_stride * sizeof(int32_t);
  const uintptr_t lo = (uintptr_t)child_table, hi = lo + (uintptr_t)n_children * child_table_stride * sizeof(int32_t);
  for (int f = 0; f < n_children; ++f) {
    const int s = parents[f];
    if (s < 0 || s >= cs.num_seqs) return fail(ctx, CC_ERR_INVALID_ARG, "parent of child %d does not exist", f);
    const int pages = (cs.kv_len[s] + (1 << g.page_shift) - 1) >> g.page_shift;
    if (child_table_stride < pages || child_table_stride <= 0)
      return fail(ctx, CC_ERR_INVALID_ARG, "child_table_stride too small for child %d", f);
    const uintptr_t from = (uintptr_t)g.table + s * row, to = from + pages * sizeof(int32_t);
    if (from < hi && lo < to) return fail(ctx, CC_ERR_INVALID_ARG, "a child's row lies on the row of a parent");
    a.parent[f] = (uint8_t)s;
  }
  a.n_children = n_children;
  a.child_stride = child_table_stride;
  a.child_table = child_table;
  a.free_pages = free_pages;
  const DeviceScope scope(ctx->device);
  if (scope.error != cudaSuccess) return cuda_fail(ctx, scope.error, "context's device");
  for (int l0 = 0; l0 < n_layers; l0 += kForkLayers) {
    a.n_layers = n_layers - l0 < kForkLayers ? n_layers - l0 : kForkLayers;
    a.write_table = l0 == 0;
    for (int l = 0; l < a.n_layers; ++l) {
      a.k[l] = (uint16_t*)k[l0 + l];
      a.v[l] = (uint16_t*)v[l0 + l];
    }
    const cudaError_t e = launch_fork(make_launch(ctx, stream), cs, g, a);
    if (e != cudaSuccess) return cuda_fail(ctx, e, "fork launch");
  }
  return CC_OK;
}

}  // extern "C"
