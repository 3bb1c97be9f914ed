// extern "C" entry points of the attention half of a layer: argument checks on
// the host, then launches on the caller's stream.
#include <math.h>
#include <stdint.h>

#include "spl.h"
#include "spl_attn.h"

namespace {

constexpr int64_t kMaxRows = (int64_t)1 << 31;       // tokens, requests, slots
constexpr int64_t kMaxElems = (int64_t)1 << 40;
constexpr int32_t kMaxHeads = 4096;

bool aligned(const void* p, uintptr_t a) { return (reinterpret_cast<uintptr_t>(p) & (a - 1)) == 0; }
bool given(const void* p, uintptr_t a) { return p && aligned(p, a); }
bool fp_dtype(int32_t d) { return d == SPL_F16 || d == SPL_BF16; }
bool page_ok(int32_t page) { return page >= 16 && page <= 256 && (page & (page - 1)) == 0; }
bool dim_ok(int32_t d) { return d == 64 || d == 96 || d == 128 || d == 256; }

// Whether any of the first `outs` arrays shares memory with another one.
struct Span {
  const void* at;
  int64_t ints;
};
bool overlap(const Span* a, int outs, int n) {
  for (int i = 0; i < outs; ++i)
    for (int j = i + 1; j < n; ++j) {
      const uintptr_t x = reinterpret_cast<uintptr_t>(a[i].at), y = reinterpret_cast<uintptr_t>(a[j].at);
      if (a[i].ints > 0 && a[j].ints > 0 && (x < y ? y - x < 4 * (uintptr_t)a[i].ints : x - y < 4 * (uintptr_t)a[j].ints))
        return true;
    }
  return false;
}

spl_status launched(hipError_t e) {
  if (e == hipSuccess) return SPL_OK;
  return e == hipErrorNotSupported ? SPL_ERR_UNSUPPORTED : SPL_ERR_DEVICE;
}

bool stride_ok(int64_t s) { return s >= 0 && s <= kMaxElems && s % 8 == 0; }
spl_status check_heads(const spl_heads* h, int64_t tokens) {
  if (!h || h->heads < 1 || h->heads > kMaxHeads || !stride_ok(h->token_stride) || !stride_ok(h->head_stride))
    return SPL_ERR_INVALID_ARG;
  return tokens == 0 || given(h->data, 16) ? SPL_OK : SPL_ERR_INVALID_ARG;
}

spl_status check_cache(const spl_kv_cache* c) {
  if (!c) return SPL_ERR_INVALID_ARG;
  if (!fp_dtype(c->dtype) || !dim_ok(c->head_dim) || !page_ok(c->page)) return SPL_ERR_UNSUPPORTED;
  if (c->heads < 1 || c->heads > kMaxHeads || c->pages < 1 || c->pages > kMaxRows / c->page - 1 || !given(c->data, 16))
    return SPL_ERR_INVALID_ARG;
  return c->data_bytes >= c->pages * c->heads * spl_kv_page_bytes(c->head_dim, c->page) ? SPL_OK : SPL_ERR_INVALID_ARG;
}

// What the norm and the rotation share, forward and backward.
spl_status check_turn(int64_t tokens, int32_t dim, int32_t dtype, const void* q_weight, const void* k_weight, float eps,
                      const int32_t* positions, const float* rope, int64_t rope_rows, int32_t rot) {
  if (tokens < 0 || tokens >= kMaxRows) return SPL_ERR_INVALID_ARG;
  if (!fp_dtype(dtype) || dim < 8 || dim > 256 || dim % 8 != 0) return SPL_ERR_UNSUPPORTED;
  if (rot < 0 || rot > dim || rot % 16 != 0) return SPL_ERR_UNSUPPORTED;
  if ((q_weight && !aligned(q_weight, 16)) || (k_weight && !aligned(k_weight, 16))) return SPL_ERR_INVALID_ARG;
  if (!(eps >= 0.0f) || !isfinite(eps)) return SPL_ERR_INVALID_ARG;
  if (rot > 0 && tokens > 0 &&
      (!given(positions, 4) || !given(rope, 4) || rope_rows < 1 || rope_rows > kMaxElems / rot))
    return SPL_ERR_INVALID_ARG;
  return SPL_OK;
}

// Launches count workgroups in 32 bits: a wave takes at least four heads.
bool rows_fit(int64_t tokens, int64_t heads, int32_t dim) {
  return tokens <= kMaxElems / (heads * dim) && tokens * (heads + 12) < kMaxRows;
}

}  // namespace

extern "C" {

int64_t spl_kv_page_bytes(int32_t head_dim, int32_t page) {
  return dim_ok(head_dim) && page_ok(page) ? spl::page_geom(head_dim, page).bytes : 0;
}

spl_status spl_block_tables(const int32_t* cached, const int32_t* fresh, int64_t requests, int64_t tokens,
                            int32_t page, int32_t* table, int64_t width, const int32_t* free_pages,
                            int64_t free_count, const int32_t* free_head, int32_t* row_start, int32_t* lens,
                            int32_t* positions, int32_t* slots, int32_t* state, hipStream_t stream) {
  if (requests < 1 || requests >= kMaxRows - 1024 || tokens < 0 || tokens >= kMaxRows || width < 1 ||
      width > kMaxElems / requests || free_count < 0 || free_count >= kMaxRows)
    return SPL_ERR_INVALID_ARG;
  if (!page_ok(page)) return SPL_ERR_UNSUPPORTED;
  if (!given(cached, 4) || !given(fresh, 4) || !given(table, 4) || !given(free_head, 4) || !given(row_start, 4) ||
      !given(lens, 4) || !given(state, 4) || (free_count > 0 && !given(free_pages, 4)) ||
      (tokens > 0 && (!given(positions, 4) || !given(slots, 4))))
    return SPL_ERR_INVALID_ARG;
  // a workgroup reads what another one may have written by then
  const Span arrays[] = {{table, requests * width}, {row_start, requests + 1}, {lens, requests}, {positions, tokens},
                         {slots, tokens},           {state, 2},                {cached, requests}, {fresh, requests},
                         {free_pages, free_count},  {free_head, 1}};
  if (overlap(arrays, 6, 10)) return SPL_ERR_INVALID_ARG;
  (void)hipGetLastError();
  return launched(spl::launch_block_tables(cached, fresh, requests, tokens, page, table, width, free_pages, free_count,
                                           free_head, row_start, lens, positions, slots, state, stream));
}

spl_status spl_qk_norm_rope(const spl_heads* q, const spl_heads* k, int64_t tokens, int32_t dim, int32_t dtype,
                            const void* q_weight, const void* k_weight, float eps, const int32_t* positions,
                            const float* rope, int64_t rope_rows, int32_t rot, int32_t interleaved, void* q_out,
                            void* k_out, hipStream_t stream) {
  spl_status st = check_turn(tokens, dim, dtype, q_weight, k_weight, eps, positions, rope, rope_rows, rot);
  if (st == SPL_OK) st = check_heads(q, tokens);
  if (st == SPL_OK) st = check_heads(k, tokens);
  if (st != SPL_OK) return st;
  if (tokens == 0) return SPL_OK;
  if (!given(q_out, 16) || !given(k_out, 16) || !rows_fit(tokens, (int64_t)q->heads + k->heads, dim))
    return SPL_ERR_INVALID_ARG;
  spl::NormRopeArgs a{};
  a.q = *q, a.k = *k, a.q_out = q_out, a.k_out = k_out, a.wq = q_weight, a.wk = k_weight, a.positions = positions;
  a.rope = rope, a.rope_rows = rope_rows, a.tokens = tokens, a.dim = dim, a.rot = rot;
  a.interleaved = interleaved ? 1 : 0, a.eps = eps;
  (void)hipGetLastError();
  return launched(spl::launch_norm_rope(a, dtype, stream));
}

spl_status spl_qk_norm_rope_append(const spl_heads* q, const spl_heads* k, const spl_heads* v, int64_t tokens,
                                   const void* q_weight, const void* k_weight, float eps, const int32_t* positions,
                                   const float* rope, int64_t rope_rows, int32_t rot, int32_t interleaved,
                                   const int32_t* slots, const spl_kv_cache* cache, void* q_out, void* k_out,
                                   hipStream_t stream) {
  spl_status st = check_cache(cache);
  if (st == SPL_OK)
    st = check_turn(tokens, cache->head_dim, cache->dtype, q_weight, k_weight, eps, positions, rope, rope_rows, rot);
  if (st == SPL_OK) st = check_heads(q, tokens);
  if (st == SPL_OK) st = check_heads(k, tokens);
  if (st == SPL_OK) st = check_heads(v, tokens);
  if (st != SPL_OK) return st;
  if (k->heads != cache->heads || v->heads != cache->heads) return SPL_ERR_INVALID_ARG;
  if (tokens == 0) return SPL_OK;
  if (!given(q_out, 16) || (k_out && !aligned(k_out, 16)) || !given(slots, 4) ||
      !rows_fit(tokens, (int64_t)q->heads + 2 * (int64_t)k->heads, cache->head_dim))
    return SPL_ERR_INVALID_ARG;
  spl::NormRopeArgs a{};
  a.q = *q, a.k = *k, a.v = *v, a.q_out = q_out, a.k_out = k_out, a.wq = q_weight, a.wk = k_weight;
  a.positions = positions, a.rope = rope, a.rope_rows = rope_rows, a.slots = slots, a.cache = *cache;
  a.tokens = tokens, a.dim = cache->head_dim, a.rot = rot, a.interleaved = interleaved ? 1 : 0, a.eps = eps;
  (void)hipGetLastError();
  return launched(spl::launch_norm_rope(a, cache->dtype, stream));
}

spl_status spl_cache_read(const spl_kv_cache* cache, const int32_t* slots, int64_t tokens, void* k, void* v,
                          hipStream_t stream) {
  const spl_status st = check_cache(cache);
  if (st != SPL_OK) return st;
  if (tokens < 0 || tokens >= kMaxRows) return SPL_ERR_INVALID_ARG;
  if (tokens == 0 || (!k && !v)) return SPL_OK;
  if (!given(slots, 4) || (k && !aligned(k, 16)) || (v && !aligned(v, 16)) ||
      tokens > kMaxElems / 8 / ((int64_t)cache->heads * cache->head_dim))
    return SPL_ERR_INVALID_ARG;
  if (spl::cache_read_threads(*cache, tokens) > spl::kMaxThreads - 255) return SPL_ERR_UNSUPPORTED;
  (void)hipGetLastError();
  return launched(spl::launch_cache_read(*cache, slots, tokens, k, v, stream));
}

int64_t spl_qk_norm_rope_grad_workspace_bytes(int64_t tokens, int32_t q_heads, int32_t k_heads, int32_t dim) {
  if (tokens < 0 || tokens >= kMaxRows || q_heads < 1 || q_heads > kMaxHeads || k_heads < 1 || k_heads > kMaxHeads ||
      dim < 8 || dim > 256 || dim % 8 != 0 || !rows_fit(tokens, (int64_t)q_heads + k_heads, dim))
    return -1;
  return tokens == 0 ? 0 : spl::norm_rope_grad_bytes(tokens, q_heads, k_heads, dim);
}

spl_status spl_qk_norm_rope_grad(const spl_heads* dq, const spl_heads* dk, const spl_heads* q, const spl_heads* k,
                                 int64_t tokens, int32_t dim, int32_t dtype, const void* q_weight,
                                 const void* k_weight, float eps, const int32_t* positions, const float* rope,
                                 int64_t rope_rows, int32_t rot, int32_t interleaved, void* dq_out, void* dk_out,
                                 float* dq_weight, float* dk_weight, void* workspace, hipStream_t stream) {
  spl_status st = check_turn(tokens, dim, dtype, q_weight, k_weight, eps, positions, rope, rope_rows, rot);
  if (st == SPL_OK) st = check_heads(dq, tokens);
  if (st == SPL_OK) st = check_heads(dk, tokens);
  if (st == SPL_OK) st = check_heads(q, q_weight ? tokens : 0);
  if (st == SPL_OK) st = check_heads(k, k_weight ? tokens : 0);
  if (st != SPL_OK) return st;
  if (dq->heads != q->heads || dk->heads != k->heads || (dq_weight && !q_weight) || (dk_weight && !k_weight) ||
      !aligned(dq_weight, 4) || !aligned(dk_weight, 4))
    return SPL_ERR_INVALID_ARG;
  (void)hipGetLastError();
  if (tokens == 0) {
    hipError_t e = hipSuccess;                                    // 2 dim 16-bit zeros are dim float zeros
    if (dq_weight) e = spl::launch_zero_fill(dq_weight, 2 * (int64_t)dim, stream);
    if (e == hipSuccess && dk_weight) e = spl::launch_zero_fill(dk_weight, 2 * (int64_t)dim, stream);
    return launched(e);
  }
  if (!given(dq_out, 16) || !given(dk_out, 16) || !given(workspace, 16) ||
      !rows_fit(tokens, (int64_t)q->heads + k->heads, dim))
    return SPL_ERR_INVALID_ARG;
  spl::NormRopeGradArgs a{};
  a.dq = *dq, a.dk = *dk, a.q = *q, a.k = *k, a.dq_out = dq_out, a.dk_out = dk_out, a.wq = q_weight, a.wk = k_weight;
  a.dwq = dq_weight, a.dwk = dk_weight, a.positions = positions, a.rope = rope, a.rope_rows = rope_rows;
  a.tokens = tokens, a.dim = dim, a.rot = rot, a.interleaved = interleaved ? 1 : 0, a.eps = eps;
  a.partial = static_cast<float*>(workspace);
  return launched(spl::launch_norm_rope_grad(a, dtype, stream));
}

static spl_status attn_sizes(const spl_kv_cache* cache, int64_t tokens, int32_t heads, int64_t requests, int64_t width,
                             int64_t max_new, int64_t max_len, spl::AttnArgs* a) {
  const spl_status st = check_cache(cache);
  if (st != SPL_OK) return st;
  if (tokens < 0 || tokens >= kMaxRows || heads < 1 || heads > kMaxHeads || heads % cache->heads != 0 || requests < 1 ||
      requests >= kMaxRows || width < 1 || width > kMaxElems / requests || width > (kMaxRows - 1) / cache->page ||
      max_new < 0 || max_new >= kMaxRows || max_len < 0 || max_len >= kMaxRows ||
      tokens > kMaxElems / ((int64_t)heads * cache->head_dim) || tokens * heads >= kMaxRows - requests)
    return SPL_ERR_INVALID_ARG;
  *a = spl::AttnArgs{};
  a->cache = *cache, a->tokens = tokens, a->requests = requests, a->width = width, a->max_new = max_new;
  a->max_len = max_len, a->q.heads = heads;
  return tokens == 0 || spl::attn_fits(*a) ? SPL_OK : SPL_ERR_UNSUPPORTED;
}

int64_t spl_attention_fp4_workspace_bytes(const spl_kv_cache* cache, int64_t tokens, int32_t heads, int64_t requests,
                                          int64_t width, int64_t max_new, int64_t max_len) {
  spl::AttnArgs a;
  if (attn_sizes(cache, tokens, heads, requests, width, max_new, max_len, &a) != SPL_OK) return -1;
  return tokens == 0 ? 0 : spl::attn_workspace_bytes(a);
}

spl_status spl_attention_fp4(const spl_heads* q, int64_t tokens, const spl_kv_cache* cache, const int32_t* table,
                             int64_t requests, int64_t width, const int32_t* lens, const int32_t* row_start,
                             int64_t max_new, int64_t max_len, float scale, int32_t window, void* out, float* lse,
                             void* workspace, hipStream_t stream) {
  spl_status st = check_heads(q, tokens);
  if (st != SPL_OK) return st;
  spl::AttnArgs a;
  st = attn_sizes(cache, tokens, q->heads, requests, width, max_new, max_len, &a);
  if (st != SPL_OK) return st;
  if (window < 0 || !isfinite(scale)) return SPL_ERR_INVALID_ARG;
  if (tokens == 0) return SPL_OK;
  if (!given(table, 4) || !given(lens, 4) || !given(row_start, 4) || !given(out, 16) || !aligned(lse, 4))
    return SPL_ERR_INVALID_ARG;
  if (spl::attn_workspace_bytes(a) > 0 && !given(workspace, 256)) return SPL_ERR_INVALID_ARG;
  a.q = *q, a.table = table, a.lens = lens, a.row_start = row_start, a.scale = scale, a.window = window;
  a.out = out, a.lse = lse, a.workspace = workspace;
  (void)hipGetLastError();
  return launched(spl::launch_attn(a, stream));
}

}  // extern "C"
