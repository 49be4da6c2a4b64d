// The calls around the paged key/value cache on gfx950 (MI355X): argument checks, launchers and their C ABI.  The kernels live in
// the headers included here.  A translation unit of its own: these kernels are compiled with NaN honoured (a value that is not
// finite reaches the rows that see it, and no other), the prefill kernels without.
#include <hip/hip_runtime.h>

#include <algorithm>
#include <cmath>
#include <cstdarg>
#include <cstdint>
#include <cstdio>

#include "shareprefill.h"

#include "cache_accept_kernel.h"
#include "cache_attn_kernels.h"
#include "cache_common.h"
#include "cache_index.h"
#include "cache_plan_kernels.h"
#include "qk_norm_rope_kernel.h"

extern "C" __attribute__((visibility("hidden"))) void sp_set_error_text(const char *text);  // what sp_last_error returns

namespace {

sp_status fail(sp_status rc, const char *fmt, ...) {
  char text[512];
  va_list ap;
  va_start(ap, fmt);
  vsnprintf(text, sizeof(text), fmt, ap);
  va_end(ap);
  sp_set_error_text(text);
  return rc;
}

sp_status launched(const char *what) {
  const hipError_t e = hipGetLastError();
  return e == hipSuccess ? SP_OK : fail(SP_ERR_HIP, "%s launch: %s", what, hipGetErrorString(e));
}

sp_status need(const void *p, size_t align, const char *name) {
  if (!p) return fail(SP_ERR_INVALID_ARG, "%s is NULL", name);
  if ((uintptr_t)p % align) return fail(SP_ERR_INVALID_ARG, "%s is not %zu-byte aligned", name, align);
  return SP_OK;
}
sp_status may(const void *p, size_t align, const char *name) { return p ? need(p, align, name) : SP_OK; }

sp_status check_workspace(const void *ws, size_t have, size_t want) {
  if (want == 0) return SP_OK;
  if (!ws) return fail(SP_ERR_WORKSPACE, "workspace is NULL (%zu bytes needed)", want);
  if ((uintptr_t)ws % 256) return fail(SP_ERR_WORKSPACE, "workspace is not 256-byte aligned");
  if (have < want) return fail(SP_ERR_WORKSPACE, "workspace too small: %zu bytes given, %zu needed", have, want);
  return SP_OK;
}

// numbers that the kernels' 32-bit loops count up to
sp_status check_counts(int64_t n_requests, int64_t n_tokens) {
  if (n_requests < 0 || n_tokens < 0) return fail(SP_ERR_INVALID_ARG, "numbers of requests and tokens must not be negative");
  if (n_requests > (1 << 20) || n_tokens > (1 << 28))
    return fail(SP_ERR_UNSUPPORTED, "more than 2^20 requests or 2^28 tokens in a call");
  return SP_OK;
}

sp_status check_page(int32_t page) {
  if (page < CACHE_MIN_PAGE || page > CACHE_MAX_PAGE || (page & (page - 1)))
    return fail(SP_ERR_UNSUPPORTED, "page_size %d unsupported (a power of two from %d to %d)", page, CACHE_MIN_PAGE, CACHE_MAX_PAGE);
  return SP_OK;
}

// `name`: whose stride; a stride between rows that do not exist counts for nothing
sp_status check_stride(int64_t s, int64_t least, int64_t count, const char *name) {
  if (s < 0 || s % 8) return fail(SP_ERR_INVALID_ARG, "%s must be a non-negative multiple of 8 elements (got %lld)", name, (long long)s);
  if (count > 1 && s < least) return fail(SP_ERR_INVALID_ARG, "%s %lld is smaller than head_dim", name, (long long)s);
  return SP_OK;
}

sp_status check_heads_of(int32_t hq, int32_t hk, int32_t d) {
  if (hq <= 0 || hk <= 0) return fail(SP_ERR_INVALID_ARG, "head counts must be positive");
  if (hq % hk) return fail(SP_ERR_INVALID_ARG, "n_q_heads (%d) is not a multiple of n_kv_heads (%d)", hq, hk);
  if (d != 64 && d != 128) return fail(SP_ERR_UNSUPPORTED, "head_dim %d unsupported (64 or 128)", d);
  if (hq > 1024) return fail(SP_ERR_UNSUPPORTED, "n_q_heads %d exceeds 1024", hq);
  return SP_OK;
}

sp_status check_cache(const sp_cache_shape *c) {
  if (!c) return fail(SP_ERR_INVALID_ARG, "cache is NULL");
  sp_status rc;
  if (c->n_pages <= 0) return fail(SP_ERR_INVALID_ARG, "n_pages must be positive");
  if ((rc = check_page(c->page_size))) return rc;
  if ((rc = check_heads_of(c->n_kv_heads, c->n_kv_heads, c->head_dim))) return rc;
  if ((int64_t)c->n_pages * c->page_size > 0x7fffffff)
    return fail(SP_ERR_UNSUPPORTED, "%d pages of %d tokens: more slots than 32 bits number", c->n_pages, c->page_size);
  if ((rc = check_stride(c->stride_page, c->head_dim, c->n_pages, "cache stride_page")) ||
      (rc = check_stride(c->stride_token, c->head_dim, c->page_size, "cache stride_token")) ||
      (rc = check_stride(c->stride_head, c->head_dim, c->n_kv_heads, "cache stride_head")))
    return rc;
  if (c->stride_token > (1 << 24)) return fail(SP_ERR_UNSUPPORTED, "cache stride_token %lld exceeds 2^24 elements", (long long)c->stride_token);
  return SP_OK;
}

int log2_of(int32_t x) { return __builtin_ctz((unsigned)x); }

// ------------------------------------------------------------------------------------------------------------------ plan
size_t plan_bytes(int32_t n) { return ((size_t)2 * n + 1) * sizeof(int32_t); }

// ------------------------------------------------------------------------------------------------------------- attention
// Rows of a workgroup's tile, by the rows (group * max_new) that a request has under one KV head.  Up to 16 the narrow kernel: 64
// contexts of 8K with 4 rows 412 us and 414 in the wide one, 32 of 3000 with 8 rows 95 and 103, 16 of 500 with 4 16.8 and 18.4
// (one of 100K 99 and 97).  Two column groups to a wavefront, which read a key's fragment from LDS once for 32 rows instead of 16, from
// 193 rows on: below, shorter steps of more workgroups are faster (us, one group and two: 12 contexts of up to 6150 with 147 rows 42
// and 52, 8 of 4000 with 128 51 and 51 and with 192 70 and 83, 4 of 30000 with 147 84 and 118), above it turns (4 of 30000 with 224
// rows 195 and 178, one of 131000 with 512 388 and 330), though not for a lone short one: of 8000 with 224 rows 31 and 43, the price of a rule by
// the rows alone.
int attn_tile_rows(const sp_step_shape *s, const sp_cache_shape *c) {
  const int64_t rows = (int64_t)s->max_new * (s->n_q_heads / c->n_kv_heads);
  return rows <= 16 ? 16 : rows <= 192 ? 64 : 128;
}
int64_t attn_most_keys(const sp_step_shape *s, const sp_cache_shape *c) { return (int64_t)s->max_pages * c->page_size; }
int64_t attn_partial_rows(const sp_step_shape *s, const sp_cache_shape *c) {
  return c->n_kv_heads * cache_partial_rows(s->n_requests, s->n_tokens, s->n_q_heads / c->n_kv_heads, attn_most_keys(s, c), c->n_kv_heads);
}
int64_t attn_items(const sp_step_shape *s, const sp_cache_shape *c) {
  return c->n_kv_heads * cache_grid(s->n_requests, s->n_tokens, s->n_q_heads / c->n_kv_heads, attn_most_keys(s, c), attn_tile_rows(s, c), c->n_kv_heads);
}
size_t attn_bytes(const sp_step_shape *s, const sp_cache_shape *c) {
  return (size_t)attn_partial_rows(s, c) * (c->head_dim + 4) * sizeof(float);
}

sp_status check_step(const sp_step_shape *s, const sp_cache_shape *c) {
  if (!s) return fail(SP_ERR_INVALID_ARG, "shape is NULL");
  sp_status rc = check_cache(c);
  if (rc) return rc;
  if ((rc = check_counts(s->n_requests, s->n_tokens))) return rc;
  if (s->max_pages <= 0 || s->max_new <= 0) return fail(SP_ERR_INVALID_ARG, "max_pages / max_new must be positive");
  if ((rc = check_heads_of(s->n_q_heads, c->n_kv_heads, c->head_dim))) return rc;
  if (s->mask_words < 0 || s->mask_words > CACHE_MAX_WORDS)
    return fail(SP_ERR_UNSUPPORTED, "mask_words %d outside [0, %d]", s->mask_words, CACHE_MAX_WORDS);
  if (s->mask_words && s->max_new > 64 * s->mask_words)
    return fail(SP_ERR_INVALID_ARG, "max_new %d does not fit %d mask words", s->max_new, s->mask_words);
  if ((int64_t)s->max_pages * c->page_size > 0x7fffffff - CACHE_MAX_PAGE)
    return fail(SP_ERR_UNSUPPORTED, "%d pages of %d tokens: longer than 32 bits number", s->max_pages, c->page_size);
  if ((rc = check_stride(s->q_stride_t, c->head_dim, s->n_tokens, "q_stride_t")) ||
      (rc = check_stride(s->q_stride_h, c->head_dim, s->n_q_heads, "q_stride_h")) ||
      (rc = check_stride(s->o_stride_t, c->head_dim, s->n_tokens, "o_stride_t")) ||
      (rc = check_stride(s->o_stride_h, c->head_dim, s->n_q_heads, "o_stride_h")))
    return rc;
  if (!(s->softmax_scale >= 0.f) || std::isinf(s->softmax_scale))
    return fail(SP_ERR_INVALID_ARG, "softmax_scale must be finite and >= 0 (0 selects 1/sqrt(head_dim))");
  if (attn_items(s, c) > 0x7fffffff || attn_partial_rows(s, c) > 0x7fffffff || (int64_t)s->n_tokens * s->n_q_heads > 0x7fffffff)
    return fail(SP_ERR_UNSUPPORTED, "grid too large");
  return SP_OK;
}

// Workgroups of a launch: each goes on with the items gridDim further on, so that a table of long rows does not make a launch of
// workgroups that find nothing to do.
constexpr int64_t CA_GRID = 2048;

template <int D>
sp_status launch_cache_attn(const CacheAttnParams &p, int tile_rows, int64_t items, hipStream_t st) {
  const dim3 grid((unsigned)std::min(items, CA_GRID)), block(CA_THREADS);
  if (tile_rows == 16)
    hipLaunchKernelGGL((cache_attn_narrow_kernel<D>), grid, block, 0, st, p);
  else if (tile_rows == 64)
    hipLaunchKernelGGL((cache_attn_wide_kernel<D, 1>), grid, block, 0, st, p);
  else
    hipLaunchKernelGGL((cache_attn_wide_kernel<D, 2>), grid, block, 0, st, p);
  const sp_status rc = launched("cache_attn_kernel");
  if (rc || !cache_any_chunks(p.most_keys)) return rc;  // no request has two chunks
  const int64_t rows = (int64_t)p.n_tok * p.hq;
  hipLaunchKernelGGL((cache_join_kernel<D>), dim3((unsigned)std::min((rows + CA_WAVES - 1) / CA_WAVES, CA_GRID)), block, 0, st, p);
  return launched("cache_join_kernel");
}

}  // namespace

extern "C" {

sp_status sp_cache_plan_workspace_bytes(int32_t n_requests, size_t *bytes) {
  sp_set_error_text("");
  if (!bytes) return fail(SP_ERR_INVALID_ARG, "bytes is NULL");
  sp_status rc = check_counts(n_requests, 0);
  if (rc) return rc;
  *bytes = plan_bytes(n_requests);
  return SP_OK;
}

sp_status sp_cache_plan(int32_t n_requests, int32_t max_tokens, int32_t page_size, int32_t max_pages, const int32_t *ctx_len,
                        const int32_t *new_len, const int32_t *n_held, int32_t *block_table, const int32_t *free_pages,
                        int32_t free_capacity, const int32_t *n_free, const int32_t *parents, int32_t mask_words,
                        int32_t *n_held_out, int32_t *n_free_out, int32_t *tok_start, int32_t *seq_len, int32_t *positions,
                        int32_t *slots, int32_t *status, uint64_t *tree_mask, void *workspace, size_t workspace_bytes,
                        void *hip_stream) {
  sp_set_error_text("");
  sp_status rc;
  if ((rc = check_counts(n_requests, max_tokens))) return rc;
  if (max_pages <= 0 || free_capacity < 0)
    return fail(SP_ERR_INVALID_ARG, "free_capacity must not be negative, max_pages must be positive");
  if ((rc = check_page(page_size))) return rc;
  if ((int64_t)max_pages * page_size > 0x7fffffff - CACHE_MAX_PAGE)
    return fail(SP_ERR_UNSUPPORTED, "%d pages of %d tokens: longer than 32 bits number", max_pages, page_size);
  if (mask_words < 0 || mask_words > CACHE_MAX_WORDS)
    return fail(SP_ERR_UNSUPPORTED, "mask_words %d outside [0, %d]", mask_words, CACHE_MAX_WORDS);
  if ((mask_words > 0) != (tree_mask != nullptr) && max_tokens > 0)
    return fail(SP_ERR_INVALID_ARG, "tree_mask and mask_words go together");
  if ((rc = need(n_free, 4, "n_free")) || (rc = need(n_free_out, 4, "n_free_out")) || (rc = need(tok_start, 4, "tok_start"))) return rc;
  if (n_requests > 0 &&
      ((rc = need(ctx_len, 4, "ctx_len")) || (rc = need(new_len, 4, "new_len")) || (rc = need(n_held, 4, "n_held")) ||
       (rc = need(block_table, 4, "block_table")) || (rc = need(n_held_out, 4, "n_held_out")) ||
       (rc = need(seq_len, 4, "seq_len")) || (rc = need(status, 4, "status"))))
    return rc;
  if (free_capacity > 0 && (rc = need(free_pages, 4, "free_pages"))) return rc;
  if (max_tokens > 0 && ((rc = need(positions, 4, "positions")) || (rc = need(slots, 4, "slots")))) return rc;
  if ((rc = may(parents, 4, "parents")) || (rc = may(tree_mask, 8, "tree_mask"))) return rc;
  if (n_requests > 0 && (seq_len == ctx_len || seq_len == new_len))
    return fail(SP_ERR_INVALID_ARG, "seq_len must not be ctx_len's or new_len's memory");
  if ((rc = check_workspace(workspace, workspace_bytes, plan_bytes(n_requests)))) return rc;
  PlanParams p{};
  p.ctx = ctx_len, p.fresh = new_len, p.held = n_held, p.free_pages = free_pages, p.n_free = n_free, p.parents = parents;
  p.table = block_table, p.held_out = n_held_out, p.n_free_out = n_free_out, p.tok_start = tok_start, p.seq_len = seq_len;
  p.positions = positions, p.slots = slots, p.status = status, p.mask = tree_mask;
  p.old_held = (int32_t *)workspace, p.page_start = p.old_held + n_requests, p.free_count = p.page_start + n_requests;
  p.n = n_requests, p.max_tokens = max_tokens, p.page_shift = log2_of(page_size), p.width = max_pages, p.words = mask_words;
  p.free_capacity = free_capacity;
  hipStream_t st = (hipStream_t)hip_stream;
  const bool spread = n_requests <= PLAN_THREADS && n_held_out != n_held && n_free_out != n_free;
  const bool one = !spread && max_tokens <= PLAN_ONE_LAUNCH;
  const unsigned groups = spread ? (unsigned)std::max((max_tokens + PLAN_THREADS - 1) / PLAN_THREADS, 1) : 1;
  hipLaunchKernelGGL(plan_kernel, dim3(groups), dim3(PLAN_THREADS), 0, st, p, spread ? PLAN_THREADS : one ? PLAN_ONE_LAUNCH : 0);
  if ((rc = launched("plan_kernel")) || spread || one) return rc;
  hipLaunchKernelGGL(plan_tokens_kernel, dim3((unsigned)((max_tokens + PLAN_PART_THREADS - 1) / PLAN_PART_THREADS)), dim3(PLAN_PART_THREADS),
                     0, st, p);
  return launched("plan_tokens_kernel");
}

sp_status sp_qk_norm_rope(const sp_rope_shape *shape, const void *q, const void *k, const void *v, const void *q_weight,
                          const void *k_weight, const float *inv_freq, const int32_t *positions, void *q_out, void *k_out,
                          const sp_cache_shape *cache, void *k_cache, void *v_cache, const int32_t *slots, void *hip_stream) {
  sp_set_error_text("");
  if (!shape) return fail(SP_ERR_INVALID_ARG, "shape is NULL");
  const sp_rope_shape &s = *shape;
  sp_status rc;
  if ((rc = check_counts(0, s.n_tokens)) || (rc = check_heads_of(s.n_q_heads, s.n_kv_heads, s.head_dim))) return rc;
  if (s.rotary_dim < 0 || s.rotary_dim > s.head_dim || s.rotary_dim % 8)
    return fail(SP_ERR_INVALID_ARG, "rotary_dim %d is not a multiple of 8 in [0, head_dim]", s.rotary_dim);
  if (!(s.eps >= 0.f) || std::isinf(s.eps)) return fail(SP_ERR_INVALID_ARG, "eps must be finite and >= 0");
  const int64_t d = s.head_dim, n = s.n_tokens;
  if ((rc = check_stride(s.q_stride_t, d, n, "q_stride_t")) || (rc = check_stride(s.q_stride_h, d, s.n_q_heads, "q_stride_h")) ||
      (rc = check_stride(s.k_stride_t, d, n, "k_stride_t")) || (rc = check_stride(s.k_stride_h, d, s.n_kv_heads, "k_stride_h")) ||
      (rc = check_stride(s.qo_stride_t, d, n, "qo_stride_t")) || (rc = check_stride(s.qo_stride_h, d, s.n_q_heads, "qo_stride_h")))
    return rc;
  if (k_out && ((rc = check_stride(s.ko_stride_t, d, n, "ko_stride_t")) || (rc = check_stride(s.ko_stride_h, d, s.n_kv_heads, "ko_stride_h"))))
    return rc;
  if (cache) {
    if ((rc = check_cache(cache))) return rc;
    if (cache->head_dim != s.head_dim || cache->n_kv_heads != s.n_kv_heads)
      return fail(SP_ERR_INVALID_ARG, "the cache has %d heads of %d, the keys %d of %d", cache->n_kv_heads, cache->head_dim, s.n_kv_heads, s.head_dim);
    if ((rc = check_stride(s.v_stride_t, d, n, "v_stride_t")) || (rc = check_stride(s.v_stride_h, d, s.n_kv_heads, "v_stride_h"))) return rc;
  }
  if (!k_out && !cache) return fail(SP_ERR_INVALID_ARG, "k_out and cache are both NULL: the keys go nowhere");
  if (n == 0) return SP_OK;
  if ((rc = need(q, 16, "q")) || (rc = need(k, 16, "k")) || (rc = need(q_out, 16, "q_out")) || (rc = may(k_out, 16, "k_out")) ||
      (rc = may(q_weight, 16, "q_weight")) || (rc = may(k_weight, 16, "k_weight")))
    return rc;
  if (s.rotary_dim && ((rc = need(inv_freq, 4, "inv_freq")) || (rc = need(positions, 4, "positions")))) return rc;
  if (cache && ((rc = need(v, 16, "v")) || (rc = need(k_cache, 16, "k_cache")) || (rc = need(v_cache, 16, "v_cache")) || (rc = need(slots, 4, "slots"))))
    return rc;
  RopeParams p{};
  p.q = (const uint16_t *)q, p.k = (const uint16_t *)k, p.v = (const uint16_t *)v;
  p.qw = (const uint16_t *)q_weight, p.kw = (const uint16_t *)k_weight;
  p.inv_freq = inv_freq, p.positions = positions, p.slots = slots;
  p.q_out = (uint16_t *)q_out, p.k_out = (uint16_t *)k_out, p.k_cache = (uint16_t *)k_cache, p.v_cache = (uint16_t *)v_cache;
  p.q_st = s.q_stride_t, p.q_sh = s.q_stride_h, p.k_st = s.k_stride_t, p.k_sh = s.k_stride_h, p.v_st = s.v_stride_t, p.v_sh = s.v_stride_h;
  p.qo_st = s.qo_stride_t, p.qo_sh = s.qo_stride_h, p.ko_st = s.ko_stride_t, p.ko_sh = s.ko_stride_h;
  p.tokens = s.n_tokens, p.hq = s.n_q_heads, p.hk = s.n_kv_heads, p.rotary = s.rotary_dim, p.interleaved = s.interleaved != 0;
  p.eps = s.eps;
  if (cache) {
    p.c_sp = cache->stride_page, p.c_st = cache->stride_token, p.c_sh = cache->stride_head;
    p.page_shift = log2_of(cache->page_size), p.n_slots = (int64_t)cache->n_pages * cache->page_size;
  }
  hipStream_t st = (hipStream_t)hip_stream;
  // A workgroup takes as many rows at a time as its threads hold.  Where a token's are no multiple of that, long calls take four tokens
  // to a workgroup (us, one and four, 32768 tokens: 12 rows of 128 of 16 at a time 54 and 39, 36 145 and 130, but 48 173 and 174 and 80
  // 265 and 280; 2048 tokens of 48 rows of 64 9.1 and 10.0, 4096 14.6 and 13.6)
  const int rows_of = s.n_q_heads + s.n_kv_heads + (cache ? s.n_kv_heads : 0);
  const bool four = s.n_tokens >= 4096 && rows_of % (ROPE_THREADS / (s.head_dim / 8)) != 0;
  const bool whole = s.rotary_dim == s.head_dim;
  auto launch = [&](auto d, auto tokens) -> sp_status {
    constexpr int D = decltype(d)::value, TB = decltype(tokens)::value;
    static_assert(ROPE_LAUNCH % TB == 0 && (int64_t)ROPE_LAUNCH / TB * ROPE_THREADS < (1ll << 32), "a launch's threads");
    for (; p.first < p.tokens; p.first += ROPE_LAUNCH) {  // (2^28 + 2^22 at most)
      const dim3 grid((unsigned)((std::min(p.tokens - p.first, ROPE_LAUNCH) + TB - 1) / TB));
      if (whole)
        hipLaunchKernelGGL((qk_norm_rope_kernel<D, TB, true>), grid, dim3(ROPE_THREADS), 0, st, p);
      else
        hipLaunchKernelGGL((qk_norm_rope_kernel<D, TB, false>), grid, dim3(ROPE_THREADS), 0, st, p);
      if (const sp_status e = launched("qk_norm_rope_kernel")) return e;
    }
    return SP_OK;
  };
  constexpr std::integral_constant<int, 128> d128{};
  constexpr std::integral_constant<int, 64> d64{};
  constexpr std::integral_constant<int, 4> t4{};
  constexpr std::integral_constant<int, 1> t1{};
  if (s.head_dim == 128) return four ? launch(d128, t4) : launch(d128, t1);
  return four ? launch(d64, t4) : launch(d64, t1);
}

sp_status sp_cache_attn_workspace_bytes(const sp_step_shape *shape, const sp_cache_shape *cache, size_t *bytes) {
  sp_set_error_text("");
  if (!bytes) return fail(SP_ERR_INVALID_ARG, "bytes is NULL");
  sp_status rc = check_step(shape, cache);
  if (rc) return rc;
  *bytes = attn_bytes(shape, cache);
  return SP_OK;
}

sp_status sp_cache_attn(const sp_step_shape *shape, const sp_cache_shape *cache, const void *q, const void *k_cache,
                        const void *v_cache, const int32_t *block_table, const int32_t *seq_len, const int32_t *tok_start,
                        const uint64_t *tree_mask, void *o, float *lse, void *workspace, size_t workspace_bytes,
                        void *hip_stream) {
  sp_set_error_text("");
  sp_status rc = check_step(shape, cache);
  if (rc) return rc;
  const sp_step_shape &s = *shape;
  const sp_cache_shape &c = *cache;
  if (s.n_tokens == 0 || s.n_requests == 0) return SP_OK;
  if ((rc = need(q, 16, "q")) || (rc = need(k_cache, 16, "k_cache")) || (rc = need(v_cache, 16, "v_cache")) ||
      (rc = need(block_table, 4, "block_table")) || (rc = need(seq_len, 4, "seq_len")) || (rc = need(tok_start, 4, "tok_start")) ||
      (rc = need(o, 16, "o")) || (rc = may(lse, 4, "lse")))
    return rc;
  if (s.mask_words && (rc = need(tree_mask, 8, "tree_mask"))) return rc;
  if (!s.mask_words && tree_mask) return fail(SP_ERR_INVALID_ARG, "tree_mask and mask_words go together");
  if ((rc = check_workspace(workspace, workspace_bytes, attn_bytes(shape, cache)))) return rc;
  CacheAttnParams p{};
  p.q = (const uint16_t *)q, p.k = (const uint16_t *)k_cache, p.v = (const uint16_t *)v_cache, p.o = (uint16_t *)o, p.lse = lse;
  p.table = block_table, p.seq = seq_len, p.start = tok_start, p.mask = tree_mask;
  p.part_o = (float *)workspace, p.part_ml = p.part_o + (size_t)attn_partial_rows(shape, cache) * c.head_dim;
  p.q_st = s.q_stride_t, p.q_sh = s.q_stride_h, p.o_st = s.o_stride_t, p.o_sh = s.o_stride_h;
  p.c_sp = c.stride_page, p.c_st = c.stride_token, p.c_sh = c.stride_head;
  p.most_keys = (int)attn_most_keys(shape, cache);
  p.n_req = s.n_requests, p.n_tok = s.n_tokens, p.hq = s.n_q_heads, p.hk = c.n_kv_heads, p.group = s.n_q_heads / c.n_kv_heads;
  p.page_shift = log2_of(c.page_size), p.n_pages = c.n_pages, p.width = s.max_pages, p.words = s.mask_words, p.many_split = cache_many_split(c.n_kv_heads);
  const float scale = s.softmax_scale > 0.f ? s.softmax_scale : 1.0f / sqrtf((float)c.head_dim);
  p.c = scale * 1.4426950408889634f;
  const int rows = attn_tile_rows(shape, cache);
  const int64_t items = attn_items(shape, cache);
  hipStream_t st = (hipStream_t)hip_stream;
  return c.head_dim == 128 ? launch_cache_attn<128>(p, rows, items, st) : launch_cache_attn<64>(p, rows, items, st);
}

sp_status sp_cache_accept(const sp_cache_shape *cache, int32_t n_layers, int64_t stride_layer, void *k_cache, void *v_cache,
                          int32_t n_requests, int32_t max_pages, const int32_t *block_table, const int32_t *ctx_len,
                          const int32_t *seq_len, int32_t max_accept, const int32_t *path, const int32_t *n_accepted,
                          int32_t *ctx_out, void *hip_stream) {
  sp_set_error_text("");
  sp_status rc = check_cache(cache);
  if (rc) return rc;
  if ((rc = check_counts(n_requests, 0))) return rc;
  if (n_layers <= 0 || n_layers > 65535 || max_pages <= 0)
    return fail(SP_ERR_INVALID_ARG, "n_layers outside [1, 65535] or max_pages not positive");
  if (max_accept < 0 || max_accept > ACCEPT_MAX) return fail(SP_ERR_UNSUPPORTED, "max_accept %d outside [0, %d]", max_accept, ACCEPT_MAX);
  if ((rc = check_stride(stride_layer, cache->head_dim, n_layers, "stride_layer"))) return rc;
  if (n_requests == 0) return SP_OK;
  if ((rc = need(k_cache, 16, "k_cache")) || (rc = need(v_cache, 16, "v_cache")) || (rc = need(block_table, 4, "block_table")) ||
      (rc = need(ctx_len, 4, "ctx_len")) || (rc = need(seq_len, 4, "seq_len")) || (rc = need(n_accepted, 4, "n_accepted")) ||
      (rc = may(ctx_out, 4, "ctx_out")))
    return rc;
  if (max_accept > 0 && (rc = need(path, 4, "path"))) return rc;
  if (ctx_out && (ctx_out == ctx_len || ctx_out == seq_len || ctx_out == n_accepted || ctx_out == path || ctx_out == block_table))
    return fail(SP_ERR_INVALID_ARG, "ctx_out must be no other argument's memory");  // other workgroups of the request read those
  AcceptParams p{};
  p.k = (uint16_t *)k_cache, p.v = (uint16_t *)v_cache;
  p.table = block_table, p.ctx = ctx_len, p.seq = seq_len, p.path = path, p.count = n_accepted, p.ctx_out = ctx_out;
  p.c_sl = stride_layer, p.c_sp = cache->stride_page, p.c_st = cache->stride_token, p.c_sh = cache->stride_head;
  p.n_pages = cache->n_pages, p.page_shift = log2_of(cache->page_size), p.width = max_pages, p.max_accept = max_accept;
  p.hk = cache->n_kv_heads, p.d8 = cache->head_dim / 8;
  const unsigned pieces = (unsigned)((2 * p.hk * p.d8 + ACCEPT_THREADS - 1) / ACCEPT_THREADS);
  hipLaunchKernelGGL(cache_accept_kernel, dim3((unsigned)n_requests, (unsigned)n_layers, pieces), dim3(ACCEPT_THREADS), 0,
                     (hipStream_t)hip_stream, p);
  return launched("cache_accept_kernel");
}

}  // extern "C"
