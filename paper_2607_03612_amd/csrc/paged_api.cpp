// C ABI of the paged key-value cache (saf3r_paged.h): host-side validation.
// Every check runs before any launch, so a call that returns an error has
// enqueued nothing.
#include <math.h>
#include <stdint.h>

#include "../../include/saf3r_paged.h"
#include "paged_internal.h"

namespace {

bool aligned(const void* p, uintptr_t bytes) { return reinterpret_cast<uintptr_t>(p) % bytes == 0; }
saf3r_status hip_status(hipError_t e) { return e == hipSuccess ? SAF3R_OK : SAF3R_ERR_HIP; }

saf3r_status check_page_size(int32_t page_size) {
  if (page_size <= 0) return SAF3R_ERR_INVALID_ARGUMENT;
  if (page_size % saf3r::kPageQuantum != 0 || page_size > saf3r::kMaxPageSize) return SAF3R_ERR_UNSUPPORTED;
  return SAF3R_OK;
}

// A stride of `size`-byte elements along `n` entries as bytes, in [0, limit]; -1 if it
// is none. Along one entry it says nothing and is 0.
int64_t stride_bytes(int64_t stride, int64_t n, int size, int64_t limit) {
  if (n == 1) return 0;
  if (stride < 0 || stride > limit / size || stride * size % 16 != 0) return -1;
  return stride * size;
}
// Past what entries in one device's memory can be apart, and under 2^60 bytes to the
// last of them: sums of such products fit 63 bits.
int64_t far_limit(int64_t n) {
  const int64_t most = (int64_t)1 << 44, last = ((int64_t)1 << 60) / (n > 1 ? n : 1);
  return most < last ? most : last;
}

struct Cache {
  int size;  // bytes of a value
  int64_t page, head, token;  // strides in bytes
};

saf3r_status check_cache(const saf3r_page_layout* c, Cache* out) {
  if (!c || c->pages <= 0 || c->kv_heads <= 0) return SAF3R_ERR_INVALID_ARGUMENT;
  if (c->dtype < SAF3R_CACHE_F32 || c->dtype > SAF3R_CACHE_E4M3 || c->reserved != 0) return SAF3R_ERR_INVALID_ARGUMENT;
  const saf3r_status st = check_page_size(c->page_size);
  if (st != SAF3R_OK) return st;
  if (c->head_dim != 64 && c->head_dim != 128) return SAF3R_ERR_UNSUPPORTED;
  if (c->kv_heads > saf3r::kMaxPagedHeads) return SAF3R_ERR_UNSUPPORTED;
  if ((int64_t)c->pages * c->page_size > INT32_MAX) return SAF3R_ERR_UNSUPPORTED;
  out->size = c->dtype == SAF3R_CACHE_F32 ? 4 : c->dtype == SAF3R_CACHE_BF16 ? 2 : 1;
  out->page = stride_bytes(c->page_stride, c->pages, out->size, far_limit(c->pages));
  out->head = stride_bytes(c->head_stride, c->kv_heads, out->size, far_limit(c->kv_heads));
  out->token = stride_bytes(c->token_stride, c->page_size, out->size, (((int64_t)1 << 30) - 1) / c->page_size);
  if (out->page < 0 || out->head < 0 || out->token < 0) return SAF3R_ERR_INVALID_ARGUMENT;
  return SAF3R_OK;
}

saf3r_status check_step(const saf3r_page_step* p) {
  if (!p || p->requests <= 0 || p->max_pages <= 0 || p->pages <= 0 || p->tokens < 0 || p->in_place < 0 ||
      p->in_place > 1)
    return SAF3R_ERR_INVALID_ARGUMENT;
  const saf3r_status st = check_page_size(p->page_size);
  if (st != SAF3R_OK) return st;
  if (p->requests > saf3r::kMaxRequests || (int64_t)p->max_pages * p->page_size > saf3r::kMaxRowTokens ||
      (int64_t)p->pages * p->page_size > INT32_MAX || p->tokens > saf3r::kMaxStepTokens)
    return SAF3R_ERR_UNSUPPORTED;
  return SAF3R_OK;
}

saf3r_status check_decode(const saf3r_page_layout* cache, const saf3r_decode* d, Cache* c, saf3r::DecodeArgs* a) {
  saf3r_status st = check_cache(cache, c);
  if (st != SAF3R_OK) return st;
  if (!d || d->requests <= 0 || d->q_heads <= 0 || d->max_pages <= 0 || d->anchor < 0 || d->window < 0)
    return SAF3R_ERR_INVALID_ARGUMENT;
  const float scale_log2 = d->scale * 1.4426950408889634f;  // log2(e)
  if (!(d->scale > 0.0f) || !isfinite(scale_log2)) return SAF3R_ERR_INVALID_ARGUMENT;
  if (d->requests > saf3r::kMaxRequests || d->q_heads > saf3r::kMaxPagedHeads || d->q_heads % cache->kv_heads != 0 ||
      (int64_t)d->max_pages * cache->page_size > saf3r::kMaxRowTokens)
    return SAF3R_ERR_UNSUPPORTED;
  const int wide = cache->dtype == SAF3R_CACHE_F32 ? 4 : 2;
  const int64_t strides[4] = {d->q_head_stride, d->q_request_stride, d->out_head_stride, d->out_request_stride};
  int64_t* to[4] = {&a->q_head, &a->q_request, &a->out_head, &a->out_request};
  for (int i = 0; i < 4; ++i) {
    const int64_t n = i % 2 == 0 ? d->q_heads : d->requests;
    const int64_t bytes = stride_bytes(strides[i], n, wide, far_limit(n));
    if (bytes < 0) return SAF3R_ERR_INVALID_ARGUMENT;
    *to[i] = bytes / wide;
  }
  a->requests = d->requests;
  a->q_heads = d->q_heads;
  a->kv_heads = cache->kv_heads;
  a->group = d->q_heads / cache->kv_heads;
  a->qtiles = (a->group + 15) / 16;
  a->max_pages = d->max_pages;
  a->pages = cache->pages;
  a->anchor = d->anchor;
  a->window = d->window;
  a->scale_log2 = scale_log2;
  a->page = saf3r::page_div(cache->page_size);
  a->token_stride = (int32_t)c->token;
  a->page_stride = c->page;
  a->head_stride = c->head;
  return SAF3R_OK;
}

// The arrays of exponents: there for an 8-bit cache, absent for others.
bool exps_ok(int dtype, const uint8_t* k, const uint8_t* v) {
  if (dtype != SAF3R_CACHE_E4M3) return !k && !v;
  return k && v && aligned(k, 4) && aligned(v, 4);
}

}  // namespace

extern "C" {

int64_t saf3r_page_tables_workspace_bytes(const saf3r_page_step* step) {
  const saf3r_status st = check_step(step);
  if (st != SAF3R_OK) return st;
  if (saf3r::page_tables_in_one(step->requests, step->tokens, step->in_place != 0)) return 0;
  return (int64_t)step->requests * (int64_t)sizeof(saf3r::RequestRecord);
}

saf3r_status saf3r_page_tables(const saf3r_page_step* step, const int32_t* lengths,
                               const int32_t* new_tokens, int32_t* free_pages,
                               const int32_t* free_count, int32_t* page_table,
                               int32_t* lengths_out, int32_t* free_count_out,
                               int32_t* token_start, int32_t* slots, void* workspace,
                               int64_t workspace_bytes, void* stream) {
  const saf3r_status st = check_step(step);
  if (st != SAF3R_OK) return st;
  const void* words[] = {lengths, new_tokens, free_pages, free_count, page_table, lengths_out, free_count_out, token_start};
  for (const void* p : words)
    if (!p || !aligned(p, 4)) return SAF3R_ERR_INVALID_ARGUMENT;
  if (!step->in_place && (lengths_out == lengths || free_count_out == free_count)) return SAF3R_ERR_INVALID_ARGUMENT;
  const int64_t need = saf3r_page_tables_workspace_bytes(step);
  if ((step->tokens > 0 && !slots) || !aligned(slots, 4) || (need > 0 && !workspace) || !aligned(workspace, 16) ||
      workspace_bytes < 0)
    return SAF3R_ERR_INVALID_ARGUMENT;
  if (workspace_bytes < need) return SAF3R_ERR_CAPACITY;
  saf3r::StepArgs a{};
  a.requests = step->requests;
  a.max_pages = step->max_pages;
  a.pages = step->pages;
  a.tokens = step->tokens;
  a.in_place = step->in_place;
  a.page = saf3r::page_div(step->page_size);
  return hip_status(saf3r::launch_page_tables(lengths, new_tokens, free_pages, free_count, page_table, lengths_out,
                                              free_count_out, token_start, slots,
                                              static_cast<saf3r::RequestRecord*>(workspace), a,
                                              static_cast<hipStream_t>(stream)));
}

saf3r_status saf3r_cache_append(const saf3r_page_layout* cache, const saf3r_token_layout* rows,
                                const void* k, const void* v, const int32_t* slots, void* k_pages,
                                void* v_pages, uint8_t* k_exp, uint8_t* v_exp, void* stream) {
  Cache c;
  const saf3r_status st = check_cache(cache, &c);
  if (st != SAF3R_OK) return st;
  if (!rows || rows->tokens < 0 || rows->reserved != 0) return SAF3R_ERR_INVALID_ARGUMENT;
  if (rows->tokens > saf3r::kMaxAppendTokens) return SAF3R_ERR_UNSUPPORTED;
  const int wide = cache->dtype == SAF3R_CACHE_F32 ? 4 : 2;
  saf3r::AppendArgs a{};
  a.row_head = stride_bytes(rows->head_stride, cache->kv_heads, wide, far_limit(cache->kv_heads));
  a.row_token = stride_bytes(rows->token_stride, rows->tokens, wide, far_limit(rows->tokens));
  if (a.row_head < 0 || a.row_token < 0) return SAF3R_ERR_INVALID_ARGUMENT;
  if (!k_pages || !v_pages || !aligned(k_pages, 16) || !aligned(v_pages, 16) || !exps_ok(cache->dtype, k_exp, v_exp))
    return SAF3R_ERR_INVALID_ARGUMENT;
  if (rows->tokens == 0) return SAF3R_OK;
  if (!k || !v || !slots || !aligned(k, 16) || !aligned(v, 16) || !aligned(slots, 4)) return SAF3R_ERR_INVALID_ARGUMENT;
  a.tokens = rows->tokens;
  a.heads = cache->kv_heads;
  a.slots = cache->pages * cache->page_size;
  a.page = saf3r::page_div(cache->page_size);
  a.page_stride = c.page;
  a.head_stride = c.head;
  a.token_stride = c.token;
  return hip_status(saf3r::launch_cache_append(cache->dtype, cache->head_dim, k, v, slots, k_pages, v_pages, k_exp, v_exp,
                                               a, static_cast<hipStream_t>(stream)));
}

int64_t saf3r_paged_attention_workspace_bytes(const saf3r_page_layout* cache, const saf3r_decode* step) {
  Cache c;
  saf3r::DecodeArgs a{};
  const saf3r_status st = check_decode(cache, step, &c, &a);
  if (st != SAF3R_OK) return st;
  return saf3r::paged_attention_workspace(cache->dtype, cache->head_dim, a);
}

saf3r_status saf3r_paged_attention(const saf3r_page_layout* cache, const saf3r_decode* step,
                                   const void* q, const void* k_pages, const void* v_pages,
                                   const uint8_t* k_exp, const uint8_t* v_exp,
                                   const int32_t* page_table, const int32_t* lengths, void* out,
                                   float* lse_or_null, void* workspace, int64_t workspace_bytes,
                                   void* stream) {
  Cache c;
  saf3r::DecodeArgs a{};
  const saf3r_status st = check_decode(cache, step, &c, &a);
  if (st != SAF3R_OK) return st;
  const void* wide[] = {q, k_pages, v_pages, out};
  for (const void* p : wide)
    if (!p || !aligned(p, 16)) return SAF3R_ERR_INVALID_ARGUMENT;
  const int64_t need = saf3r::paged_attention_workspace(cache->dtype, cache->head_dim, a);
  if ((need > 0 && !workspace) || !aligned(workspace, 16)) return SAF3R_ERR_INVALID_ARGUMENT;
  if (!page_table || !lengths || !aligned(page_table, 4) || !aligned(lengths, 4) || !aligned(lse_or_null, 4) ||
      !exps_ok(cache->dtype, k_exp, v_exp) || workspace_bytes < 0)
    return SAF3R_ERR_INVALID_ARGUMENT;
  if (workspace_bytes < need) return SAF3R_ERR_CAPACITY;
  return hip_status(saf3r::launch_paged_attention(cache->dtype, cache->head_dim, q, k_pages, v_pages, k_exp, v_exp,
                                                  page_table, lengths, out, lse_or_null, workspace, a,
                                                  static_cast<hipStream_t>(stream)));
}

}  // extern "C"
