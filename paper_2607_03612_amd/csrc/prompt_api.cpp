// C ABI of saf3r_prompt.h: host-side validation. Every check runs before any
// launch, so a call that returns an error has enqueued nothing.
#include "../../include/saf3r_prompt.h"
#include "paged_check.h"

namespace {

saf3r_status check_prompt(const saf3r_page_layout* cache, const saf3r_prompt* p, saf3r::PromptArgs* a) {
  Cache c;
  if (!p) return SAF3R_ERR_INVALID_ARGUMENT;
  // what a step of one token for each request has as well
  const saf3r_decode one{p->requests, p->q_heads, p->max_pages, p->anchor, p->window, p->scale, 0, 0, 0, 0};
  saf3r::DecodeArgs d{};
  saf3r_status st = check_decode(cache, &one, &c, &d);
  if (st == SAF3R_OK) st = check_cap(p->scale, p->cap, &a->cap_in, &a->cap_out);
  if (st != SAF3R_OK) return st;
  if (p->tokens < 0) return SAF3R_ERR_INVALID_ARGUMENT;
  if (p->tokens > saf3r::kMaxPromptTokens) return SAF3R_ERR_UNSUPPORTED;
  const int wide = cache->dtype == SAF3R_CACHE_F32 ? 4 : 2;
  const int64_t strides[4] = {p->q_head_stride, p->q_token_stride, p->out_head_stride, p->out_token_stride};
  int64_t* to[4] = {&a->q_head, &a->q_token, &a->out_head, &a->out_token};
  for (int i = 0; i < 4; ++i) {
    const int64_t n = i % 2 == 0 ? p->q_heads : p->tokens;
    const int64_t bytes = stride_bytes(strides[i], n, wide, far_limit(n));
    if (bytes < 0) return SAF3R_ERR_INVALID_ARGUMENT;
    *to[i] = bytes / wide;
  }
  a->requests = d.requests;
  a->tokens = p->tokens;
  a->q_heads = d.q_heads;
  a->kv_heads = d.kv_heads;
  a->group = d.group;
  a->max_pages = d.max_pages;
  a->pages = d.pages;
  // a row has no more tokens: what lies beyond says the same, and places stay in 32 bits
  const int32_t most = (int32_t)saf3r::kMaxRowTokens;
  a->anchor = p->anchor < most ? p->anchor : most;
  a->window = p->window < most ? p->window : most;
  a->scale_log2 = d.scale_log2;
  a->page = d.page;
  a->token_stride = d.token_stride;
  a->page_stride = d.page_stride;
  a->head_stride = d.head_stride;
  a->far_cap = p->cap > saf3r::kNearCap || !isfinite(a->cap_in * saf3r::kTwoLog2e);
  saf3r::plan_prompt(cache->dtype, cache->head_dim, a);
  return SAF3R_OK;
}

}  // namespace

extern "C" {

saf3r_status saf3r_cache_read(const saf3r_page_layout* cache, const saf3r_token_layout* rows,
                              const int32_t* slots, const void* k_pages, const void* v_pages,
                              const uint8_t* k_exp, const uint8_t* v_exp, void* k, void* v,
                              void* stream) {
  Cache c;
  saf3r::AppendArgs a{};
  const saf3r_status st = check_tokens(cache, rows, &c, &a);
  if (st != SAF3R_OK) return st;
  if (!k_pages || !v_pages || !aligned(k_pages, 16) || !aligned(v_pages, 16) || !exps_ok(cache->dtype, k_exp, v_exp))
    return SAF3R_ERR_INVALID_ARGUMENT;
  if ((cache->kv_heads > 1 && a.row_head == 0) || (rows->tokens > 1 && a.row_token == 0)) return SAF3R_ERR_INVALID_ARGUMENT;
  if (rows->tokens == 0) return SAF3R_OK;
  if (!k || !v || !slots || !aligned(k, 16) || !aligned(v, 16) || !aligned(slots, 4)) return SAF3R_ERR_INVALID_ARGUMENT;
  return hip_status(saf3r::launch_cache_read(cache->dtype, cache->head_dim, k, v, slots, k_pages, v_pages, k_exp, v_exp, a,
                                             static_cast<hipStream_t>(stream)));
}

saf3r_status saf3r_paged_attention_scored(const saf3r_page_layout* cache, const saf3r_decode* step,
                                          float cap, const float* slopes_or_null, const void* q,
                                          const void* k_pages, const void* v_pages,
                                          const uint8_t* k_exp, const uint8_t* v_exp,
                                          const int32_t* page_table, const int32_t* lengths, void* out,
                                          float* lse_or_null, void* workspace, int64_t workspace_bytes,
                                          void* stream) {
  return decode_call(cache, step, cap, slopes_or_null, q, k_pages, v_pages, k_exp, v_exp, page_table, lengths, out,
                     lse_or_null, workspace, workspace_bytes, stream);
}

int64_t saf3r_prompt_attention_workspace_bytes(const saf3r_page_layout* cache, const saf3r_prompt* step) {
  saf3r::PromptArgs a{};
  const saf3r_status st = check_prompt(cache, step, &a);
  if (st != SAF3R_OK) return st;
  return saf3r::prompt_workspace(cache->head_dim, a);
}

saf3r_status saf3r_prompt_attention(const saf3r_page_layout* cache, const saf3r_prompt* step,
                                    const float* slopes_or_null, const void* q, const void* k_pages,
                                    const void* v_pages, const uint8_t* k_exp, const uint8_t* v_exp,
                                    const int32_t* page_table, const int32_t* lengths,
                                    const int32_t* token_start, const int32_t* prefix_or_null, void* out,
                                    float* lse_or_null, void* workspace, int64_t workspace_bytes,
                                    void* stream) {
  saf3r::PromptArgs a{};
  const saf3r_status st = check_prompt(cache, step, &a);
  if (st != SAF3R_OK) return st;
  if (!k_pages || !v_pages || !aligned(k_pages, 16) || !aligned(v_pages, 16) || !exps_ok(cache->dtype, k_exp, v_exp))
    return SAF3R_ERR_INVALID_ARGUMENT;
  const int32_t* words[] = {page_table, lengths, token_start};
  for (const int32_t* p : words)
    if (!p || !aligned(p, 4)) return SAF3R_ERR_INVALID_ARGUMENT;
  const int64_t need = saf3r::prompt_workspace(cache->head_dim, a);
  if (!aligned(prefix_or_null, 4) || !aligned(slopes_or_null, 4) || !aligned(lse_or_null, 4) || workspace_bytes < 0 ||
      (need > 0 && !workspace) || !aligned(workspace, 16))
    return SAF3R_ERR_INVALID_ARGUMENT;
  if (workspace_bytes < need) return SAF3R_ERR_CAPACITY;
  if (step->tokens == 0) return SAF3R_OK;
  if (!q || !out || !aligned(q, 16) || !aligned(out, 16)) return SAF3R_ERR_INVALID_ARGUMENT;
  a.slopes = slopes_or_null;
  return hip_status(saf3r::launch_prompt_attention(cache->dtype, cache->head_dim, q, k_pages, v_pages, k_exp, v_exp, page_table,
                                                   lengths, token_start, prefix_or_null, out, lse_or_null, workspace, a,
                                                   static_cast<hipStream_t>(stream)));
}

}  // extern "C"
