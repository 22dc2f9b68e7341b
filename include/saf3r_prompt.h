/*
 * saf3r_prompt.h -- more over the paged key-value cache of saf3r_paged.h, whose
 * conventions hold:
 *
 *   saf3r_cache_read    the cached tokens of given slots as contiguous rows
 *   saf3r_paged_attention_scored  attention of one token per request whose scores are
 *                       capped or lowered by the distance of query and key
 *   saf3r_prompt_attention  attention of several new tokens per request over its pages:
 *                       a prompt, its next part, a frame, drafted tokens
 *
 * Changed scores: with z = scale * q . k of a query at place p of its sequence and the
 * key at place j,
 *   z' = cap * tanh(z / cap)    where cap > 0 (0: z' = z), then
 *   z" = z' - slopes[h] * |p - j|    where there are slopes, float32 [q_heads], 4-byte
 *                               aligned, in the GPU's memory; finite, of either sign
 * in fp32: off by a few roundings of the cap and of the bias. scale / cap must be a
 * normal fp32 number and cap * log2(e) finite; where a bias is not finite, outputs are
 * undefined.
 */
#ifndef SAF3R_PROMPT_H
#define SAF3R_PROMPT_H

#include "saf3r_paged.h"

#ifdef __cplusplus
extern "C" {
#endif

/* The way back of saf3r_cache_append: the values that the slots hold. Token t's rows of
 * head h go to h * head_stride + t * token_stride elements of k and v (strides > 0 along
 * more than one entry, multiples of 16 bytes, no two rows in one place, be they of k or v). A slot outside
 * [0, pages * page_size) gives zeros; slots may repeat. bf16 is exact for what an 8-bit
 * or 4-bit cache holds (from 2^-126 on; an E2M1 block of exponent 255 is NaN).
 *   slots          int32 [tokens]
 *   k_pages, v_pages, k_exp, v_exp  as in saf3r_cache_append
 *   k, v           [kv_heads][tokens][head_dim], fp32 for SAF3R_CACHE_F32 and bf16
 *                  otherwise, 16-byte aligned; written
 * tokens 0 .. 2^26; none is not an error. */
saf3r_status saf3r_cache_read(const saf3r_page_layout* cache, const saf3r_token_layout* rows,
                              const int32_t* slots, const void* k_pages, const void* v_pages,
                              const uint8_t* k_exp, const uint8_t* v_exp, void* k, void* v,
                              void* stream);

/* saf3r_paged_attention with changed scores, the query of request r being its last token
 * (p = lengths[r] - 1); softmax, lse and masks are those of the changed ones. The other
 * arguments and the workspace are saf3r_paged_attention's. */
saf3r_status saf3r_paged_attention_scored(const saf3r_page_layout* cache, const saf3r_decode* step,
                                          float cap, const float* slopes_or_null, const void* q,
                                          const void* k_pages, const void* v_pages,
                                          const uint8_t* k_exp, const uint8_t* v_exp,
                                          const int32_t* page_table, const int32_t* lengths, void* out,
                                          float* lse_or_null, void* workspace, int64_t workspace_bytes,
                                          void* stream);

/* Attention of the new tokens of a step over their requests' cached tokens, their own
 * among them (saf3r_page_tables and saf3r_cache_append come first). The new tokens of all
 * requests lie one after another, those of r from token_start[r] to token_start[r + 1];
 * they are the last ones of its lengths[r] tokens, so with c of them and
 * n = lengths[r] (read as 0 .. max_pages * page_size) the i-th is at place
 * p = n - c + i. It sees the keys j < n with
 *   j < prefix[r], or j <= p and (window = 0 or j < anchor or j > p - window).
 * prefix int32 [requests] or NULL (0 everywhere; below 0 counts as 0): its first tokens are
 * seen by all new ones, earlier ones among these too; with prefix[r] >= n the new tokens
 * see everything, like a frame's. Scores may be changed as above (cap 0 and no slopes: as
 * they are). Query head h reads key-value head h / (q_heads / kv_heads).
 *   out = sum_j softmax(z)_j v_j,  lse = log(sum_j exp(z_j)) over the keys seen
 * A token that sees none gives zeros and lse -inf: so one without a place, its request having
 * fewer tokens than new ones (p < 0), that no prefix shows any, and one whose scores are all -inf. Keys whose page-table entry
 * lies outside [0, pages) are left out like masked ones. Tokens before token_start[0] and
 * from token_start[requests] on belong to nobody: their rows stay as they were. A request
 * that saf3r_page_tables refused kept its length: its new tokens count as its last ones, and
 * their rows mean nothing. token_start is read as 0 .. tokens and has to ascend; of a
 * request whose end lies before its start there are no new tokens, and where starts go
 * back, the rows of out and lse mean nothing.
 * What lies in the cache behind a sequence's end does not reach the output, infinities and
 * NaN included; such values among a request's own keys and values are undefined, those of
 * a query reach its own row only.
 * Scores of any size are taken, as fp32 holds them: scale * log2(e) * q . k has to be finite.
 * fp32 caches: fp32 products. The others: exact bf16 operands with fp32 accumulation,
 * softmax and sums in fp32, the weights rounded to bf16 (2^-8) for the product with V.
 * Same inputs, same bits.
 *   q, out          element (h, t, d) at h * head_stride + t * token_stride + d;
 *                   strides >= 0, multiples of 16 bytes; 16-byte aligned; the rows of out
 *                   distinct
 *   page_table      int32 [requests][max_pages]; read up to ceil(n / page_size)
 *   lengths         int32 [requests]
 *   token_start     int32 [requests + 1]
 *   lse_or_null     NULL, or float32 [q_heads][tokens]
 *   workspace       saf3r_prompt_attention_workspace_bytes, 16-byte aligned; may be NULL
 *                   if these are 0
 * Limits: as saf3r_paged_attention's, and tokens 0 .. 2^22; none is not an error. */
typedef struct {
  int32_t requests;
  int32_t tokens; /* rows of q and out */
  int32_t q_heads;
  int32_t max_pages;
  int32_t anchor;
  int32_t window;
  float scale;
  float cap;
  int64_t q_head_stride;
  int64_t q_token_stride;
  int64_t out_head_stride;
  int64_t out_token_stride;
} saf3r_prompt;

/* Bytes of the workspace, or a negative saf3r_status. */
int64_t saf3r_prompt_attention_workspace_bytes(const saf3r_page_layout* cache, const saf3r_prompt* step);

saf3r_status saf3r_prompt_attention(const saf3r_page_layout* cache, const saf3r_prompt* step,
                                    const float* slopes_or_null, const void* q, const void* k_pages,
                                    const void* v_pages, const uint8_t* k_exp, const uint8_t* v_exp,
                                    const int32_t* page_table, const int32_t* lengths,
                                    const int32_t* token_start, const int32_t* prefix_or_null, void* out,
                                    float* lse_or_null, void* workspace, int64_t workspace_bytes,
                                    void* stream);

#ifdef __cplusplus
}
#endif

#endif /* SAF3R_PROMPT_H */
