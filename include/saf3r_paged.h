/*
 * saf3r_paged.h -- the paged key-value cache: C ABI of libsaf3r.so beside
 * saf3r.h, for AMD Instinct MI355X (gfx950).
 *
 * saf3r.h attends over whole sequences that lie contiguous in memory. A stream
 * of frames or tokens, or many sequences of changing length, keeps K and V in
 * pages of a fixed number of tokens instead, and asks for the attention of one
 * new token of each sequence ("request") at a time:
 *
 *   saf3r_page_tables      one step's bookkeeping on the GPU: pages for the new
 *                          tokens, the slot of each, ended sequences' pages back
 *   saf3r_cache_append     K and V of the new tokens into their slots
 *   saf3r_paged_attention  softmax attention of one token per request over its
 *                          pages
 *
 * Conventions of saf3r.h hold: device pointers owned by the caller, valid for
 * the sizes stated and not aliasing one another unless said otherwise; host
 * structs read during the call only; every argument the host can see checked
 * before anything is launched, an error meaning that nothing was enqueued;
 * work enqueued on `stream`, on the current device, which must be the
 * pointers'; no allocation and no state between calls, so calls may be captured
 * into graphs and run at once on several streams when their outputs and
 * workspaces do not overlap. A workspace is overwritten and holds nothing
 * between calls; calls that share one must be ordered on the GPU.
 *
 * Strides count elements; a stride along a dimension of one entry is not looked at. Along
 * n entries it is at most 2^44 bytes, and n times it at most 2^60.
 *
 * What the GPU reads from lengths, tables and slots is bounded there: a bad
 * entry gives no access outside the arrays, as each call says.
 *
 * The cache: K pages and V pages, each [pages][kv_heads][page_size][head_dim]
 * addressed by the strides of a saf3r_page_layout, the same for both, with head_dim
 * contiguous; so token-major pages do as well. Slot s is token s % page_size of
 * page s / page_size. Element types:
 *   SAF3R_CACHE_F32   fp32, with fp32 tokens, queries and outputs;
 *   SAF3R_CACHE_BF16  bf16, with bf16 ones;
 *   SAF3R_CACHE_E4M3  8-bit OCP e4m3, with bf16 tokens, queries and outputs, and
 *                     one power of two per token and head: the value is
 *                     code * 2^(exp - 127), exp a uint8 of 1 .. 254 in
 *                     [pages][kv_heads][page_size] (contiguous, one array for K
 *                     and one for V);
 *   SAF3R_CACHE_E2M1  4-bit OCP e2m1, two codes a byte, the first in the low half, with
 *                     bf16 tokens, queries and outputs, and one power of two per 32
 *                     values of a row: exp of 2 .. 252 in
 *                     [pages][kv_heads][page_size][head_dim / 32] (contiguous). An
 *                     element of the pages is a byte: strides count those.
 */
#ifndef SAF3R_PAGED_H
#define SAF3R_PAGED_H

#include "saf3r.h"

#ifdef __cplusplus
extern "C" {
#endif

typedef enum {
  SAF3R_CACHE_F32 = 0,
  SAF3R_CACHE_BF16 = 1,
  SAF3R_CACHE_E4M3 = 2,
  SAF3R_CACHE_E2M1 = 4
} saf3r_cache_dtype;

typedef struct {
  int32_t pages;        /* >= 1; pages * page_size < 2^31 */
  int32_t page_size;    /* tokens, a multiple of 16, 16 .. 1024 */
  int32_t kv_heads;     /* 1 .. 256 */
  int32_t head_dim;     /* 64 or 128 */
  int32_t dtype;        /* saf3r_cache_dtype */
  int32_t reserved;     /* 0 */
  int64_t page_stride;  /* every stride >= 0 and a multiple of 16 bytes, */
  int64_t head_stride;  /*   page_size * token_stride under 2^30 bytes */
  int64_t token_stride;
} saf3r_page_layout;

/* One step's bookkeeping for a batch of requests. Request r holds lengths[r]
 * tokens in the first ceil(lengths[r] / page_size) entries of its table row, and
 * free_pages[0 .. *free_count) is the stack of the pages that nobody holds.
 * new_tokens[r] >= 0: that many tokens follow (0: nothing); < 0: the sequence
 * ends. In this order:
 *   1. ended sequences, in the order of r, push their pages on the stack, a row's
 *      first page first; their lengths become 0, their rows stay as they were;
 *   2. the others, in the order of r, take the pages that they lack for
 *      lengths[r] + new_tokens[r] tokens from the top of the stack, the first
 *      taken being the first that the row lacks.
 * A page taken or looked up that lies outside [0, pages) gives slots -1.
 * The new tokens of all requests lie one after another, in the order of r:
 * token_start[r] is where those of r start (token_start[requests]: their number;
 * no entry exceeds `tokens`), and slots[t] the cache slot of each, -1 for places
 * behind the last one.
 * A request is refused (its length and row stay, its tokens' slots are -1, it
 * takes no page) if the stack has too few pages left for it, if its length would
 * pass max_pages * page_size, or if its tokens do not end within `tokens`. A
 * length below 0 or above max_pages * page_size counts as refused whatever
 * new_tokens says. What the stack lacks for one request it also lacks for the
 * later ones that need a page. Pushes past `pages` entries are dropped.
 *   lengths, new_tokens       int32 [requests]
 *   free_pages                int32 [pages]: in, the stack; out, the pushed pages
 *                             behind its old top
 *   free_count                int32 [1]; read as 0 .. pages
 *   page_table                int32 [requests][max_pages]; only the entries of
 *                             the pages taken are written
 *   lengths_out               int32 [requests]; with in_place it may be `lengths`
 *   free_count_out            int32 [1]; with in_place it may be `free_count`
 *   token_start               int32 [requests + 1]
 *   slots                     int32 [tokens]
 *   workspace                 16-byte aligned, saf3r_page_tables_workspace_bytes;
 *                             may be NULL if these are 0 (up to 1024 requests,
 *                             with in_place up to 4096 tokens)
 * With separate outputs the call may be repeated: it reads nothing it writes
 * but the pages pushed. All pointers but the workspace 4-byte aligned.
 * Limits: requests 1 .. 65536, max_pages * page_size <= 2^29, tokens 0 .. 2^30. */
typedef struct {
  int32_t requests;
  int32_t page_size;  /* as in saf3r_page_layout */
  int32_t max_pages;  /* entries of a table row, >= 1 */
  int32_t pages;      /* entries of free_pages, >= 1 */
  int32_t tokens;     /* entries of slots */
  int32_t in_place;   /* 0 or 1 */
} saf3r_page_step;

/* Bytes of the workspace, or a negative saf3r_status. */
int64_t saf3r_page_tables_workspace_bytes(const saf3r_page_step* step);

saf3r_status saf3r_page_tables(const saf3r_page_step* step, const int32_t* lengths,
                               const int32_t* new_tokens, int32_t* free_pages,
                               const int32_t* free_count, int32_t* page_table,
                               int32_t* lengths_out, int32_t* free_count_out,
                               int32_t* token_start, int32_t* slots, void* workspace,
                               int64_t workspace_bytes, void* stream);

/* K and V of `tokens` new tokens into their slots. Token t's rows of head h start
 * at h * head_stride + t * token_stride elements of k and v (any strides >= 0
 * that are multiples of 16 bytes; head_dim contiguous). A slot outside
 * [0, pages * page_size) writes nothing. Slots must be distinct: of two tokens in one
 * slot either may be kept, and in an 8-bit cache parts of both. Every other
 * entry of the cache stays as it was.
 * E4M3: exp - 127 is the least e >= -126 with max|x| <= 448 * 2^e over the
 * row's finite x, and the codes are x / 2^e rounded to the nearest e4m3 (ties to
 * even); infinities and NaN become NaN.
 * E2M1: for each 32 values of a row exp - 127 is the least e of -125 .. 125 with
 * max|x| <= 6 * 2^e, and the codes are x / 2^e rounded to the nearest of 0, 1/2, 1, 3/2,
 * 2, 3, 4, 6 (ties to even codes, 6 past it), with their sign. 32 values with an infinity
 * or NaN among them become exp 255 and codes 7: NaN to saf3r_cache_read.
 *   k, v           [kv_heads][tokens][head_dim], fp32 for SAF3R_CACHE_F32 and bf16
 *                  otherwise, 16-byte aligned
 *   slots          int32 [tokens]
 *   k_pages, v_pages  16-byte aligned
 *   k_exp, v_exp   the exponents of an E4M3 cache (4-byte aligned) or an E2M1 one (16),
 *                  else NULL
 * tokens 0 .. 2^26; none is not an error. */
typedef struct {
  int32_t tokens;
  int32_t reserved; /* 0 */
  int64_t head_stride;
  int64_t token_stride;
} saf3r_token_layout;

saf3r_status saf3r_cache_append(const saf3r_page_layout* cache, const saf3r_token_layout* rows,
                                const void* k, const void* v, const int32_t* slots, void* k_pages,
                                void* v_pages, uint8_t* k_exp, uint8_t* v_exp, void* stream);

/* Attention of one query token per request over the request's cached tokens.
 * Query head h reads key-value head h / (q_heads / kv_heads); K and V are read once for
 * each 16 query heads that share them. For request r with
 * n = lengths[r] (read as 0 .. max_pages * page_size):
 *   z_j = scale * q . k_j   over the tokens j < n, with window > 0 only those with
 *                           j < anchor or j >= n - window
 *   out = sum_j softmax(z)_j v_j,  lse = log(sum_j exp(z_j))
 * anchor + window are the one-token forms of the anchor-frame and frame-local
 * classes (Sec. 4.1): the first tokens of a stream and its last ones. A token
 * whose page-table entry lies outside [0, pages) is left out like a masked one.
 * A request without a token gives a row of zeros and lse -inf; so does one
 * whose scores are all -inf. What lies in the cache behind a sequence's end or
 * outside its window does not reach the output, infinities and NaN included.
 * Infinite or NaN values among a request's own keys and values are undefined.
 * Scores of any size are taken, as fp32 holds them: scale * log2(e) * q . k has to be finite.
 * QK^T and PV run on the matrix cores with fp32 accumulation, softmax and sums in
 * fp32. fp32 caches: fp32 products. The others: exact bf16 operands,
 * the weights as two bf16 parts each (16 bits), so that the output's error is
 * its own rounding to bf16.
 * The keys of all requests are shared out evenly among the chip's workgroups,
 * whatever the lengths; the parts of a sequence that fell to several are joined
 * in a fixed order (same inputs, same bits). Where max_pages * page_size tokens of a
 * head's K and V are at most 384 KB (256 KB in 8 bits, in 4 2048 tokens), a workgroup takes each row whole
 * instead, in one launch: a table no wider than its sequences is faster for short ones.
 *   q, out          element (h, r, d) at h * head_stride + r * request_stride + d;
 *                   strides >= 0, multiples of 16 bytes; 16-byte aligned; the rows
 *                   of out distinct
 *   page_table      int32 [requests][max_pages]; read up to ceil(n / page_size)
 *   lengths         int32 [requests]
 *   k_exp, v_exp    of an E4M3 cache (4-byte aligned) or an E2M1 one (16), else NULL
 *   lse_or_null     NULL, or float32 [q_heads][requests]
 *   workspace       saf3r_paged_attention_workspace_bytes, 16-byte aligned; may be
 *                   NULL if these are 0
 * Limits: q_heads 1 .. 256 and a multiple of kv_heads, requests 1 .. 65536,
 * max_pages * page_size <= 2^29, anchor >= 0, window >= 0, scale > 0 and
 * scale * log2(e) finite in fp32. */
typedef struct {
  int32_t requests;
  int32_t q_heads;
  int32_t max_pages;
  int32_t anchor;
  int32_t window;
  float scale;
  int64_t q_head_stride;
  int64_t q_request_stride;
  int64_t out_head_stride;
  int64_t out_request_stride;
} saf3r_decode;

/* Bytes of the workspace, or a negative saf3r_status. */
int64_t saf3r_paged_attention_workspace_bytes(const saf3r_page_layout* cache, const saf3r_decode* step);

saf3r_status saf3r_paged_attention(const saf3r_page_layout* cache, const saf3r_decode* step,
                                   const void* q, const void* k_pages, const void* v_pages,
                                   const uint8_t* k_exp, const uint8_t* v_exp,
                                   const int32_t* page_table, const int32_t* lengths, void* out,
                                   float* lse_or_null, void* workspace, int64_t workspace_bytes,
                                   void* stream);

#ifdef __cplusplus
}
#endif

#endif /* SAF3R_PAGED_H */
