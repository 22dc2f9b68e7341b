// Internal declarations of the paged key-value cache (saf3r_paged.h).
#pragma once

#include <hip/hip_runtime.h>
#include <stdint.h>

namespace saf3r {

constexpr int kPageQuantum = 16;       // a page holds a multiple of 16 tokens: a tile's 16 keys lie in one page
constexpr int kMaxPageSize = 1024;
constexpr int kMaxPagedHeads = 256;
constexpr int kMaxRequests = 65536;
constexpr int64_t kMaxRowTokens = (int64_t)1 << 29;  // of a request: max_pages * page_size
constexpr int64_t kMaxStepTokens = (int64_t)1 << 30;

// x / page_size for 0 <= x < 2^29 + kMaxPageSize, as one high product: with d =
// page_size / 16 <= 64 and m = ceil(2^31 / d), floor(x / 16) * (m d - 2^31) < 2^31.
struct PageDiv {
  uint32_t magic;  // ceil(2^31 / (page_size / 16)), at most 2^31
  int32_t size;
};
inline PageDiv page_div(int32_t page_size) {
  const uint32_t d = (uint32_t)page_size / kPageQuantum;
  return PageDiv{(uint32_t)((((uint64_t)1 << 31) + d - 1) / d), page_size};
}
__host__ __device__ inline int32_t div_page(PageDiv p, int32_t x) {
  return (int32_t)(((uint64_t)(((uint32_t)x >> 4) << 1) * p.magic) >> 32);
}

// ---------------------------------------------------------------- page tables

struct StepArgs {
  int32_t requests;
  int32_t max_pages;
  int32_t pages;
  int32_t tokens;
  int32_t in_place;
  PageDiv page;
};

// What the slot pass needs of a request.
struct RequestRecord {
  int32_t length;  // tokens before the step
  int32_t top;     // stack index of the first page it takes (the next ones lie below), -1 if refused
  int32_t held;    // pages before the step
};

// Whether a step is one launch, without a workspace.
bool page_tables_in_one(int32_t requests, int32_t tokens, bool in_place);
hipError_t launch_page_tables(const int32_t* lengths, const int32_t* new_tokens, int32_t* free_pages,
                              const int32_t* free_count, int32_t* table, int32_t* lengths_out,
                              int32_t* count_out, int32_t* start, int32_t* slots,
                              RequestRecord* records, const StepArgs& a, hipStream_t s);

// ---------------------------------------------------------------- append

// Strides in bytes.
struct AppendArgs {
  int32_t tokens;
  int32_t heads;
  int32_t slots;  // pages * page_size
  PageDiv page;
  int64_t row_head, row_token;                // of k and v
  int64_t page_stride, head_stride, token_stride;  // of the pages
};

hipError_t launch_cache_append(int dtype, int dim, const void* k, const void* v, const int32_t* slots,
                               void* k_pages, void* v_pages, uint8_t* k_exp, uint8_t* v_exp,
                               const AppendArgs& a, hipStream_t s);

// ---------------------------------------------------------------- attention

// Strides of the pages in bytes, of q and out in elements.
struct DecodeArgs {
  int32_t requests;
  int32_t q_heads, kv_heads;
  int32_t group;   // query heads of a key-value head
  int32_t qtiles;  // ceil(group / 16)
  int32_t max_pages;
  int32_t pages;
  int32_t anchor, window;
  float scale_log2;  // scale * log2(e)
  PageDiv page;
  int32_t token_stride;
  int64_t page_stride, head_stride;
  int64_t q_head, q_request, out_head, out_request;
};

hipError_t launch_paged_attention(int dtype, int dim, const void* q, const void* k_pages,
                                  const void* v_pages, const uint8_t* k_exp, const uint8_t* v_exp,
                                  const int32_t* table, const int32_t* lengths, void* out, float* lse,
                                  void* workspace, const DecodeArgs& a, hipStream_t s);
int64_t paged_attention_workspace(int dtype, int dim, const DecodeArgs& a);

}  // namespace saf3r
