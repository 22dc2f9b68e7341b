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
// A launch's threads in one dimension stay under 2^32: of append_kernel 32 a token,
// of paged_rows_kernel 256 a row.
constexpr int64_t kMaxAppendTokens = (int64_t)1 << 26;
constexpr int64_t kMaxWholeRows = (int64_t)1 << 23;

// x / page_size for 0 <= x < 2^31, as one high product and a shift: with d =
// page_size / 16, l = floor(log2 d) and m = ceil(2^(31 + l) / d) < 2^32 (2^31 where d is
// a power of two), m d is less than d above 2^(31 + l), and floor(x / 16) < 2^27 times
// that is below 2^27 * 2^(l + 1) < 2^(31 + l): never a whole quotient too many.
struct PageDiv {
  uint32_t magic;  // m
  int32_t shift;   // l
  int32_t size;
};
inline PageDiv page_div(int32_t page_size) {
  const uint32_t d = (uint32_t)page_size / kPageQuantum;
  int32_t l = 0;
  while (d >> (l + 1)) ++l;
  return PageDiv{(uint32_t)((((uint64_t)1 << (31 + l)) + d - 1) / d), l, page_size};
}
__host__ __device__ inline int32_t div_page(PageDiv p, int32_t x) {
  return (int32_t)((uint32_t)(((uint64_t)(((uint32_t)x >> 4) << 1) * p.magic) >> 32) >> p.shift);
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

// Steps of up to so many requests are one launch, without a workspace, of up to so many
// workgroups, a token a thread if that is enough. In place the workgroups would read
// what the first one writes, so there it is one, for steps of few tokens.
constexpr int kStepRequests = 1024;
constexpr int kStepGroups = 512;
constexpr int kStepInPlaceTokens = 4096;
inline bool page_tables_in_one(int32_t requests, int32_t tokens, bool in_place) {
  return requests <= kStepRequests && (!in_place || tokens <= kStepInPlaceTokens);
}
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

// Shared-out launches: 512 workgroups of four waves, two waves to a SIMD (with 1024, 8
// sequences of 2100 tokens over 8 heads 20.0 -> 25.3 us in fp32 of 64, 16.7 -> 19.9 in 8
// bits of 128; of 8192 55 -> 59 and 34 -> 39; 32 of 8192 190 -> 193 and 105 -> 105).
constexpr int kThreads = 256;
constexpr int kGroupWaves = kThreads / 64;
constexpr int kWorkgroups = 512;
constexpr int kWaves = kWorkgroups * kGroupWaves;  // a power of two
// Whole-row launches: four waves share a row. With eight, 27.5 -> 30.9 us for 2048 rows of
// 256 tokens in bf16 of 64, 34 -> 50 in 8 bits of 128; 4.3 and 4.3 for 8 rows of 256; 10.2
// -> 9.3 and 12.1 -> 11.7 for 128 rows of 1024.
constexpr int kRowThreads = 256;
constexpr int kRowWaves = kRowThreads / 64;

// Rows are not shared out where the longest that the table has room for (the
// lengths themselves are the GPU's) is this short, a CU's intake being 40 to 60 bytes
// a ns, less in 8 bits. us, whole rows / shared out, 8 rows of four query heads at 256,
// 384, 512 KB: bf16 of dimension 64 8.3 / 9.6, 10.9 / 9.7, 13.4 / 9.7; of dimension 128
// 7.9 / 10.3, 10.0 / 10.5, 12.2 / 10.5; fp32 8.9 / 11.4, 11.6 / 11.6, 14.3 / 11.4; 8
// bits of dimension 128 10.3 / 10.2, 13.3 / 10.3, 16.6 / 10.3. With more rows whole ones
// stay ahead: at 384 KB 11.6 / 16.4 for 128 rows, 74 / 78 for 1024 (bf16, 128), and in 8
// bits 15.8 / 17.9 and 76 / 81 above the limit; but the same table may hold one long
// sequence and short ones, which whole rows leave to one CU. Shared out takes a second
// launch, about 4 us of the host's time.
constexpr int64_t kWholeRowBytes = 384 << 10, kWholeRowBytes8 = 256 << 10;
inline bool whole_rows(int dtype, int dim, const DecodeArgs& a) {
  const int size = dtype == 0 ? 4 : dtype == 1 ? 2 : 1;
  return (int64_t)a.max_pages * a.page.size * dim * size * 2 <= (dtype == 2 ? kWholeRowBytes8 : kWholeRowBytes) &&
         (int64_t)a.requests * a.kv_heads * a.qtiles <= kMaxWholeRows;
}

// Query heads of a row, and the workspace: an int4 per workgroup, and two parts of a
// row each, of a float2 and dim sums per query head.
__host__ __device__ inline int piece_heads(const DecodeArgs& a) { return a.group < 16 ? a.group : 16; }
constexpr int64_t kCutBytes = (int64_t)kWorkgroups * sizeof(int4);
inline int64_t paged_attention_workspace(int dtype, int dim, const DecodeArgs& a) {
  if (whole_rows(dtype, dim, a)) return 0;
  return kCutBytes + (int64_t)2 * kWorkgroups * piece_heads(a) * (int64_t)(sizeof(float2) + dim * sizeof(float));
}

hipError_t launch_paged_attention(int dtype, int dim, const void* q, const void* k_pages,
                                  const void* v_pages, const uint8_t* k_exp, const uint8_t* v_exp,
                                  const int32_t* table, const int32_t* lengths, void* out, float* lse,
                                  void* workspace, const DecodeArgs& a, hipStream_t s);

}  // namespace saf3r
