// Launch stand-ins of the paged cache for the host-layer sanitizer build, beside
// launch_stubs.cpp: csrc/paged_api.cpp runs against these instead of the kernels.
// Each checks the arguments that the host layer built and returns
// hipErrorInvalidValue (SAF3R_ERR_HIP) when one is off. Nothing here touches a GPU.
#include <math.h>
#include <stdint.h>

#include "../../paper_2607_03612_amd/csrc/paged_internal.h"

namespace saf3r {
namespace {

hipError_t paged_status(bool ok) { return ok ? hipSuccess : hipErrorInvalidValue; }
bool page_ok(const PageDiv& p) {
  return p.size >= 16 && p.size <= kMaxPageSize && p.size % 16 == 0 && p.magic == page_div(p.size).magic;
}
int launches = 0;  // of the kind last asked for: 1 one launch or whole rows, 2 otherwise

}  // namespace

extern "C" int saf3r_stub_paged_launches() { return launches; }
extern "C" int32_t saf3r_stub_div_page(int32_t size, int32_t x) { return div_page(page_div(size), x); }

hipError_t launch_page_tables(const int32_t* lengths, const int32_t* new_tokens, int32_t* free_pages,
                              const int32_t* free_count, int32_t* table, int32_t* lengths_out, int32_t* count_out,
                              int32_t* start, int32_t* slots, RequestRecord* records, const StepArgs& a, hipStream_t) {
  const bool one = page_tables_in_one(a.requests, a.tokens, a.in_place != 0);
  launches = one ? 1 : 2;
  bool ok = lengths && new_tokens && free_pages && free_count && table && lengths_out && count_out && start &&
            (slots || a.tokens == 0) && (records || one) && page_ok(a.page) && a.requests >= 1 &&
            a.requests <= kMaxRequests && a.max_pages >= 1 && a.pages >= 1 && a.tokens >= 0 && a.tokens <= kMaxStepTokens &&
            (int64_t)a.max_pages * a.page.size <= kMaxRowTokens;
  // the workgroups of one launch read what the first one writes only if there is no other
  ok = ok && (!one || a.tokens <= kStepInPlaceTokens || (lengths != lengths_out && free_count != count_out));
  return paged_status(ok);
}

hipError_t launch_cache_append(int dtype, int dim, const void* k, const void* v, const int32_t* slots, void* k_pages,
                               void* v_pages, uint8_t* k_exp, uint8_t* v_exp, const AppendArgs& a, hipStream_t) {
  const bool eight = dtype == 2;
  return paged_status(dtype >= 0 && dtype <= 2 && (dim == 64 || dim == 128) && k && v && slots && k_pages && v_pages &&
                      (k_exp != nullptr) == eight && (v_exp != nullptr) == eight && page_ok(a.page) && a.tokens >= 1 &&
                      (int64_t)a.tokens * 32 < ((int64_t)1 << 32) && a.heads >= 1 && a.heads <= kMaxPagedHeads && a.slots >= a.page.size && a.slots % a.page.size == 0 &&
                      a.row_head % 16 == 0 && a.row_token % 16 == 0 && a.page_stride % 16 == 0 && a.head_stride % 16 == 0 &&
                      a.token_stride % 16 == 0 && a.page_stride >= 0 && a.row_head >= 0);
}

hipError_t launch_paged_attention(int dtype, int dim, const void* q, const void* k_pages, const void* v_pages,
                                  const uint8_t* k_exp, const uint8_t* v_exp, const int32_t* table, const int32_t* lengths,
                                  void* out, float*, void* workspace, const DecodeArgs& a, hipStream_t) {
  const bool eight = dtype == 2;
  const bool whole = whole_rows(dtype, dim, a);
  launches = whole ? 1 : 2;
  const int64_t grid = (int64_t)a.requests * a.kv_heads * a.qtiles;
  return paged_status(dtype >= 0 && dtype <= 2 && (dim == 64 || dim == 128) && q && k_pages && v_pages && table && lengths &&
                      out && (workspace || whole) && (k_exp != nullptr) == eight && (v_exp != nullptr) == eight &&
                      page_ok(a.page) && a.kv_heads >= 1 && a.group >= 1 && a.group * a.kv_heads == a.q_heads &&
                      a.q_heads <= kMaxPagedHeads && a.qtiles == (a.group + 15) / 16 && (!whole || grid * kRowThreads < ((int64_t)1 << 32)) &&
                      (int64_t)a.max_pages * a.page.size <= kMaxRowTokens && (int64_t)a.page.size * a.token_stride < (1 << 30) &&
                      a.scale_log2 > 0 && isfinite(a.scale_log2) && a.anchor >= 0 && a.window >= 0);
}

}  // namespace saf3r
