// The paged cache's bookkeeping and its writes.
#include "paged_internal.h"

namespace saf3r {
namespace {

constexpr int kScanThreads = 1024;
constexpr int kScanWaves = kScanThreads / 64;
constexpr int kSlotThreads = 256;

// Sums stop at a limit of at most 2^30 + 1: a + b fits 32 bits, and the order
// of additions does not matter.
__device__ inline uint32_t add_to(uint32_t a, uint32_t b, uint32_t limit) { return min(a + b, limit); }

// Sums of the threads before this one; `total` gets the sum of all.
__device__ inline uint32_t scan(uint32_t x, uint32_t limit, uint32_t* waves, uint32_t& total) {
  const int lane = threadIdx.x & 63, wave = threadIdx.x >> 6;
#pragma unroll
  for (int d = 1; d < 64; d <<= 1) {
    const uint32_t y = __shfl_up(x, d);
    if (lane >= d) x = add_to(x, y, limit);
  }
  __syncthreads();  // the last scan's reads of `waves`
  if (lane == 63) waves[wave] = x;
  __syncthreads();
  uint32_t before = 0, all = 0;
#pragma unroll
  for (int w = 0; w < kScanWaves; ++w) {
    if (w == wave) before = all;
    all = add_to(all, waves[w], limit);
  }
  total = all;
  const uint32_t y = __shfl_up(x, 1);
  return lane == 0 ? before : add_to(before, y, limit);
}

// One workgroup: the order of the requests is the order of its threads, 1024
// requests a turn. Ended sequences' pages go on the stack first, since what they
// give back decides who fits; then the pages that the others need are summed.
__global__ __launch_bounds__(kScanThreads) void page_scan_kernel(
    const int32_t* lengths, const int32_t* __restrict__ new_tokens, int32_t* free_pages,
    const int32_t* free_count, const int32_t* table, int32_t* lengths_out, int32_t* count_out,
    int32_t* __restrict__ start_out, RequestRecord* __restrict__ records, StepArgs a) {
  __shared__ uint32_t waves[kScanWaves];
  const int lane = threadIdx.x & 63;
  const int32_t capacity = a.max_pages * a.page.size;
  const uint32_t token_limit = (uint32_t)a.tokens + 1, page_limit = (uint32_t)a.pages + 1;
  const uint32_t count = (uint32_t)min(max(*free_count, 0), a.pages);
  uint32_t tokens_before = 0, back_before = 0;
  for (int r0 = 0; r0 < a.requests; r0 += kScanThreads) {
    const int r = r0 + threadIdx.x;
    int32_t length = -1, fresh = 0;
    if (r < a.requests) {
      length = lengths[r];
      fresh = new_tokens[r];
    }
    const bool good = length >= 0 && length <= capacity;
    const bool ends = good && fresh < 0;
    const int32_t held = good ? div_page(a.page, length + a.page.size - 1) : 0;
    const uint32_t grow = min((uint32_t)max(fresh, 0), token_limit);
    uint32_t total;
    const uint32_t first = add_to(tokens_before, scan(grow, token_limit, waves, total), token_limit);
    tokens_before = add_to(tokens_before, total, token_limit);
    const uint32_t back = ends ? min((uint32_t)held, page_limit) : 0;
    const uint32_t back_first = add_to(back_before, scan(back, page_limit, waves, total), page_limit);
    back_before = add_to(back_before, total, page_limit);
    if (r < a.requests) {
      start_out[r] = (int32_t)min(first, (uint32_t)a.tokens);
      // top: provisional, whether the request may take pages at all
      records[r] = RequestRecord{(int32_t)min(first, (uint32_t)a.tokens), length,
                                 good && !ends && first + grow < token_limit ? 0 : -1, held};
    }
    // a wave copies its ended requests' rows one after another
    uint64_t todo = __ballot(back > 0);
    while (todo) {
      const int src = __ffsll((unsigned long long)todo) - 1;
      todo &= todo - 1;
      const int rr = r0 + (int)(threadIdx.x & ~63u) + src;
      const uint32_t n = __shfl(back, src);
      const uint32_t at = count + __shfl(back_first, src);  // a sum at its limit lies past the stack's end
      for (uint32_t j = lane; j < n; j += 64)
        if (at + j < (uint32_t)a.pages) free_pages[at + j] = table[(int64_t)rr * a.max_pages + j];
    }
  }
  if (threadIdx.x == 0) start_out[a.requests] = (int32_t)min(tokens_before, (uint32_t)a.tokens);
  const uint32_t top = min(count + back_before, (uint32_t)a.pages);
  uint32_t need_before = 0, taken = 0;
  for (int r0 = 0; r0 < a.requests; r0 += kScanThreads) {
    const int r = r0 + threadIdx.x;
    RequestRecord rec{0, -1, -1, 0};
    int32_t fresh = 0;
    if (r < a.requests) {
      rec = records[r];
      fresh = new_tokens[r];
    }
    const bool may = rec.top == 0 && fresh <= capacity - rec.length;
    const int32_t after = may ? rec.length + fresh : 0;
    const uint32_t need = may ? min((uint32_t)(div_page(a.page, after + a.page.size - 1) - rec.held), page_limit) : 0;
    uint32_t total;
    const uint32_t need_first = add_to(need_before, scan(need, page_limit, waves, total), page_limit);
    const uint32_t need_to = add_to(need_first, need, page_limit);
    need_before = add_to(need_before, total, page_limit);
    const bool fits = may && (need == 0 || need_to <= top);
    if (r < a.requests) {
      rec.top = !fits ? -1 : need == 0 ? 0 : (int32_t)(top - 1 - need_first);
      records[r].top = rec.top;
      const bool ends = fresh < 0 && rec.length >= 0 && rec.length <= capacity;
      lengths_out[r] = ends ? 0 : fits ? after : rec.length;
    }
    // the sums grow with r, so the pages taken are the last sum that fits
    uint32_t mine = fits && need > 0 ? need_to : 0;
#pragma unroll
    for (int d = 32; d >= 1; d >>= 1) mine = max(mine, (uint32_t)__shfl_xor((int)mine, d));
    __syncthreads();
    if (lane == 0) waves[threadIdx.x >> 6] = mine;
    __syncthreads();
#pragma unroll
    for (int w = 0; w < kScanWaves; ++w) taken = max(taken, waves[w]);
  }
  if (threadIdx.x == 0) *count_out = (int32_t)(top - taken);
}

// One thread per new token: its request by bisection of the starts, its slot,
// and, where it is a page's first token, the page's entry in the table.
__global__ __launch_bounds__(kSlotThreads) void page_slots_kernel(
    const int32_t* __restrict__ free_pages, int32_t* table, const int32_t* __restrict__ start,
    int32_t* __restrict__ slots, const RequestRecord* __restrict__ records, StepArgs a) {
  const int t = blockIdx.x * kSlotThreads + threadIdx.x;
  if (t >= a.tokens) return;
  int32_t slot = -1;
  if (t < start[a.requests]) {
    int lo = 0, hi = a.requests;  // the last request that starts at or before t
    while (hi - lo > 1) {
      const int mid = (lo + hi) >> 1;
      if (start[mid] <= t) lo = mid;
      else hi = mid;
    }
    const RequestRecord rec = records[lo];
    if (rec.top >= 0) {
      const int32_t pos = rec.length + (t - rec.start);
      const int32_t i = div_page(a.page, pos);
      const int32_t in = pos - i * a.page.size;
      int32_t* entry = table + (int64_t)lo * a.max_pages + i;
      int32_t page;
      if (i >= rec.held) {
        page = free_pages[rec.top - (i - rec.held)];
        if (in == 0) *entry = page;
      } else {
        page = *entry;
      }
      // a table or stack entry that is no page has no slots
      if (page >= 0 && page < a.pages) slot = page * a.page.size + in;
    }
  }
  slots[t] = slot;
}

// One row (token, head, K or V) to kDim * esz / 16 lanes of 16 bytes each; a
// workgroup's rows are consecutive tokens of one head, so that both the framework's
// [heads, N, dim] tokens and a page are read and written as long runs.
template <int kType, int kDim>
__global__ __launch_bounds__(256) void append_kernel(const char* __restrict__ k, const char* __restrict__ v,
                                                     const int32_t* __restrict__ slots, char* __restrict__ kp,
                                                     char* __restrict__ vp, uint8_t* __restrict__ ke,
                                                     uint8_t* __restrict__ ve, AppendArgs a) {
  constexpr int kIn = kType == 0 ? 4 : 2;
  constexpr int kLanes = kDim * kIn / 16;
  constexpr int kRows = 256 / kLanes;
  const int lane = threadIdx.x % kLanes;
  const int64_t t = (int64_t)blockIdx.x * kRows + threadIdx.x / kLanes;
  const int h = blockIdx.y;
  const bool value = blockIdx.z != 0;
  const int32_t slot = t < a.tokens ? slots[t] : -1;
  const bool keep = slot >= 0 && slot < a.slots;
  uint4 x{0, 0, 0, 0};
  if (keep) x = *reinterpret_cast<const uint4*>((value ? v : k) + h * a.row_head + t * a.row_token + lane * 16);
  const int32_t page = keep ? div_page(a.page, slot) : 0;
  const int32_t in = slot - page * a.page.size;
  char* to = (value ? vp : kp) + page * a.page_stride + h * a.head_stride + in * a.token_stride;
  if constexpr (kType != 2) {
    if (keep) *reinterpret_cast<uint4*>(to + lane * 16) = x;
  } else {
    const uint32_t w[4] = {x.x, x.y, x.z, x.w};
    uint32_t largest = 0;
#pragma unroll
    for (int i = 0; i < 4; ++i) {
      const uint32_t lo = (w[i] << 16) & 0x7fffffffu, hi = w[i] & 0x7fff0000u;
      largest = max(largest, lo < 0x7f800000u ? lo : 0u);
      largest = max(largest, hi < 0x7f800000u ? hi : 0u);
    }
#pragma unroll
    for (int d = kLanes / 2; d >= 1; d >>= 1) largest = max(largest, (uint32_t)__shfl_xor((int)largest, d));
    // 448 = 1.75 * 2^8: the carry out of the mantissa is there from 1.75 on
    const int e = max((int)((largest + 0x1fffffu) >> 23) - 135, -126);
    const float inv = __uint_as_float((uint32_t)(127 - e) << 23);  // e <= 120
    uint32_t codes[2];
#pragma unroll
    for (int i = 0; i < 2; ++i) {
      float y[4];
#pragma unroll
      for (int c = 0; c < 4; ++c) {
        const uint32_t word = w[2 * i + (c >> 1)];
        const uint32_t bits = c & 1 ? word & 0xffff0000u : word << 16;
        y[c] = (bits & 0x7f800000u) == 0x7f800000u ? __uint_as_float(0x7fc00000u) : __uint_as_float(bits) * inv;
      }
      int packed = __builtin_amdgcn_cvt_pk_fp8_f32(y[0], y[1], 0, false);
      packed = __builtin_amdgcn_cvt_pk_fp8_f32(y[2], y[3], packed, true);
      codes[i] = (uint32_t)packed;
    }
    if (keep) {
      *reinterpret_cast<uint2*>(to + lane * 8) = uint2{codes[0], codes[1]};
      if (lane == 0) (value ? ve : ke)[((int64_t)page * a.heads + h) * a.page.size + in] = (uint8_t)(e + 127);
    }
  }
}

template <int kType, int kDim>
hipError_t append(const void* k, const void* v, const int32_t* slots, void* kp, void* vp, uint8_t* ke, uint8_t* ve,
                  const AppendArgs& a, hipStream_t s) {
  constexpr int kRows = 256 / (kDim * (kType == 0 ? 4 : 2) / 16);
  const dim3 grid((unsigned)((a.tokens + kRows - 1) / kRows), (unsigned)a.heads, 2);
  hipLaunchKernelGGL((append_kernel<kType, kDim>), grid, dim3(256), 0, s, static_cast<const char*>(k),
                     static_cast<const char*>(v), slots, static_cast<char*>(kp), static_cast<char*>(vp), ke, ve, a);
  return hipGetLastError();
}

}  // namespace

hipError_t launch_page_tables(const int32_t* lengths, const int32_t* new_tokens, int32_t* free_pages,
                              const int32_t* free_count, int32_t* table, int32_t* lengths_out,
                              int32_t* count_out, int32_t* start, int32_t* slots,
                              RequestRecord* records, const StepArgs& a, hipStream_t s) {
  hipLaunchKernelGGL(page_scan_kernel, dim3(1), dim3(kScanThreads), 0, s, lengths, new_tokens, free_pages, free_count,
                     table, lengths_out, count_out, start, records, a);
  const hipError_t e = hipGetLastError();
  if (e != hipSuccess || a.tokens == 0) return e;
  hipLaunchKernelGGL(page_slots_kernel, dim3((unsigned)((a.tokens + kSlotThreads - 1) / kSlotThreads)),
                     dim3(kSlotThreads), 0, s, free_pages, table, start, slots, records, a);
  return hipGetLastError();
}

hipError_t launch_cache_append(int dtype, int dim, const void* k, const void* v, const int32_t* slots,
                               void* k_pages, void* v_pages, uint8_t* k_exp, uint8_t* v_exp,
                               const AppendArgs& a, hipStream_t s) {
  if (a.tokens == 0) return hipSuccess;
  if (dtype == 0)
    return dim == 64 ? append<0, 64>(k, v, slots, k_pages, v_pages, k_exp, v_exp, a, s)
                     : append<0, 128>(k, v, slots, k_pages, v_pages, k_exp, v_exp, a, s);
  if (dtype == 1)
    return dim == 64 ? append<1, 64>(k, v, slots, k_pages, v_pages, k_exp, v_exp, a, s)
                     : append<1, 128>(k, v, slots, k_pages, v_pages, k_exp, v_exp, a, s);
  return dim == 64 ? append<2, 64>(k, v, slots, k_pages, v_pages, k_exp, v_exp, a, s)
                   : append<2, 128>(k, v, slots, k_pages, v_pages, k_exp, v_exp, a, s);
}

}  // namespace saf3r
