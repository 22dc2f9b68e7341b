// The paged cache's bookkeeping and its writes.
#include "paged_internal.h"

namespace saf3r {
namespace {

constexpr int kSlotThreads = 256;
// Sums stop at a limit of at most 2^30 + 1: a + b fits 32 bits, and the order
// of additions does not matter.
__device__ inline uint32_t add_to(uint32_t a, uint32_t b, uint32_t limit) { return min(a + b, limit); }

// Sums of the threads before this one; `total` gets the sum of all.
template <int kScanThreads>
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
  for (int w = 0; w < kScanThreads / 64; ++w) {
    if (w == wave) before = all;
    all = add_to(all, waves[w], limit);
  }
  total = all;
  const uint32_t y = __shfl_up(x, 1);
  return lane == 0 ? before : add_to(before, y, limit);
}

// The last of `n` ascending entries, the first of which is at most x, that is.
__device__ inline int last_up_to(const uint32_t* from, int n, uint32_t x) {
  int lo = 0, hi = n;
  while (hi - lo > 1) {
    const int mid = (lo + hi) >> 1;
    if (from[mid] <= x) lo = mid;
    else hi = mid;
  }
  return lo;
}

// A new token's slot, and, where it is a page's first token, the page's entry in
// the table. stack(i): entry i of the stack that the pages are taken from.
template <typename Stack>
__device__ inline int32_t slot_of(int32_t t, const uint32_t* start, const RequestRecord* records, Stack stack,
                                  int32_t* table, const StepArgs& a) {
  const int r = last_up_to(start, a.requests, (uint32_t)t);
  const RequestRecord rec = records[r];
  if (rec.top < 0) return -1;
  const int32_t pos = rec.length + (t - (int32_t)start[r]);
  const int32_t i = div_page(a.page, pos);
  const int32_t in = pos - i * a.page.size;
  int32_t* entry = table + (int64_t)r * a.max_pages + i;
  int32_t page;
  if (i >= rec.held) {
    page = stack(rec.top - (i - rec.held));
    if (in == 0) *entry = page;
  } else {
    page = *entry;
  }
  // an entry of the table or the stack that is no page has no slots
  return page >= 0 && page < a.pages ? page * a.page.size + in : -1;
}

// What a thread knows of its request after the first pass over them.
struct Request {
  RequestRecord rec;      // top: provisional, 0 where the request may take pages at all
  int32_t fresh;          // its entry of new_tokens
  uint32_t first;         // where its new tokens start
  uint32_t back, behind;  // pages it gives back, and those of the requests before it
};

template <int kThreads>
__device__ inline Request read_request(int r, const int32_t* lengths, const int32_t* __restrict__ new_tokens, const StepArgs& a,
                                       uint32_t* waves, uint32_t& tokens_before, uint32_t& back_before) {
  const uint32_t token_limit = (uint32_t)a.tokens + 1, page_limit = (uint32_t)a.pages + 1;
  const int32_t capacity = a.max_pages * a.page.size;
  int32_t length = -1, fresh = 0;
  if (r < a.requests) {
    length = lengths[r];
    fresh = new_tokens[r];
  }
  const bool good = length >= 0 && length <= capacity;
  const bool ends = good && fresh < 0;
  const int32_t held = good ? div_page(a.page, length + a.page.size - 1) : 0;
  const uint32_t grow = min((uint32_t)max(fresh, 0), token_limit);
  Request q;
  uint32_t total;
  q.first = add_to(tokens_before, scan<kThreads>(grow, token_limit, waves, total), token_limit);
  tokens_before = add_to(tokens_before, total, token_limit);
  q.back = ends ? min((uint32_t)held, page_limit) : 0;
  q.behind = add_to(back_before, scan<kThreads>(q.back, page_limit, waves, total), page_limit);
  back_before = add_to(back_before, total, page_limit);
  q.rec = RequestRecord{length, good && !ends && q.first + grow < token_limit ? 0 : -1, held};
  q.fresh = fresh;
  return q;
}

// A wave copies its ended requests' rows to the stack one after another; a sum at
// its limit lies past the stack's end.
__device__ inline void push_pages(int r, const Request& q, uint32_t count, int32_t* free_pages, const int32_t* table,
                                  const StepArgs& a) {
  const int lane = threadIdx.x & 63;
  uint64_t todo = __ballot(q.back > 0);
  while (todo) {
    const int src = __ffsll((unsigned long long)todo) - 1;
    todo &= todo - 1;
    const int rr = r - lane + src;
    const uint32_t n = __shfl(q.back, src), at = count + __shfl(q.behind, src);
    for (uint32_t j = lane; j < n; j += 64)
      if (at + j < (uint32_t)a.pages) free_pages[at + j] = table[(int64_t)rr * a.max_pages + j];
  }
}

// The second pass: the pages that a request takes, and its length after the step.
template <int kThreads>
__device__ inline int32_t take_pages(RequestRecord& rec, int32_t fresh, uint32_t top, const StepArgs& a, uint32_t* waves,
                                     uint32_t& need_before, uint32_t& taken) {
  const uint32_t page_limit = (uint32_t)a.pages + 1;
  const int32_t capacity = a.max_pages * a.page.size;
  const bool ends = fresh < 0 && rec.length >= 0 && rec.length <= capacity;
  const bool may = rec.top == 0 && fresh <= capacity - rec.length;
  const int32_t after = may ? rec.length + fresh : 0;
  const uint32_t need = may ? min((uint32_t)(div_page(a.page, after + a.page.size - 1) - rec.held), page_limit) : 0;
  uint32_t total;
  const uint32_t first = add_to(need_before, scan<kThreads>(need, page_limit, waves, total), page_limit);
  const uint32_t to = add_to(first, need, page_limit);
  need_before = add_to(need_before, total, page_limit);
  const bool fits = may && (need == 0 || to <= top);
  rec.top = !fits ? -1 : need == 0 ? 0 : (int32_t)(top - 1 - first);
  // the sums grow with r, so the pages taken are the last sum that fits
  uint32_t mine = fits && need > 0 ? to : 0;
#pragma unroll
  for (int d = 32; d >= 1; d >>= 1) mine = max(mine, (uint32_t)__shfl_xor((int)mine, d));
  __syncthreads();
  if ((threadIdx.x & 63) == 0) waves[threadIdx.x >> 6] = mine;
  __syncthreads();
#pragma unroll
  for (int w = 0; w < kThreads / 64; ++w) taken = max(taken, waves[w]);
  return ends ? 0 : fits ? after : rec.length;
}

// A step of up to kThreads requests. The order of the requests is the order of the
// threads: ended sequences' pages are counted first, since what they give back
// decides who fits, then the pages that the others need. Every workgroup does this
// for itself and then finds the slots of its own new tokens; the first one writes
// what belongs to the requests. No workgroup waits for another: a page that an ended
// sequence gave back is read from that sequence's row, not from the stack. (Two
// launches, one to count and one with a thread per token: 10.2 us for 1000 requests
// at 4096 to 16384 tokens, and 4 us more of the host's time.)
template <int kThreads>
__global__ __launch_bounds__(kThreads) void page_step_kernel(
    const int32_t* lengths, const int32_t* __restrict__ new_tokens, int32_t* free_pages, const int32_t* free_count,
    int32_t* table, int32_t* lengths_out, int32_t* count_out, int32_t* __restrict__ start_out,
    int32_t* __restrict__ slots, StepArgs a) {
  __shared__ uint32_t waves[kThreads / 64];
  __shared__ uint32_t starts[kThreads];
  __shared__ uint32_t behind[kThreads];
  __shared__ RequestRecord records[kThreads];
  const int r = threadIdx.x;
  const uint32_t count = (uint32_t)min(max(*free_count, 0), a.pages);
  uint32_t tokens = 0, back = 0;
  Request q = read_request<kThreads>(r, lengths, new_tokens, a, waves, tokens, back);
  starts[r] = min(q.first, (uint32_t)a.tokens);
  behind[r] = q.behind;
  const int32_t end = (int32_t)min(tokens, (uint32_t)a.tokens);
  const uint32_t top = min(count + back, (uint32_t)a.pages);
  uint32_t need = 0, taken = 0;
  const int32_t after = take_pages<kThreads>(q.rec, q.fresh, top, a, waves, need, taken);
  records[r] = q.rec;
  if (blockIdx.x == 0) {
    if (r < a.requests) {
      start_out[r] = (int32_t)starts[r];
      lengths_out[r] = after;
    }
    if (r == 0) {
      start_out[a.requests] = end;
      *count_out = (int32_t)(top - taken);
    }
    push_pages(r, q, count, free_pages, table, a);
  }
  __syncthreads();
  const auto stack = [&](int32_t i) {
    if ((uint32_t)i < count) return free_pages[i];
    const uint32_t off = (uint32_t)i - count;
    const int from = last_up_to(behind, a.requests, off);
    return table[(int64_t)from * a.max_pages + (off - behind[from])];
  };
  const int32_t first = (int32_t)blockIdx.x * (kThreads * kSlotsEach);
#pragma unroll
  for (int i = 0; i < kSlotsEach; ++i) {
    const int32_t t = first + i * kThreads + r;
    if (t < a.tokens) slots[t] = t < end ? slot_of(t, starts, records, stack, table, a) : -1;
  }
}

// A step of any number of requests, kScanThreads a turn, by one workgroup; the slots
// follow in a launch of their own.
constexpr int kScanThreads = 1024;
__global__ __launch_bounds__(kScanThreads) void page_scan_kernel(
    const int32_t* lengths, const int32_t* __restrict__ new_tokens, int32_t* free_pages,
    const int32_t* free_count, const int32_t* table, int32_t* lengths_out, int32_t* count_out,
    int32_t* __restrict__ start_out, RequestRecord* __restrict__ records, StepArgs a) {
  __shared__ uint32_t waves[kScanThreads / 64];
  const uint32_t count = (uint32_t)min(max(*free_count, 0), a.pages);
  uint32_t tokens = 0, back = 0;
  for (int r0 = 0; r0 < a.requests; r0 += kScanThreads) {
    const int r = r0 + threadIdx.x;
    const Request q = read_request<kScanThreads>(r, lengths, new_tokens, a, waves, tokens, back);
    if (r < a.requests) {
      start_out[r] = (int32_t)min(q.first, (uint32_t)a.tokens);
      records[r] = q.rec;
    }
    push_pages(r, q, count, free_pages, table, a);
  }
  const uint32_t top = min(count + back, (uint32_t)a.pages);
  uint32_t need = 0, taken = 0;
  for (int r0 = 0; r0 < a.requests; r0 += kScanThreads) {
    const int r = r0 + threadIdx.x;
    RequestRecord rec{-1, -1, 0};
    int32_t fresh = 0;
    if (r < a.requests) {
      rec = records[r];
      fresh = new_tokens[r];
    }
    const int32_t after = take_pages<kScanThreads>(rec, fresh, top, a, waves, need, taken);
    if (r < a.requests) {
      records[r].top = rec.top;
      lengths_out[r] = after;
    }
  }
  if (threadIdx.x == 0) {
    start_out[a.requests] = (int32_t)min(tokens, (uint32_t)a.tokens);
    *count_out = (int32_t)(top - taken);
  }
}

// One thread per new token.
__global__ __launch_bounds__(kSlotThreads) void page_slots_kernel(
    const int32_t* __restrict__ free_pages, int32_t* table, const int32_t* __restrict__ start,
    int32_t* __restrict__ slots, const RequestRecord* __restrict__ records, StepArgs a) {
  const int t = blockIdx.x * kSlotThreads + threadIdx.x;
  if (t >= a.tokens) return;
  const auto stack = [&](int32_t i) { return free_pages[i]; };
  slots[t] = t < start[a.requests] ? slot_of(t, reinterpret_cast<const uint32_t*>(start), records, stack, table, a) : -1;
}

// One row (token, head, K or V) to the lanes that its 16 bytes (in 8 bits: 32 of its
// input) each make up; a workgroup's rows are consecutive tokens of one head, so that
// both the framework's [heads, N, dim] tokens and a page are read and written as long
// runs.
template <int kType, int kDim>
struct AppendShape {
  static constexpr int kIn = kType == 0 ? 4 : 2;
  static constexpr int kVecs = kType == 2 ? 2 : 1;  // 16-byte loads of a lane
  static constexpr int kLanes = kDim * kIn / 16 / kVecs;
  static constexpr int kRows = 256 / kLanes;
};
template <int kType, int kDim>
__global__ __launch_bounds__(256) void append_kernel(const char* __restrict__ k, const char* __restrict__ v,
                                                     const int32_t* __restrict__ slots, char* __restrict__ kp,
                                                     char* __restrict__ vp, uint8_t* __restrict__ ke,
                                                     uint8_t* __restrict__ ve, AppendArgs a) {
  using S = AppendShape<kType, kDim>;
  const int lane = threadIdx.x % S::kLanes;
  const int64_t t = (int64_t)blockIdx.x * S::kRows + threadIdx.x / S::kLanes;
  const int h = blockIdx.y;
  const bool value = blockIdx.z != 0;
  const int32_t slot = t < a.tokens ? slots[t] : -1;
  const bool keep = slot >= 0 && slot < a.slots;
  uint4 x[S::kVecs];
  const uint4* from = reinterpret_cast<const uint4*>((value ? v : k) + h * a.row_head + t * a.row_token) + lane * S::kVecs;
#pragma unroll
  for (int i = 0; i < S::kVecs; ++i) x[i] = keep ? from[i] : uint4{0, 0, 0, 0};
  const int32_t page = keep ? div_page(a.page, slot) : 0;
  const int32_t in = slot - page * a.page.size;
  char* to = (value ? vp : kp) + page * a.page_stride + h * a.head_stride + in * a.token_stride;
  if constexpr (kType != 2) {
    if (keep) *reinterpret_cast<uint4*>(to + lane * 16) = x[0];
  } else {
    const uint32_t w[8] = {x[0].x, x[0].y, x[0].z, x[0].w, x[1].x, x[1].y, x[1].z, x[1].w};
    uint32_t largest = 0;
#pragma unroll
    for (int i = 0; i < 8; ++i) {
      const uint32_t lo = (w[i] << 16) & 0x7fffffffu, hi = w[i] & 0x7fff0000u;
      largest = max(largest, lo < 0x7f800000u ? lo : 0u);
      largest = max(largest, hi < 0x7f800000u ? hi : 0u);
    }
#pragma unroll
    for (int d = S::kLanes / 2; d >= 1; d >>= 1) largest = max(largest, (uint32_t)__shfl_xor((int)largest, d));
    // 448 = 1.75 * 2^8: the carry out of the mantissa is there from 1.75 on
    const int e = max((int)((largest + 0x1fffffu) >> 23) - 135, -126);
    const float inv = __uint_as_float((uint32_t)(127 - e) << 23);  // e <= 120
    uint32_t codes[4];
#pragma unroll
    for (int i = 0; i < 4; ++i) {
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
      *reinterpret_cast<uint4*>(to + lane * 16) = uint4{codes[0], codes[1], codes[2], codes[3]};
      if (lane == 0) (value ? ve : ke)[((int64_t)page * a.heads + h) * a.page.size + in] = (uint8_t)(e + 127);
    }
  }
}

template <int kType, int kDim>
hipError_t append(const void* k, const void* v, const int32_t* slots, void* kp, void* vp, uint8_t* ke, uint8_t* ve,
                  const AppendArgs& a, hipStream_t s) {
  constexpr int kRows = AppendShape<kType, kDim>::kRows;
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
  if (page_tables_in_one(a.requests, a.tokens, a.in_place != 0)) {
    // four waves where they are enough (64 requests, 1024 tokens: 5.7 us, 6.6 with 16)
    const bool small = a.requests <= 256 && a.tokens <= 256 * kSlotsEach;
    const int each = (small ? 256 : kStepRequests) * kSlotsEach;
    const dim3 grid((unsigned)(a.tokens > each ? (a.tokens + each - 1) / each : 1));
    if (small)
      hipLaunchKernelGGL(page_step_kernel<256>, grid, dim3(256), 0, s, lengths, new_tokens, free_pages, free_count, table,
                         lengths_out, count_out, start, slots, a);
    else
      hipLaunchKernelGGL(page_step_kernel<kStepRequests>, grid, dim3(kStepRequests), 0, s, lengths, new_tokens, free_pages,
                         free_count, table, lengths_out, count_out, start, slots, a);
    return hipGetLastError();
  }
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
