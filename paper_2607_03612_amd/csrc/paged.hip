// The paged cache's bookkeeping and its writes.
#include "paged_internal.h"

namespace saf3r {
namespace {

constexpr int kSlotThreads = 256;
// Sums stop at a limit of at most 2^30 + 1: a + b fits 32 bits, and the order
// of additions does not matter.
__device__ inline uint32_t add_to(uint32_t a, uint32_t b, uint32_t limit) { return min(a + b, limit); }

// The sum over a wave's lanes up to and with this one: within rows of 16 lanes, then
// each row's last lane to the rows behind it, all in registers.
template <int kCtrl, int kRows>
__device__ inline uint32_t shifted(uint32_t x) {
  return (uint32_t)__builtin_amdgcn_update_dpp(0, (int)x, kCtrl, kRows, 0xf, false);
}
__device__ inline uint32_t wave_scan(uint32_t x, uint32_t limit) {
  x = add_to(x, shifted<0x111, 0xf>(x), limit);  // from 1, 2, 4, 8 lanes before
  x = add_to(x, shifted<0x112, 0xf>(x), limit);
  x = add_to(x, shifted<0x114, 0xf>(x), limit);
  x = add_to(x, shifted<0x118, 0xf>(x), limit);
  x = add_to(x, shifted<0x142, 0xa>(x), limit);  // lane 15 to row 1, 47 to row 3
  x = add_to(x, shifted<0x143, 0xc>(x), limit);  // lane 31 to rows 2 and 3
  return x;
}

// Sums of the threads before this one, for kSums values at once; `total` gets those
// of all.
template <int kThreads, int kSums>
__device__ inline void scan(const uint32_t (&x)[kSums], const uint32_t (&limit)[kSums], uint32_t (*waves)[kThreads / 64],
                            uint32_t (&before)[kSums], uint32_t (&total)[kSums]) {
  const int lane = threadIdx.x & 63, wave = threadIdx.x >> 6;
  uint32_t to[kSums];
#pragma unroll
  for (int i = 0; i < kSums; ++i) to[i] = wave_scan(x[i], limit[i]);
  __syncthreads();  // the last scan's reads of `waves`
#pragma unroll
  for (int i = 0; i < kSums; ++i)
    if (lane == 63) waves[i][wave] = to[i];
  __syncthreads();
#pragma unroll
  for (int i = 0; i < kSums; ++i) {
    uint32_t ahead = 0, all = 0;
#pragma unroll
    for (int w = 0; w < kThreads / 64; ++w) {
      if (w == wave) ahead = all;
      all = add_to(all, waves[i][w], limit[i]);
    }
    total[i] = all;
    const uint32_t y = __shfl_up(to[i], 1);
    before[i] = lane == 0 ? ahead : add_to(ahead, y, limit[i]);
  }
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

// Sums over the requests so far.
struct Sums {
  uint32_t tokens, back;  // of the first pass: new tokens, pages given back
  uint32_t need;          // of the second: pages asked for
};

template <int kThreads>
__device__ inline Request read_request(int r, const int32_t* lengths, const int32_t* __restrict__ new_tokens, const StepArgs& a,
                                       uint32_t (*waves)[kThreads / 64], Sums& sums) {
  const uint32_t limit[2] = {(uint32_t)a.tokens + 1, (uint32_t)a.pages + 1};
  const int32_t capacity = a.max_pages * a.page.size;
  int32_t length = -1, fresh = 0;
  if (r < a.requests) {
    length = lengths[r];
    fresh = new_tokens[r];
  }
  const bool good = length >= 0 && length <= capacity;
  const bool ends = good && fresh < 0;
  const int32_t held = good ? div_page(a.page, length + a.page.size - 1) : 0;
  const uint32_t x[2] = {min((uint32_t)max(fresh, 0), limit[0]), ends ? min((uint32_t)held, limit[1]) : 0};
  uint32_t before[2], total[2];
  scan<kThreads, 2>(x, limit, waves, before, total);
  Request q;
  q.first = add_to(sums.tokens, before[0], limit[0]);
  sums.tokens = add_to(sums.tokens, total[0], limit[0]);
  q.back = x[1];
  q.behind = add_to(sums.back, before[1], limit[1]);
  sums.back = add_to(sums.back, total[1], limit[1]);
  q.rec = RequestRecord{length, good && !ends && q.first + x[0] < limit[0] ? 0 : -1, held};
  q.fresh = fresh;
  return q;
}

// The second pass: the pages that a request takes, and its length after the step. The
// sums grow with r, so the pages taken in all are the last sum that fits.
template <int kThreads>
__device__ inline int32_t take_pages(RequestRecord& rec, int32_t fresh, uint32_t top, const StepArgs& a,
                                     uint32_t (*waves)[kThreads / 64], Sums& sums, uint32_t* taken) {
  const uint32_t limit[1] = {(uint32_t)a.pages + 1};
  const int32_t capacity = a.max_pages * a.page.size;
  const bool ends = fresh < 0 && rec.length >= 0 && rec.length <= capacity;
  const bool may = rec.top == 0 && fresh <= capacity - rec.length;
  const int32_t after = may ? rec.length + fresh : 0;
  const uint32_t need[1] = {may ? min((uint32_t)(div_page(a.page, after + a.page.size - 1) - rec.held), limit[0]) : 0};
  uint32_t before[1], total[1];
  scan<kThreads, 1>(need, limit, waves, before, total);
  const uint32_t first = add_to(sums.need, before[0], limit[0]), to = add_to(first, need[0], limit[0]);
  sums.need = add_to(sums.need, total[0], limit[0]);
  const bool fits = may && (need[0] == 0 || to <= top);
  rec.top = !fits ? -1 : need[0] == 0 ? 0 : (int32_t)(top - 1 - first);
  const uint64_t some = __ballot(fits && need[0] > 0);
  if (some && (threadIdx.x & 63) == 63 - __clzll((long long)some)) atomicMax(taken, to);
  return ends ? 0 : fits ? after : rec.length;
}

// A step of up to kThreads requests. The order of the requests is the order of the
// threads: ended sequences' pages are counted first, since what they give back
// decides who fits, then the pages that the others need. Every workgroup does this
// for itself and then finds the slots of its share of the new tokens and copies its
// share of the pages given back; the first one writes what belongs to the requests. No
// workgroup waits for another: a page that an ended sequence gave back is read from
// that sequence's row, not from the stack. Bound by the chain of lengths, sums, table
// and stores: 2.7 us for 64 requests and as many tokens, 7.2 for 1000 with 21000 tokens
// and 37 that end. (Two launches, one to count and one with a thread per token: 10.3 us
// for a request more than the 1024 that take 5.2 here, and 4 us more of the host's time.)
template <int kThreads>
__global__ __launch_bounds__(kThreads) void page_step_kernel(
    const int32_t* lengths, const int32_t* __restrict__ new_tokens, int32_t* free_pages, const int32_t* free_count,
    int32_t* table, int32_t* lengths_out, int32_t* count_out, int32_t* __restrict__ start_out,
    int32_t* __restrict__ slots, StepArgs a) {
  __shared__ uint32_t waves[2][kThreads / 64];
  __shared__ uint32_t starts[kThreads];
  __shared__ uint32_t behind[kThreads];
  __shared__ RequestRecord records[kThreads];
  __shared__ uint32_t taken;
  const int r = threadIdx.x;
  if (r == 0) taken = 0;
  const uint32_t count = (uint32_t)min(max(*free_count, 0), a.pages);
  Sums sums{0, 0, 0};
  Request q = read_request<kThreads>(r, lengths, new_tokens, a, waves, sums);
  starts[r] = min(q.first, (uint32_t)a.tokens);
  behind[r] = q.behind;
  const int32_t end = (int32_t)min(sums.tokens, (uint32_t)a.tokens);
  const uint32_t top = min(count + sums.back, (uint32_t)a.pages);
  const int32_t after = take_pages<kThreads>(q.rec, q.fresh, top, a, waves, sums, &taken);
  records[r] = q.rec;
  if (blockIdx.x == 0 && r < a.requests) {
    start_out[r] = (int32_t)starts[r];
    lengths_out[r] = after;
  }
  __syncthreads();
  if (blockIdx.x == 0 && r == 0) {
    start_out[a.requests] = end;
    *count_out = (int32_t)(top - taken);
  }
  const auto given_back = [&](uint32_t i) {
    const int from = last_up_to(behind, a.requests, i);
    return table[(int64_t)from * a.max_pages + (i - behind[from])];
  };
  const auto stack = [&](int32_t i) { return (uint32_t)i < count ? free_pages[i] : given_back((uint32_t)i - count); };
  const uint32_t mine = blockIdx.x * kThreads + r, all = gridDim.x * kThreads;
  for (uint32_t t = mine; t < (uint32_t)a.tokens; t += all)
    slots[t] = (int32_t)t < end ? slot_of((int32_t)t, starts, records, stack, table, a) : -1;
  for (uint32_t i = mine; i < top - count; i += all) free_pages[count + i] = given_back(i);
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

// A step of any number of requests, kScanThreads a turn, by one workgroup that goes over
// them twice; the slots follow in a launch of their own. Bound by the chain of reads and
// sums, about 1.2 us for a turn of one pass. Both launches: 6.7 us for 100 requests with
// 137400 tokens in place, 10.3 for 1025 requests with a token each, 16 for 4096, 43 for
// 16384, 150 for 65536. Pages that are given back come on top, a wave's ended requests
// one after another: 7 us for 11300 pages of 128 requests among 4096, 73 for 23100 of
// 2048 among 65536.
constexpr int kScanThreads = 1024;
__global__ __launch_bounds__(kScanThreads) void page_scan_kernel(
    const int32_t* lengths, const int32_t* __restrict__ new_tokens, int32_t* free_pages,
    const int32_t* free_count, const int32_t* table, int32_t* lengths_out, int32_t* count_out,
    int32_t* __restrict__ start_out, RequestRecord* __restrict__ records, StepArgs a) {
  __shared__ uint32_t waves[2][kScanThreads / 64];
  __shared__ uint32_t taken;
  if (threadIdx.x == 0) taken = 0;
  const uint32_t count = (uint32_t)min(max(*free_count, 0), a.pages);
  Sums sums{0, 0, 0};
  for (int r0 = 0; r0 < a.requests; r0 += kScanThreads) {
    const int r = r0 + threadIdx.x;
    const Request q = read_request<kScanThreads>(r, lengths, new_tokens, a, waves, sums);
    if (r < a.requests) {
      start_out[r] = (int32_t)min(q.first, (uint32_t)a.tokens);
      records[r] = q.rec;
    }
    push_pages(r, q, count, free_pages, table, a);
  }
  const uint32_t top = min(count + sums.back, (uint32_t)a.pages);
  for (int r0 = 0; r0 < a.requests; r0 += kScanThreads) {
    const int r = r0 + threadIdx.x;
    RequestRecord rec{-1, -1, 0};
    int32_t fresh = 0;
    if (r < a.requests) {
      rec = records[r];
      fresh = new_tokens[r];
    }
    const int32_t after = take_pages<kScanThreads>(rec, fresh, top, a, waves, sums, &taken);
    if (r < a.requests) {
      records[r].top = rec.top;
      lengths_out[r] = after;
    }
  }
  __syncthreads();
  if (threadIdx.x == 0) {
    start_out[a.requests] = (int32_t)min(sums.tokens, (uint32_t)a.tokens);
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
// runs. Bound by HBM: 137400 tokens of 16 heads of 64 in bf16 201 us, 5.6 TB/s read and
// written; 43968 into 8 bits 48.6 us, the same rate (63 with 16 bytes of input a lane).
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
    // four waves where they are as many as the requests ask for; in place, one
    // workgroup and more of them for many tokens
    const bool small = a.requests <= 256 && (!a.in_place || a.tokens <= 1024);
    const int threads = small ? 256 : kStepRequests;
    const int64_t want = ((int64_t)a.tokens + threads - 1) / threads;
    const dim3 grid(a.in_place || want < 1 ? 1u : (unsigned)(want < kStepGroups ? want : kStepGroups));
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
