// Attention of several new tokens per request over a paged cache.
//
// The rows of a request are its new tokens times the query heads that share a
// key-value head; a workgroup takes a tile of them and walks the keys that any of them
// sees, 32 at a time, K and V of these in LDS for its four waves:
//   S^T = K Q^T   (keys x rows), so a lane owns a row and half of the 32 keys
//   O^T += V^T P^T
// on the 32x32 products, with an online softmax. P^T is taken where S^T left it: which
// keys share a lane is free as long as V^T has them in the same places.
// Caches of 8 and 4 bits become bf16 on their way into LDS, exactly.
#include <type_traits>

#include "paged_deal.h"
#include "paged_scores.h"

namespace saf3r {
namespace {

typedef __bf16 bf16x8 __attribute__((ext_vector_type(8)));
typedef __bf16 bf16x4 __attribute__((ext_vector_type(4)));
typedef __bf16 bf16x2 __attribute__((ext_vector_type(2)));
typedef float f32x4 __attribute__((ext_vector_type(4)));
typedef float f32x16 __attribute__((ext_vector_type(16)));
typedef uint32_t u32x4 __attribute__((ext_vector_type(4)));
typedef uint32_t u32x2 __attribute__((ext_vector_type(2)));
typedef __attribute__((address_space(3))) bf16x4 lds_bf16x4;

constexpr float kLn2 = 0.6931471805599453f, kLog2e = 1.4426950408889634f;

__device__ inline float pair_max(float x) {
  const auto s = __builtin_amdgcn_permlane32_swap(__float_as_uint(x), __float_as_uint(x), false, false);
  return fmaxf(__uint_as_float(s[0]), __uint_as_float(s[1]));
}
__device__ inline float pair_sum(float x) {
  const auto s = __builtin_amdgcn_permlane32_swap(__float_as_uint(x), __float_as_uint(x), false, false);
  return __uint_as_float(s[0]) + __uint_as_float(s[1]);
}

// The same for a whole wave; r: a request at or before the one that has number x.
template <int kRows>
__device__ inline Tile next_tile(const PromptArgs& a, const int32_t* __restrict__ lengths, const int32_t* __restrict__ start,
                                 const int32_t* __restrict__ prefix, int32_t r, int32_t x) {
  int32_t first = start_of(a, start, r), end = start_of(a, start, r + 1);
  while (r + 1 < a.requests && number_of<kRows>(a, end, r + 1) <= x) {
    ++r;
    first = end;
    end = start_of(a, start, r + 1);
  }
  Tile t = tile_of<kRows>(a, lengths, prefix, __builtin_amdgcn_readfirstlane(r), __builtin_amdgcn_readfirstlane(first),
                          __builtin_amdgcn_readfirstlane(end), x);
  t.n = __builtin_amdgcn_readfirstlane(t.n);
  t.prefix = __builtin_amdgcn_readfirstlane(t.prefix);
  t.head = __builtin_amdgcn_readfirstlane(t.head);
  t.skip = __builtin_amdgcn_readfirstlane(t.skip);
  t.count = __builtin_amdgcn_readfirstlane(t.count);
  return t;
}
// The request that has number x, by a whole wave, 64 requests at a time: three turns at
// most; 0 where x lies before all.
template <int kRows>
__device__ inline int32_t request_of(const PromptArgs& a, const int32_t* __restrict__ start, int32_t x) {
  const int lane = threadIdx.x & 63;
  int32_t lo = 0, hi = a.requests;
  while (true) {
    const int32_t step = (hi - lo + 63) / 64, r = lo + lane * step;
    const uint64_t reached = __ballot(r < hi && number_of<kRows>(a, start_of(a, start, r), r) <= x);
    if (!reached) return 0;
    lo += (63 - __clzll((long long)reached)) * step;
    if (step == 1) return __builtin_amdgcn_readfirstlane(lo);
    hi = min(lo + step, hi);
  }
}

// ---------------------------------------------- steps dealt out among workgroups

// The steps of all tiles of all key-value heads, head by head, in equal runs of
// neighbouring ones to a.groups workgroups, whatever the lengths (the GPU's), as the one-token
// kernel does with its tiles. A tile that falls to several leaves a part in each, workgroup w's in
// slot 2w if it began before and in slot 2w + 1 if it begins there: of each row kDim sums
// and (m, l). With a workgroup for each tile instead, 16 drafted tokens for each of 4
// sequences of 10992 took 429 us, not 88, a frame of 1374 over 137400 with 16 heads 3079, not
// 1048. Where tiles are many, dealing out costs: 10992 tokens at once 1309 us, not 982
// (neighbours then stand at different keys, and miss L2), 12 ragged prompts 406, not 374.
struct Cut {
  int32_t row, rows, first, h;
  int32_t from, to;
};
static_assert(sizeof(Cut) == kCutRecord, "the workspace's size counts on it");
struct Parts {
  float* o;    // [2 groups][slot_rows][kDim]
  float2* ml;  // [2 groups][slot_rows]
  // a tile that begins in workgroup w and ends in a later one: its first row, rows from there
  // on, first token, key-value head; w, the last one; else w < 0
  Cut* cut;
};
template <int kDim>
__device__ inline Parts parts_of(const PromptArgs& a, void* workspace) {
  Parts p;
  p.cut = static_cast<Cut*>(workspace);
  p.ml = reinterpret_cast<float2*>(p.cut + a.groups);
  p.o = reinterpret_cast<float*>(p.ml + (int64_t)2 * a.groups * a.slot_rows);
  return p;
}
// A run's place: its tile, head and step in the tile, and the steps left.
struct Run {
  Tile t;
  int32_t x, h, step;
  int64_t left;
  int64_t at, total;  // of the run's next step among all, and their number
  bool nothing;       // some tile has rows but no step
};

constexpr int kStarts = kMaxDealt;  // their starts are kept in LDS
template <int kThreads>
struct DealLds {
  int64_t before[kThreads];  // steps of the tiles before a thread's
  int64_t wave_sum[kThreads / 64];
  int32_t starts[kStarts + 1];
};

// Counts the steps, each thread those of neighbouring tiles, and finds the run of workgroup w.
template <int kThreads, int kRows>
__device__ inline Run find_run(const PromptArgs& a, const int32_t* __restrict__ lengths, const int32_t* __restrict__ start,
                               const int32_t* __restrict__ prefix, int w, DealLds<kThreads>& lds) {
  const int lane = threadIdx.x & 63, wave = threadIdx.x >> 6;
  for (int i = threadIdx.x; i <= a.requests; i += kThreads) lds.starts[i] = start_of(a, start, i);
  __syncthreads();
  const auto at = [&](int32_t r) { return lds.starts[r]; };
  const int32_t each = (a.tiles + kThreads - 1) / kThreads, x0 = threadIdx.x * each;
  int64_t mine = 0;
  bool nothing = false;
  if (x0 < a.tiles) {
    int32_t r = 0, hi = a.requests;
    while (hi - r > 1) {
      const int32_t mid = (r + hi) >> 1;
      if (number_of<kRows>(a, at(mid), mid) <= x0) r = mid;
      else hi = mid;
    }
    int32_t first = at(r), end = at(r + 1);
    for (int32_t x = x0; x < min(x0 + each, a.tiles); ++x) {
      while (r + 1 < a.requests && number_of<kRows>(a, end, r + 1) <= x) {
        ++r;
        first = end;
        end = at(r + 1);
      }
      const int64_t row = (int64_t)(x - number_of<kRows>(a, first, r)) * kRows;
      if (row < 0 || row >= (int64_t)(end - first) * a.group) continue;
      const int32_t count = tile_of<kRows>(a, lengths, prefix, r, first, end, x).count;
      mine += count;
      nothing |= count == 0;
    }
  }
  int64_t sum = mine;
#pragma unroll
  for (int d = 1; d < 64; d <<= 1) {
    const int64_t y = __shfl_up(sum, d);
    if (lane >= d) sum += y;
  }
  if (lane == 63) lds.wave_sum[wave] = sum;
  __syncthreads();
  int64_t head = 0;
#pragma unroll
  for (int i = 0; i < kThreads / 64; ++i) {
    if (i == wave) sum += head;
    head += lds.wave_sum[i];
  }
  lds.before[threadIdx.x] = sum - mine;
  Run run;
  run.nothing = __syncthreads_or(nothing);
  run.total = head * a.kv_heads;
  run.at = run_start(a, run.total, w);
  run.left = run_start(a, run.total, w + 1) - run.at;
  if (run.left <= 0) return run;
  run.h = (int32_t)(run.at / head);
  int64_t off = run.at - run.h * head;
  int owner = -1;
#pragma unroll
  for (int i = 0; i < kThreads / 64; ++i) owner += __popcll(__ballot(lds.before[64 * i + lane] <= off));
  off -= lds.before[owner];
  run.x = __builtin_amdgcn_readfirstlane(owner * each);
  int32_t r = request_of<kRows>(a, lds.starts, run.x);
  // ends before the last number; behind it only where starts go back and the counts differ
  for (; run.x < a.tiles; ++run.x) {
    run.t = next_tile<kRows>(a, lengths, lds.starts, prefix, r, run.x);
    r = run.t.r;
    if (off < run.t.count) break;
    off -= run.t.count;
  }
  if (run.x == a.tiles) run.left = 0;
  run.h = __builtin_amdgcn_readfirstlane(run.h);
  run.step = __builtin_amdgcn_readfirstlane((int32_t)off);
  return run;
}
// Behind a tile's last step: the next one that has any. There is one while steps are left;
// where starts go back there may be none, and the run ends.
template <int kRows>
__device__ inline void next_of(const PromptArgs& a, const int32_t* __restrict__ lengths, const int32_t* __restrict__ start,
                               const int32_t* __restrict__ prefix, Run& run) {
  run.step = 0;
  int32_t r = run.t.r;
  do {
    if (++run.x == a.tiles) {
      run.x = 0;
      r = 0;
      if (++run.h >= a.kv_heads) {
        run.left = 0;
        return;
      }
    }
    run.t = next_tile<kRows>(a, lengths, start, prefix, r, run.x);
    r = run.t.r;
  } while (run.t.count == 0);
}

// 32 keys of K or V in LDS. bf16: panels of 64 dimensions, rows of 128 bytes; 16-byte piece
// c of row r lies at place c ^ f(r), so that the reads of both products touch every bank
// once. fp32: rows with 16 bytes behind them, to the same end.
__device__ inline int swz_f(int r) { return ((r >> 2) & 1) | (r & 2) | (((r ^ (r >> 1) ^ (r >> 3)) & 1) << 2); }
__device__ inline int swz(int r, int c) { return r * 128 + ((c ^ swz_f(r)) << 4); }

__device__ inline uint32_t fp8_pair(uint32_t codes, bool high, float scale) {
  const bf16x2 x = high ? __builtin_amdgcn_cvt_scalef32_pk_bf16_fp8(codes, scale, true)
                        : __builtin_amdgcn_cvt_scalef32_pk_bf16_fp8(codes, scale, false);
  return __builtin_bit_cast(uint32_t, x);
}
template <int kByte>
__device__ inline uint32_t fp4_pair(uint32_t codes, float scale) {
  return __builtin_bit_cast(uint32_t, (bf16x2)__builtin_amdgcn_cvt_scalef32_pk_bf16_fp4(codes, scale, kByte));
}

// A row's output.
template <bool kF32, int kDim, int kTq>
__device__ __forceinline__ void put_row(const PromptArgs& a, const f32x16 (&o)[kDim / 32][kTq], int tq, int hf, int32_t head, int32_t token,
                                        float m, float l, char* __restrict__ out, float* __restrict__ lse) {
  const float f = l > 0.0f ? 1.0f / l : l;  // 0 and NaN stay
  const int64_t at = head * a.out_head + token * a.out_token;
#pragma unroll
  for (int c = 0; c < kDim / 32; ++c)
#pragma unroll
    for (int g = 0; g < 4; ++g) {
      const f32x4 x = f32x4{o[c][tq][4 * g], o[c][tq][4 * g + 1], o[c][tq][4 * g + 2], o[c][tq][4 * g + 3]} * f;
      const int64_t d = at + 32 * c + 8 * g + 4 * hf;
      if constexpr (kF32)
        *reinterpret_cast<f32x4*>(reinterpret_cast<float*>(out) + d) = x;
      else
        *reinterpret_cast<bf16x4*>(reinterpret_cast<__bf16*>(out) + d) = __builtin_convertvector(x, bf16x4);
    }
  if (lse && hf == 0) lse[(int64_t)head * a.tokens + token] = (m + __log2f(l)) * kLn2;
}
// A row's part of a tile's keys.
template <int kDim, int kTq>
__device__ __forceinline__ void put_part(const Parts& p, const f32x16 (&o)[kDim / 32][kTq], int tq, int hf, int64_t at, float m, float l) {
  if (hf == 0) p.ml[at] = float2{m, l};
#pragma unroll
  for (int c = 0; c < kDim / 32; ++c)
#pragma unroll
    for (int g = 0; g < 4; ++g)
      *reinterpret_cast<f32x4*>(p.o + at * kDim + 32 * c + 8 * g + 4 * hf) =
          f32x4{o[c][tq][4 * g], o[c][tq][4 * g + 1], o[c][tq][4 * g + 2], o[c][tq][4 * g + 3]};
}
// Rows that see nothing have no step: their outputs, by the workgroups in turn.
template <bool kF32, int kDim, int kRows>
__device__ inline void put_nothing(const PromptArgs& a, const int32_t* __restrict__ lengths, const int32_t* __restrict__ start,
                                   const int32_t* __restrict__ prefix, int32_t x, int32_t h, int threads, char* __restrict__ out,
                                   float* __restrict__ lse) {
  const Tile t = next_tile<kRows>(a, lengths, start, prefix, request_of<kRows>(a, start, x), x);
  if (t.count > 0 || x < number_of<kRows>(a, t.first, t.r)) return;
  const int64_t row0 = (int64_t)(x - number_of<kRows>(a, t.first, t.r)) * kRows;
  constexpr int kLanes = kDim / 4;
  for (int i = threadIdx.x; i < kRows * kLanes; i += threads) {
    const int64_t row = row0 + i / kLanes;
    if (row >= t.rows) break;
    const int32_t token = t.first + (int32_t)row / a.group, head = h * a.group + (int32_t)row % a.group, d = i % kLanes * 4;
    const int64_t at = head * a.out_head + token * a.out_token + d;
    if constexpr (kF32)
      *reinterpret_cast<f32x4*>(reinterpret_cast<float*>(out) + at) = f32x4{0, 0, 0, 0};
    else
      *reinterpret_cast<u32x2*>(reinterpret_cast<__bf16*>(out) + at) = u32x2{0, 0};
    if (lse && d == 0) lse[(int64_t)head * a.tokens + token] = -INFINITY;
  }
}

// What a workgroup needs between its tiles, in LDS: in registers it would push the
// walk's own out of them.
template <int kThreads>
struct Desk {
  PromptArgs a;
  const int32_t *lengths, *start, *prefix;
  char* out;
  float* lse;
  void* workspace;
  int32_t w;
  Run run;
  DealLds<kThreads> deal;
};
__device__ inline int32_t uniform(int32_t x) { return __builtin_amdgcn_readfirstlane(x); }

// What a workgroup does: with a.groups its run of steps, else one tile. segment(t, h, lo,
// hi, done) goes through the tile's steps lo .. hi - 1 and calls done(o, tq, hf, row, m, l) for
// each of the lane's rows.
template <bool kF32, int kDim, int kRows, int kThreads, typename Segment>
__device__ __forceinline__ void work(const PromptArgs& args, const int32_t* __restrict__ lengths, const int32_t* __restrict__ start,
                                     const int32_t* __restrict__ prefix, char* __restrict__ out, float* __restrict__ lse,
                                     void* __restrict__ workspace, Desk<kThreads>& desk, Segment segment) {
  {
    Run run;
    int w = 0;
    if (args.groups == 0) {
      // a request's longest rows first, of all heads; neighbouring workgroups run on
      // different XCDs, so with 8 heads each XCD has one of them
      run.x = args.tiles - 1 - (int)(blockIdx.y * kTilesAcross + blockIdx.x / args.kv_heads);
      if (run.x < 0) return;
      run.h = blockIdx.x % args.kv_heads;
      run.t = next_tile<kRows>(args, lengths, start, prefix, request_of<kRows>(args, start, run.x), run.x);
      run.step = 0;
      run.left = run.t.count;
      run.at = run.total = 0;
      if (run.t.count == 0) {
        put_nothing<kF32, kDim, kRows>(args, lengths, start, prefix, run.x, run.h, kThreads, out, lse);
        return;
      }
    } else {
      // workgroup b runs on XCD b % 8, which has neighbouring runs
      w = (blockIdx.x & 7) * (args.groups / 8) + (blockIdx.x >> 3);
      run = find_run<kThreads, kRows>(args, lengths, start, prefix, w, desk.deal);
      if (threadIdx.x == 0) parts_of<kDim>(args, workspace).cut[w].from = -1;
      if (run.nothing)
        for (int64_t i = w; i < (int64_t)args.tiles * args.kv_heads; i += args.groups)
          put_nothing<kF32, kDim, kRows>(args, lengths, start, prefix, (int32_t)(i / args.kv_heads), (int32_t)(i % args.kv_heads), kThreads,
                                         out, lse);
      if (run.left <= 0) return;
    }
    if (threadIdx.x == 0) {
      desk.a = args;
      desk.lengths = lengths;
      desk.start = start;
      desk.prefix = prefix;
      desk.out = out;
      desk.lse = lse;
      desk.workspace = workspace;
      desk.w = w;
      desk.run = run;
    }
  }
  while (true) {
    __syncthreads();
    Tile t;
    t.r = uniform(desk.run.t.r);
    t.n = uniform(desk.run.t.n);
    t.first = uniform(desk.run.t.first);
    t.fresh = uniform(desk.run.t.fresh);
    t.rows = uniform(desk.run.t.rows);
    t.row = uniform(desk.run.t.row);
    t.prefix = uniform(desk.run.t.prefix);
    t.head = uniform(desk.run.t.head);
    t.skip = uniform(desk.run.t.skip);
    const int32_t lo = uniform(desk.run.step), hi = uniform((int32_t)min((int64_t)desk.run.t.count, lo + desk.run.left));
    segment(desk.a, t, uniform(desk.run.h), lo, hi, [&](const auto& o, int tq, int hf, int32_t number, float m, float l) {
      const PromptArgs& a = desk.a;
      const Run& run = desk.run;
      if (number >= run.t.rows) return;
      const int32_t h = run.h;
      if (run.step == 0 && run.t.count <= run.left) {
        const Row row = row_of(a, run.t, number);
        put_row<kF32, kDim>(a, o, tq, hf, h * a.group + row.head, row.token, m, l, desk.out, desk.lse);
      } else {
        const int64_t slot = (int64_t)(2 * desk.w + (run.step == 0 ? 1 : 0)) * a.slot_rows;
        put_part<kDim>(parts_of<kDim>(a, desk.workspace), o, tq, hf, slot + (number - run.t.row), m, l);
      }
    });
    Run run = desk.run;
    if (run.step == 0 && run.t.count > run.left && threadIdx.x == 0)
      parts_of<kDim>(desk.a, desk.workspace).cut[desk.w] =
          Cut{run.t.row, min(run.t.rows - run.t.row, kRows), run.t.first, run.h, desk.w, run_of(desk.a, run.total, run.at + (run.t.count - 1))};
    const int32_t steps = (int32_t)min((int64_t)(run.t.count - run.step), run.left);
    if (run.left == steps) return;  // the whole workgroup
    run.left -= steps;
    run.at += steps;
    next_of<kRows>(desk.a, desk.lengths, desk.start, desk.prefix, run);
    __syncthreads();
    if (!uniform(run.left > 0)) return;
    if (threadIdx.x == 0) desk.run = run;
  }
}

// 64 entries of the request's row of the table, one a lane.
struct Entries {
  int32_t base, page;
};
// Entries i and i + 1 are among them afterwards.
__device__ inline void reach(const PromptArgs& a, const int32_t* __restrict__ row, int32_t n, int32_t i, Entries& e) {
  if ((uint32_t)(i - e.base) >= 63u) {
    e.base = i;
    const int32_t j = i + (threadIdx.x & 63);
    e.page = (int64_t)j * a.page.size < n ? row[j] : -1;
    e.page = (uint32_t)e.page < (uint32_t)a.pages ? e.page : -1;
    asm volatile("" : "+v"(e.page));  // waited for here, not at every use
  }
}

// ------------------------------------------------------------------ fp32 products

// Four waves of 32 rows, one step after the other, keys asked for a step ahead: the matrix
// cores' fp32 products take 64 cycles each, 64 to 128 a step. 1044 tokens of 16 heads of 64: 65
// us with the join, 23 of it around the steps.
constexpr int kThreadsF32 = 256;
template <int kDim, bool kScored>
__global__ __launch_bounds__(kThreadsF32) void prompt_f32_kernel(
    const char* __restrict__ q, const char* __restrict__ k, const char* __restrict__ v, const int32_t* __restrict__ table,
    const int32_t* __restrict__ lengths, const int32_t* __restrict__ start, const int32_t* __restrict__ prefix, char* __restrict__ out,
    float* __restrict__ lse, void* __restrict__ workspace, PromptArgs a) {
  constexpr int kRows = 128, kThreads = kThreadsF32, kC = kDim / 32, kRow = kDim * 4 + 16;
  __shared__ __attribute__((aligned(1024))) char lds_k[kKeys * kRow];
  __shared__ __attribute__((aligned(1024))) char lds_v[kKeys * kRow];
  __shared__ Desk<kThreads> desk;
  const int lane = threadIdx.x & 63, wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
  const int l32 = lane & 31, hf = lane >> 5;
  work<true, kDim, kRows, kThreads>(a, lengths, start, prefix, out, lse, workspace, desk, [&](const PromptArgs& b, const Tile& t, int h, int32_t lo, int32_t hi, auto done) {
    const int32_t number = t.row + wave * 32 + l32;
    const Row row = row_of(b, t, number);
    const int head = h * b.group + row.head;
    const float slope = kScored && b.slopes ? b.slopes[head] * kLog2e : 0.0f;
    const char* from = q + (head * b.q_head + row.token * b.q_token) * 4;
    u32x4 qw[kDim / 8];  // dimensions kDim / 2 hf + 4i ..
#pragma unroll
    for (int i = 0; i < kDim / 8; ++i) qw[i] = *reinterpret_cast<const u32x4*>(from + kDim * 2 * hf + 16 * i);
    f32x16 o[kC][1];  // register e of o[c]: dimension 32c + 8 (e / 4) + 4 hf + e % 4 of the row
#pragma unroll
    for (int c = 0; c < kC; ++c)
#pragma unroll
      for (int e = 0; e < 16; ++e) o[c][0][e] = 0.0f;
    float m = -INFINITY, l = 0.0f;

    // a step's keys are asked for while the one before is worked on
    constexpr int kPieces = kDim / 4, kEach = kKeys * kPieces / kThreads;
    u32x4 kw[kEach], vw[kEach];
    uint32_t next_absent = 0;  // bit u: keys 16u .. 16u + 15 have no page
    const auto base_of = [&](int32_t x) { return (x < t.head ? x : x + t.skip) * kKeys; };
    Entries entries{0x7fffffff - 64, -1};  // none yet
    const auto fetch = [&](int32_t base) {
      int32_t page[2];
      next_absent = 0;
      reach(a, table + (int64_t)t.r * a.max_pages, t.n, div_page(a.page, base), entries);
#pragma unroll
      for (int u = 0; u < 2; ++u) {
        const int32_t j = base + 16 * u;
        const int32_t entry = __builtin_amdgcn_readlane(entries.page, div_page(a.page, j) - entries.base);
        page[u] = j < t.n ? entry : -1;
        if (page[u] < 0) next_absent |= 1u << u;
      }
#pragma unroll
      for (int i = 0; i < kEach; ++i) {
        const int id = threadIdx.x + i * kThreads, key = id / kPieces, piece = id % kPieces;
        const int32_t j = base + key;
        kw[i] = vw[i] = u32x4{0, 0, 0, 0};
        if (j < t.n && !(next_absent >> (key >> 4) & 1u)) {
          const int64_t pg = key < 16 ? page[0] : page[1];
          const int32_t in = j - div_page(a.page, j) * a.page.size;
          const int64_t at = pg * a.page_stride + h * a.head_stride + (int64_t)in * a.token_stride + 16 * piece;
          kw[i] = *reinterpret_cast<const u32x4*>(k + at);
          vw[i] = *reinterpret_cast<const u32x4*>(v + at);
        }
      }
    };
    fetch(base_of(lo));
    for (int32_t x = lo; x < hi; ++x) {
      const int32_t base = base_of(x);
      const uint32_t absent = next_absent;
      __syncthreads();
#pragma unroll
      for (int i = 0; i < kEach; ++i) {
        const int id = threadIdx.x + i * kThreads, at = id / kPieces * kRow + 16 * (id % kPieces);
        *reinterpret_cast<u32x4*>(lds_k + at) = kw[i];
        *reinterpret_cast<u32x4*>(lds_v + at) = vw[i];
      }
      __syncthreads();
      if (x + 1 < hi) fetch(base_of(x + 1));
      f32x16 z = {};
#pragma unroll
      for (int i = 0; i < kDim / 8; ++i) {
        const f32x4 kw = *reinterpret_cast<const f32x4*>(lds_k + l32 * kRow + kDim * 2 * hf + 16 * i);
        const f32x4 qf = __builtin_bit_cast(f32x4, qw[i]);
#pragma unroll
        for (int e = 0; e < 4; ++e) z = __builtin_amdgcn_mfma_f32_32x32x2f32(kw[e], qf[e], z, 0, 0, 0);
      }
      float top = -INFINITY;
#pragma unroll
      for (int e = 0; e < 16; ++e) {
        const int key = 8 * (e >> 2) + 4 * hf + (e & 3);
        const int32_t j = base + key;
        float y = z[e];
        if constexpr (kScored) {
          y = a.cap_in != 0.0f ? a.cap_out * tanh_of(y * a.cap_in) : y * a.scale_log2;
          y = fmaf(-slope, fabsf((float)(row.place - j)), y);
        } else {
          y *= a.scale_log2;
        }
        const bool keep = (j < row.below || (j >= row.from && j <= row.place)) && !(absent >> (key >> 4) & 1u);
        z[e] = keep ? y : -INFINITY;
        top = fmaxf(top, z[e]);
      }
      const float to = fmaxf(m, pair_max(top));
      const float f = to == -INFINITY ? 1.0f : __builtin_amdgcn_exp2f(m - to), mm = to == -INFINITY ? 0.0f : to;
      m = to;
      l *= f;
#pragma unroll
      for (int c = 0; c < kC; ++c) o[c][0] *= f;
#pragma unroll
      for (int e = 0; e < 16; ++e) {
        z[e] = __builtin_amdgcn_exp2f(z[e] - mm);
        l += z[e];
      }
#pragma unroll
      for (int e = 0; e < 16; ++e)
#pragma unroll
        for (int c = 0; c < kC; ++c) {
          const float vw = *reinterpret_cast<const float*>(lds_v + (8 * (e >> 2) + 4 * hf + (e & 3)) * kRow + (32 * c + l32) * 4);
          o[c][0] = __builtin_amdgcn_mfma_f32_32x32x2f32(vw, z[e], o[c][0], 0, 0, 0);
        }
    }
    done(o, 0, hf, number, m, pair_sum(l));
  });
}

// ------------------------------------------------ bf16 products, in a pipeline

typedef __attribute__((address_space(3))) void lds_void;
typedef __attribute__((address_space(3))) char lds_char;
typedef __attribute__((address_space(3))) const bf16x8 lds_bf16x8;
typedef __attribute__((address_space(3))) u32x4 lds_u32x4;

constexpr int kRing = 4;  // buffers of K and of V
constexpr uint32_t kRsrcWord3 = 0x00020000u;  // a buffer of raw 32-bit data
// Offsets in a page are below 2^30: kOutside and 128 bytes on lie past the extent, where
// reads give zeros.
constexpr uint32_t kExtent = 0x7fffffffu, kOutside = 0x80000000u;

// Where 32 keys lie: their places in the sequence, and of the 16 that a wave brings in
// (of each 16, where it brings in some of both) the bytes to the first one's row of the
// head and, for exponents, its number among all tokens of all heads.
template <int kType, int kDim>
struct Spot {
  static constexpr int kParts = kType != 1 && kDim == 128 ? 2 : 1;
  int32_t base;
  uint32_t absent;  // bit u: keys 16u .. 16u + 15 have no page
  int64_t at[kParts], token[kParts];
};

// A thread's share of 32 keys in 8 or 4 bits between the pages and LDS: pieces of 8 values.
template <int kType, int kDim>
struct Raw {
  static constexpr int kEach = kDim / 64;  // of K and of V
  uint32_t k[kEach][2], v[kEach][2];       // 4 bits: the first word
  uint32_t ke[kEach], ve[kEach];
};

struct Limits {
  int32_t place, below, from;
  int32_t lost;  // see Rows::again
};

// A weight is 2^(z scale - m) with the product unrounded and m its rounded maximum: from here on
// the rounding is a power of two and more, as much as that of the scores themselves.
constexpr float kFarMaximum = 16777216.0f;

// kScored: 0 as they are, 1 lowered by the distance, 2 capped (and lowered).
template <int kDim, int kScored>
struct Rows {
  static constexpr int kC = kDim / 32, kS = kDim / 16;
  bf16x8 q[2][kS];      // Q^T as the B operand: dimensions 16 s + 8 hf .. of row 32 tq + l32
  f32x16 o[kC][2];      // register e: dimension 32 c + 8 (e / 4) + 4 hf + e % 4
  float nm[2], l[2];    // minus the running maximum (log2), this lane's share of the sum
  float slope[2];       // of the row's head
  int32_t place[2];     // changed scores: the row's place
  // Lane parts of LDS addresses, of a panel. An empty asm defines them anew at each use, so
  // that a buffer's own address goes into the instruction's offset and not, added to
  // each part, into a register of its own for each of eight buffers.
  int kpart[4], vpart[2][2];

  __device__ __forceinline__ void read_k(lds_char* b, bf16x8 (&x)[kS]) {
#pragma unroll
    for (int s = 0; s < 4; ++s) asm volatile("" : "+v"(kpart[s]));
#pragma unroll
    for (int s = 0; s < kS; ++s) x[s] = *(lds_bf16x8*)(b + 4096 * (s >> 2) + kpart[s & 3]);
  }
  __device__ __forceinline__ void read_v(lds_char* b, bf16x8 (&x)[2][kC]) {
#pragma unroll
    for (int c = 0; c < 2; ++c)
#pragma unroll
      for (int r = 0; r < 2; ++r) asm volatile("" : "+v"(vpart[c][r]));
#pragma unroll
    for (int u = 0; u < 2; ++u)
#pragma unroll
      for (int c = 0; c < kC; ++c) {
        lds_char* const at = b + 4096 * (c >> 1) + 2048 * u;
        const bf16x4 lo = __builtin_amdgcn_ds_read_tr16_b64_v4bf16((lds_bf16x4*)(at + vpart[c & 1][0]));
        const bf16x4 hi = __builtin_amdgcn_ds_read_tr16_b64_v4bf16((lds_bf16x4*)(at + vpart[c & 1][1]));
        x[u][c] = bf16x8{lo[0], lo[1], lo[2], lo[3], hi[0], hi[1], hi[2], hi[3]};
      }
  }
  __device__ __forceinline__ void mfma_s(const bf16x8 (&x)[kS], f32x16 (&z)[2]) const {
    f32x16 z0 = {}, z1 = {};
#pragma unroll
    for (int s = 0; s < kS; ++s) {
      z0 = __builtin_amdgcn_mfma_f32_32x32x16_bf16(x[s], q[0][s], z0, 0, 0, 0);
      z1 = __builtin_amdgcn_mfma_f32_32x32x16_bf16(x[s], q[1][s], z1, 0, 0, 0);
    }
    z[0] = z0;
    z[1] = z1;
  }
  __device__ __forceinline__ void mfma_pv(const bf16x8 (&x)[2][kC], const bf16x8 (&p)[2][2]) {
#pragma unroll
    for (int u = 0; u < 2; ++u)
#pragma unroll
      for (int c = 0; c < kC; ++c)
#pragma unroll
        for (int tq = 0; tq < 2; ++tq) o[c][tq] = __builtin_amdgcn_mfma_f32_32x32x16_bf16(x[u][c], p[u][tq], o[c][tq], 0, 0, 0);
  }
  // A score in log2 units, capped and lowered; far: the distance to the lane's first key.
  __device__ __forceinline__ float lowered(float z, int tq, int e, float far) const {
    return fmaf(-slope[tq], fabsf(far - (float)(8 * (e >> 2) + (e & 3))), z);
  }
  __device__ __forceinline__ float change(const PromptArgs& a, float z, int tq, int e, float far) const {
    return lowered(kScored == 2 ? a.cap_out * tanh_of(z * a.cap_in) : z * a.scale_log2, tq, e, far);
  }
  // The cap as cap - 2 cap / (1 + e^2y): five vector instructions' time less than the above, off
  // by 5 2^-24 of the cap. At a cap of 2048 and below that is less than 2^-10, where the weights'
  // own rounding is 2^-8 of each; beyond, scores are changed by the above ahead of the products.
  // So they are where the factor below would be infinite, and a score of 0 times it no number.
  __device__ __forceinline__ float capped(const PromptArgs& a, float z) const {
    const float t = __builtin_amdgcn_exp2f(z * (a.cap_in * kTwoLog2e));
    return fmaf(-2.0f * a.cap_out, __builtin_amdgcn_rcpf(1.0f + t), a.cap_out);
  }
  __device__ __forceinline__ float far_of(int tq, int32_t base, int hf) const { return (float)(place[tq] - base - 4 * hf); }
  // Of the wave's rows what each sees, from LDS: needed at the borders only.
  __device__ __forceinline__ void mask(f32x16 (&z)[2], int32_t base, int lane, uint32_t absent, const Limits* of) const {
#pragma unroll
    for (int tq = 0; tq < 2; ++tq) {
      const Limits y = of[32 * tq + (lane & 31)];
      const int32_t at = base + 4 * (lane >> 5);
#pragma unroll
      for (int e = 0; e < 16; ++e) {
        const int32_t j = at + 8 * (e >> 2) + (e & 3);
        const bool keep = (j < y.below || (j >= y.from && j <= y.place)) && !(absent >> (e >> 3) & 1u);
        z[tq][e] = keep ? z[tq][e] : -INFINITY;
      }
    }
  }
  // P = 2^(z scale - m) with the running maximum as it stands, rounded to bf16 for the
  // product: an output is off by up to 2^-8 more. The sum is that of the weights in fp32, for
  // the lse's sake (that of the rounded ones took half the instructions and put 1e-4 on it).
  __device__ __forceinline__ static bf16x2 pair(float z0, float z1, float sc, float nmu, float& sum) {
    const float x = __builtin_amdgcn_exp2f(fmaf(z0, sc, nmu)), y = __builtin_amdgcn_exp2f(fmaf(z1, sc, nmu));
    sum += x;
    sum += y;
    return bf16x2{(__bf16)x, (__bf16)y};
  }
  // kAgain: from a maximum of 2^24 on scores are scaled first, so that the largest one's weight is 1.
  template <bool kAgain>
  __device__ __forceinline__ void weights(const f32x16 (&z)[2], const float (&nmu)[2], float sc, bf16x8 (&p)[2][2], float (&sum)[2]) const {
#pragma unroll
    for (int tq = 0; tq < 2; ++tq) {
      sum[tq] = 0.0f;
      const bool far = kAgain && fabsf(nmu[tq]) >= kFarMaximum;
      const float by = far ? sc : 1.0f, then = far ? 1.0f : sc;
#pragma unroll
      for (int u = 0; u < 2; ++u) {
        bf16x2 x[4];
#pragma unroll
        for (int e = 0; e < 4; ++e) {
          const float z0 = z[tq][8 * u + 2 * e], z1 = z[tq][8 * u + 2 * e + 1];
          x[e] = pair(kAgain ? z0 * by : z0, kAgain ? z1 * by : z1, kAgain ? then : sc, nmu[tq], sum[tq]);
        }
        p[u][tq] = bf16x8{x[0][0], x[0][1], x[1][0], x[1][1], x[2][0], x[2][1], x[3][0], x[3][1]};
      }
    }
  }

  // A step's work in one order: each product followed by its share of the softmax of the
  // present scores, so that the matrix cores and the vector unit work side by side; the
  // operands come from LDS two pairs of products ahead. (The compiler, left to itself or given
  // groups to interleave, puts the products of the wider form in a row: 1390 us for 10992
  // tokens at once, 1117 so, both without what the step does beside.)
  template <typename Beside>
  __device__ __forceinline__ void fused(const PromptArgs& a, lds_char* kb, lds_char* vb, const bf16x8 (&p)[2][2], float sc, bool changed, int32_t base, int hf,
                                        f32x16 (&z)[2], f32x16 (&next)[2], bf16x8 (&pn)[2][2], float (&sum)[2], Beside beside) {
    constexpr int kProducts = 2 * kS + 4 * kC, kEach = 32 / kProducts;  // scores a product
#if defined(__HIP_DEVICE_COMPILE__)
    if constexpr (kDim == 128) {  // Q in accumulation registers, where the products read it as well
#pragma unroll
      for (int tq = 0; tq < 2; ++tq)
#pragma unroll
        for (int s = 0; s < kS; ++s) asm("" : "+a"(q[tq][s]));
    }
#endif
#pragma unroll
    for (int s = 0; s < 4; ++s) asm volatile("" : "+v"(kpart[s]));
#pragma unroll
    for (int c = 0; c < 2; ++c)
#pragma unroll
      for (int r = 0; r < 2; ++r) asm volatile("" : "+v"(vpart[c][r]));
    bf16x8 kw[kS], vw[2 * kC];
    const auto get_k = [&](int s) { kw[s] = *(lds_bf16x8*)(kb + 4096 * (s >> 2) + kpart[s & 3]); };
    const auto get_v = [&](int i) {
      const int c = i % kC, u = i / kC;
      lds_char* const at = vb + 4096 * (c >> 1) + 2048 * u;
      const bf16x4 lo = __builtin_amdgcn_ds_read_tr16_b64_v4bf16((lds_bf16x4*)(at + vpart[c & 1][0]));
      const bf16x4 hi = __builtin_amdgcn_ds_read_tr16_b64_v4bf16((lds_bf16x4*)(at + vpart[c & 1][1]));
      vw[i] = bf16x8{lo[0], lo[1], lo[2], lo[3], hi[0], hi[1], hi[2], hi[3]};
    };
    float far[2];
    if constexpr (kScored) {
      far[0] = far_of(0, base, hf);
      far[1] = far_of(1, base, hf);
      asm volatile("" : "+v"(far[0]), "+v"(far[1]));  // or 32 distances are taken ahead of the branch before this
    }
    // scores that are changed already: lowered by nothing
    const float scale = changed ? 1.0f : a.scale_log2, by[2] = {changed ? 0.0f : slope[0], changed ? 0.0f : slope[1]};
    bf16x2 x[2][8];
    float even;  // a pair's first weight
    sum[0] = sum[1] = 0.0f;
    const auto share = [&](int product) {
#pragma unroll
      for (int i = 0; i < kEach; ++i) {
        const int n = product * kEach + i, tq = n >> 4, e = n & 15;
        if constexpr (kScored == 1) z[tq][e] = fmaf(-by[tq], fabsf(far[tq] - (float)(8 * (e >> 2) + (e & 3))), z[tq][e] * scale);
        if constexpr (kScored == 2) {
          const float y = lowered(capped(a, z[tq][e]), tq, e, far[tq]);
          z[tq][e] = changed ? z[tq][e] : y;
        }
        const float y = __builtin_amdgcn_exp2f(fmaf(z[tq][e], sc, nm[tq]));
        sum[tq] += y;
        if (e & 1) x[tq][e >> 1] = bf16x2{(__bf16)even, (__bf16)y};
        even = y;
      }
      beside(product);
      __builtin_amdgcn_sched_barrier(0);
    };
    constexpr int kLead = 2;
#pragma unroll
    for (int s = 0; s < kLead; ++s) get_k(s);
    __builtin_amdgcn_sched_barrier(0);
#pragma unroll
    for (int s = 0; s < kS; ++s) {
      if (s + kLead < kS) get_k(s + kLead);
      else get_v(s + kLead - kS);
#pragma unroll
      for (int tq = 0; tq < 2; ++tq) {
        const f32x16 none = {};
        next[tq] = __builtin_amdgcn_mfma_f32_32x32x16_bf16(kw[s], q[tq][s], s == 0 ? none : next[tq], 0, 0, 0);
        share(2 * s + tq);
      }
    }
#pragma unroll
    for (int i = 0; i < 2 * kC; ++i) {
      if (i + kLead < 2 * kC) get_v(i + kLead);
#pragma unroll
      for (int tq = 0; tq < 2; ++tq) {
        o[i % kC][tq] = __builtin_amdgcn_mfma_f32_32x32x16_bf16(vw[i], p[i / kC][tq], o[i % kC][tq], 0, 0, 0);
        share(2 * kS + 2 * i + tq);
      }
    }
#pragma unroll
    for (int u = 0; u < 2; ++u)
#pragma unroll
      for (int tq = 0; tq < 2; ++tq) {
        const bf16x2 (&y)[8] = x[tq];
        pn[u][tq] = bf16x8{y[4 * u][0],     y[4 * u][1],     y[4 * u + 1][0], y[4 * u + 1][1],
                           y[4 * u + 2][0], y[4 * u + 2][1], y[4 * u + 3][0], y[4 * u + 3][1]};
      }
  }
  // The maximum moves only where a row's sum leaves [0, 2^12]: at its first key, where the
  // maximum is still none and the sum infinite or NaN, and where scores grew by much. A
  // row without a key so far keeps m = -inf and weights of 0; a row whose sum is in order
  // keeps its maximum, whatever the others of the wave do. kAgain: a lost row's follows every score.
  template <bool kAgain = false>
  __device__ __forceinline__ void settle(const f32x16 (&z)[2], float sc, bf16x8 (&p)[2][2], float (&sum)[2], int l32 = 0, const Limits* of = nullptr) {
    if (kAgain || __ballot(__float_as_uint(sum[0]) > 0x45800000u || __float_as_uint(sum[1]) > 0x45800000u)) {
      float use[2];
#pragma unroll
      for (int tq = 0; tq < 2; ++tq) {
        const auto both = __builtin_amdgcn_permlane32_swap(__float_as_uint(sum[tq]), __float_as_uint(sum[tq]), false, false);
        const bool moves = max((uint32_t)both[0], (uint32_t)both[1]) > 0x45800000u || (kAgain && of[32 * tq + l32].lost);
        float top = z[tq][0];
        asm volatile("" : "+v"(top));  // the maximum is taken here only, not ahead of the branch
#pragma unroll
        for (int e = 1; e < 16; ++e) top = fmaxf(top, z[tq][e]);
        const float to = moves ? fminf(-(pair_max(top) * sc), nm[tq]) : nm[tq];
        const float f = to == INFINITY ? 1.0f : __builtin_amdgcn_exp2f(to - nm[tq]);
        nm[tq] = to;
        use[tq] = to == INFINITY ? 0.0f : to;
        l[tq] *= f;
        if constexpr (kAgain) asm volatile("" : "+v"(l[tq]));  // rounded here, as behind the branch elsewhere
#pragma unroll
        for (int c = 0; c < kC; ++c) o[c][tq] *= f;
      }
      weights<kAgain>(z, use, sc, p, sum);
    }
    l[0] += sum[0];
    l[1] += sum[1];
  }
  __device__ __forceinline__ void clear() {
#pragma unroll
    for (int tq = 0; tq < 2; ++tq) {
      nm[tq] = INFINITY;
      l[tq] = 0.0f;
#pragma unroll
      for (int c = 0; c < kC; ++c)
#pragma unroll
        for (int e = 0; e < 16; ++e) o[c][tq][e] = 0.0f;
    }
  }
  // Whether a row's weights, or their products with V, may have left the exponent's range: the
  // maximum is far, or sums are no numbers. A row without a key has neither.
  __device__ __forceinline__ bool is_lost(int tq) const {
    float none = l[tq] * 0.0f;
#pragma unroll
    for (int c = 0; c < kC; ++c)
#pragma unroll
      for (int e = 0; e < 16; ++e) none = fmaf(o[c][tq][e], 0.0f, none);
    return none != 0.0f || (kScored == 0 && fabsf(nm[tq]) >= kFarMaximum && nm[tq] < INFINITY);
  }
  // Lost rows are noted; all sums from the start.
  __device__ __forceinline__ void again(int l32, Limits* of) {
#pragma unroll
    for (int tq = 0; tq < 2; ++tq)
      if (is_lost(tq)) of[32 * tq + l32].lost = 1;  // by either of its lanes
    clear();
  }
};

// Four waves of 64 rows each. Step t issues S^T of keys t + 1 and the product with V of
// keys t - 1 on the matrix cores while the vector unit runs the softmax of keys t.
// K and V lie in rings of four buffers each, K of keys x in buffer x % 4, V likewise; right
// after a step's barrier what step t - 1 read is filled again (K t + 4, V t + 2),
// three steps before it is read. In 8 and 4 bits a step writes K t + 2 and V t, which were
// asked for one step before, or four. 64 rows a wave: with 32 the LDS reads of K and V
// alone would take as long as the products. 10992 tokens at once, 32 heads on 8 of 128 in
// bf16: 989 us, 1002 TFLOP/s, where a library product reaches 1199; a step's 32 products
// take 1024 of about 2400 cycles. 8 frames of 1374 tokens over 10992, 16 heads of 64: in 8
// bits 844 us, 660 TFLOP/s, bound by what goes beside a step's 16 products (156 vector and 107
// scalar instructions: softmax, codes to bf16, lookups and addresses); in bf16 732, 760 TFLOP/s.
constexpr int kWaves = 4;
template <int kType, int kDim, int kScored>
__global__ __launch_bounds__(64 * kWaves) __attribute__((amdgpu_waves_per_eu(kDim == 64 ? 2 : 1, kDim == 64 ? 2 : 1))) void
prompt_bf16_kernel(const char* __restrict__ q, const char* __restrict__ k, const char* __restrict__ v,
                   const uint8_t* __restrict__ k_exp, const uint8_t* __restrict__ v_exp, const int32_t* __restrict__ table,
                   const int32_t* __restrict__ lengths, const int32_t* __restrict__ start, const int32_t* __restrict__ prefix,
                   char* __restrict__ out, float* __restrict__ lse, void* __restrict__ workspace, PromptArgs a) {
  constexpr int kThreads = 64 * kWaves, kBytes = kKeys * kDim * 2, kRows = 64 * kWaves, kPanels = kDim / 64;
  // written by the waves themselves there are never more than two in use
  constexpr int kLong = kType == 1 ? kBytes : 16;
  __shared__ __attribute__((aligned(1024))) char k0[kBytes], k1[kBytes], k2[kLong], k3[kLong];
  __shared__ __attribute__((aligned(1024))) char v0[kBytes], v1[kBytes], v2[kLong], v3[kLong];
  __shared__ Desk<kThreads> desk;
  __shared__ Limits limits[kRows];  // read by the waves that write them, behind a barrier
  lds_char* const kring[kRing] = {(lds_char*)k0, (lds_char*)k1, (lds_char*)(kType == 1 ? k2 : k0), (lds_char*)(kType == 1 ? k3 : k1)};
  lds_char* const vring[kRing] = {(lds_char*)v0, (lds_char*)v1, (lds_char*)(kType == 1 ? v2 : v0), (lds_char*)(kType == 1 ? v3 : v1)};
  const int lane = threadIdx.x & 63, wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
  const int l32 = lane & 31, hf = lane >> 5;
  const float sc = kScored ? 1.0f : a.scale_log2;

  work<false, kDim, kRows, kThreads>(a, lengths, start, prefix, out, lse, workspace, desk, [&](const PromptArgs& b, const Tile& t, int h, int32_t lo, int32_t hi, auto done) {
  using W = Rows<kDim, kScored>;
  W w;
#pragma unroll
  for (int tq = 0; tq < 2; ++tq) {
    const Row row = row_of(b, t, t.row + wave * 64 + tq * 32 + l32);
    const int head = h * b.group + row.head;
    w.slope[tq] = kScored && b.slopes ? b.slopes[head] * kLog2e : 0.0f;
    w.place[tq] = row.place;
    if (hf == 0) limits[wave * 64 + tq * 32 + l32] = Limits{row.place, row.below, row.from, 0};
    const char* from = q + (head * b.q_head + row.token * b.q_token) * 2;
#pragma unroll
    for (int s = 0; s < w.kS; ++s) w.q[tq][s] = *reinterpret_cast<const bf16x8*>(from + 32 * s + 16 * hf);
  }
  w.clear();
  const int tr_row = 4 * hf + ((lane & 15) >> 2), tr_col = 16 * ((lane >> 4) & 1) + 4 * (lane & 3);
#pragma unroll
  for (int s = 0; s < 4; ++s) w.kpart[s] = swz(l32, 2 * s + hf);
#pragma unroll
  for (int c = 0; c < 2; ++c)
#pragma unroll
    for (int r = 0; r < 2; ++r) w.vpart[c][r] = swz(tr_row + 8 * r, (32 * c + tr_col) >> 3) + (tr_col & 7) * 2;
  // keys that every row of the wave sees: those below all_below, and [all_from, all_place]
  int32_t all_below, all_from, all_place;
  {
    const Row low = row_of(b, t, t.row + wave * 64), high = row_of(b, t, t.row + wave * 64 + 63);
    all_below = __builtin_amdgcn_readfirstlane(low.below);
    all_from = __builtin_amdgcn_readfirstlane(high.from);
    all_place = __builtin_amdgcn_readfirstlane(low.place);
  }
  const auto is_whole = [&](int32_t base, uint32_t absent) {
    return absent == 0 && (base + kKeys <= all_below || (base >= all_from && base + kKeys - 1 <= all_place));
  };

  const int32_t* const entries_row = table + (int64_t)t.r * a.max_pages;
  Entries entries{0x7fffffff - 64, -1};  // none yet
  using Y = Spot<kType, kDim>;
  // Where keys x lie, in three pieces that a step has between its products.
  int32_t page_i, page_in;
  const auto base_of = [&](int32_t x) {
    x = min(x, hi - 1);
    return (x < t.head ? x : x + t.skip) * kKeys;
  };
  const auto locate_begin = [&](int32_t base, Y& y) {
    y.base = base;
    y.absent = 0;
    y.at[0] = y.token[0] = 0;
    page_i = div_page(a.page, base);
    page_in = base - page_i * a.page.size;
  };
  const auto locate_part = [&](int u, Y& y) {
    if (u == 1) {
      page_in += 16;
      const bool over = page_in == a.page.size;
      page_in = over ? 0 : page_in;
      page_i += over ? 1 : 0;
    }
    const int32_t entry = __builtin_amdgcn_readlane(entries.page, page_i - entries.base);
    const int32_t page = y.base + 16 * u < t.n ? entry : -1;
    y.absent |= (uint32_t)(page < 0) << u;
    // selected, not branched over: a branch would part the products
    const int64_t at = max(page, 0) * a.page_stride + h * a.head_stride + (int64_t)page_in * a.token_stride;
    const int64_t token = ((int64_t)max(page, 0) * a.kv_heads + h) * a.page.size + page_in;
    const bool mine = Y::kParts == 2 || u == wave >> 1;
    y.at[u % Y::kParts] = mine ? at : y.at[u % Y::kParts];
    y.token[u % Y::kParts] = mine ? token : y.token[u % Y::kParts];
  };
  const auto locate = [&](int32_t x) {
    Y y;
    const int32_t base = base_of(x);
    reach(a, entries_row, t.n, div_page(a.page, base), entries);
    locate_begin(base, y);
    locate_part(0, y);
    locate_part(1, y);
    return y;
  };
  // bf16: memory to LDS directly, a KB an instruction: 8 rows of a panel
  const auto dma = [&](const char* from, const Y& y, lds_char* buf) {
    const int u = wave >> 1, row = 8 * (wave & 1) + (lane >> 3);  // of the 16 keys of u
    const auto r = __builtin_amdgcn_make_buffer_rsrc(const_cast<char*>(from + y.at[0]), (short)0, (int)kExtent, (int)kRsrcWord3);
    const bool there = !(y.absent >> u & 1u) && y.base + 16 * u + row < t.n;
    const uint32_t off = there ? (uint32_t)(row * a.token_stride + 16 * ((lane & 7) ^ swz_f(row))) : kOutside;
#pragma unroll
    for (int p = 0; p < kPanels; ++p)
      __builtin_amdgcn_raw_ptr_buffer_load_lds(r, (lds_void*)(buf + 4096 * p + 1024 * wave), 16, (int)(off + 128 * p), 0, 0, 0);
  };
  // others: through registers, where they become bf16
  using R = Raw<kType, kDim>;
  constexpr int kPieces = kDim / 8, kPieceBytes = kType == 2 ? 8 : 4, kBlocks = kType == 2 ? 1 : kDim / kExpBlock;
  // a thread takes one piece of rows kStep apart
  constexpr int kStep = kThreads / kPieces;
  const int piece = threadIdx.x % kPieces, piece_row = threadIdx.x / kPieces;
  const auto fetch = [&](const char* from, const uint8_t* exp, const Y& y, uint32_t (&to)[R::kEach][2], uint32_t (&e)[R::kEach]) {
#pragma unroll
    for (int i = 0; i < R::kEach; ++i) {
      const int u = R::kEach == 1 ? wave >> 1 : i * kStep / 16;  // the 16 keys of the wave's
      const int row = R::kEach == 1 ? piece_row & 15 : piece_row + i * kStep - 16 * u;
      const int part = Y::kParts == 1 ? 0 : u;
      const auto r = __builtin_amdgcn_make_buffer_rsrc(const_cast<char*>(from + y.at[part]), (short)0, (int)kExtent, (int)kRsrcWord3);
      const auto re = __builtin_amdgcn_make_buffer_rsrc(const_cast<uint8_t*>(exp + y.token[part] * kBlocks), (short)0, (int)kExtent,
                                                        (int)kRsrcWord3);
      const bool there = !(y.absent >> u & 1u) && y.base + 16 * u + row < t.n;
      const uint32_t at = there ? (uint32_t)(row * a.token_stride + piece * kPieceBytes) : kOutside;
      if constexpr (kType == 2) {
        const u32x2 x = __builtin_bit_cast(u32x2, __builtin_amdgcn_raw_buffer_load_b64(r, (int)at, 0, 0));
        to[i][0] = x[0];
        to[i][1] = x[1];
      } else {
        to[i][0] = __builtin_amdgcn_raw_buffer_load_b32(r, (int)at, 0, 0);
      }
      const uint32_t of = there ? (uint32_t)(row * kBlocks + (kType == 2 ? 0 : piece / 4)) : kOutside;
      e[i] = __builtin_amdgcn_raw_buffer_load_b8(re, (int)of, 0, 0);
    }
  };
  const auto put = [&](const uint32_t (&x)[R::kEach][2], const uint32_t (&e)[R::kEach], lds_char* buf) {
#pragma unroll
    for (int i = 0; i < R::kEach; ++i) {
      const float scale = __uint_as_float(e[i] << 23);
      u32x4 y;
      if constexpr (kType == 2)
        y = u32x4{fp8_pair(x[i][0], false, scale), fp8_pair(x[i][0], true, scale), fp8_pair(x[i][1], false, scale),
                  fp8_pair(x[i][1], true, scale)};
      else
        y = u32x4{fp4_pair<0>(x[i][0], scale), fp4_pair<1>(x[i][0], scale), fp4_pair<2>(x[i][0], scale), fp4_pair<3>(x[i][0], scale)};
      *(lds_u32x4*)(buf + 4096 * (piece >> 3) + swz(piece_row + i * kStep, piece & 7)) = y;
    }
  };
  // what goes to LDS in this step and, at width 128, in the next three: there is one
  // workgroup on a CU there, and no other's work while a load is on its way
  constexpr int kAhead = kDim == 64 ? 1 : 4;
  R raw[kAhead];
  const auto fetch_both = [&](const Y& yk, const Y& yv, R& to) {
    fetch(k, k_exp, yk, to.k, to.ke);
    fetch(v, v_exp, yv, to.v, to.ve);
  };

  f32x16 z[2];
  bf16x8 p[2][2] = {};
  // the steps' keys from the present one on; what is asked for last in a step is that of K
  constexpr int kQueue = kType == 1 ? 5 : 3 + kAhead;
  Y spots[kQueue];
  constexpr int kLoads = 2 * kPanels;  // of a wave and step
  const auto sync = [&](auto all) {
    if constexpr (kType == 1)  // loads of three steps ago and before, all LDS reads
      __builtin_amdgcn_s_waitcnt(decltype(all)::value ? 0x0070 : 0x0070 | (2 * kLoads));
    else
      __builtin_amdgcn_s_waitcnt(0xC07F);
    asm volatile("s_barrier" ::: "memory");
  };

  if (lo < hi) {
#pragma unroll
    for (int x = 0; x < kQueue - 1; ++x) spots[x + 1] = locate(lo + x);
    // V of keys -1: any that is finite, its weights are 0
    if constexpr (kType == 1) {
#pragma unroll
      for (int x = 0; x < kRing; ++x) dma(k, spots[x + 1], kring[x]);
      dma(v, spots[1], vring[3]);
      dma(v, spots[1], vring[0]);
      dma(v, spots[2], vring[1]);
    } else {
      R r[2];
      fetch_both(spots[1], spots[1], r[0]);
      fetch_both(spots[2], spots[2], r[1]);
#pragma unroll
      for (int x = 0; x < kAhead; ++x) fetch_both(spots[x + 3 < kQueue ? x + 3 : kQueue - 1], spots[x + 1], raw[x]);
      put(r[0].k, r[0].ke, kring[0]);
      put(r[1].k, r[1].ke, kring[1]);
      put(r[0].v, r[0].ve, vring[3]);
    }
    sync(std::true_type{});
    {
      bf16x8 kw[W::kS];
      w.read_k(kring[0], kw);
      w.mfma_s(kw, z);
    }
    // step x, its place in the rings P
    const auto step = [&](auto place, int32_t x) {
      constexpr int P = decltype(place)::value;
      sync(std::false_type{});
      const int32_t base = spots[1].base;
      const uint32_t absent = spots[1].absent;
      const int32_t new_base = base_of(x + kQueue - 1);
      reach(a, entries_row, t.n, div_page(a.page, new_base), entries);
      // the step's other work, behind its products: a wave has its SIMD, or half of it, for
      // itself, and what it does ahead of them the matrix cores wait for
      const auto beside = [&](int product) {
        if (product == 1) {
#pragma unroll
          for (int i = 0; i + 1 < kQueue; ++i) spots[i] = spots[i + 1];
          locate_begin(new_base, spots[kQueue - 1]);
        }
        if (product == 3) locate_part(0, spots[kQueue - 1]);
        if (product == 5) locate_part(1, spots[kQueue - 1]);
        if constexpr (kType == 1) {
          if (product == 7) dma(k, spots[4], kring[P]);
          if (product == 9) dma(v, spots[2], vring[(P + 2) & 3]);
        } else {
          R& r = raw[P % kAhead];
          if (product == 0) put(r.k, r.ke, kring[(P + 2) & 3]);
          if (product == 2) put(r.v, r.ve, vring[P]);
          if (product == 7) fetch(k, k_exp, spots[2 + kAhead], r.k, r.ke);
          if (product == 9) fetch(v, v_exp, spots[kAhead], r.v, r.ve);
        }
      };
      const bool whole = is_whole(base, absent);
      lds_char* const kb = kring[(P + 1) & 3];
      lds_char* const vb = vring[(P + 3) & 3];
      f32x16 next[2];
      bf16x8 pn[2][2];
      float sum[2];
      // A mask comes behind the scores' change: there the scores are changed ahead of the step's
      // work, elsewhere along with it.
      const bool changed = kScored && (!whole || (kScored == 2 && a.far_cap));
      if (changed) {
#pragma unroll
        for (int tq = 0; tq < 2; ++tq) {
          const float far = w.far_of(tq, base, hf);
#pragma unroll
          for (int e = 0; e < 16; ++e) z[tq][e] = w.change(a, z[tq][e], tq, e, far);
        }
      }
      if (!whole) w.mask(z, base, lane, absent, limits + wave * 64);
      w.fused(a, kb, vb, p, sc, changed, base, hf, z, next, pn, sum, beside);
      w.settle(z, sc, pn, sum);
#pragma unroll
      for (int u = 0; u < 2; ++u)
#pragma unroll
        for (int tq = 0; tq < 2; ++tq) p[u][tq] = pn[u][tq];
      z[0] = next[0];
      z[1] = next[1];
    };
    using P0 = std::integral_constant<int, 0>;
    using P1 = std::integral_constant<int, 1>;
    using P2 = std::integral_constant<int, 2>;
    using P3 = std::integral_constant<int, 3>;
    int32_t x = lo;
    for (; x + 4 <= hi; x += 4) {
      step(P0{}, x);
      step(P1{}, x + 1);
      step(P2{}, x + 2);
      step(P3{}, x + 3);
    }
    const int rest = hi - x;
    if (rest > 0) step(P0{}, x);
    if (rest > 1) step(P1{}, x + 1);
    if (rest > 2) step(P2{}, x + 2);
    sync(std::true_type{});
    // the last keys' V
    bf16x8 vw[2][W::kC];
    w.read_v(rest == 0 ? vring[3] : rest == 1 ? vring[0] : rest == 2 ? vring[1] : vring[2], vw);
    w.mfma_pv(vw, p);
  }
  // Lost rows take the plainest walk, one step after the other, in which their maximum follows
  // every score; the tile's others get the same bits again. (Far maxima told apart in each step's
  // settle: 827 -> 855 us for 8 frames.)
  if (__syncthreads_or(w.is_lost(0) || w.is_lost(1))) {
    w.again(l32, limits + wave * 64);
    for (int32_t x = lo; x < hi; ++x) {
      const Y y = locate(x);
      __syncthreads();
      if constexpr (kType == 1) {
        dma(k, y, kring[0]);
        dma(v, y, vring[0]);
      } else {
        R r;
        fetch_both(y, y, r);
        put(r.k, r.ke, kring[0]);
        put(r.v, r.ve, vring[0]);
      }
      sync(std::true_type{});
      bf16x8 kw[W::kS], vw[2][W::kC];
      w.read_k(kring[0], kw);
      w.mfma_s(kw, z);
      if constexpr (kScored) {
        const bool brief = kScored == 2 && !a.far_cap && is_whole(y.base, y.absent);
#pragma unroll
        for (int tq = 0; tq < 2; ++tq) {
          const float far = w.far_of(tq, y.base, hf);
          if (brief) {
#pragma unroll
            for (int e = 0; e < 16; ++e) z[tq][e] = w.lowered(w.capped(a, z[tq][e]), tq, e, far);
          } else {
#pragma unroll
            for (int e = 0; e < 16; ++e) z[tq][e] = w.change(a, z[tq][e], tq, e, far);
          }
        }
      }
      w.mask(z, y.base, lane, y.absent, limits + wave * 64);
      float sum[2];
      w.template weights<true>(z, w.nm, sc, p, sum);
      w.template settle<true>(z, sc, p, sum, l32, limits + wave * 64);
      w.read_v(vring[0], vw);
      w.mfma_pv(vw, p);
    }
  }

#pragma unroll
  for (int tq = 0; tq < 2; ++tq) done(w.o, tq, hf, t.row + wave * 64 + tq * 32 + l32, -w.nm[tq], pair_sum(w.l[tq]));
  });
}

// The tiles that fell to several workgroups, in the order of these: one workgroup for each
// join_rows rows, 16 bytes of sums a lane.
constexpr int kJoinThreads = 256;
constexpr int join_rows(int dim) { return kJoinThreads / (dim / 4); }
template <bool kF32, int kDim>
__global__ __launch_bounds__(kJoinThreads) void prompt_join_kernel(char* __restrict__ out, float* __restrict__ lse,
                                                                   void* __restrict__ workspace, PromptArgs a) {
  constexpr int kLanes = kDim / 4;
  const Parts p = parts_of<kDim>(a, workspace);
  const Cut cut = p.cut[blockIdx.x];
  if (cut.from < 0) return;
  const int row = blockIdx.y * join_rows(kDim) + threadIdx.x / kLanes, d = threadIdx.x % kLanes * 4;
  if (row >= cut.rows) return;
  float m = -INFINITY, l = 0.0f;
  f32x4 o = {0, 0, 0, 0};
  constexpr int kAtOnce = 8;  // parts asked for together
  for (int w0 = cut.from; w0 <= cut.to; w0 += kAtOnce) {
    float2 x[kAtOnce];
    f32x4 y[kAtOnce];
#pragma unroll
    for (int u = 0; u < kAtOnce; ++u) {
      const int w = min(w0 + u, cut.to);
      const int64_t at = (int64_t)(2 * w + (w == cut.from ? 1 : 0)) * a.slot_rows + row;
      x[u] = p.ml[at];
      y[u] = *reinterpret_cast<const f32x4*>(p.o + at * kDim + d);
    }
    float to = m;
#pragma unroll
    for (int u = 0; u < kAtOnce; ++u) to = fmaxf(to, x[u].x);
    const float f = to == -INFINITY ? 1.0f : __builtin_amdgcn_exp2f(m - to);
    o *= f;
    l *= f;
    m = to;
#pragma unroll
    for (int u = 0; u < kAtOnce; ++u) {
      const float g = w0 + u > cut.to ? 0.0f : to == -INFINITY ? 1.0f : __builtin_amdgcn_exp2f(x[u].x - to);
      if (w0 + u <= cut.to) o += y[u] * g;
      l = fmaf(x[u].y, g, l);
    }
  }
  o *= l > 0.0f ? 1.0f / l : l;
  const int32_t number = cut.row + row, i_token = number / a.group;
  const int head = cut.h * a.group + (number - i_token * a.group), token = cut.first + i_token;
  const int64_t at = head * a.out_head + token * a.out_token + d;
  if constexpr (kF32)
    *reinterpret_cast<f32x4*>(reinterpret_cast<float*>(out) + at) = o;
  else
    *reinterpret_cast<bf16x4*>(reinterpret_cast<__bf16*>(out) + at) = __builtin_convertvector(o, bf16x4);
  if (lse && d == 0) lse[(int64_t)head * a.tokens + token] = (m + __log2f(l)) * kLn2;
}

template <int kType, int kDim, int kScored>
hipError_t launch(const void* q, const void* kp, const void* vp, const uint8_t* ke, const uint8_t* ve, const int32_t* table,
                  const int32_t* lengths, const int32_t* start, const int32_t* prefix, void* out, float* lse, void* workspace,
                  const PromptArgs& a, hipStream_t s) {
  const dim3 grid(a.groups ? (unsigned)a.groups : (unsigned)(a.tiles < kTilesAcross ? a.tiles : kTilesAcross) * (unsigned)a.kv_heads,
                  a.groups ? 1u : (unsigned)((a.tiles + kTilesAcross - 1) / kTilesAcross));
  const char *qc = static_cast<const char*>(q), *kc = static_cast<const char*>(kp), *vc = static_cast<const char*>(vp);
  char* oc = static_cast<char*>(out);
  if constexpr (kType == 0)
    hipLaunchKernelGGL((prompt_f32_kernel<kDim, kScored != 0>), grid, dim3(kThreadsF32), 0, s, qc, kc, vc, table, lengths, start, prefix, oc,
                       lse, workspace, a);
  else
    hipLaunchKernelGGL((prompt_bf16_kernel<kType, kDim, kScored>), grid, dim3(64 * kWaves), 0, s, qc, kc, vc, ke, ve, table, lengths,
                       start, prefix, oc, lse, workspace, a);
  const hipError_t e = hipGetLastError();
  if (e != hipSuccess || a.groups == 0) return e;
  hipLaunchKernelGGL((prompt_join_kernel<kType == 0, kDim>), dim3((unsigned)a.groups, (unsigned)((a.slot_rows + join_rows(kDim) - 1) / join_rows(kDim))),
                     dim3(kJoinThreads), 0, s, oc, lse, workspace, a);
  return hipGetLastError();
}

}  // namespace

hipError_t launch_prompt_attention(int dtype, int dim, const void* q, const void* k_pages, const void* v_pages,
                                   const uint8_t* k_exp, const uint8_t* v_exp, const int32_t* table,
                                   const int32_t* lengths, const int32_t* start, const int32_t* prefix, void* out,
                                   float* lse, void* workspace, const PromptArgs& a, hipStream_t s) {
#define SAF3R_ARGS q, k_pages, v_pages, k_exp, v_exp, table, lengths, start, prefix, out, lse, workspace, a, s
#define SAF3R_CASE(T, D)                                                     \
  if (dtype == T && dim == D)                                                \
  return a.cap_in != 0.0f ? launch<T, D, 2>(SAF3R_ARGS) : a.slopes ? launch<T, D, 1>(SAF3R_ARGS) : launch<T, D, 0>(SAF3R_ARGS)
  SAF3R_CASE(0, 64);
  SAF3R_CASE(0, 128);
  SAF3R_CASE(1, 64);
  SAF3R_CASE(1, 128);
  SAF3R_CASE(2, 64);
  SAF3R_CASE(2, 128);
  SAF3R_CASE(4, 64);
  SAF3R_CASE(4, 128);
#undef SAF3R_ARGS
#undef SAF3R_CASE
  return hipErrorInvalidValue;
}

}  // namespace saf3r
