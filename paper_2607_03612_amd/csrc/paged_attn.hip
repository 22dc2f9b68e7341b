// Attention of one new token per request over a paged cache.
//
// For a key-value head the up to 16 query heads that share it are the columns of
// the matrix products, 16 keys of a page the rows:
//   S^T = K Q^T   (A = K, B = Q^T)      O^T += V^T P^T   (A = V^T, B = P^T)
// A lane of the 16x16 products holds, of S^T, the four keys 4g .. 4g + 3 (g = lane
// / 16) of query lane % 16. P^T is wanted with eight keys per lane for a product
// over 32: which keys share a lane is free as long as V^T has them in the same
// places, so two 16-key results side by side are P^T as they are, and no lane
// gives a weight to another. The same freedom lets every operand come from
// memory straight into its registers: K's rows in 16-byte pieces along the head
// (Q is laid out alike), V's rows with head_dim / 16 neighbouring dimensions per
// lane, transposed in the lane by byte permutes. No tile passes through LDS.
#include "paged_internal.h"

namespace saf3r {
namespace {

typedef __bf16 bf16x8 __attribute__((ext_vector_type(8)));
typedef __bf16 bf16x2 __attribute__((ext_vector_type(2)));
typedef float f32x4 __attribute__((ext_vector_type(4)));
typedef uint32_t u32x4 __attribute__((ext_vector_type(4)));
typedef uint32_t u32x2 __attribute__((ext_vector_type(2)));

constexpr int kThreads = 256;
constexpr int kCuCount = 256;
// Waves of a launch, two to a SIMD: every wave takes the same number of tiles, at
// least kMinTiles, so that a short launch does not spend itself on joining.
constexpr int kWaves = kCuCount * 8;
constexpr int kMinTiles = 2;
constexpr float kLn2 = 0.6931471805599453f;

// kType: 0 fp32, 1 bf16, 2 e4m3.
template <int kType, int kDim>
struct Shape {
  static constexpr int kSize = kType == 0 ? 4 : kType == 1 ? 2 : 1;  // bytes of a cached value
  static constexpr int kVDims = kDim / 16;                           // dimensions of V per lane
  // 16-key groups of a tile: 32 to 64 registers of K and V in flight per lane
  static constexpr int kGroups = kType == 0 ? (kDim == 64 ? 2 : 1) : kType == 1 ? 2 : 4;
  static constexpr int kTile = 16 * kGroups;            // keys
  static constexpr int kKWords = kDim * kSize / 16;     // words of K per lane and group
  static constexpr int kVWords = kVDims * kSize / 4;    // words of V per lane and key
  static constexpr int kQWords = kType == 0 ? kDim / 4 : kDim / 8;
};

template <int kType, int kDim>
struct KeyTile {
  using S = Shape<kType, kDim>;
  uint32_t w[S::kGroups][S::kKWords];
  uint32_t exp[S::kGroups];  // e4m3: of key lane % 16
};
template <int kType, int kDim>
struct ValueTile {
  using S = Shape<kType, kDim>;
  uint32_t w[S::kGroups][4][S::kVWords];
  uint32_t exp[S::kGroups];  // e4m3: of keys 4g .. 4g + 3
};

template <int kType, int kDim>
struct State {
  f32x4 o[kDim / 16];  // O^T: register r of o[i] is dimension (4g + r) kDim/16 + i of query lane % 16
  float m, l;          // largest score (in log2) and this lane's part of the sum
};

__device__ inline float exp2_fast(float x) { return __builtin_amdgcn_exp2f(x); }
__device__ inline float across_groups_max(float x) {
  x = fmaxf(x, __shfl_xor(x, 16));
  return fmaxf(x, __shfl_xor(x, 32));
}
__device__ inline float across_groups_sum(float x) {
  x += __shfl_xor(x, 16);
  return x + __shfl_xor(x, 32);
}

// Tokens of a request that are attended, in tiles: the first `head` tiles, and
// after them the tiles from `head + skip` on, `count` in all.
struct Span {
  int32_t n;       // tokens
  int32_t anchor;  // tokens [0, anchor) and [from, n) are kept
  int32_t from;
  int32_t head, skip, count;
};

template <int kTile>
__device__ inline Span span_of(const DecodeArgs& a, int32_t length) {
  Span s;
  s.n = min(max(length, 0), a.max_pages * a.page.size);
  const int32_t all = (s.n + kTile - 1) / kTile;
  if (a.window == 0) {
    s.anchor = 0;
    s.from = 0;
    s.head = 0;
    s.skip = 0;
    s.count = all;
  } else {
    s.anchor = min(a.anchor, s.n);
    s.from = max(s.n - a.window, 0);
    s.head = (s.anchor + kTile - 1) / kTile;
    const int32_t tail = max(s.from / kTile, s.head);
    s.skip = tail - s.head;
    s.count = s.head + max(all - tail, 0);
  }
  return s;
}

// One tile of a request's row: what it is and where its keys lie.
template <int kGroups>
struct Place {
  int32_t r;     // request
  int32_t row;   // of its rows (key-value head, tile of query heads)
  int32_t x;     // tile of the row, of s.count
  int32_t tile;  // the same counted from the sequence's start
  Span s;
  int32_t page[kGroups];  // -1 for a page that holds no token or whose entry is no page
  int64_t at[kGroups];    // bytes from a head's pages to the group's first key
  int64_t exp[kGroups];   // entries to its exponents
};

template <int kGroups>
__device__ inline void look_up(const DecodeArgs& a, const int32_t* __restrict__ table, Place<kGroups>& p) {
  p.tile = p.x < p.s.head ? p.x : p.x + p.s.skip;
  const int h = p.row / a.qtiles;
#pragma unroll
  for (int u = 0; u < kGroups; ++u) {
    const int32_t pos = p.tile * (16 * kGroups) + 16 * u;
    const int32_t i = div_page(a.page, pos);
    int32_t page = pos < p.s.n ? table[(int64_t)p.r * a.max_pages + i] : -1;
    page = page < 0 || page >= a.pages ? -1 : page;
    // an absent page's keys are read from page 0, which exists, and masked
    const int32_t in = page < 0 ? 0 : pos - i * a.page.size;
    const int64_t from = max(page, 0);
    p.page[u] = page;
    p.at[u] = from * a.page_stride + h * a.head_stride + (int64_t)in * a.token_stride;
    p.exp[u] = (from * a.kv_heads + h) * a.page.size + in;
  }
}

template <int kWords>
__device__ inline void load_words(uint32_t* to, const char* from) {
  if constexpr (kWords % 4 == 0) {
#pragma unroll
    for (int w = 0; w < kWords; w += 4) {
      const u32x4 x = *reinterpret_cast<const u32x4*>(from + 4 * w);
      to[w] = x[0];
      to[w + 1] = x[1];
      to[w + 2] = x[2];
      to[w + 3] = x[3];
    }
  } else if constexpr (kWords == 2) {
    const u32x2 x = *reinterpret_cast<const u32x2*>(from);
    to[0] = x[0];
    to[1] = x[1];
  } else {
    static_assert(kWords == 1, "words of a V row per lane");
    to[0] = *reinterpret_cast<const uint32_t*>(from);
  }
}

// Reads stay inside pages: a group's 16 keys lie in one page, whole.
template <int kType, int kDim>
__device__ inline void load_keys(const DecodeArgs& a, const char* __restrict__ k, const uint8_t* __restrict__ exp,
                                 const Place<Shape<kType, kDim>::kGroups>& p, KeyTile<kType, kDim>& t) {
  using S = Shape<kType, kDim>;
  const int lane = threadIdx.x & 63, g = lane >> 4, c = lane & 15;
  const uint32_t off = (uint32_t)(c * a.token_stride + g * 16);
#pragma unroll
  for (int u = 0; u < S::kGroups; ++u) {
    // row lane % 16, the pieces of 16 bytes g, g + 4, ...
#pragma unroll
    for (int w = 0; w < S::kKWords / 4; ++w) load_words<4>(&t.w[u][4 * w], k + p.at[u] + off + 64 * w);
    if constexpr (kType == 2) t.exp[u] = exp[p.exp[u] + c];
  }
}
template <int kType, int kDim>
__device__ inline void load_values(const DecodeArgs& a, const char* __restrict__ v, const uint8_t* __restrict__ exp,
                                   const Place<Shape<kType, kDim>::kGroups>& p, ValueTile<kType, kDim>& t) {
  using S = Shape<kType, kDim>;
  const int lane = threadIdx.x & 63, g = lane >> 4, c = lane & 15;
  const uint32_t off = (uint32_t)(4 * g * a.token_stride + c * (S::kVDims * S::kSize));
#pragma unroll
  for (int u = 0; u < S::kGroups; ++u) {
    // rows 4g .. 4g + 3, dimensions from (lane % 16) kDim / 16 on
#pragma unroll
    for (int r = 0; r < 4; ++r) load_words<S::kVWords>(t.w[u][r], v + p.at[u] + (off + (uint32_t)(r * a.token_stride)));
    if constexpr (kType == 2) t.exp[u] = *reinterpret_cast<const uint32_t*>(exp + p.exp[u] + 4 * g);
  }
}

__device__ inline bf16x8 as_bf16x8(uint32_t a, uint32_t b, uint32_t c, uint32_t d) {
  return __builtin_bit_cast(bf16x8, u32x4{a, b, c, d});
}
__device__ inline uint32_t fp8_pair(uint32_t codes, bool high, float scale) {
  const bf16x2 x = high ? __builtin_amdgcn_cvt_scalef32_pk_bf16_fp8(codes, scale, true)
                        : __builtin_amdgcn_cvt_scalef32_pk_bf16_fp8(codes, scale, false);
  return __builtin_bit_cast(uint32_t, x);
}
// Two fp32 as bf16 (nearest, ties to even), the first in the low half.
__device__ inline uint32_t bf16_pair(float x, float y) {
  return __builtin_bit_cast(uint32_t, bf16x2{(__bf16)x, (__bf16)y});
}

// S^T of a tile.
template <int kType, int kDim>
__device__ inline void score_tile(const KeyTile<kType, kDim>& t, const uint32_t (&q)[Shape<kType, kDim>::kQWords],
                                  f32x4 (&z)[Shape<kType, kDim>::kGroups]) {
  using S = Shape<kType, kDim>;
#pragma unroll
  for (int u = 0; u < S::kGroups; ++u) {
    z[u] = f32x4{0, 0, 0, 0};
    if constexpr (kType == 0) {
#pragma unroll
      for (int w = 0; w < kDim / 4; ++w)
        z[u] = __builtin_amdgcn_mfma_f32_16x16x4f32(__uint_as_float(t.w[u][w]), __uint_as_float(q[w]), z[u], 0, 0, 0);
    } else if constexpr (kType == 1) {
#pragma unroll
      for (int w = 0; w < kDim / 32; ++w)
        z[u] = __builtin_amdgcn_mfma_f32_16x16x32_bf16(
            as_bf16x8(t.w[u][4 * w], t.w[u][4 * w + 1], t.w[u][4 * w + 2], t.w[u][4 * w + 3]),
            as_bf16x8(q[4 * w], q[4 * w + 1], q[4 * w + 2], q[4 * w + 3]), z[u], 0, 0, 0);
    } else {
      const float scale = __uint_as_float(t.exp[u] << 23);
#pragma unroll
      for (int w = 0; w < kDim / 32; ++w) {
        const uint32_t c0 = t.w[u][2 * w], c1 = t.w[u][2 * w + 1];
        z[u] = __builtin_amdgcn_mfma_f32_16x16x32_bf16(
            as_bf16x8(fp8_pair(c0, false, scale), fp8_pair(c0, true, scale), fp8_pair(c1, false, scale),
                      fp8_pair(c1, true, scale)),
            as_bf16x8(q[4 * w], q[4 * w + 1], q[4 * w + 2], q[4 * w + 3]), z[u], 0, 0, 0);
      }
    }
  }
}

// Tiles at an end of the kept tokens, or with an absent page: a masked key's
// score is -inf and its V row 0, whatever memory holds there.
template <int kGroups>
__device__ inline bool is_whole(const Place<kGroups>& p) {
  const int32_t first = p.tile * (16 * kGroups), last = first + 16 * kGroups;
  bool whole = last <= p.s.n && (last <= p.s.anchor || first >= p.s.from);
#pragma unroll
  for (int u = 0; u < kGroups; ++u) whole = whole && p.page[u] >= 0;
  return whole;
}

// A tile's scores and V into the running softmax. With scores z in log2 units and
// the running maximum m, every new maximum scales what is summed so far by 2^(m - m').
template <int kType, int kDim>
__device__ inline void add_tile(const DecodeArgs& a, const Place<Shape<kType, kDim>::kGroups>& pl, f32x4 (&z)[Shape<kType, kDim>::kGroups],
                                ValueTile<kType, kDim>& t, State<kType, kDim>& st) {
  using S = Shape<kType, kDim>;
  const int g = (threadIdx.x & 63) >> 4;
  if (!is_whole(pl)) {
    const int32_t first = pl.tile * S::kTile;
#pragma unroll
    for (int u = 0; u < S::kGroups; ++u)
#pragma unroll
      for (int r = 0; r < 4; ++r) {
        const int32_t j = first + 16 * u + 4 * g + r;
        const bool keep = pl.page[u] >= 0 && j < pl.s.n && (j < pl.s.anchor || j >= pl.s.from);
        if (!keep) {
          z[u][r] = -INFINITY;
#pragma unroll
          for (int w = 0; w < S::kVWords; ++w) t.w[u][r][w] = 0;
          if constexpr (kType == 2) t.exp[u] = (t.exp[u] & ~(0xffu << (8 * r))) | 1u << (8 * r);
        }
      }
  }
  float top = fmaxf(fmaxf(z[0][0], z[0][1]), fmaxf(z[0][2], z[0][3]));
#pragma unroll
  for (int u = 1; u < S::kGroups; ++u)
    top = fmaxf(top, fmaxf(fmaxf(z[u][0], z[u][1]), fmaxf(z[u][2], z[u][3])));
  top = across_groups_max(top) * a.scale_log2;
  if (__any(top > st.m)) {
    const float to = fmaxf(st.m, top);
    const float f = to == -INFINITY ? 1.0f : exp2_fast(st.m - to);
    st.m = to;
    st.l *= f;
#pragma unroll
    for (int i = 0; i < S::kVDims; ++i) st.o[i] *= f;
  }
  const float m = st.m == -INFINITY ? 0.0f : st.m;  // every score so far -inf: weights 2^-inf = 0
  float p[S::kGroups][4];
#pragma unroll
  for (int u = 0; u < S::kGroups; ++u)
#pragma unroll
    for (int r = 0; r < 4; ++r) {
      p[u][r] = exp2_fast(fmaf(z[u][r], a.scale_log2, -m));
      st.l += p[u][r];
    }
  if constexpr (kType == 0) {
#pragma unroll
    for (int u = 0; u < S::kGroups; ++u)
#pragma unroll
      for (int r = 0; r < 4; ++r)
#pragma unroll
        for (int i = 0; i < S::kVDims; ++i)
          st.o[i] = __builtin_amdgcn_mfma_f32_16x16x4f32(__uint_as_float(t.w[u][r][i]), p[u][r], st.o[i], 0, 0, 0);
  } else {
#pragma unroll
    for (int u = 0; u < S::kGroups; u += 2) {
      // a weight as the sum of two bf16 (16 of its 24 bits): one alone would add
      // as much error as the output's own rounding
      uint32_t hi[4], lo[4];
#pragma unroll
      for (int x = 0; x < 4; ++x) {
        const float p0 = p[u + (x >> 1)][2 * (x & 1)], p1 = p[u + (x >> 1)][2 * (x & 1) + 1];
        hi[x] = bf16_pair(p0, p1);
        lo[x] = bf16_pair(p0 - __uint_as_float(hi[x] << 16), p1 - __uint_as_float(hi[x] & 0xffff0000u));
      }
      const bf16x8 ph = as_bf16x8(hi[0], hi[1], hi[2], hi[3]), pl = as_bf16x8(lo[0], lo[1], lo[2], lo[3]);
      // two dimensions of eight keys
      uint32_t vw[8][S::kVDims / 2];
#pragma unroll
      for (int x = 0; x < 8; ++x)
#pragma unroll
        for (int w = 0; w < S::kVDims / 2; ++w) {
          if constexpr (kType == 1) {
            vw[x][w] = t.w[u + (x >> 2)][x & 3][w];
          } else {
            const float scale = __uint_as_float(((t.exp[u + (x >> 2)] >> (8 * (x & 3))) & 0xffu) << 23);
            vw[x][w] = fp8_pair(t.w[u + (x >> 2)][x & 3][w >> 1], w & 1, scale);
          }
        }
#pragma unroll
      for (int i = 0; i < S::kVDims; ++i) {
        const uint32_t sel = i & 1 ? 0x07060302u : 0x05040100u;  // the high or the low halves of two words
        uint32_t e[4];
#pragma unroll
        for (int x = 0; x < 4; ++x) e[x] = __builtin_amdgcn_perm(vw[2 * x + 1][i >> 1], vw[2 * x][i >> 1], sel);
        const bf16x8 va = as_bf16x8(e[0], e[1], e[2], e[3]);
        st.o[i] = __builtin_amdgcn_mfma_f32_16x16x32_bf16(va, ph, st.o[i], 0, 0, 0);
        st.o[i] = __builtin_amdgcn_mfma_f32_16x16x32_bf16(va, pl, st.o[i], 0, 0, 0);
      }
    }
  }
}

// The queries of a tile of 16 heads: lane % 16 is the query, the pieces of its
// row those of K's rows. Heads past the group are zeros.
template <int kType, int kDim>
__device__ inline void load_queries(const DecodeArgs& a, const char* __restrict__ q, int r, int row,
                                    uint32_t (&w)[Shape<kType, kDim>::kQWords]) {
  using S = Shape<kType, kDim>;
  const int qt = row % a.qtiles, first = row / a.qtiles * a.group + 16 * qt;
  const int heads = min(a.group - 16 * qt, 16);
  const int lane = threadIdx.x & 63, g = lane >> 4, c = lane & 15;
  constexpr int kIn = kType == 0 ? 4 : 2;
#pragma unroll
  for (int x = 0; x < S::kQWords; ++x) w[x] = 0;
  if (c < heads) {
    const char* row = q + ((first + c) * a.q_head + r * a.q_request) * kIn;
    if constexpr (kType == 2) {
      // K's piece of 16 codes is two products' share: 32 bytes of q
#pragma unroll
      for (int x = 0; x < S::kQWords / 8; ++x) {
        load_words<4>(&w[8 * x], row + 128 * x + 32 * g);
        load_words<4>(&w[8 * x + 4], row + 128 * x + 32 * g + 16);
      }
    } else {
#pragma unroll
      for (int x = 0; x < S::kQWords / 4; ++x) load_words<4>(&w[4 * x], row + 64 * x + 16 * g);
    }
  }
}

// Where a launch's pieces go: a row that falls to several waves leaves a part in
// each, wave w's in slot 2w if the row began before the wave's tiles and in slot
// 2w + 1 if it begins among them. Each part: kDim sums per query, and (m, l).
struct Pieces {
  float* o;    // [2 kWaves][heads][kDim]
  float2* ml;  // [2 kWaves][heads]
  int4* cut;   // a row that starts in wave w and ends in a later one: (request, row, w, last wave), else w < 0
};
constexpr int64_t kCutBytes = (int64_t)kWaves * sizeof(int4);

__host__ __device__ inline Pieces pieces(void* workspace, int heads) {
  Pieces p;
  p.cut = static_cast<int4*>(workspace);
  p.ml = reinterpret_cast<float2*>(static_cast<char*>(workspace) + kCutBytes);
  p.o = reinterpret_cast<float*>(p.ml + 2 * kWaves * heads);
  return p;
}
__host__ __device__ inline int piece_heads(const DecodeArgs& a) { return a.group < 16 ? a.group : 16; }

// A wave's part of a row: the output where it has the whole row, else a piece.
template <int kType, int kDim>
__device__ inline void put_row(const DecodeArgs& a, const State<kType, kDim>& st, int r, int row, int slot, char* __restrict__ out,
                               float* __restrict__ lse, const Pieces& pc) {
  using S = Shape<kType, kDim>;
  const int lane = threadIdx.x & 63, g = lane >> 4, c = lane & 15;
  const int qt = row % a.qtiles, first = row / a.qtiles * a.group + 16 * qt;
  const int heads = min(a.group - 16 * qt, 16);
  const float l = across_groups_sum(st.l);
  if (c >= heads) return;
  if (slot >= 0) {
    const int at = slot * piece_heads(a) + c;
    if (g == 0) pc.ml[at] = float2{st.m, l};
#pragma unroll
    for (int x = 0; x < 4; ++x)
#pragma unroll
      for (int i = 0; i < S::kVDims; i += 4)
        *reinterpret_cast<f32x4*>(pc.o + (int64_t)at * kDim + (4 * g + x) * S::kVDims + i) =
            f32x4{st.o[i][x], st.o[i + 1][x], st.o[i + 2][x], st.o[i + 3][x]};
    return;
  }
  const float f = l > 0.0f ? 1.0f / l : l;  // 0 and NaN stay
  const int head = first + c;
  const int64_t at = head * a.out_head + r * a.out_request;
#pragma unroll
  for (int x = 0; x < 4; ++x)
#pragma unroll
    for (int i = 0; i < S::kVDims; i += 4) {
      const int64_t to = at + (4 * g + x) * S::kVDims + i;
      const f32x4 y = f32x4{st.o[i][x], st.o[i + 1][x], st.o[i + 2][x], st.o[i + 3][x]} * f;
      if constexpr (kType == 0)
        *reinterpret_cast<f32x4*>(reinterpret_cast<float*>(out) + to) = y;
      else
        *reinterpret_cast<u32x2*>(reinterpret_cast<uint16_t*>(out) + to) = u32x2{bf16_pair(y[0], y[1]), bf16_pair(y[2], y[3])};
    }
  if (lse && g == 0) lse[(int64_t)head * a.requests + r] = (st.m + __log2f(l)) * kLn2;
}

// The next request after r that has tiles (64 lengths at a time), or `requests`.
template <int kTile>
__device__ inline int next_request(const DecodeArgs& a, const int32_t* __restrict__ lengths, int r) {
  const int lane = threadIdx.x & 63;
  for (++r; r < a.requests; r += 64) {
    const bool some = r + lane < a.requests && lengths[r + lane] > 0;
    const uint64_t found = __ballot(some);
    if (found) return r + __ffsll((unsigned long long)found) - 1;
  }
  return a.requests;
}

// The tiles of all requests' rows, request by request and row by row, are dealt
// out to the waves in equal runs of neighbouring tiles. A wave goes through its
// run without a stop: while it works on one tile's scores the next one's K is on
// the way, while it works on V the next V.
template <int kType, int kDim>
__global__ __launch_bounds__(kThreads, 2) void paged_attention_kernel(
    const char* __restrict__ q, const char* __restrict__ k, const char* __restrict__ v,
    const uint8_t* __restrict__ k_exp, const uint8_t* __restrict__ v_exp, const int32_t* __restrict__ table,
    const int32_t* __restrict__ lengths, char* __restrict__ out, float* __restrict__ lse, void* __restrict__ workspace,
    DecodeArgs a) {
  using S = Shape<kType, kDim>;
  __shared__ int64_t before[kThreads + 1];  // tiles of the requests before a thread's
  __shared__ int64_t wave_sum[kThreads / 64];
  const int lane = threadIdx.x & 63, wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
  const int rows = a.kv_heads * a.qtiles;
  const Pieces pc = pieces(workspace, piece_heads(a));

  // requests without a token
  for (int r = blockIdx.x; r < a.requests; r += gridDim.x) {
    if (lengths[r] > 0) continue;
    for (int i = threadIdx.x; i < a.q_heads * (kDim / 4); i += kThreads) {
      const int head = i / (kDim / 4), d = i % (kDim / 4) * 4;
      const int64_t at = head * a.out_head + r * a.out_request + d;
      if constexpr (kType == 0)
        *reinterpret_cast<f32x4*>(reinterpret_cast<float*>(out) + at) = f32x4{0, 0, 0, 0};
      else
        *reinterpret_cast<u32x2*>(reinterpret_cast<uint16_t*>(out) + at) = u32x2{0, 0};
      if (lse && d == 0) lse[(int64_t)head * a.requests + r] = -INFINITY;
    }
  }

  // where the runs lie: each thread counts neighbouring requests
  const int each = (a.requests + kThreads - 1) / kThreads;
  int64_t mine = 0;
  for (int i = 0; i < each; ++i) {
    const int r = threadIdx.x * each + i;
    if (r < a.requests) mine += span_of<S::kTile>(a, lengths[r]).count;
  }
  mine *= rows;
  int64_t sum = mine;
#pragma unroll
  for (int d = 1; d < 64; d <<= 1) {
    const int64_t y = __shfl_up(sum, d);
    if (lane >= d) sum += y;
  }
  if (lane == 63) wave_sum[wave] = sum;
  __syncthreads();
  int64_t total = 0;
#pragma unroll
  for (int w = 0; w < kThreads / 64; ++w) {
    if (w == wave) sum += total;
    total += wave_sum[w];
  }
  before[threadIdx.x] = sum - mine;
  __syncthreads();

  const int64_t run = max((total + kWaves - 1) / kWaves, (int64_t)kMinTiles);
  const int w = wave * gridDim.x + blockIdx.x;  // neighbouring runs on different CUs
  const int64_t lo = w * run, hi = min(lo + run, total);
  if (lane == 0) pc.cut[w].z = -1;
  if (lo >= hi) return;

  // the first tile's request: the thread whose requests hold it, then these one by one
  int owner = 0;
#pragma unroll
  for (int i = 0; i < kThreads / 64; ++i) owner += __popcll(__ballot(before[64 * i + lane] <= lo));
  owner -= 1;
  Place<S::kGroups> next;
  next.r = owner * each;
  int64_t off = lo - before[owner];
  next.s = span_of<S::kTile>(a, lengths[next.r]);
  while (off >= (int64_t)next.s.count * rows) {
    off -= (int64_t)next.s.count * rows;
    next.s = span_of<S::kTile>(a, lengths[++next.r]);
  }
  next.r = __builtin_amdgcn_readfirstlane(next.r);
  next.s = span_of<S::kTile>(a, lengths[next.r]);
  next.row = (int32_t)(off / next.s.count);
  next.row = __builtin_amdgcn_readfirstlane(next.row);
  next.x = __builtin_amdgcn_readfirstlane((int32_t)(off - (int64_t)next.row * next.s.count));

  KeyTile<kType, kDim> kt;
  ValueTile<kType, kDim> vt;
  State<kType, kDim> st;
  uint32_t qw[S::kQWords], qn[S::kQWords];
  look_up<S::kGroups>(a, table, next);
  load_queries<kType, kDim>(a, q, next.r, next.row, qn);
  load_keys<kType, kDim>(a, k, k_exp, next, kt);
  load_values<kType, kDim>(a, v, v_exp, next, vt);
  bool begins = true;         // the tile is the wave's first of its row
  bool from_start = next.x == 0;  // and the row's first
  int64_t left = hi - lo;
  while (true) {
    const Place<S::kGroups> now = next;
    if (begins) {
#pragma unroll
      for (int i = 0; i < S::kQWords; ++i) qw[i] = qn[i];
      st.m = -INFINITY;
      st.l = 0.0f;
#pragma unroll
      for (int i = 0; i < S::kVDims; ++i) st.o[i] = f32x4{0, 0, 0, 0};
      from_start = now.x == 0;
    }
    f32x4 z[S::kGroups];
    score_tile<kType, kDim>(kt, qw, z);
    const bool ends = now.x + 1 == now.s.count;
    --left;
    if (left > 0) {
      if (!ends) {
        ++next.x;
      } else {
        next.x = 0;
        if (++next.row == rows) {
          next.row = 0;
          next.r = __builtin_amdgcn_readfirstlane(next_request<S::kTile>(a, lengths, next.r));
          next.s = span_of<S::kTile>(a, lengths[next.r]);
        }
        load_queries<kType, kDim>(a, q, next.r, next.row, qn);
      }
      look_up<S::kGroups>(a, table, next);
      load_keys<kType, kDim>(a, k, k_exp, next, kt);
    }
    add_tile<kType, kDim>(a, now, z, vt, st);
    if (left > 0) load_values<kType, kDim>(a, v, v_exp, next, vt);
    begins = ends;
    if (ends || left == 0) {
      const bool whole = ends && from_start;
      put_row<kType, kDim>(a, st, now.r, now.row, whole ? -1 : from_start ? 2 * w + 1 : 2 * w, out, lse, pc);
      if (!ends && from_start && lane == 0) {
        // tiles of the row behind this run, a run each wave
        const int64_t behind = now.s.count - 1 - now.x;
        pc.cut[w] = int4{now.r, now.row, w, w + (int)((behind + run - 1) / run)};
      }
    }
    if (left == 0) break;
  }
}

// The rows that fell to several waves: one workgroup per such row and query, its
// 16-byte lanes spread over kThreads * 4 / kDim pieces at a time, in the order of
// the waves.
template <int kType, int kDim>
__global__ __launch_bounds__(kThreads) void paged_join_kernel(const void* __restrict__ workspace, char* __restrict__ out,
                                                              float* __restrict__ lse, DecodeArgs a) {
  constexpr int kLanes = kDim / 4, kAtOnce = kThreads / kLanes;
  __shared__ f32x4 part[kAtOnce][kLanes];
  __shared__ float2 part_ml[kAtOnce];
  const Pieces pc = pieces(const_cast<void*>(workspace), piece_heads(a));
  const int4 cut = pc.cut[blockIdx.x];
  if (cut.z < 0) return;
  const int qt = cut.y % a.qtiles, n = blockIdx.y;
  if (n >= min(a.group - 16 * qt, 16)) return;
  const int head = cut.y / a.qtiles * a.group + 16 * qt + n;
  const int slot = threadIdx.x / kLanes, d = threadIdx.x % kLanes;
  const int count = cut.w - cut.z + 1;
  float m = -INFINITY, l = 0.0f;
  f32x4 o{0, 0, 0, 0};
  for (int i = slot; i < count; i += kAtOnce) {
    const int at = (2 * (cut.z + i) + (i == 0 ? 1 : 0)) * piece_heads(a) + n;
    const float2 ml = pc.ml[at];
    const f32x4 x = *reinterpret_cast<const f32x4*>(pc.o + (int64_t)at * kDim + 4 * d);
    const float to = fmaxf(m, ml.x);
    const float f = to == -INFINITY ? 1.0f : exp2_fast(m - to), g = to == -INFINITY ? 1.0f : exp2_fast(ml.x - to);
    o = o * f + x * g;
    l = l * f + ml.y * g;
    m = to;
  }
  part[slot][d] = o;
  if (d == 0) part_ml[slot] = float2{m, l};
  __syncthreads();
  if (slot > 0) return;
#pragma unroll
  for (int i = 1; i < kAtOnce; ++i) {
    const float2 ml = part_ml[i];
    const float to = fmaxf(m, ml.x);
    const float f = to == -INFINITY ? 1.0f : exp2_fast(m - to), g = to == -INFINITY ? 1.0f : exp2_fast(ml.x - to);
    o = o * f + part[i][d] * g;
    l = l * f + ml.y * g;
    m = to;
  }
  o *= l > 0.0f ? 1.0f / l : l;
  const int64_t to = head * a.out_head + cut.x * a.out_request + 4 * d;
  if constexpr (kType == 0)
    *reinterpret_cast<f32x4*>(reinterpret_cast<float*>(out) + to) = o;
  else
    *reinterpret_cast<u32x2*>(reinterpret_cast<uint16_t*>(out) + to) = u32x2{bf16_pair(o[0], o[1]), bf16_pair(o[2], o[3])};
  if (lse && d == 0) lse[(int64_t)head * a.requests + cut.x] = (m + __log2f(l)) * kLn2;
}

template <int kType, int kDim>
hipError_t launch(const void* q, const void* kp, const void* vp, const uint8_t* ke, const uint8_t* ve, const int32_t* table,
                  const int32_t* lengths, void* out, float* lse, void* workspace, const DecodeArgs& a, hipStream_t s) {
  hipLaunchKernelGGL((paged_attention_kernel<kType, kDim>), dim3(kWaves / (kThreads / 64)), dim3(kThreads), 0, s,
                     static_cast<const char*>(q), static_cast<const char*>(kp), static_cast<const char*>(vp), ke, ve, table,
                     lengths, static_cast<char*>(out), lse, workspace, a);
  const hipError_t e = hipGetLastError();
  if (e != hipSuccess) return e;
  hipLaunchKernelGGL((paged_join_kernel<kType, kDim>), dim3(kWaves, (unsigned)piece_heads(a)), dim3(kThreads), 0, s, workspace,
                     static_cast<char*>(out), lse, a);
  return hipGetLastError();
}

}  // namespace

int64_t paged_attention_workspace(int dim, const DecodeArgs& a) {
  return kCutBytes + (int64_t)2 * kWaves * piece_heads(a) * ((int64_t)sizeof(float2) + dim * (int64_t)sizeof(float));
}

hipError_t launch_paged_attention(int dtype, int dim, const void* q, const void* k_pages,
                                  const void* v_pages, const uint8_t* k_exp, const uint8_t* v_exp,
                                  const int32_t* table, const int32_t* lengths, void* out, float* lse,
                                  void* workspace, const DecodeArgs& a, hipStream_t s) {
#define SAF3R_CASE(T, D)     \
  if (dtype == T && dim == D) \
  return launch<T, D>(q, k_pages, v_pages, k_exp, v_exp, table, lengths, out, lse, workspace, a, s)
  SAF3R_CASE(0, 64);
  SAF3R_CASE(0, 128);
  SAF3R_CASE(1, 64);
  SAF3R_CASE(1, 128);
  SAF3R_CASE(2, 64);
  SAF3R_CASE(2, 128);
#undef SAF3R_CASE
  return hipErrorInvalidValue;
}

}  // namespace saf3r
