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
#include "paged_scores.h"

namespace saf3r {
namespace {

typedef __bf16 bf16x8 __attribute__((ext_vector_type(8)));
typedef __bf16 bf16x2 __attribute__((ext_vector_type(2)));
typedef float f32x4 __attribute__((ext_vector_type(4)));
typedef uint32_t u32x4 __attribute__((ext_vector_type(4)));
typedef uint32_t u32x2 __attribute__((ext_vector_type(2)));

constexpr float kLn2 = 0.6931471805599453f, kLog2e = 1.4426950408889634f;

// kType: 0 fp32, 1 bf16, 2 e4m3, 4 e2m1.
template <int kType, int kDim>
struct Shape {
  static constexpr int kBits = cache_bits(kType);  // of a cached value
  static constexpr int kVDims = kDim / 16;         // dimensions of V per lane
  // 16-key groups of a tile: 32 to 64 registers of K and V in flight per lane (four for
  // bf16 of 64 as well: 26.7 -> 28.3 us for 1024 rows of 512 tokens, 10.2 -> 9.7 for 128
  // rows of 1024; e2m1 with two 220 -> 237 us for 192 ragged sequences of width 128, with
  // six 229; one of 274800 tokens of width 64 79 -> 100 with two, 79 with six and eight)
  static constexpr int kGroups = kType == 0 ? (kDim == 64 ? 2 : 1) : kType == 1 ? 2 : 4;
  static constexpr int kTile = 16 * kGroups;            // keys
  // A wave's share in a shared-out launch is at least 64 keys. For 16 rows of 2100
  // tokens: with half as many as that, 12.4 -> 12.8 us in fp32 of 64, 11.8 -> 12.2 in bf16
  // of 128; with twice, 12.4 -> 16.0, 11.8 -> 14.3 and in 8 bits of 128 11.1 -> 13.6.
  static constexpr int kMinTiles = 64 / kTile;
  static constexpr int kKWords = kDim * kBits / 128;    // words of K per lane and group
  static constexpr int kVBytes = kVDims * kBits / 8;    // bytes of V per lane and key
  static constexpr int kVWords = (kVBytes + 3) / 4;     // and words
  static constexpr int kBlocks = kDim / kExpBlock;      // e2m1: exponents of a row
  // words of the exponents of a lane's four keys of V
  static constexpr int kVExps = kType == 4 ? kBlocks : 1;
  static constexpr int kQWords = kType == 0 ? kDim / 4 : kDim / 8;
};

template <int kType, int kDim>
struct KeyTile {
  using S = Shape<kType, kDim>;
  uint32_t w[S::kGroups][S::kKWords];
  uint32_t exp[S::kGroups];  // e4m3, e2m1: of key lane % 16 (and the lane's dimensions)
};
template <int kType, int kDim>
struct ValueTile {
  using S = Shape<kType, kDim>;
  uint32_t w[S::kGroups][4][S::kVWords];
  uint32_t exp[S::kGroups][S::kVExps];  // e4m3, e2m1: of keys 4g .. 4g + 3, in e2m1 all of the rows
};

template <int kType, int kDim>
struct State {
  f32x4 o[kDim / 16];  // O^T: register r of o[i] is dimension (4g + r) kDim/16 + i of query lane % 16
  float m, l;          // largest score (in log2) and this lane's part of the sum
};

// A query head's share of the changed scores: its slope times log2(e).
template <bool kScored>
struct Bias {
  float slope = 0.0f;
};
template <>
struct Bias<false> {};

__device__ inline float exp2_fast(float x) { return __builtin_amdgcn_exp2f(x); }
// Over the four lanes of a query: lanes 32 and 16 apart, exchanged in registers.
__device__ inline float across_groups_max(float x) {
  const uint32_t w = __float_as_uint(x);
  const auto s = __builtin_amdgcn_permlane32_swap(w, w, false, false);
  const uint32_t y = __float_as_uint(fmaxf(__uint_as_float(s[0]), __uint_as_float(s[1])));
  const auto t = __builtin_amdgcn_permlane16_swap(y, y, false, false);
  return fmaxf(__uint_as_float(t[0]), __uint_as_float(t[1]));
}
__device__ inline float across_groups_sum(float x) {
  const uint32_t w = __float_as_uint(x);
  const auto s = __builtin_amdgcn_permlane32_swap(w, w, false, false);
  const uint32_t y = __float_as_uint(__uint_as_float(s[0]) + __uint_as_float(s[1]));
  const auto t = __builtin_amdgcn_permlane16_swap(y, y, false, false);
  return __uint_as_float(t[0]) + __uint_as_float(t[1]);
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

// One tile of a row: what it is and where its keys lie. A row is a request's
// key-value head h with up to 16 of the query heads that share it.
template <int kGroups>
struct Place {
  int32_t r;             // request
  int32_t h, qt;         // key-value head, tile of its query heads
  int32_t first, heads;  // query heads first .. first + heads - 1
  int32_t x;             // tile of the row, of s.count
  int32_t tile;          // the same counted from the sequence's start
  Span s;
  uint32_t absent;       // bit u: group u's page holds no token, or its entry is no page
  int64_t head, exp_head;  // bytes to the head in a page, tokens to its exponents
  int64_t at[kGroups];   // bytes to the group's first key
  int64_t exp[kGroups];  // tokens to its exponents
  __device__ void set_row(const DecodeArgs& a) {
    first = h * a.group + 16 * qt;
    heads = min(a.group - 16 * qt, 16);
    head = h * a.head_stride;
    exp_head = (int64_t)h * a.page.size;
  }
  // the next row of the request; false if that was its last
  __device__ bool next_row(const DecodeArgs& a) {
    x = 0;
    bool more = true;
    if (++qt == a.qtiles) {
      qt = 0;
      if (++h == a.kv_heads) {
        h = 0;
        more = false;
      }
    }
    set_row(a);
    return more;
  }
};

// 64 entries of a request's row of the table, one a lane: a tile's pages come from
// there without a trip to memory.
struct Entries {
  int32_t r, base;
  int32_t page;  // entry base + lane; -1 past the request's pages and for what is no page
};

template <int kType, int kGroups>
__device__ inline void look_up(const DecodeArgs& a, const int32_t* __restrict__ table, Entries& e, Place<kGroups>& p) {
  p.tile = p.x < p.s.head ? p.x : p.x + p.s.skip;
  p.absent = 0;
  const int32_t pos = p.tile * (16 * kGroups);
  int32_t i = div_page(a.page, pos), in = pos - i * a.page.size;
#pragma unroll
  for (int u = 0; u < kGroups; ++u) {
    if (u > 0) {
      in += 16;
      if (in == a.page.size) {
        in = 0;
        ++i;
      }
    }
    if (u == 0 || in == 0) {
      if (p.r != e.r || (uint32_t)(i - e.base) >= 64u) {
        e.r = p.r;
        e.base = i;
        const int32_t j = i + (threadIdx.x & 63);
        e.page = j * a.page.size < p.s.n ? table[(int64_t)p.r * a.max_pages + j] : -1;
        e.page = (uint32_t)e.page < (uint32_t)a.pages ? e.page : -1;
        // waited for here: left to its first use, the wait would be one for every
        // load in flight on every tile
        asm volatile("" : "+v"(e.page));
      }
      // an absent page's keys are read from page 0, which exists, and masked
      const int32_t page = __builtin_amdgcn_readlane(e.page, i - e.base);
      p.absent |= (uint32_t)(page < 0) << u;
      const uint32_t from = (uint32_t)max(page, 0);
      p.at[u] = p.head + from * a.page_stride + (int64_t)in * a.token_stride;
      if constexpr (kType == 2 || kType == 4) p.exp[u] = p.exp_head + from * (int64_t)(a.kv_heads * a.page.size) + in;
    } else {
      p.absent |= (p.absent >> (u - 1) & 1u) << u;
      p.at[u] = p.at[u - 1] + 16 * a.token_stride;
      if constexpr (kType == 2 || kType == 4) p.exp[u] = p.exp[u - 1] + 16;
    }
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
    static_assert(kWords == 1, "words of a row per lane");
    to[0] = *reinterpret_cast<const uint32_t*>(from);
  }
}

// Reads stay inside pages: a group's 16 keys lie in one page, whole.
template <int kType, int kDim>
__device__ inline void load_keys(const DecodeArgs& a, const char* __restrict__ k, const uint8_t* __restrict__ exp,
                                 const Place<Shape<kType, kDim>::kGroups>& p, KeyTile<kType, kDim>& t) {
  using S = Shape<kType, kDim>;
  const int lane = threadIdx.x & 63, g = lane >> 4, c = lane & 15;
  constexpr int kPiece = S::kKWords < 4 ? S::kKWords : 4;  // words
  const uint32_t off = (uint32_t)(c * a.token_stride + g * (4 * kPiece));
#pragma unroll
  for (int u = 0; u < S::kGroups; ++u) {
    // row lane % 16, the pieces of 16 bytes g, g + 4, ... (of 4-bit rows a quarter each)
#pragma unroll
    for (int w = 0; w < S::kKWords / kPiece; ++w) load_words<kPiece>(&t.w[u][4 * w], k + p.at[u] + off + 64 * w);
    if constexpr (kType == 2) t.exp[u] = exp[p.exp[u] + c];
    if constexpr (kType == 4) t.exp[u] = exp[p.exp[u] * S::kBlocks + (c * S::kBlocks + g * S::kBlocks / 4)];
  }
}
template <int kType, int kDim>
__device__ inline void load_values(const DecodeArgs& a, const char* __restrict__ v, const uint8_t* __restrict__ exp,
                                   const Place<Shape<kType, kDim>::kGroups>& p, ValueTile<kType, kDim>& t) {
  using S = Shape<kType, kDim>;
  const int lane = threadIdx.x & 63, g = lane >> 4, c = lane & 15;
  const uint32_t off = (uint32_t)(4 * g * a.token_stride + c * S::kVBytes);
#pragma unroll
  for (int u = 0; u < S::kGroups; ++u) {
    // rows 4g .. 4g + 3, dimensions from (lane % 16) kDim / 16 on
#pragma unroll
    for (int r = 0; r < 4; ++r) {
      const char* from = v + p.at[u] + (off + (uint32_t)(r * a.token_stride));
      if constexpr (S::kVBytes == 2)
        t.w[u][r][0] = *reinterpret_cast<const uint16_t*>(from);
      else
        load_words<S::kVWords>(t.w[u][r], from);
    }
    if constexpr (kType == 2) t.exp[u][0] = *reinterpret_cast<const uint32_t*>(exp + p.exp[u] + 4 * g);
    if constexpr (kType == 4)
      load_words<S::kVExps>(t.exp[u], reinterpret_cast<const char*>(exp) + p.exp[u] * S::kBlocks + 4 * g * S::kBlocks);
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
// The two values of one byte, each exact in bf16.
template <int kByte>
__device__ inline uint32_t fp4_pair(uint32_t codes, float scale) {
  return __builtin_bit_cast(uint32_t, (bf16x2)__builtin_amdgcn_cvt_scalef32_pk_bf16_fp4(codes, scale, kByte));
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
      // four sums of a quarter of the dimensions each: shorter chains, and a quarter
      // of the roundings that the score of a single one would go through
      f32x4 part[4] = {z[u], z[u], z[u], z[u]};
#pragma unroll
      for (int w = 0; w < kDim / 4; ++w)
        part[w & 3] = __builtin_amdgcn_mfma_f32_16x16x4f32(__uint_as_float(t.w[u][w]), __uint_as_float(q[w]), part[w & 3], 0, 0, 0);
      z[u] = (part[0] + part[1]) + (part[2] + part[3]);
    } else if constexpr (kType == 1) {
#pragma unroll
      for (int w = 0; w < kDim / 32; ++w)
        z[u] = __builtin_amdgcn_mfma_f32_16x16x32_bf16(
            as_bf16x8(t.w[u][4 * w], t.w[u][4 * w + 1], t.w[u][4 * w + 2], t.w[u][4 * w + 3]),
            as_bf16x8(q[4 * w], q[4 * w + 1], q[4 * w + 2], q[4 * w + 3]), z[u], 0, 0, 0);
    } else if constexpr (kType == 4) {
      const float scale = __uint_as_float(t.exp[u] << 23);
#pragma unroll
      for (int w = 0; w < kDim / 32; ++w) {
        const uint32_t c = t.w[u][w];
        z[u] = __builtin_amdgcn_mfma_f32_16x16x32_bf16(
            as_bf16x8(fp4_pair<0>(c, scale), fp4_pair<1>(c, scale), fp4_pair<2>(c, scale), fp4_pair<3>(c, scale)),
            as_bf16x8(q[4 * w], q[4 * w + 1], q[4 * w + 2], q[4 * w + 3]), z[u], 0, 0, 0);
      }
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
  return p.absent == 0 && last <= p.s.n && (last <= p.s.anchor || first >= p.s.from);
}

// A tile's scores and V into the running softmax. With scores z in log2 units and
// the running maximum m, every new maximum scales what is summed so far by 2^(m - m').
// kScored: z are first capped and lowered by the distance of query and key.
template <int kType, int kDim, bool kScored>
__device__ inline void add_tile(const DecodeArgs& a, const Place<Shape<kType, kDim>::kGroups>& pl, f32x4 (&z)[Shape<kType, kDim>::kGroups],
                                ValueTile<kType, kDim>& t, State<kType, kDim>& st, const Bias<kScored>& bias) {
  using S = Shape<kType, kDim>;
  const int g = (threadIdx.x & 63) >> 4;
  const float scale_log2 = kScored ? 1.0f : a.scale_log2;
  if constexpr (kScored) {
    // the query is the last token; fp32 counts exactly up to 2^24, a farther key's
    // distance is off by its own rounding
    const float far = (float)(pl.s.n - 1 - pl.tile * S::kTile - 4 * g);
#pragma unroll
    for (int u = 0; u < S::kGroups; ++u)
#pragma unroll
      for (int r = 0; r < 4; ++r) {
        z[u][r] = a.cap_in != 0.0f ? a.cap_out * tanh_of(z[u][r] * a.cap_in) : z[u][r] * a.scale_log2;
        z[u][r] = fmaf(-bias.slope, far - (float)(16 * u + r), z[u][r]);
      }
  }
  if (!is_whole(pl)) {
    const int32_t first = pl.tile * S::kTile;
#pragma unroll
    for (int u = 0; u < S::kGroups; ++u)
#pragma unroll
      for (int r = 0; r < 4; ++r) {
        const int32_t j = first + 16 * u + 4 * g + r;
        const bool keep = !(pl.absent >> u & 1u) && j < pl.s.n && (j < pl.s.anchor || j >= pl.s.from);
        if (!keep) {
          z[u][r] = -INFINITY;
#pragma unroll
          for (int w = 0; w < S::kVWords; ++w) t.w[u][r][w] = 0;
          if constexpr (kType == 2) t.exp[u][0] = (t.exp[u][0] & ~(0xffu << (8 * r))) | 1u << (8 * r);
          if constexpr (kType == 4 && S::kBlocks == 4) t.exp[u][r] = 0x01010101u;
          if constexpr (kType == 4 && S::kBlocks == 2)
            t.exp[u][r >> 1] = (t.exp[u][r >> 1] & ~(0xffffu << (16 * (r & 1)))) | 0x0101u << (16 * (r & 1));
        }
      }
  }
  float top = fmaxf(fmaxf(z[0][0], z[0][1]), fmaxf(z[0][2], z[0][3]));
#pragma unroll
  for (int u = 1; u < S::kGroups; ++u)
    top = fmaxf(top, fmaxf(fmaxf(z[u][0], z[u][1]), fmaxf(z[u][2], z[u][3])));
  top = across_groups_max(top) * scale_log2;
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
  const auto weights = [&](float by, float then) {
#pragma unroll
    for (int u = 0; u < S::kGroups; ++u)
#pragma unroll
      for (int r = 0; r < 4; ++r) {
        p[u][r] = exp2_fast(fmaf(z[u][r] * by, then, -m));
        st.l += p[u][r];
      }
  };
  // From a maximum of 2^24 on its rounding is a power of two and more, as much as that of the
  // scores themselves: they are scaled first, so that the largest one's weight is 1.
  const bool far = !kScored && fabsf(m) >= 16777216.0f;
  if (__any(far))
    weights(far ? scale_log2 : 1.0f, far ? 1.0f : scale_log2);
  else
    weights(1.0f, scale_log2);
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
          } else if constexpr (kType == 4) {
            const int c = threadIdx.x & 15, r = x & 3;
            // of the lane's block: dimensions from c kDim / 16 on
            const uint32_t (&e)[S::kVExps] = t.exp[u + (x >> 2)];
            const uint32_t exp = S::kBlocks == 4 ? e[r] >> (8 * (c >> 2)) : e[r >> 1] >> (16 * (r & 1) + 8 * (c >> 3));
            const float scale = __uint_as_float((exp & 0xffu) << 23);
            const uint32_t codes = t.w[u + (x >> 2)][r][0];
            vw[x][w] = w == 0 ? fp4_pair<0>(codes, scale) : w == 1 ? fp4_pair<1>(codes, scale)
                       : w == 2 ? fp4_pair<2>(codes, scale) : fp4_pair<3>(codes, scale);
          } else {
            const float scale = __uint_as_float(((t.exp[u + (x >> 2)][0] >> (8 * (x & 3))) & 0xffu) << 23);
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
__device__ inline void load_queries(const DecodeArgs& a, const char* __restrict__ q,
                                    const Place<Shape<kType, kDim>::kGroups>& p, uint32_t (&w)[Shape<kType, kDim>::kQWords]) {
  using S = Shape<kType, kDim>;
  const int lane = threadIdx.x & 63, g = lane >> 4, c = lane & 15;
  constexpr int kIn = kType == 0 ? 4 : 2;
#pragma unroll
  for (int x = 0; x < S::kQWords; ++x) w[x] = 0;
  if (c < p.heads) {
    const char* row = q + ((p.first + c) * a.q_head + p.r * a.q_request) * kIn;
    if constexpr (kType == 2) {
      // K's piece of 16 codes is two products' share: 32 bytes of q
#pragma unroll
      for (int x = 0; x < S::kQWords / 8; ++x) {
        load_words<4>(&w[8 * x], row + 128 * x + 32 * g);
        load_words<4>(&w[8 * x + 4], row + 128 * x + 32 * g + 16);
      }
    } else if constexpr (kType == 4) {
      // a quarter of the row
#pragma unroll
      for (int x = 0; x < S::kQWords / 4; ++x) load_words<4>(&w[4 * x], row + kDim / 2 * g + 16 * x);
    } else {
#pragma unroll
      for (int x = 0; x < S::kQWords / 4; ++x) load_words<4>(&w[4 * x], row + 64 * x + 16 * g);
    }
  }
}
template <bool kScored, int kGroups>
__device__ inline Bias<kScored> load_bias(const DecodeArgs& a, const Place<kGroups>& p) {
  Bias<kScored> b;
  if constexpr (kScored) {
    const int c = threadIdx.x & 15;
    if (a.slopes && c < p.heads) b.slope = a.slopes[p.first + c] * kLog2e;
  }
  return b;
}

// Parts of rows in LDS: of each its sums and (m, l) per query.
template <int kDim, int kSlots>
struct Parts {
  float o[kSlots][16][kDim + 4];
  float2 ml[kSlots][16];
};

template <int kType, int kDim, int kSlots>
__device__ inline void put_part(Parts<kDim, kSlots>& lds, int slot, const State<kType, kDim>& st) {
  using S = Shape<kType, kDim>;
  const int lane = threadIdx.x & 63, g = lane >> 4, c = lane & 15;
  const float l = across_groups_sum(st.l);
  if (g == 0) lds.ml[slot][c] = float2{st.m, l};
#pragma unroll
  for (int x = 0; x < 4; ++x)
#pragma unroll
    for (int i = 0; i < S::kVDims; i += 4)
      *reinterpret_cast<f32x4*>(&lds.o[slot][c][(4 * g + x) * S::kVDims + i]) =
          f32x4{st.o[i][x], st.o[i + 1][x], st.o[i + 2][x], st.o[i + 3][x]};
}

// kWidth neighbouring sums of a query, and its (m, l).
template <int kWidth>
struct Sums {
  float o[kWidth];
  float m, l;
  __device__ void clear() {
    m = -INFINITY;
    l = 0.0f;
#pragma unroll
    for (int i = 0; i < kWidth; ++i) o[i] = 0.0f;
  }
  __device__ void add(const float* x, float2 ml) {
    const float to = fmaxf(m, ml.x);
    const float f = to == -INFINITY ? 1.0f : exp2_fast(m - to), g = to == -INFINITY ? 1.0f : exp2_fast(ml.x - to);
#pragma unroll
    for (int i = 0; i < kWidth; ++i) o[i] = fmaf(x[i], g, o[i] * f);
    l = fmaf(ml.y, g, l * f);
    m = to;
  }
};

template <int kType, int kWidth>
__device__ inline void put_values(const DecodeArgs& a, char* __restrict__ out, int r, int head, int d, const float* x) {
  static_assert(kWidth == 4 || kWidth == 8, "stores of 8 or 16 bytes in bf16");
  const int64_t at = head * a.out_head + r * a.out_request + d;
  if constexpr (kType == 0) {
#pragma unroll
    for (int i = 0; i < kWidth; i += 4)
      *reinterpret_cast<f32x4*>(reinterpret_cast<float*>(out) + at + i) = f32x4{x[i], x[i + 1], x[i + 2], x[i + 3]};
  } else {
    uint32_t w[kWidth / 2];
#pragma unroll
    for (int i = 0; i < kWidth / 2; ++i) w[i] = bf16_pair(x[2 * i], x[2 * i + 1]);
    uint16_t* to = reinterpret_cast<uint16_t*>(out) + at;
    if constexpr (kWidth == 8)
      *reinterpret_cast<u32x4*>(to) = u32x4{w[0], w[1], w[2], w[3]};
    else
      *reinterpret_cast<u32x2*>(to) = u32x2{w[0], w[1]};
  }
}

// The finished output of kWidth dimensions; a query without a key has l = 0.
template <int kType, int kWidth>
__device__ inline void put_output(const DecodeArgs& a, char* __restrict__ out, float* __restrict__ lse, int r, int head, int d,
                                  const float* o, float m, float l) {
  const float f = l > 0.0f ? 1.0f / l : l;  // 0 and NaN stay
  float x[kWidth];
#pragma unroll
  for (int i = 0; i < kWidth; ++i) x[i] = o[i] * f;
  put_values<kType, kWidth>(a, out, r, head, d, x);
  if (lse && d == 0) lse[(int64_t)head * a.requests + r] = (m + __log2f(l)) * kLn2;
}

// A row that one wave has whole.
template <int kType, int kDim>
__device__ inline void put_row(const DecodeArgs& a, const State<kType, kDim>& st,
                               const Place<Shape<kType, kDim>::kGroups>& p, char* __restrict__ out, float* __restrict__ lse) {
  using S = Shape<kType, kDim>;
  const int lane = threadIdx.x & 63, g = lane >> 4, c = lane & 15;
  const float l = across_groups_sum(st.l);
  if (c >= p.heads) return;
#pragma unroll
  for (int x = 0; x < 4; ++x) {
    float o[S::kVDims];
#pragma unroll
    for (int i = 0; i < S::kVDims; ++i) o[i] = st.o[i][x];
    put_output<kType, S::kVDims>(a, out, lse, p.r, p.first + c, (4 * g + x) * S::kVDims, o, st.m, l);
  }
}

// A wave goes through `left` > 0 tiles from `next` on without a stop: the next tile's
// K is asked for as soon as the present scores are there, its V behind the present
// sums. advance(next) goes to the following tile and says whether it begins another
// row; done(state, place, from_start, ends) takes the part of a row. (Both asked for
// a whole tile ahead, in registers of their own: no faster anywhere, 16.7 / 20.7 us
// for 1024 rows of 512 tokens. One CU takes in 40 to 60 bytes a ns either way.)
template <int kType, int kDim, bool kScored, typename Advance, typename Done>
__device__ inline void walk(const DecodeArgs& a, const char* __restrict__ q, const char* __restrict__ k,
                            const char* __restrict__ v, const uint8_t* __restrict__ k_exp, const uint8_t* __restrict__ v_exp,
                            const int32_t* __restrict__ table, Place<Shape<kType, kDim>::kGroups>& next, int64_t left,
                            Advance advance, Done done) {
  using S = Shape<kType, kDim>;
  KeyTile<kType, kDim> kt;
  ValueTile<kType, kDim> vt;
  State<kType, kDim> st;
  uint32_t qw[S::kQWords], qn[S::kQWords];
  Bias<kScored> bias, bias_next = load_bias<kScored>(a, next);
  Entries entries{-1, 0, -1};
  load_queries<kType, kDim>(a, q, next, qn);
  look_up<kType>(a, table, entries, next);
  load_keys<kType, kDim>(a, k, k_exp, next, kt);
  load_values<kType, kDim>(a, v, v_exp, next, vt);
  bool begins = true;      // the tile is the wave's first of its row
  bool from_start = true;  // and that the row's first
  while (true) {
    const Place<S::kGroups> now = next;
    if (begins) {
#pragma unroll
      for (int i = 0; i < S::kQWords; ++i) qw[i] = qn[i];
      bias = bias_next;
      st.m = -INFINITY;
      st.l = 0.0f;
#pragma unroll
      for (int i = 0; i < S::kVDims; ++i) st.o[i] = f32x4{0, 0, 0, 0};
      from_start = now.x == 0;
    }
    f32x4 z[S::kGroups];
    score_tile<kType, kDim>(kt, qw, z);
    const bool ends = now.x + 1 == now.s.count;
    const bool last = --left == 0;
    if (!last) {
      if (advance(next)) {
        load_queries<kType, kDim>(a, q, next, qn);
        bias_next = load_bias<kScored>(a, next);
      }
      look_up<kType>(a, table, entries, next);
      load_keys<kType, kDim>(a, k, k_exp, next, kt);
    }
    add_tile<kType, kDim, kScored>(a, now, z, vt, st, bias);
    if (!last) load_values<kType, kDim>(a, v, v_exp, next, vt);
    begins = ends;
    if (ends || last) done(st, now, from_start, ends);
    if (last) break;
  }
}

// ------------------------------------------------- rows shared out among all

// Where a launch's pieces go: a row that falls to several workgroups leaves a part
// in each, workgroup w's in slot 2w if the row began before it and in slot 2w + 1 if
// it begins there. Each part: kDim sums per query, and (m, l).
struct Pieces {
  float* o;    // [2 kWorkgroups][heads][kDim]
  float2* ml;  // [2 kWorkgroups][heads]
  int4* cut;   // a row that begins in workgroup w and ends in a later one: (request, first query head and, from
               // bit 16 on, their number, w, last one), else z < 0
};
__host__ __device__ inline Pieces pieces(void* workspace, int heads) {
  Pieces p;
  p.cut = static_cast<int4*>(workspace);
  p.ml = reinterpret_cast<float2*>(static_cast<char*>(workspace) + kCutBytes);
  p.o = reinterpret_cast<float*>(p.ml + 2 * kWorkgroups * heads);
  return p;
}
// The next request after r that has tiles (64 lengths at a time), or `requests`.
__device__ inline int next_request(const DecodeArgs& a, const int32_t* __restrict__ lengths, int r) {
  const int lane = threadIdx.x & 63;
  for (++r; r < a.requests; r += 64) {
    const bool some = r + lane < a.requests && lengths[r + lane] > 0;
    const uint64_t found = __ballot(some);
    if (found) return __builtin_amdgcn_readfirstlane(r + __ffsll((unsigned long long)found) - 1);
  }
  return a.requests;
}

// The first tile of a wave's run.
template <int kMinTiles>
__device__ inline int64_t run_start(int64_t total, int wave) {
  return total < (int64_t)kWaves * kMinTiles ? min((int64_t)wave * kMinTiles, total) : total * wave / kWaves;
}
// The wave whose run holds tile x.
template <int kMinTiles>
__device__ inline int run_of(int64_t total, int64_t x) {
  return total < (int64_t)kWaves * kMinTiles ? (int)(x / kMinTiles) : (int)(((x + 1) * kWaves - 1) / total);
}

// The outputs of requests without a token, every kWorkgroups-th request; `first` is
// the first one's length.
template <int kType, int kDim>
__device__ inline void zero_rows(const DecodeArgs& a, const int32_t* __restrict__ lengths, char* __restrict__ out,
                                 float* __restrict__ lse, int w, int32_t first) {
  for (int r = w; r < a.requests; r += kWorkgroups) {
    if ((r == w ? first : lengths[r]) > 0) continue;
    for (int i = threadIdx.x; i < a.q_heads * (kDim / 4); i += kThreads) {
      const float none[4] = {0, 0, 0, 0};
      put_output<kType, 4>(a, out, lse, r, i / (kDim / 4), i % (kDim / 4) * 4, none, -INFINITY, 0.0f);
    }
  }
}

struct PartHead {
  int32_t r;
  int32_t first, heads;
  int32_t behind;  // tiles of the row behind the part
};

// The tiles of all requests' rows, request by request and row by row, are dealt out
// to the waves in equal runs of neighbouring tiles. Bound by HBM where the runs are
// long: one sequence of 274800 tokens 188 us with 16 heads of 64 in bf16 (6.0 TB/s of K
// and V), 64 of up to 10992 with 8 heads of 128 247 us (5.8), 192 in 8 bits 382 (5.7).
// Of a short launch 2 us go into counting and seeking, 1 to 4 into the first page and
// its K, 1 into the parts; the waves of a full chip end within 6 us of one another,
// those that came to the memory first ahead. In 4 bits 217 us for the 192 sequences (5.3
// TB/s); the long one of width 64, 77 us (3.9), is bound by instructions: two bytes of V a
// lane and key. With kScored the 64 take 249 us, as without; in 4
// bits, where the vector unit is busy already, the 192 248 (cap) and 254 (cap and bias), the long one 107.
template <int kType, int kDim, bool kScored>
__global__ __launch_bounds__(kThreads, 2) void paged_attention_kernel(
    const char* __restrict__ q, const char* __restrict__ k, const char* __restrict__ v,
    const uint8_t* __restrict__ k_exp, const uint8_t* __restrict__ v_exp, const int32_t* __restrict__ table,
    const int32_t* __restrict__ lengths, char* __restrict__ out, float* __restrict__ lse, void* __restrict__ workspace,
    DecodeArgs a) {
  using S = Shape<kType, kDim>;
  constexpr int kSlots = 2 * kGroupWaves;  // a wave's first row may have begun before it, its last may go on
  __shared__ union {
    struct {
      int64_t before[kThreads];  // tiles of the requests before a thread's
      int64_t wave_sum[kGroupWaves];
      int32_t length[kThreads];  // of a thread's first request
    } deal;
    Parts<kDim, kSlots> parts;
  } lds;
  __shared__ PartHead heads_of[kSlots];
  __shared__ int32_t ends_of[kSlots];  // 1: the row's last tile is in the part; 0: not; -1: no part
  const int lane = threadIdx.x & 63, wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
  const int rows = a.kv_heads * a.qtiles;
  const int w = blockIdx.x;
  const Pieces pc = pieces(workspace, piece_heads(a));

  const int32_t own_length = w < a.requests ? lengths[w] : 1;
  // where the runs lie: each thread counts neighbouring requests
  const int each = (a.requests + kThreads - 1) / kThreads;
  int64_t mine = 0;
  for (int i = 0; i < each; ++i) {
    const int r = threadIdx.x * each + i;
    const int32_t length = r < a.requests ? lengths[r] : 0;
    if (i == 0) lds.deal.length[threadIdx.x] = length;
    mine += span_of<S::kTile>(a, length).count;
  }
  mine *= rows;
  int64_t sum = mine;
#pragma unroll
  for (int d = 1; d < 64; d <<= 1) {
    const int64_t y = __shfl_up(sum, d);
    if (lane >= d) sum += y;
  }
  if (lane == 63) lds.deal.wave_sum[wave] = sum;
  if (threadIdx.x < kSlots) ends_of[threadIdx.x] = -1;
  __syncthreads();
  int64_t total = 0;
#pragma unroll
  for (int i = 0; i < kGroupWaves; ++i) {
    if (i == wave) sum += total;
    total += lds.deal.wave_sum[i];
  }
  lds.deal.before[threadIdx.x] = sum - mine;
  __syncthreads();

  if (threadIdx.x == 0) pc.cut[w].z = -1;
  if (run_start<S::kMinTiles>(total, w * kGroupWaves) >= total) {  // the whole workgroup
    zero_rows<kType, kDim>(a, lengths, out, lse, w, own_length);
    return;
  }
  const int64_t lo = run_start<S::kMinTiles>(total, w * kGroupWaves + wave);
  const int64_t hi = run_start<S::kMinTiles>(total, w * kGroupWaves + wave + 1);

  Place<S::kGroups> next;
  if (lo < hi) {
    // the first tile's request: the thread whose requests hold it, then these one by one
    int owner = -1;
#pragma unroll
    for (int i = 0; i < kGroupWaves; ++i) owner += __popcll(__ballot(lds.deal.before[64 * i + lane] <= lo));
    int64_t off = lo - lds.deal.before[owner];
    next.r = __builtin_amdgcn_readfirstlane(owner * each);
    next.s = span_of<S::kTile>(a, __builtin_amdgcn_readfirstlane(lds.deal.length[owner]));
    while (off >= (int64_t)next.s.count * rows) {
      off -= (int64_t)next.s.count * rows;
      next.s = span_of<S::kTile>(a, lengths[++next.r]);
    }
    // a division of 64 bits is a tenth of the time before the first load
    const int32_t row = __builtin_amdgcn_readfirstlane(
        off >> 32 == 0 ? (int32_t)((uint32_t)off / (uint32_t)next.s.count) : (int32_t)(off / next.s.count));
    next.x = __builtin_amdgcn_readfirstlane((int32_t)(off - (int64_t)row * next.s.count));
    next.h = a.qtiles == 1 ? row : row / a.qtiles;
    next.qt = row - next.h * a.qtiles;
    next.set_row(a);
  }
  __syncthreads();  // the parts go where the counts were
  if (lo < hi) {
    walk<kType, kDim, kScored>(
        a, q, k, v, k_exp, v_exp, table, next, hi - lo,
        [&](Place<S::kGroups>& p) {
          if (++p.x < p.s.count) return false;
          if (!p.next_row(a)) {
            p.r = next_request(a, lengths, p.r);
            p.s = span_of<S::kTile>(a, lengths[p.r]);
          }
          return true;
        },
        [&](const State<kType, kDim>& st, const Place<S::kGroups>& p, bool from_start, bool ends) {
          if (from_start && ends) {
            put_row<kType, kDim>(a, st, p, out, lse);
          } else {
            const int slot = 2 * wave + (from_start ? 1 : 0);
            put_part<kType>(lds.parts, slot, st);
            if (lane == 0) {
              heads_of[slot] = PartHead{p.r, p.first, p.heads, p.s.count - 1 - p.x};
              ends_of[slot] = ends ? 1 : 0;
            }
          }
        });
  }
  __syncthreads();

  // the parts in their order: those of one row follow one another
  constexpr int kWidth = kDim * 16 / kThreads;
  const int c = threadIdx.x >> 4, d = (threadIdx.x & 15) * kWidth;
  Sums<kWidth> sums;
  bool open = false, begun = false;
  int32_t ends[kSlots];
#pragma unroll
  for (int i = 0; i < kSlots; ++i) ends[i] = __builtin_amdgcn_readfirstlane(ends_of[i]);
  int last = -1;  // the last slot that holds a part
#pragma unroll
  for (int i = 0; i < kSlots; ++i) last = ends[i] >= 0 ? i : last;
#pragma unroll
  for (int slot = 0; slot < kSlots; ++slot) {
    if (ends[slot] < 0) continue;
    if (!open) {
      sums.clear();
      begun = (slot & 1) != 0;
      open = true;
    }
    sums.add(&lds.parts.o[slot][c][d], lds.parts.ml[slot][c]);
    if (ends[slot] == 0 && slot < last) continue;  // the row goes on in this workgroup
    open = false;
    const PartHead h = heads_of[slot];
    const bool mine_too = c < h.heads;
    if (begun && ends[slot] == 1) {
      if (mine_too) put_output<kType, kWidth>(a, out, lse, h.r, h.first + c, d, sums.o, sums.m, sums.l);
    } else {
      if (mine_too) {
        const int at = (2 * w + (begun ? 1 : 0)) * piece_heads(a) + c;
        if (d == 0) pc.ml[at] = float2{sums.m, sums.l};
#pragma unroll
        for (int i = 0; i < kWidth; i += 4)
          *reinterpret_cast<f32x4*>(pc.o + (int64_t)at * kDim + d + i) = f32x4{sums.o[i], sums.o[i + 1], sums.o[i + 2], sums.o[i + 3]};
      }
      if (begun && threadIdx.x == 0) {
        const int64_t end = run_start<S::kMinTiles>(total, (w + 1) * kGroupWaves) + h.behind - 1;  // the row's last tile
        pc.cut[w] = int4{h.r, h.first | h.heads << 16, w, run_of<S::kMinTiles>(total, end) / kGroupWaves};
      }
    }
  }
  zero_rows<kType, kDim>(a, lengths, out, lse, w, own_length);
}

// The rows that fell to several workgroups, in the order of these: one workgroup per
// such row and query; its 16-byte lanes take kThreads * 4 / kDim pieces at a time. 2.7
// to 4.9 us: the latency of the list, the pieces and the last sums.
template <int kType, int kDim>
__global__ __launch_bounds__(kThreads) void paged_join_kernel(const void* __restrict__ workspace, char* __restrict__ out,
                                                              float* __restrict__ lse, DecodeArgs a) {
  constexpr int kLanes = kDim / 4, kAtOnce = kThreads / kLanes;
  __shared__ float part[kAtOnce][kDim];
  __shared__ float2 part_ml[kAtOnce];
  const Pieces pc = pieces(const_cast<void*>(workspace), piece_heads(a));
  const int4 cut = pc.cut[blockIdx.x];
  if (cut.z < 0) return;
  const int n = blockIdx.y;
  if (n >= cut.y >> 16) return;
  const int slot = threadIdx.x / kLanes, d = threadIdx.x % kLanes * 4;
  const int count = cut.w - cut.z + 1;
  Sums<4> sums;
  sums.clear();
  for (int i = slot; i < count; i += kAtOnce) {
    const int at = (2 * (cut.z + i) + (i == 0 ? 1 : 0)) * piece_heads(a) + n;
    const f32x4 x = *reinterpret_cast<const f32x4*>(pc.o + (int64_t)at * kDim + d);
    const float y[4] = {x[0], x[1], x[2], x[3]};
    sums.add(y, pc.ml[at]);
  }
#pragma unroll
  for (int i = 0; i < 4; ++i) part[slot][d + i] = sums.o[i];
  if (d == 0) part_ml[slot] = float2{sums.m, sums.l};
  __syncthreads();
  if (slot > 0) return;
#pragma unroll
  for (int i = 1; i < kAtOnce; ++i) sums.add(&part[i][d], part_ml[i]);
  put_output<kType, 4>(a, out, lse, cut.x, (cut.y & 0xffff) + n, d, sums.o, sums.m, sums.l);
}

// --------------------------------------------------------------- whole rows

// One workgroup per row: its waves take equal runs of the row's tiles and add up in
// LDS. No counting, no pieces, no second launch. Bound by one CU's intake where rows are
// few and long (whole_rows), by memory where they are many. Short ones wait for a chain
// of latencies (a length, the table, K and V, the sums): requests of up to 261 tokens of 4
// heads of 64 in bf16 take 5.3 us, be it one or 32, 256 of them (35 MB) 9.8, 1024 33 (4.3
// TB/s), 2048 62 (4.6 TB/s).
template <int kType, int kDim, bool kScored>
__global__ __launch_bounds__(kRowThreads, 2) void paged_rows_kernel(
    const char* __restrict__ q, const char* __restrict__ k, const char* __restrict__ v,
    const uint8_t* __restrict__ k_exp, const uint8_t* __restrict__ v_exp, const int32_t* __restrict__ table,
    const int32_t* __restrict__ lengths, char* __restrict__ out, float* __restrict__ lse, DecodeArgs a) {
  using S = Shape<kType, kDim>;
  __shared__ Parts<kDim, kRowWaves> lds;
  const int wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
  const int rows = a.kv_heads * a.qtiles;
  Place<S::kGroups> next;
  next.r = blockIdx.x / rows;
  next.h = (blockIdx.x - next.r * rows) / a.qtiles;
  next.qt = blockIdx.x - next.r * rows - next.h * a.qtiles;
  next.set_row(a);
  next.s = span_of<S::kTile>(a, lengths[next.r]);
  const int32_t lo = (int32_t)((int64_t)next.s.count * wave / kRowWaves), hi = (int32_t)((int64_t)next.s.count * (wave + 1) / kRowWaves);
  next.x = lo;
  State<kType, kDim> none;
  none.m = -INFINITY;
  none.l = 0.0f;
#pragma unroll
  for (int i = 0; i < S::kVDims; ++i) none.o[i] = f32x4{0, 0, 0, 0};
  const int r = next.r, first = next.first, heads = next.heads;
  if (lo < hi)
    walk<kType, kDim, kScored>(
        a, q, k, v, k_exp, v_exp, table, next, hi - lo,
        [&](Place<S::kGroups>& p) {
          ++p.x;
          return false;
        },
        [&](const State<kType, kDim>& st, const Place<S::kGroups>&, bool, bool) { put_part<kType>(lds, wave, st); });
  else
    put_part<kType>(lds, wave, none);
  __syncthreads();
  constexpr int kWidth = kDim * 16 / kRowThreads;
  const int c = threadIdx.x / (kRowThreads / 16), d = threadIdx.x % (kRowThreads / 16) * kWidth;
  if (c >= heads) return;
  Sums<kWidth> sums;
  sums.clear();
#pragma unroll
  for (int i = 0; i < kRowWaves; ++i) sums.add(&lds.o[i][c][d], lds.ml[i][c]);
  put_output<kType, kWidth>(a, out, lse, r, first + c, d, sums.o, sums.m, sums.l);
}

template <int kType, int kDim, bool kScored>
hipError_t launch(const void* q, const void* kp, const void* vp, const uint8_t* ke, const uint8_t* ve, const int32_t* table,
                  const int32_t* lengths, void* out, float* lse, void* workspace, const DecodeArgs& a, hipStream_t s) {
  if (whole_rows(kType, kDim, a)) {
    hipLaunchKernelGGL((paged_rows_kernel<kType, kDim, kScored>), dim3((unsigned)(a.requests * a.kv_heads * a.qtiles)), dim3(kRowThreads),
                       0, s, static_cast<const char*>(q), static_cast<const char*>(kp), static_cast<const char*>(vp), ke, ve,
                       table, lengths, static_cast<char*>(out), lse, a);
    return hipGetLastError();
  }
  hipLaunchKernelGGL((paged_attention_kernel<kType, kDim, kScored>), dim3(kWorkgroups), dim3(kThreads), 0, s,
                     static_cast<const char*>(q), static_cast<const char*>(kp), static_cast<const char*>(vp), ke, ve, table,
                     lengths, static_cast<char*>(out), lse, workspace, a);
  const hipError_t e = hipGetLastError();
  if (e != hipSuccess) return e;
  hipLaunchKernelGGL((paged_join_kernel<kType, kDim>), dim3(kWorkgroups, (unsigned)piece_heads(a)), dim3(kThreads), 0, s, workspace,
                     static_cast<char*>(out), lse, a);
  return hipGetLastError();
}

}  // namespace

hipError_t launch_paged_attention(int dtype, int dim, const void* q, const void* k_pages,
                                  const void* v_pages, const uint8_t* k_exp, const uint8_t* v_exp,
                                  const int32_t* table, const int32_t* lengths, void* out, float* lse,
                                  void* workspace, const DecodeArgs& a, hipStream_t s) {
  const bool scored = a.cap_in != 0.0f || a.slopes;
#define SAF3R_CASE(T, D)                                                                                                      \
  if (dtype == T && dim == D)                                                                                                 \
  return scored ? launch<T, D, true>(q, k_pages, v_pages, k_exp, v_exp, table, lengths, out, lse, workspace, a, s) \
                : launch<T, D, false>(q, k_pages, v_pages, k_exp, v_exp, table, lengths, out, lse, workspace, a, s)
  SAF3R_CASE(0, 64);
  SAF3R_CASE(0, 128);
  SAF3R_CASE(1, 64);
  SAF3R_CASE(1, 128);
  SAF3R_CASE(2, 64);
  SAF3R_CASE(2, 128);
  SAF3R_CASE(4, 64);
  SAF3R_CASE(4, 128);
#undef SAF3R_CASE
  return hipErrorInvalidValue;
}

}  // namespace saf3r
