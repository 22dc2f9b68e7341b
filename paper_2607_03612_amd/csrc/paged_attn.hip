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

constexpr int kWaves = 4;
constexpr int kThreads = 64 * kWaves;
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
struct Tile {
  using S = Shape<kType, kDim>;
  uint32_t k[S::kGroups][S::kKWords];
  uint32_t v[S::kGroups][4][S::kVWords];
  uint32_t k_exp[S::kGroups];  // e4m3: of key lane % 16
  uint32_t v_exp[S::kGroups];  // of keys 4g .. 4g + 3
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

// A request's row of the table and a head of the pages.
struct Source {
  const int32_t* row;
  const char* k;
  const char* v;
  const uint8_t* k_exp;
  const uint8_t* v_exp;
  int64_t exp_page;  // entries of a page's exponents
};

// The pages of a tile's groups; -1 for one that holds no token or whose entry is
// no page.
template <int kGroups>
__device__ inline void look_up(const DecodeArgs& a, const Source& src, const Span& s, int32_t tile, int32_t (&page)[kGroups]) {
#pragma unroll
  for (int u = 0; u < kGroups; ++u) {
    const int32_t pos = tile * (16 * kGroups) + 16 * u;
    page[u] = -1;
    if (pos < s.n) page[u] = src.row[div_page(a.page, pos)];
    if (page[u] < 0 || page[u] >= a.pages) page[u] = -1;
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

// Reads stay inside pages: an absent page's keys are read from page 0 (which
// exists) and masked, and so are the tokens of the last page behind the end.
template <int kType, int kDim>
__device__ inline void load_tile(const DecodeArgs& a, const Source& src, int32_t tile,
                                 const int32_t (&page)[Shape<kType, kDim>::kGroups], Tile<kType, kDim>& t) {
  using S = Shape<kType, kDim>;
  const int lane = threadIdx.x & 63, g = lane >> 4, c = lane & 15;
#pragma unroll
  for (int u = 0; u < S::kGroups; ++u) {
    const int32_t pos = tile * S::kTile + 16 * u;
    const int32_t p = max(page[u], 0);
    const int32_t in = page[u] < 0 ? 0 : pos - div_page(a.page, pos) * a.page.size;
    const int64_t at = p * a.page_stride + (int64_t)in * a.token_stride;
    // K: row lane % 16, the pieces of 16 bytes g, g + 4, ...
    const char* k = src.k + at + (uint32_t)(c * a.token_stride + g * 16);
#pragma unroll
    for (int w = 0; w < S::kKWords / 4; ++w) load_words<4>(&t.k[u][4 * w], k + 64 * w);
    // V: rows 4g .. 4g + 3, dimensions from (lane % 16) kDim / 16 on
#pragma unroll
    for (int r = 0; r < 4; ++r)
      load_words<S::kVWords>(t.v[u][r], src.v + at + (uint32_t)((4 * g + r) * a.token_stride + c * (S::kVDims * S::kSize)));
    if constexpr (kType == 2) {
      const int64_t e = p * src.exp_page + in;
      t.k_exp[u] = src.k_exp[e + c];
      t.v_exp[u] = *reinterpret_cast<const uint32_t*>(src.v_exp + e + 4 * g);
    }
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

// One tile into the running softmax. With scores z in log2 units and the running
// maximum m, every new maximum scales what is summed so far by 2^(m - m').
template <int kType, int kDim>
__device__ inline void attend_tile(const DecodeArgs& a, const Span& s, int32_t tile,
                                   const int32_t (&page)[Shape<kType, kDim>::kGroups], Tile<kType, kDim>& t,
                                   const uint32_t (&q)[Shape<kType, kDim>::kQWords], State<kType, kDim>& st) {
  using S = Shape<kType, kDim>;
  const int g = (threadIdx.x & 63) >> 4;
  f32x4 z[S::kGroups];
#pragma unroll
  for (int u = 0; u < S::kGroups; ++u) {
    z[u] = f32x4{0, 0, 0, 0};
    if constexpr (kType == 0) {
#pragma unroll
      for (int w = 0; w < kDim / 4; ++w)
        z[u] = __builtin_amdgcn_mfma_f32_16x16x4f32(__uint_as_float(t.k[u][w]), __uint_as_float(q[w]), z[u], 0, 0, 0);
    } else if constexpr (kType == 1) {
#pragma unroll
      for (int w = 0; w < kDim / 32; ++w)
        z[u] = __builtin_amdgcn_mfma_f32_16x16x32_bf16(
            as_bf16x8(t.k[u][4 * w], t.k[u][4 * w + 1], t.k[u][4 * w + 2], t.k[u][4 * w + 3]),
            as_bf16x8(q[4 * w], q[4 * w + 1], q[4 * w + 2], q[4 * w + 3]), z[u], 0, 0, 0);
    } else {
      const float scale = __uint_as_float(t.k_exp[u] << 23);
#pragma unroll
      for (int w = 0; w < kDim / 32; ++w) {
        const uint32_t c0 = t.k[u][2 * w], c1 = t.k[u][2 * w + 1];
        z[u] = __builtin_amdgcn_mfma_f32_16x16x32_bf16(
            as_bf16x8(fp8_pair(c0, false, scale), fp8_pair(c0, true, scale), fp8_pair(c1, false, scale),
                      fp8_pair(c1, true, scale)),
            as_bf16x8(q[4 * w], q[4 * w + 1], q[4 * w + 2], q[4 * w + 3]), z[u], 0, 0, 0);
      }
    }
  }
  // tiles at an end of the kept tokens, or with an absent page: a masked key's
  // score is -inf and its V row 0, whatever memory holds there
  const int32_t first = tile * S::kTile, last = first + S::kTile;
  bool whole = last <= s.n && (last <= s.anchor || first >= s.from);
#pragma unroll
  for (int u = 0; u < S::kGroups; ++u) whole = whole && page[u] >= 0;
  if (!whole) {
#pragma unroll
    for (int u = 0; u < S::kGroups; ++u)
#pragma unroll
      for (int r = 0; r < 4; ++r) {
        const int32_t j = first + 16 * u + 4 * g + r;
        const bool keep = page[u] >= 0 && j < s.n && (j < s.anchor || j >= s.from);
        if (!keep) {
          z[u][r] = -INFINITY;
#pragma unroll
          for (int w = 0; w < S::kVWords; ++w) t.v[u][r][w] = 0;
          if constexpr (kType == 2) t.v_exp[u] = (t.v_exp[u] & ~(0xffu << (8 * r))) | 1u << (8 * r);
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
          st.o[i] = __builtin_amdgcn_mfma_f32_16x16x4f32(__uint_as_float(t.v[u][r][i]), p[u][r], st.o[i], 0, 0, 0);
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
            vw[x][w] = t.v[u + (x >> 2)][x & 3][w];
          } else {
            const float scale = __uint_as_float(((t.v_exp[u + (x >> 2)] >> (8 * (x & 3))) & 0xffu) << 23);
            vw[x][w] = fp8_pair(t.v[u + (x >> 2)][x & 3][w >> 1], w & 1, scale);
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
__device__ inline void load_queries(const DecodeArgs& a, const char* q, int r, int first, int heads,
                                    uint32_t (&w)[Shape<kType, kDim>::kQWords]) {
  using S = Shape<kType, kDim>;
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

template <int kType, int kDim>
struct Merge {
  static constexpr int kRow = kDim + 4;  // floats of a query's row in LDS
  float o[kWaves][16][kRow];
  float m[kWaves][16];
  float l[kWaves][16];
};

template <int kType, int kDim>
__device__ inline void put_state(Merge<kType, kDim>& lds, int wave, const State<kType, kDim>& st) {
  using S = Shape<kType, kDim>;
  const int lane = threadIdx.x & 63, g = lane >> 4, c = lane & 15;
  const float l = across_groups_sum(st.l);
  if (g == 0) {
    lds.m[wave][c] = st.m;
    lds.l[wave][c] = l;
  }
#pragma unroll
  for (int r = 0; r < 4; ++r)
#pragma unroll
    for (int i = 0; i < S::kVDims; i += 4)
      *reinterpret_cast<f32x4*>(&lds.o[wave][c][(4 * g + r) * S::kVDims + i]) =
          f32x4{st.o[i][r], st.o[i + 1][r], st.o[i + 2][r], st.o[i + 3][r]};
}

// The outputs of one thread: kDim / 16 dimensions of query threadIdx.x / 16.
template <int kType, int kDim>
__device__ inline void put_output(const DecodeArgs& a, char* out, float* lse, int r, int head, const float* o, float m, float l) {
  constexpr int kVDims = kDim / 16;
  const float f = l > 0.0f ? 1.0f / l : l == 0.0f ? 0.0f : l;  // NaN stays
  const int64_t at = head * a.out_head + r * a.out_request + (threadIdx.x & 15) * kVDims;
  if constexpr (kType == 0) {
    float* to = reinterpret_cast<float*>(out) + at;
#pragma unroll
    for (int i = 0; i < kVDims; i += 4) *reinterpret_cast<f32x4*>(to + i) = f32x4{o[i] * f, o[i + 1] * f, o[i + 2] * f, o[i + 3] * f};
  } else {
    uint32_t* to = reinterpret_cast<uint32_t*>(reinterpret_cast<uint16_t*>(out) + at);
#pragma unroll
    for (int i = 0; i < kVDims; i += 4)
      *reinterpret_cast<u32x2*>(to + i / 2) = u32x2{bf16_pair(o[i] * f, o[i + 1] * f), bf16_pair(o[i + 2] * f, o[i + 3] * f)};
  }
  if (lse && (threadIdx.x & 15) == 0) lse[(int64_t)head * a.requests + r] = (m + __log2f(l)) * kLn2;
}

// One workgroup per request, key-value head and tile of its query heads; its
// four waves take the tiles in turn.
template <int kType, int kDim>
__global__ __launch_bounds__(kThreads, 2) void paged_attention_kernel(
    const char* __restrict__ q, const char* __restrict__ k, const char* __restrict__ v,
    const uint8_t* __restrict__ k_exp, const uint8_t* __restrict__ v_exp, const int32_t* __restrict__ table,
    const int32_t* __restrict__ lengths, char* __restrict__ out, float* __restrict__ lse, DecodeArgs a) {
  using S = Shape<kType, kDim>;
  __shared__ Merge<kType, kDim> lds;
  const int wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
  const int qt = blockIdx.x % a.qtiles;
  const int h = blockIdx.x / a.qtiles % a.kv_heads;
  const int r = blockIdx.x / a.qtiles / a.kv_heads;
  const int heads = min(a.group - 16 * qt, 16), first = h * a.group + 16 * qt;
  Source src;
  src.row = table + (int64_t)r * a.max_pages;
  src.k = k + h * a.head_stride;
  src.v = v + h * a.head_stride;
  src.exp_page = (int64_t)a.kv_heads * a.page.size;
  src.k_exp = k_exp + h * a.page.size;
  src.v_exp = v_exp + h * a.page.size;
  const Span s = span_of<S::kTile>(a, lengths[r]);
  uint32_t qw[S::kQWords];
  load_queries<kType, kDim>(a, q, r, first, heads, qw);
  State<kType, kDim> st;
  st.m = -INFINITY;
  st.l = 0.0f;
#pragma unroll
  for (int i = 0; i < S::kVDims; ++i) st.o[i] = f32x4{0, 0, 0, 0};
  for (int32_t x = wave; x < s.count; x += kWaves) {
    const int32_t tile = x < s.head ? x : x + s.skip;
    int32_t page[S::kGroups];
    Tile<kType, kDim> t;
    look_up<S::kGroups>(a, src, s, tile, page);
    load_tile<kType, kDim>(a, src, tile, page, t);
    attend_tile<kType, kDim>(a, s, tile, page, t, qw, st);
  }
  put_state<kType, kDim>(lds, wave, st);
  __syncthreads();
  const int query = threadIdx.x >> 4, part = threadIdx.x & 15;
  if (query >= heads) return;
  float m = -INFINITY;
#pragma unroll
  for (int w = 0; w < kWaves; ++w) m = fmaxf(m, lds.m[w][query]);
  float l = 0.0f, o[S::kVDims] = {};
#pragma unroll
  for (int w = 0; w < kWaves; ++w) {
    const float f = lds.m[w][query] == -INFINITY ? 0.0f : exp2_fast(lds.m[w][query] - m);
    l = fmaf(lds.l[w][query], f, l);
#pragma unroll
    for (int i = 0; i < S::kVDims; ++i) o[i] = fmaf(lds.o[w][query][part * S::kVDims + i], f, o[i]);
  }
  put_output<kType, kDim>(a, out, lse, r, first + query, o, m, l);
}

template <int kType, int kDim>
hipError_t launch(const void* q, const void* kp, const void* vp, const uint8_t* ke, const uint8_t* ve, const int32_t* table,
                  const int32_t* lengths, void* out, float* lse, const DecodeArgs& a, hipStream_t s) {
  const int64_t groups = (int64_t)a.requests * a.kv_heads * a.qtiles;
  hipLaunchKernelGGL((paged_attention_kernel<kType, kDim>), dim3((unsigned)groups), dim3(kThreads), 0, s,
                     static_cast<const char*>(q), static_cast<const char*>(kp), static_cast<const char*>(vp), ke, ve, table,
                     lengths, static_cast<char*>(out), lse, a);
  return hipGetLastError();
}

}  // namespace

int64_t paged_attention_workspace(int, const DecodeArgs&) { return 0; }

hipError_t launch_paged_attention(int dtype, int dim, const void* q, const void* k_pages,
                                  const void* v_pages, const uint8_t* k_exp, const uint8_t* v_exp,
                                  const int32_t* table, const int32_t* lengths, void* out, float* lse,
                                  void*, const DecodeArgs& a, hipStream_t s) {
#define SAF3R_CASE(T, D) \
  if (dtype == T && dim == D) return launch<T, D>(q, k_pages, v_pages, k_exp, v_exp, table, lengths, out, lse, a, s)
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
