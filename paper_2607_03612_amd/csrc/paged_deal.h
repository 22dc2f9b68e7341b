// How the attention of several new tokens cuts its work: the tiles of a request's rows, the
// keys of a tile, and the runs of steps that workgroups take.
#pragma once

#include "paged_internal.h"

namespace saf3r {

constexpr int kKeys = 32;  // of a step

// A workgroup's tile of rows, and the keys that some row of it sees: in steps of 32
// keys, the first `head` and from step head + skip on, `count` in all.
struct Tile {
  int32_t r, n;         // request, its tokens
  int32_t first;        // its first new token, of q
  int32_t fresh, rows;  // its new tokens; times the heads of a group
  int32_t row;          // the tile's first row
  int32_t prefix;
  int32_t head, skip, count;
};

// A row: a token and a query head, and the keys that it sees: [0, below) and [from, place].
struct Row {
  int32_t token, head;  // of q's, the head within the group
  int32_t place, below, from;
};
__host__ __device__ inline Row row_of(const PromptArgs& a, const Tile& t, int32_t m) {
  m = min(m, t.rows - 1);
  Row w;
  const int32_t i = m / a.group;
  w.token = t.first + i;
  w.head = m - i * a.group;
  w.place = t.n - t.fresh + i;
  w.below = t.prefix;
  w.from = 0;
  if (a.window > 0) {
    w.below = max(w.below, min(a.anchor, w.place + 1));
    w.from = w.place + 1 - a.window;
  }
  return w;
}

// The number of a request's first tile: floor(its first row / rows of a tile) + r, so that
// between two requests' lie as many as the first has, or more, without a sum over requests.
__host__ __device__ inline int32_t start_of(const PromptArgs& a, const int32_t* __restrict__ start, int32_t r) {
  return min(max(start[r], 0), a.tokens);
}
template <int kRows>
__host__ __device__ inline int32_t number_of(const PromptArgs& a, int32_t first, int32_t r) {
  return first * a.group / kRows + r;
}

// Tile number x as one of request r's; count 0 if it has no such tile.
template <int kRows>
__host__ __device__ inline Tile tile_of(const PromptArgs& a, const int32_t* __restrict__ lengths, const int32_t* __restrict__ prefix,
                                        int32_t r, int32_t first, int32_t end, int32_t x) {
  Tile t;
  t.r = r;
  t.first = first;
  t.fresh = end - first;
  t.rows = t.fresh * a.group;  // none where the end lies before the start
  t.count = 0;
  const int64_t row = (int64_t)(x - number_of<kRows>(a, first, r)) * kRows;
  if (row < 0 || row >= t.rows) return t;  // before all requests, or none of its own
  t.row = (int32_t)row;
  t.n = min(max(lengths[r], 0), a.max_pages * a.page.size);
  t.prefix = prefix ? min(max(prefix[r], 0), t.n) : 0;
  const Row low = row_of(a, t, t.row), high = row_of(a, t, t.row + kRows - 1);
  t.head = (high.below + kKeys - 1) / kKeys;
  const int32_t from = max(max(low.from, 0) / kKeys, t.head), end_step = (max(high.place, -1) + kKeys) / kKeys;
  t.skip = from - t.head;
  t.count = t.head + max(end_step - from, 0);
  return t;
}

// A run is this long or longer: what lies ahead of a run's first step and behind its last
// takes as long as several.
constexpr int kMinRun = 8;
__host__ __device__ inline int64_t run_start(const PromptArgs& a, int64_t total, int w) {
  return total < (int64_t)a.groups * kMinRun ? min((int64_t)w * kMinRun, total) : total * w / a.groups;
}
// The run that has step x. Where starts go back, the count of the steps and the walk over them may
// give a tile to different requests, and a tile's last step lie behind the last one counted: it
// is the last run's then, whose part is there to be read.
__host__ __device__ inline int run_of(const PromptArgs& a, int64_t total, int64_t x) {
  const int64_t w = total < (int64_t)a.groups * kMinRun ? x / kMinRun : ((x + 1) * a.groups - 1) / total;
  return (int)min(w, (int64_t)a.groups - 1);
}

}  // namespace saf3r
