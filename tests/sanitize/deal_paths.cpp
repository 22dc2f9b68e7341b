// The dealing out of prompt attention's steps (paged_deal.h) as its kernels go through it, on the CPU: a workgroup's
// search for its run, its walk from tile to tile, the parts it leaves and the list of cut tiles. Every index into the
// workspace and the rows has to lie inside, whatever the starts and lengths; where the starts ascend every step has to
// be taken once, and a cut tile's last part be where the list says. Prints the first case that fails; 0 if none does.
#include <algorithm>
#include <cstdio>
#include <cstring>
#include <random>
#include <set>
#include <tuple>
#include <vector>

using std::max;
using std::min;
#include "../../paper_2607_03612_amd/csrc/paged_deal.h"

using namespace saf3r;

namespace {

constexpr int kThreads = 256;

struct Case {
  int dtype, dim;
  PromptArgs a;
  std::vector<int32_t> lengths, start, prefix;
};

// 64 requests at a time, the highest that is reached, as a wave does.
template <int kRows>
int32_t request_of(const Case& c, int32_t x) {
  int32_t lo = 0, hi = c.a.requests;
  while (true) {
    const int32_t step = (hi - lo + 63) / 64;
    int best = -1;
    for (int lane = 0; lane < 64; ++lane) {
      const int32_t r = lo + lane * step;
      if (r < hi && number_of<kRows>(c.a, start_of(c.a, c.start.data(), r), r) <= x) best = lane;
    }
    if (best < 0) return 0;
    lo += best * step;
    if (step == 1) return lo;
    hi = min(lo + step, hi);
  }
}

template <int kRows>
Tile next_tile(const Case& c, int32_t r, int32_t x) {
  const PromptArgs& a = c.a;
  int32_t first = start_of(a, c.start.data(), r), end = start_of(a, c.start.data(), r + 1);
  while (r + 1 < a.requests && number_of<kRows>(a, end, r + 1) <= x) {
    ++r;
    first = end;
    end = start_of(a, c.start.data(), r + 1);
  }
  return tile_of<kRows>(a, c.lengths.data(), c.prefix.empty() ? nullptr : c.prefix.data(), r, first, end, x);
}

#define NEED(what)                                    \
  do {                                                \
    if (!(what)) {                                    \
      std::printf("failed: %s\n", #what);             \
      return false;                                   \
    }                                                 \
  } while (0)

template <int kRows>
bool check(const Case& c, bool ascending) {
  const PromptArgs& a = c.a;
  if (a.groups == 0) return true;
  NEED(a.requests <= kMaxDealt && a.groups <= kMaxGroups);  // as many starts are kept in LDS
  // find_run's count, each thread that of neighbouring tiles
  const int32_t each = (a.tiles + kThreads - 1) / kThreads;
  std::vector<int64_t> before(kThreads);
  int64_t head = 0;
  for (int thread = 0; thread < kThreads; ++thread) {
    before[thread] = head;
    const int32_t x0 = thread * each;
    if (x0 >= a.tiles) continue;
    int32_t r = 0, hi = a.requests;
    while (hi - r > 1) {
      const int32_t mid = (r + hi) >> 1;
      if (number_of<kRows>(a, start_of(a, c.start.data(), mid), mid) <= x0) r = mid;
      else hi = mid;
    }
    for (int32_t x = x0; x < min(x0 + each, a.tiles); ++x) {
      const Tile t = next_tile<kRows>(c, r, x);
      r = t.r;
      head += t.count;
    }
  }
  const int64_t total = head * a.kv_heads;
  // where the steps taken so far end: in this tile of this head before this step, of so many
  int last_x = -1, last_h = 0, last_step = 0, last_count = 0;
  int64_t taken = 0;
  std::set<std::tuple<int, int, int>> parts;  // slot: tile, head and whose it is
  std::vector<std::tuple<int, int, int, int>> cuts;  // first and last workgroup, tile, head
  for (int w = 0; w < a.groups; ++w) {
    int64_t at = run_start(a, total, w), left = run_start(a, total, w + 1) - at;
    NEED(at >= 0 && left >= 0 && at + left <= total);
    if (left <= 0) continue;
    int32_t h = (int32_t)(at / head);
    int64_t off = at - h * head;
    int owner = -1;
    for (int i = 0; i < kThreads; ++i) owner += before[i] <= off;
    NEED(owner >= 0);
    off -= before[owner];
    int32_t x = owner * each;
    Tile t{};
    int32_t r = request_of<kRows>(c, x);
    for (; x < a.tiles; ++x) {
      t = next_tile<kRows>(c, r, x);
      r = t.r;
      if (off < t.count) break;
      off -= t.count;
    }
    if (x == a.tiles) {
      NEED(!ascending);
      continue;
    }
    int32_t step = (int32_t)off;
    while (true) {
      const int32_t hi = (int32_t)min((int64_t)t.count, step + left);
      NEED(step >= 0 && step < hi && h >= 0 && h < a.kv_heads);
      NEED(t.row >= 0 && t.row < t.rows && t.first >= 0 && t.first + t.fresh <= a.tokens);
      NEED(((hi - 1 < t.head ? hi - 1 : hi - 1 + t.skip) * (int64_t)kKeys) < t.n);
      if (ascending) {
        if (x == last_x && h == last_h)
          NEED(step == last_step);
        else
          NEED(step == 0 && last_step == last_count && (h > last_h || (h == last_h && x > last_x)));
        last_x = x;
        last_h = h;
        last_step = hi;
        last_count = t.count;
        taken += hi - step;
      }
      const bool whole = step == 0 && t.count <= left;
      if (!whole) {
        const int slot = 2 * w + (step == 0 ? 1 : 0);
        NEED(slot < 2 * a.groups && min(t.rows - t.row, kRows) <= a.slot_rows);
        parts.insert({slot, x, h});
      }
      if (step == 0 && t.count > left) {
        const int to = run_of(a, total, at + (t.count - 1));
        // the join reads the parts of workgroups w .. to
        NEED(to >= w && to < a.groups);
        cuts.push_back({w, to, x, h});
      }
      const int32_t steps = (int32_t)min((int64_t)(t.count - step), left);
      if (left == steps) break;
      left -= steps;
      at += steps;
      step = 0;
      bool over = false;
      r = t.r;
      do {
        if (++x == a.tiles) {
          x = 0;
          r = 0;
          if (++h >= a.kv_heads) {
            over = true;
            break;
          }
        }
        t = next_tile<kRows>(c, r, x);
        r = t.r;
      } while (t.count == 0);
      if (over) {
        NEED(!ascending);
        break;
      }
    }
  }
  if (!ascending) return true;
  NEED(taken == total && last_step == last_count);
  for (const auto& [w, to, x, h] : cuts)
    for (int i = w; i <= to; ++i) NEED(parts.count({2 * i + (i == w ? 1 : 0), x, h}));
  return true;
}

}  // namespace

int main() {
  std::mt19937 g(1);
  const auto below = [&](int32_t n) { return (int32_t)(g() % (uint32_t)n); };
  const auto spread = [&](int32_t most) {  // over its logarithm
    return min(most, (int32_t)(below(8) + 1) << below(22));
  };
  int dealt = 0, back = 0;
  for (int i = 0; i < 6000; ++i) {
    Case c;
    const int types[] = {0, 1, 2, 4};
    c.dtype = types[below(4)];
    c.dim = below(2) ? 64 : 128;
    PromptArgs& a = c.a;
    std::memset(&a, 0, sizeof a);
    a.requests = 1 + below(i % 7 == 0 ? 300 : i % 11 == 0 ? 1500 : 6);
    a.tokens = 1 + below(i % 3 == 0 ? 40 : 8000);
    a.group = below(2) ? 1 : 1 + below(20);
    a.kv_heads = below(2) ? 1 : 1 + below(12);
    a.page = page_div(16 << below(7));
    a.max_pages = ((1 << 20) + a.page.size - 1) / a.page.size;
    if (below(3) == 0) {
      a.anchor = spread(1 << 20);
      a.window = spread(1 << 20);
    }
    const bool ascending = below(2) != 0;
    for (int r = 0; r <= a.requests; ++r) c.start.push_back(below(a.tokens + 1));
    if (ascending) std::sort(c.start.begin(), c.start.end());
    else if (below(3) == 0) c.start[below(a.requests + 1)] = below(2) ? INT32_MIN : INT32_MAX;
    for (int r = 0; r < a.requests; ++r) c.lengths.push_back(below(8) == 0 ? -1 : spread(1 << 20) - below(2));
    if (below(2))
      for (int r = 0; r < a.requests; ++r) c.prefix.push_back(spread(1 << 20) - 3);
    if (i == 0) {  // starts that go back, a long request behind a short one
      a.requests = 3;
      a.tokens = 7168;
      a.group = a.kv_heads = 1;
      a.anchor = a.window = 0;
      c.dtype = 1;
      c.dim = 64;
      c.start = {0, 7168, 0, 3584};
      c.lengths = {7168, 1, 1 << 20};
      c.prefix.clear();
    }
    plan_prompt(c.dtype, c.dim, &a);
    dealt += a.groups != 0;
    back += a.groups != 0 && !ascending;
    const bool ok = c.dtype == 0 ? check<128>(c, ascending && i != 0) : check<256>(c, ascending && i != 0);
    if (!ok) {
      std::printf("case %d: type %d width %d, %d requests, %d tokens, %d heads on each of %d, anchor %d window %d\nstarts", i, c.dtype, c.dim,
                  a.requests, a.tokens, a.group, a.kv_heads, a.anchor, a.window);
      for (int32_t s : c.start) std::printf(" %d", s);
      std::printf("\nlengths");
      for (int32_t s : c.lengths) std::printf(" %d", s);
      std::printf("\n");
      return 1;
    }
  }
  std::printf("%d cases dealt out, %d with starts that go back\n", dealt, back);
  return dealt > 1000 && back > 500 ? 0 : 1;
}
