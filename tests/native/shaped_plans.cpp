// Plans over the keys that a window and prefix masks leave, built by the library's planner for 256
// CUs in 8 XCDs and checked on the host, for random batches:
//  - every (sequence, kv head, query tile) covers its keys exactly once: from the key tile of the
//    first key that its first row sees to the last one that some row sees, in ranges that start
//    at multiples of a key tile, partial slots in key order in one merge group;
//  - without a window and a prefix mask the items are those of the plan without limits.
// Prints how many plans were cut; exits 0 on success.
#include <algorithm>
#include <cstdio>
#include <cstdlib>
#include <cstring>
#include <map>
#include <random>
#include <tuple>

#include "planner.h"

using namespace cw;

namespace {

constexpr int kTile = 64, kCus = 256, kXcds = 8, kRows = 256;

#define CHECK(c, ...)                                  \
  do {                                                 \
    if (!(c)) {                                        \
      std::fprintf(stderr, "FAIL line %d: ", __LINE__); \
      std::fprintf(stderr, __VA_ARGS__);               \
      std::fprintf(stderr, "\n");                      \
      std::exit(1);                                    \
    }                                                  \
  } while (0)

void check(const ExtendPlan& p, const std::vector<int32_t>& lp, const std::vector<int32_t>& ls, const std::vector<int32_t>& full,
           int window, int hkv, int g, int d) {
  std::map<std::tuple<int, int, int>, std::vector<WorkItem>> tiles;
  for (const WorkItem& w : p.items)
    if (w.seq >= 0) tiles[{w.seq, w.kvh, w.q_row0}].push_back(w);
  std::map<std::tuple<int, int, int>, CombineGroup> groups;
  for (const CombineGroup& c : p.groups) CHECK(groups.emplace(std::make_tuple(c.seq, c.kvh, c.q_row0), c).second, "two groups");
  std::vector<char> used(size_t(p.n_parts), 0);
  size_t n = 0;
  for (size_t b = 0; b < lp.size(); ++b)
    for (int h = 0; h < hkv; ++h)
      for (int64_t r = 0; r < int64_t(ls[b]) * g; r += kRows, ++n) {
        const int rows = int(std::min<int64_t>(kRows, int64_t(ls[b]) * g - r));
        const int first = lp[b] + int(r / g), last = lp[b] + int((r + rows - 1) / g);
        const int begin = window > 0 ? std::max(0, first - window + 1) / kTile * kTile : 0;
        const int end = std::max(last + 1, std::min(full[b], lp[b] + ls[b]));
        auto it = tiles.find({int(b), h, int(r)});
        CHECK(it != tiles.end(), "no tile");
        auto& v = it->second;
        std::sort(v.begin(), v.end(), [](const WorkItem& x, const WorkItem& y) { return x.kv_begin < y.kv_begin; });
        CHECK(v.front().kv_begin == begin && v.back().kv_end == end, "keys [%d, %d), expected [%d, %d)", v.front().kv_begin,
              v.back().kv_end, begin, end);
        for (size_t i = 0; i < v.size(); ++i) {
          CHECK(v[i].kv_end > v[i].kv_begin && v[i].kv_begin % kTile == 0 && v[i].rows == rows, "range");
          CHECK(i == 0 || v[i].kv_begin == v[i - 1].kv_end, "gap before key %d", v[i].kv_begin);
          if (v.size() == 1) {
            CHECK(v[i].part == -1 && groups.count(it->first) == 0, "a whole tile has a part");
            continue;
          }
          CHECK(v[i].part >= 0 && v[i].part < p.n_parts && !used[v[i].part], "part %d", v[i].part);
          used[v[i].part] = 1;
          CHECK(groups.count(it->first) == 1, "no group");
          const CombineGroup& c = groups[it->first];
          CHECK(c.rows == rows && c.n_parts == int(v.size()) && v[i].part == c.part0 + int(i), "group");
        }
      }
  CHECK(n == tiles.size(), "%zu tiles, %zu expected", tiles.size(), n);
  CHECK(std::count(used.begin(), used.end(), 0) == 0, "unused slots");
  const size_t slots = size_t(p.n_parts) * p.part_rows;
  CHECK(p.part_f32 && p.part_rows == kRows && (slots == 0 || (p.off_part_ml >= p.off_part_o + slots * d * 4 &&
                                                             p.total_bytes >= p.off_part_ml + slots * 8)), "workspace");
}

}  // namespace

int main() {
  std::mt19937 rng(7);
  auto pick = [&](int lo, int hi) { return int(std::uniform_int_distribution<int>(lo, hi)(rng)); };
  int cut = 0, plans = 0;
  for (int round = 0; round < 400; ++round) {
    const int n = pick(1, 9), hkv = 1 << pick(0, 4), g = pick(1, 16), d = pick(0, 1) ? 64 : 128;
    const int top = pick(0, 3) == 0 ? 40000 : 3000;
    std::vector<int32_t> lp, ls, full;
    for (int b = 0; b < n; ++b) {
      lp.push_back(pick(0, 2) == 0 ? 0 : pick(0, top));
      ls.push_back(pick(0, 5) == 0 ? 0 : pick(1, 2500));
      full.push_back(pick(0, 2) ? 0 : pick(0, 6000));
    }
    KeyLimits lim;
    lim.window = pick(0, 2) == 0 ? 0 : pick(0, 1) ? pick(1, 200) : pick(1, 20000);
    lim.full_lens = pick(0, 1) ? full.data() : nullptr;
    Tuning t{};
    if (round % 5 == 0) t.kv_chunk_tiles = pick(1, 7);
    if (round % 5 == 1) t.target_wgs = pick(1, 600);
    const ExtendPlan p = build_extend_plan(lp.data(), ls.data(), n, hkv, g, d, kRows, 1, kCus, kXcds, t, nullptr, nullptr, 1, 0, &lim);
    std::vector<int32_t> none(n, 0);
    check(p, lp, ls, lim.full_lens ? full : none, lim.window, hkv, g, d);
    cut += p.n_parts > 0;
    ++plans;
    if (lim.window == 0 && lim.full_lens == nullptr) {
      const ExtendPlan q = build_extend_plan(lp.data(), ls.data(), n, hkv, g, d, kRows, 1, kCus, kXcds, t);
      CHECK(p.items.size() == q.items.size() &&
                (p.items.empty() || std::memcmp(p.items.data(), q.items.data(), p.items.size() * sizeof(WorkItem)) == 0),
            "limits that limit nothing change the plan");
    }
  }
  std::printf("ok: %d of %d plans cut\n", cut, plans);
  return 0;
}
