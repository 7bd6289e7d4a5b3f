// Plans with two softmax maps per row (differential attention), built by the library's planner for
// 256 CUs in 8 XCDs and checked on the host:
//  - every (sequence, key pair, query tile) covers its keys exactly once, in ranges that start at
//    multiples of a key tile, their partial slots in key order and listed in one merge group;
//  - the workspace holds every slot of both maps in fp32;
//  - decode chunks start at page and tile boundaries and span at most 64 pages;
//  - whether tiles are cut follows the bytes of the call's K/V, and cutting ends earlier.
// Prints how many plans were cut; exits 0 on success.
#include <algorithm>
#include <cstdio>
#include <cstdlib>
#include <map>
#include <random>
#include <tuple>

#include "planner.h"

using namespace cw;

namespace {

constexpr int kTile = 64, kCus = 256, kXcds = 8;

#define CHECK(c, ...)                                  \
  do {                                                 \
    if (!(c)) {                                        \
      std::fprintf(stderr, "FAIL line %d: ", __LINE__); \
      std::fprintf(stderr, __VA_ARGS__);               \
      std::fprintf(stderr, "\n");                      \
      std::exit(1);                                    \
    }                                                  \
  } while (0)

void check_parts(const ExtendPlan& p, int rows, int width, int unit) {
  std::map<std::tuple<int, int, int>, std::vector<WorkItem>> tiles;
  for (const WorkItem& w : p.items)
    if (w.seq >= 0) tiles[{w.seq, w.kvh, w.q_row0}].push_back(w);
  std::map<std::tuple<int, int, int>, CombineGroup> groups;
  for (const CombineGroup& g : p.groups) CHECK(groups.emplace(std::make_tuple(g.seq, g.kvh, g.q_row0), g).second, "two groups of one tile");
  std::vector<char> used(size_t(p.n_parts), 0);
  for (auto& [key, v] : tiles) {
    std::sort(v.begin(), v.end(), [](const WorkItem& a, const WorkItem& b) { return a.kv_begin < b.kv_begin; });
    CHECK(v[0].kv_begin == 0, "keys start at %d", v[0].kv_begin);
    for (size_t i = 0; i < v.size(); ++i) {
      CHECK(v[i].kv_end > v[i].kv_begin && v[i].kv_begin % unit == 0, "range [%d, %d)", v[i].kv_begin, v[i].kv_end);
      CHECK(i == 0 || v[i].kv_begin == v[i - 1].kv_end, "gap before key %d", v[i].kv_begin);
      CHECK(v[i].rows == v[0].rows, "rows");
      if (v.size() == 1) {
        CHECK(v[i].part == -1 && groups.count(key) == 0, "a whole tile has a part");
        continue;
      }
      CHECK(v[i].part >= 0 && v[i].part < p.n_parts && !used[v[i].part], "part %d", v[i].part);
      used[v[i].part] = 1;
      CHECK(groups.count(key) == 1, "no group");
      const CombineGroup& g = groups[key];
      CHECK(g.rows == v[i].rows && g.n_parts == int(v.size()) && v[i].part == g.part0 + int(i), "group");
    }
  }
  CHECK(std::count(used.begin(), used.end(), 0) == 0, "unused slots");
  CHECK(p.part_rows == 2 * rows && p.part_f32, "slots of %d rows", p.part_rows);
  const size_t n = size_t(p.n_parts) * p.part_rows;
  CHECK(n == 0 || (p.off_part_o >= p.meta_bytes && p.off_part_ml >= p.off_part_o + n * width * 4 &&
                   p.total_bytes >= p.off_part_ml + n * 8),
        "workspace of %zu bytes for %zu rows", p.total_bytes, n);
}

// every tile's last key, and the number of tiles
void check_extend(const ExtendPlan& p, const std::vector<int32_t>& lp, const std::vector<int32_t>& ls, int pairs, int g, int width) {
  check_parts(p, DIFF_BLOCK_M, width, kTile);
  std::map<std::tuple<int, int, int>, int> last;
  for (const WorkItem& w : p.items)
    if (w.seq >= 0) last[{w.seq, w.kvh, w.q_row0}] = std::max(last[{w.seq, w.kvh, w.q_row0}], w.kv_end);
  size_t n = 0;
  for (size_t b = 0; b < lp.size(); ++b)
    for (int j = 0; j < pairs; ++j)
      for (int r = 0; r < ls[b] * g; r += DIFF_BLOCK_M, ++n) {
        const int rows = std::min(DIFF_BLOCK_M, ls[b] * g - r);
        const auto it = last.find({int(b), j, r});
        CHECK(it != last.end() && it->second == lp[b] + (r + rows - 1) / g + 1, "keys of sequence %zu row %d", b, r);
      }
  CHECK(n == last.size(), "%zu tiles, %zu expected", last.size(), n);
}

ExtendPlan extend(const std::vector<int32_t>& lp, const std::vector<int32_t>& ls, int pairs, int g, int d, int64_t kv_bytes) {
  return build_extend_plan(lp.data(), ls.data(), int(lp.size()), pairs, g, 2 * d, DIFF_BLOCK_M, 1, kCus, kXcds, Tuning{}, nullptr,
                           nullptr, 2, kv_bytes);
}

// The time the last workgroup ends, in key tiles (an item costs 2.5 more): one workgroup per CU,
// item i on XCD i % 8.
double makespan(const ExtendPlan& p) {
  double end = 0;
  for (int x = 0; x < kXcds; ++x) {
    std::vector<double> cu(kCus / kXcds, 0.0);
    for (size_t i = x; i < p.items.size(); i += kXcds) {
      const WorkItem& w = p.items[i];
      if (w.seq < 0) continue;
      auto it = std::min_element(cu.begin(), cu.end());
      *it += 2.5 + (w.kv_end - w.kv_begin + kTile - 1) / kTile;
      end = std::max(end, *it);
    }
  }
  return end;
}

}  // namespace

int main() {
  std::mt19937 rng(7);
  auto pick = [&](int lo, int hi) { return std::uniform_int_distribution<int>(lo, hi)(rng); };
  int cut = 0, cut_shared = 0;
  for (int n = 0; n < 1500; ++n) {
    const int seqs = pick(1, 12), pairs = 1 << pick(0, 3), g = pick(1, 16), d = pick(0, 1) ? 64 : 128;
    std::vector<int32_t> lp(seqs), ls(seqs);
    const int pre = pick(0, 3) ? pick(1, 40000) : 0, suf = pick(2, 3000);
    int64_t kv = 0;
    for (int b = 0; b < seqs; ++b) {
      lp[b] = pick(0, pre);
      ls[b] = pick(0, 9) ? pick(1, suf) : 0;
      kv += int64_t(lp[b] + ls[b]) * 8 * d * pairs;
    }
    const ExtendPlan p = extend(lp, ls, pairs, g, d, kv);
    check_extend(p, lp, ls, pairs, g, 2 * d);
    cut += p.n_parts > 0;
    cut_shared += p.n_parts > 0 && kv > (int64_t(192) << 20);
  }
  CHECK(cut > 100 && cut_shared > 20, "%d plans cut, %d of them with much K/V", cut, cut_shared);

  // Three thousand rows on 48000 keys, 4 key pairs: 376 tiles on 256 CUs.  Cut while the K/V fits the
  // memory-side cache, whole when it does not (what cutting gains is then lost to K/V read again).
  const std::vector<int32_t> lp{48000}, ls{3000};
  const ExtendPlan near = extend(lp, ls, 4, 4, 128, int64_t(94) << 20), far = extend(lp, ls, 4, 4, 128, int64_t(400) << 20);
  check_extend(near, lp, ls, 4, 4, 256);
  check_extend(far, lp, ls, 4, 4, 256);
  CHECK(near.n_parts > 0 && far.n_parts == 0, "%lld and %lld parts", (long long)near.n_parts, (long long)far.n_parts);
  CHECK(makespan(near) < 0.85 * makespan(far), "ends at %.0f and %.0f", makespan(near), makespan(far));

  for (int n = 0; n < 1500; ++n) {
    const int seqs = pick(1, 60), pairs = 1 << pick(0, 3), g = pick(1, 16), page = pick(0, 1) ? 16 : 64, d = pick(0, 1) ? 64 : 128;
    std::vector<int32_t> lp1(seqs);
    const int pre = pick(0, 70000);
    for (int32_t& x : lp1) x = pick(0, pre);
    const ExtendPlan p = build_decode_plan(lp1.data(), seqs, pairs, g, 2 * d, page, 32, pick(2, 6), kCus, Tuning{}, 0, nullptr, nullptr, 2);
    check_parts(p, g, 2 * d, std::max(32, page));
    std::map<std::pair<int, int>, int> keys;
    for (const WorkItem& w : p.items) {
      CHECK(w.kv_end - w.kv_begin <= 64 * page, "a chunk of %d keys", w.kv_end - w.kv_begin);
      keys[{w.seq, w.kvh}] += w.kv_end - w.kv_begin;
    }
    CHECK(keys.size() == size_t(seqs) * pairs, "sequences left out");
    for (const auto& [k, total] : keys) CHECK(total == lp1[k.first] + 1, "%d keys of %d", total, lp1[k.first] + 1);
  }
  std::printf("ok: %d of 1500 plans cut, %d with K/V past the memory-side cache\n", cut, cut_shared);
  return 0;
}
