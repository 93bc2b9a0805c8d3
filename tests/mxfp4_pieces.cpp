// Host-only checks of the workgroups that the planner makes of the tree-walk lists for MXFP4 pools: every block of every set of rows is in
// one piece, merges name all pieces of a set, and lists that length patches bring up to date stay covered.
#include <algorithm>
#include <climits>
#include <cstdio>
#include <cstdlib>
#include <map>
#include <random>
#include <vector>

#include "../paper_2605_10195_amd/csrc/launch_shape.hpp"
#include "../paper_2605_10195_amd/csrc/planner.hpp"

using namespace spex;

static int failures = 0, cut = 0, alone = 0, mixed = 0, two_tiles = 0, patched = 0;
#define CHECK(cond, ...) \
  do { \
    if (!(cond) && ++failures < 20) { std::printf("line %d: " #cond " ", __LINE__); std::printf(__VA_ARGS__); std::printf("\n"); } \
  } while (0)

static void check(const Plan &pl, int head_dim, const char *what) {
  const int ints = pl.item_ints(), NW = pl.walk_waves, G = pl.num_q_heads / pl.num_kv_heads;
  const int tiles = mx_row_tiles(head_dim, pl.walk_row_tiles), n_items = static_cast<int>(pl.walk_items.size()) / ints;
  const size_t rest = pl.walk_pieces.size() % (4 * Plan::kPieceInts);
  CHECK(rest == 0, "%s: part of a workgroup", what);
  std::map<std::pair<int, int>, std::vector<std::pair<int, std::vector<int>>>> of;  // set: pieces by their first block
  std::vector<char> used(static_cast<size_t>(pl.walk_partial_rows), 0);
  bool some_alone = false, some_together = false;
  for (size_t g = 0; g < pl.walk_pieces.size(); g += 4 * Plan::kPieceInts) {
    const int32_t *r = &pl.walk_pieces[g];
    const bool together = r[5] != 0;
    for (int k = 0; k < 4; ++k) {
      const int32_t *p = r + k * Plan::kPieceInts;
      if (p[0] < 0) continue;
      CHECK((p[5] != 0) == together, "%s: a workgroup of both kinds", what);
      if (together) CHECK(std::equal(p, p + Plan::kPieceInts, r), "%s: four records", what);
      (together ? some_together : some_alone) = true;
      if (together && k > 0) continue;
      CHECK(p[0] < n_items, "%s: item %d", what, p[0]);
      of[{p[0], p[1]}].push_back({p[2], std::vector<int>(p, p + Plan::kPieceInts)});
    }
  }
  std::map<std::pair<int, int>, std::pair<int, int>> merges;  // set: slot, pieces
  for (size_t m = 0; m < pl.walk_merges.size(); m += Plan::kMergeInts) {
    const int32_t *r = &pl.walk_merges[m];
    CHECK((merges.insert({{r[0], r[1]}, {r[2], r[3]}}).second), "%s: merged twice", what);
    CHECK(r[3] > 1 && r[3] <= 64, "%s: %d pieces", what, r[3]);
  }
  for (int i = 0; i < n_items; ++i) {
    const int32_t *rec = &pl.walk_items[static_cast<size_t>(i) * ints];
    for (int w = 0; w < NW; ++w) {
      const int rows = rec[3 + 2 * NW + w] * G;
      for (int s = 0; s * 16 * tiles < rows; ++s) {
        auto it = of.find({i, w | s << 8});
        CHECK(it != of.end(), "%s: item %d wavefront %d set %d is in no piece", what, i, w, s);
        if (it == of.end()) continue;
        auto &v = it->second;
        std::sort(v.begin(), v.end());
        const int n = static_cast<int>(v.size());
        auto m = merges.find(it->first);
        CHECK((n > 1) == (m != merges.end()), "%s: %d pieces and a merge or none", what, n);
        if (n > 1) CHECK(m != merges.end() && m->second.second == n, "%s: a merge of other pieces", what);
        int next = 0;
        for (int p = 0; p < n; ++p) {
          const std::vector<int> &r = v[static_cast<size_t>(p)].second;
          CHECK(r[2] == next, "%s: piece %d begins at %d behind %d", what, p, r[2], next);
          next = r[3];
          if (n > 1) {
            CHECK(r[4] == m->second.first + p * 16 * tiles, "%s: place of piece %d", what, p);
            CHECK(r[4] >= 0 && r[4] + 16 * tiles <= pl.walk_partial_rows, "%s: room", what);
            for (int k = r[4]; k < r[4] + 16 * tiles && k < pl.walk_partial_rows; ++k) {
              CHECK(!used[static_cast<size_t>(k)], "%s: a row of two pieces", what);
              used[static_cast<size_t>(k)] = 1;
            }
          } else {
            CHECK(r[4] == -1, "%s: a whole set", what);
          }
        }
        CHECK(next == INT_MAX, "%s: the last piece has an end", what);
        of.erase(it);
      }
    }
  }
  CHECK(of.empty(), "%s: pieces of no set", what);
  cut += !merges.empty();
  alone += some_alone;
  mixed += some_alone && some_together;
  two_tiles += tiles == 2;
}

int main(int argc, char **argv) {
  const int rounds = argc > 1 ? std::atoi(argv[1]) : 60;
  std::mt19937 rng(1);
  auto pick = [&](int lo, int hi) { return lo + static_cast<int>(rng() % static_cast<unsigned>(hi - lo + 1)); };
  for (int t = 0; t < rounds; ++t) {
    const int kind = t % 6, dims = 32 * pick(1, 8), Hkv = pick(1, 8), G = kind == 5 ? pick(1, 64) : pick(1, 16);
    // few long paths, many short ones, many and a long one, bushes, one root of many branches, wide groups
    const int roots = kind == 0 ? pick(1, 6) : (kind == 1 || kind == 2 ? pick(500, 900) : (kind == 4 ? 1 : pick(1, 40)));
    PageTable pt(400000, 16, nullptr);
    std::vector<int32_t> leaves, lens;
    for (int r = 0; r < roots; ++r) {
      const int u = pt.fork(kNoNode, 1);
      pt.append(u, kind == 0 ? pick(100, 60000) : (kind == 2 && r == 7 ? 20000 : pick(1, kind == 1 || kind == 2 ? 90 : 900)), nullptr);
      const int n = kind == 0 ? pick(0, 3) : (kind == 1 || kind == 2 ? pick(0, 4) : (kind == 4 ? pick(50, 300) : pick(0, 30)));
      if (n == 0) {
        leaves.push_back(u);
        lens.push_back(1);
        continue;
      }
      const int f = pt.fork(u, n);
      for (int k = 0; k < n; ++k) {
        const int len = pick(1, 130);
        pt.append(f + k, len, nullptr);
        leaves.push_back(f + k);
        lens.push_back(pick(0, 4) ? 1 : pick(1, std::min(len, 40)));
      }
    }
    Planner planner;
    planner.pool = {true, false, dims, 1, true};
    Plan plan;
    const int row_tiles = t % 4 == 3 ? 2 : 0, waves = t % 5 == 4 ? 8 : 0;
    char what[96];
    std::snprintf(what, sizeof what, "case %d: %d roots, %d requests, heads %d / %d / %d", t, roots, static_cast<int>(leaves.size()), G * Hkv, Hkv, dims);
    const int32_t n = static_cast<int32_t>(leaves.size());
    const PlanError e = planner.begin(pt, leaves.data(), lens.data(), nullptr, n, G * Hkv, Hkv, 0, 0, row_tiles, waves, &plan);
    CHECK(e == PlanError::kOk, "%s: begin", what);
    if (e != PlanError::kOk) continue;
    planner.ensure_walk(pt, &plan);
    if (!plan.walk_ok) continue;
    check(plan, dims, what);
    std::vector<int32_t> patches;
    for (int step = 0; step < 40; ++step) {
      for (int32_t u : leaves) pt.append(u, 1, nullptr);
      patches.clear();
      if (!planner.patch_lengths(pt, &plan, &patches)) break;
      ++patched;
      if (step % 8 == 7) check(plan, dims, what);
    }
  }
  if (failures) return 1;
  if (cut < 5 || alone < 5 || mixed < 1 || two_tiles < 3 || patched < 50) {
    std::printf("too few cases: %d cut, %d alone, %d mixed, %d of two tiles, %d patched\n", cut, alone, mixed, two_tiles, patched);
    return 1;
  }
  std::printf("ok\n");
  return 0;
}
