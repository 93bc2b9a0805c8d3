// Host-only checks of which kernels the planner chooses over MXFP4 pools: the tree walk, but for one set of rows on a path for which a
// set's pieces are too few.
#include <cstdio>

#include "../paper_2605_10195_amd/csrc/planner.hpp"

using namespace spex;

// Whether the walk is chosen for `paths` requests on nodes of their own of `tokens` tokens.
static bool walks(int Hq, int Hkv, int dim, int tokens, int paths) {
  PageTable pt(400000, 16, nullptr);
  std::vector<int32_t> nodes;
  for (int i = 0; i < paths; ++i) {
    nodes.push_back(pt.fork(kNoNode, 1));
    pt.append(nodes.back(), tokens, nullptr);
  }
  Planner planner;
  planner.pool = {true, false, dim, 1, true};
  Plan plan;
  if (planner.begin(pt, nodes.data(), nullptr, nullptr, paths, Hq, Hkv, 0, 0, 0, 0, &plan) != PlanError::kOk) return false;
  const bool walk = planner.prefers_walk(pt, &plan);
  planner.ensure_walk(pt, &plan);
  if (!plan.walk_ok || planner.prefers_walk(pt, &plan) != walk) std::printf("%d/%d/%d: no lists, or another choice\n", Hq, Hkv, dim);
  return walk;
}

int main() {
  const struct {
    int Hq, Hkv, dim, tokens, paths;
    bool walk;
  } cases[] = {
      {4, 1, 128, 64000, 1, true},   {4, 1, 128, 700000, 1, true},    {4, 1, 128, 917472, 1, true},    {4, 1, 128, 917504, 1, false},
      {4, 1, 128, 2000000, 1, false}, {8, 2, 128, 2000000, 1, true},  {4, 1, 128, 2000000, 2, true},   {32, 1, 128, 1000000, 1, true},
      {32, 1, 128, 2000000, 1, false}, {4, 1, 256, 2000000, 1, true}, {16, 1, 64, 1000000, 1, false},
  };
  int wrong = 0;
  for (const auto &c : cases)
    if (walks(c.Hq, c.Hkv, c.dim, c.tokens, c.paths) != c.walk && ++wrong)
      std::printf("%d/%d/%d, %d paths of %d tokens: %s the walk\n", c.Hq, c.Hkv, c.dim, c.paths, c.tokens, c.walk ? "not" : "takes");
  if (!wrong) std::printf("ok\n");
  return wrong != 0;
}
