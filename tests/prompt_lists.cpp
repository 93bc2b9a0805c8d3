// The lists of spex_prompt_attention, built by test_prompt_attention.py from the library's own host source with the launches replaced by
// the test's own: every row set of every prompt and kv head is worked on exactly once, in launches of bounded size.
#include <hip/hip_runtime.h>

#include <cstdio>
#include <cstdlib>
#include <map>
#include <random>
#include <vector>

#include "../include/spex_prompt.h"
#include "../paper_2605_10195_amd/csrc/prompt.hpp"

static int failures = 0;
#define CHECK(ok, ...)                                                                   \
  do {                                                                                   \
    if (!(ok) && ++failures < 20) {                                                      \
      std::printf("line %d: ", __LINE__), std::printf(__VA_ARGS__), std::printf("\n");   \
    }                                                                                    \
  } while (0)

struct Range {
  int64_t from, to;  // items of a prompt
};
static std::map<int, std::vector<Range>> ranges;  // by the prompt's first token
static std::map<int, int> lengths;
static long launches = 0;
static int sets_of_a_group = 4;

namespace spex {
bool hip_failed(hipError_t e, const char *) { return e != hipSuccess; }
PromptKernel prompt_kernel(bool f32, bool wide, int32_t, int64_t, int32_t) { return {f32, wide, false, false, false, sets_of_a_group}; }
int64_t prompt_items(const PromptKernel &k, int32_t heads_per_kv, int32_t len) {
  return ((static_cast<int64_t>(len) + kPromptRows - 1) / kPromptRows * heads_per_kv + k.sets - 1) / k.sets;
}
hipError_t launch_prompt(const PromptKernel &, const PromptArgs &a, int64_t items, hipStream_t) {
  ++launches;
  CHECK(items > 0 && items * a.Hkv <= (int64_t(1) << 23), "%ld items", static_cast<long>(items));
  CHECK(a.n > 0 && a.n <= kMaxPromptsPerLaunch, "%d prompts", a.n);
  for (int i = 0; i < a.n; ++i) {
    const int64_t end = i + 1 < a.n ? a.first[i + 1] : items, begin = i ? a.first[i] : 0;
    CHECK(i == 0 || a.first[i] > 0, "prompt %d begins before the launch", i);
    CHECK(begin < end, "prompt %d without items", i);
    ranges[a.start[i]].push_back({begin - a.first[i], end - a.first[i]});
    CHECK(lengths[a.start[i]] == a.len[i], "length of prompt %d", i);
  }
  for (int i = a.n; i < kMaxPromptsPerLaunch; ++i) CHECK(a.first[i] == INT32_MAX, "list behind its end");
  return hipSuccess;
}
}  // namespace spex

static void one(int heads, int kv_heads, const std::vector<int32_t> &lens) {
  spex_prompt_config_t c{};
  c.num_q_heads = heads;
  c.num_kv_heads = kv_heads;
  c.head_dim = 1;
  c.dtype = SPEX_BF16;
  char any[16];
  ranges.clear();
  lengths.clear();
  int at = 0;
  for (int32_t n : lens) {
    if (n) lengths[at] = n;
    at += n;
  }
  const spex_status_t st = spex_prompt_attention(&c, lens.data(), static_cast<int32_t>(lens.size()), any, any, any, any, nullptr, 1.f, nullptr);
  CHECK(st == SPEX_OK, "status %d", st);
  CHECK(ranges.size() == lengths.size(), "%zu prompts of %zu", ranges.size(), lengths.size());
  for (auto &p : ranges) {
    int64_t next = 0;
    for (const Range &r : p.second) {
      CHECK(r.from == next, "items of prompt %d", p.first);
      next = r.to;
    }
    const int64_t sets = (static_cast<int64_t>(lengths[p.first]) + 31) / 32 * (heads / kv_heads);
    CHECK(next == (sets + sets_of_a_group - 1) / sets_of_a_group, "items of prompt %d", p.first);
  }
}

int main() {
  std::mt19937 rng(1);
  for (int sets : {1, 4}) {
    sets_of_a_group = sets;
    for (int heads : {1, 32, 255, 255 * 40, 255 * 4000})
      for (int kv : {1, 255})
        for (int round = 0; round < 6; ++round) {
          if (heads % kv) continue;
          std::vector<int32_t> lens;
          for (int n = 1 + rng() % 200; n > 0; --n) lens.push_back(rng() % 5 ? rng() % 300 : rng() % (1 << (heads > 40000 ? 10 : 18)));
          one(heads, kv, lens);
        }
    launches = 0;
    one(64, 8, {1 << 24});
    CHECK(launches == (sets == 1 ? 4 : 1), "%ld launches of the longest prompt", launches);
    launches = 0;
    one(4080, 255, {5, 1 << 24, 70, 1 << 24, 0, 1 << 20});
    CHECK(launches > (sets == 1 ? 500 : 120), "%ld launches of long prompts", launches);
    one(4095, 1, {1 << 24});
  }
  if (failures == 0) std::printf("ok\n");
  return failures != 0;
}
