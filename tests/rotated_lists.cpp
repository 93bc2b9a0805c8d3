// The lists of spex_tree_append_rotated, built by test_append_rotated.py from the library's own host sources over a HIP
// runtime that is made here: every launch is checked against a model of the tree, and its patches are applied to the plan.
#include <hip/hip_runtime.h>

#include <algorithm>
#include <cstdio>
#include <cstdlib>
#include <cstring>
#include <map>
#include <random>
#include <vector>

#include "../include/spex_tree.h"
#include "../paper_2605_10195_amd/csrc/kernels.hpp"

static int failures = 0;
#define CHECK(ok, ...)                                                              \
  do {                                                                              \
    if (!(ok) && ++failures < 20) {                                                 \
      std::printf("line %d: ", __LINE__), std::printf(__VA_ARGS__), std::printf("\n"); \
    }                                                                               \
  } while (0)

extern "C" {
const char *hipGetErrorString(hipError_t) { return "an error made by the test"; }
hipError_t hipGetDevice(int *d) { return *d = 0, hipSuccess; }
hipError_t hipGetSymbolAddress(void **p, const void *) { return *p = nullptr, hipErrorUnknown; }
hipError_t hipMalloc(void **p, size_t n) { return *p = std::malloc(n), hipSuccess; }
hipError_t hipFree(void *p) { return std::free(p), hipSuccess; }
hipError_t hipMemcpy(void *d, const void *s, size_t n, hipMemcpyKind) { return std::memcpy(d, s, n), hipSuccess; }
hipError_t hipMemcpyAsync(void *d, const void *s, size_t n, hipMemcpyKind, hipStream_t) { return std::memcpy(d, s, n), hipSuccess; }
hipError_t hipHostMalloc(void **p, size_t n, unsigned) { return *p = std::malloc(n), hipSuccess; }
hipError_t hipHostFree(void *p) { return std::free(p), hipSuccess; }
hipError_t hipDeviceSynchronize() { return hipSuccess; }
hipError_t hipStreamSynchronize(hipStream_t) { return hipSuccess; }
hipError_t hipEventCreate(hipEvent_t *e) { return *e = nullptr, hipSuccess; }
hipError_t hipEventCreateWithFlags(hipEvent_t *e, unsigned) { return hipEventCreate(e); }
hipError_t hipEventDestroy(hipEvent_t) { return hipSuccess; }
hipError_t hipEventElapsedTime(float *, hipEvent_t, hipEvent_t) { return hipErrorUnknown; }
hipError_t hipEventRecord(hipEvent_t, hipStream_t) { return hipSuccess; }
hipError_t hipEventSynchronize(hipEvent_t) { return hipSuccess; }
}

struct Seen {
  int page, lo, n, tok0, pos0, new_index;
  bool is_new;
};
static std::vector<Seen> seen;
static std::vector<int> positions_seen;
static long launches = 0, from_memory = 0, patched = 0;

namespace spex {
bool has_mfma_kernel(const Shape &) { return true; }
bool has_rowmajor_kernel(const Shape &, const AttnArgs &) { return false; }
hipError_t launch_split(const Shape &, const AttnArgs &, const ItemLists &, hipStream_t) { return hipSuccess; }
hipError_t launch_split_phases(const Shape &, const AttnArgs &, const ItemLists &, hipStream_t) { return hipSuccess; }
hipError_t launch_generic_attention(const Shape &, const AttnArgs &, int, hipStream_t) { return hipSuccess; }
hipError_t launch_merge(const Shape &, const MergeArgs &, hipStream_t) { return hipSuccess; }
hipError_t launch_scatter(const Shape &, const ScatterArgs &, hipStream_t) { return hipSuccess; }
hipError_t launch_scatter_quantise(const Shape &, const ScatterArgs &, hipStream_t) { return hipSuccess; }
hipError_t launch_gather(const Shape &, const GatherArgs &, hipStream_t) { return hipSuccess; }
hipError_t launch_patch(int32_t *blob, const int32_t *p, int32_t n, hipStream_t) {
  for (int i = 0; i < n; ++i) blob[p[2 * i]] = p[2 * i + 1];
  return hipSuccess;
}
hipError_t launch_tree_walk(const Shape &, const WalkArgs &, int, int, bool, bool, hipStream_t) { return hipSuccess; }
hipError_t launch_append_tokens(const Shape &, const AppendTokensArgs &, hipStream_t) { return hipErrorUnknown; }
hipError_t launch_append_rotated(const Shape &, const RotateArgs &a, const RotateLists &in, hipStream_t) {
  const int32_t *h = a.lists ? a.lists : in.ints;
  ++launches;
  from_memory += a.lists != nullptr;
  int tokens = 0, most = 0;
  for (int i = 0; i < a.n_recs; ++i) {
    const int32_t *r = h + i * kVisitInts;
    const int lo = r[1] & 0xff, hi = (r[1] >> 8) & 0xff;
    seen.push_back({r[0], lo, hi - lo, r[2], r[3], r[4], (r[1] >> 16) != 0});
    tokens += hi - lo;
    most = std::max(most, hi - lo);
  }
  CHECK(most == a.most_tokens, "most tokens of a record");
  if (a.has_positions) positions_seen.assign(h + a.n_recs * kVisitInts, h + a.n_recs * kVisitInts + tokens);
  CHECK(a.lists || a.patches + 2 * a.n_patches <= kInlineInts, "lists longer than the arguments hold");
  for (int i = 0; i < a.n_patches; ++i) a.plan[h[a.patches + 2 * i]] = h[a.patches + 2 * i + 1];
  patched += a.n_patches > 0;
  return hipSuccess;
}
}  // namespace spex

int main() {
  std::vector<int32_t> pages(2000), valid(2000);
  for (int page_size : {1, 16, 64})
    for (int round = 0; round < 12; ++round) {
      std::mt19937 rng(1000 * page_size + round);
      auto below = [&](int n) { return static_cast<int>(rng() % n); };
      char pool[16];
      spex_tree_t *t = nullptr;
      spex_config_t c{};
      c.num_q_heads = c.num_kv_heads = 1;
      c.head_dim = 64;
      c.page_size = page_size;
      c.q_dtype = c.kv_dtype = SPEX_BF16;
      c.num_pages = 60000;
      c.k_pool = c.v_pool = pool;
      CHECK(spex_tree_create(&c, &t) == SPEX_OK, "create");
      double freq[32] = {};
      CHECK(spex_tree_set_rotation(t, 64, freq, 0) == SPEX_OK, "rotation");
      spex_node_t root;
      CHECK(spex_tree_fork(t, SPEX_NO_NODE, 1, &root) == SPEX_OK, "fork");
      const int prompt = below(70);
      if (prompt) CHECK(spex_tree_append_step(t, root, prompt, nullptr, nullptr, nullptr, nullptr, nullptr) == SPEX_OK, "prompt");
      const int n = 1 + below(round % 3 == 0 ? 300 : 40);
      std::vector<spex_node_t> nodes(n);
      CHECK(spex_tree_fork(t, root, n, nodes.data()) == SPEX_OK, "fork");
      std::map<int, int> length;
      std::vector<float> out(n * 64);
      bool asked = false;
      for (int call = 0; call < 30; ++call) {
        if (below(2)) std::shuffle(nodes.begin(), nodes.end(), rng);
        if (asked || below(2)) {  // a plan for the appends to be patched into
          bool full = true;
          for (int u : nodes) full = full && length[u] > 0;
          if (full) {
            std::vector<spex_node_t> in_order(nodes);
            std::sort(in_order.begin(), in_order.end());
            CHECK(spex_tree_decode_attention(t, in_order.data(), nullptr, n, pool, out.data(), nullptr, 0.1f, nullptr) == SPEX_OK, "decode");
            asked = true;
          }
        }
        const bool one_each = below(2), given = below(3) == 0;
        std::vector<int32_t> counts(n), positions;
        int total = 0;
        for (int &x : counts) total += x = one_each ? 1 : (below(4) ? below(8) : below(3 * page_size + 2));
        for (int i = 0; i < total; ++i) positions.push_back(below(INT32_MAX));
        spex_rotated_t d{};
        d.k = d.v = pool;
        seen.clear();
        const spex_status_t st =
            spex_tree_append_rotated(t, nodes.data(), one_each ? nullptr : counts.data(), n, given ? positions.data() : nullptr, &d, nullptr);
        CHECK(st == SPEX_OK, "append: %d", st);
        size_t at = 0;
        int token = 0, started = 0;
        for (int i = 0; i < n; ++i) {
          int32_t n_pages = 0;
          const int end = length[nodes[i]] + counts[i];
          if (counts[i] == 0) continue;
          CHECK(spex_tree_path_pages(t, nodes[i], pages.data(), valid.data(), 2000, &n_pages) == SPEX_OK, "pages");
          const int own = (end + page_size - 1) / page_size;
          for (int from = length[nodes[i]]; from < end;) {
            const int page = from / page_size, lo = from % page_size, take = std::min(page_size - lo, end - from);
            CHECK(at < seen.size(), "too few records");
            if (at >= seen.size()) return 1;
            const Seen s = seen[at++];
            CHECK(s.page == pages[n_pages - own + page] && s.lo == lo && s.n == take && s.tok0 == token, "record %zu", at);
            CHECK(s.is_new == (lo == 0) && (given || s.pos0 == prompt + from), "start and position of record %zu", at);
            CHECK(!s.is_new || s.new_index == started, "order of the started pages");
            started += s.is_new;
            token += take;
            from += take;
          }
          length[nodes[i]] = end;
        }
        CHECK(at == seen.size(), "too many records");
        if (given && total) CHECK(positions_seen == positions, "positions");
      }
      spex_tree_destroy(t);
    }
  CHECK(launches > 500 && from_memory > 100 && from_memory < launches - 100 && patched > 50, "%ld launches, %ld lists in memory, %ld with patches",
        launches, from_memory, patched);
  if (failures == 0) std::printf("ok\n");
  return failures != 0;
}
