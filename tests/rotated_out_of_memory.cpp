// spex_tree_append_rotated without host memory: every allocation of a call fails in turn, over the HIP runtime of rotated_lists.cpp.  A call
// either changes nothing and says SPEX_ERR_CAPACITY, or appends everything and launches it.
#define main lists_main
#include "rotated_lists.cpp"
#undef main

#include <new>

static long allocations = 0, fail_at = -1;
static void *get(std::size_t n) {
  if (fail_at >= 0 && allocations++ == fail_at) throw std::bad_alloc();
  void *p = std::malloc(n ? n : 1);
  if (!p) throw std::bad_alloc();
  return p;
}
void *operator new(std::size_t n) { return get(n); }
void *operator new[](std::size_t n) { return get(n); }
void operator delete(void *p) noexcept { std::free(p); }
void operator delete[](void *p) noexcept { std::free(p); }
void operator delete(void *p, std::size_t) noexcept { std::free(p); }
void operator delete[](void *p, std::size_t) noexcept { std::free(p); }

struct State {
  std::vector<int> tokens, pages, free;
  bool operator==(const State &o) const { return tokens == o.tokens && pages == o.pages && free == o.free; }
};
static State state(spex_tree_t *t, const std::vector<spex_node_t> &nodes) {
  State s;
  int32_t n = 0;
  for (int u : nodes) {
    spex_node_info_t info;
    CHECK(spex_tree_node_info(t, u, &info) == SPEX_OK, "info");
    s.tokens.push_back(info.n_tokens);
    s.pages.push_back(info.n_pages);
  }
  s.free.resize(4000);
  CHECK(spex_tree_free_pages(t, s.free.data(), 4000, &n) == SPEX_OK, "free pages");
  s.free.resize(n);
  return s;
}

int main() {
  long failed = 0, plans_dropped = 0;
  char pool[16];
  for (int count : {1, 5, 40})
    for (int n : {3, 90})
      for (bool planned : {false, true})
        for (bool descending : {false, true})
          for (long at = 0;; ++at) {
            spex_tree_t *t = nullptr;
            spex_config_t c{};
            c.num_q_heads = c.num_kv_heads = 1;
            c.head_dim = 64;
            c.page_size = 16;
            c.q_dtype = c.kv_dtype = SPEX_BF16;
            c.num_pages = 4000;
            c.k_pool = c.v_pool = pool;
            CHECK(spex_tree_create(&c, &t) == SPEX_OK, "create");
            double freq[32] = {};
            CHECK(spex_tree_set_rotation(t, 64, freq, 0) == SPEX_OK, "rotation");
            std::vector<spex_node_t> nodes(n);
            CHECK(spex_tree_fork(t, SPEX_NO_NODE, n, nodes.data()) == SPEX_OK, "fork");
            std::vector<float> out(n * 64);
            std::vector<int32_t> counts(n);
            for (int i = 0; i < n; ++i) {
              counts[i] = count + i % 3;
              CHECK(spex_tree_append_step(t, nodes[i], 3 + i % 14, nullptr, nullptr, nullptr, nullptr, nullptr) == SPEX_OK, "prompt");
            }
            if (planned)
              CHECK(spex_tree_decode_attention(t, nodes.data(), nullptr, n, pool, out.data(), nullptr, 0.1f, nullptr) == SPEX_OK, "decode");
            std::vector<spex_node_t> order(nodes);
            if (descending) std::reverse(order.begin(), order.end());
            const State before = state(t, order);
            spex_rotated_t d{};
            d.k = d.v = pool;
            seen.clear();
            seen.reserve(10000);
            allocations = 0;
            fail_at = at;
            const spex_status_t st = spex_tree_append_rotated(t, order.data(), counts.data(), n, nullptr, &d, nullptr);
            const bool reached = allocations > at;
            fail_at = -1;
            const State after = state(t, order);
            if (st == SPEX_OK) {
              int tokens = 0, launched = 0;
              for (int i = 0; i < n; ++i) {
                CHECK(after.tokens[i] == before.tokens[i] + counts[i], "node %d", i);
                tokens += counts[i];
              }
              for (const Seen &s : seen) launched += s.n;
              CHECK(launched == tokens, "%d of %d tokens launched", launched, tokens);
              if (reached) ++plans_dropped;
            } else {
              CHECK(st == SPEX_ERR_CAPACITY && reached, "status %d", st);
              CHECK(after == before && seen.empty(), "allocation %ld of %d nodes, %d tokens: the tree has changed", at, n, count);
              ++failed;
              CHECK(spex_tree_append_rotated(t, order.data(), counts.data(), n, nullptr, &d, nullptr) == SPEX_OK, "again");
            }
            CHECK(spex_tree_decode_attention(t, nodes.data(), nullptr, n, pool, out.data(), nullptr, 0.1f, nullptr) == SPEX_OK, "decode");
            spex_tree_destroy(t);
            if (!reached) break;
          }
  CHECK(failed > 50 && plans_dropped > 3, "%ld calls failed, %ld plans dropped", failed, plans_dropped);
  if (failures == 0) std::printf("ok\n");
  return failures != 0;
}
