// The frequencies of spex_tree_set_rotation on their way to the device, over the HIP runtime of rotated_lists.cpp, with copies as the runtime's
// documentation allows them: of pageable memory, which may be changed once the call has returned, to the device when somebody waits.
#include <hip/hip_runtime.h>

#include "../paper_2605_10195_amd/csrc/kernels.hpp"
#define main lists_main
#define hipMemcpy lists_memcpy
#define hipMemcpyAsync lists_memcpy_async
#define hipDeviceSynchronize lists_device_synchronize
#define hipStreamSynchronize lists_stream_synchronize
#define launch_append_rotated lists_launch
namespace spex {
hipError_t lists_launch(const Shape &, const RotateArgs &, const RotateLists &, hipStream_t);
}
#include "rotated_lists.cpp"
#undef main
#undef hipMemcpy
#undef hipMemcpyAsync
#undef hipDeviceSynchronize
#undef hipStreamSynchronize
#undef launch_append_rotated

#include <cmath>

struct Copy {
  void *to;
  std::vector<char> from;
  hipStream_t stream;
};
static std::vector<Copy> under_way;
static std::vector<const spex::Turns *> running;  // launches that nobody has waited for, which read there

static void land(bool all, hipStream_t s) {
  for (size_t i = 0; i < under_way.size();)
    if (all || under_way[i].stream == s) {
      for (const spex::Turns *at : running) CHECK(at != under_way[i].to, "frequencies replaced under a launch");
      std::memcpy(under_way[i].to, under_way[i].from.data(), under_way[i].from.size());
      under_way.erase(under_way.begin() + i);
    } else {
      ++i;
    }
}
extern "C" {
hipError_t hipMemcpyAsync(void *d, const void *s, size_t n, hipMemcpyKind, hipStream_t stream) {
  under_way.push_back({d, std::vector<char>(static_cast<const char *>(s), static_cast<const char *>(s) + n), stream});
  return hipSuccess;
}
hipError_t hipMemcpy(void *d, const void *s, size_t n, hipMemcpyKind k) { return hipMemcpyAsync(d, s, n, k, nullptr); }
hipError_t hipDeviceSynchronize() {
  running.clear();
  land(true, nullptr);
  return hipSuccess;
}
hipError_t hipStreamSynchronize(hipStream_t s) {
  land(false, s);
  return hipSuccess;
}
}
static double expected = 0.0;
namespace spex {
hipError_t launch_append_rotated(const Shape &, const RotateArgs &a, const RotateLists &, hipStream_t) {
  const double turns = a.freq[0].hi + a.freq[0].lo;
  CHECK(std::fabs(turns * 6.283185307179586 - expected) < 1e-12, "the launch reads %g, the setting is %g", turns * 6.283185307179586, expected);
  running.push_back(a.freq);
  return hipSuccess;
}
}  // namespace spex

int main() {
  char pool[16], streams[3];
  spex_tree_t *t = nullptr;
  spex_config_t c{};
  c.num_q_heads = c.num_kv_heads = 1;
  c.head_dim = 64;
  c.page_size = 16;
  c.q_dtype = c.kv_dtype = SPEX_BF16;
  c.num_pages = 100;
  c.k_pool = c.v_pool = pool;
  CHECK(spex_tree_create(&c, &t) == SPEX_OK, "create");
  spex_node_t root;
  CHECK(spex_tree_fork(t, SPEX_NO_NODE, 1, &root) == SPEX_OK, "fork");
  for (int i = 0; i < 20; ++i) {
    if (i % 3 == 0) {
      double freq[32];
      for (double &f : freq) f = expected = 0.25 + i;
      CHECK(spex_tree_set_rotation(t, 64, freq, 0) == SPEX_OK, "rotation");
    }
    spex_rotated_t d{};
    d.k = d.v = pool;
    CHECK(spex_tree_append_rotated(t, &root, nullptr, 1, nullptr, &d, reinterpret_cast<hipStream_t>(streams + i % 3)) == SPEX_OK, "append");
  }
  spex_tree_destroy(t);
  if (failures == 0) std::printf("ok\n");
  return failures != 0;
}
