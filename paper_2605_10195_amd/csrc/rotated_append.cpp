// spex_tree_set_rotation and spex_tree_append_rotated: argument checks, the page table's part and the launch's lists.  See
// include/spex_tree.h.
#include <algorithm>
#include <cmath>
#include <cstring>
#include <new>
#include <vector>

#include "tree.hpp"

namespace {

// The frequencies to the device.  Launches that read others there are waited for, and so is the copy, since later launches may come on
// other streams.
spex_status_t upload_rotation(spex_tree *t, hipStream_t stream) {
  if (t->freq_on_device) return SPEX_OK;
  if (t->d_freq)
    HIP_TRY(hipDeviceSynchronize());
  else
    HIP_TRY(hipMalloc(&t->d_freq, sizeof(t->freq)));
  HIP_TRY(hipMemcpyAsync(t->d_freq, t->freq, sizeof(t->freq), hipMemcpyHostToDevice, stream));
  HIP_TRY(hipStreamSynchronize(stream));
  t->freq_on_device = true;
  return SPEX_OK;
}

spex_status_t append_rotated_impl(spex_tree_t *t, const spex_node_t *nodes, const int32_t *counts, int32_t n_nodes, const int32_t *positions,
                                  const spex_rotated_t *data, void *hip_stream) {
  if (!t || !data || n_nodes < 0 || (n_nodes > 0 && !nodes)) return SPEX_ERR_INVALID_ARG;
  if (!t->cfg.k_pool || t->rotary_dim == 0) return SPEX_ERR_INVALID_ARG;
  const bool fp8 = t->cfg.kv_dtype == SPEX_FP8_E4M3;
  if ((data->q == nullptr) != (data->q_out == nullptr) || (data->k_scales == nullptr) != (data->v_scales == nullptr) ||
      (data->k_scales && !fp8))
    return SPEX_ERR_INVALID_ARG;
  const int64_t q_row = static_cast<int64_t>(t->cfg.num_q_heads) * t->cfg.head_dim;
  const int64_t kv_row = static_cast<int64_t>(t->cfg.num_kv_heads) * t->cfg.head_dim;
  const int64_t given[5] = {data->q_stride, data->k_stride, data->v_stride, data->q_out_stride, data->k_out_stride};
  const int64_t dense[5] = {q_row, kv_row, kv_row, q_row, kv_row};
  int64_t stride[5];
  for (int i = 0; i < 5; ++i) {
    stride[i] = given[i] ? given[i] : dense[i];
    if (stride[i] < dense[i]) return SPEX_ERR_INVALID_ARG;
    if (stride[i] > INT32_MAX) return SPEX_ERR_UNSUPPORTED;
  }
  // in place means every element in its own place
  if ((data->q && data->q == data->q_out && stride[0] != stride[3]) || (data->k && data->k == data->k_out && stride[1] != stride[4]))
    return SPEX_ERR_INVALID_ARG;

  // Check everything before touching the table: the call is all or nothing.
  const int32_t P = t->cfg.page_size, shift = __builtin_ctz(P);  // a division takes as long as the rest of a node's work
  int64_t need = 0, visits = 0, tokens = 0;
  bool ascending = true;
  for (int32_t i = 0; i < n_nodes; ++i) {
    const int32_t u = nodes[i], c = counts ? counts[i] : 1;
    if (c < 0) return SPEX_ERR_INVALID_ARG;
    if (!t->pt->valid(u)) return SPEX_ERR_BAD_NODE;
    const spex::Node &nd = t->pt->node(u);
    if (nd.n_live_children > 0) return SPEX_ERR_NOT_LEAF;
    if (static_cast<int64_t>(nd.n_tokens) + c > INT32_MAX / 2) return SPEX_ERR_UNSUPPORTED;
    ascending = ascending && (i == 0 || nodes[i - 1] < u);
    tokens += c;
    if (c == 0) continue;
    const int32_t last = (nd.n_tokens + c - 1) >> shift;
    need += last + 1 - static_cast<int64_t>(nd.pages.size());
    visits += last - (nd.n_tokens >> shift) + 1;
  }
  std::vector<int32_t> sorted;
  if (!ascending) {
    sorted.assign(nodes, nodes + n_nodes);
    std::sort(sorted.begin(), sorted.end());
    if (std::adjacent_find(sorted.begin(), sorted.end()) != sorted.end()) return SPEX_ERR_INVALID_ARG;
  }
  if (tokens > INT32_MAX || visits > (1 << 22)) return SPEX_ERR_UNSUPPORTED;
  if (tokens == 0) return SPEX_OK;
  if (!data->k || !data->v) return SPEX_ERR_INVALID_ARG;
  if (positions)
    for (int64_t i = 0; i < tokens; ++i)
      if (positions[i] < 0) return SPEX_ERR_INVALID_ARG;
  if (data->k_scales && data->n_scales < need) return SPEX_ERR_INVALID_ARG;
  if (need > t->pt->free_pages()) return SPEX_ERR_OOM_PAGES;
  // Tokens before each node's own: nodes of a list are mostly siblings, so the last parent's sum is kept.
  std::vector<int32_t> before(positions ? 0 : static_cast<size_t>(n_nodes));
  if (!positions) {
    int32_t parent = spex::kNoNode;
    int64_t sum = 0;
    for (int32_t i = 0; i < n_nodes; ++i) {
      const spex::Node &nd = t->pt->node(nodes[i]);
      if (nd.parent != parent) {
        parent = nd.parent;
        sum = 0;
        for (int32_t w = parent; w != spex::kNoNode; w = t->pt->node(w).parent) sum += t->pt->node(w).n_tokens;
      }
      if (sum + nd.n_tokens + (counts ? counts[i] : 1) > INT32_MAX) return SPEX_ERR_UNSUPPORTED;
      before[i] = static_cast<int32_t>(sum) + nd.n_tokens;
    }
  }

  if (need > 0)
    for (int32_t i = 0; i < n_nodes; ++i) t->pt->reserve(nodes[i], counts ? counts[i] : 1);

  hipStream_t stream = static_cast<hipStream_t>(hip_stream);
  const spex_status_t us = upload_rotation(t, stream);
  if (us != SPEX_OK) return us;
  // The lists go into the kernel arguments if they fit, with some room for length patches of the cached plan, and else into
  // the ring, with room for 32 patches a node as in append_tokens_impl.  A call through the ring takes 5 us more on the host (an event
  // behind the kernel; 140 and 141 nodes of one token: 5.1 / 10.2) and 1.3 on the GPU (records read over the bus; 32/8/128: 6.7 / 8.0).
  const size_t rec_ints = static_cast<size_t>(visits) * spex::kVisitInts;
  const size_t pos_ints = positions ? static_cast<size_t>(tokens) : 0, patch_at = rec_ints + pos_ints;
  const bool plan_follows = t->plan.valid && t->plan_on_device;
  const bool ring = patch_at + (plan_follows ? 8 * static_cast<size_t>(n_nodes) : 0) > spex::kInlineInts;
  const size_t patch_room = ring ? static_cast<size_t>(n_nodes) * 32 : (spex::kInlineInts - patch_at) / 2;
  spex::RotateLists lists;
  int32_t *h = lists.ints;
  if (ring) {
    const spex_status_t rs = spex::ring_reserve(t, (patch_at + 2 * patch_room) * sizeof(int32_t), &h);
    if (rs != SPEX_OK) return rs;
  }
  int32_t *rec = h, most = 0;
  int32_t token = 0, started = 0;
  for (int32_t i = 0; i < n_nodes; ++i) {
    const int32_t u = nodes[i], c = counts ? counts[i] : 1;
    if (c == 0) continue;
    const int32_t old_tokens = t->pt->node(u).n_tokens;
    int32_t first_new = 0;
    t->pt->append(u, c, &first_new);  // cannot fail: the pages were counted and their lists have room
    const spex::Node &nd = t->pt->node(u);
    for (int32_t at = old_tokens; at < old_tokens + c;) {
      const int32_t page = at >> shift, lo = at & (P - 1), n = std::min(P - lo, old_tokens + c - at);
      const bool is_new = page >= first_new;
      rec[0] = nd.pages[page];
      rec[1] = lo | (lo + n) << 8 | (is_new ? 1 << 16 : 0);
      rec[2] = token;
      rec[3] = positions ? 0 : before[i] + at - old_tokens;
      rec[4] = is_new ? started++ : 0;
      rec += spex::kVisitInts;
      most = std::max(most, n);
      token += n;
      at += n;
    }
  }
  if (positions) std::memcpy(h + rec_ints, positions, pos_ints * sizeof(int32_t));
  const size_t n_patch = spex::follow_append(t, h + patch_at, patch_room);

  spex::RotateArgs a{};
  a.k_pool = t->cfg.k_pool;
  a.v_pool = t->cfg.v_pool;
  a.k_scale = t->cfg.k_scale;
  a.v_scale = t->cfg.v_scale;
  a.q = data->q;
  a.k = data->k;
  a.v = data->v;
  a.q_out = data->q_out;
  a.k_out = data->k_out;
  a.q_stride = stride[0];
  a.k_stride = stride[1];
  a.v_stride = stride[2];
  a.q_out_stride = stride[3];
  a.k_out_stride = stride[4];
  a.k_scale_src = data->k_scales;
  a.v_scale_src = data->v_scales;
  a.freq = static_cast<const spex::Turns *>(t->d_freq);
  a.lists = ring ? h : nullptr;
  a.has_positions = positions != nullptr;
  a.n_recs = static_cast<int32_t>(visits);
  a.rotary_dim = t->rotary_dim;
  a.interleaved = t->interleaved;
  a.most_tokens = most;
  a.plan = static_cast<int32_t *>(t->d_plan);
  a.patches = static_cast<int32_t>(patch_at);
  a.n_patches = static_cast<int32_t>(n_patch);
  HIP_TRY(spex::launch_append_rotated(t->shape, a, lists, stream));
  return ring ? spex::ring_commit(t, (patch_at + 2 * n_patch) * sizeof(int32_t), stream) : SPEX_OK;
}

}  // namespace

extern "C" {

spex_status_t spex_tree_set_rotation(spex_tree_t *t, int32_t rotary_dim, const double *inv_freq, int32_t interleaved) {
  if (!t || rotary_dim < 0 || rotary_dim > t->cfg.head_dim || rotary_dim % 2 != 0 || (rotary_dim > 0) != (inv_freq != nullptr))
    return SPEX_ERR_INVALID_ARG;
  const int32_t n = rotary_dim / 2;
  for (int32_t i = 0; i < n; ++i)
    if (!std::isfinite(inv_freq[i])) return SPEX_ERR_INVALID_ARG;
  for (int32_t i = 0; i < n; ++i) {
    const long double turns = static_cast<long double>(inv_freq[i]) / 6.283185307179586476925286766559005768L;
    t->freq[2 * i] = static_cast<double>(turns);
    t->freq[2 * i + 1] = static_cast<double>(turns - static_cast<long double>(t->freq[2 * i]));
  }
  t->rotary_dim = rotary_dim;
  t->interleaved = interleaved != 0;
  t->freq_on_device = false;
  return SPEX_OK;
}

spex_status_t spex_tree_append_rotated(spex_tree_t *t, const spex_node_t *nodes, const int32_t *counts, int32_t n_nodes,
                                       const int32_t *positions, const spex_rotated_t *data, void *hip_stream) {
  try {
    return append_rotated_impl(t, nodes, counts, n_nodes, positions, data, hip_stream);
  } catch (const std::bad_alloc &) {
    return SPEX_ERR_CAPACITY;
  }
}

}  // extern "C"
