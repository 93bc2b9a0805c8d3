// MXFP4 pools: what the calls on such a handle go through, and spex_tree_read_back, its argument checks and the launch's lists.  See
// include/spex_tree.h.
#include <algorithm>
#include <new>

#include "tree.hpp"

namespace {

spex_status_t read_back_impl(spex_tree_t *t, const spex_node_t *nodes, const int32_t *firsts, const int32_t *counts, int32_t n_nodes,
                             void *k_out, void *v_out, int64_t *n_tokens, void *hip_stream) {
  const int32_t P = t->cfg.page_size;
  int64_t tokens = 0, visits = 0;
  for (int32_t i = 0; i < n_nodes; ++i) {
    if (!t->pt->valid(nodes[i])) return SPEX_ERR_BAD_NODE;
    const int64_t have = t->pt->node(nodes[i]).n_tokens, first = firsts ? firsts[i] : 0, n = counts ? counts[i] : have - first;
    if (first < 0 || n < 0 || first + n > have) return SPEX_ERR_INVALID_ARG;
    tokens += n;
    if (n > 0) visits += (first + n - 1) / P - first / P + 1;
  }
  if (tokens > INT32_MAX || visits > (1 << 22)) return SPEX_ERR_UNSUPPORTED;
  const bool count_only = !k_out && !v_out && n_tokens;
  if (tokens > 0 && !count_only && (!k_out || !v_out || !t->cfg.k_pool)) return SPEX_ERR_INVALID_ARG;
  if (tokens == 0 || count_only) {
    if (n_tokens) *n_tokens = tokens;
    return SPEX_OK;
  }

  hipStream_t stream = static_cast<hipStream_t>(hip_stream);
  const size_t ints = static_cast<size_t>(visits) * spex::kReadInts;
  const bool ring = ints > spex::kInlineInts;
  spex::RotateLists lists;
  int32_t *h = lists.ints;
  if (ring) {
    const spex_status_t rs = spex::ring_reserve(t, ints * sizeof(int32_t), &h);
    if (rs != SPEX_OK) return rs;
  }
  int32_t *rec = h, token = 0;
  for (int32_t i = 0; i < n_nodes; ++i) {
    const spex::Node &nd = t->pt->node(nodes[i]);
    const int32_t first = firsts ? firsts[i] : 0, end = counts ? first + counts[i] : nd.n_tokens;
    for (int32_t at = first; at < end;) {
      const int32_t page = at / P, lo = at % P, n = std::min(P - lo, end - at);
      rec[0] = nd.pages[page];
      rec[1] = lo | (lo + n) << 8;
      rec[2] = token;
      rec += spex::kReadInts;
      token += n;
      at += n;
    }
  }
  spex::ReadBackArgs a{};
  a.k_pool = t->cfg.k_pool;
  a.v_pool = t->cfg.v_pool;
  a.k_out = k_out;
  a.v_out = v_out;
  a.lists = ring ? h : nullptr;
  a.n_recs = static_cast<int32_t>(visits);
  HIP_TRY(spex::launch_mxfp4_read(t->shape, a, lists, stream));
  if (n_tokens) *n_tokens = tokens;
  return ring ? spex::ring_commit(t, ints * sizeof(int32_t), stream) : SPEX_OK;
}

spex_status_t read_back(spex_tree_t *t, const spex_node_t *nodes, const int32_t *firsts, const int32_t *counts, int32_t n_nodes,
                        void *k_out, void *v_out, int64_t *n_tokens, void *hip_stream) {
  try {
    return read_back_impl(t, nodes, firsts, counts, n_nodes, k_out, v_out, n_tokens, hip_stream);
  } catch (const std::bad_alloc &) {
    return SPEX_ERR_CAPACITY;
  }
}

const spex::Mxfp4Calls kCalls = {spex::append_quantised, read_back, spex::launch_mxfp4_split, spex::launch_mxfp4_walk};
const bool kKnown = (spex::mxfp4_calls = &kCalls, true);

}  // namespace

extern "C" spex_status_t spex_tree_read_back(spex_tree_t *t, const spex_node_t *nodes, const int32_t *firsts, const int32_t *counts,
                                             int32_t n_nodes, void *k_out, void *v_out, int64_t *n_tokens, void *hip_stream) {
  if (!t || n_nodes < 0 || (n_nodes > 0 && !nodes)) return SPEX_ERR_INVALID_ARG;
  if (t->cfg.kv_dtype != SPEX_MXFP4) return SPEX_ERR_UNSUPPORTED;
  return read_back(t, nodes, firsts, counts, n_nodes, k_out, v_out, n_tokens, hip_stream);
}
