// spex_prompt_attention: argument checks and the lists of its launches.  See include/spex_prompt.h.
#include "../../include/spex_prompt.h"

#include <algorithm>
#include <new>
#include <vector>

#include "kernels.hpp"
#include "prompt.hpp"

namespace {

constexpr int32_t kMaxPromptTokens = 1 << 24;
// Workgroups of a launch: with 256 threads each, a launch stays below 2^32 threads.
constexpr int64_t kMaxLaunchGroups = int64_t(1) << 23;

bool aligned16(const void *x) { return (reinterpret_cast<uintptr_t>(x) & 15) == 0; }

// A checked call.
struct Call {
  int64_t strides[4];  // of q, k, v and out
  int64_t total;       // tokens
  spex::PromptKernel kernel;
};

spex_status_t check(const spex_prompt_config_t *cfg, const int32_t *lens, int32_t n_prompts, const void *q, const void *k, const void *v,
                    const void *out, Call *call) {
  if (!cfg || n_prompts < 0 || (n_prompts > 0 && !lens)) return SPEX_ERR_INVALID_ARG;
  if (cfg->num_q_heads <= 0 || cfg->num_kv_heads <= 0 || cfg->num_kv_heads > 255 || cfg->num_q_heads % cfg->num_kv_heads != 0 ||
      cfg->head_dim < 1 || cfg->head_dim > 256)
    return SPEX_ERR_INVALID_ARG;
  if (cfg->dtype != SPEX_F32 && cfg->dtype != SPEX_BF16) return SPEX_ERR_UNSUPPORTED;
  const int64_t q_row = static_cast<int64_t>(cfg->num_q_heads) * cfg->head_dim;
  const int64_t kv_row = static_cast<int64_t>(cfg->num_kv_heads) * cfg->head_dim;
  const int64_t given[4] = {cfg->q_stride, cfg->k_stride, cfg->v_stride, cfg->out_stride}, dense[4] = {q_row, kv_row, kv_row, q_row};
  for (int i = 0; i < 4; ++i) {
    call->strides[i] = given[i] ? given[i] : dense[i];
    if (call->strides[i] < dense[i]) return SPEX_ERR_INVALID_ARG;
  }
  for (int64_t s : call->strides)
    if (s > INT32_MAX) return SPEX_ERR_UNSUPPORTED;
  int64_t total = 0, row_sets = 0;
  int32_t longest = 0;
  for (int32_t i = 0; i < n_prompts; ++i) {
    if (lens[i] < 0) return SPEX_ERR_INVALID_ARG;
    if (lens[i] > kMaxPromptTokens) return SPEX_ERR_UNSUPPORTED;
    total += lens[i];
    longest = std::max(longest, lens[i]);
    row_sets += (lens[i] + spex::kPromptRows - 1) / spex::kPromptRows;
  }
  // the kernels count a prompt's row sets of one kv head in 32 bits, with a workgroup's to spare
  const int64_t longest_sets = (static_cast<int64_t>(longest) + spex::kPromptRows - 1) / spex::kPromptRows;
  if (total > INT32_MAX || longest_sets * (cfg->num_q_heads / cfg->num_kv_heads) > INT32_MAX - 64) return SPEX_ERR_UNSUPPORTED;
  call->total = total;
  if (total == 0) return SPEX_OK;
  if (!q || !k || !v || !out) return SPEX_ERR_INVALID_ARG;

  const int64_t per16 = cfg->dtype == SPEX_F32 ? 4 : 8;
  bool wide = cfg->head_dim % per16 == 0 && aligned16(q) && aligned16(k) && aligned16(v) && aligned16(out);
  for (int64_t s : call->strides) wide = wide && s % per16 == 0;
  // offsets inside a tile of up to 64 tokens are 32 bits
  wide = wide && std::max({call->strides[0], call->strides[1], call->strides[2]}) * (16 / per16) < (int64_t(1) << 24);
  call->kernel = spex::prompt_kernel(cfg->dtype == SPEX_F32, wide, cfg->head_dim, row_sets * cfg->num_q_heads, longest);
  return SPEX_OK;
}

}  // namespace

extern "C" spex_status_t spex_prompt_form(const spex_prompt_config_t *cfg, const int32_t *lens, int32_t n_prompts, const void *q,
                                          const void *k, const void *v, const void *out, int32_t *form) {
  if (!form) return SPEX_ERR_INVALID_ARG;
  Call call;
  const spex_status_t st = check(cfg, lens, n_prompts, q, k, v, out, &call);
  if (st != SPEX_OK) return st;
  const spex::PromptKernel &kn = call.kernel;
  if (call.total == 0)
    *form = -1;
  else if (!kn.wide)
    *form = 0;
  else if (kn.split)
    *form = kn.eight ? 4 : 3;
  else
    *form = kn.short_tiles ? 2 : 1;
  return SPEX_OK;
}

extern "C" spex_status_t spex_prompt_attention(const spex_prompt_config_t *cfg, const int32_t *lens, int32_t n_prompts,
                                               const void *q, const void *k, const void *v, void *out, float *lse,
                                               float sm_scale, void *hip_stream) {
  Call call;
  const spex_status_t st = check(cfg, lens, n_prompts, q, k, v, out, &call);
  if (st != SPEX_OK) return st;
  if (!(sm_scale >= 1e-38f && sm_scale <= 1e37f)) return SPEX_ERR_INVALID_ARG;  // times log2(e) it has a reciprocal in fp32
  if (call.total == 0) return SPEX_OK;
  const spex::PromptKernel &kernel = call.kernel;
  const int32_t G = cfg->num_q_heads / cfg->num_kv_heads;

  struct Prompt {
    int32_t start, len;
  };
  Prompt few[64], *list = few;
  std::vector<Prompt> many;
  try {
    if (n_prompts > 64) {
      many.resize(static_cast<size_t>(n_prompts));
      list = many.data();
    }
  } catch (const std::bad_alloc &) {
    return SPEX_ERR_CAPACITY;
  }
  int32_t n = 0, at = 0;
  for (int32_t i = 0; i < n_prompts; ++i) {
    if (lens[i] > 0) {
      list[n++] = {at, lens[i]};
    }
    at += lens[i];
  }
  // Longest first: the workgroups with most work start first, within a prompt and over all of them.
  std::sort(list, list + n, [](const Prompt &a, const Prompt &b) { return a.len != b.len ? a.len > b.len : a.start < b.start; });

  spex::PromptArgs a;
  a.q = q;
  a.k = k;
  a.v = v;
  a.out = out;
  a.lse = lse;
  a.q_stride = call.strides[0];
  a.k_stride = call.strides[1];
  a.v_stride = call.strides[2];
  a.out_stride = call.strides[3];
  a.scale_log2 = sm_scale * 1.4426950408889634f;
  a.Hkv = cfg->num_kv_heads;
  a.G = G;
  a.D = cfg->head_dim;
  const int64_t room = kMaxLaunchGroups / cfg->num_kv_heads;
  int64_t done = 0;  // items of prompt i that launches before have taken
  for (int32_t i = 0; i < n;) {
    int64_t items = 0;
    for (a.n = 0; i < n && a.n < spex::kMaxPromptsPerLaunch && items < room; ++a.n) {
      const int64_t left = spex::prompt_items(kernel, G, list[i].len) - done, take = std::min(left, room - items);
      a.first[a.n] = static_cast<int32_t>(items - done);
      a.start[a.n] = list[i].start;
      a.len[a.n] = list[i].len;
      items += take;
      done = take < left ? done + take : 0;
      if (done == 0) ++i;
    }
    for (int32_t j = a.n; j < spex::kMaxPromptsPerLaunch; ++j) {
      a.first[j] = INT32_MAX;
      a.start[j] = a.len[j] = 0;
    }
    if (spex::hip_failed(spex::launch_prompt(kernel, a, items, static_cast<hipStream_t>(hip_stream)), "launch_prompt"))
      return SPEX_ERR_DEVICE;
  }
  return SPEX_OK;
}
