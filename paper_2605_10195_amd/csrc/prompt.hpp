// Launch interface between spex_prompt_attention and its kernels.
#pragma once

#include <hip/hip_runtime.h>

#include <cstdint>

namespace spex {

// Prompts of one launch.  Their list travels in the kernel arguments (1.5 KB), so that a call needs no memory of its
// own; more prompts take more launches.
constexpr int kMaxPromptsPerLaunch = 128;
// Rows (tokens of one query head) of a wavefront.
constexpr int kPromptRows = 32;

struct PromptArgs {
  const void *q, *k, *v;
  void *out;
  float *lse;  // may be null
  int64_t q_stride, k_stride, v_stride, out_stride;  // elements between tokens
  float scale_log2;
  int32_t Hkv, G, D;
  int32_t n;                                // prompts of this launch, longest first
  // work items (of one kv head) before the prompt's, less those of it that an earlier launch has taken; INT32_MAX behind the last
  int32_t first[kMaxPromptsPerLaunch];
  int32_t start[kMaxPromptsPerLaunch];      // first token
  int32_t len[kMaxPromptsPerLaunch];        // tokens
};

// The kernel for the launches of one call.
struct PromptKernel {
  bool f32, wide;    // type; rows of 16-byte pieces (else element by element)
  bool split;        // a workgroup splits the keys of its rows over its wavefronts
  bool eight;        // eight of them instead of four
  bool short_tiles;  // tiles of 32 keys instead of 64
  int32_t sets;      // row sets of kPromptRows rows a work item has
};
// row_sets: of all prompts and query heads; longest: tokens of the longest prompt
PromptKernel prompt_kernel(bool f32, bool wide, int32_t head_dim, int64_t row_sets, int32_t longest);
// Work items of one kv head that a prompt of `len` tokens makes.
int64_t prompt_items(const PromptKernel &k, int32_t heads_per_kv, int32_t len);
// a.first / start / len filled for a.n prompts, `items` of them together for one kv head.
hipError_t launch_prompt(const PromptKernel &k, const PromptArgs &a, int64_t items, hipStream_t stream);

}  // namespace spex
