// A handle of spex_tree.h and what the files behind its entry points share.
#pragma once

#include <hip/hip_runtime.h>

#include <cstddef>
#include <cstdint>
#include <vector>

#include "../../include/spex_tree.h"
#include "kernels.hpp"
#include "page_table.hpp"
#include "planner.hpp"

#define HIP_TRY(expr)                                            \
  do {                                                           \
    if (spex::hip_failed((expr), #expr)) return SPEX_ERR_DEVICE; \
  } while (0)

namespace spex {

// Device copy of a Plan: one blob, arrays at 256-byte aligned offsets.
struct DevicePlan {
  const int32_t *prefix_items = nullptr, *suffix_items = nullptr, *pg_rec = nullptr, *qt_rec = nullptr;
  const int32_t *part_indptr = nullptr, *part_base = nullptr, *part_hstride = nullptr, *merge_qt = nullptr;
  const int32_t *coop_items[2] = {nullptr, nullptr};
  const int32_t *walk_items = nullptr, *walk_blocks = nullptr, *walk_qt = nullptr, *qt_mask = nullptr;
};

}  // namespace spex

struct spex_tree {
  spex_config_t cfg{};
  spex::Shape shape{};
  spex::PageTable *pt = nullptr;
  spex::Planner planner;
  spex::Plan plan;
  bool plan_on_device = false, device_has_split = false, device_has_walk = false;
  bool plan_patched_by_append = false;  // the cached plan was brought up to date by an append call
  spex::DevicePlan dplan;
  size_t blob_off[14] = {}, blob_ints[14] = {};  // byte offset and length of each list in the blob
  std::vector<int32_t> pending_patches;          // {array, index, value} not yet on the device
  void *d_patch = nullptr;
  size_t d_patch_cap = 0;

  void *d_plan = nullptr;
  size_t d_plan_cap = 0;
  // Pinned staging for host -> device copies (plans and their patches).  Two slots
  // used in turn: the host may fill one while the copy out of the other is still queued behind
  // earlier kernels, so it can prepare the next call while the GPU runs the current one.
  struct Stage {
    void *h = nullptr;
    size_t cap = 0;
    hipEvent_t event = nullptr;
    bool pending = false;
  } stage[2];
  int stage_cur = 0;
  void *h_stage = nullptr;  // the slot reserved last (stage[stage_cur].h)
  // Pinned lists that the append kernel reads where they are: one block cut into segments that are filled
  // one after the other, several calls to a segment, so that the host may run that many calls ahead of the GPU.
  struct Ring {
    static constexpr int kSegments = 4, kCalls = 16;  // calls to a segment: at most kCalls
    char *base = nullptr;
    size_t seg_bytes = 0, used = 0;  // bytes of the current segment that calls have taken
    int cur = 0;
    struct Segment {
      hipEvent_t event[kCalls] = {};  // one behind each call's kernel, made when first needed
      int calls = 0;                  // calls whose lists lie in the segment
    } seg[kSegments];
  } ring;

  // Position rotation: frequencies in turns a position, two doubles each, and their copy on the device.
  int32_t rotary_dim = 0;
  bool interleaved = false, freq_on_device = false;
  double freq[256] = {};
  void *d_freq = nullptr;

  float *d_part_o = nullptr, *d_part_ml = nullptr;
  int64_t part_cap_rows = 0;
  std::vector<char> static_stage;  // host image of the lists for the entry point that allocates nothing

  int32_t prefix_chunk = 0, suffix_chunk = 0, kernel_mode = 0, walk_row_tiles = 0, walk_waves = 0;
  // Profiling: a ring of event sets, one per decode_attention call since it was enabled.
  static constexpr int kProfSlots = 256;
  struct ProfSlot {
    hipEvent_t ev[8] = {nullptr, nullptr, nullptr, nullptr, nullptr, nullptr, nullptr, nullptr};
    bool valid[4] = {false, false, false, false};
  };
  bool profiling = false;
  std::vector<ProfSlot> prof;
  int64_t prof_calls = 0;  // calls recorded since profiling was enabled / last read
  int64_t info[8] = {0, 0, 0, 0, 0, 0, 0, 0};
};

namespace spex {

// Pinned lists of a launch, in api.cpp: room for up to `bytes`, and, behind the kernel that reads the first `bytes` of them, their event.
spex_status_t ring_reserve(spex_tree *t, size_t bytes, int32_t **out);
spex_status_t ring_commit(spex_tree *t, size_t bytes, hipStream_t stream);
// Behind an append to the page table, in api.cpp: the cached plan's patches as {index, value} pairs for the append's launch, at most
// `room` of them (0 where there are none, or more).
size_t follow_append(spex_tree *t, int32_t *pairs, size_t room);

}  // namespace spex
