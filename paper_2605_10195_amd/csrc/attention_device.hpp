// Device code shared by the attention kernels: reads of the launch lists, work items, exchanges between the lanes of a row.
#pragma once

#include <hip/hip_runtime.h>

#include <climits>
#include <cstdint>

#include "kernels.hpp"

namespace spex {
namespace {

typedef __bf16 bf16x8 __attribute__((ext_vector_type(8)));
typedef _Float16 f16x8 __attribute__((ext_vector_type(8)));
typedef _Float16 f16x2 __attribute__((ext_vector_type(2)));
typedef float f32x4 __attribute__((ext_vector_type(4)));
typedef float f32x2 __attribute__((ext_vector_type(2)));
typedef uint32_t u32x4 __attribute__((ext_vector_type(4)));
typedef uint32_t u32x2 __attribute__((ext_vector_type(2)));

constexpr float kNegInf = -__builtin_huge_valf();

__device__ __forceinline__ int uniform(int v) { return __builtin_amdgcn_readfirstlane(v); }

// Wave-uniform read of plan data through the scalar (constant) path.  The plan arrays are
// written by the host before the launch and never by a kernel.  Going through scalar loads keeps
// these small reads out of the vector-memory queue, whose in-order completion counter would
// otherwise make every page-record lookup wait for all K/V loads in flight.
typedef const int32_t __attribute__((address_space(4))) const_i32;
__device__ __forceinline__ int sload(const int32_t *base, int64_t idx) {
  return ((const_i32 *)(uintptr_t)base)[idx];
}

__device__ __forceinline__ float fast_exp2(float x) { return __builtin_amdgcn_exp2f(x); }

// Maximum over lanes l, l^16, l^32, l^48 (the four lane groups that hold one query row), by the
// gfx950 row-swap instructions: v_permlane16_swap exchanges the odd 16-lane rows of its first
// operand with the even rows of its second, v_permlane32_swap the upper half of the first with
// the lower half of the second; with both operands equal, the pair afterwards holds the value of
// the lane and of its partner.  Two wait states separate a vector write from a swap that reads it.
// The compiler does not track hazards of instructions inside inline assembly, so the argument must
// be the result of an ordinary vector ALU instruction (here: the v_max that folds in the running
// maximum) -- never directly of an MFMA, whose results need many more wait states before they can
// be read.
__device__ __forceinline__ float row_group_max(float v) {
  float a = v, b = v;
  asm("s_nop 1\n\t"
      "v_permlane16_swap_b32 %0, %1\n\t"
      "v_max_f32 %0, %0, %1\n\t"
      "v_mov_b32 %1, %0\n\t"
      "s_nop 1\n\t"
      "v_permlane32_swap_b32 %0, %1\n\t"
      "v_max_f32 %0, %0, %1"
      : "+v"(a), "+v"(b));
  return a;
}

// Wave-uniform description of one work item.
struct Item {
  int pg_begin, pg_count, qt_begin, qt_count, pbase, flags, g, row0;
};

__device__ __forceinline__ Item load_item(const int32_t *items, int idx) {
  const int64_t r = static_cast<int64_t>(uniform(idx)) * 8;
  Item it;
  it.pg_begin = sload(items, r + 0);
  it.pg_count = sload(items, r + 1);
  it.qt_begin = sload(items, r + 2);
  it.qt_count = sload(items, r + 3);
  it.pbase = sload(items, r + 4);
  it.flags = sload(items, r + 5);
  it.g = sload(items, r + 6);
  it.row0 = sload(items, r + 7);
  return it;
}

// Page ids / valid counts / positions of one 32-token block, wave-uniform.
struct BlockMeta {
  int pid_a, pid_b, vp_a, vp_b;  // vp = position << 7 | valid; vp_b = 0 when the block has one page
};

__device__ __forceinline__ BlockMeta load_block_meta(const int32_t *pg_rec, const Item &it, int b) {
  const int ia = it.pg_begin + 2 * b;
  const bool has_b = 2 * b + 1 < it.pg_count;
  const int ib = has_b ? ia + 1 : ia;
  BlockMeta bm;
  bm.pid_a = sload(pg_rec, 2 * ia);
  bm.vp_a = sload(pg_rec, 2 * ia + 1);
  bm.pid_b = sload(pg_rec, 2 * ib);
  bm.vp_b = has_b ? sload(pg_rec, 2 * ib + 1) : 0;
  return bm;
}

// The work items of a launch, in up to four lists: workgroup wg_end[k - 1] .. wg_end[k] - 1 belong to
// list k.
struct SplitLists {
  static constexpr int kLists = 4;
  const int32_t *items[kLists];
  int32_t wg_end[kLists];
  int32_t n_items[kLists];
  int32_t span[kLists];     // rows an item of the list covers from its first row on
};
// The list the workgroup belongs to and its index there.
struct ListPos {
  int k, local, n_items, span;
  const int32_t *items;
};
__device__ __forceinline__ ListPos list_of(const SplitLists &ls, int wg) {
  ListPos r = {0, wg, ls.n_items[0], ls.span[0], ls.items[0]};
#pragma unroll
  for (int i = 1; i < SplitLists::kLists; ++i) {  // member by member: as a whole the lists go through scratch memory
    const bool in = wg >= ls.wg_end[i - 1];
    r.k = in ? i : r.k;
    r.local = in ? wg - ls.wg_end[i - 1] : r.local;
    r.n_items = in ? ls.n_items[i] : r.n_items;
    r.span = in ? ls.span[i] : r.span;
    r.items = in ? ls.items[i] : r.items;
  }
  return r;
}

// rows_per_wg: rows of an item one workgroup takes.  n_wg < 0: too many.
inline SplitLists make_lists(const ItemLists &l, int rows_per_wg, int64_t *n_wg) {
  SplitLists ls{};
  *n_wg = 0;
  for (int k = 0; k < SplitLists::kLists; ++k) {
    ls.items[k] = l.items[k];
    ls.n_items[k] = l.n_items[k] > 0 ? l.n_items[k] : 1;  // a divisor
    ls.span[k] = l.span[k];
    *n_wg += static_cast<int64_t>(l.n_items[k]) * ((l.span[k] + rows_per_wg - 1) / rows_per_wg);
    ls.wg_end[k] = static_cast<int32_t>(*n_wg);
    if (*n_wg > INT32_MAX) {
      *n_wg = -1;
      break;
    }
  }
  return ls;
}

}  // namespace
}  // namespace spex
