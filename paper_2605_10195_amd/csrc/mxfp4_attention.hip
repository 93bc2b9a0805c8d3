// HIP kernels of decode attention over microscaled 4-bit (MXFP4) pools on gfx950 (CDNA4, 64-lane wavefronts).
//
//   spex_mxfp4_split_kernel
//       The split path's items, a workgroup for up to 16 NT rows of one: its four wavefronts take every fourth block of 32 tokens
//       and join their softmax states through LDS.  Partial states go to the merge kernel, as for the other pools.
//   spex_mxfp4_walk_kernel
//       The tree walk: the same over the whole path of up to 16 NT rows, from the root to the requested nodes, by a wavefront or by
//       four.  Nothing but finished rows is written, except where long paths go in pieces.
//   spex_mxfp4_merge_kernel
//       Merges the pieces' states of every row.
//
// Mathematics: S^T = K Q^T, p = 2^(c S^T - m), l += sum p, O += P V, out = O / l, with keys and values code * 2^E.
// Keys become bf16 operands, which hold code * 2^E exactly (two significant bits), values fp16, which do as well since the values' E is
// bounded; v_cvt_scalef32_pk_* makes two of them from a byte and the scale.  Queries are the caller's bf16.  Weights go into the product
// as two fp16 pieces, 22 bits, so that nothing is rounded to fewer bits than fp32 sums lose.
//
// Bound: the instructions a SIMD can issue.  A block of 32 tokens and a tile of 16 rows of a head of 128 are 26 products of 16 cycles and
// about 145 vector instructions of 4 (64 conversions, 70 for the weights), and the two kinds of a SIMD's wavefronts hardly run side by
// side; a second row tile shares the conversions.  The second piece of the weights is a third of the products.  Few rows on long paths
// are bound by how fast wavefronts get their blocks.
//
// No LDS in the loop: a tile is held in the order in which its lanes consume it (mxfp4_device.hpp), so a block's codes go from memory
// into the registers they are converted in.  A ring of blocks in LDS, filled by copies of its own three or four ahead, was slower
// (64 roots of 2500 tokens with 32 branches of 256: 190 us against 171).
#include <algorithm>
#include <type_traits>

#include "attention_device.hpp"
#include "kernels.hpp"
#include "mxfp4_device.hpp"

namespace spex {
namespace {

typedef uint32_t u32x8 __attribute__((ext_vector_type(8)));
typedef _Float16 f16x16 __attribute__((ext_vector_type(16)));
typedef u32x4 u32x4_q __attribute__((aligned(2)));   // queries: any alignment of their type
typedef f32x4 f32x4_out __attribute__((aligned(4)));
typedef f32x2 f32x2_out __attribute__((aligned(4)));

// Start of a row's softmax reference: finite, so that (-inf) - m stays -inf, and below any score.
constexpr float kMInit = -1.0e30f;
// How far a score may exceed the reference before that moves, and the exponent of a weight at the reference: weights stay below 2^15,
// fp16's largest, and the smallest fp16 step is 2^-31 of a row's largest weight at most.
constexpr float kSlackLog2 = 8.f, kWeightLog2 = 7.f, kWeightUnit = 1.f / 128.f;  // (2^-kWeightLog2)
// Places of a sparse product's weights: 0 and 2, or 1 and 3, of every four.
constexpr int kEvenDims = static_cast<int>(0x88888888u), kOddDims = static_cast<int>(0xddddddddu);
// From here on references are subtracted as scores.  Scaled ones are rounded by up to 2^-2 here, by 1 from 2^24 on, and all weights are off
// by as much: more would take them out of fp16.
constexpr float kFarLog2 = 4194304.f;

// A reference as it is subtracted from scaled scores.  Finite: a row that has met no score keeps kMInit, whatever the scale, and a score that
// it does not see has to stay -inf.
__device__ __forceinline__ float scaled_reference(float m, float c) { return fmaxf(__builtin_fmaf(m, c, -kWeightLog2), -3.0e38f); }

// A block of 32 tokens: pages a and b, wave-uniform.
struct MxBlock {
  int64_t at[2];   // where the pages' tiles begin in a pool
  int vp_a, vp_b;  // position << 7 | kMasked | kRowMasked | valid tokens; vp_b 0: no page b
  int rows;        // first row | (last row + 1) << 16 of the row block whose path holds it
  bool live;       // there is such a block
};
constexpr int kMasked = 64, kRowMasked = 32, kValid = 31;  // of page a: some row sees a part of the block; some row is not on its path

// The keys and the values of a block as they lie in memory.
template <int M>
struct MxKeys {
  static constexpr int kScales = kMxRun<M> ? (M == 8 ? 2 : 1) : M;
  uint32_t w[2][M];
  uint32_t scale[2][kScales];  // a byte each
};
template <int M>
struct MxValues {
  static constexpr int kScales = kMxRun<M> ? 1 : M;
  uint32_t w[2 * M];           // of the lane's first four tokens, of its second
  uint32_t scale[2][kScales];  // four tokens' bytes each
};

template <int N>
__device__ __forceinline__ void load_words(const char *p, uint32_t (&w)[N]) {
  typedef uint32_t word4 __attribute__((ext_vector_type(4), aligned(4)));
  typedef uint32_t word3 __attribute__((ext_vector_type(3), aligned(4)));
  typedef uint32_t word2 __attribute__((ext_vector_type(2), aligned(4)));
#pragma unroll
  for (int i = 0; i < N; i += 4) {
    if (N - i >= 4) {
      const word4 x = *reinterpret_cast<const word4 *>(p + 4 * i);
#pragma unroll
      for (int j = 0; j < 4; ++j) w[i + j] = x[j];
    } else if (N - i == 3) {
      const word3 x = *reinterpret_cast<const word3 *>(p + 4 * i);
#pragma unroll
      for (int j = 0; j < 3; ++j) w[i + j] = x[j];
    } else if (N - i == 2) {
      const word2 x = *reinterpret_cast<const word2 *>(p + 4 * i);
      w[i] = x[0];
      w[i + 1] = x[1];
    } else {
      w[i] = *reinterpret_cast<const uint32_t *>(p + 4 * i);
    }
  }
}

// Lane (g, t): token t of both pages.  A block that is not there, and page b of a block without one, are read at another place of the pool.
template <int M>
__device__ __forceinline__ void load_keys(MxKeys<M> &x, const MxBlock &b, const void *pool) {
  const int lane = threadIdx.x & 63, c = lane & 15, jj = lane >> 4;
#pragma unroll
  for (int p = 0; p < 2; ++p) {
    const char *tile = static_cast<const char *>(pool) + b.at[p];
    load_words<M>(tile + static_cast<uint32_t>(lane * 4 * M), x.w[p]);
#pragma unroll
    for (int i = 0; i < MxKeys<M>::kScales; ++i) {
      const int block = kMxRun<M> ? (M >= 4 ? jj * (M / 4) + i : jj * M / 4) : i;
      x.scale[p][i] = *reinterpret_cast<const uint8_t *>(tile + static_cast<uint32_t>(mx_key_scale_at<M>(block, c)));
    }
  }
}
// Lane (g, c): page g % 2, tokens 4 (g / 2) .. + 3 and 8 further on, the order in which the sparse product takes them (block_values).
template <int M>
__device__ __forceinline__ void load_values(MxValues<M> &x, const MxBlock &b, const void *pool) {
  const int lane = threadIdx.x & 63, c = lane & 15, page = (lane >> 4) & 1, tg = lane >> 5;
  const char *tile = static_cast<const char *>(pool) + (b.at[0] + ((b.at[1] - b.at[0]) & -static_cast<int64_t>(page)));
  load_words<2 * M>(tile + (16 * tg + c) * 8 * M, x.w);
#pragma unroll
  for (int i = 0; i < MxValues<M>::kScales; ++i) {
    const u32x2 e = *reinterpret_cast<const u32x2 *>(tile + mx_value_scale_at<M>(kMxRun<M> ? c * M / 16 : i, tg));
    x.scale[0][i] = e[0];
    x.scale[1][i] = e[1];
  }
}

// A wavefront's rows, 16 to a tile: lane (c = lane % 16, jj = lane / 16) has row c of every tile; its scores are of tokens 4 jj .. + 3
// of page a, then of page b; its accumulators 2 j and 2 j + 1 are of rows 4 jj .. + 3 and the dims mx_value_dim(c, j) and the one behind.
template <int M, int NT>
struct MxRows {
  bf16x8 q[NT][M];
  int limit[NT], qtok[NT], qidx[NT];
  uint32_t dmask[NT];
  f32x4 o[NT][2 * M];
  f32x4 l[NT];                 // the weights' sums of rows 4 jj .. + 3, as a product with ones gives them
  float m[NT], mc[NT];         // reference as a score, and scaled less kWeightLog2
  int seen_end;                // path positions from here on no row sees (wave-uniform)
  int far;                     // wave-uniform: bit nt, some reference of tile nt is beyond kFarLog2
};

// A state's weights are 2^(c s - mc) with mc as it is rounded.  Log2 of how much less that is than 2^(c (s - m) + kWeightLog2): up to half a unit
// of mc, 2^-3 just below kFarLog2, which states with other references do not share.  Joins make up for it.
template <int M, int NT>
__device__ __forceinline__ float rounded_off(const MxRows<M, NT> &st, int nt, float c) {
  return (st.far >> nt & 1) != 0 || st.m[nt] == kMInit ? 0.f : -__builtin_fmaf(st.m[nt], c, -(st.mc[nt] + kWeightLog2));
}

template <int M, int NT, bool TREE>
__device__ __forceinline__ void load_rows(MxRows<M, NT> &st, const void *q, const int32_t *qt_rec, const int32_t *qt_mask, int qt_begin,
                                          int row_base, int rows, int g, const Shape &sh, float c) {
  const int lane = threadIdx.x & 63, jj = lane >> 4;
  int end = 0;
#pragma unroll
  for (int nt = 0; nt < NT; ++nt) {
    const int r = row_base + 16 * nt + (lane & 15);
    st.limit[nt] = INT_MAX;
    st.qtok[nt] = st.qidx[nt] = 0;
    st.dmask[nt] = 0;
    st.m[nt] = kMInit;
    st.mc[nt] = scaled_reference(kMInit, c);
    st.l[nt] = f32x4{0.f, 0.f, 0.f, 0.f};
#pragma unroll
    for (int i = 0; i < 2 * M; ++i) st.o[nt][i] = f32x4{0.f, 0.f, 0.f, 0.f};
    if (r < rows) {
      const int2 qr = *reinterpret_cast<const int2 *>(qt_rec + 2 * (static_cast<int64_t>(qt_begin) + r / sh.G));
      st.qtok[nt] = qr.x;
      st.limit[nt] = qr.y;
      end = max(end, qr.y + (TREE ? 31 : 0));
      if (TREE) {
        const int2 dm = *reinterpret_cast<const int2 *>(qt_mask + 2 * static_cast<int64_t>(qr.x));
        st.qidx[nt] = dm.x;
        st.dmask[nt] = static_cast<uint32_t>(dm.y);
      }
      const uint16_t *qp = static_cast<const uint16_t *>(q) + (static_cast<int64_t>(qr.x) * sh.Hq + g * sh.G + r % sh.G) * (32 * M);
#pragma unroll
      for (int s = 0; s < M; ++s) st.q[nt][s] = __builtin_bit_cast(bf16x8, *reinterpret_cast<const u32x4_q *>(qp + mx_key_dim<M>(jj, s)));
    } else {
#pragma unroll
      for (int s = 0; s < M; ++s) st.q[nt][s] = __builtin_bit_cast(bf16x8, u32x4{0, 0, 0, 0});
    }
  }
#pragma unroll
  for (int o = 8; o >= 1; o >>= 1) end = max(end, __shfl_xor(end, o));
  st.seen_end = uniform(end);
  st.far = 0;
}

// Which of the lane's four tokens of a page the row sees, as bits.
template <bool TREE, bool REMAKE>
__device__ __forceinline__ uint32_t seen_bits(int limit, int qidx, uint32_t dmask, int vp, int first) {
  const int valid = (vp & kValid) - first, pos = (vp >> 7) + first;
  if (TREE) {  // positions below base, and base + k for the set bits k of the mask
    if (REMAKE) asm volatile("" : "+v"(dmask));  // the word below is made here and not kept in two registers for the whole path
    const int shift = pos - (limit - 1 - qidx) + 32;
    const uint64_t bits = (static_cast<uint64_t>(dmask) << 32) | 0xffffffffull;
    const uint32_t seen = shift <= 0 ? 0xfu : (shift >= 64 ? 0u : static_cast<uint32_t>(bits >> shift));
    return seen & ((1u << min(max(valid, 0), 4)) - 1u);
  }
  return (1u << min(max(min(valid, limit - pos), 0), 4)) - 1u;
}

// p - h for the two halves of hh, rounded toward zero to fp16.  The mixed fma takes an fp16 operand as it is.
__device__ __forceinline__ uint32_t rest_of(uint32_t hh, float p0, float p1) {
  float r0, r1;
  asm("v_fma_mix_f32 %0, %1, -1.0, %2 op_sel_hi:[1,0,0]" : "=v"(r0) : "v"(hh), "v"(p0));
  asm("v_fma_mix_f32 %0, %1, -1.0, %2 op_sel:[1,0,0] op_sel_hi:[1,0,0]" : "=v"(r1) : "v"(hh), "v"(p1));
  return __builtin_bit_cast(uint32_t, __builtin_amdgcn_cvt_pkrtz(r0, r1));
}

template <int M>
__device__ __forceinline__ bf16x8 key_operand(uint32_t w, float scale) {
  u32x4 r;
  r[0] = __builtin_bit_cast(uint32_t, __builtin_amdgcn_cvt_scalef32_pk_bf16_fp4(w, scale, 0));
  r[1] = __builtin_bit_cast(uint32_t, __builtin_amdgcn_cvt_scalef32_pk_bf16_fp4(w, scale, 1));
  r[2] = __builtin_bit_cast(uint32_t, __builtin_amdgcn_cvt_scalef32_pk_bf16_fp4(w, scale, 2));
  r[3] = __builtin_bit_cast(uint32_t, __builtin_amdgcn_cvt_scalef32_pk_bf16_fp4(w, scale, 3));
  return __builtin_bit_cast(bf16x8, r);
}

// Scores of a block's 32 tokens, eight a lane and row: the four of page a, the four of page b.
template <int NT>
struct MxScores {
  f32x4 s[NT][2];
};
// (T0, T1: the first row tile concerned, and the one behind the last.)
template <int T0, int T1, bool OVERLAP, int M, int NT>
__device__ __forceinline__ void block_scores(MxScores<NT> &y, const MxRows<M, NT> &st, const MxKeys<M> &x) {
#pragma unroll
  for (int p = 0; p < 2; ++p) {
    float scale[MxKeys<M>::kScales];
    if (!OVERLAP && p == 1) __builtin_amdgcn_sched_barrier(0);
#pragma unroll
    for (int i = 0; i < MxKeys<M>::kScales; ++i) scale[i] = mx_scale(x.scale[p][i]);
#pragma unroll
    for (int nt = T0; nt < T1; ++nt) y.s[nt][p] = f32x4{0.f, 0.f, 0.f, 0.f};
#pragma unroll
    for (int i = 0; i < M; ++i) {
      const bf16x8 kf = key_operand<M>(x.w[p][i], scale[kMxRun<M> ? (M == 8 ? i / 4 : 0) : i]);
#pragma unroll
      for (int nt = T0; nt < T1; ++nt) y.s[nt][p] = __builtin_amdgcn_mfma_f32_16x16x32_bf16(kf, st.q[nt][i], y.s[nt][p], 0, 0, 0);
    }
  }
}
// Those that a row does not see become -inf.  row0: the wavefront's first row in the row block.
template <int T0, int T1, bool TREE, int M, int NT>
__device__ __forceinline__ void mask_block(MxScores<NT> &y, const MxRows<M, NT> &st, const MxBlock &b, int row0) {
  if (!(b.vp_a & (kMasked | kRowMasked))) return;
  // Two tiles of a head of 64 have no registers for their mask words, and spill.  (One tile of a head of 128 reloads its word where a block has
  // masks, and spills queries if the word is remade.)
  constexpr bool kRemake = NT == 2 && mx_occupancy(32 * M, NT) > 2;
  const int lane = threadIdx.x & 63, jj = lane >> 4;
  int lo = b.rows & 0xffff, hi = static_cast<int>(static_cast<uint32_t>(b.rows) >> 16), vp_a = b.vp_a, vp_b = b.vp_b;
  asm volatile("" : "+s"(lo), "+s"(hi), "+s"(vp_a), "+s"(vp_b));  // nothing of this is computed ahead of the branch
#pragma unroll
  for (int nt = T0; nt < T1; ++nt) {
    const int row = row0 + 16 * nt + (lane & 15);
    const bool on_path = row >= lo && row < hi;
    uint32_t seen = 0xff;
    if (vp_a & kMasked)
      seen = seen_bits<TREE, kRemake>(st.limit[nt], st.qidx[nt], st.dmask[nt], vp_a, 4 * jj) |
             seen_bits<TREE, kRemake>(st.limit[nt], st.qidx[nt], st.dmask[nt], vp_b, 4 * jj) << 4;
    if (!on_path) seen = 0;
#pragma unroll
    for (int i = 0; i < 8; ++i) {
      const uint32_t keep = static_cast<uint32_t>(static_cast<int32_t>(seen << (31 - i)) >> 31);
      const float score = y.s[nt][i >> 2][i & 3];  // a select here compiles to three instructions a score
      y.s[nt][i >> 2][i & 3] = __builtin_bit_cast(float, (__builtin_bit_cast(uint32_t, score) & keep) | (0xff800000u & ~keep));
    }
  }
}

// x *= by and x -= by.  IN_PLACE: in assembly, because the compiler gives results in a branch registers of their own and copies them back, 36 of
// them for a head of 128.  (Not where blocks overlap: there it would copy for the assembly what it does not copy without.)
template <bool IN_PLACE>
__device__ __forceinline__ void scale_by(f32x4 &x, const f32x4 by) {
  if constexpr (IN_PLACE) {
#pragma unroll
    for (int i = 0; i < 4; ++i) {
      float e = x[i];
      asm("v_mul_f32 %0, %1, %0" : "+v"(e) : "v"(by[i]));
      x[i] = e;
    }
  } else {
    x *= by;
  }
}
template <bool IN_PLACE>
__device__ __forceinline__ void lower_by(f32x4 &x, float by) {
  if constexpr (IN_PLACE) {
#pragma unroll
    for (int i = 0; i < 4; ++i) {
      float e = x[i];
      asm("v_sub_f32 %0, %0, %1" : "+v"(e) : "v"(by));
      x[i] = e;
    }
  } else {
    x -= by;
  }
}

// Moves the references that a block's scores are far above; scores of far rows become differences to theirs.
template <int T0, int T1, bool OVERLAP, int M, int NT>
__device__ __forceinline__ void move_references(MxRows<M, NT> &st, MxScores<NT> &y, float c, float slack) {
  float top[NT];
  bool above = false;
#pragma unroll
  for (int nt = T0; nt < T1; ++nt) {
    const f32x4 a = y.s[nt][0], b = y.s[nt][1];
    top[nt] = fmaxf(fmaxf(fmaxf(a[0], a[1]), fmaxf(a[2], a[3])), fmaxf(fmaxf(b[0], b[1]), fmaxf(b[2], b[3])));
    above = above || top[nt] > st.m[nt] + slack;
  }
  if (__any(above)) {
#pragma unroll
    for (int nt = T0; nt < T1; ++nt) {
      const float m_new = row_group_max(fmaxf(top[nt], st.m[nt]));
      const float less = __builtin_fmaf(st.m[nt] - m_new, c, rounded_off(st, nt, c));
      st.m[nt] = m_new;
      st.mc[nt] = scaled_reference(m_new, c);
      st.far |= (__any(fabsf(st.mc[nt]) >= kFarLog2 && m_new != kMInit) ? 1 : 0) << nt;
      const float alpha = fast_exp2(less - rounded_off(st, nt, c));
      f32x4 of_rows;  // the lane's accumulators are of four rows
#pragma unroll
      for (int i = 0; i < 4; ++i) of_rows[i] = __shfl(alpha, 4 * (static_cast<int>(threadIdx.x & 63) >> 4) + i);
      scale_by<!OVERLAP>(st.l[nt], of_rows);
#pragma unroll
      for (int i = 0; i < 2 * M; ++i) scale_by<!OVERLAP>(st.o[nt][i], of_rows);
    }
  }
  if (st.far) {
#pragma unroll
    for (int nt = T0; nt < T1; ++nt) {
      const bool far = (st.far >> nt & 1) != 0;
      const float by = far ? st.m[nt] : 0.f;
      lower_by<!OVERLAP>(y.s[nt][0], by);
      lower_by<!OVERLAP>(y.s[nt][1], by);
      if (OVERLAP) st.mc[nt] = far ? -kWeightLog2 : st.mc[nt];
    }
  }
}

// Weights of a block's scores and their product with its values.
template <int T0, int T1, bool OVERLAP, int M, int NT>
__device__ __forceinline__ void block_values(MxRows<M, NT> &st, const MxScores<NT> &y, const MxValues<M> &x, float c) {
  f16x8 ph[NT], pl[NT];
#pragma unroll
  for (int nt = T0; nt < T1; ++nt) {
    float w[8];
    const float mc = !OVERLAP && (st.far >> nt & 1) != 0 ? -kWeightLog2 : st.mc[nt];
#pragma unroll
    for (int i = 0; i < 8; ++i) w[i] = fast_exp2(__builtin_fmaf(y.s[nt][i >> 2][i & 3], c, -mc));
    u32x4 h, rest;
#pragma unroll
    for (int i = 0; i < 4; ++i) {
      h[i] = __builtin_bit_cast(uint32_t, f16x2{static_cast<_Float16>(w[2 * i]), static_cast<_Float16>(w[2 * i + 1])});
      rest[i] = rest_of(h[i], w[2 * i], w[2 * i + 1]);
    }
    ph[nt] = __builtin_bit_cast(f16x8, h);
    pl[nt] = __builtin_bit_cast(f16x8, rest);
    const _Float16 one = static_cast<_Float16>(1.f);
    const f16x8 ones = {one, one, one, one, one, one, one, one};
    st.l[nt] = __builtin_amdgcn_mfma_f32_16x16x32_f16(ph[nt], ones, st.l[nt], 0, 0, 0);
    st.l[nt] = __builtin_amdgcn_mfma_f32_16x16x32_f16(pl[nt], ones, st.l[nt], 0, 0, 0);
  }
  if (!OVERLAP) __builtin_amdgcn_sched_barrier(0);  // the values' conversions ahead of the weights would take the registers of a wavefront
  float vs[2][4];
#pragma unroll
  for (int j = 0; j < M; ++j) {
    if (j == 0 || !kMxRun<M>) {
#pragma unroll
      for (int h = 0; h < 2; ++h)
#pragma unroll
        for (int t = 0; t < 4; ++t) vs[h][t] = mx_scale(x.scale[h][kMxRun<M> ? 0 : j], t);
    }
    // A byte of a word is the dims d, d + 1 of one token, which one conversion puts side by side, where a product over tokens wants
    // two tokens of one dim.  So the product is one over (token, dim) pairs of which every second weight is zero: the sparse one,
    // which takes two of four at a dense product's rate; kEvenDims and kOddDims choose d and d + 1.  It wants a lane's values in the
    // order in which load_values has taken them.
    if (!OVERLAP && j > 0 && j % 2 == 0) __builtin_amdgcn_sched_barrier(0);
    u32x8 r;
#pragma unroll
    for (int h = 0; h < 2; ++h) {
      r[4 * h] = __builtin_bit_cast(uint32_t, __builtin_amdgcn_cvt_scalef32_pk_f16_fp4(x.w[h * M + j], vs[h][0], 0));
      r[4 * h + 1] = __builtin_bit_cast(uint32_t, __builtin_amdgcn_cvt_scalef32_pk_f16_fp4(x.w[h * M + j], vs[h][1], 1));
      r[4 * h + 2] = __builtin_bit_cast(uint32_t, __builtin_amdgcn_cvt_scalef32_pk_f16_fp4(x.w[h * M + j], vs[h][2], 2));
      r[4 * h + 3] = __builtin_bit_cast(uint32_t, __builtin_amdgcn_cvt_scalef32_pk_f16_fp4(x.w[h * M + j], vs[h][3], 3));
    }
    const f16x16 vf = __builtin_bit_cast(f16x16, r);
#pragma unroll
    for (int nt = T0; nt < T1; ++nt) {
      st.o[nt][2 * j] = __builtin_amdgcn_smfmac_f32_16x16x64_f16(ph[nt], vf, st.o[nt][2 * j], kEvenDims, 0, 0);
      st.o[nt][2 * j + 1] = __builtin_amdgcn_smfmac_f32_16x16x64_f16(ph[nt], vf, st.o[nt][2 * j + 1], kOddDims, 0, 0);
    }
#pragma unroll
    for (int nt = T0; nt < T1; ++nt) {
      st.o[nt][2 * j] = __builtin_amdgcn_smfmac_f32_16x16x64_f16(pl[nt], vf, st.o[nt][2 * j], kEvenDims, 0, 0);
      st.o[nt][2 * j + 1] = __builtin_amdgcn_smfmac_f32_16x16x64_f16(pl[nt], vf, st.o[nt][2 * j + 1], kOddDims, 0, 0);
    }
  }
}

// Where a finished or partial row goes.
struct RowPlace {
  int64_t at;  // row of the destination, or -1: none
  float inv;
};
// LDS of a set of wavefronts that hold the same rows: softmax states, factors and places, and of several wavefronts a stage of 16 rows each.
template <int M, int NT>
struct MxJoin {
  static constexpr int kRow = 32 * M + 4;  // the pad spreads rows over the banks
  static constexpr int kStage = 16 * kRow;
  static constexpr int floats(int waves) { return waves * ((waves > 1 ? kStage : 0) + 3 * 16 * NT + 16) + 4 * 16; }
};

// Joins the states of the KS wavefronts (number ks of them calls) that hold the same rows, and writes the rows.  Several: called by all
// of a workgroup together.  place(nt, row of the tile): the destination row or -1.  ml (of several): the rows are partial states, weights
// 2^(c (s - m)) with m a score, because of two far references only the difference may be scaled; else they are finished.
template <int M, int NT, int KS, class Place>
__device__ __forceinline__ void join_rows(MxRows<M, NT> &st, int ks, float c, float *area, float *dst, float *ml, float *lse, Place place) {
  constexpr int kRow = MxJoin<M, NT>::kRow, kStage = KS > 1 ? MxJoin<M, NT>::kStage : 0, D = 32 * M;
  constexpr int kRun = kMxRun<M> ? 2 * M : 2;  // dims of a lane that follow each other
  const int lane = threadIdx.x & 63, row = lane & 15, jj = lane >> 4;
  RowPlace *places = reinterpret_cast<RowPlace *>(area);
  float *states = area + 4 * 16;  // [wavefront][m of all rows, l of all rows, what was rounded off m c]
  float *factors = states + KS * 3 * 16 * NT + 16 * ks;
  float *stage = states + KS * (3 * 16 * NT + 16);
  auto meet = [&]() {
    if (KS > 1) {
      __syncthreads();
    } else {
      __builtin_amdgcn_fence(__ATOMIC_ACQ_REL, "wavefront");
      __builtin_amdgcn_wave_barrier();
    }
  };
#pragma unroll
  for (int nt = 0; nt < NT; ++nt) {
    float *mine = states + ks * 3 * 16 * NT + 16 * nt;
    if (jj == 0) {
      mine[row] = st.m[nt];
      mine[2 * 16 * NT + row] = rounded_off(st, nt, c);
    }
    if (row == 0) *reinterpret_cast<f32x4 *>(mine + 16 * NT + 4 * jj) = st.l[nt];
  }
  meet();
#pragma unroll
  for (int nt = 0; nt < NT; ++nt) {
    const float *of = states + 16 * nt + row;
    float m = st.m[nt], l = of[16 * NT], factor = 1.f;
    if (KS > 1) {
#pragma unroll
      for (int k = 0; k < KS; ++k) m = fmaxf(m, of[3 * k * 16 * NT]);
      auto weight = [&](int k) { return fast_exp2(__builtin_fmaf(of[3 * k * 16 * NT] - m, c, of[(3 * k + 2) * 16 * NT])); };
      l = 0.f;
#pragma unroll
      for (int k = 0; k < KS; ++k) l += of[(3 * k + 1) * 16 * NT] * weight(k);
      factor = weight(ks);
      if (ml) {
        l *= kWeightUnit;
        factor *= kWeightUnit;
      }
    }
    if (jj == 0) {
      const float inv = KS > 1 && ml ? 1.f : 1.f / l;
      if (ks == 0) {
        const int64_t at = place(nt, row);
        places[row] = {at, inv};
        if (at >= 0) {
          if (KS > 1 && ml)
            *reinterpret_cast<f32x2 *>(ml + 2 * at) = f32x2{m, l};
          else if (lse)
            lse[at] = (__builtin_fmaf(m, c, -kWeightLog2) + (__builtin_log2f(l) + (KS > 1 ? 0.f : of[2 * 16 * NT]))) * 0.6931471805599453f;
        }
      }
      factors[row] = factor;
    }
    __builtin_amdgcn_fence(__ATOMIC_ACQ_REL, "wavefront");
    __builtin_amdgcn_wave_barrier();
    const f32x4 f = *reinterpret_cast<const f32x4 *>(factors + 4 * jj);
#pragma unroll
    for (int i = 0; i < 4; ++i) {
      const RowPlace to = places[4 * jj + i];
      const float by = KS > 1 ? f[i] : to.inv;
      if (KS == 1 && to.at < 0) continue;
      float *out = KS > 1 ? stage + ks * kStage + (4 * jj + i) * kRow : dst + to.at * D;
#pragma unroll
      for (int j = 0; j < M; j += kRun / 2) {
        float *p = out + mx_value_dim<M>(row, j);
        if constexpr (kRun >= 4) {
#pragma unroll
          for (int k = 0; k < kRun; k += 4) {
            const f32x4 *o = st.o[nt] + 2 * j + k;
            *reinterpret_cast<f32x4_out *>(p + k) = f32x4{o[0][i], o[1][i], o[2][i], o[3][i]} * by;
          }
        } else {
          *reinterpret_cast<f32x2_out *>(p) = f32x2{st.o[nt][2 * j][i], st.o[nt][2 * j + 1][i]} * by;
        }
      }
    }
    meet();
    if (KS > 1) {
      for (int i = ks * 64 + lane; i < 16 * (D / 4); i += 64 * KS) {
        const int r = i / (D / 4), d = i % (D / 4) * 4;
        const RowPlace to = places[r];
        f32x4 v = *reinterpret_cast<const f32x4 *>(stage + r * kRow + d);
#pragma unroll
        for (int k = 1; k < KS; ++k) v += *reinterpret_cast<const f32x4 *>(stage + k * kStage + r * kRow + d);
        if (to.at >= 0) *reinterpret_cast<f32x4_out *>(dst + to.at * D + d) = v * to.inv;
      }
      if (nt + 1 < NT) meet();
    }
  }
}

constexpr int kWaves = 4;  // of a workgroup
// Private blocks of a set from which on those of one row tile have rounds of their own: 64 trees of 32 branches of eight blocks took
// 171 us without and 160 with; two or three blocks a branch 140 and 152.
constexpr int kAlone = 16;

// The blocks of one of the wavefronts that hold the same rows: every stride-th record of a list, 64 of them at a time in registers, a lane
// each.  Read::fetch(i): record i as it lies in memory, for a lane; Read::make(raw, i, r): what it says, false where it does not concern the
// wavefront's rows.
struct MxLanes {
  int page[2], vp_a, vp_b, rows;
};
template <int M>
__device__ __forceinline__ int64_t tile_at(int page, int page_tiles, int g) {
  return (static_cast<int64_t>(page) * page_tiles + g) * mx_tile_bytes(M);
}
// Rows from row_end on are not there and need no mask (eight of sixteen rows on 48 paths of 16000 tokens: 30 us with one, 26 without).
// Records from number `alone` on whose rows lie in one tile are left out of those for all tiles, and are the only ones of a single tile.
template <int T0, int T1, int M, int NT, class Read>
struct MxSource {
  Read read;
  int n, at, stride, alone, row0, row_end, g, page_tiles;
  bool &left_out;
  uint64_t left;
  MxLanes r;
  __device__ __forceinline__ typename Read::Raw fetch() const {
    const int i = at + stride * static_cast<int>(threadIdx.x & 63);
    return i < n ? read.fetch(i) : typename Read::Raw{};
  }
  __device__ __forceinline__ void take(const typename Read::Raw &raw) {
    const int i = at + stride * static_cast<int>(threadIdx.x & 63);
    bool concerns = i < n;
    if (concerns) concerns = read.make(raw, i, r);
    const int lo = r.rows & 0xffff, hi = static_cast<int>(static_cast<uint32_t>(r.rows) >> 16);
    if (NT > 1 && T1 - T0 == NT) {
      const bool one = i >= alone && (lo >= row0 + 16 || hi <= row0 + 16);
      left_out = left_out || __any(concerns && one);
      concerns = concerns && !one;
    } else if (NT > 1) {
      concerns = concerns && (T0 == 0 ? hi <= row0 + 16 : lo >= row0 + 16);
    }
    if (lo > row0 + 16 * T0 || hi < min(row0 + 16 * T1, row_end)) r.vp_a |= kRowMasked;
    left = __ballot(concerns);
    at += 64 * stride;
  }
  __device__ __forceinline__ MxBlock next() {
    while (left == 0 && at < n) take(fetch());
    MxBlock b;
    b.live = left != 0;
    const int l = b.live ? __builtin_ctzll(left) : 0;
    const int none = b.live ? 0 : kRowMasked;  // a block that is not there is one of no rows
    left &= left - 1;
#pragma unroll
    for (int p = 0; p < 2; ++p) b.at[p] = tile_at<M>(__builtin_amdgcn_readlane(r.page[p], l), page_tiles, g);
    b.vp_a = __builtin_amdgcn_readlane(r.vp_a, l) | none;
    b.vp_b = __builtin_amdgcn_readlane(r.vp_b, l);
    b.rows = b.live ? __builtin_amdgcn_readlane(r.rows, l) : 0;
    return b;
  }
};

// Blocks first, first + stride, .. of n, for the row tiles T0 .. T1.  OVERLAP: a block's scores are computed beside the weights and values
// of the block before, so that matrix and vector instructions of one wavefront run at the same time; keys are requested two blocks ahead,
// values one.  Otherwise a block at a time, the next one's keys and values requested where this one's have been used.
template <int T0, int T1, bool TREE, bool OVERLAP, int M, int NT, class Read>
__device__ __forceinline__ void walk_tiles(MxRows<M, NT> &st, const void *k, const void *v, int row0, int row_end, float c, int n, int first,
                                           int stride, int alone, int g, int page_tiles, bool &left_out, const Read &read,
                                           const typename Read::Raw *raw) {
  const float slack = kSlackLog2 / c;
  MxSource<T0, T1, M, NT, Read> src{read, n, first, stride, alone, row0, row_end, g, page_tiles, left_out, 0, {}};
  MxKeys<M> k0;
  MxValues<M> v0;
  MxScores<NT> y0;
  if (raw) src.take(*raw);
  MxBlock b0 = src.next();
  if (!b0.live) return;
  load_keys<M>(k0, b0, k);
  load_values<M>(v0, b0, v);
  if constexpr (OVERLAP) {
    MxKeys<M> k1;
    MxValues<M> v1;
    MxScores<NT> y1;
    MxBlock b1 = src.next();
    load_keys<M>(k1, b1, k);
    block_scores<T0, T1, OVERLAP>(y0, st, k0);
    mask_block<T0, T1, TREE>(y0, st, b0, row0);
    // y, x: of block b; the block behind it has its keys in nk and its place in nb, the one behind that is requested into b and k
    auto step = [&](MxScores<NT> &y, MxValues<M> &x, MxKeys<M> &key, MxBlock &b, MxScores<NT> &ny, MxValues<M> &nx, MxKeys<M> &nk, MxBlock &nb) {
      b = src.next();
      load_keys<M>(key, b, k);
      load_values<M>(nx, nb, v);
      move_references<T0, T1, OVERLAP>(st, y, c, slack);
      block_scores<T0, T1, OVERLAP>(ny, st, nk);
      block_values<T0, T1, OVERLAP>(st, y, x, c);
      mask_block<T0, T1, TREE>(ny, st, nb, row0);
    };
    do {  // two at a time: a block that is not there is one of no rows
      step(y0, v0, k0, b0, y1, v1, k1, b1);
      step(y1, v1, k1, b1, y0, v0, k0, b0);
    } while (b0.live);
  } else {
    auto step = [&](MxKeys<M> &key, MxValues<M> &x, MxBlock &at) {
      const MxBlock b = at;
      at = src.next();
      block_scores<T0, T1, OVERLAP>(y0, st, key);
      load_keys<M>(key, at, k);
      mask_block<T0, T1, TREE>(y0, st, b, row0);
      move_references<T0, T1, OVERLAP>(st, y0, c, slack);
      block_values<T0, T1, OVERLAP>(st, y0, x, c);
      load_values<M>(x, at, v);
    };
    do step(k0, v0, b0);
    while (b0.live);
  }
}
// Of two tiles, blocks that concern one of them only have rounds of their own from record `alone` on: half the products and weights.
// raw: the first 64 records, fetched before the rows were loaded.
template <bool TREE, bool OVERLAP, int M, int NT, class Read>
__device__ __forceinline__ void walk_blocks(MxRows<M, NT> &st, const void *k, const void *v, int row0, int row_end, float c, int n, int first,
                                            int stride, int alone, int g, int page_tiles, const Read &read,
                                            const typename Read::Raw &raw) {
  bool left_out = false;
  walk_tiles<0, NT, TREE, OVERLAP>(st, k, v, row0, row_end, c, n, first, stride, alone, g, page_tiles, left_out, read, &raw);
  if constexpr (NT == 2) {
    if (!left_out) return;
    const int from = first >= alone ? first : first + (alone - first + stride - 1) / stride * stride;
    walk_tiles<0, 1, TREE, OVERLAP>(st, k, v, row0, row_end, c, n, from, stride, alone, g, page_tiles, left_out, read, nullptr);
    walk_tiles<1, 2, TREE, OVERLAP>(st, k, v, row0, row_end, c, n, from, stride, alone, g, page_tiles, left_out, read, nullptr);
  }
}

// With one row tile the registers go to more wavefronts instead, four a SIMD: 157 us for the 64 trees above, 177 with two that overlap, 165
// with three that do not.  A second block of keys and values under way took three back and was no faster.
constexpr bool mx_overlap(int blocks, int row_tiles) { return row_tiles == 2; }

// Blocks of a split item: pairs of its pages' records {page, position << 7 | valid tokens}.
struct SplitRecords {
  struct Raw {
    int2 a, b;
  };
  const int2 *pages;
  int count;
  bool masked;
  int seen_end;
  __device__ __forceinline__ Raw fetch(int i) const { return {pages[2 * i], pages[min(2 * i + 1, count - 1)]}; }
  __device__ __forceinline__ bool make(const Raw &x, int i, MxLanes &r) const {
    const bool has_b = 2 * i + 1 < count;
    r = {{x.a.x, x.b.x}, x.a.y | (masked || !has_b ? kMasked : 0), has_b ? x.b.y : 0, static_cast<int>(0xffff0000u)};
    return (x.a.y >> 7) < seen_end;
  }
};

// For lists that the walk does not hold and where the caller asks for it: every item's rows cost a partial state of each, so that 64 trees as above
// take 414 us.  48 paths of 16000 tokens with one query each and heads of 64 take 24 here and 27 through the walk, whose lists are longer.
template <int M, int NT, bool TREE>
__global__ __launch_bounds__(64 * kWaves, mx_occupancy(32 * M, NT)) void spex_mxfp4_split_kernel(AttnArgs p, Shape sh, SplitLists ls) {
  __shared__ __attribute__((aligned(16))) float lds[MxJoin<M, NT>::floats(kWaves)];
  const ListPos at = list_of(ls, static_cast<int>(blockIdx.x));
  const int tile = at.local / at.n_items;
  Item cur = load_item(at.items, at.local - tile * at.n_items);
  cur.row0 += tile * 16 * NT;
  const int G = sh.G, rows = cur.qt_count * G;
  if (cur.pg_count == 0 || cur.row0 >= rows) return;  // whole workgroup: padding item, or no such tile
  const int w = uniform(threadIdx.x >> 6), g = cur.g;
  const float c = p.scale_log2;
  const int n_blocks = (cur.pg_count + 1) >> 1, first = w + kWaves * static_cast<int>(threadIdx.x & 63);
  SplitRecords records{reinterpret_cast<const int2 *>(p.pg_rec) + cur.pg_begin, cur.pg_count, (cur.flags & 1) != 0, 0};
  const auto raw = first < n_blocks ? records.fetch(first) : SplitRecords::Raw{};
  MxRows<M, NT> st;
  load_rows<M, NT, TREE>(st, p.q, p.qt_rec, p.qt_mask, cur.qt_begin, cur.row0, rows, g, sh, c);
  records.seen_end = st.seen_end;
  walk_blocks<TREE, mx_overlap(M, NT)>(st, p.k_pool, p.v_pool, 0, INT_MAX, c, n_blocks, w, kWaves, INT_MAX, g, sh.page_tiles, records, raw);
  join_rows<M, NT, kWaves>(st, w, c, lds, p.finish ? p.out : p.part_o, p.finish ? nullptr : p.part_ml, p.lse, [&](int nt, int row) {
    const int r = cur.row0 + 16 * nt + row;
    if (r >= rows) return static_cast<int64_t>(-1);
    return p.finish ? static_cast<int64_t>(st.qtok[nt]) * sh.Hq + g * G + r % G
                    : static_cast<int64_t>(cur.pbase) + static_cast<int64_t>(g) * rows + r;
  });
}

// A set of up to 16 NT rows of a work item of the tree-walk lists: those of tile set `part >> 8` of its wavefront of rows `part & 0xff`.
struct MxSet {
  int g, rows, row_base;      // rows of the wavefront, the set's first one among them
  int row0;                   // the same in the row block
  int qt_begin;
  int blk_begin, n_shared, priv_begin, n_priv;
};
template <int NT>
__device__ __forceinline__ MxSet load_set(const int32_t *items, int item, int part, int nw, int ntw, int G) {
  const int64_t ir = static_cast<int64_t>(item) * (nw <= 4 ? 16 : 32);
  const int w = part & 0xff;
  // The whole record in one load, a lane an int.
  const int x = items[ir + min(static_cast<int>(threadIdx.x & 63), nw <= 4 ? 15 : 31)];
  auto field = [&](int i) { return __builtin_amdgcn_readlane(x, i); };
  MxSet t;
  t.g = field(0);
  t.blk_begin = field(1);
  t.n_shared = field(2);
  t.n_priv = field(3 + w) & 0xffff;  // blocks | room << 16
  t.priv_begin = t.blk_begin + t.n_shared;
  for (int v = 0; v < w; ++v) t.priv_begin += static_cast<int>(static_cast<uint32_t>(field(3 + v)) >> 16);
  t.qt_begin = field(3 + nw + w);
  t.rows = field(3 + 2 * nw + w) * G;
  t.row_base = (part >> 8) * 16 * NT;
  t.row0 = w * 16 * ntw + t.row_base;
  return t;
}

// Blocks of a set: records {page a, position << 7 | valid tokens, page b, valid tokens or 0, rows, flags}, first the shared ones.
struct WalkRecords {
  struct Raw {
    u32x4 a, b;
  };
  const u32x4 *blocks;
  int shared_begin, n_shared, priv_less_shared, row0, row1, seen_end;
  __device__ __forceinline__ Raw fetch(int i) const {
    const u32x4 *rec = blocks + 2 * static_cast<int64_t>((i < n_shared ? shared_begin : priv_less_shared) + i);
    return {rec[0], rec[1]};
  }
  __device__ __forceinline__ bool make(const Raw &x, int, MxLanes &r) const {
    const int lo = static_cast<int>(x.b[0] & 0xffffu), hi = static_cast<int>(x.b[0] >> 16);
    r.page[0] = static_cast<int>(x.a[0]);
    r.page[1] = static_cast<int>(x.a[3] != 0 ? x.a[2] : x.a[0]);
    r.vp_a = static_cast<int>(x.a[1]) | ((x.b[1] & 1) != 0 ? kMasked : 0);
    r.vp_b = static_cast<int>(x.a[3]);
    r.rows = static_cast<int>(x.b[0]);
    return lo < row1 && hi > row0 && (r.vp_a >> 7) < seen_end;
  }
};

// A workgroup of four pieces, a wavefront each, or of one whose blocks the four wavefronts take in turn (Planner::build_pieces).
// Measured, heads 32 / 8 / 128: 64 trees of 2500 tokens with 32 branches of 256 (474 MB) 150 us, 3.2 TB/s, 115 without the arithmetic; 32 trees
// of 16 branches (137 MB) 27 us, 5.1 TB/s; 16 trees of 4 branches with 100 queries each 187 us, 600 TFLOP/s of the products that the
// definition has, 980 with those of the second pieces; one document of 64000 tokens and 8 branches (71 MB) 24 us and 5 to merge.
template <int M, int NT, bool TREE>
__global__ __launch_bounds__(64 * kWaves, mx_occupancy(32 * M, NT)) void spex_mxfp4_walk_kernel(WalkArgs p, Shape sh, int nw, int ntw) {
  constexpr int kOne = MxJoin<M, NT>::floats(1), kAll = MxJoin<M, NT>::floats(kWaves);
  __shared__ __attribute__((aligned(16))) float lds[kWaves * kOne > kAll ? kWaves * kOne : kAll];
  const int w = uniform(threadIdx.x >> 6);
  const int64_t pr = (static_cast<int64_t>(blockIdx.x) * kWaves + w) * 8;
  const int item = sload(p.pieces, pr), begin = sload(p.pieces, pr + 2), end = sload(p.pieces, pr + 3), slot = sload(p.pieces, pr + 4);
  const bool together = sload(p.pieces, pr + 5) != 0;  // all of the workgroup or none
  if (item < 0) return;  // padding
  const MxSet t = load_set<NT>(p.items, item, sload(p.pieces, pr + 1), nw, ntw, sh.G);
  const int G = sh.G;
  const float c = p.scale_log2;
  const int stride = together ? kWaves : 1, first = begin + (together ? w : 0), n = min(end, t.n_shared + t.n_priv);
  WalkRecords records{reinterpret_cast<const u32x4 *>(p.blocks), t.blk_begin, t.n_shared, t.priv_begin - t.n_shared, t.row0, t.row0 + 16 * NT, 0};
  const int mine = first + stride * static_cast<int>(threadIdx.x & 63);
  const auto raw = mine < n ? records.fetch(mine) : WalkRecords::Raw{};
  MxRows<M, NT> st;
  load_rows<M, NT, TREE>(st, p.q, p.qt_rec, p.qt_mask, t.qt_begin, t.row_base, t.rows, t.g, sh, c);
  records.seen_end = st.seen_end;
  walk_blocks<TREE, mx_overlap(M, NT)>(st, p.k_pool, p.v_pool, t.row0, t.row0 + t.rows - t.row_base, c, n, first, stride,
                                       t.n_priv >= kAlone * stride ? t.n_shared : INT_MAX, t.g, sh.page_tiles, records, raw);
  const bool whole = slot < 0;
  float *dst = whole ? p.out : p.part_o, *ml = whole ? nullptr : p.part_ml;
  auto place = [&](int nt, int row) {
    const int r = t.row_base + 16 * nt + row;
    if (r >= t.rows) return static_cast<int64_t>(-1);
    return whole ? static_cast<int64_t>(st.qtok[nt]) * sh.Hq + t.g * G + r % G : static_cast<int64_t>(slot) + 16 * nt + row;
  };
  if (together)
    join_rows<M, NT, kWaves>(st, w, c, lds, dst, ml, p.lse, place);
  else
    join_rows<M, NT, 1>(st, 0, c, lds + w * kOne, p.out, nullptr, p.lse, place);  // pieces are walked together
}

// Rows whose path was walked in pieces (256 rows of 63 pieces, 8 MB: 4.4 to 5.2 us, of it 1.6 an empty launch): a workgroup a row; threads
// of four dims each, in as many groups as fit, which take the pieces in turn and are summed through LDS.  Up to 64 pieces: a lane holds the weight of one.
template <int M, int NT>
__global__ __launch_bounds__(256) void spex_mxfp4_merge_kernel(WalkArgs p, Shape sh, int nw, int ntw) {
  constexpr int D = 32 * M, kLanes = D / 4, kGroups = 256 / kLanes, kEach = (64 + kGroups - 1) / kGroups, kBatch = kEach < 8 ? kEach : 8;
  __shared__ __attribute__((aligned(16))) float lds[kGroups * D];
  const int tid = threadIdx.x, lane = tid & 63;
  const int merge = static_cast<int>(blockIdx.x) / (16 * NT), row = static_cast<int>(blockIdx.x) - merge * 16 * NT;
  const int item = sload(p.merges, 4 * static_cast<int64_t>(merge)), part = sload(p.merges, 4 * static_cast<int64_t>(merge) + 1);
  const int64_t slot = sload(p.merges, 4 * static_cast<int64_t>(merge) + 2);
  const int n = sload(p.merges, 4 * static_cast<int64_t>(merge) + 3);
  f32x2 ml = {kNegInf, 0.f};
  if (lane < n) ml = *reinterpret_cast<const f32x2 *>(p.part_ml + 2 * (slot + static_cast<int64_t>(lane) * 16 * NT + row));
  const int group = tid / kLanes, d = (tid - group * kLanes) * 4;
  const float *src = p.part_o + (slot + row) * D + d;
  constexpr int64_t kStep = static_cast<int64_t>(16 * NT) * D;
  f32x4 x[kBatch];
#pragma unroll
  for (int k = 0; k < kBatch; ++k) {
    const int at = group + k * kGroups;
    x[k] = *reinterpret_cast<const f32x4 *>(src + (group < kGroups && at < n ? at : 0) * kStep);
  }
  const MxSet t = load_set<NT>(p.items, item, part, nw, ntw, sh.G);  // behind the loads, which do not wait for it
  const int r = t.row_base + row;
  if (r >= t.rows) return;  // the whole workgroup; what it loaded is room of its set's states
  float m = ml[0];
#pragma unroll
  for (int o = 32; o >= 1; o >>= 1) m = fmaxf(m, __shfl_xor(m, o));
  const float weight = fast_exp2((ml[0] - m) * p.scale_log2);
  float l = weight * ml[1];
#pragma unroll
  for (int o = 32; o >= 1; o >>= 1) l += __shfl_xor(l, o);
  f32x4 o = {0.f, 0.f, 0.f, 0.f};
  for (int i = group; i - group < n; i += kBatch * kGroups) {  // every lane goes round as often: the weights are exchanged
#pragma unroll
    for (int k = 0; k < kBatch; ++k) {
      const int at = i + k * kGroups;
      const float f = __shfl(weight, min(at, 63));
      o += x[k] * (at < n ? f : 0.f);
    }
#pragma unroll
    for (int k = 0; k < kBatch; ++k) {
      const int at = i + (kBatch + k) * kGroups;
      if (at < n && group < kGroups) x[k] = *reinterpret_cast<const f32x4 *>(src + at * kStep);
    }
  }
  if (group < kGroups) *reinterpret_cast<f32x4 *>(lds + group * D + d) = o;
  __syncthreads();
  if (tid >= kLanes) return;
#pragma unroll
  for (int k = 1; k < kGroups; ++k) o += *reinterpret_cast<const f32x4 *>(lds + k * D + d);
  const int qtok = sload(p.qt_rec, 2 * (static_cast<int64_t>(t.qt_begin) + r / sh.G));
  const int64_t at = static_cast<int64_t>(qtok) * sh.Hq + t.g * sh.G + r % sh.G;
  *reinterpret_cast<f32x4_out *>(p.out + at * D + d) = o * (1.f / l);
  if (tid == 0 && p.lse) p.lse[at] = __builtin_fmaf(m, p.scale_log2, __builtin_log2f(l)) * 0.6931471805599453f;
}

// f(integral constant M)
template <class F>
hipError_t with_blocks(int head_dim, F f) {
  switch (head_dim) {
    case 32: return f(std::integral_constant<int, 1>());
    case 64: return f(std::integral_constant<int, 2>());
    case 96: return f(std::integral_constant<int, 3>());
    case 128: return f(std::integral_constant<int, 4>());
    case 160: return f(std::integral_constant<int, 5>());
    case 192: return f(std::integral_constant<int, 6>());
    case 224: return f(std::integral_constant<int, 7>());
    case 256: return f(std::integral_constant<int, 8>());
  }
  return hipErrorInvalidValue;
}

template <int M, int NT>
hipError_t launch_split(const Shape &sh, const AttnArgs &a, const ItemLists &l, hipStream_t stream) {
  int64_t n_wg = 0;
  const SplitLists ls = make_lists(l, 16 * NT, &n_wg);
  if (n_wg < 0) return hipErrorInvalidValue;
  if (n_wg == 0) return hipSuccess;
  const dim3 grid(static_cast<unsigned>(n_wg)), block(64 * kWaves);
  if (a.qt_mask)
    hipLaunchKernelGGL((spex_mxfp4_split_kernel<M, NT, true>), grid, block, 0, stream, a, sh, ls);
  else
    hipLaunchKernelGGL((spex_mxfp4_split_kernel<M, NT, false>), grid, block, 0, stream, a, sh, ls);
  return hipGetLastError();
}

template <int M, int NT>
hipError_t launch_walk(const Shape &sh, const WalkArgs &a, int ntw, int waves, hipStream_t stream) {
  const dim3 grid(static_cast<unsigned>(a.n_pieces / kWaves)), block(64 * kWaves);
  if (a.qt_mask)
    hipLaunchKernelGGL((spex_mxfp4_walk_kernel<M, NT, true>), grid, block, 0, stream, a, sh, waves, ntw);
  else
    hipLaunchKernelGGL((spex_mxfp4_walk_kernel<M, NT, false>), grid, block, 0, stream, a, sh, waves, ntw);
  const hipError_t e = hipGetLastError();
  if (e != hipSuccess || a.n_merges == 0) return e;
  hipLaunchKernelGGL((spex_mxfp4_merge_kernel<M, NT>), dim3(static_cast<unsigned>(a.n_merges) * 16 * NT), dim3(256), 0, stream, a, sh, waves, ntw);
  return hipGetLastError();
}

}  // namespace

hipError_t launch_mxfp4_split(const Shape &sh, const AttnArgs &a, const ItemLists &l, hipStream_t stream) {
  return with_blocks(sh.D, [&](auto m) {
    constexpr int M = decltype(m)::value;
    return std::max({l.span[0], l.span[1], l.span[2], l.span[3]}) <= 16 ? launch_split<M, 1>(sh, a, l, stream)
                                                                       : launch_split<M, mx_row_tiles(32 * M, 2)>(sh, a, l, stream);
  });
}

hipError_t launch_mxfp4_walk(const Shape &sh, const WalkArgs &a, int ntw, int waves, hipStream_t stream) {
  if (a.n_pieces <= 0) return hipSuccess;
  if ((ntw != 1 && ntw != 2 && ntw != 4) || (waves != 2 && waves != 4 && waves != 8)) return hipErrorInvalidValue;
  return with_blocks(sh.D, [&](auto m) {
    constexpr int M = decltype(m)::value;
    return ntw == 1 ? launch_walk<M, 1>(sh, a, ntw, waves, stream) : launch_walk<M, mx_row_tiles(32 * M, 2)>(sh, a, ntw, waves, stream);
  });
}

}  // namespace spex
