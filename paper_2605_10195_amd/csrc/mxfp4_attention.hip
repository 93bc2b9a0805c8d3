// HIP kernels of decode attention over microscaled 4-bit (MXFP4) pools on gfx950 (CDNA4, 64-lane wavefronts).
//
//   spex_mxfp4_split_kernel
//       The split path's items, a workgroup for up to 16 NT rows of one: its four wavefronts take every fourth block of 32 tokens
//       and join their softmax states through LDS.  Partial states go to the merge kernel, as for the other pools.
//   spex_mxfp4_walk_kernel
//       The tree walk: the same over the whole path of up to 16 NT rows, from the root to the requested nodes.  Nothing but finished
//       rows is written.
//
// Mathematics: S^T = K Q^T, p = 2^(c S^T - m), l += sum p, O^T += V^T P^T, out = O / l, with keys and values code * 2^E.
// Keys become bf16 operands, which hold code * 2^E exactly (two significant bits), values fp16, which do as well since the values' E is
// bounded; v_cvt_scalef32_pk_* makes two of them from a byte and the scale.  Queries are the caller's bf16.  Weights go into the product
// as two fp16 pieces, 22 bits, so that nothing is rounded to fewer bits than fp32 sums lose.
//
// No LDS in the loop: a tile is held in the order in which its lanes consume it (mxfp4_device.hpp), so a block's codes go from memory
// into the registers they are converted in, and sharing converted tiles between wavefronts would cost as many LDS reads
// as the conversions take vector instructions.
#include <algorithm>
#include <type_traits>

#include "attention_device.hpp"
#include "kernels.hpp"
#include "mxfp4_device.hpp"

namespace spex {
namespace {

typedef uint32_t u32x3 __attribute__((ext_vector_type(3)));
typedef u32x4 u32x4_q __attribute__((aligned(2)));   // queries: any alignment of their type
typedef f32x4 f32x4_out __attribute__((aligned(4)));

// Start of a row's softmax reference: finite, so that (-inf) - m stays -inf, and below any score.
constexpr float kMInit = -1.0e30f;
// How far a score may exceed the reference before that moves, and the exponent of a weight at the reference: weights stay below 2^15,
// fp16's largest, and the smallest fp16 step is 2^-31 of a row's largest weight at most.
constexpr float kSlackLog2 = 8.f, kWeightLog2 = 7.f;
// Scaled references from here on are not subtracted in scaled form: their rounding would shift weights by many units.
constexpr float kFarLog2 = 4194304.f;

// A block of 32 tokens: pages a and b, wave-uniform.
struct MxBlock {
  int pid_a, vp_a, pid_b, vp_b;  // vp: position << 7 | valid tokens; vp_b 0: no page b
  int lo, hi;                    // rows of the row block whose path holds it
  bool masked, live;             // live: there is such a block
};

// The words of a block as they lie in memory.
template <int M>
struct MxRaw {
  static constexpr int kKeyScales = kMxRun<M> ? (M == 8 ? 2 : 1) : M, kValueScales = kMxRun<M> ? 1 : M;
  uint32_t k[2][M], v[2][M];
  uint32_t ks[2][kKeyScales];    // a byte each
  uint32_t vs[2][kValueScales];  // four tokens' bytes each
};

typedef __amdgpu_buffer_rsrc_t rsrc_t;

template <int M>
__device__ __forceinline__ void load_words(rsrc_t r, int at, uint32_t (&w)[M]) {
#pragma unroll
  for (int i = 0; i < M; i += 4) {
    if (M - i >= 4) {
      const u32x4 x = __builtin_bit_cast(u32x4, __builtin_amdgcn_raw_buffer_load_b128(r, at + 4 * i, 0, 0));
#pragma unroll
      for (int j = 0; j < 4; ++j) w[i + j] = x[j];
    } else if (M - i == 3) {
      const u32x3 x = __builtin_bit_cast(u32x3, __builtin_amdgcn_raw_buffer_load_b96(r, at + 4 * i, 0, 0));
#pragma unroll
      for (int j = 0; j < 3; ++j) w[i + j] = x[j];
    } else if (M - i == 2) {
      const u32x2 x = __builtin_bit_cast(u32x2, __builtin_amdgcn_raw_buffer_load_b64(r, at + 4 * i, 0, 0));
      w[i] = x[0];
      w[i + 1] = x[1];
    } else {
      w[i] = __builtin_amdgcn_raw_buffer_load_b32(r, at + 4 * i, 0, 0);
    }
  }
}

// Requests a block.  A block or page that is not there has no bytes: its loads give zeros and move nothing.
template <int M>
__device__ __forceinline__ void load_block(MxRaw<M> &x, const MxBlock &b, const char *kpool, const char *vpool, int page_tiles, int g) {
  const int lane = threadIdx.x & 63, c = lane & 15, jj = lane >> 4;
#pragma unroll
  for (int p = 0; p < 2; ++p) {
    const int64_t at = (static_cast<int64_t>(p ? b.pid_b : b.pid_a) * page_tiles + g) * mx_tile_bytes(M);
    const int bytes = b.live && (p ? b.vp_b : b.vp_a) != 0 ? mx_tile_bytes(M) : 0;
    const rsrc_t kr = __builtin_amdgcn_make_buffer_rsrc(const_cast<char *>(kpool + at), 0, bytes, 0x00020000);
    const rsrc_t vr = __builtin_amdgcn_make_buffer_rsrc(const_cast<char *>(vpool + at), 0, bytes, 0x00020000);
    load_words<M>(kr, lane * 4 * M, x.k[p]);
#pragma unroll
    for (int i = 0; i < MxRaw<M>::kKeyScales; ++i) {
      const int block = kMxRun<M> ? (M >= 4 ? jj * (M / 4) + i : jj * M / 4) : i;
      x.ks[p][i] = __builtin_amdgcn_raw_buffer_load_b8(kr, mx_scale_at<M>(block, c), 0, 0);
    }
    load_words<M>(vr, lane * 4 * M, x.v[p]);
#pragma unroll
    for (int i = 0; i < MxRaw<M>::kValueScales; ++i) {
      const int block = kMxRun<M> ? c * M / 16 : i;
      x.vs[p][i] = __builtin_amdgcn_raw_buffer_load_b32(vr, mx_scale_at<M>(block, 4 * jj), 0, 0);
    }
  }
}

// A wavefront's rows, 16 to a tile: lane (c = lane % 16, jj = lane / 16) has row c of every tile; its scores are of tokens 4 jj .. + 3
// of page a, then of page b, its accumulators of the dims mx_value_dim(4 jj + i, j) and the one behind, i < 4.
template <int M, int NT>
struct MxRows {
  bf16x8 q[NT][M];
  int limit[NT], qtok[NT], qidx[NT];
  uint32_t dmask[NT];
  f32x4 o[NT][2 * M];
  float m[NT], mc[NT], l[NT];  // reference as a score, and scaled less kWeightLog2; l is the lane's share
  int seen_end;                // path positions from here on no row sees (wave-uniform)
  bool far;                    // wave-uniform: some reference is beyond kFarLog2
};

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
    st.mc[nt] = kMInit * c - kWeightLog2;
    st.l[nt] = 0.f;
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
  st.far = false;
}

// Which of the lane's four tokens of a page the row sees, as bits.
template <bool TREE>
__device__ __forceinline__ uint32_t seen_bits(int limit, int qidx, uint32_t dmask, int vp, int first) {
  const int valid = (vp & 127) - first, pos = (vp >> 7) + first;
  if (TREE) {  // positions below base, and base + k for the set bits k of the mask
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

// A block against the wavefront's rows.  row0: the first of them in the row block.
template <int M, int NT, bool TREE>
__device__ __forceinline__ void block_step(MxRows<M, NT> &st, const MxRaw<M> &x, const MxBlock &b, int row0, float c, float slack) {
  const int lane = threadIdx.x & 63, jj = lane >> 4;
  f32x4 s[NT][2];
#pragma unroll
  for (int p = 0; p < 2; ++p) {
    float scale[MxRaw<M>::kKeyScales];
#pragma unroll
    for (int i = 0; i < MxRaw<M>::kKeyScales; ++i) scale[i] = mx_scale(x.ks[p][i]);
#pragma unroll
    for (int nt = 0; nt < NT; ++nt) s[nt][p] = f32x4{0.f, 0.f, 0.f, 0.f};
#pragma unroll
    for (int i = 0; i < M; ++i) {
      const bf16x8 kf = key_operand<M>(x.k[p][i], scale[kMxRun<M> ? (M == 8 ? i / 4 : 0) : i]);
#pragma unroll
      for (int nt = 0; nt < NT; ++nt) s[nt][p] = __builtin_amdgcn_mfma_f32_16x16x32_bf16(kf, st.q[nt][i], s[nt][p], 0, 0, 0);
    }
  }
  f16x8 ph[NT], pl[NT];
#pragma unroll
  for (int nt = 0; nt < NT; ++nt) {
    float y[8];
#pragma unroll
    for (int i = 0; i < 4; ++i) {
      y[i] = s[nt][0][i];
      y[4 + i] = s[nt][1][i];
    }
    const int first_row = row0 + 16 * nt;
    if (b.masked || b.lo > first_row || b.hi < first_row + 16) {
      const int row = first_row + (lane & 15);
      uint32_t seen = seen_bits<TREE>(st.limit[nt], st.qidx[nt], st.dmask[nt], b.vp_a, 4 * jj) |
                      seen_bits<TREE>(st.limit[nt], st.qidx[nt], st.dmask[nt], b.vp_b, 4 * jj) << 4;
      if (row < b.lo || row >= b.hi) seen = 0;
#pragma unroll
      for (int i = 0; i < 8; ++i) y[i] = (seen >> i) & 1 ? y[i] : kNegInf;
    }
    const float top = fmaxf(fmaxf(fmaxf(y[0], y[1]), fmaxf(y[2], y[3])), fmaxf(fmaxf(y[4], y[5]), fmaxf(y[6], y[7])));
    if (__any(top > st.m[nt] + slack)) {
      const float m_new = row_group_max(fmaxf(top, st.m[nt]));
      const float alpha = fast_exp2((st.m[nt] - m_new) * c);
      st.m[nt] = m_new;
      st.mc[nt] = __builtin_fmaf(m_new, c, -kWeightLog2);
      st.far = st.far || __any(fabsf(st.mc[nt]) >= kFarLog2 && m_new != kMInit);
      st.l[nt] *= alpha;
#pragma unroll
      for (int i = 0; i < 2 * M; ++i) st.o[nt][i] *= alpha;
    }
    if (st.far) {
#pragma unroll
      for (int i = 0; i < 8; ++i) y[i] = fast_exp2(__builtin_fmaf(y[i] - st.m[nt], c, kWeightLog2));
    } else {
#pragma unroll
      for (int i = 0; i < 8; ++i) y[i] = fast_exp2(__builtin_fmaf(y[i], c, -st.mc[nt]));
    }
    st.l[nt] += ((y[0] + y[1]) + (y[2] + y[3])) + ((y[4] + y[5]) + (y[6] + y[7]));
    u32x4 h, rest;
#pragma unroll
    for (int i = 0; i < 4; ++i) {
      h[i] = __builtin_bit_cast(uint32_t, f16x2{static_cast<_Float16>(y[2 * i]), static_cast<_Float16>(y[2 * i + 1])});
      rest[i] = rest_of(h[i], y[2 * i], y[2 * i + 1]);
    }
    ph[nt] = __builtin_bit_cast(f16x8, h);
    pl[nt] = __builtin_bit_cast(f16x8, rest);
  }
  float vs[2][4];
#pragma unroll
  for (int j = 0; j < M; ++j) {
    if (j == 0 || !kMxRun<M>) {
#pragma unroll
      for (int p = 0; p < 2; ++p)
#pragma unroll
        for (int t = 0; t < 4; ++t) vs[p][t] = mx_scale((x.vs[p][kMxRun<M> ? 0 : j] >> (8 * t)) & 255u);
    }
    // a word: dims d, d + 1 of four tokens, a byte each -> the rows of d and of d + 1, tokens side by side
    u32x4 r0, r1;
#pragma unroll
    for (int p = 0; p < 2; ++p) {
      uint32_t w[4];
      w[0] = __builtin_bit_cast(uint32_t, __builtin_amdgcn_cvt_scalef32_pk_f16_fp4(x.v[p][j], vs[p][0], 0));
      w[1] = __builtin_bit_cast(uint32_t, __builtin_amdgcn_cvt_scalef32_pk_f16_fp4(x.v[p][j], vs[p][1], 1));
      w[2] = __builtin_bit_cast(uint32_t, __builtin_amdgcn_cvt_scalef32_pk_f16_fp4(x.v[p][j], vs[p][2], 2));
      w[3] = __builtin_bit_cast(uint32_t, __builtin_amdgcn_cvt_scalef32_pk_f16_fp4(x.v[p][j], vs[p][3], 3));
#pragma unroll
      for (int t = 0; t < 2; ++t) {
        r0[2 * p + t] = __builtin_amdgcn_perm(w[2 * t + 1], w[2 * t], 0x05040100u);
        r1[2 * p + t] = __builtin_amdgcn_perm(w[2 * t + 1], w[2 * t], 0x07060302u);
      }
    }
    const f16x8 a0 = __builtin_bit_cast(f16x8, r0), a1 = __builtin_bit_cast(f16x8, r1);
#pragma unroll
    for (int nt = 0; nt < NT; ++nt) {
      st.o[nt][2 * j] = __builtin_amdgcn_mfma_f32_16x16x32_f16(a0, ph[nt], st.o[nt][2 * j], 0, 0, 0);
      st.o[nt][2 * j] = __builtin_amdgcn_mfma_f32_16x16x32_f16(a0, pl[nt], st.o[nt][2 * j], 0, 0, 0);
      st.o[nt][2 * j + 1] = __builtin_amdgcn_mfma_f32_16x16x32_f16(a1, ph[nt], st.o[nt][2 * j + 1], 0, 0, 0);
      st.o[nt][2 * j + 1] = __builtin_amdgcn_mfma_f32_16x16x32_f16(a1, pl[nt], st.o[nt][2 * j + 1], 0, 0, 0);
    }
  }
}

// Where a finished or partial row goes.
struct RowPlace {
  int64_t at;  // row of the destination, or -1: none
  float inv;
};
// LDS of a set of wavefronts that hold the same rows: a stage of 16 rows each, softmax states, places.
template <int M, int NT>
struct MxJoin {
  static constexpr int kRow = 32 * M + 4;  // the pad spreads rows over the banks
  static constexpr int kStage = 16 * kRow;
  static constexpr int floats(int waves) { return waves * (kStage + 2 * 16 * NT) + 4 * 16; }
};

// Joins the states of the KS wavefronts (number ks of them calls) that hold the same rows, and writes the rows.  Called by all of a
// workgroup's wavefronts together, with an area of their own for each set.  place(nt, row of the tile): the destination row or -1.
template <int M, int NT, int KS, class Place>
__device__ __forceinline__ void join_rows(MxRows<M, NT> &st, int ks, float c, float *area, float *dst, float *ml, float *lse, Place place) {
  constexpr int kRow = MxJoin<M, NT>::kRow, kStage = MxJoin<M, NT>::kStage, D = 32 * M;
  const int lane = threadIdx.x & 63, row = lane & 15, jj = lane >> 4;
  float *states = area + KS * kStage;  // [wavefront][row]{m, l}
  RowPlace *places = reinterpret_cast<RowPlace *>(states + KS * 2 * 16 * NT);
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
    st.l[nt] += __shfl_xor(st.l[nt], 16);
    st.l[nt] += __shfl_xor(st.l[nt], 32);
    if (KS > 1 && jj == 0) *reinterpret_cast<f32x2 *>(states + (ks * 16 * NT + 16 * nt + row) * 2) = f32x2{st.m[nt], st.l[nt]};
  }
  if (KS > 1) __syncthreads();
#pragma unroll
  for (int nt = 0; nt < NT; ++nt) {
    float m = st.m[nt], l = st.l[nt], factor = 1.f;
    if (KS > 1) {
      f32x2 all[KS];
#pragma unroll
      for (int k = 0; k < KS; ++k) {
        all[k] = *reinterpret_cast<const f32x2 *>(states + (k * 16 * NT + 16 * nt + row) * 2);
        m = fmaxf(m, all[k][0]);
      }
      l = 0.f;
#pragma unroll
      for (int k = 0; k < KS; ++k) l += all[k][1] * fast_exp2((all[k][0] - m) * c);
      factor = fast_exp2((st.m[nt] - m) * c);
    }
    float *stage = area + ks * kStage;
#pragma unroll
    for (int i = 0; i < 4; ++i)
#pragma unroll
      for (int j = 0; j < 2 * M; j += (kMxRun<M> && M > 1 ? 4 : 2)) {
        float *to = stage + row * kRow + mx_value_dim<M>(4 * jj + i, j / 2);
        if constexpr (kMxRun<M> && M > 1)
          *reinterpret_cast<f32x4 *>(to) = f32x4{st.o[nt][j][i], st.o[nt][j + 1][i], st.o[nt][j + 2][i], st.o[nt][j + 3][i]} * factor;
        else
          *reinterpret_cast<f32x2 *>(to) = f32x2{st.o[nt][j][i], st.o[nt][j + 1][i]} * factor;
      }
    if (ks == 0 && jj == 0) {
      const int64_t at = place(nt, row);
      places[row] = {at, ml ? 1.f : 1.f / l};
      if (at >= 0) {
        if (ml)
          *reinterpret_cast<f32x2 *>(ml + 2 * at) = f32x2{__builtin_fmaf(m, c, -kWeightLog2), l};
        else if (lse)
          lse[at] = (__builtin_fmaf(m, c, -kWeightLog2) + __builtin_log2f(l)) * 0.6931471805599453f;
      }
    }
    meet();
    for (int i = ks * 64 + lane; i < 16 * (D / 4); i += 64 * KS) {
      const int r = i / (D / 4), d = i % (D / 4) * 4;
      const RowPlace to = places[r];
      f32x4 v = *reinterpret_cast<const f32x4 *>(area + r * kRow + d);
#pragma unroll
      for (int k = 1; k < KS; ++k) v += *reinterpret_cast<const f32x4 *>(area + k * kStage + r * kRow + d);
      if (to.at >= 0) *reinterpret_cast<f32x4_out *>(dst + to.at * D + d) = v * to.inv;
    }
    if (nt + 1 < NT) meet();
  }
}

constexpr int kWaves = 4;  // of a workgroup: they hold the same rows

// The blocks of wavefront w of a workgroup: records w, w + 4, .. of a list, 64 of them at a time in registers, a lane each.
// read(i): record i, for a lane; lanes whose record does not concern the wavefront's rows drop out.
struct MxLanes {
  int pid_a, vp_a, pid_b, vp_b, rows, flags;
};
template <class Read>
struct MxSource {
  Read read;
  int n, at;
  uint64_t left;
  MxLanes r;
  __device__ __forceinline__ MxBlock next() {
    while (left == 0 && at < n) {
      const int i = at + kWaves * (threadIdx.x & 63);
      bool concerns = i < n;
      if (concerns) concerns = read(i, r);
      left = __ballot(concerns);
      at += 64 * kWaves;
    }
    MxBlock b;
    b.live = left != 0;
    const int l = b.live ? __builtin_ctzll(left) : 0;
    left &= left - 1;
    b.pid_a = __builtin_amdgcn_readlane(r.pid_a, l);
    b.vp_a = __builtin_amdgcn_readlane(r.vp_a, l);
    b.pid_b = __builtin_amdgcn_readlane(r.pid_b, l);
    b.vp_b = __builtin_amdgcn_readlane(r.vp_b, l);
    const int rows = __builtin_amdgcn_readlane(r.rows, l);
    b.lo = rows & 0xffff;
    b.hi = static_cast<int>(static_cast<uint32_t>(rows) >> 16);
    b.masked = __builtin_amdgcn_readlane(r.flags, l) & 1;
    return b;
  }
};

// One block is worked on while the next is on its way, in registers of its own.
template <int M, int NT, bool TREE, class Read>
__device__ __forceinline__ void walk_blocks(MxRows<M, NT> &st, const void *k, const void *v, int page_tiles, int g, int row0, float c, int n, int w,
                                            Read read) {
  const char *kpool = static_cast<const char *>(k), *vpool = static_cast<const char *>(v);
  const float slack = kSlackLog2 / c;
  MxSource<Read> src{read, n, w, 0, {}};
  MxRaw<M> x0, x1;
  MxBlock b0 = src.next();
  load_block<M>(x0, b0, kpool, vpool, page_tiles, g);
  MxBlock b1 = src.next();
  load_block<M>(x1, b1, kpool, vpool, page_tiles, g);
  while (b0.live) {
    block_step<M, NT, TREE>(st, x0, b0, row0, c, slack);
    b0 = src.next();
    load_block<M>(x0, b0, kpool, vpool, page_tiles, g);
    if (!b1.live) break;
    block_step<M, NT, TREE>(st, x1, b1, row0, c, slack);
    b1 = src.next();
    load_block<M>(x1, b1, kpool, vpool, page_tiles, g);
  }
}

// Wavefronts a SIMD: with one the compiler keeps accumulators in the other half of the register file and moves them for every block.
constexpr int mx_occupancy(int blocks, int row_tiles) { return blocks * row_tiles <= 4 ? 3 : 2; }

template <int M, int NT, bool TREE>
__global__ __launch_bounds__(64 * kWaves, mx_occupancy(M, NT)) void spex_mxfp4_split_kernel(AttnArgs p, Shape sh, SplitLists ls) {
  __shared__ __attribute__((aligned(16))) float lds[MxJoin<M, NT>::floats(kWaves)];
  const ListPos at = list_of(ls, static_cast<int>(blockIdx.x));
  const int tile = at.local / at.n_items;
  Item cur = load_item(at.items, at.local - tile * at.n_items);
  cur.row0 += tile * 16 * NT;
  const int G = sh.G, rows = cur.qt_count * G;
  if (cur.pg_count == 0 || cur.row0 >= rows) return;  // whole workgroup: padding item, or no such tile
  const int w = uniform(threadIdx.x >> 6), g = cur.g;
  const float c = p.scale_log2;
  MxRows<M, NT> st;
  load_rows<M, NT, TREE>(st, p.q, p.qt_rec, p.qt_mask, cur.qt_begin, cur.row0, rows, g, sh, c);
  walk_blocks<M, NT, TREE>(st, p.k_pool, p.v_pool, sh.page_tiles, g, 0, c, (cur.pg_count + 1) >> 1, w, [&](int i, MxLanes &r) {
    const int2 *pages = reinterpret_cast<const int2 *>(p.pg_rec) + cur.pg_begin + 2 * i;
    const bool has_b = 2 * i + 1 < cur.pg_count;
    const int2 a = pages[0], b = pages[has_b ? 1 : 0];
    r = {a.x, a.y, b.x, has_b ? b.y : 0, static_cast<int>(0xffff0000u), cur.flags | (has_b ? 0 : 1)};
    return (a.y >> 7) < st.seen_end;
  });
  join_rows<M, NT, kWaves>(st, w, c, lds, p.finish ? p.out : p.part_o, p.finish ? nullptr : p.part_ml, p.lse, [&](int nt, int row) {
    const int r = cur.row0 + 16 * nt + row;
    if (r >= rows) return static_cast<int64_t>(-1);
    return p.finish ? static_cast<int64_t>(st.qtok[nt]) * sh.Hq + g * G + r % G
                    : static_cast<int64_t>(cur.pbase) + static_cast<int64_t>(g) * rows + r;
  });
}

// One workgroup for each set of 16 NT rows of the row blocks' NW wavefronts of 16 ntw.  The sets of a row block read its shared blocks
// one beside the other: they are eight workgroups apart, which is one XCD.
template <int M, int NT, bool TREE>
__global__ __launch_bounds__(64 * kWaves, mx_occupancy(M, NT)) void spex_mxfp4_walk_kernel(WalkArgs p, Shape sh, int nw, int ntw) {
  __shared__ __attribute__((aligned(16))) float lds[MxJoin<M, NT>::floats(kWaves)];
  const int groups = ntw / NT, sets = nw * groups;
  const int batch = static_cast<int>(blockIdx.x) / (8 * sets), within = static_cast<int>(blockIdx.x) - batch * 8 * sets;
  const int set = within >> 3, item = batch * 8 + (within & 7);
  if (item >= p.n_items) return;
  const int rw = set / groups, row_base = (set - rw * groups) * 16 * NT;
  const int64_t ir = static_cast<int64_t>(item) * (nw <= 4 ? 16 : 32);
  const int rows = sload(p.items, ir + 3 + 2 * nw + rw) * sh.G;
  if (row_base >= rows) return;  // padding, a wavefront without rows, or no such tile
  const int g = sload(p.items, ir), blk_begin = sload(p.items, ir + 1), n_shared = sload(p.items, ir + 2);
  // per wavefront: private blocks | room << 16
  const int n_priv = sload(p.items, ir + 3 + rw) & 0xffff;
  int priv_begin = blk_begin + n_shared;
  for (int v = 0; v < rw; ++v) priv_begin += static_cast<int>(static_cast<uint32_t>(sload(p.items, ir + 3 + v)) >> 16);
  const int row0 = rw * 16 * ntw + row_base, qt_begin = sload(p.items, ir + 3 + nw + rw), G = sh.G, w = uniform(threadIdx.x >> 6);
  const float c = p.scale_log2;
  MxRows<M, NT> st;
  load_rows<M, NT, TREE>(st, p.q, p.qt_rec, p.qt_mask, qt_begin, row_base, rows, g, sh, c);
  walk_blocks<M, NT, TREE>(st, p.k_pool, p.v_pool, sh.page_tiles, g, row0, c, n_shared + n_priv, w, [&](int i, MxLanes &r) {
    const u32x4 *rec = reinterpret_cast<const u32x4 *>(p.blocks) + 2 * static_cast<int64_t>(i < n_shared ? blk_begin + i : priv_begin + i - n_shared);
    const u32x4 a = rec[0], b = rec[1];
    r = {static_cast<int>(a[0]), static_cast<int>(a[1]), static_cast<int>(a[2]), static_cast<int>(a[3]), static_cast<int>(b[0]), static_cast<int>(b[1])};
    return static_cast<int>(b[0] & 0xffffu) < row0 + 16 * NT && static_cast<int>(b[0] >> 16) > row0 && (r.vp_a >> 7) < st.seen_end;
  });
  join_rows<M, NT, kWaves>(st, w, c, lds, p.out, nullptr, p.lse, [&](int nt, int row) {
    const int r = row_base + 16 * nt + row;
    return r < rows ? static_cast<int64_t>(st.qtok[nt]) * sh.Hq + g * G + r % G : static_cast<int64_t>(-1);
  });
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

// Row tiles of a workgroup: two where there are rows for them; wide heads have registers for one.
constexpr int mx_row_tiles(int blocks) { return blocks <= 4 ? 2 : 1; }

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
  const int64_t n_wg = (static_cast<int64_t>(a.n_items) + 7) / 8 * 8 * waves * (ntw / NT);
  if (n_wg > INT32_MAX) return hipErrorInvalidValue;
  const dim3 grid(static_cast<unsigned>(n_wg)), block(64 * kWaves);
  if (a.qt_mask)
    hipLaunchKernelGGL((spex_mxfp4_walk_kernel<M, NT, true>), grid, block, 0, stream, a, sh, waves, ntw);
  else
    hipLaunchKernelGGL((spex_mxfp4_walk_kernel<M, NT, false>), grid, block, 0, stream, a, sh, waves, ntw);
  return hipGetLastError();
}

}  // namespace

hipError_t launch_mxfp4_split(const Shape &sh, const AttnArgs &a, const ItemLists &l, hipStream_t stream) {
  return with_blocks(sh.D, [&](auto m) {
    constexpr int M = decltype(m)::value;
    return std::max({l.span[0], l.span[1], l.span[2], l.span[3]}) <= 16 ? launch_split<M, 1>(sh, a, l, stream)
                                                                       : launch_split<M, mx_row_tiles(M)>(sh, a, l, stream);
  });
}

hipError_t launch_mxfp4_walk(const Shape &sh, const WalkArgs &a, int ntw, int waves, hipStream_t stream) {
  if (a.n_items <= 0) return hipSuccess;
  if ((ntw != 1 && ntw != 2 && ntw != 4) || (waves != 2 && waves != 4 && waves != 8)) return hipErrorInvalidValue;
  return with_blocks(sh.D, [&](auto m) {
    constexpr int M = decltype(m)::value;
    return ntw == 1 ? launch_walk<M, 1>(sh, a, ntw, waves, stream) : launch_walk<M, mx_row_tiles(M)>(sh, a, ntw, waves, stream);
  });
}

}  // namespace spex
