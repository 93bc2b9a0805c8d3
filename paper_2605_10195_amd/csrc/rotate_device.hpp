// Device code shared by the kernels that append rotated tokens.
#pragma once

#include "kernels.hpp"

namespace spex {
namespace {

typedef float f32x4 __attribute__((ext_vector_type(4)));
typedef float f32x2 __attribute__((ext_vector_type(2)));
typedef uint32_t u32x4 __attribute__((ext_vector_type(4)));
typedef uint32_t u32x2 __attribute__((ext_vector_type(2)));

__device__ __forceinline__ int uniform(int v) { return __builtin_amdgcn_readfirstlane(v); }
__device__ __forceinline__ float wave_max(float v) {
#pragma unroll
  for (int o = 32; o >= 1; o >>= 1) v = fmaxf(v, __shfl_xor(v, o));
  return v;
}
__device__ __forceinline__ float bf16_bits_to_float(uint16_t b) {
  return __builtin_bit_cast(float, static_cast<uint32_t>(b) << 16);
}
__device__ __forceinline__ uint16_t half_word(const u32x4 &v, int i) {
  return static_cast<uint16_t>(v[i >> 1] >> (16 * (i & 1)));
}

// Cosine and sine of 2 pi p (f.hi + f.lo).  p f.hi is split exactly into its rounded value and the rest; after whole turns and
// quarter turns at most an eighth of a turn is left, where the Taylor series to the 13th and 14th power are off by less than 3e-14.
// Nothing is contracted: t - rint(t) made into one fma of x f.hi would hold the rest already, and it would count twice.
__device__ __forceinline__ f32x2 cos_sin_turns(int p, const Turns f) {
#pragma clang fp contract(off)
  const double x = static_cast<double>(p);
  const double t = x * f.hi, rest = __builtin_fma(x, f.hi, -t) + x * f.lo;
  const double r = (t - __builtin_rint(t)) + rest;         // in [-0.5, 0.5], almost
  const double quarter = __builtin_rint(4.0 * r);
  const double a = 6.283185307179586476925 * __builtin_fma(-0.25, quarter, r);
  const double a2 = a * a;
  double s = 1.0 / 6227020800.0;
  s = __builtin_fma(s, a2, -1.0 / 39916800.0);
  s = __builtin_fma(s, a2, 1.0 / 362880.0);
  s = __builtin_fma(s, a2, -1.0 / 5040.0);
  s = __builtin_fma(s, a2, 1.0 / 120.0);
  s = __builtin_fma(s, a2, -1.0 / 6.0);
  s = __builtin_fma(s * a2, a, a);
  double c = -1.0 / 87178291200.0;
  c = __builtin_fma(c, a2, 1.0 / 479001600.0);
  c = __builtin_fma(c, a2, -1.0 / 3628800.0);
  c = __builtin_fma(c, a2, 1.0 / 40320.0);
  c = __builtin_fma(c, a2, -1.0 / 720.0);
  c = __builtin_fma(c, a2, 1.0 / 24.0);
  c = __builtin_fma(c, a2, -0.5);
  c = __builtin_fma(c, a2, 1.0);
  const int n = static_cast<int>(quarter) & 3;
  const double cn = (n & 1) ? s : c, sn = (n & 1) ? c : s;
  return f32x2{static_cast<float>(n == 1 || n == 2 ? -cn : cn), static_cast<float>(n >= 2 ? -sn : sn)};
}

__device__ __forceinline__ f32x2 turned(float x1, float x2, f32x2 cs) {
#pragma clang fp contract(off)
  return f32x2{x1 * cs[0] - x2 * cs[1], x2 * cs[0] + x1 * cs[1]};
}

// A record: tokens tok0 .. tok0 + hi - lo - 1 of the call go to slots [lo, hi) of the page.
struct PageVisit {
  int page, lo, hi, fill, tok0, pos0, new_index;
  bool is_new;  // this call starts the page: slots up to fill = P are written, zeros behind the tokens
};
// Lists of up to kInlineInts travel in the kernel arguments; longer ones are read where the host wrote them, in pinned memory.
__device__ __forceinline__ PageVisit page_visit(const RotateArgs &a, const RotateLists &in, int P) {
  int r[kVisitInts];
  const int at = static_cast<int>(blockIdx.x) * kVisitInts;
  if (a.lists) {  // one access a wavefront: the lanes read an int each
    const int x = a.lists[at + min(static_cast<int>(threadIdx.x) & 63, kVisitInts - 1)];
#pragma unroll
    for (int i = 0; i < kVisitInts; ++i) r[i] = __builtin_amdgcn_readlane(x, i);
  } else {
#pragma unroll
    for (int i = 0; i < kVisitInts; ++i) r[i] = uniform(in.ints[at + i]);
  }
  PageVisit v;
  v.page = r[0];
  v.tok0 = r[2];
  v.pos0 = r[3];
  v.new_index = r[4];
  v.lo = r[1] & 0xff;
  v.hi = (r[1] >> 8) & 0xff;
  v.is_new = (r[1] >> 16) != 0;
  v.fill = v.is_new ? P : v.hi;
  return v;
}
// Position of token t of a record.
__device__ __forceinline__ int position(const RotateArgs &a, const RotateLists &in, const PageVisit &v, int t) {
  if (!a.has_positions) return v.pos0 + t;
  const int at = a.n_recs * kVisitInts + v.tok0 + t;
  return a.lists ? a.lists[at] : in.ints[at];
}

// Where token t begins; strides are below 2^31.
__device__ __forceinline__ int64_t token_at(int t, int64_t stride) {
  return static_cast<int64_t>(static_cast<uint64_t>(static_cast<uint32_t>(t)) * static_cast<uint32_t>(stride));
}
__device__ __forceinline__ uint16_t half_of(uint32_t w, int i) { return static_cast<uint16_t>(w >> (16 * i)); }

__device__ __forceinline__ void apply_patches(const RotateArgs &a, const RotateLists &in) {
  if (blockIdx.y != 0) return;
  for (int i = static_cast<int>(blockIdx.x * 256 + threadIdx.x); i < a.n_patches; i += static_cast<int>(gridDim.x) * 256) {
    const int at = a.patches + 2 * i;
    if (a.lists)
      a.plan[a.lists[at]] = a.lists[at + 1];
    else
      a.plan[in.ints[at]] = in.ints[at + 1];
  }
}

// Eight dims of a row.
struct Eight {
  float x[8];
};
template <bool F32>
__device__ __forceinline__ Eight load_eight(const void *base, int64_t at) {
  Eight r;
  if (F32) {
    const f32x4 *p = reinterpret_cast<const f32x4 *>(static_cast<const float *>(base) + at);
    const f32x4 a = p[0], b = p[1];
#pragma unroll
    for (int i = 0; i < 4; ++i) r.x[i] = a[i], r.x[4 + i] = b[i];
  } else {
    const u32x4 w = *reinterpret_cast<const u32x4 *>(static_cast<const uint16_t *>(base) + at);
#pragma unroll
    for (int i = 0; i < 8; ++i) r.x[i] = bf16_bits_to_float(half_word(w, i));
  }
  return r;
}
__device__ __forceinline__ uint32_t pair_bf16(float a, float b) {
  typedef __bf16 bf16x2 __attribute__((ext_vector_type(2)));
  return __builtin_bit_cast(uint32_t, bf16x2{static_cast<__bf16>(a), static_cast<__bf16>(b)});
}
template <bool F32>
__device__ __forceinline__ void store_eight(void *base, int64_t at, const Eight &e) {
  if (F32) {
    f32x4 *p = reinterpret_cast<f32x4 *>(static_cast<float *>(base) + at);
    p[0] = f32x4{e.x[0], e.x[1], e.x[2], e.x[3]};
    p[1] = f32x4{e.x[4], e.x[5], e.x[6], e.x[7]};
  } else {
    *reinterpret_cast<u32x4 *>(static_cast<uint16_t *>(base) + at) =
        u32x4{pair_bf16(e.x[0], e.x[1]), pair_bf16(e.x[2], e.x[3]), pair_bf16(e.x[4], e.x[5]), pair_bf16(e.x[6], e.x[7])};
  }
}
__device__ __forceinline__ float largest(const Eight &e) {
  float m = 0.f;
#pragma unroll
  for (int i = 0; i < 8; ++i) m = fmaxf(m, __builtin_fabsf(e.x[i]));
  return m;
}

}  // namespace
}  // namespace spex
