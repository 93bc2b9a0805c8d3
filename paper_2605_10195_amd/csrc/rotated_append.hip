// HIP kernels of spex_tree_append_rotated on gfx950.
//
//   spex_append_rotated_kernel
//       Tiled pools.  One workgroup per (page that the call writes to, range of kv heads): the cosines and sines of its tokens into
//       LDS, then queries, keys and values in jobs of a wavefront.
//   spex_append_rotated_rows_kernel
//       Row-major pools: the same, 16 bytes of a row at a time.
//   spex_append_rotated_any_kernel
//       The same element by element, for rows, buffers or rotated parts that are not made of 16-byte pieces.
//
// Bound: memory.  Runs of prompts move at the rate of a large copy (5 TB/s here): 211 MB of bf16 prompts take 40 us, 1.08 GB into
// an fp8 cache 254 us (4.3 TB/s, encoding beside it), 92 MB of drafts, six tokens a page, 25 us.  Steps of one token are bound
// by latency, a launch, the angles, one round of loads and stores: 16 branches of 32/8/128 take 4.9 us, 1024 of 28/4/128 13.5
// (21 MB, 4 us by bytes; the rest is the one round of every workgroup behind its record, which comes over the bus: 1.3 us at 141 nodes).
//
// Mathematics: the pair (x1, x2) number i of a head at position p turns by the angle p * inv_freq[i],
//   y1 = x1 cos - x2 sin,  y2 = x2 cos + x1 sin.
// The angle is taken in 64 bits, as turns, so that whole turns can be dropped exactly however far the position; cosine
// and sine are rounded to fp32, products and sums are fp32 operations rounded one by one, and the result is rounded once to the
// type it is stored in.
#include <algorithm>
#include <type_traits>

#include "kernels.hpp"
#include "rotate_device.hpp"

namespace spex {
namespace {

// Where the attention kernels expect token t, dim d of a tile.
template <int KV, int LAYOUT>
__device__ __forceinline__ int k_offset(int t, int d, int D) {
  if (LAYOUT == kRowMajor) return t * D + d;
  const int tt = 4 * (t >> 3) + (t & 3);
  if (KV == kFP8)
    return ((t >> 2) & 1) * 8 * D + (d >> 6) * 512 + ((d & 31) >> 3) * 128 + tt * 16 +
           ((d >> 5) & 1) * 8 + (d & 7);
  return ((t >> 2) & 1) * 8 * D + (d >> 5) * 256 + ((d & 31) >> 3) * 64 + tt * 8 + (d & 7);
}
template <int KV, int LAYOUT>
__device__ __forceinline__ int v_offset(int t, int d, int D) {
  if (LAYOUT == kRowMajor) return t * D + d;
  if (KV == kFP8)
    return (d >> 5) * 512 + (t >> 3) * 256 + (d & 15) * 16 + ((d >> 4) & 1) * 8 + (t & 7);
  return (d >> 4) * 256 + (t >> 3) * 128 + (d & 15) * 8 + (t & 7);
}
// Tiled bf16 pools hold V in IEEE half precision, rounded toward zero.
template <int KV, int LAYOUT>
__device__ __forceinline__ constexpr bool v_is_f16() {
  return KV == kBF16 && LAYOUT == kMfmaTiled;
}
__device__ __forceinline__ uint16_t bf16_bits_to_f16_bits(uint16_t b) {
  return static_cast<uint16_t>(__builtin_bit_cast(uint32_t, __builtin_amdgcn_cvt_pkrtz(bf16_bits_to_float(b), 0.f)));
}
// fp32 -> e4m3: to nearest even, saturating, NaN kept, by integer arithmetic.
__device__ __forceinline__ uint32_t encode_e4m3(float y) {
  const uint32_t u = __builtin_bit_cast(uint32_t, y);
  const uint32_t sign = (u >> 24) & 0x80u, a = u & 0x7fffffffu;
  uint32_t code;
  if (a > 0x7f800000u) {
    code = 0x7fu;
  } else if (a >= 0x43e00000u) {  // 448.0f and above (infinity included)
    code = 0x7eu;
  } else if (a >= 0x3c800000u) {  // 2^-6
    const uint32_t r = a + 0x7ffffu + ((a >> 20) & 1u);
    code = (((r >> 23) - 120u) << 3) | ((r >> 20) & 7u);
  } else {
    code = static_cast<uint32_t>(__builtin_rintf(__builtin_bit_cast(float, a) * 512.0f));
  }
  return code | sign;
}

// The reciprocal of a page's scale.  A scale of 0 is a page of zeros: finite here, so that 0 times it is 0.
__device__ __forceinline__ float inverse_scale(float s) { return fminf(1.0f / s, __FLT_MAX__); }
__device__ __forceinline__ float page_scale(float amax) { return fmaxf(amax / 448.0f, 0x1p-40f); }

// Two pieces of eight dims that are turned together: unit u of a row of D dims has dims d[0] .. + 7 and, where it has a second
// piece, d[1] .. + 7.  Halves: pair i is (i, i + R/2); interleaved: (2i, 2i + 1).
template <bool F32, bool INTER>
struct Unit {
  Eight e[2];
  int d[2];
  bool two, rotated[2];
  __device__ __forceinline__ void place(int u, int D, int R) {
    const bool halves = !INTER && 16 * u < R;
    d[0] = halves ? 8 * u : 16 * u;
    d[1] = halves ? 8 * u + R / 2 : 16 * u + 8;
    two = d[1] < D;
    rotated[0] = d[0] < R;
    rotated[1] = d[1] < R;
  }
  __device__ __forceinline__ void load(const void *base, int64_t row) {
    e[0] = load_eight<F32>(base, row + d[0]);
    e[1] = two ? load_eight<F32>(base, row + d[1]) : e[0];
  }
  __device__ __forceinline__ void clear() {
#pragma unroll
    for (int j = 0; j < 8; ++j) e[0].x[j] = e[1].x[j] = 0.f;
  }
  // cs: cosines and sines of the token's pairs.
  __device__ __forceinline__ void turn(const f32x2 *cs) {
    if (INTER) {
#pragma unroll
      for (int k = 0; k < 2; ++k)
        if (rotated[k]) {
#pragma unroll
          for (int i = 0; i < 4; ++i) {
            const f32x2 y = turned(e[k].x[2 * i], e[k].x[2 * i + 1], cs[d[k] / 2 + i]);
            e[k].x[2 * i] = y[0];
            e[k].x[2 * i + 1] = y[1];
          }
        }
    } else if (rotated[0]) {
#pragma unroll
      for (int i = 0; i < 8; ++i) {
        const f32x2 y = turned(e[0].x[i], e[1].x[i], cs[d[0] + i]);
        e[0].x[i] = y[0];
        e[1].x[i] = y[1];
      }
    }
  }
  __device__ __forceinline__ void store(void *base, int64_t row) const {
    store_eight<F32>(base, row + d[0], e[0]);
    if (two) store_eight<F32>(base, row + d[1], e[1]);
  }
  __device__ __forceinline__ float top() const { return fmaxf(largest(e[0]), two ? largest(e[1]) : 0.f); }
};

// e4m3 codes of a, b, c, d, as encode_e4m3 gives them: values clamped to +-448, then converted to nearest even two at a time.
// The clamp would take a NaN to a number, so four values with one among them are encoded one by one.
__device__ __forceinline__ uint32_t encode_four(float a, float b, float c, float d) {
  const uint32_t top = max(max(__builtin_bit_cast(uint32_t, a) & 0x7fffffffu, __builtin_bit_cast(uint32_t, b) & 0x7fffffffu),
                           max(__builtin_bit_cast(uint32_t, c) & 0x7fffffffu, __builtin_bit_cast(uint32_t, d) & 0x7fffffffu));
  if (top > 0x7f800000u) return encode_e4m3(a) | encode_e4m3(b) << 8 | encode_e4m3(c) << 16 | encode_e4m3(d) << 24;
  int r = __builtin_amdgcn_cvt_pk_fp8_f32(__builtin_amdgcn_fmed3f(a, -448.f, 448.f), __builtin_amdgcn_fmed3f(b, -448.f, 448.f), 0, false);
  r = __builtin_amdgcn_cvt_pk_fp8_f32(__builtin_amdgcn_fmed3f(c, -448.f, 448.f), __builtin_amdgcn_fmed3f(d, -448.f, 448.f), r, true);
  return static_cast<uint32_t>(r);
}
__device__ __forceinline__ u32x2 encode_eight(const Eight &e, float inv) {
  return u32x2{encode_four(e.x[0] * inv, e.x[1] * inv, e.x[2] * inv, e.x[3] * inv),
               encode_four(e.x[4] * inv, e.x[5] * inv, e.x[6] * inv, e.x[7] * inv)};
}
// Eight dims of a token into a tile.
template <int KV>
__device__ __forceinline__ void put_eight(char *tile, int at, const Eight &e, float inv) {
  if (KV == kFP8)
    *reinterpret_cast<u32x2 *>(tile + at) = encode_eight(e, inv);
  else
    store_eight<KV == kF32>(tile, at, e);
}

// Tiled pools.  A workgroup's work is cut into jobs of a wavefront, dealt to its four wavefronts in turn: a kv head's values (D 64:
// two heads'; of a few tokens, rows), a page's worth of units of keys, two units of queries a lane.  Loads of a job are all under way before the first is used.
template <int KV, int D, bool INTER>
__global__ __launch_bounds__(256) void spex_append_rotated_kernel(RotateArgs a, Shape sh, RotateLists in) {
  constexpr bool FP8 = KV == kFP8;
  constexpr int P = 16, U = D / 16, N = P * U / 64, ESZ = FP8 ? 1 : 2;
  extern __shared__ __attribute__((aligned(16))) char lds_[];
  f32x2 *cs = reinterpret_cast<f32x2 *>(lds_);  // [token][R / 2]
  const int R = a.rotary_dim, half = R / 2, tid = threadIdx.x, lane = tid & 63;
  const PageVisit pv = page_visit(a, in, P);
  apply_patches(a, in);
  const int n = pv.hi - pv.lo;  // tokens
  for (int i = tid; i < n * half; i += 256) {
    const int t = i / half, pair = i - t * half;
    cs[i] = cos_sin_turns(position(a, in, pv, t), a.freq[pair]);
  }
  __syncthreads();
  const int g0 = static_cast<int>(blockIdx.y) * sh.Hkv / a.parts, ng = (static_cast<int>(blockIdx.y) + 1) * sh.Hkv / a.parts - g0;
  const int nq = ng * sh.G, slots = pv.fill - pv.lo, n_q = a.q ? n * nq * U : 0, n_k = slots * ng * U;
  const int64_t tile0 = static_cast<int64_t>(pv.page) * sh.page_tiles + g0;
  constexpr int64_t kTileBytes = static_cast<int64_t>(P) * D * ESZ;
  constexpr int kHeadLanes = D / 2;  // values
  // Values of a few tokens behind others have no eight slots that can be written at once: a lane takes eight dims of a token.
  const bool few = !pv.is_new && n < 8;
  const int n_v = few ? n * ng * (D / 8) : ng * kHeadLanes, v_jobs = (n_v + 63) / 64, k_jobs = (n_k + 64 * N - 1) / (64 * N), q_jobs = (n_q + 127) / 128;
  for (int j = uniform(tid >> 6); j < v_jobs + k_jobs + q_jobs; j += 4) {
    if (j < v_jobs && few) {
      const int i = j * 64 + lane, r = i / (D / 8), t = r / ng, gi = r - t * ng, d = i % (D / 8) * 8;
      if (i >= n_v) continue;
      const Eight e = load_eight<false>(a.v, token_at(pv.tok0 + t, a.v_stride) + (g0 + gi) * D + d);
      const float inv = FP8 ? inverse_scale(a.v_scale[pv.page * sh.Hkv + g0 + gi]) : 1.f;
      char *tile = static_cast<char *>(a.v_pool) + (tile0 + gi) * kTileBytes;
      const u32x2 c = encode_eight(e, inv);
#pragma unroll
      for (int k = 0; k < 8; ++k) {
        const int at = v_offset<KV, kMfmaTiled>(pv.lo + t, d + k, D);
        if (FP8)
          tile[at] = static_cast<char>(c[k >> 2] >> (8 * (k & 3)));
        else
          reinterpret_cast<uint16_t *>(tile)[at] = static_cast<uint16_t>(__builtin_bit_cast(uint32_t, __builtin_amdgcn_cvt_pkrtz(e.x[k], 0.f)));
      }
    } else if (j < v_jobs) {
      // Values lie token-minor: a lane takes two dims of all tokens.
      const int gi = (j * 64 + lane) / kHeadLanes, d = lane % kHeadLanes * 2;
      if (gi >= ng) continue;
      const char *src = static_cast<const char *>(a.v) + 2 * (token_at(pv.tok0, a.v_stride) + (g0 + gi) * D + d);
      uint32_t w[P];
#pragma unroll
      for (int s = 0; s < P; ++s) {
        w[s] = 0;
        if (s >= pv.lo && s < pv.hi) w[s] = *reinterpret_cast<const uint32_t *>(src + 2 * token_at(s - pv.lo, a.v_stride));
      }
      float inv = 1.f;
      if (FP8) {
        const int at = pv.page * sh.Hkv + g0 + gi;
        float s;
        if (!pv.is_new) {
          s = a.v_scale[at];
        } else {
          if (a.v_scale_src) {
            s = a.v_scale_src[static_cast<int64_t>(pv.new_index) * sh.Hkv + g0 + gi];
          } else {
            float top = 0.f;
#pragma unroll
            for (int i = 0; i < P; ++i)
              top = fmaxf(top, fmaxf(__builtin_fabsf(bf16_bits_to_float(half_of(w[i], 0))), __builtin_fabsf(bf16_bits_to_float(half_of(w[i], 1)))));
#pragma unroll
            for (int o = kHeadLanes / 2; o >= 1; o >>= 1) top = fmaxf(top, __shfl_xor(top, o));
            s = page_scale(top);
          }
          if (d == 0) a.v_scale[at] = s;
        }
        inv = inverse_scale(s);
      }
      char *tile = static_cast<char *>(a.v_pool) + (tile0 + gi) * kTileBytes;
#pragma unroll
      for (int t0 = 0; t0 < P; t0 += 8) {
        if (t0 + 8 <= pv.lo || t0 >= pv.fill) continue;
        const bool whole = t0 >= pv.lo && t0 + 8 <= pv.fill;
#pragma unroll
        for (int k = 0; k < 2; ++k) {
          char *dst = tile + ESZ * v_offset<KV, kMfmaTiled>(t0, d + k, D);
          float x[8];
#pragma unroll
          for (int s = 0; s < 8; ++s) x[s] = bf16_bits_to_float(half_of(w[t0 + s], k));
          if (FP8) {
            const u32x2 c = {encode_four(x[0] * inv, x[1] * inv, x[2] * inv, x[3] * inv), encode_four(x[4] * inv, x[5] * inv, x[6] * inv, x[7] * inv)};
            if (whole) {
              *reinterpret_cast<u32x2 *>(dst) = c;
            } else {
#pragma unroll
              for (int s = 0; s < 8; ++s)
                if (t0 + s >= pv.lo && t0 + s < pv.fill) dst[s] = static_cast<char>(c[s >> 2] >> (8 * (s & 3)));
            }
          } else {
            u32x4 h;
#pragma unroll
            for (int s = 0; s < 4; ++s) h[s] = __builtin_bit_cast(uint32_t, __builtin_amdgcn_cvt_pkrtz(x[2 * s], x[2 * s + 1]));
            if (whole) {
              *reinterpret_cast<u32x4 *>(dst) = h;
            } else {
#pragma unroll
              for (int s = 0; s < 8; ++s)
                if (t0 + s >= pv.lo && t0 + s < pv.fill) *reinterpret_cast<uint16_t *>(dst + 2 * s) = static_cast<uint16_t>(h[s >> 1] >> (16 * (s & 1)));
            }
          }
        }
      }
    } else if (j < v_jobs + k_jobs) {
      // Keys.  Of a page the call starts a job has one head; four lanes beside each other have four tokens, which lie beside each
      // other in the tile.
      Unit<false, INTER> un[N];
      int t[N], gi[N];
#pragma unroll
      for (int k = 0; k < N; ++k) {
        const int i = ((j - v_jobs) * N + k) * 64 + lane;
        int u;
        if (pv.is_new) {
          gi[k] = j - v_jobs;
          t[k] = (k * 64 + lane) / (4 * U) * 4 + (lane & 3);
          u = lane / 4 % U;
        } else {
          const int r = i / U;
          u = i - r * U;
          gi[k] = r / slots;
          t[k] = r - gi[k] * slots;
        }
        un[k].place(u, D, R);
        un[k].clear();
        if (i >= n_k) gi[k] = -1;
        if (gi[k] >= 0 && t[k] < n) un[k].load(a.k, token_at(pv.tok0 + t[k], a.k_stride) + (g0 + gi[k]) * D);
      }
      float top = 0.f;
#pragma unroll
      for (int k = 0; k < N; ++k) {
        if (gi[k] < 0 || t[k] >= n) continue;
        un[k].turn(cs + t[k] * half);
        if (a.k_out) un[k].store(a.k_out, token_at(pv.tok0 + t[k], a.k_out_stride) + (g0 + gi[k]) * D);
        if (FP8) top = fmaxf(top, un[k].top());
      }
      float started = 1.f;
      if (FP8 && pv.is_new) {
        const int g = g0 + j - v_jobs;
        started = a.k_scale_src ? a.k_scale_src[static_cast<int64_t>(pv.new_index) * sh.Hkv + g] : page_scale(wave_max(top));
        if (lane == 0) a.k_scale[pv.page * sh.Hkv + g] = started;
        started = inverse_scale(started);
      }
#pragma unroll
      for (int k = 0; k < N; ++k) {
        if (gi[k] < 0) continue;
        float inv = started;
        if (FP8 && !pv.is_new) inv = inverse_scale(a.k_scale[pv.page * sh.Hkv + g0 + gi[k]]);
        char *tile = static_cast<char *>(a.k_pool) + (tile0 + gi[k]) * kTileBytes;
        put_eight<KV>(tile, k_offset<KV, kMfmaTiled>(pv.lo + t[k], un[k].d[0], D), un[k].e[0], inv);
        put_eight<KV>(tile, k_offset<KV, kMfmaTiled>(pv.lo + t[k], un[k].d[1], D), un[k].e[1], inv);
      }
    } else {
      Unit<false, INTER> un[2];
      int t[2], at[2];
#pragma unroll
      for (int k = 0; k < 2; ++k) {
        const int i = (j - v_jobs - k_jobs) * 128 + k * 64 + lane, r = i / U;
        t[k] = i < n_q ? r / nq : -1;
        at[k] = (g0 * sh.G + r - t[k] * nq) * D;
        un[k].place(i - r * U, D, R);
        if (t[k] >= 0) un[k].load(a.q, token_at(pv.tok0 + t[k], a.q_stride) + at[k]);
      }
#pragma unroll
      for (int k = 0; k < 2; ++k) {
        if (t[k] < 0) continue;
        un[k].turn(cs + t[k] * half);
        un[k].store(a.q_out, token_at(pv.tok0 + t[k], a.q_out_stride) + at[k]);
      }
    }
  }
}

// Row-major pools.
template <int KV, bool INTER>
__global__ __launch_bounds__(256) void spex_append_rotated_rows_kernel(RotateArgs a, Shape sh, RotateLists in) {
  constexpr bool F32 = KV == kF32, FP8 = KV == kFP8;
  constexpr int ESZ = F32 ? 4 : (FP8 ? 1 : 2);
  extern __shared__ __attribute__((aligned(16))) char lds_[];
  f32x2 *cs = reinterpret_cast<f32x2 *>(lds_);  // [token][R / 2]
  const int D = sh.D, P = sh.P, U = (D + 15) / 16, R = a.rotary_dim;
  const int tid = threadIdx.x, lane = tid & 63, wave = uniform(tid >> 6);
  const PageVisit pv = page_visit(a, in, P);
  apply_patches(a, in);
  const int n = pv.hi - pv.lo;  // tokens
  for (int i = tid; i < n * (R / 2); i += 256) {
    const int t = i / (R / 2), pair = i - t * (R / 2);
    cs[i] = cos_sin_turns(position(a, in, pv, t), a.freq[pair]);
  }
  __syncthreads();
  const int g0 = static_cast<int>(blockIdx.y) * sh.Hkv / a.parts, g1 = (static_cast<int>(blockIdx.y) + 1) * sh.Hkv / a.parts, ng = g1 - g0;
  Unit<F32, INTER> un;
  if (a.q) {
    const int nq = ng * sh.G;
    for (int i = tid; i < n * nq * U; i += 256) {
      const int r = i / U, t = r / nq, head = g0 * sh.G + r - t * nq;
      un.place(i - r * U, D, R);
      un.load(a.q, token_at(pv.tok0 + t, a.q_stride) + static_cast<int64_t>(head) * D);
      un.turn(cs + t * (R / 2));
      un.store(a.q_out, token_at(pv.tok0 + t, a.q_out_stride) + static_cast<int64_t>(head) * D);
    }
  }
  const int64_t tile0 = static_cast<int64_t>(pv.page) * sh.page_tiles, tile_bytes = static_cast<int64_t>(P) * D * ESZ;
  const int slots = pv.fill - pv.lo;
  // Keys.  fp8: a wavefront a kv head, because the page's scale comes from all of its tokens.
  const int first = FP8 ? lane : tid, step = FP8 ? 64 : 256;
  for (int gi = FP8 ? wave : 0; gi < (FP8 ? ng : 1); gi += FP8 ? 4 : 1) {
    const int heads = FP8 ? 1 : ng;
    float inv = 1.f;
    if (FP8) {
      const int g = g0 + gi;
      const int64_t at = static_cast<int64_t>(pv.page) * sh.Hkv + g;
      float s;
      if (!pv.is_new) {
        s = a.k_scale[at];
      } else if (a.k_scale_src) {
        s = a.k_scale_src[static_cast<int64_t>(pv.new_index) * sh.Hkv + g];
      } else {
        float top = 0.f;
        for (int i = lane; i < n * U; i += 64) {
          const int t = i / U;
          un.place(i - t * U, D, R);
          un.load(a.k, token_at(pv.tok0 + t, a.k_stride) + static_cast<int64_t>(g) * D);
          un.turn(cs + t * (R / 2));
          top = fmaxf(top, un.top());
        }
        s = page_scale(wave_max(top));
      }
      if (pv.is_new && lane == 0) a.k_scale[at] = s;
      inv = inverse_scale(s);
    }
    for (int i = first; i < slots * heads * U; i += step) {
      const int r = i / U, t = r / heads, g = g0 + (FP8 ? gi : r - t * heads);
      const int slot = pv.lo + t;
      un.place(i - r * U, D, R);
      if (t < n) {
        un.load(a.k, token_at(pv.tok0 + t, a.k_stride) + static_cast<int64_t>(g) * D);
        un.turn(cs + t * (R / 2));
        if (a.k_out) un.store(a.k_out, token_at(pv.tok0 + t, a.k_out_stride) + static_cast<int64_t>(g) * D);
      } else {
        un.clear();
      }
      char *tile = static_cast<char *>(a.k_pool) + (tile0 + g) * tile_bytes;
      put_eight<KV>(tile, k_offset<KV, kRowMajor>(slot, un.d[0], D), un.e[0], inv);
      if (un.two) put_eight<KV>(tile, k_offset<KV, kRowMajor>(slot, un.d[1], D), un.e[1], inv);
    }
  }
  // Values: as the keys, unturned.
  const int C = D / 8;
  for (int gi = FP8 ? wave : 0; gi < (FP8 ? ng : 1); gi += FP8 ? 4 : 1) {
    const int heads = FP8 ? 1 : ng;
    float inv = 1.f;
    if (FP8) {
      const int g = g0 + gi;
      const int64_t at = static_cast<int64_t>(pv.page) * sh.Hkv + g;
      float s;
      if (!pv.is_new) {
        s = a.v_scale[at];
      } else if (a.v_scale_src) {
        s = a.v_scale_src[static_cast<int64_t>(pv.new_index) * sh.Hkv + g];
      } else {
        float top = 0.f;
        for (int i = lane; i < n * C; i += 64)
          top = fmaxf(top, largest(load_eight<F32>(a.v, token_at(pv.tok0 + i / C, a.v_stride) + static_cast<int64_t>(g) * D + i % C * 8)));
        s = page_scale(wave_max(top));
      }
      if (pv.is_new && lane == 0) a.v_scale[at] = s;
      inv = inverse_scale(s);
    }
    for (int i = first; i < slots * heads * C; i += step) {
      const int r = i / C, t = r / heads, g = g0 + (FP8 ? gi : r - t * heads), d = (i - r * C) * 8;
      Eight e = {};
      if (t < n) e = load_eight<F32>(a.v, token_at(pv.tok0 + t, a.v_stride) + static_cast<int64_t>(g) * D + d);
      put_eight<KV>(static_cast<char *>(a.v_pool) + (tile0 + g) * tile_bytes, (pv.lo + t) * D + d, e, inv);
    }
  }
}

// Element by element: a workgroup per (page, kv head), with the query heads of the kv head; a thread turns whole pairs.
template <int KV, int LAYOUT>
__global__ __launch_bounds__(256) void spex_append_rotated_any_kernel(RotateArgs a, Shape sh, RotateLists in) {
  typedef typename std::conditional<KV == kF32, float, typename std::conditional<KV == kBF16, uint16_t, uint8_t>::type>::type T;
  typedef typename std::conditional<KV == kF32, float, uint16_t>::type S;
  constexpr bool FP8 = KV == kFP8;
  __shared__ float red[2][4];
  const int D = sh.D, P = sh.P, R = a.rotary_dim, half = R / 2, per = half + D - R;  // per: pairs and single dims of a row
  const int tid = threadIdx.x, g = blockIdx.y;
  const PageVisit pv = page_visit(a, in, P);
  apply_patches(a, in);
  const int n = pv.hi - pv.lo, slots = pv.fill - pv.lo;
  auto widen = [](S x) { return KV == kF32 ? static_cast<float>(x) : bf16_bits_to_float(static_cast<uint16_t>(x)); };
  auto narrow = [](float x) {
    if (KV == kF32) return static_cast<S>(x);
    return static_cast<S>(__builtin_bit_cast(uint16_t, static_cast<__bf16>(x)));
  };
  // Values and dims of element j of a row: a turned pair (j < half) or a dim behind the turned part (twice).
  struct Two {
    float x[2];
    int d[2];
  };
  auto element = [&](const void *base, int64_t row, int t, int j) {
    Two e;
    e.d[0] = j >= half ? R + j - half : (a.interleaved ? 2 * j : j);
    e.d[1] = j >= half ? e.d[0] : (a.interleaved ? 2 * j + 1 : j + half);
    e.x[0] = widen(static_cast<const S *>(base)[row + e.d[0]]);
    e.x[1] = widen(static_cast<const S *>(base)[row + e.d[1]]);
    if (j < half) {
      const f32x2 y = turned(e.x[0], e.x[1], cos_sin_turns(position(a, in, pv, t), a.freq[j]));
      e.x[0] = y[0];
      e.x[1] = y[1];
    }
    return e;
  };
  if (a.q)
    for (int i = tid; i < n * sh.G * per; i += 256) {
      const int t = i / per / sh.G, head = g * sh.G + i / per % sh.G;
      const Two e = element(a.q, (pv.tok0 + t) * a.q_stride + static_cast<int64_t>(head) * D, t, i % per);
      S *o = static_cast<S *>(a.q_out) + (pv.tok0 + t) * a.q_out_stride + static_cast<int64_t>(head) * D;
      o[e.d[0]] = narrow(e.x[0]);
      o[e.d[1]] = narrow(e.x[1]);
    }
  const int64_t tile = (static_cast<int64_t>(pv.page) * sh.page_tiles + g) * (static_cast<int64_t>(P) * D);
  T *kp = static_cast<T *>(a.k_pool) + tile, *vp = static_cast<T *>(a.v_pool) + tile;
  auto k_row = [&](int t) { return (pv.tok0 + t) * a.k_stride + static_cast<int64_t>(g) * D; };
  auto v_row = [&](int t) { return (pv.tok0 + t) * a.v_stride + static_cast<int64_t>(g) * D; };
  float kinv = 1.f, vinv = 1.f;
  if (FP8) {
    const int64_t at = static_cast<int64_t>(pv.page) * sh.Hkv + g;
    float ks, vs;
    if (!pv.is_new) {
      ks = a.k_scale[at];
      vs = a.v_scale[at];
    } else {
      if (a.k_scale_src) {
        ks = a.k_scale_src[static_cast<int64_t>(pv.new_index) * sh.Hkv + g];
        vs = a.v_scale_src[static_cast<int64_t>(pv.new_index) * sh.Hkv + g];
      } else {
        float ka = 0.f, va = 0.f;
        for (int i = tid; i < n * per; i += 256) {
          const Two e = element(a.k, k_row(i / per), i / per, i % per);
          ka = fmaxf(ka, fmaxf(__builtin_fabsf(e.x[0]), __builtin_fabsf(e.x[1])));
        }
        for (int i = tid; i < n * D; i += 256) va = fmaxf(va, __builtin_fabsf(widen(static_cast<const S *>(a.v)[v_row(i / D) + i % D])));
        ka = wave_max(ka);
        va = wave_max(va);
        if ((tid & 63) == 0) {
          red[0][tid >> 6] = ka;
          red[1][tid >> 6] = va;
        }
        __syncthreads();
        ks = page_scale(fmaxf(fmaxf(red[0][0], red[0][1]), fmaxf(red[0][2], red[0][3])));
        vs = page_scale(fmaxf(fmaxf(red[1][0], red[1][1]), fmaxf(red[1][2], red[1][3])));
      }
      if (tid == 0) {
        a.k_scale[at] = ks;
        a.v_scale[at] = vs;
      }
    }
    kinv = inverse_scale(ks);
    vinv = inverse_scale(vs);
    // k_out may be k: every thread has read the whole page's keys before one of them is replaced
    __syncthreads();
  }
  for (int i = tid; i < slots * per; i += 256) {
    const int t = i / per, slot = pv.lo + t;
    if (t < n) {
      const Two e = element(a.k, k_row(t), t, i % per);
      if (a.k_out) {
        S *o = static_cast<S *>(a.k_out) + (pv.tok0 + t) * a.k_out_stride + static_cast<int64_t>(g) * D;
        o[e.d[0]] = narrow(e.x[0]);
        o[e.d[1]] = narrow(e.x[1]);
      }
#pragma unroll
      for (int k = 0; k < 2; ++k)
        kp[k_offset<KV, LAYOUT>(slot, e.d[k], D)] = FP8 ? static_cast<T>(encode_e4m3(e.x[k] * kinv)) : static_cast<T>(narrow(e.x[k]));
    } else {
      const int j = i % per, d0 = j >= half ? R + j - half : j;
      kp[k_offset<KV, LAYOUT>(slot, d0, D)] = T(0);
      if (j < half) kp[k_offset<KV, LAYOUT>(slot, j + half, D)] = T(0);
    }
  }
  for (int i = tid; i < slots * D; i += 256) {
    const int t = i / D, d = i % D;
    T x = T(0);
    if (t < n) {
      const S s = static_cast<const S *>(a.v)[v_row(t) + d];
      if (FP8)
        x = static_cast<T>(encode_e4m3(widen(s) * vinv));
      else
        x = v_is_f16<KV, LAYOUT>() ? static_cast<T>(bf16_bits_to_f16_bits(static_cast<uint16_t>(s))) : static_cast<T>(s);
    }
    vp[v_offset<KV, LAYOUT>(pv.lo + t, d, D)] = x;
  }
}

}  // namespace

static bool aligned16(const void *x) { return (reinterpret_cast<uintptr_t>(x) & 15) == 0; }

// DT: head_dim of tiled pools, else 0.
template <int KV, int DT, bool INTER>
static void append_rotated_wide(const Shape &sh, const RotateArgs &a, const RotateLists &in, hipStream_t stream) {
  const dim3 grid(static_cast<unsigned>(a.n_recs), static_cast<unsigned>(a.parts)), block(256);
  const size_t lds = static_cast<size_t>(a.most_tokens) * (a.rotary_dim / 2) * sizeof(float) * 2;
  if constexpr (DT > 0)
    hipLaunchKernelGGL((spex_append_rotated_kernel<KV, DT, INTER>), grid, block, lds, stream, a, sh, in);
  else
    hipLaunchKernelGGL((spex_append_rotated_rows_kernel<KV, INTER>), grid, block, lds, stream, a, sh, in);
}
template <int KV, int DT>
static void append_rotated_wide(const Shape &sh, const RotateArgs &a, const RotateLists &in, hipStream_t stream) {
  if (a.interleaved)
    append_rotated_wide<KV, DT, true>(sh, a, in, stream);
  else
    append_rotated_wide<KV, DT, false>(sh, a, in, stream);
}

template <int KV>
static hipError_t append_rotated(const Shape &sh, const RotateArgs &args, const RotateLists &in, hipStream_t stream) {
  RotateArgs a = args;
  const bool tiled = sh.layout == kMfmaTiled;
  const int64_t per16 = KV == kF32 ? 4 : 8;
  bool wide = sh.D % 8 == 0 && a.rotary_dim % (a.interleaved ? 8 : 16) == 0;
  for (const void *x : {a.q, a.k, a.v, static_cast<const void *>(a.q_out), static_cast<const void *>(a.k_out),
                        static_cast<const void *>(a.k_pool), static_cast<const void *>(a.v_pool)})
    wide = wide && aligned16(x);
  for (int64_t s : {a.q_stride, a.k_stride, a.v_stride, a.q_out_stride, a.k_out_stride}) wide = wide && s % per16 == 0;
  if (!wide) {
    const dim3 grid(static_cast<unsigned>(a.n_recs), static_cast<unsigned>(sh.Hkv)), block(256);
    a.parts = sh.Hkv;
    if (tiled)
      hipLaunchKernelGGL((spex_append_rotated_any_kernel<KV, KV == kF32 ? kRowMajor : kMfmaTiled>), grid, block, 0, stream, a, sh, in);
    else
      hipLaunchKernelGGL((spex_append_rotated_any_kernel<KV, kRowMajor>), grid, block, 0, stream, a, sh, in);
    return hipGetLastError();
  }
  // Pages few in number are shared by several workgroups, each with some kv heads, up to as many as the card holds at once (four
  // a CU).  16 tokens of 8 kv heads: 5.0 us against 7.7 with a workgroup a page; 512 pages of 6 tokens, fp8: 26.3 us with 1024
  // workgroups, 31.8 with 512, 30.4 with 2048, 35.2 with 4096.
  a.parts = static_cast<int32_t>(std::max<int64_t>(1, std::min<int64_t>(sh.Hkv, 1024 / a.n_recs)));
  if (KV != kF32 && tiled && sh.D == 64)
    append_rotated_wide<KV, KV == kF32 ? 0 : 64>(sh, a, in, stream);
  else if (KV != kF32 && tiled)
    append_rotated_wide<KV, KV == kF32 ? 0 : 128>(sh, a, in, stream);
  else
    append_rotated_wide<KV, 0>(sh, a, in, stream);
  return hipGetLastError();
}

hipError_t launch_append_rotated(const Shape &sh, const RotateArgs &a, const RotateLists &in, hipStream_t stream) {
  if (a.n_recs <= 0) return hipSuccess;
  switch (sh.kv_dtype) {
    case kF32: return append_rotated<kF32>(sh, a, in, stream);
    case kBF16: return append_rotated<kBF16>(sh, a, in, stream);
    case kFP8: return append_rotated<kFP8>(sh, a, in, stream);
    case kMXFP4: return launch_mxfp4_append(sh, a, in, stream);
  }
  return hipErrorInvalidValue;
}

}  // namespace spex
