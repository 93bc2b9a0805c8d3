// HIP kernels that write and read microscaled 4-bit (MXFP4) pools on gfx950.
//
//   spex_mxfp4_append_kernel
//       The appends: a workgroup per (page that the call writes to, range of kv heads).  Queries and keys are rotated by position
//       where a rotation is set and written back where wanted, keys and values quantised into the tiles.
//   spex_mxfp4_read_kernel
//       Tokens of many nodes as bf16 values, a workgroup per page and range of kv heads.
//
// Mathematics, per block of 32 dims of a token's key (rotated, in fp32) or value, with amax its largest magnitude:
//   E = floor(log2 amax) - 2, at least -126 and at most 125 (values: -23 and 13),
//   code = the e2m1 number (0, 0.5, 1, 1.5, 2, 3, 4, 6) nearest to x 2^-E, ties to the even code, at most 6 in magnitude.
// This is the conversion of the OCP microscaling formats.  E comes from amax's exponent bits, x 2^-E is exact, so the rounding to four
// bits is the only one.  The bounds of the values' E keep code * 2^E an IEEE half without rounding, as which attention multiplies it.
//
// Bound: memory.  8763 tokens of 8 prompts (32 / 8 heads of 128, rotated keys written back) are appended in 45 to 49 us, 207 MB, 88 to 96 % of
// a large copy's rate; 48000 tokens are read in 42 to 44, 249 MB, at more than that rate (the codes come out of the last-level cache).
// Steps of one token: latency, 4.7 us for 16 nodes, of it 1.6 an empty launch, and 12.9 for 1024, whose records come over the bus.
// Values are handled four tokens at a time, because a word of a tile holds four, keys by the token: their words do.
#include <algorithm>
#include <type_traits>

#include "kernels.hpp"
#include "mxfp4_device.hpp"
#include "rotate_device.hpp"

namespace spex {
namespace {

constexpr int kMinKeyE = -126, kMaxKeyE = 125, kMinValueE = -23, kMaxValueE = 13;
constexpr uint32_t kEmptyScale = 127;  // of slots without a token

__device__ __forceinline__ float element(const void *base, int64_t at) {
  return bf16_bits_to_float(static_cast<const uint16_t *>(base)[at]);
}
// Dims 8 chunk .. + 7 of a row, rotated.  A row lies in one wavefront, whose loads of all its dims come before its stores: out may be in.
// WIDE: rows, buffers and the rotated part's halves are made of 16-byte pieces, so that a chunk and its partner are one load each.
template <bool WIDE>
__device__ __forceinline__ Eight turned_chunk(const void *base, int64_t row, int chunk, int R, bool interleaved, const f32x2 *cs) {
  const int d0 = 8 * chunk, half = R / 2;
  Eight e;
  if (WIDE) {
    e = load_eight<false>(base, row + d0);
    if (d0 >= R) return e;
    if (interleaved) {
#pragma unroll
      for (int i = 0; i < 4; ++i) {
        const f32x2 y = turned(e.x[2 * i], e.x[2 * i + 1], cs[d0 / 2 + i]);
        e.x[2 * i] = y[0];
        e.x[2 * i + 1] = y[1];
      }
      return e;
    }
    const bool second = d0 >= half;
    const Eight o = load_eight<false>(base, row + (second ? d0 - half : d0 + half));
#pragma unroll
    for (int i = 0; i < 8; ++i) {
      const f32x2 y = turned(second ? o.x[i] : e.x[i], second ? e.x[i] : o.x[i], cs[(second ? d0 - half : d0) + i]);
      e.x[i] = second ? y[1] : y[0];
    }
    return e;
  }
  Eight o;
#pragma unroll
  for (int i = 0; i < 8; ++i) {
    const int d = d0 + i;
    e.x[i] = o.x[i] = element(base, row + d);
    if (d < R) o.x[i] = element(base, row + (interleaved ? d ^ 1 : (d < half ? d + half : d - half)));
  }
#pragma unroll
  for (int i = 0; i < 8; ++i) {
    const int d = d0 + i;
    if (d >= R) continue;
    const bool second = interleaved ? d & 1 : d >= half;
    const int pair = interleaved ? d >> 1 : (second ? d - half : d);
    const f32x2 y = turned(second ? o.x[i] : e.x[i], second ? e.x[i] : o.x[i], cs[pair]);
    e.x[i] = second ? y[1] : y[0];
  }
  return e;
}
template <bool WIDE>
__device__ __forceinline__ void store_chunk(void *base, int64_t at, const Eight &e) {
  if (WIDE) {
    store_eight<false>(base, at, e);
  } else {
#pragma unroll
    for (int i = 0; i < 8; ++i)
      static_cast<uint16_t *>(base)[at + i] = __builtin_bit_cast(uint16_t, static_cast<__bf16>(e.x[i]));
  }
}

// The exponent byte of a block whose four chunks lie in four neighbouring lanes, `top` the largest magnitude of the lane's own.
__device__ __forceinline__ uint32_t block_exponent(float top, int least, int most) {
  top = fmaxf(top, __shfl_xor(top, 1));
  top = fmaxf(top, __shfl_xor(top, 2));
  const int e = static_cast<int>(__builtin_bit_cast(uint32_t, top) >> 23) - 2;  // top >= 0: no sign; below the normal numbers: 0
  return static_cast<uint32_t>(min(max(e, least + 127), most + 127));
}
__device__ __forceinline__ uint32_t encode_chunk(const Eight &e, float scale) {
  uint32_t w = 0;
  w = __builtin_amdgcn_cvt_scalef32_pk_fp4_f32(w, e.x[0], e.x[1], scale, 0);
  w = __builtin_amdgcn_cvt_scalef32_pk_fp4_f32(w, e.x[2], e.x[3], scale, 1);
  w = __builtin_amdgcn_cvt_scalef32_pk_fp4_f32(w, e.x[4], e.x[5], scale, 2);
  return __builtin_amdgcn_cvt_scalef32_pk_fp4_f32(w, e.x[6], e.x[7], scale, 3);
}

// Byte b of r[j] = byte j of w[b].
__device__ __forceinline__ void transpose_bytes(const uint32_t (&w)[4], uint32_t (&r)[4]) {
  const uint32_t lo01 = __builtin_amdgcn_perm(w[1], w[0], 0x05010400u), hi01 = __builtin_amdgcn_perm(w[1], w[0], 0x07030602u);
  const uint32_t lo23 = __builtin_amdgcn_perm(w[3], w[2], 0x05010400u), hi23 = __builtin_amdgcn_perm(w[3], w[2], 0x07030602u);
  r[0] = __builtin_amdgcn_perm(lo23, lo01, 0x05040100u);
  r[1] = __builtin_amdgcn_perm(lo23, lo01, 0x07060302u);
  r[2] = __builtin_amdgcn_perm(hi23, hi01, 0x05040100u);
  r[3] = __builtin_amdgcn_perm(hi23, hi01, 0x07060302u);
}

template <int M, bool WIDE>
__global__ __launch_bounds__(256) void spex_mxfp4_append_kernel(RotateArgs a, Shape sh, RotateLists in) {
  constexpr int P = 16, D = 32 * M, C = 4 * M, RW = 64 / C;  // C: lanes a row; RW: rows of a wavefront's job
  extern __shared__ __attribute__((aligned(16))) char lds_[];
  f32x2 *cs = reinterpret_cast<f32x2 *>(lds_);  // [token][R / 2]
  const int R = a.rotary_dim, half = R / 2, tid = threadIdx.x, lane = tid & 63;
  const PageVisit pv = page_visit(a, in, P);
  apply_patches(a, in);
  const int n = pv.hi - pv.lo;  // tokens
  if (R > 0) {
    for (int i = tid; i < n * half; i += 256) {
      const int t = i / half, pair = i - t * half;
      cs[i] = cos_sin_turns(position(a, in, pv, t), a.freq[pair]);
    }
    __syncthreads();
  }
  const int g0 = static_cast<int>(blockIdx.y) * sh.Hkv / a.parts, ng = (static_cast<int>(blockIdx.y) + 1) * sh.Hkv / a.parts - g0;
  const int nq = ng * sh.G, slots = pv.fill - pv.lo, tg0 = pv.lo / 4, n_tg = (pv.fill + 3) / 4 - tg0;
  const int n_v = n_tg * ng, n_k = slots * ng, n_q = a.q ? n * nq : 0;
  const int v_jobs = (n_v + RW - 1) / RW, k_jobs = (n_k + RW - 1) / RW, q_jobs = (n_q + RW - 1) / RW;
  const int sub = lane / C, chunk = lane - sub * C;
  const int64_t tile0 = static_cast<int64_t>(pv.page) * sh.page_tiles + g0;
  for (int j = uniform(tid >> 6); j < v_jobs + k_jobs + q_jobs; j += 4) {
    if (j < v_jobs) {
      // Values: four tokens of eight dims a lane.
      const int i = j * RW + sub, gi = i / n_tg, tg = tg0 + i - gi * n_tg;
      const bool live = sub < RW && i < n_v;
      Eight e[4];
#pragma unroll
      for (int k = 0; k < 4; ++k) {
        const int s = 4 * tg + k;
        e[k] = Eight{};
        if (live && s >= pv.lo && s < pv.hi)
          e[k] = turned_chunk<WIDE>(a.v, token_at(pv.tok0 + s - pv.lo, a.v_stride) + (g0 + gi) * D, chunk, 0, false, cs);
      }
      uint32_t w[4], r[4], scales = 0;
#pragma unroll
      for (int k = 0; k < 4; ++k) {
        const int s = 4 * tg + k;
        uint32_t b = block_exponent(largest(e[k]), kMinValueE, kMaxValueE);
        w[k] = encode_chunk(e[k], mx_scale(b));
        if (s >= pv.hi) b = kEmptyScale;
        scales |= b << (8 * k);
      }
      if (!live) continue;
      transpose_bytes(w, r);
      char *tile = static_cast<char *>(a.v_pool) + (tile0 + gi) * mx_tile_bytes(M);
      const bool whole = 4 * tg >= pv.lo && 4 * tg + 4 <= pv.fill;
#pragma unroll
      for (int k = 0; k < 4; ++k) {
        char *dst = tile + mx_value_at<M>(4 * chunk + k, tg);
        if (whole) {
          *reinterpret_cast<uint32_t *>(dst) = r[k];
        } else {
#pragma unroll
          for (int b = 0; b < 4; ++b)
            if (4 * tg + b >= pv.lo && 4 * tg + b < pv.fill) dst[b] = static_cast<char>(r[k] >> (8 * b));
        }
      }
      if ((chunk & 3) == 0) {
        char *dst = tile + mx_value_scale_at<M>(chunk >> 2, tg);
        if (whole) {
          *reinterpret_cast<uint32_t *>(dst) = scales;
        } else {
#pragma unroll
          for (int b = 0; b < 4; ++b)
            if (4 * tg + b >= pv.lo && 4 * tg + b < pv.fill) dst[b] = static_cast<char>(scales >> (8 * b));
        }
      }
    } else if (j < v_jobs + k_jobs) {
      const int i = (j - v_jobs) * RW + sub, gi = i / slots, t = i - gi * slots;
      const bool live = sub < RW && i < n_k, token = live && t < n;
      Eight e = {};
      if (token) {
        e = turned_chunk<WIDE>(a.k, token_at(pv.tok0 + t, a.k_stride) + (g0 + gi) * D, chunk, R, a.interleaved, cs + t * half);
        if (a.k_out) store_chunk<WIDE>(a.k_out, token_at(pv.tok0 + t, a.k_out_stride) + (g0 + gi) * D + 8 * chunk, e);
      }
      const uint32_t b = block_exponent(largest(e), kMinKeyE, kMaxKeyE);
      if (!live) continue;
      char *tile = static_cast<char *>(a.k_pool) + (tile0 + gi) * mx_tile_bytes(M);
      *reinterpret_cast<uint32_t *>(tile + mx_key_at<M>(chunk, pv.lo + t)) = encode_chunk(e, mx_scale(b));
      if ((chunk & 3) == 0) tile[mx_key_scale_at<M>(chunk >> 2, pv.lo + t)] = static_cast<char>(token ? b : kEmptyScale);
    } else {
      const int i = (j - v_jobs - k_jobs) * RW + sub, t = i / nq, head = g0 * sh.G + i - t * nq;
      if (sub >= RW || i >= n_q) continue;
      const Eight e = turned_chunk<WIDE>(a.q, token_at(pv.tok0 + t, a.q_stride) + head * D, chunk, R, a.interleaved, cs + t * half);
      store_chunk<WIDE>(a.q_out, token_at(pv.tok0 + t, a.q_out_stride) + head * D + 8 * chunk, e);
    }
  }
}

// Eight values of a row.
template <bool WIDE>
__device__ __forceinline__ void put_values(void *base, int64_t at, uint32_t codes, float scale) {
  const u32x4 v = {__builtin_bit_cast(uint32_t, __builtin_amdgcn_cvt_scalef32_pk_bf16_fp4(codes, scale, 0)),
                   __builtin_bit_cast(uint32_t, __builtin_amdgcn_cvt_scalef32_pk_bf16_fp4(codes, scale, 1)),
                   __builtin_bit_cast(uint32_t, __builtin_amdgcn_cvt_scalef32_pk_bf16_fp4(codes, scale, 2)),
                   __builtin_bit_cast(uint32_t, __builtin_amdgcn_cvt_scalef32_pk_bf16_fp4(codes, scale, 3))};
  uint16_t *dst = static_cast<uint16_t *>(base) + at;
  if (WIDE) {
    *reinterpret_cast<u32x4 *>(dst) = v;
  } else {
#pragma unroll
    for (int i = 0; i < 8; ++i) dst[i] = half_word(v, i);
  }
}

// Records of kReadInts ints: page id, first slot | slot behind the last << 8, place of the first token in the output.
template <int M, bool WIDE>
__global__ __launch_bounds__(256) void spex_mxfp4_read_kernel(ReadBackArgs a, Shape sh, RotateLists in) {
  constexpr int D = 32 * M, C = 4 * M, RW = 64 / C;
  const int tid = threadIdx.x, lane = tid & 63, sub = lane / C, chunk = lane - sub * C;
  const int at = static_cast<int>(blockIdx.x) * kReadInts;
  int r[kReadInts];
  if (a.lists) {  // one access a wavefront
    const int x = a.lists[at + min(lane, kReadInts - 1)];
#pragma unroll
    for (int i = 0; i < kReadInts; ++i) r[i] = __builtin_amdgcn_readlane(x, i);
  } else {
#pragma unroll
    for (int i = 0; i < kReadInts; ++i) r[i] = uniform(in.ints[at + i]);
  }
  const int lo = r[1] & 0xff, hi = r[1] >> 8, n = hi - lo, tg0 = lo / 4, n_tg = (hi + 3) / 4 - tg0;
  const int g0 = static_cast<int>(blockIdx.y) * sh.Hkv / a.parts, ng = (static_cast<int>(blockIdx.y) + 1) * sh.Hkv / a.parts - g0;
  const int64_t tile0 = static_cast<int64_t>(r[0]) * sh.page_tiles + g0;
  const int n_v = n_tg * ng, n_k = n * ng, v_jobs = (n_v + RW - 1) / RW, k_jobs = (n_k + RW - 1) / RW;
  auto row_of = [&](int t, int gi) { return (static_cast<int64_t>(r[2] + t) * sh.Hkv + g0 + gi) * D + 8 * chunk; };
  if (sub >= RW) return;
  for (int j = uniform(tid >> 6); j < v_jobs + k_jobs; j += 4) {
    if (j < v_jobs) {
      const int i = j * RW + sub, gi = i / n_tg, tg = tg0 + i - gi * n_tg;
      if (i >= n_v) continue;
      const char *tile = static_cast<const char *>(a.v_pool) + (tile0 + gi) * mx_tile_bytes(M);
      uint32_t w[4], c[4];
#pragma unroll
      for (int k = 0; k < 4; ++k) w[k] = *reinterpret_cast<const uint32_t *>(tile + mx_value_at<M>(4 * chunk + k, tg));
      const uint32_t scales = *reinterpret_cast<const uint32_t *>(tile + mx_value_scale_at<M>(chunk >> 2, tg));
      transpose_bytes(w, c);
#pragma unroll
      for (int k = 0; k < 4; ++k) {
        const int s = 4 * tg + k;
        if (s < lo || s >= hi) continue;
        put_values<WIDE>(a.v_out, row_of(s - lo, gi), c[k], mx_scale(scales, k));
      }
    } else {
      const int i = (j - v_jobs) * RW + sub, t = i / ng, gi = i - t * ng;
      if (i >= n_k) continue;
      const char *tile = static_cast<const char *>(a.k_pool) + (tile0 + gi) * mx_tile_bytes(M);
      const uint32_t w = *reinterpret_cast<const uint32_t *>(tile + mx_key_at<M>(chunk, lo + t));
      put_values<WIDE>(a.k_out, row_of(t, gi), w, mx_scale(static_cast<uint8_t>(tile[mx_key_scale_at<M>(chunk >> 2, lo + t)])));
    }
  }
}

// Ranges of kv heads that a page's work is cut into.
int32_t parts_of(const Shape &sh, int32_t n_recs, int32_t workgroups) { return std::max(1, std::min(sh.Hkv, workgroups / n_recs)); }
bool aligned16(const void *x) { return (reinterpret_cast<uintptr_t>(x) & 15) == 0; }

// f(integral constant M)
template <class F>
hipError_t with_blocks(int head_dim, F f) {
  switch (head_dim) {
    case 32: f(std::integral_constant<int, 1>()); break;
    case 64: f(std::integral_constant<int, 2>()); break;
    case 96: f(std::integral_constant<int, 3>()); break;
    case 128: f(std::integral_constant<int, 4>()); break;
    case 160: f(std::integral_constant<int, 5>()); break;
    case 192: f(std::integral_constant<int, 6>()); break;
    case 224: f(std::integral_constant<int, 7>()); break;
    case 256: f(std::integral_constant<int, 8>()); break;
    default: return hipErrorInvalidValue;
  }
  return hipGetLastError();
}

}  // namespace

hipError_t launch_mxfp4_append(const Shape &sh, const RotateArgs &args, const RotateLists &in, hipStream_t stream) {
  if (args.n_recs <= 0) return hipSuccess;
  RotateArgs a = args;
  bool wide = a.rotary_dim % (a.interleaved ? 8 : 16) == 0;
  for (const void *x : {a.q, a.k, a.v, static_cast<const void *>(a.q_out), static_cast<const void *>(a.k_out)}) wide = wide && aligned16(x);
  for (int64_t s : {a.q_stride, a.k_stride, a.v_stride, a.q_out_stride, a.k_out_stride}) wide = wide && s % 8 == 0;
  // Workgroups wanted.  Pages of 16 tokens (550 of 8 heads) take 57.8 us in 1024, 48.0 in 2048, 51.7 in 4096; single tokens (1024 of 4
  // heads), where the record and the angles are most of a workgroup's time, 12.8 / 14.4 / 17.4.
  a.parts = parts_of(sh, a.n_recs, a.most_tokens > 4 ? 2048 : 1024);
  const dim3 grid(static_cast<unsigned>(a.n_recs), static_cast<unsigned>(a.parts)), block(256);
  const size_t lds = static_cast<size_t>(a.most_tokens) * (a.rotary_dim / 2) * sizeof(float) * 2;
  return with_blocks(sh.D, [&](auto m) {
    if (wide)
      hipLaunchKernelGGL((spex_mxfp4_append_kernel<decltype(m)::value, true>), grid, block, lds, stream, a, sh, in);
    else
      hipLaunchKernelGGL((spex_mxfp4_append_kernel<decltype(m)::value, false>), grid, block, lds, stream, a, sh, in);
  });
}

hipError_t launch_mxfp4_read(const Shape &sh, const ReadBackArgs &args, const RotateLists &in, hipStream_t stream) {
  if (args.n_recs <= 0) return hipSuccess;
  ReadBackArgs a = args;
  const bool wide = aligned16(a.k_out) && aligned16(a.v_out);
  // 550 pages of 8 heads of 128 take 10.5 us in 2048 workgroups, 12.8 in 1024, 11.2 in 4096; 1024 of 4 9.0 / 9.3 / 10.3.  Many pages
  // that are in no cache, us in one part / two: 8 heads of 128 79.1 / 72.0, 98.9 / 90.5, 75.6 / 67.0; 4 of 128 98.7 / 104.8, 4 of 96
  // 51.7 / 53.3, 2 of 128 58.2 / 66.2, 2 of 64 32.8 / 41.8.
  a.parts = std::max(sh.Hkv > 1 && sh.Hkv * sh.D >= 1024 ? 2 : 1, parts_of(sh, a.n_recs, 2048));
  const dim3 grid(static_cast<unsigned>(a.n_recs), static_cast<unsigned>(a.parts)), block(256);
  return with_blocks(sh.D, [&](auto m) {
    if (wide)
      hipLaunchKernelGGL((spex_mxfp4_read_kernel<decltype(m)::value, true>), grid, block, 0, stream, a, sh, in);
    else
      hipLaunchKernelGGL((spex_mxfp4_read_kernel<decltype(m)::value, false>), grid, block, 0, stream, a, sh, in);
  });
}

}  // namespace spex
