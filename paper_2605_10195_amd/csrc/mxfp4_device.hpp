// Tiles of a microscaled 4-bit (MXFP4) pool: where their codes and scales lie.  Device code shared by the kernels that write, read and
// attend over them.
//
// A tile holds 16 tokens of one kv head, D = 32 M dims: 8 D bytes of e2m1 codes, two dims to a byte with the even one in the low half,
// and behind them M x 16 bytes of exponents, [block of 32 dims][token], a byte e for the scale 2^(e - 127).  The codes lie in the order in
// which a wavefront consumes them, M 32-bit words a lane, so that a tile's keys (or values) are one load of a lane, each lane beside the next:
//   keys    the words of lane (g, t) = 16 g + t hold token t; word s is a chunk of 8 dims, the k-step s of the MFMA 16x16x32 S^T = K Q^T
//   values  the words of lane (g, c) = 16 g + c, g < 2, hold tokens 4 g .. 4 g + 3, a byte each, and behind them tokens 8 further on; word j
//           of either M is a pair of dims, columns c of the products O += P V number 2 j and 2 j + 1.  A block's exponents stand in the
//           same order: tokens 0 .. 3, 8 .. 11, 4 .. 7, 12 .. 15.
// Which chunk and which pair is free, because sums over dims may go in any order.  With M a power of two a lane's dims follow each
// other, chunk g M + s and pair c M + j, so that it needs one scale (M = 8 for keys: two); otherwise they are dealt so that word i
// belongs to block i, chunk 4 s + g and pair 16 j + c.
#pragma once

#include <hip/hip_runtime.h>

#include <cstdint>

namespace spex {
namespace {

template <int M>
constexpr bool kMxRun = (M & (M - 1)) == 0;  // a lane's dims follow each other
constexpr int mx_tile_bytes(int M) { return 272 * M; }
template <int M>
__device__ __forceinline__ constexpr int mx_key_scale_at(int block, int t) { return 256 * M + 16 * block + t; }
// Of tokens 4 tg .. 4 tg + 3, a word.
template <int M>
__device__ __forceinline__ constexpr int mx_value_scale_at(int block, int tg) { return 256 * M + 16 * block + 8 * (tg & 1) + 4 * (tg >> 1); }
// Byte offset of the word with chunk `chunk` of token t's key.
template <int M>
__device__ __forceinline__ int mx_key_at(int chunk, int t) {
  const int g = kMxRun<M> ? chunk / M : chunk & 3, s = kMxRun<M> ? chunk % M : chunk >> 2;
  return ((16 * g + t) * M + s) * 4;
}
// Byte offset of the word with dims 2 pair, 2 pair + 1 of the values of tokens 4 tg .. 4 tg + 3.
template <int M>
__device__ __forceinline__ int mx_value_at(int pair, int tg) {
  const int c = kMxRun<M> ? pair / M : pair & 15, j = kMxRun<M> ? pair % M : pair >> 4;
  return (((16 * (tg & 1) + c) * 2 + (tg >> 1)) * M + j) * 4;
}
// The first dim of chunk s of lane group g; of pair j of lane c.
template <int M>
__device__ __forceinline__ constexpr int mx_key_dim(int g, int s) { return kMxRun<M> ? 8 * (g * M + s) : 8 * (4 * s + g); }
template <int M>
__device__ __forceinline__ constexpr int mx_value_dim(int c, int j) { return kMxRun<M> ? 2 * (c * M + j) : 2 * (16 * j + c); }

// The scale of exponent byte i of a word, for the conversions that make numbers of codes: they read its exponent bits and none of the others
// (all codes and exponents compared on the device with the other bits set).
__device__ __forceinline__ float mx_scale(uint32_t e, int i = 0) { return __builtin_bit_cast(float, i < 3 ? e << (23 - 8 * i) : e >> 1); }

}  // namespace
}  // namespace spex
