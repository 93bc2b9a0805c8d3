// HIP kernels for causal attention over packed prompts on gfx950 (CDNA4, 64-lane wavefronts).
//
//   spex_prompt_bf16_kernel
//       One workgroup takes NW sets of 32 query rows of one kv head, a wavefront each: the pair (block of 32
//       tokens, query head) number i of a prompt goes to wavefront i mod NW of work item i / NW, so that all
//       wavefronts share the K and V tiles they stage in LDS, however many query heads a kv head has.
//   spex_prompt_f32_kernel
//       The same with the fp32 MFMA.
//   spex_prompt_generic_kernel
//       Same contract without matrix cores, for rows that are not made of 16-byte pieces.
//
// Mathematics: one pass over the keys with the running maximum m and sum l of a softmax,
//   S^T = K Q^T,  p = 2^(S^T scale log2(e) - m),  l += sum p,  O^T += V^T P^T,  out = O / l.
// With the scores transposed a lane holds scores of one query row only (column lane % 32 of the MFMA result), so m and l
// are one register each, and the weights of 16 keys are, as they lie, the B operand of the PV product for the
// key order {8 j + 4 (lane / 32) + i}: V is read from LDS in that order by the transposing load.
#include "prompt.hpp"

#include <climits>

namespace spex {
namespace {

typedef __bf16 bf16x8 __attribute__((ext_vector_type(8)));
typedef __bf16 bf16x2 __attribute__((ext_vector_type(2)));
typedef short s16x4 __attribute__((ext_vector_type(4)));
typedef float f32x2 __attribute__((ext_vector_type(2)));
typedef float f32x4 __attribute__((ext_vector_type(4)));
typedef float f32x16 __attribute__((ext_vector_type(16)));
typedef uint32_t u32x2 __attribute__((ext_vector_type(2)));
typedef uint32_t u32x4 __attribute__((ext_vector_type(4)));
typedef __attribute__((address_space(3))) char lds_char;
typedef __attribute__((address_space(3))) s16x4 lds_s16x4;
typedef __attribute__((address_space(3))) u32x4 lds_u32x4;
typedef __attribute__((address_space(3))) u32x2 lds_u32x2;
typedef __attribute__((address_space(3))) float lds_float;

// Start value of the running maximum: finite, and below any score that the rows can have.
constexpr float kMInit = -1.0e30f;
// A row's reference m stays while its scores are below m + 8: weights reach 2^8, sums stay far inside fp32, and the
// accumulators are rescaled a few times a row instead of once a tile.
constexpr float kSlack = 8.0f;

__device__ __forceinline__ int uniform(int v) { return __builtin_amdgcn_readfirstlane(v); }
__device__ __forceinline__ float fast_exp2(float x) { return __builtin_amdgcn_exp2f(x); }

// The value of lane l ^ 32.
__device__ __forceinline__ float other_half(float v) {
  const u32x2 r = __builtin_amdgcn_permlane32_swap(__builtin_bit_cast(uint32_t, v), __builtin_bit_cast(uint32_t, v), false, false);
  return __builtin_bit_cast(float, (threadIdx.x & 32) ? r[0] : r[1]);
}

__device__ __forceinline__ uint32_t pack_bf16(float a, float b) {
  return __builtin_bit_cast(uint32_t, bf16x2{static_cast<__bf16>(a), static_cast<__bf16>(b)});
}

// What a wavefront works on.
struct RowSet {
  int head;      // query head
  int q0;        // first token of its 32, within the prompt
  int len;       // tokens of the prompt
  int64_t row0;  // the prompt's first token among all
  int kv;        // kv head
  int last;      // last token any wavefront of the workgroup has (none: -1)
  bool live;
};
// Items run from a prompt's last tokens to its first: those with most keys start first.
template <int NW>
__device__ __forceinline__ RowSet row_set(const PromptArgs &p, int wave) {
  RowSet r;
  r.kv = static_cast<int>(blockIdx.x) % p.Hkv;
  const int item = static_cast<int>(blockIdx.x) / p.Hkv, lane = threadIdx.x & 63;
  int idx = -1;
#pragma unroll
  for (int i = 0; i < kMaxPromptsPerLaunch; i += 64) idx += __builtin_popcountll(__ballot(p.first[i + lane] <= item));
  r.len = p.len[idx];
  r.row0 = p.start[idx];
  const int blocks = (r.len + kPromptRows - 1) / kPromptRows, pairs = blocks * p.G;
  const int group = (pairs + NW - 1) / NW - 1 - (item - p.first[idx]);
  const int pair = group * NW + wave;
  r.live = pair < pairs;
  r.q0 = pair / p.G * kPromptRows;
  r.head = r.kv * p.G + pair % p.G;
  const int most = min(group * NW + NW - 1, pairs - 1) / p.G;
  r.last = min(most * kPromptRows + kPromptRows, r.len) - 1;
  return r;
}

// 16 bytes a lane from memory to LDS, to lds + 16 * lane.  In assembly, because the compiler lets every transposing read wait for
// all such copies under way, those into the other buffers too; tile_barrier() is what waits for them.  (The compiler keeps nothing
// in m0 between instructions of its own.)
__device__ __forceinline__ void copy_to_lds(const u32x4 rows, int lane_off, int off, lds_char *lds) {
  asm volatile("s_mov_b32 m0, %0\n\ts_nop 0\n\tbuffer_load_dwordx4 %1, %2, %3 offen lds" ::"s"(
                   uniform(static_cast<int>(reinterpret_cast<uintptr_t>(lds)))),
               "v"(lane_off), "s"(rows), "s"(off)
               : "memory");
}
// Behind it every wavefront's copies have landed, and none of them reads LDS of the step before.
__device__ __forceinline__ void tile_barrier() { asm volatile("s_waitcnt vmcnt(0) lgkmcnt(0)\n\ts_barrier" ::: "memory"); }

// ---- bf16 ----------------------------------------------------------------------------------------
// LDS tiles: 64 keys, rows of ROWB bytes (128, 256 or 512), 16-byte piece c of row t at place c ^ swz(t).  A K operand read
// has 32 rows at one piece, a V read four rows at two neighbouring pieces: with the bits of t in this order both
// spread over all banks.
template <int ROWB>
__device__ __forceinline__ int swz(int t) {
  if (ROWB == 128) return (((t >> 1) & 1) << 1) | (((t >> 2) & 1) << 2) | ((t >> 3) & 1);
  return ((t & 3) << 2) | (((t >> 2) & 1) << 1) | ((t >> 3) & 1);
}

template <int DP>
struct TileB {
  static constexpr int kKeys = 64;
  static constexpr int kRowB = DP <= 64 ? 128 : (DP <= 128 ? 256 : 512);
  static constexpr int kBytes = kKeys * kRowB;
};

// Copies tiles of KEYS tokens of one head, ROWB bytes a row in LDS, into LDS; Place::at(t, c) is where piece c of row t lies in its
// row.  Tokens past the prompt lie behind the end of the buffer and come out as zeros; pieces past the head repeat its last, which
// meet zeros of q or dims that are not stored.  A wavefront's rounds are a fixed number of rows apart, so that a lane's
// offsets are the same from tile to tile and the rest is scalar.
template <int KEYS, int ROWB, int NW, class Place>
struct Stager {
  static constexpr int PER = ROWB / 16, ROUNDS = KEYS * ROWB / 1024 / NW, STEP = NW * 64 / PER;  // STEP: rows a round
  static constexpr int KINDS = STEP >= 16 ? 1 : 16 / STEP;  // rounds whose pieces lie differently: places repeat every 16 rows
  static_assert(ROUNDS % KINDS == 0, "");
  uint64_t at;    // first row of the next tile
  int64_t left;   // bytes from there to the end of the prompt's last row
  int64_t tile_b; // bytes from tile to tile
  int step_b, off[KINDS];
  // base: first row
  __device__ __forceinline__ Stager(const char *base, int64_t stride_b, int len, int row_b, int wave, int lane)
      : at(reinterpret_cast<uint64_t>(base)), left((len - 1) * stride_b + row_b), tile_b(KEYS * stride_b), step_b(KINDS * STEP * static_cast<int>(stride_b)) {
#pragma unroll
    for (int k = 0; k < KINDS; ++k) {
      const int n = (k * NW + wave) * 64 + lane, row = n / PER;
      off[k] = row * static_cast<int>(stride_b) + min(Place::at(row, n % PER), row_b / 16 - 1) * 16;
    }
  }
  // The next tile; lds: of the wavefront's first round
  __device__ __forceinline__ void next(lds_char *lds) {
    const u32x4 rows = {static_cast<uint32_t>(at), static_cast<uint32_t>(at >> 32) & 0xffffu,
                        (left >> 31) != 0 ? 0x7fffffffu : static_cast<uint32_t>(left), 0x00020000u};
#pragma unroll
    for (int i = 0; i < ROUNDS; ++i) copy_to_lds(rows, off[i % KINDS], i / KINDS * step_b, lds + i * NW * 1024);
    at += tile_b;
    left -= tile_b;
  }
};
template <int ROWB>
struct PlaceB {
  static __device__ __forceinline__ int at(int t, int c) { return c ^ swz<ROWB>(t); }
};
struct PlaceF {
  static __device__ __forceinline__ int at(int t, int c) { return c ^ (t & 15); }
};

template <int DP, int NW>
__global__ __launch_bounds__(64 * NW, DP <= 128 ? 2 : 1) void spex_prompt_bf16_kernel(PromptArgs p) {
  constexpr int ROWB = TileB<DP>::kRowB, TILE = TileB<DP>::kBytes, KS = DP / 16, DT = DP / 32;
  __shared__ __attribute__((aligned(1024))) char lds_[4 * TILE];
  lds_char *lds = (lds_char *)lds_;
  const int lane = threadIdx.x & 63, wave = uniform(threadIdx.x >> 6), col = lane & 31, h = lane >> 5;
  const RowSet rs = row_set<NW>(p, wave);
  const int pieces = p.D / 8;
  Stager<64, ROWB, NW, PlaceB<ROWB>> ks(static_cast<const char *>(p.k) + (rs.row0 * p.k_stride + rs.kv * p.D) * 2, p.k_stride * 2, rs.len, p.D * 2, wave, lane);
  Stager<64, ROWB, NW, PlaceB<ROWB>> vs(static_cast<const char *>(p.v) + (rs.row0 * p.v_stride + rs.kv * p.D) * 2, p.v_stride * 2, rs.len, p.D * 2, wave, lane);
  const int tiles = rs.last / 64 + 1, mine = rs.live ? min(rs.q0 + kPromptRows - 1, rs.len - 1) / 64 + 1 : 0;
  lds_char *const mine_at = lds + wave * 1024;  // where this wavefront's copies into the first buffer go
  // Queries and results cross LDS, so that memory sees whole rows: as the operands lie a load or store has 32 or 16 bytes of
  // each of 32 rows.  Every wavefront has 32 rows of the buffer that is free then: a quarter of a tile of K and one of V.
  static_assert(NW == 4, "");
  auto rows_at = [&](int buffer) { return lds + ((wave >> 1) * 2 + buffer) * TILE + (wave & 1) * (TILE / 2); };
  const int64_t row = rs.row0 + rs.q0, head0 = static_cast<int64_t>(rs.live ? rs.head : 0) * p.D;
  if (rs.live) {
    Stager<32, ROWB, 1, PlaceB<ROWB>> qs(static_cast<const char *>(p.q) + (row * p.q_stride + head0) * 2, p.q_stride * 2, rs.len - rs.q0, p.D * 2, 0, lane);
    qs.next(rows_at(1));
  }
  ks.next(mine_at);
  vs.next(mine_at + 2 * TILE);
  // Places of the operand pieces in a tile; the other keys of the tile lie at constant distances.
  int koff[KS], voff[DT][2];
#pragma unroll
  for (int s = 0; s < KS; ++s) koff[s] = col * ROWB + ((2 * s + h) ^ swz<ROWB>(col)) * 16;
#pragma unroll
  for (int dt = 0; dt < DT; ++dt)
#pragma unroll
    for (int j = 0; j < 2; ++j) {
      const int t = 8 * j + 4 * h + ((lane & 15) >> 2), c = 4 * dt + 2 * ((lane >> 4) & 1) + ((lane & 3) >> 1);
      voff[dt][j] = t * ROWB + (c ^ swz<ROWB>(t)) * 16 + (lane & 1) * 8;
    }
  bf16x8 qf[KS];
  asm volatile("s_waitcnt vmcnt(%0)" ::"n"(2 * TILE / 1024 / NW) : "memory");  // the copies of K and V are younger
  {
    const lds_char *rows = rows_at(1);
#pragma unroll
    for (int s = 0; s < KS; ++s) {
      u32x4 x = *(const lds_u32x4 *)(rows + koff[s]);
      if (2 * s + h >= pieces) x = u32x4{0, 0, 0, 0};
      qf[s] = __builtin_bit_cast(bf16x8, x);
    }
  }
  f32x16 o[DT];
#pragma unroll
  for (int dt = 0; dt < DT; ++dt)
#pragma unroll
    for (int r = 0; r < 16; ++r) o[dt][r] = 0.f;
  float m = kMInit, l = 0.f, limit = -__builtin_huge_valf();  // limit: scores up to here need no other reference point
  const float inv_scale = 1.0f / p.scale_log2;
  const int qpos = rs.q0 + col;

  for (int t = 0; t < tiles; ++t) {
    tile_barrier();
    lds_char *kt = lds + (t & 1) * TILE, *vt = lds + (2 + (t & 1)) * TILE;
    if (t + 1 < tiles) {
      lds_char *to = mine_at + (~t & 1) * TILE;
      ks.next(to);
      vs.next(to + 2 * TILE);
    }
    if (t >= mine) continue;
    f32x16 s[2];
#pragma unroll
    for (int kt2 = 0; kt2 < 2; ++kt2) {
#pragma unroll
      for (int r = 0; r < 16; ++r) s[kt2][r] = 0.f;
#pragma unroll
      for (int i = 0; i < KS; ++i) {
        const bf16x8 kf = __builtin_bit_cast(bf16x8, *(const lds_u32x4 *)(kt + koff[i] + kt2 * 32 * ROWB));
        s[kt2] = __builtin_amdgcn_mfma_f32_32x32x16_bf16(kf, qf[i], s[kt2], 0, 0, 0);
      }
    }
    if (t * 64 + 63 > rs.q0) {
#pragma unroll
      for (int kt2 = 0; kt2 < 2; ++kt2)
#pragma unroll
        for (int r = 0; r < 16; ++r)
          if (t * 64 + kt2 * 32 + 8 * (r / 4) + 4 * h + r % 4 > qpos) s[kt2][r] = -__builtin_huge_valf();
    }
    float mx = s[0][0];
#pragma unroll
    for (int r = 1; r < 32; ++r) mx = fmaxf(mx, s[r / 16][r % 16]);
    if (__any(mx > limit)) {
      const float mn = fmaxf(m, fmaxf(mx, other_half(mx)) * p.scale_log2), f = fast_exp2(m - mn);
      m = mn;
      limit = (m + kSlack) * inv_scale;
      l *= f;
#pragma unroll
      for (int dt = 0; dt < DT; ++dt)
#pragma unroll
        for (int r = 0; r < 16; ++r) o[dt][r] *= f;
    }
    uint32_t pw[16];
#pragma unroll
    for (int r = 0; r < 32; r += 2) {
      const float a = fast_exp2(__builtin_fmaf(s[r / 16][r % 16], p.scale_log2, -m));
      const float b = fast_exp2(__builtin_fmaf(s[r / 16][r % 16 + 1], p.scale_log2, -m));
      l += a + b;
      pw[r / 2] = pack_bf16(a, b);
    }
#pragma unroll
    for (int sl = 0; sl < 4; ++sl) {
      const bf16x8 pf = __builtin_bit_cast(bf16x8, u32x4{pw[4 * sl], pw[4 * sl + 1], pw[4 * sl + 2], pw[4 * sl + 3]});
#pragma unroll
      for (int dt = 0; dt < DT; ++dt) {
        const s16x4 v0 = __builtin_amdgcn_ds_read_tr16_b64_v4i16((lds_s16x4 *)(vt + voff[dt][0] + sl * 16 * ROWB));
        const s16x4 v1 = __builtin_amdgcn_ds_read_tr16_b64_v4i16((lds_s16x4 *)(vt + voff[dt][1] + sl * 16 * ROWB));
        const u32x2 a0 = __builtin_bit_cast(u32x2, v0), a1 = __builtin_bit_cast(u32x2, v1);
        o[dt] = __builtin_amdgcn_mfma_f32_32x32x16_bf16(__builtin_bit_cast(bf16x8, u32x4{a0[0], a0[1], a1[0], a1[1]}), pf, o[dt], 0, 0, 0);
      }
    }
  }
  if (!rs.live) return;
  l += other_half(l);
  const float inv = 1.0f / l;
  lds_char *rows = rows_at(tiles & 1);  // the last tile lies in the others
#pragma unroll
  for (int dt = 0; dt < DT; ++dt)
#pragma unroll
    for (int j = 0; j < 4; ++j)
      *(lds_u32x2 *)(rows + col * ROWB + ((4 * dt + j) ^ swz<ROWB>(col)) * 16 + 8 * h) =
          u32x2{pack_bf16(o[dt][4 * j] * inv, o[dt][4 * j + 1] * inv), pack_bf16(o[dt][4 * j + 2] * inv, o[dt][4 * j + 3] * inv)};
  constexpr int PER = ROWB / 16;
  char *out = static_cast<char *>(p.out) + (row * p.out_stride + head0) * 2;
#pragma unroll
  for (int i = 0; i < 32 * PER / 64; ++i) {
    const int r = (i * 64 + lane) / PER, c = lane % PER;
    const u32x4 x = *(const lds_u32x4 *)(rows + r * ROWB + (c ^ swz<ROWB>(r)) * 16);
    if (rs.q0 + r < rs.len && c < pieces) *reinterpret_cast<u32x4 *>(out + r * p.out_stride * 2 + c * 16) = x;
  }
  if (p.lse && h == 0 && qpos < rs.len)
    p.lse[(row + col) * (static_cast<int64_t>(p.Hkv) * p.G) + rs.head] = (m + __builtin_log2f(l)) * 0.6931471805599453f;
}

// ---- fp32 ----------------------------------------------------------------------------------------
// Tiles of 32 keys; piece c (four dims) of row t at place c ^ (t & 15).
template <int DP, int NW>
__global__ __launch_bounds__(64 * NW, DP <= 128 ? 2 : 1) void spex_prompt_f32_kernel(PromptArgs p) {
  constexpr int ROWB = DP * 4, TILE = 32 * ROWB, KS = DP / 8, DT = DP / 32;
  __shared__ __attribute__((aligned(1024))) char lds_[4 * TILE];
  lds_char *lds = (lds_char *)lds_;
  const int lane = threadIdx.x & 63, wave = uniform(threadIdx.x >> 6), col = lane & 31, h = lane >> 5;
  const RowSet rs = row_set<NW>(p, wave);
  const int pieces = p.D / 4;
  Stager<32, ROWB, NW, PlaceF> ks(static_cast<const char *>(p.k) + (rs.row0 * p.k_stride + rs.kv * p.D) * 4, p.k_stride * 4, rs.len, p.D * 4, wave, lane);
  Stager<32, ROWB, NW, PlaceF> vs(static_cast<const char *>(p.v) + (rs.row0 * p.v_stride + rs.kv * p.D) * 4, p.v_stride * 4, rs.len, p.D * 4, wave, lane);
  const int tiles = rs.last / 32 + 1, mine = rs.live ? min(rs.q0 + kPromptRows - 1, rs.len - 1) / 32 + 1 : 0;
  lds_char *const mine_at = lds + wave * 1024;  // where this wavefront's copies into the first buffer go
  ks.next(mine_at);
  vs.next(mine_at + 2 * TILE);
  f32x4 qf[KS];
  {
    const char *qrow = static_cast<const char *>(p.q) +
                       ((rs.row0 + min(rs.q0 + col, rs.len - 1)) * p.q_stride + static_cast<int64_t>(rs.live ? rs.head : 0) * p.D) * 4;
#pragma unroll
    for (int s = 0; s < KS; ++s) {
      const int c = 2 * s + h;
      qf[s] = *reinterpret_cast<const f32x4 *>(qrow + min(c, pieces - 1) * 16);
      if (c >= pieces) qf[s] = f32x4{0.f, 0.f, 0.f, 0.f};
    }
  }
  // Place of dim col of key 4 h + i; keys 8 further and dims 32 further lie at constant distances.
  int voff[4];
#pragma unroll
  for (int i = 0; i < 4; ++i) voff[i] = (4 * h + i) * ROWB + ((col >> 2) ^ (4 * h + i)) * 16 + (col & 3) * 4;
  f32x16 o[DT];
#pragma unroll
  for (int dt = 0; dt < DT; ++dt)
#pragma unroll
    for (int r = 0; r < 16; ++r) o[dt][r] = 0.f;
  float m = kMInit, l = 0.f;
  const int qpos = rs.q0 + col;
  for (int t = 0; t < tiles; ++t) {
    tile_barrier();
    lds_char *kt = lds + (t & 1) * TILE, *vt = lds + (2 + (t & 1)) * TILE;
    if (t + 1 < tiles) {
      lds_char *to = mine_at + (~t & 1) * TILE;
      ks.next(to);
      vs.next(to + 2 * TILE);
    }
    if (t >= mine) continue;
    f32x16 s;
#pragma unroll
    for (int r = 0; r < 16; ++r) s[r] = 0.f;
#pragma unroll
    for (int i = 0; i < KS; ++i) {
      const f32x4 kf = __builtin_bit_cast(f32x4, *(const lds_u32x4 *)(kt + col * ROWB + ((2 * i + h) ^ (col & 15)) * 16));
#pragma unroll
      for (int e = 0; e < 4; ++e) s = __builtin_amdgcn_mfma_f32_32x32x2f32(kf[e], qf[i][e], s, 0, 0, 0);
    }
    if (t * 32 + 31 > rs.q0) {
#pragma unroll
      for (int r = 0; r < 16; ++r)
        if (t * 32 + 8 * (r / 4) + 4 * h + r % 4 > qpos) s[r] = -__builtin_huge_valf();
    }
    float mx = s[0];
#pragma unroll
    for (int r = 1; r < 16; ++r) mx = fmaxf(mx, s[r]);
    mx = fmaxf(mx, other_half(mx)) * p.scale_log2;
    if (__any(mx > m + kSlack)) {
      const float mn = fmaxf(m, mx), f = fast_exp2(m - mn);
      m = mn;
      l *= f;
#pragma unroll
      for (int dt = 0; dt < DT; ++dt)
#pragma unroll
        for (int r = 0; r < 16; ++r) o[dt][r] *= f;
    }
#pragma unroll
    for (int r = 0; r < 16; ++r) {
      s[r] = fast_exp2(__builtin_fmaf(s[r], p.scale_log2, -m));
      l += s[r];
    }
#pragma unroll
    for (int r = 0; r < 16; ++r) {
#pragma unroll
      for (int dt = 0; dt < DT; ++dt) {
        const float vf = *(const lds_float *)(vt + voff[r % 4] + r / 4 * 8 * ROWB + (dt ^ (r / 4 & 1)) * 128);
        o[dt] = __builtin_amdgcn_mfma_f32_32x32x2f32(vf, s[r], o[dt], 0, 0, 0);
      }
    }
  }
  if (!rs.live || qpos >= rs.len) return;
  l += other_half(l);
  const int64_t row = rs.row0 + qpos;
  const float inv = 1.0f / l;
  float *out = static_cast<float *>(p.out) + row * p.out_stride + static_cast<int64_t>(rs.head) * p.D;
#pragma unroll
  for (int dt = 0; dt < DT; ++dt)
#pragma unroll
    for (int j = 0; j < 4; ++j) {
      const int d = 32 * dt + 8 * j + 4 * h;
      if (d < p.D)
        *reinterpret_cast<f32x4 *>(out + d) = f32x4{o[dt][4 * j] * inv, o[dt][4 * j + 1] * inv, o[dt][4 * j + 2] * inv, o[dt][4 * j + 3] * inv};
    }
  if (p.lse && h == 0) p.lse[row * (static_cast<int64_t>(p.Hkv) * p.G) + rs.head] = (m + __builtin_log2f(l)) * 0.6931471805599453f;
}

// ---- any rows ------------------------------------------------------------------------------------
template <bool F32>
__device__ __forceinline__ float load(const void *p, int64_t i) {
  if (F32) return static_cast<const float *>(p)[i];
  return __builtin_bit_cast(float, static_cast<uint32_t>(static_cast<const uint16_t *>(p)[i]) << 16);
}

// One wavefront a query row: 64 keys at a time, a key a lane for the scores, dims lane, lane + 64, .. for the values.
template <bool F32>
__global__ __launch_bounds__(64) void spex_prompt_generic_kernel(PromptArgs p) {
  const RowSet rs = row_set<1>(p, 0);
  const int lane = threadIdx.x, D = p.D;
  for (int i = 0; i < kPromptRows; ++i) {
    const int qpos = rs.q0 + i;
    if (qpos >= rs.len) return;
    const int64_t q = (rs.row0 + qpos) * p.q_stride + static_cast<int64_t>(rs.head) * D, k = rs.row0 * p.k_stride + rs.kv * D,
                  v = rs.row0 * p.v_stride + rs.kv * D;
    float m = kMInit, l = 0.f, o[4] = {0.f, 0.f, 0.f, 0.f};
    for (int t0 = 0; t0 <= qpos; t0 += 64) {
      const int t = min(t0 + lane, qpos);
      float x = 0.f;
      for (int d = 0; d < D; ++d) x = __builtin_fmaf(load<F32>(p.q, q + d), load<F32>(p.k, k + t * p.k_stride + d), x);
      x = t0 + lane <= qpos ? x * p.scale_log2 : -__builtin_huge_valf();
      float mx = x;
#pragma unroll
      for (int w = 32; w >= 1; w >>= 1) mx = fmaxf(mx, __shfl_xor(mx, w));
      const float mn = fmaxf(m, mx), f = fast_exp2(m - mn), w = fast_exp2(x - mn);
      m = mn;
      l = l * f + w;
#pragma unroll
      for (int c = 0; c < 4; ++c) o[c] *= f;
      const int n = min(64, qpos + 1 - t0);
      for (int j = 0; j < n; ++j) {
        const float wj = __shfl(w, j);
#pragma unroll
        for (int c = 0; c < 4; ++c)
          if (lane + 64 * c < D) o[c] = __builtin_fmaf(wj, load<F32>(p.v, v + static_cast<int64_t>(t0 + j) * p.v_stride + lane + 64 * c), o[c]);
      }
    }
#pragma unroll
    for (int w = 32; w >= 1; w >>= 1) l += __shfl_xor(l, w);
    const int64_t row = rs.row0 + qpos, out = row * p.out_stride + static_cast<int64_t>(rs.head) * D;
#pragma unroll
    for (int c = 0; c < 4; ++c) {
      const int d = lane + 64 * c;
      if (d >= D) continue;
      if (F32)
        static_cast<float *>(p.out)[out + d] = o[c] / l;
      else
        static_cast<__bf16 *>(p.out)[out + d] = static_cast<__bf16>(o[c] / l);
    }
    if (p.lse && lane == 0) p.lse[row * (static_cast<int64_t>(p.Hkv) * p.G) + rs.head] = (m + __builtin_log2f(l)) * 0.6931471805599453f;
  }
}

constexpr int kWaves = 4;

}  // namespace

PromptKernel prompt_kernel(bool f32, bool wide) { return {f32, wide, wide ? kWaves : 1}; }

int64_t prompt_items(const PromptKernel &k, int32_t heads_per_kv, int32_t len) {
  const int64_t pairs = (static_cast<int64_t>(len) + kPromptRows - 1) / kPromptRows * heads_per_kv;
  return (pairs + k.waves - 1) / k.waves;
}

hipError_t launch_prompt(const PromptKernel &k, const PromptArgs &a, int64_t items, hipStream_t stream) {
  const dim3 grid(static_cast<unsigned>(items * a.Hkv));
  void (*kernel)(PromptArgs) = nullptr;
  if (!k.wide)
    kernel = k.f32 ? spex_prompt_generic_kernel<true> : spex_prompt_generic_kernel<false>;
  else if (k.f32)
    kernel = a.D <= 64 ? spex_prompt_f32_kernel<64, kWaves> : (a.D <= 128 ? spex_prompt_f32_kernel<128, kWaves> : spex_prompt_f32_kernel<256, kWaves>);
  else
    kernel = a.D <= 64 ? spex_prompt_bf16_kernel<64, kWaves>
                       : (a.D <= 96 ? spex_prompt_bf16_kernel<96, kWaves>
                                    : (a.D <= 128 ? spex_prompt_bf16_kernel<128, kWaves>
                                                  : (a.D <= 192 ? spex_prompt_bf16_kernel<192, kWaves> : spex_prompt_bf16_kernel<256, kWaves>)));
  hipLaunchKernelGGL(kernel, grid, dim3(static_cast<unsigned>(64 * k.waves)), 0, stream, a);
  return hipGetLastError();
}

}  // namespace spex
