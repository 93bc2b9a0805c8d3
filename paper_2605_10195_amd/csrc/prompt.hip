// HIP kernels for causal attention over packed prompts on gfx950 (CDNA4, 64-lane wavefronts).
//
//   spex_prompt_bf16_kernel
//       One workgroup takes NW sets of 32 query rows of one kv head, a wavefront each: the pair (block of 32
//       tokens, query head) number i of a prompt goes to wavefront i mod NW of work item i / NW, so that all
//       wavefronts share the K and V tiles they stage in LDS, however many query heads a kv head has.
//   spex_prompt_f32_kernel
//       The same with the fp32 MFMA.
//   spex_prompt_split_kernel
//       The same for launches of few rows: a workgroup takes one set of 32 rows, its wavefronts every NW-th 32 keys each,
//       and joins their states in the end.
//   spex_prompt_generic_kernel
//       Same contract without matrix cores, for rows that are not made of 16-byte pieces.
//
// Mathematics: one pass over the keys with the running maximum m and sum l of a softmax,
//   S^T = K Q^T,  p = 2^(S^T scale log2(e) - m),  l += sum p,  O^T += V^T P^T,  out = O / l.
// With the scores transposed a lane holds scores of one query row only (column lane % 32 of the MFMA result), so m and l
// are one register each, and the weights of 16 keys are, as they lie, the B operand of the PV product for the
// key order {8 j + 4 (lane / 32) + i}: V is read from LDS in that order by the transposing load.
// bf16: the weights are rounded to bf16, half a step of 2^-8 each, because the product with V takes its operands so; two parts of a weight
// would keep 16 bits and double that product's matrix instructions.  l sums them as they were before.
//
// Bound: the matrix cores, and with them power (at 1.0 PFLOP/s the clock falls from 2.4 to 1.75 GHz; on zeros the same launch is a
// third faster).  bf16, 8 prompts of 4096 tokens: D 64 0.82 PFLOP/s (the exponentials take a larger share), 96 0.87, 128 1.04, 192 1.0,
// 256 (4 prompts) 0.9; one of 16000, 32/8/128: 1.1; a bf16 matrix product of 16384 reaches 1.35.  Prompts below 1000 tokens are bound by
// the first loads and last stores of their workgroups: 64 of 128 .. 1024 tokens, 28/4/128: 294 us, 16 of 1024: 0.8 PFLOP/s.  fp32:
// 105 TFLOP/s at D 128 (matrix product: 154).  One prompt of a few hundred tokens: 10 us, launch and latency.
#include "prompt.hpp"

#include <climits>
#include <type_traits>

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

// Start value of the running maximum: finite, and far below any scaled score (+-1e30 log2(e)) that the rows can have.
constexpr float kMInit = -3.0e38f;
// A row's reference m stays while its scores are below m + 8: weights reach 2^8, sums stay far inside fp32, and the
// accumulators are rescaled a few times a row instead of once a tile.
constexpr float kSlack = 8.0f;

__device__ __forceinline__ int uniform(int v) { return __builtin_amdgcn_readfirstlane(v); }
__device__ __forceinline__ float fast_exp2(float x) { return __builtin_amdgcn_exp2f(x); }

// The reference point of a row: its weights are 2^((s - base) scale_log2 - m).  A row near zero has base 0, so that a weight is one fma and
// one exponential; the key that set m then has the weight 2^(what rounding the product to m left), not 1, which is of no account as long as that
// is a few units.  Rows whose |m| reaches kFar -- where fp32 holds no fractions, and from 2^31 on no unit below 128 -- have m 0
// and the score itself as base, subtracted from the scores of every tile before they are scaled.
constexpr float kFar = 16777216.0f;
struct Reference {
  float m = kMInit, base = 0.f;
  // Moves it up to `top`, the row's largest score of a tile (at least once before the first weight); the factor of the weights so far.
  __device__ __forceinline__ float move(float top, float scale) {
    const float ref = base != 0.f ? fmaxf(base, top) : top, scaled = ref * scale;
    const float mn = base != 0.f ? scaled : fmaxf(m, scaled);
    const bool far = __builtin_fabsf(mn) >= kFar;  // mn is then that of ref
    const float new_base = far ? ref : 0.f, new_m = far ? 0.f : mn;
    const float f = fast_exp2(__builtin_fmaf(base - new_base, scale, m - new_m));
    base = new_base;
    m = new_m;
    return f;
  }
  __device__ __forceinline__ bool far() const { return base != 0.f; }
  // In log2 units, rounded.
  __device__ __forceinline__ float value(float scale) const { return __builtin_fmaf(base, scale, m); }
};

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
// LDS tiles: rows of ROWB bytes (128, 256 or 512), 16-byte piece c of row t at place c ^ swz(t).  A K operand read
// has 32 rows at one piece, a V read four rows at two neighbouring pieces: with the bits of t in this order both
// spread over all banks.
template <int ROWB>
__device__ __forceinline__ int swz(int t) {
  if (ROWB == 128) return (((t >> 1) & 1) << 1) | (((t >> 2) & 1) << 2) | ((t >> 3) & 1);
  return ((t & 3) << 2) | (((t >> 2) & 1) << 1) | ((t >> 3) & 1);
}

template <int DP>
struct TileB {
  static constexpr int kRowB = DP <= 64 ? 128 : (DP <= 128 ? 256 : 512);
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
  // base: first row; tile number `first` comes first, then every `every`-th
  __device__ __forceinline__ Stager(const char *base, int64_t stride_b, int len, int row_b, int wave, int lane, int first = 0, int every = 1)
      : at(reinterpret_cast<uint64_t>(base) + first * (KEYS * stride_b)), left((len - 1 - first * KEYS) * stride_b + row_b),
        tile_b(every * (KEYS * stride_b)), step_b(KINDS * STEP * static_cast<int>(stride_b)) {
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

// KEYS: keys of a tile.  64 means half the barriers, 32 half the LDS: two workgroups then fit into a CU where a row has 512 bytes, three
// where it has 256.  Rows of 512 bytes always take 32: 8 prompts of 4096, 16/4/192: 1115 us with 64 keys, 825 with 32 (1.0
// PFLOP/s); 4 of 4096, 16/4/256: 850 and 611 (0.9).  The others: prompt_kernel.
template <int DP, int KEYS, int NW>
__global__ __launch_bounds__(64 * NW, 2) void spex_prompt_bf16_kernel(PromptArgs p) {
  constexpr int ROWB = TileB<DP>::kRowB, TILE = KEYS * ROWB, KS = DP / 16, DT = DP / 32, HALVES = KEYS / 32;
  __shared__ __attribute__((aligned(1024))) char lds_[4 * TILE];
  lds_char *lds = (lds_char *)lds_;
  const int lane = threadIdx.x & 63, wave = uniform(threadIdx.x >> 6), col = lane & 31, h = lane >> 5;
  const RowSet rs = row_set<NW>(p, wave);
  const int pieces = p.D / 8;
  Stager<KEYS, ROWB, NW, PlaceB<ROWB>> ks(static_cast<const char *>(p.k) + (rs.row0 * p.k_stride + rs.kv * p.D) * 2, p.k_stride * 2, rs.len, p.D * 2, wave, lane);
  Stager<KEYS, ROWB, NW, PlaceB<ROWB>> vs(static_cast<const char *>(p.v) + (rs.row0 * p.v_stride + rs.kv * p.D) * 2, p.v_stride * 2, rs.len, p.D * 2, wave, lane);
  const int tiles = rs.last / KEYS + 1, mine = rs.live ? min(rs.q0 + kPromptRows - 1, rs.len - 1) / KEYS + 1 : 0;
  lds_char *const mine_at = lds + wave * 1024;  // where this wavefront's copies into the first buffer go
  // Queries and results cross LDS, so that memory sees whole rows: as the operands lie a load or store has 32 or 16 bytes of
  // each of 32 rows.  Every wavefront has 32 rows of the buffer that is free then, half a tile; tiles of 32 keys leave no room beside a
  // buffer in use, so all of them are free at those times.
  static_assert(NW == 4, "");
  auto rows_at = [&](int buffer) { return HALVES == 2 ? lds + ((wave >> 1) * 2 + buffer) * TILE + (wave & 1) * (TILE / 2) : lds + wave * TILE; };
  const int64_t row = rs.row0 + rs.q0, head0 = static_cast<int64_t>(rs.live ? rs.head : 0) * p.D;
  if (rs.live) {
    Stager<32, ROWB, 1, PlaceB<ROWB>> qs(static_cast<const char *>(p.q) + (row * p.q_stride + head0) * 2, p.q_stride * 2, rs.len - rs.q0, p.D * 2, 0, lane);
    qs.next(rows_at(1));
  }
  if (HALVES == 2) {
    ks.next(mine_at);
    vs.next(mine_at + 2 * TILE);
  }
  // Places of the operand pieces in a tile; the other keys of the tile and the other half of a row of 512 bytes lie at constant
  // distances.
  constexpr int KO = KS < 8 ? KS : 8, VO = DT < 4 ? DT : 4;
  int koff[KO], voff[VO][2];
#pragma unroll
  for (int s = 0; s < KO; ++s) koff[s] = col * ROWB + ((2 * s + h) ^ swz<ROWB>(col)) * 16;
#pragma unroll
  for (int dt = 0; dt < VO; ++dt)
#pragma unroll
    for (int j = 0; j < 2; ++j) {
      const int t = 8 * j + 4 * h + ((lane & 15) >> 2), c = 4 * dt + 2 * ((lane >> 4) & 1) + ((lane & 3) >> 1);
      voff[dt][j] = t * ROWB + (c ^ swz<ROWB>(t)) * 16 + (lane & 1) * 8;
    }
  bf16x8 qf[KS];
  asm volatile("s_waitcnt vmcnt(%0)" ::"n"(HALVES == 2 ? 2 * TILE / 1024 / NW : 0) : "memory");  // the copies of K and V are younger
  {
    const lds_char *rows = rows_at(1);
#pragma unroll
    for (int s = 0; s < KS; ++s) {
      u32x4 x = *(const lds_u32x4 *)(rows + koff[s % KO] + s / KO * 256);
      if (2 * s + h >= pieces) x = u32x4{0, 0, 0, 0};
      qf[s] = __builtin_bit_cast(bf16x8, x);
    }
  }
  if (HALVES == 1) {
    tile_barrier();
    ks.next(mine_at);
    vs.next(mine_at + 2 * TILE);
  }
  f32x16 o[DT];
#pragma unroll
  for (int dt = 0; dt < DT; ++dt)
#pragma unroll
    for (int r = 0; r < 16; ++r) o[dt][r] = 0.f;
  Reference ref;
  float l = 0.f, limit = -__builtin_huge_valf();  // limit: scores up to here need no other reference point, of a far row none
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
    f32x16 s[HALVES];
#pragma unroll
    for (int kt2 = 0; kt2 < HALVES; ++kt2) {
#pragma unroll
      for (int r = 0; r < 16; ++r) s[kt2][r] = 0.f;
#pragma unroll
      for (int i = 0; i < KS; ++i) {
        const bf16x8 kf = __builtin_bit_cast(bf16x8, *(const lds_u32x4 *)(kt + koff[i % KO] + i / KO * 256 + kt2 * 32 * ROWB));
        s[kt2] = __builtin_amdgcn_mfma_f32_32x32x16_bf16(kf, qf[i], s[kt2], 0, 0, 0);
      }
    }
    if (t * KEYS + KEYS - 1 > rs.q0) {
#pragma unroll
      for (int kt2 = 0; kt2 < HALVES; ++kt2)
#pragma unroll
        for (int r = 0; r < 16; ++r)
          if (t * KEYS + kt2 * 32 + 8 * (r / 4) + 4 * h + r % 4 > qpos) s[kt2][r] = -__builtin_huge_valf();
    }
    float mx = s[0][0];
#pragma unroll
    for (int r = 1; r < KEYS / 2; ++r) mx = fmaxf(mx, s[r / 16][r % 16]);
    if (__any(mx > limit)) {
      const float f = ref.move(fmaxf(mx, other_half(mx)), p.scale_log2);
      limit = ref.far() ? -__builtin_huge_valf() : (ref.m + kSlack) * inv_scale;
      l *= f;
#pragma unroll
      for (int dt = 0; dt < DT; ++dt)
#pragma unroll
        for (int r = 0; r < 16; ++r) o[dt][r] *= f;
      if (__any(ref.far())) {
#pragma unroll
        for (int r = 0; r < KEYS / 2; ++r) s[r / 16][r % 16] -= ref.base;
      }
    }
    uint32_t pw[KEYS / 4];
#pragma unroll
    for (int r = 0; r < KEYS / 2; r += 2) {
      const float a = fast_exp2(__builtin_fmaf(s[r / 16][r % 16], p.scale_log2, -ref.m));
      const float b = fast_exp2(__builtin_fmaf(s[r / 16][r % 16 + 1], p.scale_log2, -ref.m));
      l += a + b;
      pw[r / 2] = pack_bf16(a, b);
    }
#pragma unroll
    for (int sl = 0; sl < KEYS / 16; ++sl) {
      const bf16x8 pf = __builtin_bit_cast(bf16x8, u32x4{pw[4 * sl], pw[4 * sl + 1], pw[4 * sl + 2], pw[4 * sl + 3]});
#pragma unroll
      for (int dt = 0; dt < DT; ++dt) {
        const s16x4 v0 = __builtin_amdgcn_ds_read_tr16_b64_v4i16((lds_s16x4 *)(vt + voff[dt % VO][0] + dt / VO * 256 + sl * 16 * ROWB));
        const s16x4 v1 = __builtin_amdgcn_ds_read_tr16_b64_v4i16((lds_s16x4 *)(vt + voff[dt % VO][1] + dt / VO * 256 + sl * 16 * ROWB));
        const u32x2 a0 = __builtin_bit_cast(u32x2, v0), a1 = __builtin_bit_cast(u32x2, v1);
        o[dt] = __builtin_amdgcn_mfma_f32_32x32x16_bf16(__builtin_bit_cast(bf16x8, u32x4{a0[0], a0[1], a1[0], a1[1]}), pf, o[dt], 0, 0, 0);
      }
    }
  }
  if (HALVES == 1) tile_barrier();
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
    p.lse[(row + col) * (static_cast<int64_t>(p.Hkv) * p.G) + rs.head] = (ref.value(p.scale_log2) + __builtin_log2f(l)) * 0.6931471805599453f;
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
  Reference ref;
  float l = 0.f;
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
    mx = fmaxf(mx, other_half(mx));
    if (__any(mx * p.scale_log2 > ref.m + kSlack || ref.far())) {
      const float f = ref.move(mx, p.scale_log2);
      l *= f;
#pragma unroll
      for (int dt = 0; dt < DT; ++dt)
#pragma unroll
        for (int r = 0; r < 16; ++r) o[dt][r] *= f;
      if (__any(ref.far())) {
#pragma unroll
        for (int r = 0; r < 16; ++r) s[r] -= ref.base;
      }
    }
#pragma unroll
    for (int r = 0; r < 16; ++r) {
      s[r] = fast_exp2(__builtin_fmaf(s[r], p.scale_log2, -ref.m));
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
  if (p.lse && h == 0) p.lse[row * (static_cast<int64_t>(p.Hkv) * p.G) + rs.head] = (ref.value(p.scale_log2) + __builtin_log2f(l)) * 0.6931471805599453f;
}

// ---- few rows ------------------------------------------------------------------------------------
// A workgroup takes 32 rows of one query head; wavefront w units w, w + NW, .. of 32 keys, which it copies into LDS of its own and
// waits for alone.  In the end the wavefronts' states go through LDS: with M the largest m of a row,
// l = sum_w l_w 2^(m_w - M), out = sum_w O_w 2^(m_w - M) / l.  Where M is far from zero the differences are those of the scores themselves.
// Rows far from zero are left to a second pass of the wavefront that met one: with references of both kinds in the first, one prompt
// of 512 tokens, 32/8/128, takes 11.6 us; so 11.2 (11.05 with none but ordinary rows).
// What bounds such launches is the way of the longest row set from launch to store; its keys are worked on NW at a time here.
template <bool F32, int DP, int NW>
__global__ __launch_bounds__(64 * NW, 2 * NW * 32 * (F32 ? DP * 4 : TileB<DP>::kRowB) <= 65536 ? 2 : 1) void spex_prompt_split_kernel(PromptArgs p) {
  constexpr int ESZ = F32 ? 4 : 2, ROWB = F32 ? DP * 4 : TileB<DP>::kRowB, UNIT = 32 * ROWB, DT = DP / 32;
  constexpr int KS = F32 ? DP / 8 : DP / 16;  // steps of 16 bytes a lane
  typedef typename std::conditional<F32, PlaceF, PlaceB<ROWB>>::type Place;
  constexpr int CP = UNIT / 1024;             // copies of a unit
  constexpr int PER = DP / 4;                 // pieces of four dims of a row of results
  static_assert(32 * DP * 4 <= 2 * UNIT, "a wavefront's results fit its own LDS");
  __shared__ __attribute__((aligned(1024))) char lds_[2 * NW * UNIT];
  __shared__ float ml[NW][3][32];  // a row's m (where it is far, only that and on which side), l and base
  const int lane = threadIdx.x & 63, wave = uniform(threadIdx.x >> 6), col = lane & 31, h = lane >> 5;
  lds_char *const kt = (lds_char *)lds_ + wave * (2 * UNIT), *const vt = kt + UNIT;
  const RowSet rs = row_set<1>(p, 0);
  const int units = rs.q0 / 32 + 1, pieces = p.D * ESZ / 16;
  const int64_t row = rs.row0 + rs.q0, head0 = static_cast<int64_t>(rs.head) * p.D, kv0 = static_cast<int64_t>(rs.kv) * p.D;
  const Stager<32, ROWB, 1, Place> first_k(static_cast<const char *>(p.k) + (rs.row0 * p.k_stride + kv0) * ESZ, p.k_stride * ESZ, rs.len, p.D * ESZ, 0, lane, wave, NW);
  const Stager<32, ROWB, 1, Place> first_v(static_cast<const char *>(p.v) + (rs.row0 * p.v_stride + kv0) * ESZ, p.v_stride * ESZ, rs.len, p.D * ESZ, 0, lane, wave, NW);
  // Places of the operand pieces, as in the other kernels.
  int koff[KS], voff[F32 ? 4 : 2 * DT];
#pragma unroll
  for (int s = 0; s < KS; ++s) koff[s] = col * ROWB + Place::at(col, 2 * s + h) * 16;
  if (F32) {
#pragma unroll
    for (int i = 0; i < 4; ++i) voff[i] = (4 * h + i) * ROWB + ((col >> 2) ^ (4 * h + i)) * 16 + (col & 3) * 4;
  } else {
#pragma unroll
    for (int i = 0; i < 2 * DT; ++i) {
      const int t = 8 * (i & 1) + 4 * h + ((lane & 15) >> 2), c = 4 * (i >> 1) + 2 * ((lane >> 4) & 1) + ((lane & 3) >> 1);
      voff[i] = t * ROWB + Place::at(t, c) * 16 + (lane & 1) * 8;
    }
  }
  f32x16 o[DT];
  Reference ref;
  float l = 0.f, farthest = 0.f;
  // Over the wavefront's units.  FAR: with references that may be far from zero; without, farthest tells where a row would have needed one.
  auto pass = [&](auto any_reference) __attribute__((always_inline)) {
    constexpr bool FAR = decltype(any_reference)::value;
    Stager<32, ROWB, 1, Place> ks = first_k, vs = first_v;
#pragma unroll
    for (int dt = 0; dt < DT; ++dt)
#pragma unroll
      for (int r = 0; r < 16; ++r) o[dt][r] = 0.f;
    ref = Reference();
    l = 0.f;
    // the queries by way of the room for values
    Stager<32, ROWB, 1, Place> qs(static_cast<const char *>(p.q) + (row * p.q_stride + head0) * ESZ, p.q_stride * ESZ, rs.len - rs.q0, p.D * ESZ, 0, lane);
    qs.next(vt);
    ks.next(kt);
    u32x4 qf[KS];
    asm volatile("s_waitcnt vmcnt(%0)" ::"n"(CP) : "memory");
#pragma unroll
    for (int s = 0; s < KS; ++s) {
      qf[s] = *(const lds_u32x4 *)(vt + koff[s]);
      if (2 * s + h >= pieces) qf[s] = u32x4{0, 0, 0, 0};
    }
    asm volatile("s_waitcnt lgkmcnt(0)" ::: "memory");
    vs.next(vt);
    for (int u = wave; u < units; u += NW) {
      asm volatile("s_waitcnt vmcnt(%0)" ::"n"(CP) : "memory");  // the keys have landed, the values may be under way
      f32x16 s;
#pragma unroll
      for (int r = 0; r < 16; ++r) s[r] = 0.f;
#pragma unroll
      for (int i = 0; i < KS; ++i) {
        const u32x4 kf = *(const lds_u32x4 *)(kt + koff[i]);
        if (F32) {
#pragma unroll
          for (int e = 0; e < 4; ++e)
            s = __builtin_amdgcn_mfma_f32_32x32x2f32(__builtin_bit_cast(f32x4, kf)[e], __builtin_bit_cast(f32x4, qf[i])[e], s, 0, 0, 0);
        } else {
          s = __builtin_amdgcn_mfma_f32_32x32x16_bf16(__builtin_bit_cast(bf16x8, kf), __builtin_bit_cast(bf16x8, qf[i]), s, 0, 0, 0);
        }
      }
      // No branch between the products and the first use of their results: the compiler has left out the wait states on the
      // shorter of two ways here.
      const bool more = u + NW < units;
      const int seen = u == units - 1 ? col - 4 * h : 32;  // keys behind a row's own token lie in the last unit
#pragma unroll
      for (int r = 0; r < 16; ++r)
        if (8 * (r / 4) + r % 4 > seen) s[r] = -__builtin_huge_valf();
      float mx = s[0];
#pragma unroll
      for (int r = 1; r < 16; ++r) mx = fmaxf(mx, s[r]);
      mx = fmaxf(mx, other_half(mx));
      asm volatile("s_waitcnt lgkmcnt(0)" ::: "memory");  // the keys have been read
      if (more) ks.next(kt);
      const float mn = fmaxf(ref.m, mx * p.scale_log2);
      if (!FAR) farthest = fmaxf(farthest, __builtin_fabsf(mn));
      if (FAR || __any(mn > ref.m)) {
        float f;
        if (FAR) {
          f = ref.move(mx, p.scale_log2);
#pragma unroll
          for (int r = 0; r < 16; ++r) s[r] -= ref.base;
        } else {
          f = fast_exp2(ref.m - mn);
          ref.m = mn;
        }
        l *= f;
#pragma unroll
        for (int dt = 0; dt < DT; ++dt)
#pragma unroll
          for (int r = 0; r < 16; ++r) o[dt][r] *= f;
      }
#pragma unroll
      for (int r = 0; r < 16; ++r) {
        s[r] = fast_exp2(__builtin_fmaf(s[r], p.scale_log2, -ref.m));
        l += s[r];
      }
      if (more)
        asm volatile("s_waitcnt vmcnt(%0)" ::"n"(CP) : "memory");
      else
        asm volatile("s_waitcnt vmcnt(0)" ::: "memory");
      if (F32) {
#pragma unroll
        for (int r = 0; r < 16; ++r)
#pragma unroll
          for (int dt = 0; dt < DT; ++dt)
            o[dt] = __builtin_amdgcn_mfma_f32_32x32x2f32(*(const lds_float *)(vt + voff[r % 4] + r / 4 * 8 * ROWB + (dt ^ (r / 4 & 1)) * 128), s[r], o[dt], 0, 0, 0);
      } else {
#pragma unroll
        for (int sl = 0; sl < 2; ++sl) {
          const bf16x8 pf = __builtin_bit_cast(bf16x8, u32x4{pack_bf16(s[8 * sl], s[8 * sl + 1]), pack_bf16(s[8 * sl + 2], s[8 * sl + 3]),
                                                             pack_bf16(s[8 * sl + 4], s[8 * sl + 5]), pack_bf16(s[8 * sl + 6], s[8 * sl + 7])});
#pragma unroll
          for (int dt = 0; dt < DT; ++dt) {
            const u32x2 a0 = __builtin_bit_cast(u32x2, __builtin_amdgcn_ds_read_tr16_b64_v4i16((lds_s16x4 *)(vt + voff[(2 * dt) % (F32 ? 4 : 2 * DT)] + sl * 16 * ROWB)));
            const u32x2 a1 = __builtin_bit_cast(u32x2, __builtin_amdgcn_ds_read_tr16_b64_v4i16((lds_s16x4 *)(vt + voff[(2 * dt + 1) % (F32 ? 4 : 2 * DT)] + sl * 16 * ROWB)));
            o[dt] = __builtin_amdgcn_mfma_f32_32x32x16_bf16(__builtin_bit_cast(bf16x8, u32x4{a0[0], a0[1], a1[0], a1[1]}), pf, o[dt], 0, 0, 0);
          }
        }
      }
      asm volatile("s_waitcnt lgkmcnt(0)" ::: "memory");  // the values have been read
      if (more) vs.next(vt);
    }
    l += other_half(l);
  };
  if (wave < units) {
    pass(std::false_type());
    if (__builtin_expect(__any(farthest >= kFar), 0)) pass(std::true_type());
  } else {
#pragma unroll
    for (int dt = 0; dt < DT; ++dt)
#pragma unroll
      for (int r = 0; r < 16; ++r) o[dt][r] = 0.f;
  }
  // Results into this wavefront's LDS: piece c of row r at place c ^ (r & 7), so that rows do not fall on the same banks.
  if (h == 0) {
    ml[wave][0][col] = ref.far() ? __builtin_copysignf(-kMInit / 16, ref.base) : ref.m;
    ml[wave][1][col] = l;
    ml[wave][2][col] = ref.base;
  }
#pragma unroll
  for (int dt = 0; dt < DT; ++dt)
#pragma unroll
    for (int j = 0; j < 4; ++j)
      *(__attribute__((address_space(3))) f32x4 *)(kt + col * (DP * 4) + ((8 * dt + 2 * j + h) ^ (col & 7)) * 16) =
          f32x4{o[dt][4 * j], o[dt][4 * j + 1], o[dt][4 * j + 2], o[dt][4 * j + 3]};
  __syncthreads();
  for (int i = threadIdx.x; i < 32 * PER; i += 64 * NW) {
    const int r = i / PER, c = i % PER, d = 4 * c;
    float top = kMInit;
#pragma unroll
    for (int w = 0; w < NW; ++w) top = fmaxf(top, ml[w][0][r]);
    float below[NW];
#pragma unroll
    for (int w = 0; w < NW; ++w) below[w] = ml[w][0][r] - top;
    const bool far = __builtin_fabsf(top) >= kFar - 256.0f;  // else far states lie below by so much that they count nothing
    if (__builtin_expect(__any(far), 0)) {
      if (far) {
        float base = -__FLT_MAX__;  // the largest
#pragma unroll
        for (int w = 0; w < NW; ++w)
          if (ml[w][2][r] != 0.f) base = fmaxf(base, ml[w][2][r]);
        const bool near = __builtin_fabsf(top) < kFar;
#pragma unroll
        for (int w = 0; w < NW; ++w) {
          const float b = ml[w][2][r], m = b != 0.f ? 0.f : ml[w][0][r];
          below[w] = near ? __builtin_fmaf(b, p.scale_log2, m - top) : __builtin_fmaf(b - base, p.scale_log2, m);
        }
        if (!near) top = base * p.scale_log2;
      }
    }
    float sum = 0.f;
    f32x4 x = {0.f, 0.f, 0.f, 0.f};
#pragma unroll
    for (int w = 0; w < NW; ++w) {
      const float f = fast_exp2(below[w]);
      sum += ml[w][1][r] * f;
      const f32x4 y = *(const __attribute__((address_space(3))) f32x4 *)((const lds_char *)lds_ + w * (2 * UNIT) + r * (DP * 4) + (c ^ (r & 7)) * 16);
#pragma unroll
      for (int e = 0; e < 4; ++e) x[e] += y[e] * f;
    }
    if (rs.q0 + r >= rs.len || d >= p.D) continue;
    const float inv = 1.0f / sum;
    char *out = static_cast<char *>(p.out) + ((row + r) * p.out_stride + head0 + d) * ESZ;
    if (F32)
      *reinterpret_cast<f32x4 *>(out) = f32x4{x[0] * inv, x[1] * inv, x[2] * inv, x[3] * inv};
    else
      *reinterpret_cast<u32x2 *>(out) = u32x2{pack_bf16(x[0] * inv, x[1] * inv), pack_bf16(x[2] * inv, x[3] * inv)};
    if (p.lse && c == 0) p.lse[(row + r) * (static_cast<int64_t>(p.Hkv) * p.G) + rs.head] = (top + __builtin_log2f(sum)) * 0.6931471805599453f;
  }
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
    float m = -__FLT_MAX__, l = 0.f, o[4] = {0.f, 0.f, 0.f, 0.f};  // m: as a score, not scaled
    for (int t0 = 0; t0 <= qpos; t0 += 64) {
      const int t = min(t0 + lane, qpos);
      float x = 0.f;
      for (int d = 0; d < D; ++d) x = __builtin_fmaf(load<F32>(p.q, q + d), load<F32>(p.k, k + t * p.k_stride + d), x);
      if (t0 + lane > qpos) x = -__builtin_huge_valf();
      float mx = x;
#pragma unroll
      for (int w = 32; w >= 1; w >>= 1) mx = fmaxf(mx, __shfl_xor(mx, w));
      const float mn = fmaxf(m, mx), f = fast_exp2((m - mn) * p.scale_log2), w = fast_exp2((x - mn) * p.scale_log2);
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
    if (p.lse && lane == 0) p.lse[row * (static_cast<int64_t>(p.Hkv) * p.G) + rs.head] = __builtin_fmaf(m, p.scale_log2, __builtin_log2f(l)) * 0.6931471805599453f;
  }
}

constexpr int kWaves = 4;

}  // namespace

PromptKernel prompt_kernel(bool f32, bool wide, int32_t D, int64_t row_sets, int32_t longest) {
  PromptKernel k{f32, wide, false, false, false, wide ? kWaves : 1};
  if (!wide || (f32 && D > 128)) return k;
  // Keys are split over the wavefronts of a workgroup where all row sets run at once that way (by LDS), or where the way of the
  // longest, in units of 32 keys, is shorter by enough: a workgroup has some other work as long as `fixed` units, and keys
  // and values are then not shared by four row sets.  us, whole / split; heads 32/8/128, one prompt of 1: 4.9 / 4.1, 256: 8.6 / 6.8,
  // 512 (512 row sets): 13.0 / 9.9, 768: 17.7 / 18.0, 1024: 22.2 / 23.1, 2048: 45.9 / 61.3; 8/2/128, 2048: 37.4 / 21.9, 4096 (1024):
  // 70.7 / 57.7, 8192: 164 / 194; 8 of 128, 32/8/128 (1024): 7.3 / 12.1; 16/2/64, 2048 (1024): 32.7 / 20.3; 16/4/256, 512 (256): 27.4 / 17.0,
  // 1024 (512): 49 / 34, 1500 (752): 68 / 65, 2048 (1024): 93 / 100, 16/4/192, 1500 (752): 44 / 54; fp32 8/2/64, 256: 23.1 / 9.1,
  // 32/8/128, 256 (256): 38.7 / 15.8, 512: 71.7 / 34.3, 32 of 64 (2048): 29 / 67.
  const int32_t row_b = f32 ? (D <= 64 ? 256 : 512) : (D <= 64 ? 128 : (D <= 128 ? 256 : 512));
  const int64_t at_once = 256 * (512 / row_b), rounds = (row_sets + at_once - 1) / at_once;
  const double units = (longest + 31) / 32, fixed = f32 ? 0.5 : 3.0, shared = f32 ? 1.3 : (D <= 128 ? 1.5 : 1.2);
  k.split = rounds <= 1 || shared * static_cast<double>(rounds) * (units / kWaves + fixed) < units;
  if (k.split) k.sets = 1;
  // Eight wavefronts where their LDS (128 KB where a row has 256 bytes) still holds all row sets at once and the longest has more units than
  // four of them take in one go, two of a bf16 head of more than 96 dims, where joining eight states costs more.  us, four / eight:
  // 8/2/128, 256: 6.3 / 6.5, 512: 8.4 / 7.9, 1024: 12.3 / 10.7; 4/2/96, 2048: 19.4 / 14.7; 16/2/64, 256: 5.0 / 4.7, 1024: 10.1 / 9.2; 4 of 200, 8/2/128:
  // 6.5 / 6.6; fp32 8/2/64, 160: 8.9 / 8.5, 256: 9.2 / 8.9, 1024: 25.3 / 22.8.
  k.eight = k.split && row_b <= 256 && row_sets <= 256 * (256 / row_b) && longest > (f32 || D <= 96 ? 1 : 2) * 32 * kWaves;
  // Heads of 97 to 128 dims, tiles of 64 / 32 keys: a third workgroup on a CU pays once there are some rounds of them, and a single
  // round is bound by the way of its longest.  us; 32/8/128, one prompt of 1024 (1024 row sets): 22.4 / 28.0, 2048:
  // 47.9 / 56.4, 4096 (4096): 150.6 / 149.7; 12/4/128, 12 of 200 .. 1500 (3288): 40.8 / 46.6; 16/4/128, 4 of 2000 (4032): 86.6 / 90.0; 40/8/128,
  // 4 of 900 (4640): 50.7 / 51.5; 28/4/128, 16 of 512 (7168): 52.9 / 51.9; 64 of 128 .. 1024 (32 thousand): 331 / 307; 64/8/128, 32 of 2048:
  // 2394 / 2302.  96 dims: 8 of 4096 alike, 12 of 200 .. 1500 34.2 / 40.3; 64 dims: 8 of 4096 345 / 354.
  k.short_tiles = !f32 && (D > 128 || (D > 96 && row_sets > 2 * (3 * 256 * kWaves)));
  return k;
}

int64_t prompt_items(const PromptKernel &k, int32_t heads_per_kv, int32_t len) {
  const int64_t pairs = (static_cast<int64_t>(len) + kPromptRows - 1) / kPromptRows * heads_per_kv;
  return (pairs + k.sets - 1) / k.sets;
}

template <int DP>
static void (*bf16_kernel(const PromptKernel &k))(PromptArgs) {
  if constexpr (DP <= 128)
    if (k.eight) return spex_prompt_split_kernel<false, DP, 2 * kWaves>;
  if (k.split) return spex_prompt_split_kernel<false, DP, kWaves>;
  if constexpr (DP >= 128)
    if (DP > 128 || k.short_tiles) return spex_prompt_bf16_kernel<DP, 32, kWaves>;
  if constexpr (DP <= 128) return spex_prompt_bf16_kernel<DP, 64, kWaves>;
}

hipError_t launch_prompt(const PromptKernel &k, const PromptArgs &a, int64_t items, hipStream_t stream) {
  const dim3 grid(static_cast<unsigned>(items * a.Hkv));
  void (*kernel)(PromptArgs) = nullptr;
  if (!k.wide)
    kernel = k.f32 ? spex_prompt_generic_kernel<true> : spex_prompt_generic_kernel<false>;
  else if (k.f32 && k.eight)
    kernel = spex_prompt_split_kernel<true, 64, 2 * kWaves>;
  else if (k.f32 && k.split)
    kernel = a.D <= 64 ? spex_prompt_split_kernel<true, 64, kWaves> : spex_prompt_split_kernel<true, 128, kWaves>;
  else if (k.f32)
    kernel = a.D <= 64 ? spex_prompt_f32_kernel<64, kWaves> : (a.D <= 128 ? spex_prompt_f32_kernel<128, kWaves> : spex_prompt_f32_kernel<256, kWaves>);
  else
    kernel = a.D <= 64 ? bf16_kernel<64>(k) : (a.D <= 96 ? bf16_kernel<96>(k) : (a.D <= 128 ? bf16_kernel<128>(k) : (a.D <= 192 ? bf16_kernel<192>(k) : bf16_kernel<256>(k))));
  hipLaunchKernelGGL(kernel, grid, dim3(k.wide ? (k.eight ? 128 * kWaves : 64 * kWaves) : 64), 0, stream, a);
  return hipGetLastError();
}

}  // namespace spex
