// decode.hip -- attention of one new token per sequence over bf16 or fp32 pages, for gfx950: the
// tiles of keys that decode_kernel.h's kernel works on.
//
// Four rollouts of 47 to 94 thousand tokens, 12 heads of 128, bf16 (1.66 GB): 247 us with the
// join, 6.7 TB/s, with plain instead of nontemporal loads 272; 48 sequences of 100 to 16,000 tokens,
// 40 query heads over 8 (617 MB): 101 us with the join, 6.1 TB/s.  With 64 instead of 32 tokens a
// unit the waves' loads differ more (5% for the 48 sequences).
#include "decode_kernel.h"

namespace omnimem {
namespace {

constexpr float kBelow = 1.f - 1.f / 256;  // of a probability: what its first bf16 piece is cut from

// A wave's tile of KEYS keys.  S^T = K Q^T and O^T += V^T P^T, so that query heads are the
// columns of both (lane % 16) and the scores' layout is the B operand of the second product:
// lane group j = lane / 16 holds, of 32 bf16 keys, keys 8 j .. 8 j + 7 (two K row tiles whose
// rows are taken in the order 8 j + 4 a + r), of 16 fp32 keys, keys 4 j + r of step r.  Both
// operands of QK take the 16 bytes 4 s + j of their rows as step s; the order of a contraction is free.
template <typename T, int D>
struct Tile;

template <int D>
struct Tile<uint16_t, D> {
  typedef uint16_t Io;
  static constexpr int kDim = D;
  static constexpr bool kScaled = false;
  static constexpr int wgs(int) { return 2; }
  static constexpr bool kTwoPolicies = true;
  static constexpr int ROW = D * 2, KEYS = 8192 / ROW, KB = KEYS / 32, QS = ROW / 64, VW = D / 16;
  static constexpr int RT = KEYS / 16;  // 16-key row tiles
  static constexpr int UNIT = KEYS;
  typedef uint32_t vraw __attribute__((ext_vector_type(VW / 2)));  // a lane's V dims of one key
  u32x4 k[KB][2][QS];
  vraw v[KB][8];

  __device__ __forceinline__ static int key(int t, int r, int j) { return 32 * (t / 2) + 8 * j + 4 * (t % 2) + r; }

  template <int POLICY>
  __device__ __forceinline__ void load_k(__amdgpu_buffer_rsrc_t rs, int i, int j) {
    const int at = (8 * (i / 4) + i % 4) * ROW + j * 16;
#pragma unroll
    for (int b = 0; b < KB; ++b)
#pragma unroll
      for (int a = 0; a < 2; ++a)
#pragma unroll
        for (int s = 0; s < QS; ++s)
          k[b][a][s] = __builtin_amdgcn_raw_buffer_load_b128(rs, at + (32 * b + 4 * a) * ROW + s * 64, 0, POLICY);
  }
  template <int POLICY>
  __device__ __forceinline__ void load_v(__amdgpu_buffer_rsrc_t rs, int i, int j) {
    const int at = 8 * j * ROW + i * VW * 2;
#pragma unroll
    for (int b = 0; b < KB; ++b)
#pragma unroll
      for (int e = 0; e < 8; ++e) {
        const int from = at + (32 * b + e) * ROW;
        if constexpr (VW == 8) v[b][e] = __builtin_amdgcn_raw_buffer_load_b128(rs, from, 0, POLICY);
        else v[b][e] = __builtin_amdgcn_raw_buffer_load_b64(rs, from, 0, POLICY);
      }
  }
  __device__ __forceinline__ void clear_v_below(int lo, int j) {
#pragma unroll
    for (int b = 0; b < KB; ++b)
#pragma unroll
      for (int e = 0; e < 8; ++e)
        if (32 * b + 8 * j + e < lo) v[b][e] = vraw{};
  }
  // a lane's part of a query, and the scores of a tile
  __device__ __forceinline__ static void load_q(const uint16_t* row, int j, u32x4 (&q)[QS]) {
    const char* at = reinterpret_cast<const char*>(row) + j * 16;
#pragma unroll
    for (int s = 0; s < QS; ++s) q[s] = *reinterpret_cast<const u32x4*>(at + s * 64);
  }
  template <int NT>
  __device__ __forceinline__ void scores(const u32x4 (&q)[NT][QS], f32x4 (&s)[NT][RT]) const {
#pragma unroll
    for (int n = 0; n < NT; ++n)
#pragma unroll
      for (int r = 0; r < RT; ++r) s[n][r] = qk(q[n], r);
  }
  // scores of row tile t
  __device__ __forceinline__ f32x4 qk(const u32x4 (&q)[QS], int t) const {
    f32x4 c{};
#pragma unroll
    for (int s = 0; s < QS; ++s)
      c = __builtin_amdgcn_mfma_f32_16x16x32_bf16(__builtin_bit_cast(bf16x8, k[t / 2][t % 2][s]),
                                                  __builtin_bit_cast(bf16x8, q[s]), c, 0, 0, 0);
    return c;
  }
  // O^T row tiles m: dims VW * (row of the tile) + m.  A word of the A operand holds dim m of two
  // keys, picked out of the keys' rows.  P goes in two bf16 pieces: the first is a truncation of
  // somewhat less than P, between P (1 - 3 * 2^-8) and P, so that the second is not 0 and an
  // infinite value stays infinite in the sum; the second, rounded by 2^-8 of itself, leaves P
  // 3 * 2^-16 off, and the output's rounding is what O is off by.
  template <int NT>
  __device__ __forceinline__ void pv(const f32x4 (&p)[NT][RT], f32x4 (&o)[NT][VW]) const {
#pragma unroll
    for (int b = 0; b < KB; ++b) {
      bf16x8 high[NT], low[NT];
#pragma unroll
      for (int n = 0; n < NT; ++n) {
        u32x4 w;
#pragma unroll
        for (int e = 0; e < 8; e += 2) {
          const f32x4 x = p[n][2 * b + e / 4];
          const uint32_t a0 = __float_as_uint(x[e % 4] * kBelow), a1 = __float_as_uint(x[e % 4 + 1] * kBelow);
          w[e / 2] = __builtin_amdgcn_perm(a1, a0, 0x07060302u);
          low[n][e] = static_cast<__bf16>(x[e % 4] - __uint_as_float(a0 & 0xffff0000u));
          low[n][e + 1] = static_cast<__bf16>(x[e % 4 + 1] - __uint_as_float(a1 & 0xffff0000u));
        }
        high[n] = __builtin_bit_cast(bf16x8, w);
      }
#pragma unroll
      for (int m = 0; m < VW; ++m) {
        u32x4 w;
#pragma unroll
        for (int e = 0; e < 4; ++e)
          w[e] = __builtin_amdgcn_perm(v[b][2 * e + 1][m / 2], v[b][2 * e][m / 2], m % 2 ? 0x07060302u : 0x05040100u);
#pragma unroll
        for (int n = 0; n < NT; ++n) {
          o[n][m] = __builtin_amdgcn_mfma_f32_16x16x32_bf16(__builtin_bit_cast(bf16x8, w), high[n], o[n][m], 0, 0, 0);
          o[n][m] = __builtin_amdgcn_mfma_f32_16x16x32_bf16(__builtin_bit_cast(bf16x8, w), low[n], o[n][m], 0, 0, 0);
        }
      }
    }
  }
  // first of the four consecutive dims that tiles 4 x .. 4 x + 3 hold of their row
  __device__ __forceinline__ static int dim(int row, int x) { return VW * row + 4 * x; }
};

template <int D>
struct Tile<float, D> {
  typedef float Io;
  static constexpr int kDim = D;
  static constexpr bool kScaled = false;
  static constexpr int wgs(int) { return 2; }
  static constexpr bool kTwoPolicies = true;
  static constexpr int ROW = D * 4, KEYS = 8192 / ROW, RT = KEYS / 16, QS = ROW / 64, VW = D / 16, UNIT = 32;
  u32x4 k[RT][QS];
  u32x4 v[RT][4][VW / 4];

  __device__ __forceinline__ static int key(int t, int r, int j) { return 16 * t + 4 * j + r; }

  template <int POLICY>
  __device__ __forceinline__ void load_k(__amdgpu_buffer_rsrc_t rs, int i, int j) {
    const int at = i * ROW + j * 16;
#pragma unroll
    for (int t = 0; t < RT; ++t)
#pragma unroll
      for (int s = 0; s < QS; ++s)
        k[t][s] = __builtin_amdgcn_raw_buffer_load_b128(rs, at + 16 * t * ROW + s * 64, 0, POLICY);
  }
  template <int POLICY>
  __device__ __forceinline__ void load_v(__amdgpu_buffer_rsrc_t rs, int i, int j) {
    const int at = 4 * j * ROW + i * 16;
#pragma unroll
    for (int t = 0; t < RT; ++t)
#pragma unroll
      for (int r = 0; r < 4; ++r)
#pragma unroll
        for (int x = 0; x < VW / 4; ++x)
          v[t][r][x] = __builtin_amdgcn_raw_buffer_load_b128(rs, at + (16 * t + r) * ROW + x * 256, 0, POLICY);
  }
  __device__ __forceinline__ void clear_v_below(int lo, int j) {
#pragma unroll
    for (int t = 0; t < RT; ++t)
#pragma unroll
      for (int r = 0; r < 4; ++r)
#pragma unroll
        for (int x = 0; x < VW / 4; ++x)
          if (16 * t + 4 * j + r < lo) v[t][r][x] = u32x4{};
  }
  // a lane's part of a query, and the scores of a tile
  __device__ __forceinline__ static void load_q(const float* row, int j, u32x4 (&q)[QS]) {
    const char* at = reinterpret_cast<const char*>(row) + j * 16;
#pragma unroll
    for (int s = 0; s < QS; ++s) q[s] = *reinterpret_cast<const u32x4*>(at + s * 64);
  }
  template <int NT>
  __device__ __forceinline__ void scores(const u32x4 (&q)[NT][QS], f32x4 (&s)[NT][RT]) const {
#pragma unroll
    for (int n = 0; n < NT; ++n)
#pragma unroll
      for (int r = 0; r < RT; ++r) s[n][r] = qk(q[n], r);
  }
  __device__ __forceinline__ f32x4 qk(const u32x4 (&q)[QS], int t) const {
    f32x4 c{};
#pragma unroll
    for (int s = 0; s < QS; ++s)
#pragma unroll
      for (int e = 0; e < 4; ++e)
        c = __builtin_amdgcn_mfma_f32_16x16x4f32(__uint_as_float(k[t][s][e]), __uint_as_float(q[s][e]), c, 0, 0, 0);
    return c;
  }
  template <int NT>
  __device__ __forceinline__ void pv(const f32x4 (&p)[NT][RT], f32x4 (&o)[NT][VW]) const {
#pragma unroll
    for (int t = 0; t < RT; ++t)
#pragma unroll
      for (int r = 0; r < 4; ++r)
#pragma unroll
        for (int m = 0; m < VW; ++m)
#pragma unroll
          for (int n = 0; n < NT; ++n)
            o[n][m] = __builtin_amdgcn_mfma_f32_16x16x4f32(__uint_as_float(v[t][r][m / 4][m % 4]), p[n][t][r], o[n][m],
                                                           0, 0, 0);
  }
  __device__ __forceinline__ static int dim(int row, int x) { return 64 * x + 4 * row; }
};

template <typename L>
hipError_t launch_tile(const DecodeArgs& A, const DecodePlan& p, hipStream_t stream) {
  using T = typename L::Io;
  constexpr int D = L::kDim;
  const auto join = p.join_rows == 1   ? k_decode_join<T, D, 1>
                    : p.join_rows == 2 ? k_decode_join<T, D, 2>
                                       : k_decode_join<T, D, 4>;
  return launch_with_join(p.tile_rows == kDecodeHeadRows ? kernel_of<L, 1>(p) : kernel_of<L, 2>(p), kThreads, join, 256, A, p, stream);
}

}  // namespace

hipError_t launch_decode(const SeqGeom& g, const DecodePlan& p, const DecodeLaunch& a, void* workspace,
                         hipStream_t stream) {
  const DecodeArgs A = decode_args(g, p, a, workspace);
  if (a.dtype == OMNIMEM_BF16)
    return a.D == 128 ? launch_tile<Tile<uint16_t, 128>>(A, p, stream) : launch_tile<Tile<uint16_t, 64>>(A, p, stream);
  return a.D == 128 ? launch_tile<Tile<float, 128>>(A, p, stream) : launch_tile<Tile<float, 64>>(A, p, stream);
}

}  // namespace omnimem
