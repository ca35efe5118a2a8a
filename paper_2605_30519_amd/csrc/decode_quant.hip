// decode_quant.hip -- attention of one new token per sequence over 8-bit pages, for gfx950: the tiles
// of keys that decode_kernel.h's kernel works on.
//
//   O = sum_t softmax_t(scale k_s <q, k_t>) v_s v_t, k_t and v_t e4m3 codes, k_s and v_s their pages' scales
//
// A code is a bf16 number as it stands, so codes are widened to bf16 in registers, two an
// instruction, and both products run on bf16 MFMA without an error of their own; K's scale goes into
// the scores' factor and V's into the probabilities, a scalar each for a tile of one page.
//
// Bound by the stream of K and V, of half the bytes of bf16 pages: four rollouts of 47 to 94 thousand
// tokens, 12 heads of 128 (829 MB), 131 us with the join, 6.3 TB/s (bf16 pages 248 us); 48 sequences of
// 100 to 16,000 tokens, 40 query heads over 8 (309 MB), 59 us (102), of which the join and its launch are 6; 12
// sequences of 4,000 to 30,000, 16 heads of 64 (317 MB), 58 us, whose 4 KB slabs stream 4% slower.  The matrix
// cores are 14% busy, the vector units 36%.
#include "decode_kernel.h"

namespace omnimem {
namespace {

// Two codes of a word, its low or its high half.
template <bool HIGH>
__device__ __forceinline__ uint32_t widen2(uint32_t codes) {
  return __builtin_bit_cast(uint32_t, __builtin_amdgcn_cvt_scalef32_pk_bf16_fp8(codes, 1.f, HIGH));
}

// The parts of x that its first, second and third 8 significant bits make up; cut off, not rounded, so
// that three of them are all of an fp32 number.
__device__ __forceinline__ uint32_t cut(float& x) {
  const uint32_t high = __float_as_uint(x) & 0xffff0000u;
  x -= __uint_as_float(high);
  return high;
}

// 64 keys of a page; the layouts are those of the bf16 tile.  Both operands of QK take the 16 dims
// 16 (4 s + j) .. of their rows as two steps; a step is 8 of them for each lane group j.
// PIECES: bf16 numbers that a query is held in, 3 for fp32 (all of its 24 bits); P, with V's scale,
// goes in one more than a bf16 query, 2^-15 off, or in 3.
template <typename T, int D>
struct TileQuant {
  typedef T Io;
  static constexpr int kDim = D;
  static constexpr bool kScaled = true;
  static constexpr bool kF32 = sizeof(T) == 4;
  static constexpr int ROW = D, KEYS = 64, UNIT = 64, KB = 2, RT = 4, VW = D / 16;
  static constexpr int KC = D / 64;  // 16-byte chunks of a lane's part of a key
  static constexpr int PIECES = kF32 ? 3 : 1, STEPS = 2 * KC, QS = STEPS * PIECES;
  static constexpr int P_PIECES = kF32 ? 3 : 2;
  static constexpr int wgs(int nt) { return nt == 2 && D == 128 ? 1 : 2; }
  // fp32 queries of 128 dims leave no registers for a second loop (56 spilled: 32 windows of 2,500
  // tokens, 8 key heads, 147 us instead of 38); the one that is left spills two or three over a line, 8 to 12 bytes of
  // scratch memory a lane: four rollouts of 47 to 94 thousand tokens, 12 heads, 135 us, 129 with bf16 queries
  static constexpr bool kTwoPolicies = !(kF32 && D == 128);
  typedef uint32_t vraw __attribute__((ext_vector_type(VW / 4)));  // a lane's V dims of one key
  u32x4 k[KB][2][KC];
  vraw v[KB][8];

  __device__ __forceinline__ static int key(int t, int r, int j) { return 32 * (t / 2) + 8 * j + 4 * (t % 2) + r; }

  // piece p of step x in q[p * STEPS + x]
  __device__ __forceinline__ static void load_q(const T* row, int j, u32x4 (&q)[QS]) {
#pragma unroll
    for (int x = 0; x < STEPS; ++x) {
      const T* at = row + 16 * (x / 2 * 4 + j) + 8 * (x % 2);
      if constexpr (!kF32) {
        q[x] = *reinterpret_cast<const u32x4*>(at);
      } else {
        f32x4 f[2] = {*reinterpret_cast<const f32x4*>(at), *reinterpret_cast<const f32x4*>(at + 4)};
#pragma unroll
        for (int p = 0; p < PIECES; ++p)
#pragma unroll
          for (int e = 0; e < 8; e += 2) {
            float a = f[e / 4][e % 4], b = f[e / 4][e % 4 + 1];
            q[p * STEPS + x][e / 2] = __builtin_amdgcn_perm(cut(b), cut(a), 0x07060302u);
            f[e / 4][e % 4] = a;
            f[e / 4][e % 4 + 1] = b;
          }
      }
    }
  }
  template <int POLICY>
  __device__ __forceinline__ void load_k(__amdgpu_buffer_rsrc_t rs, int i, int j) {
    const int at = (8 * (i / 4) + i % 4) * ROW + j * 16;
#pragma unroll
    for (int b = 0; b < KB; ++b)
#pragma unroll
      for (int a = 0; a < 2; ++a)
#pragma unroll
        for (int s = 0; s < KC; ++s)
          k[b][a][s] = __builtin_amdgcn_raw_buffer_load_b128(rs, at + (32 * b + 4 * a) * ROW + s * 64, 0, POLICY);
  }
  template <int POLICY>
  __device__ __forceinline__ void load_v(__amdgpu_buffer_rsrc_t rs, int i, int j) {
    const int at = 8 * j * ROW + i * VW;
#pragma unroll
    for (int b = 0; b < KB; ++b)
#pragma unroll
      for (int e = 0; e < 8; ++e) {
        const int from = at + (32 * b + e) * ROW;
        if constexpr (VW == 8) v[b][e] = __builtin_amdgcn_raw_buffer_load_b64(rs, from, 0, POLICY);
        else v[b][e][0] = __builtin_amdgcn_raw_buffer_load_b32(rs, from, 0, POLICY);
      }
  }
  __device__ __forceinline__ void clear_v_below(int lo, int j) {
#pragma unroll
    for (int b = 0; b < KB; ++b)
#pragma unroll
      for (int e = 0; e < 8; ++e)
        if (32 * b + 8 * j + e < lo) v[b][e] = vraw{};
  }
  template <int NT>
  __device__ __forceinline__ void scores(const u32x4 (&q)[NT][QS], f32x4 (&s)[NT][RT]) const {
    // the row tiles' chains side by side: a product waits for the one before it in its own
#pragma unroll
    for (int x = 0; x < STEPS; ++x) {
      u32x4 a[RT];
#pragma unroll
      for (int t = 0; t < RT; ++t) {
        const u32x4 c = k[t / 2][t % 2][x / 2];
        const int w = x % 2 * 2;
        a[t] = u32x4{widen2<false>(c[w]), widen2<true>(c[w]), widen2<false>(c[w + 1]), widen2<true>(c[w + 1])};
      }
#pragma unroll
      for (int p = 0; p < PIECES; ++p)
#pragma unroll
        for (int n = 0; n < NT; ++n)
#pragma unroll
          for (int t = 0; t < RT; ++t)
            s[n][t] = __builtin_amdgcn_mfma_f32_16x16x32_bf16(
                __builtin_bit_cast(bf16x8, a[t]), __builtin_bit_cast(bf16x8, q[n][p * STEPS + x]),
                x == 0 && p == 0 ? f32x4{} : s[n][t], 0, 0, 0);
    }
  }
  // O^T row tiles m: dims VW * (row of the tile) + m.  Four keys' words of four dims are turned into
  // four dims' words of four keys, whose halves widen to words of the A operand.
  template <int NT>
  __device__ __forceinline__ void pv(const f32x4 (&p)[NT][RT], float scale, f32x4 (&o)[NT][VW]) const {
#pragma unroll
    for (int b = 0; b < KB; ++b) {
      u32x4 piece[NT][P_PIECES];
#pragma unroll
      for (int n = 0; n < NT; ++n)
#pragma unroll
        for (int e = 0; e < 8; e += 2) {
          float x = p[n][2 * b + e / 4][e % 4] * scale, y = p[n][2 * b + e / 4][e % 4 + 1] * scale;
#pragma unroll
          for (int z = 0; z < P_PIECES; ++z) {
            if constexpr (!kF32) {
              if (z == 1) {  // the last piece, rounded
                const bf16x2 r = {static_cast<__bf16>(x), static_cast<__bf16>(y)};
                piece[n][z][e / 2] = __builtin_bit_cast(uint32_t, r);
                continue;
              }
            }
            piece[n][z][e / 2] = __builtin_amdgcn_perm(cut(y), cut(x), 0x07060302u);
          }
        }
#pragma unroll
      for (int w = 0; w < VW / 4; ++w) {
        uint32_t d[2][4];
#pragma unroll
        for (int f = 0; f < 2; ++f) {
          const uint32_t a = v[b][4 * f][w], c = v[b][4 * f + 1][w], g = v[b][4 * f + 2][w], h = v[b][4 * f + 3][w];
          const uint32_t ac0 = __builtin_amdgcn_perm(c, a, 0x05010400u), ac2 = __builtin_amdgcn_perm(c, a, 0x07030602u);
          const uint32_t gh0 = __builtin_amdgcn_perm(h, g, 0x05010400u), gh2 = __builtin_amdgcn_perm(h, g, 0x07030602u);
          d[f][0] = __builtin_amdgcn_perm(gh0, ac0, 0x05040100u);
          d[f][1] = __builtin_amdgcn_perm(gh0, ac0, 0x07060302u);
          d[f][2] = __builtin_amdgcn_perm(gh2, ac2, 0x05040100u);
          d[f][3] = __builtin_amdgcn_perm(gh2, ac2, 0x07060302u);
        }
        u32x4 a[4];
#pragma unroll
        for (int m = 0; m < 4; ++m)
          a[m] = u32x4{widen2<false>(d[0][m]), widen2<true>(d[0][m]), widen2<false>(d[1][m]), widen2<true>(d[1][m])};
#pragma unroll
        for (int z = 0; z < P_PIECES; ++z)
#pragma unroll
          for (int n = 0; n < NT; ++n)
#pragma unroll
            for (int m = 0; m < 4; ++m)
              o[n][4 * w + m] = __builtin_amdgcn_mfma_f32_16x16x32_bf16(
                  __builtin_bit_cast(bf16x8, a[m]), __builtin_bit_cast(bf16x8, piece[n][z]), o[n][4 * w + m], 0, 0, 0);
      }
    }
  }
  __device__ __forceinline__ static int dim(int row, int x) { return VW * row + 4 * x; }
};

template <typename L>
hipError_t launch_tile(const DecodeArgs& A, const DecodePlan& p, hipStream_t stream) {
  using T = typename L::Io;
  constexpr int D = L::kDim;
  auto kernel = p.tile_rows == kDecodeHeadRows   ? kernel_of<L, 1>(p)
                : !p.pair                       ? k_decode<L, 2, DecodeSplit::kLine>
                : p.split == DecodeSplit::kLine ? k_decode<L, 1, DecodeSplit::kLine, true>
                                                : k_decode<L, 1, DecodeSplit::kItem, true>;
  int threads = kThreads;
  if constexpr (D == 64) {
    if (p.eight_waves) {
      kernel = k_decode<L, 1, DecodeSplit::kItem, false, 8>;
      threads = 8 * kWave;
    }
  }
  // The shares of a long item are many, and a set of threads takes its part of them one behind the other:
  // 512 threads a row where an item has 64 shares and more (one of 100,000 tokens, 8 query heads, 15.8 ->
  // 8.5 us), else two rows of 128 with eight shares' loads in flight (18 ragged items of 24 query heads, four rows
  // and four shares 13.6, this 8.0; 32 items of 32 heads 11.4 / 5.9; 384 items 4.7 both).
  const auto join = p.join_rows == 1 ? (p.long_items ? k_decode_join<T, D, 1, 512, 8> : k_decode_join<T, D, 1>)
                                     : k_decode_join<T, D, 2, 256, 8>;
  return launch_with_join(kernel, threads, join, p.long_items ? 512 : 256, A, p, stream);
}

}  // namespace

hipError_t launch_decode_quant(const SeqGeom& g, const DecodePlan& p, const DecodeLaunch& a, void* workspace,
                               hipStream_t stream) {
  const DecodeArgs A = decode_args(g, p, a, workspace);
  if (a.dtype == OMNIMEM_BF16)
    return a.D == 128 ? launch_tile<TileQuant<uint16_t, 128>>(A, p, stream)
                      : launch_tile<TileQuant<uint16_t, 64>>(A, p, stream);
  return a.D == 128 ? launch_tile<TileQuant<float, 128>>(A, p, stream) : launch_tile<TileQuant<float, 64>>(A, p, stream);
}

}  // namespace omnimem
