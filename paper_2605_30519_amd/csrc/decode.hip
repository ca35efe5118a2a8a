// decode.hip -- attention of one new token per sequence over a paged cache, for gfx950:
//   O[i][h] = sum_t softmax_t(scale <q_i, k_t>) v_t over the tokens of sequence i.
//
// A key and a value serve the G query heads of their head alone, G flops a byte of bf16, so
// the kernel is bound by the stream of K and V from memory and built to keep it full: no LDS
// and no barrier between loads and products, tiles of 8 KB of K and 8 KB of V a wave straight
// into MFMA operand registers, the next tile's loads issued as soon as the registers of the
// present one are read.  Four rollouts of 47 to 94 thousand tokens, 12 heads of 128, bf16
// (1.66 GB): 247 us with the join, 6.7 TB/s, with plain instead of nontemporal loads 272; 48
// sequences of 100 to 16,000 tokens, 40 query heads over 8 (617 MB): 101 us with the join, 6.1 TB/s.
//
// Split.  An item is a (sequence, key/value head, tile of up to 32 query heads); its units of
// 32 tokens (64 for bf16 heads of 64) follow one another on a line of all items' units, and
// workgroup w takes the equal share [w q, (w + 1) q) of it, over item boundaries, so that any
// mix of lengths loads every workgroup alike and lengths stay on the device (a captured graph
// replays with others).  The four waves take a segment's units in turn and meet in LDS; an
// item that several workgroups share leaves (O, max, sum) a share in the workspace, which
// k_decode_join adds up in the order of the line, in a launch of its own (4 to 5 us): workgroups
// that hand results on within a launch pay more for the caches between the dies.  With 64
// instead of 32 tokens a unit the waves' loads differ more (5% for the 48 sequences).
#include <float.h>

#include "device_common.h"
#include "launch.h"
#include "seq_launch.h"

namespace omnimem {
namespace {

// What an item costs beside its units (its waves meet, its result is written), in units: lengths
// on the line count it, so that a share of short items holds fewer units.  12 sequences of 1 to
// 11,664 tokens, 40 fp32 heads of 64: 82 us without, 66 with one unit, 58 with three, 59 with six.
constexpr int kItemUnits = 3;
constexpr int kThreads = kDecodeWaves * kWave;
constexpr int kMinUnits = 4;      // units of a share: one for each wave
constexpr float kLowest = -FLT_MAX;  // below every score: a row without keys keeps sum 0
constexpr int kAskUnits = 64;     // units of a share from which it is asked whether pages are shared
constexpr int kNontemporal = 2;   // cache policy of a buffer load: read once
constexpr float kBelow = 1.f - 1.f / 256;  // of a probability: what its first bf16 piece is cut from

struct DecodeArgs {
  SeqGeom g;
  DecodeLaunch a;
  int G, head_tiles, tile_rows, rows;
  float scale2;  // scale * log2 e: the softmax runs on exp2
  float* part;
  DecodeStart* starts;
  int slot_floats;
};

// Tokens [begin, end) of a sequence and the blocks that hold them, in units of UT tokens.
struct Span {
  int begin, end, block, units;
};

__device__ __forceinline__ int block_shift(const SeqGeom& g) { return 6 + (g.B >> 7); }  // log2 B

__device__ __forceinline__ int block_of(const SeqGeom& g, int t) {
  if (g.S == g.B) return t >> block_shift(g);
  const int c = t / g.S;
  return c * g.Bpc + ((t - c * g.S) >> block_shift(g));
}

template <int UT>
__device__ __forceinline__ Span span_of(const DecodeArgs& A, int len) {
  Span s;
  s.end = min(max(len, 0), A.g.cap);
  s.begin = A.a.window > 0 ? max(0, s.end - A.a.window) : 0;
  s.block = block_of(A.g, s.begin);
  s.units = s.end > 0 ? (block_of(A.g, s.end - 1) + 1 - s.block) * (A.g.B / UT) : 0;
  return s;
}

// Inclusive prefix sums over a wave, by cross-lane moves of the VALU.
__device__ __forceinline__ int scan_lanes(int v) {
  v += __builtin_amdgcn_update_dpp(0, v, 0x111, 0xf, 0xf, false);  // row_shr:1, 2, 4, 8: within 16 lanes
  v += __builtin_amdgcn_update_dpp(0, v, 0x112, 0xf, 0xf, false);
  v += __builtin_amdgcn_update_dpp(0, v, 0x114, 0xf, 0xf, false);
  v += __builtin_amdgcn_update_dpp(0, v, 0x118, 0xf, 0xf, false);
  v += __builtin_amdgcn_update_dpp(0, v, 0x142, 0xa, 0xf, false);  // row_bcast:15 into rows 1 and 3
  v += __builtin_amdgcn_update_dpp(0, v, 0x143, 0xc, 0xf, false);  // row_bcast:31 into rows 2 and 3
  return v;
}

__device__ __forceinline__ float max_over_groups(float x) {  // over the four 16-lane groups
  const auto a = __builtin_amdgcn_permlane16_swap(__float_as_uint(x), __float_as_uint(x), false, false);
  const float y = fmaxf(__uint_as_float(a[0]), __uint_as_float(a[1]));
  const auto b = __builtin_amdgcn_permlane32_swap(__float_as_uint(y), __float_as_uint(y), false, false);
  return fmaxf(__uint_as_float(b[0]), __uint_as_float(b[1]));
}

__device__ __forceinline__ float sum_over_groups(float x) {
  const auto a = __builtin_amdgcn_permlane16_swap(__float_as_uint(x), __float_as_uint(x), false, false);
  const float y = __uint_as_float(a[0]) + __uint_as_float(a[1]);
  const auto b = __builtin_amdgcn_permlane32_swap(__float_as_uint(y), __float_as_uint(y), false, false);
  return __uint_as_float(b[0]) + __uint_as_float(b[1]);
}

// Rows [0, rows) of a tile; further rows read as zero.
__device__ __forceinline__ __amdgpu_buffer_rsrc_t tile_rsrc(const void* base, int bytes) {
  const u32x4 r = buffer_rsrc(base, bytes);
  return __builtin_amdgcn_make_buffer_rsrc(reinterpret_cast<void*>(static_cast<uint64_t>(r[1]) << 32 | r[0]), 0, r[2],
                                           r[3]);
}

// A wave's tile of KEYS keys.  S^T = K Q^T and O^T += V^T P^T, so that query heads are the
// columns of both (lane % 16) and the scores' layout is the B operand of the second product:
// lane group j = lane / 16 holds, of 32 bf16 keys, keys 8 j .. 8 j + 7 (two K row tiles whose
// rows are taken in the order 8 j + 4 a + r), of 16 fp32 keys, keys 4 j + r of step r.  Both
// operands of QK take the 16 bytes 4 s + j of their rows as step s; the order of a contraction is free.
template <typename T, int D>
struct Tile;

template <int D>
struct Tile<uint16_t, D> {
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

__device__ __forceinline__ void store_row(uint16_t* out, const f32x4 x) {
  bf16x4 w;
#pragma unroll
  for (int e = 0; e < 4; ++e) w[e] = static_cast<__bf16>(x[e]);
  *reinterpret_cast<bf16x4*>(out) = w;
}
__device__ __forceinline__ void store_row(float* out, const f32x4 x) { *reinterpret_cast<f32x4*>(out) = x; }

// One row's four dims of the sum over keys; a row without keys gives zeros.
template <typename T>
__device__ __forceinline__ void finish(const DecodeArgs& A, int seq, int hq, int d, f32x4 o, float top, float sum) {
  const float inv = sum == 0.f ? 0.f : 1.f / sum;
#pragma unroll
  for (int e = 0; e < 4; ++e) o[e] *= inv;
  store_row(static_cast<T*>(A.a.out) + (static_cast<int64_t>(seq) * A.a.Hq + hq) * A.a.D + d, o);
  if (d == 0 && A.a.lse != nullptr)
    A.a.lse[static_cast<int64_t>(hq) * A.g.N + seq] =
        sum == 0.f ? -INFINITY : (top + log2f(sum)) * 0.69314718055994531f;
}

// A workgroup's run of units of one item.
struct Segment {
  Span sp;
  int seq, head;  // head: (key/value head, tile)
  int unit, stop;
};

// LDS traffic of the workgroup only: loads from memory stay in flight across it.
__device__ __forceinline__ void lds_sync() {
  __builtin_amdgcn_fence(__ATOMIC_RELEASE, "workgroup", "local");
  __builtin_amdgcn_s_barrier();
  __builtin_amdgcn_fence(__ATOMIC_ACQUIRE, "workgroup", "local");
}

template <typename T, int D, int NT, DecodeSplit SPLIT>
__global__ __launch_bounds__(kThreads, 2) void k_decode(const DecodeArgs A) {
  using L = Tile<T, D>;
  constexpr int RT = L::RT, VW = L::VW, QS = L::QS, UT = L::UNIT;
  constexpr bool LINE = SPLIT == DecodeSplit::kLine, BY_WAVE = SPLIT == DecodeSplit::kWave;
  constexpr int TEAM = BY_WAVE ? 1 : kDecodeWaves;  // waves that share a segment
  __shared__ __align__(16) float s_o[kDecodeWaves][NT * 16][D];
  __shared__ float s_top[kDecodeWaves][NT * 16], s_sum[kDecodeWaves][NT * 16];
  const int tid = threadIdx.x, lane = tid % kWave;
  const int wave = __builtin_amdgcn_readfirstlane(tid / kWave);
  const int i = lane % 16, j = lane / 16;
  const int HH = A.a.H * A.head_tiles;
  const int N = A.g.N;

  Segment g{};
  int left = 0;  // units of the share from g.unit on
  bool long_share = false;
  if constexpr (!LINE) {
    const int item = BY_WAVE ? blockIdx.x * kDecodeWaves + wave : blockIdx.x;
    g.seq = item / HH;
    g.head = item - g.seq * HH;
    if (g.seq >= N) return;  // behind the last item, where every wave has its own
    g.sp = span_of<UT>(A, __builtin_amdgcn_readfirstlane(A.g.lens[g.seq]));
    left = g.sp.units;
    if (left == 0) {
      const int h = g.head / A.head_tiles, tile = g.head % A.head_tiles;
      const int rows = min(A.tile_rows, A.G - tile * A.tile_rows);
      for (int e = BY_WAVE ? lane : tid; e < rows * (D / 4); e += TEAM * kWave)
        finish<T>(A, g.seq, h * A.G + tile * A.tile_rows + e / (D / 4), e % (D / 4) * 4, f32x4{}, 0.f, 0.f);
      return;
    }
  } else {
    // The line, formed by every wave for itself: lane l's sequences, the units in front of
    // them, and the sequence that this share begins in.
    const int per = (N + kWave - 1) / kWave;
    const int first_seq = min(lane * per, N), last_seq = min(first_seq + per, N);
    int mine = 0, empty = 0, len = 0;
    for (int s = first_seq; s < last_seq; ++s) {
      len = A.g.lens[s];
      const int u = span_of<UT>(A, len).units;
      mine += u > 0 ? u + kItemUnits : 0;
      empty |= u == 0;
    }
    const int upto = scan_lanes(mine);
    const int all = __builtin_amdgcn_readlane(upto, kWave - 1);
    const int64_t line = static_cast<int64_t>(all) * HH;
    // positions in 32 bits where they fit, for the divisions' sake
    const bool small = line + gridDim.x <= 0x7fffffff;
    const int even = small ? static_cast<int>((static_cast<uint32_t>(line) + gridDim.x - 1) / gridDim.x)
                           : static_cast<int>((line + gridDim.x - 1) / gridDim.x);
    const int share = max(kMinUnits, even);
    long_share = share >= kAskUnits;
    const int64_t pos = static_cast<int64_t>(blockIdx.x) * share;
    // sequences without tokens get their zeros
    if (__ballot(empty) != 0) {
      const int each = (N + gridDim.x - 1) / gridDim.x;
      const int end = min(static_cast<int64_t>(N), (static_cast<int64_t>(blockIdx.x) + 1) * each);
      for (int64_t s0 = static_cast<int64_t>(blockIdx.x) * each; s0 < end; s0 += kWave) {
        uint64_t none = __ballot(s0 + lane < end && span_of<UT>(A, A.g.lens[min(s0 + lane, int64_t{N} - 1)]).units == 0);
        for (; none != 0; none &= none - 1)
          for (int e = tid; e < A.a.Hq * (D / 4); e += kThreads)
            finish<T>(A, static_cast<int>(s0) + __builtin_ctzll(none), e / (D / 4), e % (D / 4) * 4, f32x4{}, 0.f, 0.f);
      }
    }
    if (pos >= line) {
      if (tid == 0) A.starts[blockIdx.x] = DecodeStart{};
      return;
    }
    left = static_cast<int>(min(static_cast<int64_t>(share), line - pos));
    const int x = small ? static_cast<int>(static_cast<uint32_t>(pos) / static_cast<uint32_t>(HH))
                        : static_cast<int>(pos / HH);
    const int at = __builtin_ctzll(__ballot(upto > x));  // the lane whose sequences hold position x
    int before = __builtin_amdgcn_readlane(upto - mine, at);
    g.seq = at * per;
    if (per == 1) {
      g.sp = span_of<UT>(A, __builtin_amdgcn_readlane(len, at));
    } else {
      for (; g.seq < N; ++g.seq) {
        g.sp = span_of<UT>(A, __builtin_amdgcn_readfirstlane(A.g.lens[g.seq]));
        if (g.sp.units == 0) continue;
        if (x - before < g.sp.units + kItemUnits) break;
        before += g.sp.units + kItemUnits;
      }
    }
    const int64_t in = pos - static_cast<int64_t>(before) * HH;
    const int length = g.sp.units + kItemUnits;
    g.head = in <= 0x7fffffff ? static_cast<int>(static_cast<uint32_t>(in) / static_cast<uint32_t>(length))
                              : static_cast<int>(in / length);
    const int at_unit = static_cast<int>(in - static_cast<int64_t>(g.head) * length) - kItemUnits;
    g.unit = max(at_unit, 0);
    left += min(at_unit, 0);
    if (tid == 0) {
      DecodeStart st{};
      if (g.unit > 0) st = DecodeStart{pos - g.unit, g.sp.units, g.seq, g.head, share};
      A.starts[blockIdx.x] = st;
    }
    if (left <= 0) return;  // the share ends in front of the item's first unit
  }
  g.stop = min(g.sp.units, g.unit + left);
  left -= g.stop - g.unit;

  // The wave's tiles form one stream over the segments: while a segment's last tile is worked
  // on, the first one of the next segment is on its way.  The stream's own segment is f, at
  // most one in front of g; its units are looked up 64 at a time, lane l the l-th one's page and,
  // in one register, its first token row and its rows in use.
  Segment f = g;
  int next = f.unit + (BY_WAVE ? 0 : wave);
  uint64_t mask = 0;
  int l_page = 0;
  uint32_t l_rows = 0;
  int lo = 0, hi = 0, sub = 0;  // the tile's unit: rows in use, rows before the tile
  int64_t row = 0;              // the unit's first row in the pools
  auto look_up = [&]() {
    const int u = next + lane * TEAM;
    bool ok = u < f.stop;
    if (ok) {
      const int in_block = block_shift(A.g) - (UT == 64 ? 6 : 5);  // log2 of a block's units
      const int b = f.sp.block + (u >> in_block);
      const int l_row = (u & ((1 << in_block) - 1)) * UT;
      const int c = A.g.Bpc == 1 ? b : b / A.g.Bpc;
      const int in = (b - c * A.g.Bpc) * A.g.B + l_row;
      const int tok = c * A.g.S + in;
      l_page = A.g.table[static_cast<int64_t>(f.seq) * A.g.M + b];
      const int l_hi = min(UT, min(A.g.S - in, f.sp.end - tok));
      const int l_lo = max(0, f.sp.begin - tok);
      ok = l_page >= 0 && l_page < A.g.num_pages && l_lo < l_hi;
      l_rows = static_cast<uint32_t>(l_row << 16 | l_hi) | static_cast<uint32_t>(l_lo) << 8;  // where ok: <= 96, 64, 63
    }
    mask = __ballot(ok);
    next += kWave * TEAM;
  };
  auto advance = [&]() -> bool {
    if (sub + L::KEYS < hi) {
      sub += L::KEYS;
      return true;
    }
    while (mask == 0) {
      if (!LINE || next >= f.stop) {  // an item of a workgroup's own or a wave's is one look-up
        lo = hi = sub = 0;  // a tile of no rows
        return false;
      }
      look_up();
    }
    const int at = __builtin_ctzll(mask);
    mask &= mask - 1;
    const int rows = __builtin_amdgcn_readlane(l_rows, at);
    lo = rows >> 8 & 0xff;
    hi = rows & 0xff;
    row = (static_cast<int64_t>(__builtin_amdgcn_readlane(l_page, at)) * A.a.H + f.head / A.head_tiles) * A.g.B +
          (rows >> 16);
    sub = lo / L::KEYS * L::KEYS;
    return true;
  };
  auto rsrc = [&](const void* pool) {
    return tile_rsrc(static_cast<const char*>(pool) + (row + sub) * L::ROW, max(0, min(hi - sub, L::KEYS)) * L::ROW);
  };
  u32x4 q[NT][QS];
  auto load_q = [&]() {
    const int tile = f.head % A.head_tiles, hq0 = f.head / A.head_tiles * A.G + tile * A.tile_rows;
    const int rows = min(A.tile_rows, A.G - tile * A.tile_rows);
#pragma unroll
    for (int n = 0; n < NT; ++n) {  // rows past the last query head repeat it and are not written
      const char* at = reinterpret_cast<const char*>(static_cast<const T*>(A.a.q) + f.seq * A.a.q_stride +
                                                     static_cast<int64_t>(hq0 + min(n * 16 + i, rows - 1)) * D) +
                       j * 16;
#pragma unroll
      for (int s = 0; s < QS; ++s) q[n][s] = *reinterpret_cast<const u32x4*>(at + s * 64);
    }
  };
  // the stream's next segment; false behind the share's last one
  auto next_segment = [&]() -> bool {
    left -= kItemUnits;
    if (!LINE || left <= 0) return false;
    f.unit = 0;
    if (++f.head == HH) {
      f.head = 0;
      do {
        if (++f.seq >= N) return false;
        f.sp = span_of<UT>(A, __builtin_amdgcn_readfirstlane(A.g.lens[f.seq]));
      } while (f.sp.units == 0);
    }
    f.stop = min(f.sp.units, left);
    left -= f.stop;
    next = wave;
    load_q();
    return true;
  };

  L t;
  load_q();
  // A page of one sequence is read once, and marked so it comes a tenth faster; one that forked
  // sequences share is read by each, and serves them from the caches when it is not.  16 sequences
  // of 30,000 tokens, 8 key heads, on one prompt's pages: 241 us marked, 150 not; 8,000 tokens: 69
  // / 51.  On pages of their own, four of 47 to 94 thousand tokens, 12 key heads: 248 / 272.  So a
  // workgroup with a long share looks whether the row in front of or behind its first segment's has
  // the same pages.  A short share gains nothing (64 of 2,000: 45 both) and would wait 0.5 us for
  // the answer, and with more than 16 query heads to a key head a second loop costs registers that
  // there are not.
  bool shared = false;
  if constexpr (LINE && NT == 1) {
    const int u = f.unit + lane;
    bool same = false;
    if (long_share && u < f.stop && N > 1) {
      const int b = f.sp.block + (u >> (block_shift(A.g) - (UT == 64 ? 6 : 5)));
      const int32_t* at = A.g.table + static_cast<int64_t>(f.seq) * A.g.M + b;
      const int32_t before = f.seq > 0 ? at[-A.g.M] : -1, behind = f.seq + 1 < N ? at[A.g.M] : -1;
      same = before == *at || behind == *at;
    }
    shared = 2 * __popcll(__ballot(same)) > min(kWave, f.stop - f.unit);
  }
  if constexpr (!LINE) look_up();
  bool have = advance();
  auto stream = [&](auto policy) __attribute__((always_inline)) {
    constexpr int POLICY = decltype(policy)::value;
    t.template load_k<POLICY>(rsrc(A.a.k_pages), i, j);
    __builtin_amdgcn_sched_barrier(0);  // K in front of V here as in the loop, whose waits count on it
    t.template load_v<POLICY>(rsrc(A.a.v_pages), i, j);
    for (bool first = true;; first = false) {
      f32x4 o[NT][VW] = {};
      float top[NT], sum[NT];
#pragma unroll
      for (int n = 0; n < NT; ++n) {
        top[n] = kLowest;
        sum[n] = 0.f;
      }
      bool ahead = false;  // f is the segment behind g
      bool follows = false;
      while (have) {
        const int clo = lo - sub, chi = hi - sub;  // rows of the tile in use
        f32x4 s[NT][RT];
#pragma unroll
        for (int n = 0; n < NT; ++n)
#pragma unroll
          for (int r = 0; r < RT; ++r) s[n][r] = t.qk(q[n], r);
        have = advance();
        if (!have) {
          ahead = true;
          follows = next_segment();
          if (follows) advance();
        }
        t.template load_k<POLICY>(rsrc(A.a.k_pages), i, j);
        const bool whole = clo <= 0 && chi >= L::KEYS;
#pragma unroll
        for (int n = 0; n < NT; ++n) {
          float m = kLowest;
#pragma unroll
          for (int r = 0; r < RT; ++r)
#pragma unroll
            for (int e = 0; e < 4; ++e) s[n][r][e] *= A.scale2;
          if (!whole) {
#pragma unroll
            for (int r = 0; r < RT; ++r)
#pragma unroll
              for (int e = 0; e < 4; ++e) {
                const int key = L::key(r, e, j);
                s[n][r][e] = key >= clo && key < chi ? s[n][r][e] : -INFINITY;
              }
          }
#pragma unroll
          for (int r = 0; r < RT; ++r)
#pragma unroll
            for (int e = 0; e < 4; ++e) m = fmaxf(m, s[n][r][e]);
          m = fmaxf(max_over_groups(m), top[n]);
          const float keep = exp2f(top[n] - m);
          top[n] = m;
          float add = 0.f;
#pragma unroll
          for (int r = 0; r < RT; ++r)
#pragma unroll
            for (int e = 0; e < 4; ++e) {
              s[n][r][e] = __builtin_amdgcn_exp2f(s[n][r][e] - m);
              add += s[n][r][e];
            }
          sum[n] = sum[n] * keep + add;
          if (__any(keep != 1.f)) {
#pragma unroll
            for (int x = 0; x < VW; ++x)
#pragma unroll
              for (int e = 0; e < 4; ++e) o[n][x][e] *= keep;
          }
        }
        if (clo > 0) t.clear_v_below(clo, j);
        t.template pv<NT>(s, o);
        t.template load_v<POLICY>(rsrc(A.a.v_pages), i, j);
      }
      if (!ahead) {  // the wave had no tile of this segment
        follows = next_segment();
        if (follows) advance();
        t.template load_k<POLICY>(rsrc(A.a.k_pages), i, j);
        __builtin_amdgcn_sched_barrier(0);
        t.template load_v<POLICY>(rsrc(A.a.v_pages), i, j);
      }

      // the waves' results meet
      const int tile = g.head % A.head_tiles, hq0 = g.head / A.head_tiles * A.G + tile * A.tile_rows;
      const int rows = min(A.tile_rows, A.G - tile * A.tile_rows);
      if constexpr (BY_WAVE) {
#pragma unroll
        for (int n = 0; n < NT; ++n) {
          const float total = sum_over_groups(sum[n]);
          if (n * 16 + i >= rows) continue;
#pragma unroll
          for (int r = 0; r < 4; ++r)
#pragma unroll
            for (int x = 0; x < VW / 4; ++x) {
              f32x4 w;
#pragma unroll
              for (int e = 0; e < 4; ++e) w[e] = o[n][4 * x + e][r];
              finish<T>(A, g.seq, hq0 + n * 16 + i, L::dim(4 * j + r, x), w, top[n], total);
            }
        }
        return;
      }
      if (!first) lds_sync();  // the last segment's results have been read
#pragma unroll
      for (int n = 0; n < NT; ++n) {
        const float total = sum_over_groups(sum[n]);
        if (n * 16 + i < rows) {
          if (j == 0) {
            s_top[wave][n * 16 + i] = top[n];
            s_sum[wave][n * 16 + i] = total;
          }
          float* to = s_o[wave][n * 16 + i];
#pragma unroll
          for (int r = 0; r < 4; ++r)
#pragma unroll
            for (int x = 0; x < VW / 4; ++x) {
              f32x4 w;
#pragma unroll
              for (int e = 0; e < 4; ++e) w[e] = o[n][4 * x + e][r];
              *reinterpret_cast<f32x4*>(to + L::dim(4 * j + r, x)) = w;
            }
        }
      }
      lds_sync();
      const bool complete = !LINE || (g.unit == 0 && g.stop == g.sp.units);
      float* slot = A.part + (static_cast<int64_t>(blockIdx.x) * 2 + (first ? 0 : 1)) * A.slot_floats;
      for (int e = tid; e < rows * (D / 4); e += kThreads) {
        const int r = e / (D / 4), d = e % (D / 4) * 4;
        float m = s_top[0][r];
#pragma unroll
        for (int w = 1; w < kDecodeWaves; ++w) m = fmaxf(m, s_top[w][r]);
        float total = 0.f;
        f32x4 x{};
#pragma unroll
        for (int w = 0; w < kDecodeWaves; ++w) {
          const float c = exp2f(s_top[w][r] - m);
          total += c * s_sum[w][r];
          const f32x4 y = *reinterpret_cast<const f32x4*>(&s_o[w][r][d]);
#pragma unroll
          for (int v = 0; v < 4; ++v) x[v] += c * y[v];
        }
        if (complete) {
          finish<T>(A, g.seq, hq0 + r, d, x, m, total);
        } else {
          *reinterpret_cast<f32x4*>(slot + r * D + d) = x;
          if (d == 0) {
            slot[A.rows * D + r] = m;
            slot[A.rows * (D + 1) + r] = total;
          }
        }
      }
      if (!follows) return;
      g = f;
      have = hi > sub;
    }
  };
  if constexpr (LINE && NT == 1) {
    if (shared) return stream(std::integral_constant<int, 0>{});
  }
  stream(std::integral_constant<int, kNontemporal>{});
}

// The shares of an item that several workgroups took, joined in the order of the line by the
// workgroups of the item's second share.  x: that share, y: ROWS query heads of the tile.  The
// threads of a row take its dims by four, in sets that take the shares in turn and meet in LDS.
template <typename T, int D, int ROWS>
__global__ __launch_bounds__(256) void k_decode_join(const DecodeArgs A) {
  constexpr int LANES = D / 4, SETS = 256 / LANES / ROWS;
  __shared__ float s_top[ROWS][SETS], s_sum[ROWS][SETS];
  __shared__ __align__(16) float s_o[ROWS][SETS][D];
  const DecodeStart st = A.starts[blockIdx.x];
  if (st.units == 0) return;
  const int w0 = static_cast<int>(st.first / st.share);
  if (static_cast<int>(blockIdx.x) != w0 + 1) return;
  const int parts = static_cast<int>((st.first + st.units - 1) / st.share) - w0 + 1;
  const int h = st.head / A.head_tiles, tile = st.head % A.head_tiles;
  const int tid = threadIdx.x, own = tid / (LANES * SETS), set = tid / LANES % SETS, d = tid % LANES * 4;
  const int r = blockIdx.y * ROWS + own, hq = h * A.G + tile * A.tile_rows + r;
  const bool real = r < min(A.tile_rows, A.G - tile * A.tile_rows);
  // the item's first share is its workgroup's first segment, or its last one
  const int tail = static_cast<int64_t>(w0) * st.share < st.first - kItemUnits ? 1 : 0;
  float m = kLowest, total = 0.f;
  f32x4 o{};
  if (real) {
#pragma unroll 4
    for (int p = set; p < parts; p += SETS) {
      const float* s = A.part + (static_cast<int64_t>(w0 + p) * 2 + (p == 0 ? tail : 0)) * A.slot_floats;
      const float mp = s[A.rows * D + r], lp = s[A.rows * (D + 1) + r];
      const f32x4 y = *reinterpret_cast<const f32x4*>(s + r * D + d);
      const float n = fmaxf(m, mp), keep = exp2f(m - n), c = exp2f(mp - n);
      m = n;
      total = total * keep + c * lp;
#pragma unroll
      for (int v = 0; v < 4; ++v) o[v] = o[v] * keep + c * y[v];
    }
  }
  if constexpr (SETS > 1) {
    *reinterpret_cast<f32x4*>(&s_o[own][set][d]) = o;
    if (d == 0) {
      s_top[own][set] = m;
      s_sum[own][set] = total;
    }
    __syncthreads();
    if (set != 0) return;
#pragma unroll
    for (int x = 1; x < SETS; ++x) m = fmaxf(m, s_top[own][x]);
    o = f32x4{};
    total = 0.f;
#pragma unroll
    for (int x = 0; x < SETS; ++x) {
      const float c = exp2f(s_top[own][x] - m);
      total += c * s_sum[own][x];
      const f32x4 y = *reinterpret_cast<const f32x4*>(&s_o[own][x][d]);
#pragma unroll
      for (int v = 0; v < 4; ++v) o[v] += c * y[v];
    }
  }
  if (real) finish<T>(A, st.seq, hq, d, o, m, total);
}

template <typename T, int D, int NT>
hipError_t launch_rows(const DecodeArgs& A, const DecodePlan& p, hipStream_t stream) {
  const auto kernel = p.split == DecodeSplit::kLine   ? k_decode<T, D, NT, DecodeSplit::kLine>
                      : p.split == DecodeSplit::kItem ? k_decode<T, D, NT, DecodeSplit::kItem>
                                                      : k_decode<T, D, NT, DecodeSplit::kWave>;
  LaunchStatus st;
  st(kernel, dim3(p.wgs), dim3(kThreads), 0, stream, A);
  if (p.split == DecodeSplit::kLine && p.wgs > 1) {
    const auto join = p.join_rows == 1 ? k_decode_join<T, D, 1> : p.join_rows == 2 ? k_decode_join<T, D, 2> : k_decode_join<T, D, 4>;
    st(join, dim3(p.wgs, (p.rows + p.join_rows - 1) / p.join_rows), dim3(256), 0, stream, A);
  }
  return st.err;
}

template <typename T, int D>
hipError_t launch_typed(const DecodeArgs& A, const DecodePlan& p, hipStream_t stream) {
  return p.tile_rows == kDecodeHeadRows ? launch_rows<T, D, 1>(A, p, stream) : launch_rows<T, D, 2>(A, p, stream);
}

}  // namespace

hipError_t launch_decode(const SeqGeom& g, const DecodePlan& p, const DecodeLaunch& a, void* workspace,
                         hipStream_t stream) {
  char* ws = static_cast<char*>(workspace);
  DecodeArgs A{};
  A.g = g;
  A.a = a;
  A.G = p.G;
  A.head_tiles = p.head_tiles;
  A.tile_rows = p.tile_rows;
  A.rows = p.rows;
  A.scale2 = a.scale * 1.44269504088896341f;
  A.part = reinterpret_cast<float*>(ws + p.off_part);
  A.starts = reinterpret_cast<DecodeStart*>(ws + p.off_starts);
  A.slot_floats = static_cast<int>(p.slot_floats);
  if (a.dtype == OMNIMEM_BF16)
    return a.D == 128 ? launch_typed<uint16_t, 128>(A, p, stream) : launch_typed<uint16_t, 64>(A, p, stream);
  return a.D == 128 ? launch_typed<float, 128>(A, p, stream) : launch_typed<float, 64>(A, p, stream);
}

}  // namespace omnimem
