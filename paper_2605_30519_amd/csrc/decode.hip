// decode.hip -- attention of one new token per sequence over a paged cache, for gfx950:
//   O[i][h] = sum_t softmax_t(scale <q_i, k_t>) v_t over the tokens of sequence i.
//
// Every key and value is used by the G query heads of its head alone, 2 G flops a byte of
// bf16, so the kernel is bound by the stream of K and V from memory.  It is built to keep that
// stream full: no LDS and no barrier between the loads and the products, tiles of 8 KB of
// K and 8 KB of V a wave straight into MFMA operand registers, the next tile's loads issued
// as soon as the registers of the present one are read.
//
// Split.  An item is a (sequence, key/value head, tile of up to 32 query heads); its 64-token
// units follow one another on a line of all items' units, and workgroup w takes the equal
// share [w q, (w + 1) q) of it, over item boundaries, so that any mix of lengths loads
// every workgroup alike and lengths stay on the device (a captured graph replays with others).
// The four waves take a segment's units in turn and meet in LDS; an item that several
// workgroups share leaves (O, max, sum) a share in the workspace, which k_decode_join adds
// up in the order of the line.
#include <float.h>

#include "device_common.h"
#include "launch.h"
#include "seq_launch.h"

namespace omnimem {
namespace {

constexpr int kThreads = kDecodeWaves * kWave;
constexpr int kMinUnits = 4;      // units of a share: one for each wave
constexpr float kLowest = -FLT_MAX;  // below every score: a row without keys keeps sum 0
constexpr int kNontemporal = 2;   // cache policy of a buffer load

struct DecodeArgs {
  SeqGeom g;
  DecodeLaunch a;
  int G, head_tiles, tile_rows, rows;
  float scale2;  // scale * log2 e: the softmax runs on exp2
  float* part;
  DecodeStart* starts;
  int slot_floats;
};

// Tokens [begin, end) of a sequence and the blocks that hold them.
struct Span {
  int begin, end, block, units;
};

__device__ __forceinline__ Span span_of(const SeqGeom& g, int window, int len) {
  Span s;
  s.end = min(max(len, 0), g.cap);
  s.begin = window > 0 ? max(0, s.end - window) : 0;
  s.block = s.begin / g.S * g.Bpc + s.begin % g.S / g.B;
  const int last = s.end > 0 ? (s.end - 1) / g.S * g.Bpc + (s.end - 1) % g.S / g.B : -1;
  s.units = s.end > 0 ? (last + 1 - s.block) * (g.B / kUnitTokens) : 0;
  return s;
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
  typedef uint32_t vraw __attribute__((ext_vector_type(VW / 2)));  // a lane's V dims of one key
  u32x4 k[KB][2][QS];
  vraw v[KB][8];

  __device__ __forceinline__ static int key(int t, int r, int j) { return 32 * (t / 2) + 8 * j + 4 * (t % 2) + r; }

  __device__ __forceinline__ void load_k(__amdgpu_buffer_rsrc_t rs, int i, int j) {
    const int at = (8 * (i / 4) + i % 4) * ROW + j * 16;
#pragma unroll
    for (int b = 0; b < KB; ++b)
#pragma unroll
      for (int a = 0; a < 2; ++a)
#pragma unroll
        for (int s = 0; s < QS; ++s)
          k[b][a][s] = __builtin_amdgcn_raw_buffer_load_b128(rs, at + (32 * b + 4 * a) * ROW + s * 64, 0, kNontemporal);
  }
  __device__ __forceinline__ void load_v(__amdgpu_buffer_rsrc_t rs, int i, int j) {
    const int at = 8 * j * ROW + i * VW * 2;
#pragma unroll
    for (int b = 0; b < KB; ++b)
#pragma unroll
      for (int e = 0; e < 8; ++e) {
        const int from = at + (32 * b + e) * ROW;
        if constexpr (VW == 8) v[b][e] = __builtin_amdgcn_raw_buffer_load_b128(rs, from, 0, kNontemporal);
        else v[b][e] = __builtin_amdgcn_raw_buffer_load_b64(rs, from, 0, kNontemporal);
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
  // O^T row 16-dim tiles m: dims VW * (row of the tile) + m.  A word of the A operand holds dim m
  // of two keys, picked out of the keys' rows.
  template <int NT>
  __device__ __forceinline__ void pv(const f32x4 (&p)[NT][RT], f32x4 (&o)[NT][VW]) const {
#pragma unroll
    for (int b = 0; b < KB; ++b) {
      bf16x8 pb[NT];
#pragma unroll
      for (int n = 0; n < NT; ++n)
#pragma unroll
        for (int e = 0; e < 8; ++e) pb[n][e] = static_cast<__bf16>(p[n][2 * b + e / 4][e % 4]);
#pragma unroll
      for (int m = 0; m < VW; ++m) {
        u32x4 w;
#pragma unroll
        for (int e = 0; e < 4; ++e)
          w[e] = __builtin_amdgcn_perm(v[b][2 * e + 1][m / 2], v[b][2 * e][m / 2], m % 2 ? 0x07060302u : 0x05040100u);
#pragma unroll
        for (int n = 0; n < NT; ++n)
          o[n][m] = __builtin_amdgcn_mfma_f32_16x16x32_bf16(__builtin_bit_cast(bf16x8, w), pb[n], o[n][m], 0, 0, 0);
      }
    }
  }
  // first of the four consecutive dims that tiles 4 x .. 4 x + 3 hold of their row
  __device__ __forceinline__ static int dim(int row, int x) { return VW * row + 4 * x; }
};

template <int D>
struct Tile<float, D> {
  static constexpr int ROW = D * 4, KEYS = 8192 / ROW, RT = KEYS / 16, QS = ROW / 64, VW = D / 16;
  u32x4 k[RT][QS];
  u32x4 v[RT][4][VW / 4];

  __device__ __forceinline__ static int key(int t, int r, int j) { return 16 * t + 4 * j + r; }

  __device__ __forceinline__ void load_k(__amdgpu_buffer_rsrc_t rs, int i, int j) {
    const int at = i * ROW + j * 16;
#pragma unroll
    for (int t = 0; t < RT; ++t)
#pragma unroll
      for (int s = 0; s < QS; ++s)
        k[t][s] = __builtin_amdgcn_raw_buffer_load_b128(rs, at + 16 * t * ROW + s * 64, 0, kNontemporal);
  }
  __device__ __forceinline__ void load_v(__amdgpu_buffer_rsrc_t rs, int i, int j) {
    const int at = 4 * j * ROW + i * 16;
#pragma unroll
    for (int t = 0; t < RT; ++t)
#pragma unroll
      for (int r = 0; r < 4; ++r)
#pragma unroll
        for (int x = 0; x < VW / 4; ++x)
          v[t][r][x] = __builtin_amdgcn_raw_buffer_load_b128(rs, at + (16 * t + r) * ROW + x * 256, 0, kNontemporal);
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

template <typename T, int D, int NT>
__global__ __launch_bounds__(kThreads, NT == 1 ? 3 : 2) void k_decode(const DecodeArgs A) {
  using L = Tile<T, D>;
  constexpr int RT = L::RT, VW = L::VW, QS = L::QS;
  __shared__ __align__(16) float s_o[kDecodeWaves][NT * 16][D];
  __shared__ float s_top[kDecodeWaves][NT * 16], s_sum[kDecodeWaves][NT * 16];
  __shared__ int s_scan[kDecodeWaves];
  __shared__ int s_seq, s_before;
  const int tid = threadIdx.x, lane = tid % kWave;
  const int wave = __builtin_amdgcn_readfirstlane(tid / kWave);
  const int i = lane % 16, j = lane / 16;
  const int HH = A.a.H * A.head_tiles;
  const int N = A.g.N;

  // the line: units of every sequence, its total, and the sequence that this share begins in
  const int per = (N + kThreads - 1) / kThreads;
  const int first_seq = min(tid * per, N), last_seq = min(first_seq + per, N);
  int mine = 0;
  for (int s = first_seq; s < last_seq; ++s) mine += span_of(A.g, A.a.window, A.g.lens[s]).units;
  int all;
  const int before = block_exclusive_scan<kThreads>(mine, s_scan, all);
  const int64_t line = static_cast<int64_t>(all) * HH;
  const int share = static_cast<int>(max(static_cast<int64_t>(kMinUnits), (line + gridDim.x - 1) / gridDim.x));
  int64_t pos = static_cast<int64_t>(blockIdx.x) * share;
  if (pos < line) {
    int x = static_cast<int>(pos / HH) - before;
    if (x >= 0 && x < mine) {
      int s = first_seq, b = before;
      for (;; ++s) {
        const int u = span_of(A.g, A.a.window, A.g.lens[s]).units;
        if (x < u) break;
        x -= u;
        b += u;
      }
      s_seq = s;
      s_before = b;
    }
  }
  __syncthreads();
  // sequences without tokens, and rows of zeros for them
  for (int s = blockIdx.x; s < N; s += gridDim.x) {
    if (span_of(A.g, A.a.window, A.g.lens[s]).units != 0) continue;
    for (int e = tid; e < A.a.Hq * (D / 4); e += kThreads)
      finish<T>(A, s, e / (D / 4), e % (D / 4) * 4, f32x4{}, 0.f, 0.f);
  }
  if (pos >= line) {
    if (tid == 0) A.starts[blockIdx.x] = DecodeStart{};
    return;
  }
  int left = static_cast<int>(min(static_cast<int64_t>(share), line - pos));
  int seq = __builtin_amdgcn_readfirstlane(s_seq);
  Span sp = span_of(A.g, A.a.window, A.g.lens[seq]);
  int head = static_cast<int>((pos - static_cast<int64_t>(s_before) * HH) / sp.units);
  int unit = static_cast<int>((pos - static_cast<int64_t>(s_before) * HH) % sp.units);
  if (tid == 0) {
    DecodeStart st{};
    if (unit > 0) st = DecodeStart{pos - unit, sp.units, seq, head, share};
    A.starts[blockIdx.x] = st;
  }

  bool first = true;  // the share's first segment
  while (left > 0) {
    const int stop = min(sp.units, unit + left);
    const int h = head / A.head_tiles, tile = head % A.head_tiles;
    const int hq0 = h * A.G + tile * A.tile_rows;
    const int rows = min(A.tile_rows, A.G - tile * A.tile_rows);

    u32x4 q[NT][QS];
#pragma unroll
    for (int n = 0; n < NT; ++n) {
      const bool real = n * 16 + i < rows;
      const char* at = reinterpret_cast<const char*>(static_cast<const T*>(A.a.q) + seq * A.a.q_stride +
                                                     static_cast<int64_t>(hq0 + (real ? n * 16 + i : 0)) * D) +
                       j * 16;
#pragma unroll
      for (int s = 0; s < QS; ++s) {
        q[n][s] = *reinterpret_cast<const u32x4*>(at + s * 64);
        if (!real) q[n][s] = u32x4{};
      }
    }
    f32x4 o[NT][VW] = {};
    float top[NT], sum[NT];
#pragma unroll
    for (int n = 0; n < NT; ++n) {
      top[n] = kLowest;
      sum[n] = 0.f;
    }

    // The wave's units, 64 looked up at a time: lane l has the l-th one's page, first token
    // row, and rows in use.
    int next = unit + wave;
    uint64_t mask = 0;
    int l_page = 0, l_row = 0, l_lo = 0, l_hi = 0;
    const int32_t* table = A.g.table + static_cast<int64_t>(seq) * A.g.M;
    int lo = 0, hi = 0, sub = 0;   // the tile's unit: rows in use, rows before the tile
    int64_t row = 0;               // the unit's first row in the pools
    auto advance = [&]() -> bool {
      if (sub + L::KEYS < hi) {
        sub += L::KEYS;
        return true;
      }
      while (mask == 0) {
        if (next >= stop) {
          lo = hi = sub = 0;  // a tile of no rows
          return false;
        }
        const int u = next + lane * kDecodeWaves;
        bool ok = u < stop;
        if (ok) {
          const int b = sp.block + u / (A.g.B / kUnitTokens);
          l_row = u % (A.g.B / kUnitTokens) * kUnitTokens;
          const int in = b % A.g.Bpc * A.g.B + l_row;
          const int tok = b / A.g.Bpc * A.g.S + in;
          l_page = table[b];
          l_hi = min(kUnitTokens, min(A.g.S - in, sp.end - tok));
          l_lo = max(0, sp.begin - tok);
          ok = l_page >= 0 && l_page < A.g.num_pages && l_lo < l_hi;
        }
        mask = __ballot(ok);
        next += kWave * kDecodeWaves;
      }
      const int at = __builtin_ctzll(mask);
      mask &= mask - 1;
      lo = __builtin_amdgcn_readlane(l_lo, at);
      hi = __builtin_amdgcn_readlane(l_hi, at);
      row = (static_cast<int64_t>(__builtin_amdgcn_readlane(l_page, at)) * A.a.H + h) * A.g.B +
            __builtin_amdgcn_readlane(l_row, at);
      sub = lo / L::KEYS * L::KEYS;
      return true;
    };
    auto rsrc = [&](const void* pool) {
      return tile_rsrc(static_cast<const char*>(pool) + (row + sub) * L::ROW, max(0, min(hi - sub, L::KEYS)) * L::ROW);
    };

    L t;
    bool have = advance();
    t.load_k(rsrc(A.a.k_pages), i, j);
    t.load_v(rsrc(A.a.v_pages), i, j);
    while (have) {
      const int clo = lo - sub, chi = hi - sub;  // rows of the tile in use
      f32x4 s[NT][RT];
#pragma unroll
      for (int n = 0; n < NT; ++n)
#pragma unroll
        for (int r = 0; r < RT; ++r) s[n][r] = t.qk(q[n], r);
      have = advance();
      t.load_k(rsrc(A.a.k_pages), i, j);
      const bool whole = clo <= 0 && chi >= L::KEYS;
#pragma unroll
      for (int n = 0; n < NT; ++n) {
        float m = kLowest;
#pragma unroll
        for (int r = 0; r < RT; ++r)
#pragma unroll
          for (int e = 0; e < 4; ++e) {
            s[n][r][e] *= A.scale2;
            if (!whole) {
              const int key = L::key(r, e, j);
              if (key < clo || key >= chi) s[n][r][e] = -INFINITY;
            }
            m = fmaxf(m, s[n][r][e]);
          }
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
      t.load_v(rsrc(A.a.v_pages), i, j);
    }

    // the waves' results meet
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
    __syncthreads();
    const bool complete = unit == 0 && stop == sp.units;
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
        const float f = exp2f(s_top[w][r] - m);
        total += f * s_sum[w][r];
        const f32x4 y = *reinterpret_cast<const f32x4*>(&s_o[w][r][d]);
#pragma unroll
        for (int c = 0; c < 4; ++c) x[c] += f * y[c];
      }
      if (complete) {
        finish<T>(A, seq, hq0 + r, d, x, m, total);
      } else {
        *reinterpret_cast<f32x4*>(slot + r * D + d) = x;
        if (d == 0) {
          slot[A.rows * D + r] = m;
          slot[A.rows * (D + 1) + r] = total;
        }
      }
    }
    __syncthreads();
    first = false;
    left -= stop - unit;
    unit = stop;
    if (left > 0 && unit == sp.units) {
      unit = 0;
      if (++head == HH) {
        head = 0;
        do sp = span_of(A.g, A.a.window, A.g.lens[++seq]);
        while (sp.units == 0);
      }
    }
  }
}

// The shares of an item that several workgroups took, joined in the order of the line by the
// workgroup of the item's second share; x: the share, y: the query head of the tile.
template <typename T, int D>
__global__ __launch_bounds__(256) void k_decode_join(const DecodeArgs A) {
  constexpr int LANES = D / 4, SETS = 256 / LANES;
  __shared__ float s_red[4];
  __shared__ float s_sum[SETS];
  __shared__ __align__(16) float s_o[SETS][D];
  const DecodeStart st = A.starts[blockIdx.x];
  if (st.units == 0) return;
  const int64_t w0 = st.first / st.share;
  if (static_cast<int64_t>(blockIdx.x) != w0 + 1) return;
  const int parts = static_cast<int>((st.first + st.units - 1) / st.share - w0) + 1;
  const int h = st.head / A.head_tiles, tile = st.head % A.head_tiles;
  const int r = blockIdx.y, hq = h * A.G + tile * A.tile_rows + r;
  if (r >= min(A.tile_rows, A.G - tile * A.tile_rows)) return;
  const int tid = threadIdx.x, set = tid / LANES, d = tid % LANES * 4;
  // the item's first share is its workgroup's first segment, or its last one
  const int tail = w0 * st.share < st.first ? 1 : 0;
  auto slot = [&](int p) { return A.part + ((w0 + p) * 2 + (p == 0 ? tail : 0)) * A.slot_floats; };

  float m = kLowest;
  for (int p = tid; p < parts; p += 256) m = fmaxf(m, slot(p)[A.rows * D + r]);
#pragma unroll
  for (int x = 1; x < kWave; x <<= 1) m = fmaxf(m, __shfl_xor(m, x));
  if (tid % kWave == 0) s_red[tid / kWave] = m;
  __syncthreads();
  m = fmaxf(fmaxf(s_red[0], s_red[1]), fmaxf(s_red[2], s_red[3]));
  float total = 0.f;
  f32x4 o{};
#pragma unroll 4
  for (int p = set; p < parts; p += SETS) {
    const float* s = slot(p);
    const float f = exp2f(s[A.rows * D + r] - m);
    total += f * s[A.rows * (D + 1) + r];
    const f32x4 y = *reinterpret_cast<const f32x4*>(s + r * D + d);
#pragma unroll
    for (int c = 0; c < 4; ++c) o[c] += f * y[c];
  }
  *reinterpret_cast<f32x4*>(&s_o[set][d]) = o;
  if (d == 0) s_sum[set] = total;
  __syncthreads();
  if (set != 0) return;
  o = f32x4{};
  total = 0.f;
  for (int x = 0; x < SETS; ++x) {
    total += s_sum[x];
    const f32x4 y = *reinterpret_cast<const f32x4*>(&s_o[x][d]);
#pragma unroll
    for (int c = 0; c < 4; ++c) o[c] += y[c];
  }
  finish<T>(A, st.seq, hq, d, o, m, total);
}

template <typename T, int D>
hipError_t launch_typed(const DecodeArgs& A, const DecodePlan& p, hipStream_t stream) {
  LaunchStatus st;
  if (p.tile_rows == kDecodeHeadRows)
    st(k_decode<T, D, 1>, dim3(p.wgs), dim3(kThreads), 0, stream, A);
  else
    st(k_decode<T, D, 2>, dim3(p.wgs), dim3(kThreads), 0, stream, A);
  if (p.wgs > 1) st(k_decode_join<T, D>, dim3(p.wgs, p.rows), dim3(256), 0, stream, A);
  return st.err;
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
