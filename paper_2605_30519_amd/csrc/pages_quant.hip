// pages_quant.hip -- 8-bit pages of the sequence cache for gfx950: new tokens' keys and values quantised
// into them, and tokens read back.
//
// A code c of block b and head h stands for c * s, s the block's and head's scale, one for K and
// one for V.  Scales that are written are powers of two, 2^e with the smallest e >= -110 that
// has |x| <= 448 * 2^e (448: the largest e4m3 number) for the block's finite values x.  A power of two
// changes no e4m3 number's bits but the exponent's, so where a later token needs a larger scale,
// the codes in front of it are rounded again only where they fall below e4m3's normal range, and
// tokens appended one by one end up as those of one append, but for those smallest ones.
#include <type_traits>

#include "device_common.h"
#include "launch.h"
#include "seq_launch.h"

namespace omnimem {
namespace {

typedef uint32_t u32x2 __attribute__((ext_vector_type(2)));

constexpr int kThreads = 256;
constexpr uint32_t kInf = 0x7f800000u;
constexpr int kLowest = -110, kHighest = 120;  // exponents of a scale: its inverse is a normal fp32 number

__device__ __forceinline__ float power(int e) { return __uint_as_float(static_cast<uint32_t>(e + 127) << 23); }

// The exponent of the scale that values of at most |x| need, x by its fp32 bits without the sign.
__device__ __forceinline__ int exponent_for(uint32_t most) {
  return max(static_cast<int>(most >> 23) - 127 - 8 + ((most & 0x7fffffu) > 0x600000u ? 1 : 0), kLowest);
}

// A scale as memory has it, brought into [2^-110, 2^120].
__device__ __forceinline__ float scale_in_range(float s) {
  return s >= power(kLowest) ? fminf(s, power(kHighest)) : power(kLowest);
}

__device__ __forceinline__ int exponent_of(float s) {  // the smallest e with s <= 2^e
  const uint32_t u = __float_as_uint(s);
  return static_cast<int>(u >> 23) - 127 + ((u & 0x7fffffu) != 0 ? 1 : 0);
}

// Four values to four codes, rounded to nearest even; |x| <= 448, or NaN or infinite, which NaN stands for.
__device__ __forceinline__ uint32_t codes4(float a, float b, float c, float d) {
  const int low = __builtin_amdgcn_cvt_pk_fp8_f32(a, b, 0, false);
  return static_cast<uint32_t>(__builtin_amdgcn_cvt_pk_fp8_f32(c, d, low, true));
}

// x * y rounded to odd: a product that fp32 does not hold becomes the one of its two neighbours whose last bit is
// set.  So it stays on its side of the middle of two e4m3 numbers, and they are chosen by the product itself.
__device__ __forceinline__ float times_to_odd(float x, float y) {
  const float p = x * y, off = fmaf(x, y, -p);
  const uint32_t u = __float_as_uint(p), cut = u - ((__float_as_uint(off) ^ u) >> 31);  // towards 0
  return __uint_as_float(off == 0.f ? u : cut | 1);
}

__device__ __forceinline__ void values4(uint32_t codes, float (&x)[4]) {
  const auto low = __builtin_amdgcn_cvt_pk_f32_fp8(codes, false), high = __builtin_amdgcn_cvt_pk_f32_fp8(codes, true);
  x[0] = low[0];
  x[1] = low[1];
  x[2] = high[0];
  x[3] = high[1];
}

__device__ __forceinline__ int row_of_start(const int32_t* starts, int tokens, int s) {
  return min(max(starts[s], 0), tokens);
}

// ---------------------------------------------------------------- append
// A workgroup takes the new tokens of one block and one head, of K and V: it holds them in
// registers, 16 bytes of a row a thread and pass, finds their largest, rounds them by the scale, and, where the
// block's earlier tokens have a smaller scale, those again.  Bound by its bytes where there are many
// blocks: eight chunks of 4,680 tokens, 12 heads, bf16 (345 MB) 68.5 us, 5.0 TB/s (K and V in workgroups of
// their own and 16 values a thread, whose loads lie 32 bytes apart: 84.5; fp32 rows, 64 bytes apart, 39.8 instead
// of 24.1).  Else by the chain of loads that leads to them, the sequence, its rows and page, the rows: 64
// single tokens 5.6 us.
//
// Blocks are numbered through: n rows touch at most n div B + 2 blocks of a contiguous sequence, and
// n div S + n div B + 3 of one in chunks, so with `starts` ascending the numbers from
// base(i) = starts[i] div B + 2 i (+ starts[i] div S + i) on are sequence i's.
//
// Blocks of 128 tokens of 128 dims are 512 threads', which hold 16 KB of K in registers with twice the waves: 345 MB
// of bf16 rows 83.6 -> 78.4 us, 49 MB 15.6 -> 15.0, fp32 123 MB 29.3 -> 27.4; the smaller blocks lose by it (fp32
// ones of 128 x 64 dims, 192 MB, 38.7 -> 40.7).
template <int D, int B>
constexpr int kAppendThreads = D * B > 8192 ? 512 : kThreads;
// Waves a SIMD that registers leave at least: blocks of 64 x 64 need 94, and 97 for fp32 rows without this, which one wave
// less can have (12,288 begun blocks whose scales grow 57.4 us instead of 52.9).
template <int D, int B>
constexpr int kAppendWaves = D * B > 4096 ? 1 : 5;
constexpr int64_t kAppendMaxWgs = 1 << 22;  // more work than that is taken in turns

struct AppendUnits {
  int per_seq, S;  // 2, or 3 with chunks of S tokens (else 0)
};

// The new tokens of a block: its slots [from, to), slot s in row row + s.
struct NewTokens {
  int seq, from, to;
  int64_t block, row;
};

template <int B>
__device__ __forceinline__ bool find_tokens(const SeqGeom& g, const AppendQuantLaunch& a, const AppendUnits& units,
                                            int64_t u, NewTokens& x) {
  const int lane = threadIdx.x % kWave;
  int row0, row1, len;
  int64_t at = 0;  // of the sequence's touched blocks
  if (a.starts == nullptr) {
    x.seq = static_cast<int>(u);
    row0 = x.seq;
    row1 = x.seq + 1;
    len = g.lens[x.seq];
  } else {
    auto base = [&](int start, int i) -> int64_t {
      return static_cast<int64_t>(start / B) + (units.S > 0 ? start / units.S : 0) + static_cast<int64_t>(units.per_seq) * i;
    };
    int lo = 0, hi = g.N;  // a search by all lanes
    while (hi - lo > kWave) {
      const int step = (hi - lo + kWave - 1) / kWave, i = lo + lane * step;
      const uint64_t below = __ballot(i < hi && base(row_of_start(a.starts, a.tokens, min(i, g.N - 1)), i) <= u);
      lo += (max(1, static_cast<int>(__popcll(below))) - 1) * step;
      hi = min(hi, lo + step);
    }
    const int i = min(lo + lane, g.N - 1);
    const int start = row_of_start(a.starts, a.tokens, i), stop = row_of_start(a.starts, a.tokens, i + 1), l = g.lens[i];
    const uint64_t below = __ballot(lo + lane < hi && base(start, i) <= u);
    const int found = max(1, static_cast<int>(__popcll(below))) - 1;
    x.seq = lo + found;
    row0 = __builtin_amdgcn_readlane(start, found);
    row1 = __builtin_amdgcn_readlane(stop, found);
    len = __builtin_amdgcn_readlane(l, found);
    at = u - base(row0, x.seq);
    if (at < 0 || row1 <= row0) return false;
  }
  // of the tokens [first, stop), those in the at-th block that they touch
  const int64_t first = max(static_cast<int64_t>(len) - (row1 - row0), int64_t{0});
  const int64_t stop = min(len, g.cap);
  if (first >= stop) return false;
  const int f = static_cast<int>(first);
  int64_t t0;  // the block's first token
  int room = B;
  if (units.S == 0) {
    x.block = f / B + at;
    t0 = x.block * B;
  } else {
    const int c0 = f / g.S;
    x.block = static_cast<int64_t>(c0) * g.Bpc + (f - c0 * g.S) / B + at;
    if (x.block >= g.M) return false;
    const int b = static_cast<int>(x.block), c = b / g.Bpc, in = (b - c * g.Bpc) * B;
    t0 = static_cast<int64_t>(c) * g.S + in;
    room = min(B, g.S - in);
  }
  if (x.block >= g.M) return false;
  x.from = static_cast<int>(max(first - t0, int64_t{0}));
  x.to = static_cast<int>(min(stop - t0, static_cast<int64_t>(room)));
  x.row = row1 - (len - t0);  // the sequence's last row is its last token
  return x.from < x.to;
}

// The largest of a wave's lanes, in all of them.
__device__ __forceinline__ uint32_t wave_max(uint32_t x) {
  x = max(x, static_cast<uint32_t>(__builtin_amdgcn_update_dpp(0, x, 0x128, 0xf, 0xf, false)));  // row_ror:8, 4, 2, 1
  x = max(x, static_cast<uint32_t>(__builtin_amdgcn_update_dpp(0, x, 0x124, 0xf, 0xf, false)));
  x = max(x, static_cast<uint32_t>(__builtin_amdgcn_update_dpp(0, x, 0x122, 0xf, 0xf, false)));
  x = max(x, static_cast<uint32_t>(__builtin_amdgcn_update_dpp(0, x, 0x121, 0xf, 0xf, false)));
  const auto p = __builtin_amdgcn_permlane16_swap(x, x, false, false);
  x = max(p[0], p[1]);
  const auto q = __builtin_amdgcn_permlane32_swap(x, x, false, false);
  return max(q[0], q[1]);
}

// The largest |x| of 16 bytes of values, as fp32 bits; FINITE: what is not finite left out.
template <typename T, bool FINITE>
__device__ __forceinline__ uint32_t largest(const u32x4 raw) {
  uint32_t most = 0;
#pragma unroll
  for (int i = 0; i < 4; ++i) {
    if constexpr (sizeof(T) == 4) {
      const uint32_t m = raw[i] & 0x7fffffffu;
      most = max(most, FINITE && m >= kInf ? 0u : m);
    } else {
      const uint32_t low = raw[i] << 16 & 0x7fffffffu, high = raw[i] & 0x7fff0000u;
      most = max(most, max(FINITE && low >= kInf ? 0u : low, FINITE && high >= kInf ? 0u : high));
    }
  }
  return most;
}

// Stores past the caches pay for what the 256 MB memory-side cache cannot hold beside what is read:
// 115 MB of codes 71.2 -> 68.3 us, 172 MB 110 -> 101, 86 MB 51.9 both, 14 MB 12.5 -> 12.9.
constexpr int64_t kPastBytes = 96ll << 20;  // written

template <bool PAST, typename U>
__device__ __forceinline__ void store(U x, void* to) {
  if constexpr (PAST) __builtin_nontemporal_store(x, static_cast<U*>(to));
  else *static_cast<U*>(to) = x;
}

// The codes of 16 bytes of values, times inv.
template <bool PAST>
__device__ __forceinline__ void store_codes(uint16_t, const u32x4 raw, float inv, uint8_t* to) {
  float w[8];
#pragma unroll
  for (int e = 0; e < 8; ++e) w[e] = __uint_as_float(e % 2 ? raw[e / 2] & 0xffff0000u : raw[e / 2] << 16) * inv;
  store<PAST>(u32x2{codes4(w[0], w[1], w[2], w[3]), codes4(w[4], w[5], w[6], w[7])}, to);
}
template <bool PAST>
__device__ __forceinline__ void store_codes(float, const u32x4 raw, float inv, uint8_t* to) {
  float w[4];
#pragma unroll
  for (int e = 0; e < 4; ++e) w[e] = __uint_as_float(raw[e]) * inv;
  store<PAST>(codes4(w[0], w[1], w[2], w[3]), to);
}

template <typename T, int D, int B, bool PAST>
__device__ __forceinline__ void append_block(const SeqGeom& g, const AppendQuantLaunch& a, const AppendUnits& units,
                                             int64_t u, int h, uint32_t (&s_most)[2][kAppendThreads<D, B> / kWave],
                                             float2& s_own) {
  constexpr int N = 16 / sizeof(T), LANES = D / N;               // values of 16 bytes, threads of a row
  constexpr int THREADS = kAppendThreads<D, B>, ROWS = THREADS / LANES, PASSES = B / ROWS;
  static_assert(PASSES * ROWS == B, "a block in whole passes");
  const int tid = threadIdx.x, lane = tid % kWave;
  NewTokens x;
  if (!find_tokens<B>(g, a, units, u, x)) return;
  const int page = g.table[static_cast<int64_t>(x.seq) * g.M + x.block];

  const int slot = tid / LANES, dim = tid % LANES * N;
  u32x4 raw[2][PASSES];
#pragma unroll
  for (int kv = 0; kv < 2; ++kv) {
    const T* src = static_cast<const T*>(kv ? a.v : a.k) + static_cast<int64_t>(h) * D + dim;
    const int64_t stride = kv ? a.v_stride : a.k_stride;
#pragma unroll
    for (int p = 0; p < PASSES; ++p) {
      const int s = x.from + slot + p * ROWS;
      raw[kv][p] = u32x4{};
      if (s < x.to) raw[kv][p] = __builtin_nontemporal_load(reinterpret_cast<const u32x4*>(src + (x.row + s) * stride));
    }
  }
  if (page < 0 || page >= g.num_pages) return;
  const int64_t head = static_cast<int64_t>(page) * a.H + h;
  float2* scale_at = reinterpret_cast<float2*>(a.scales) + head;
  if (tid == 0 && x.from > 0) s_own = *scale_at;  // by the thread that will write it

  uint32_t most[2] = {0, 0};
  auto find_most = [&](auto finite) {
#pragma unroll
    for (int kv = 0; kv < 2; ++kv) {
      uint32_t m = 0;
#pragma unroll
      for (int p = 0; p < PASSES; ++p) m = max(m, largest<T, decltype(finite)::value>(raw[kv][p]));
      m = wave_max(m);
      if (lane == 0) s_most[kv][tid / kWave] = m;
    }
    __syncthreads();
#pragma unroll
    for (int kv = 0; kv < 2; ++kv) {
      most[kv] = s_most[kv][0];
#pragma unroll
      for (int w = 1; w < THREADS / kWave; ++w) most[kv] = max(most[kv], s_most[kv][w]);
    }
  };
  find_most(std::false_type{});
  if (max(most[0], most[1]) >= kInf) {  // infinities or NaN among them
    __syncthreads();
    find_most(std::true_type{});
  }

  float2 scale;
#pragma unroll
  for (int kv = 0; kv < 2; ++kv) {
    uint8_t* codes = static_cast<uint8_t*>(kv ? a.v_pages : a.k_pages) + head * B * D;
    int e = exponent_for(most[kv]);
    if (x.from > 0) {
      const float was = scale_in_range(kv ? s_own.y : s_own.x);
      e = max(e, exponent_of(was));
      const float ratio = was * power(-e);
      if (ratio != 1.f) {  // the earlier tokens, by the new scale
        auto again = [&](auto times) {
          for (int c = tid; c < x.from * (D / 16); c += THREADS) {
            u32x4* at = reinterpret_cast<u32x4*>(codes) + c;
            u32x4 w = *at;
#pragma unroll
            for (int i = 0; i < 4; ++i) {
              float y[4];
              values4(w[i], y);
              w[i] = codes4(times(y[0], ratio), times(y[1], ratio), times(y[2], ratio), times(y[3], ratio));
            }
            *at = w;
          }
        };
        // a power of two loses no bit of a code; with the other product there 12,288 blocks of 128 x 128 take 320 us, not 300
        if ((__float_as_uint(was) & 0x7fffffu) == 0) again([](float y, float r) { return y * r; });
        else again(times_to_odd);
      }
    }
    (kv ? scale.y : scale.x) = power(e);
#pragma unroll
    for (int p = 0; p < PASSES; ++p) {
      const int s = x.from + slot + p * ROWS;
      if (s < x.to) store_codes<PAST>(T{}, raw[kv][p], power(-e), codes + s * D + dim);
    }
  }
  if (tid == 0) *scale_at = scale;
}

template <typename T, int D, int B, bool PAST>
__global__ __launch_bounds__((kAppendThreads<D, B>), (kAppendWaves<D, B>)) void k_append_quant(
    const SeqGeom g, const AppendQuantLaunch a, const AppendUnits units, int64_t work) {
  __shared__ uint32_t s_most[2][kAppendThreads<D, B> / kWave];
  __shared__ float2 s_own;
  for (int64_t w = blockIdx.x; w < work; w += gridDim.x) {
    const int64_t u = w / a.H;
    append_block<T, D, B, PAST>(g, a, units, u, static_cast<int>(w - u * a.H), s_most, s_own);
    __syncthreads();
  }
}

template <typename T, bool PAST>
hipError_t launch_append(const SeqGeom& g, const AppendQuantLaunch& a, const AppendUnits& units, int64_t work,
                         hipStream_t stream) {
  const auto kernel = a.D == 128 ? (g.B == 128 ? k_append_quant<T, 128, 128, PAST> : k_append_quant<T, 128, 64, PAST>)
                                 : (g.B == 128 ? k_append_quant<T, 64, 128, PAST> : k_append_quant<T, 64, 64, PAST>);
  const int threads = a.D == 128 && g.B == 128 ? kAppendThreads<128, 128> : kThreads;
  const int64_t wgs = work < kAppendMaxWgs ? work : kAppendMaxWgs;
  return launch_kernel(kernel, dim3(static_cast<unsigned>(wgs)), dim3(threads), 0, stream, g, a, units, work);
}

// ---------------------------------------------------------------- read
// Chunks of 16 bytes of all rows are numbered through, as an append of unquantised tokens does; a
// workgroup looks up its rows' places and fills U * 256 of them, of K and of V.  Bound by its bytes: four
// chunks of 4,680 tokens, 12 heads, bf16 (173 MB) 31.3 us, 5.5 TB/s, into memory that is written again and
// again, 37 into fresh memory; with 16 codes a thread, whose stores lie 32 bytes apart, 32.2, ragged fp32 rows
// (64 bytes apart, 35 MB) 15.8 instead of 11.1.
constexpr int kReadUnroll = 2;  // of 1, 2 and 4: 38.1, 31.1 and 31.9 us
// Stores past the caches: 345 MB of bf16 rows 96.2 -> 91.0 us, 460 MB of fp32 rows 118 -> 115, but 230 MB 56 -> 63.
constexpr int64_t kReadPastBytes = 288ll << 20;  // written

// Codes of 16 bytes of values, and the values, times scale.
template <typename T>
struct Codes;

template <>
struct Codes<uint16_t> {
  uint2 c{};
  __device__ __forceinline__ void load(const void* p) {
    const auto v = __builtin_nontemporal_load(static_cast<const uint64_t*>(p));
    c = make_uint2(static_cast<uint32_t>(v), static_cast<uint32_t>(v >> 32));
  }
  template <bool PAST>
  __device__ __forceinline__ void write(uint16_t* to, float scale) const {
    float x[4], y[4];
    values4(c.x, x);
    values4(c.y, y);
    bf16x8 b;
#pragma unroll
    for (int e = 0; e < 4; ++e) {
      b[e] = static_cast<__bf16>(x[e] * scale);
      b[e + 4] = static_cast<__bf16>(y[e] * scale);
    }
    store<PAST>(b, to);
  }
};

template <>
struct Codes<float> {
  uint32_t c = 0;
  __device__ __forceinline__ void load(const void* p) { c = __builtin_nontemporal_load(static_cast<const uint32_t*>(p)); }
  template <bool PAST>
  __device__ __forceinline__ void write(float* to, float scale) const {
    float x[4];
    values4(c, x);
    store<PAST>(f32x4{x[0] * scale, x[1] * scale, x[2] * scale, x[3] * scale}, to);
  }
};

template <typename T, int U, bool PAST>
__global__ __launch_bounds__(kThreads) void k_read_quant(const SeqGeom g, const ReadQuantLaunch a) {
  constexpr int kChunks = U * kThreads;
  constexpr int N = 16 / sizeof(T);         // values of a chunk
  constexpr int kRows = kChunks / (64 / N) + 2;  // rows of at least one head of 64
  __shared__ int s_seq[kRows], s_page[kRows], s_slot[kRows];
  const int tid = threadIdx.x;
  const int head_shift = 6 + (a.D >> 7) - (N == 8 ? 3 : 2);  // log2 of a head's chunks
  const uint32_t row_chunks = static_cast<uint32_t>(a.H) << head_shift;
  const int64_t total = static_cast<int64_t>(a.tokens) * row_chunks;
  const int64_t c0 = static_cast<int64_t>(blockIdx.x) * kChunks;
  const int t0 = static_cast<int>(c0 / row_chunks);
  const uint32_t in0 = static_cast<uint32_t>(c0 - static_cast<int64_t>(t0) * row_chunks);  // the first chunk in its row
  const uint32_t mine = static_cast<uint32_t>(min(total - c0, int64_t{kChunks}));
  const int t1 = t0 + static_cast<int>((in0 + mine - 1) / row_chunks);
  for (int r = tid; r <= t1 - t0; r += kThreads) {
    const int seq = a.starts == nullptr ? t0 + r : -1;
    s_seq[r] = seq;
    s_slot[r] = seq < 0 ? 0 : a.first != nullptr ? a.first[seq] : max(g.lens[seq], -1) - 1;
  }
  if (a.starts != nullptr) {
    // s_slot: the row's token; one that is out of a token's range is -1
    __syncthreads();
    for (int s = tid; s < g.N; s += kThreads) {
      const int start = row_of_start(a.starts, a.tokens, s), stop = row_of_start(a.starts, a.tokens, s + 1);
      const int len = g.lens[s];
      const int64_t token0 = a.first != nullptr ? int64_t{a.first[s]} - start : int64_t{len} - stop;
      const int to = min(stop, t1 + 1);
      for (int t = max(start, t0); t < to; ++t) {
        const int64_t token = token0 + t;
        s_seq[t - t0] = s;
        s_slot[t - t0] = token >= 0 && token < len ? static_cast<int>(token) : -1;
      }
    }
    __syncthreads();
  }
  for (int r = tid; r <= t1 - t0; r += kThreads) {
    const int s = s_seq[r], t = s_slot[r];
    int page = -2, slot = 0;  // -2: a row of no sequence, left alone; -1: zeros
    if (s >= 0) {
      page = -1;
      if (t >= 0 && t < min(a.starts == nullptr ? g.lens[s] : t + 1, g.cap)) {
        const int c = t / g.S, off = t - c * g.S;
        const int at = g.table[static_cast<int64_t>(s) * g.M + static_cast<int64_t>(c) * g.Bpc + off / g.B];
        if (at >= 0 && at < g.num_pages) {
          page = at;
          slot = off % g.B;
        }
      }
    }
    s_page[r] = page;
    s_slot[r] = slot;
  }
  __syncthreads();
  Codes<T> kk[U], vv[U];
  float2 scale[U];
  int64_t to[U];
#pragma unroll
  for (int u = 0; u < U; ++u) {
    const uint32_t c = u * kThreads + tid;
    to[u] = -1;
    scale[u] = make_float2(0.f, 0.f);
    if (c >= mine) continue;
    const uint32_t row = (in0 + c) / row_chunks, in = in0 + c - row * row_chunks;
    const int page = s_page[row];
    if (page == -2) continue;
    to[u] = (c0 + c) * N;
    if (page < 0) continue;
    const uint32_t h = in >> head_shift;
    const int64_t head = static_cast<int64_t>(page) * a.H + h;
    const int64_t at = (head * g.B + s_slot[row]) * a.D + (in - (h << head_shift)) * N;
    kk[u].load(static_cast<const uint8_t*>(a.k_pages) + at);
    vv[u].load(static_cast<const uint8_t*>(a.v_pages) + at);
    scale[u] = *reinterpret_cast<const float2*>(a.scales + head * 2);
  }
#pragma unroll
  for (int u = 0; u < U; ++u) {
    if (to[u] < 0) continue;
    kk[u].template write<PAST>(static_cast<T*>(a.out_k) + to[u], scale[u].x);
    vv[u].template write<PAST>(static_cast<T*>(a.out_v) + to[u], scale[u].y);
  }
}

}  // namespace

hipError_t launch_append_kv_quant(const SeqGeom& g, const AppendQuantLaunch& a, hipStream_t stream) {
  const AppendUnits units{g.S == g.B ? 2 : 3, g.S == g.B ? 0 : g.S};
  const int64_t blocks = a.starts == nullptr ? g.N
                                             : static_cast<int64_t>(a.tokens) / g.B + (units.S > 0 ? a.tokens / units.S : 0) +
                                                   static_cast<int64_t>(units.per_seq) * g.N;
  const int64_t work = blocks * a.H;
  const bool past = static_cast<int64_t>(a.tokens) * a.H * a.D * 2 > kPastBytes;
  const auto launch = a.dtype == OMNIMEM_BF16 ? (past ? launch_append<uint16_t, true> : launch_append<uint16_t, false>)
                                              : (past ? launch_append<float, true> : launch_append<float, false>);
  return launch(g, a, units, work, stream);
}

hipError_t launch_read_kv_quant(const SeqGeom& g, const ReadQuantLaunch& a, hipStream_t stream) {
  const int64_t values = static_cast<int64_t>(a.tokens) * a.H * a.D, size = a.dtype == OMNIMEM_BF16 ? 2 : 4;
  constexpr int64_t kBytes = kReadUnroll * kThreads * 16;  // of K that a workgroup writes
  const int64_t wgs = (values * size + kBytes - 1) / kBytes;
  if (wgs > 0x7fffffff) return hipErrorInvalidConfiguration;
  const bool past = 2 * values * size > kReadPastBytes;
  constexpr int U = kReadUnroll;
  const auto kernel = a.dtype == OMNIMEM_BF16 ? (past ? k_read_quant<uint16_t, U, true> : k_read_quant<uint16_t, U, false>)
                                              : (past ? k_read_quant<float, U, true> : k_read_quant<float, U, false>);
  return launch_kernel(kernel, dim3(static_cast<unsigned>(wgs)), dim3(kThreads), 0, stream, g, a);
}

}  // namespace omnimem
