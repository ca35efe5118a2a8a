// pages_quant.hip -- 8-bit pages of the sequence cache for gfx950: new tokens' keys and values quantised
// into them, and tokens read back.
//
// A code c of block b and head h stands for c * s, s the block's and head's scale, one for K and
// one for V.  Scales that are written are powers of two, 2^e with the smallest e >= -110 that
// has |x| <= 448 * 2^e (448: the largest e4m3 number) for the block's finite values x.  A power of two
// changes no e4m3 number's bits but the exponent's, so where a later token needs a larger scale,
// the codes in front of it are rounded again only where they fall below e4m3's normal range, and
// tokens appended one by one end up as those of one append, but for those smallest ones.
#include "device_common.h"
#include "launch.h"
#include "seq_launch.h"

namespace omnimem {
namespace {

constexpr int kThreads = 256;
constexpr uint32_t kInf = 0x7f800000u;
constexpr int kLowest = -110, kHighest = 120;  // exponents of a scale: its inverse is a normal fp32 number

__device__ __forceinline__ float power(int e) { return __uint_as_float(static_cast<uint32_t>(e + 127) << 23); }

// The exponent of the scale that values of at most |x| need, x by its fp32 bits without the sign.
__device__ __forceinline__ int exponent_for(uint32_t most) {
  return max(static_cast<int>(most >> 23) - 127 - 8 + ((most & 0x7fffffu) > 0x600000u ? 1 : 0), kLowest);
}

// A scale as memory has it, brought into [2^-110, 2^120].
__device__ __forceinline__ float scale_in_range(float s) { return s >= power(kLowest) ? fminf(s, power(kHighest)) : power(kLowest); }

__device__ __forceinline__ int exponent_of(float s) {  // the smallest e with s <= 2^e
  const uint32_t u = __float_as_uint(s);
  return static_cast<int>(u >> 23) - 127 + ((u & 0x7fffffu) != 0 ? 1 : 0);
}

// Four values to four codes, rounded to nearest even; |x| <= 448, or NaN or infinite, which NaN stands for.
__device__ __forceinline__ uint32_t codes4(float a, float b, float c, float d) {
  const int low = __builtin_amdgcn_cvt_pk_fp8_f32(a, b, 0, false);
  return static_cast<uint32_t>(__builtin_amdgcn_cvt_pk_fp8_f32(c, d, low, true));
}

__device__ __forceinline__ void values4(uint32_t codes, float (&x)[4]) {
  const auto low = __builtin_amdgcn_cvt_pk_f32_fp8(codes, false), high = __builtin_amdgcn_cvt_pk_f32_fp8(codes, true);
  x[0] = low[0];
  x[1] = low[1];
  x[2] = high[0];
  x[3] = high[1];
}

__device__ __forceinline__ int row_of_start(const int32_t* starts, int tokens, int s) { return min(max(starts[s], 0), tokens); }

// ---------------------------------------------------------------- append
// A workgroup takes the new tokens of one block, of one head, of K or V: it holds them in
// registers, 16 values of a row a thread, finds their largest, rounds them by the scale, and, where the
// block's earlier tokens have a smaller scale, those again.
//
// Blocks are numbered through: n rows touch at most n div B + 2 blocks of a contiguous sequence, and
// n div S + n div B + 3 of one in chunks, so with `starts` ascending the numbers from
// base(i) = starts[i] div B + 2 i (+ starts[i] div S + i) on are sequence i's.
constexpr int64_t kAppendMaxWgs = 1 << 22;  // more work than that is taken in turns

struct AppendUnits {
  int per_seq, S;  // 2, or 3 with chunks of S tokens (else 0)
};

template <typename T, int D, int B>
__device__ __forceinline__ void append_block(const SeqGeom& g, const AppendQuantLaunch& a, const AppendUnits& units, int64_t w,
                                             uint32_t (&s_most)[kThreads / kWave]) {
  constexpr int LANES = D / 16, ROWS = kThreads / LANES, ITEMS = B / ROWS;  // threads of a row, rows of a pass, passes
  constexpr int VECS = 16 * sizeof(T) / 16;
  static_assert(ITEMS * ROWS == B, "a block in whole passes");
  const int tid = threadIdx.x, lane = tid % kWave;
  const int64_t w0 = w / a.H, u = w0 / 2;
  const int h = static_cast<int>(w - w0 * a.H), value = static_cast<int>(w0 % 2);

  // the sequence
  int seq, row0, row1;
  int64_t block_at = 0;  // of the sequence's touched blocks
  if (a.starts == nullptr) {
    seq = static_cast<int>(u);
    row0 = seq;
    row1 = seq + 1;
  } else {
    auto base = [&](int i) -> int64_t {
      const int s = row_of_start(a.starts, a.tokens, i);
      return static_cast<int64_t>(s / B) + (units.S > 0 ? s / units.S : 0) + static_cast<int64_t>(units.per_seq) * i;
    };
    int lo = 0, hi = g.N;
    while (hi - lo > 1) {
      const int step = (hi - lo + kWave - 1) / kWave;
      const int at = lo + lane * step;
      const uint64_t below = __ballot(lane * step < hi - lo && base(min(at, g.N - 1)) <= u);
      const int count = max(1, static_cast<int>(__popcll(below)));
      lo += (count - 1) * step;
      hi = min(hi, lo + step);
    }
    seq = __builtin_amdgcn_readfirstlane(lo);
    block_at = u - base(seq);
    row0 = row_of_start(a.starts, a.tokens, seq);
    row1 = row_of_start(a.starts, a.tokens, seq + 1);
  }
  if (block_at < 0 || row1 <= row0) return;

  // its block: of the tokens [first, end), those in the block_at-th block that they touch
  const int64_t end = g.lens[seq];
  const int64_t first = max(end - (row1 - row0), int64_t{0});
  const int64_t stop = min(end, static_cast<int64_t>(g.cap));
  if (first >= stop) return;
  const int f = static_cast<int>(first);
  const int f_chunk = f / g.S;
  const int64_t block = static_cast<int64_t>(f_chunk) * g.Bpc + (f - f_chunk * g.S) / B + block_at;
  if (block >= g.M) return;
  const int chunk = static_cast<int>(block / g.Bpc), in = static_cast<int>(block - static_cast<int64_t>(chunk) * g.Bpc) * B;
  const int64_t t0 = static_cast<int64_t>(chunk) * g.S + in;  // the block's first token
  const int from = static_cast<int>(max(first - t0, int64_t{0}));
  const int to = static_cast<int>(min(min(stop - t0, static_cast<int64_t>(g.S - in)), static_cast<int64_t>(B)));
  if (from >= to) return;
  const int page = g.table[static_cast<int64_t>(seq) * g.M + block];
  if (page < 0 || page >= g.num_pages) return;
  // the row of slot s: the sequence's last row is its last token
  const int64_t row = row1 - (end - t0);
  const T* src = static_cast<const T*>(value ? a.v : a.k) + static_cast<int64_t>(h) * D;
  const int64_t stride = value ? a.v_stride : a.k_stride;
  float* scale_at = a.scales + (static_cast<int64_t>(page) * a.H + h) * 2 + value;
  const float old = from > 0 ? *scale_at : 0.f;
  uint8_t* codes = static_cast<uint8_t*>(value ? a.v_pages : a.k_pages) + (static_cast<int64_t>(page) * a.H + h) * B * D;

  const int slot = from + tid / LANES, dim = tid % LANES * 16;
  uint4 raw[ITEMS][VECS];
  uint32_t most = 0;
#pragma unroll
  for (int x = 0; x < ITEMS; ++x) {
    const int s = slot + x * ROWS;
#pragma unroll
    for (int v = 0; v < VECS; ++v) raw[x][v] = make_uint4(0, 0, 0, 0);
    if (s < to) {
      const uint4* p = reinterpret_cast<const uint4*>(src + (row + s) * stride + dim);
#pragma unroll
      for (int v = 0; v < VECS; ++v) raw[x][v] = load_once(p + v);
    }
  }
#pragma unroll
  for (int x = 0; x < ITEMS; ++x)
#pragma unroll
    for (int v = 0; v < VECS; ++v) {
      float w[Vec16<T>::N];
      Vec16<T>::widen(raw[x][v], w);
#pragma unroll
      for (int e = 0; e < Vec16<T>::N; ++e) {
        const uint32_t m = __float_as_uint(w[e]) & 0x7fffffffu;
        most = max(most, m < kInf ? m : 0u);
      }
    }
#pragma unroll
  for (int m = 1; m < kWave; m <<= 1) most = max(most, static_cast<uint32_t>(__shfl_xor(static_cast<int>(most), m)));
  if (lane == 0) s_most[tid / kWave] = most;
  __syncthreads();  // and every thread has read the old scale
#pragma unroll
  for (int w = 0; w < kThreads / kWave; ++w) most = max(most, s_most[w]);

  int e = exponent_for(most);
  if (from > 0) {
    const float was = scale_in_range(old);
    e = max(e, exponent_of(was));
    const float ratio = was * power(-e);
    if (ratio != 1.f) {  // the earlier tokens, by the new scale
      for (int x = tid; x < from * LANES; x += kThreads) {
        uint4* p = reinterpret_cast<uint4*>(codes) + x;
        uint4 c = *p;
        uint32_t* cw = &c.x;
#pragma unroll
        for (int w = 0; w < 4; ++w) {
          float y[4];
          values4(cw[w], y);
          cw[w] = codes4(y[0] * ratio, y[1] * ratio, y[2] * ratio, y[3] * ratio);
        }
        *p = c;
      }
    }
  }
  const float inv = power(-e);
#pragma unroll
  for (int x = 0; x < ITEMS; ++x) {
    const int s = slot + x * ROWS;
    if (s >= to) continue;
    float w[16];
#pragma unroll
    for (int v = 0; v < VECS; ++v) {
      float y[Vec16<T>::N];
      Vec16<T>::widen(raw[x][v], y);
#pragma unroll
      for (int i = 0; i < Vec16<T>::N; ++i) w[v * Vec16<T>::N + i] = y[i] * inv;
    }
    const uint4 c = make_uint4(codes4(w[0], w[1], w[2], w[3]), codes4(w[4], w[5], w[6], w[7]),
                               codes4(w[8], w[9], w[10], w[11]), codes4(w[12], w[13], w[14], w[15]));
    *reinterpret_cast<uint4*>(codes + s * D + dim) = c;
  }
  if (tid == 0) *scale_at = power(e);
}

template <typename T, int D, int B>
__global__ __launch_bounds__(kThreads) void k_append_quant(const SeqGeom g, const AppendQuantLaunch a, const AppendUnits units,
                                                        int64_t work) {
  __shared__ uint32_t s_most[kThreads / kWave];
  for (int64_t w = blockIdx.x; w < work; w += gridDim.x) {
    append_block<T, D, B>(g, a, units, w, s_most);
    __syncthreads();
  }
}

template <typename T>
hipError_t launch_append_typed(const SeqGeom& g, const AppendQuantLaunch& a, const AppendUnits& units, int64_t work,
                               hipStream_t stream) {
  const auto kernel = a.D == 128 ? (g.B == 128 ? k_append_quant<T, 128, 128> : k_append_quant<T, 128, 64>)
                                 : (g.B == 128 ? k_append_quant<T, 64, 128> : k_append_quant<T, 64, 64>);
  const int64_t wgs = work < kAppendMaxWgs ? work : kAppendMaxWgs;
  return launch_kernel(kernel, dim3(static_cast<unsigned>(wgs)), dim3(kThreads), 0, stream, g, a, units, work);
}

// ---------------------------------------------------------------- read
// Chunks of 16 codes of all rows are numbered through, as an append of unquantised tokens does; a
// workgroup looks up its rows' places and moves kReadUnroll * 256 of them, in K and in V.
constexpr int kReadUnroll = 4;

template <typename T>
__device__ __forceinline__ void write16(T* to, const uint4 c, float scale) {
  const uint32_t w[4] = {c.x, c.y, c.z, c.w};
#pragma unroll
  for (int x = 0; x < 4; x += sizeof(T) == 2 ? 2 : 1) {
    float y[4];
    values4(w[x], y);
    if constexpr (sizeof(T) == 2) {
      float z[4];
      values4(w[x + 1], z);
      bf16x8 b;
#pragma unroll
      for (int e = 0; e < 4; ++e) {
        b[e] = static_cast<__bf16>(y[e] * scale);
        b[e + 4] = static_cast<__bf16>(z[e] * scale);
      }
      *reinterpret_cast<bf16x8*>(to + 4 * x) = b;
    } else {
      *reinterpret_cast<f32x4*>(to + 4 * x) = f32x4{y[0] * scale, y[1] * scale, y[2] * scale, y[3] * scale};
    }
  }
}

template <typename T>
__global__ __launch_bounds__(kThreads) void k_read_quant(const SeqGeom g, const ReadQuantLaunch a) {
  constexpr int U = kReadUnroll, kChunks = U * kThreads;
  constexpr int kRows = kChunks / 4 + 2;  // rows of at least 4 chunks (one head of 64)
  __shared__ int s_seq[kRows], s_page[kRows], s_slot[kRows];
  const int tid = threadIdx.x;
  const int head_chunks = a.D / 16;
  const int64_t row_chunks = static_cast<int64_t>(a.H) * head_chunks, total = a.tokens * row_chunks;
  const int64_t c0 = static_cast<int64_t>(blockIdx.x) * kChunks;
  const int t0 = static_cast<int>(c0 / row_chunks), t1 = static_cast<int>((min(c0 + kChunks, total) - 1) / row_chunks);
  for (int r = tid; r <= t1 - t0; r += kThreads) s_seq[r] = a.starts == nullptr ? t0 + r : -1;
  __syncthreads();
  if (a.starts != nullptr) {
    for (int s = tid; s < g.N; s += kThreads) {
      const int from = max(row_of_start(a.starts, a.tokens, s), t0);
      const int to = min(row_of_start(a.starts, a.tokens, s + 1), t1 + 1);
      for (int t = from; t < to; ++t) s_seq[t - t0] = s;
    }
    __syncthreads();
  }
  for (int r = tid; r <= t1 - t0; r += kThreads) {
    const int s = s_seq[r];
    int page = -2, slot = 0;  // -2: a row of no sequence, left alone; -1: zeros
    if (s >= 0) {
      page = -1;
      const int row = t0 + r;
      const int64_t end = min(g.lens[s], g.cap);
      int64_t t;
      if (a.first != nullptr) t = static_cast<int64_t>(a.first[s]) + row - (a.starts == nullptr ? row : row_of_start(a.starts, a.tokens, s));
      else t = static_cast<int64_t>(g.lens[s]) - 1 - (a.starts == nullptr ? 0 : row_of_start(a.starts, a.tokens, s + 1) - 1 - row);
      if (t >= 0 && t < end) {
        const int ti = static_cast<int>(t), c = ti / g.S, off = ti - c * g.S;
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
  uint4 kk[U], vv[U];
  float2 scale[U];
  int64_t to[U];
#pragma unroll
  for (int u = 0; u < U; ++u) {
    const int64_t c = c0 + u * kThreads + tid;
    to[u] = -1;
    kk[u] = vv[u] = make_uint4(0, 0, 0, 0);
    scale[u] = make_float2(0.f, 0.f);
    if (c >= total) continue;
    const int row = static_cast<int>(c / row_chunks), in = static_cast<int>(c - row * row_chunks);
    const int page = s_page[row - t0];
    if (page == -2) continue;
    to[u] = c * 16;
    if (page < 0) continue;
    const int h = in / head_chunks;
    const int64_t head = static_cast<int64_t>(page) * a.H + h;
    const int64_t at = (head * g.B + s_slot[row - t0]) * head_chunks + (in - h * head_chunks);
    kk[u] = load_once(static_cast<const uint4*>(a.k_pages) + at);
    vv[u] = load_once(static_cast<const uint4*>(a.v_pages) + at);
    scale[u] = *reinterpret_cast<const float2*>(a.scales + head * 2);
  }
#pragma unroll
  for (int u = 0; u < U; ++u) {
    if (to[u] < 0) continue;
    write16(static_cast<T*>(a.out_k) + to[u], kk[u], scale[u].x);
    write16(static_cast<T*>(a.out_v) + to[u], vv[u], scale[u].y);
  }
}

}  // namespace

hipError_t launch_append_kv_quant(const SeqGeom& g, const AppendQuantLaunch& a, hipStream_t stream) {
  const AppendUnits units{g.S == g.B ? 2 : 3, g.S == g.B ? 0 : g.S};
  const int64_t blocks = a.starts == nullptr ? g.N
                                             : static_cast<int64_t>(a.tokens) / g.B + (units.S > 0 ? a.tokens / units.S : 0) +
                                                   static_cast<int64_t>(units.per_seq) * g.N;
  const int64_t work = blocks * 2 * a.H;
  return a.dtype == OMNIMEM_BF16 ? launch_append_typed<uint16_t>(g, a, units, work, stream)
                                 : launch_append_typed<float>(g, a, units, work, stream);
}

hipError_t launch_read_kv_quant(const SeqGeom& g, const ReadQuantLaunch& a, hipStream_t stream) {
  const int64_t chunks = static_cast<int64_t>(a.tokens) * a.H * (a.D / 16);
  const int64_t wgs = (chunks + kReadUnroll * kThreads - 1) / (kReadUnroll * kThreads);
  if (wgs > 0x7fffffff) return hipErrorInvalidConfiguration;
  const auto kernel = a.dtype == OMNIMEM_BF16 ? k_read_quant<uint16_t> : k_read_quant<float>;
  return launch_kernel(kernel, dim3(static_cast<unsigned>(wgs)), dim3(kThreads), 0, stream, g, a);
}

}  // namespace omnimem
