// pages.hip -- the sequence cache's pages for gfx950: new tokens' keys and values into them,
// whole-page copies, and the tables of the next step (forks, growth, frees) and of a
// compacted pool.
#include <limits.h>

#include "device_common.h"
#include "launch.h"
#include "seq_launch.h"

namespace omnimem {
namespace {

template <bool PAST>
__device__ __forceinline__ void store16(const uint4 x, void* p) {
  const u32x4 v = {x.x, x.y, x.z, x.w};
  if constexpr (PAST) __builtin_nontemporal_store(v, static_cast<u32x4*>(p));
  else *static_cast<u32x4*>(p) = v;
}

__device__ __forceinline__ int block_shift(const SeqGeom& g) { return 6 + (g.B >> 7); }  // log2 B

__device__ __forceinline__ int blocks_of(const SeqGeom& g, int t) {  // blocks of t tokens
  if (g.S == g.B) return (t + g.B - 1) >> block_shift(g);
  const int c = t / g.S;
  return c * g.Bpc + ((t - c * g.S + g.B - 1) >> block_shift(g));
}

__device__ __forceinline__ bool block_begun(const SeqGeom& g, int t) {  // the token behind t tokens is not a block's first
  return ((g.S == g.B ? t : t % g.S) & (g.B - 1)) != 0;
}

__device__ __forceinline__ int clamped_len(const SeqGeom& g, int s) { return min(max(g.lens[s], 0), g.cap); }

// Stores past the caches pay for what the 256 MB memory-side cache cannot hold beside what it
// is copied from: 201 MB of copied pages 86.3 -> 77.5 us, 172 MB of appended tokens 70.7 -> 67.3;
// 100 MB of pages 35.5 -> 38.7 and 115 MB of tokens 42.6 -> 44.0 without.
constexpr int64_t kPastBytes = 144ll << 20;  // written

// ---------------------------------------------------------------- append
// Copies: a token's row of H * d values becomes H pieces of d, each 16-byte chunk of it
// moved by one lane.  Chunks of all rows are numbered through; a workgroup takes
// U * 256 of them in K and in V, all loads in flight before the lookups that say where they go:
// row -> sequence (starts), its length, and the page.  Bound by its bytes: eight chunks of
// 4,680 tokens, 12 heads, bf16 (460 MB read and written) 89 us, 5.2 TB/s; 64 single tokens 4.1 us,
// three dependent loads.
constexpr int kAppendThreads = 256, kAppendUnroll = 4;

template <bool PAST>
__global__ __launch_bounds__(kAppendThreads) void k_append_kv(const SeqGeom g, const AppendLaunch a) {
  constexpr int U = kAppendUnroll, kChunks = U * kAppendThreads;
  constexpr int kRows = kChunks / 8 + 2;  // rows of at least 8 chunks (one head of 64 bf16)
  __shared__ int s_seq[kRows];
  __shared__ int64_t s_to[kRows];  // chunk of head 0's piece in the pools, or -1
  const int tid = threadIdx.x;
  const int64_t total = static_cast<int64_t>(a.tokens) * a.row_chunks;
  const int64_t c0 = static_cast<int64_t>(blockIdx.x) * kChunks;
  const int t0 = static_cast<int>(c0 / a.row_chunks);
  const int t1 = static_cast<int>((min(c0 + kChunks, total) - 1) / a.row_chunks);  // last row

  uint4 kk[U], vv[U];
  int row[U], in[U];
#pragma unroll
  for (int u = 0; u < U; ++u) {
    const int64_t c = c0 + u * kAppendThreads + tid;
    row[u] = -1;
    if (c >= total) continue;
    row[u] = static_cast<int>(c / a.row_chunks);
    in[u] = static_cast<int>(c - row[u] * a.row_chunks);
    kk[u] = load_once(static_cast<const uint4*>(a.k) + row[u] * a.k_stride + in[u]);
    vv[u] = load_once(static_cast<const uint4*>(a.v) + row[u] * a.v_stride + in[u]);
  }
  // the rows' sequences: each sequence marks its own rows of this workgroup
  for (int r = tid; r <= t1 - t0; r += kAppendThreads) s_seq[r] = a.starts == nullptr ? t0 + r : -1;
  __syncthreads();
  if (a.starts != nullptr) {
    for (int s = tid; s < g.N; s += kAppendThreads) {
      const int from = max(min(max(a.starts[s], 0), a.tokens), t0);
      const int to = min(min(max(a.starts[s + 1], 0), a.tokens), t1 + 1);
      for (int t = from; t < to; ++t) s_seq[t - t0] = s;
    }
    __syncthreads();
  }
  for (int r = tid; r <= t1 - t0; r += kAppendThreads) {
    const int s = s_seq[r];
    int64_t to = -1;
    if (s >= 0) {
      // the sequence's last row is its last token
      const int64_t behind = a.starts == nullptr ? 0 : min(max(a.starts[s + 1], 0), a.tokens) - 1 - (t0 + r);
      const int64_t t = static_cast<int64_t>(g.lens[s]) - 1 - behind;
      if (t >= 0 && t < g.cap) {
        const int ti = static_cast<int>(t), c = ti / g.S, off = ti % g.S;
        const int page = g.table[static_cast<int64_t>(s) * g.M + c * g.Bpc + off / g.B];
        if (page >= 0 && page < g.num_pages)
          to = (static_cast<int64_t>(page) * a.H * g.B + off % g.B) * a.head_chunks;
      }
    }
    s_to[r] = to;
  }
  __syncthreads();
#pragma unroll
  for (int u = 0; u < U; ++u) {
    if (row[u] < 0) continue;
    const int64_t to = s_to[row[u] - t0];
    if (to < 0) continue;
    const int h = in[u] / a.head_chunks;
    const int64_t at = to + static_cast<int64_t>(h) * g.B * a.head_chunks + (in[u] - h * a.head_chunks);
    store16<PAST>(kk[u], static_cast<uint4*>(a.k_pages) + at);
    store16<PAST>(vv[u], static_cast<uint4*>(a.v_pages) + at);
  }
}

// ---------------------------------------------------------------- copies of pages
// A grid that is resident at once walks pieces of 16 KB of (pair, layer, pool); the number of
// pairs is read on the device.  Bound by its bytes: 300 pages of 12 heads x 64 x 128 bf16 in six
// layers (1.4 GB read and written) 279 us, 5.1 TB/s, as a large tensor copy (5.0); 16 pages 4.2 us.
constexpr int kCopyThreads = 256, kCopyUnroll = 4, kCopyPiece = kCopyThreads * kCopyUnroll;
constexpr int kCopyMaxWgs = 2048;

template <bool PAST>
__device__ __forceinline__ void copy_pieces(const CopyLaunch& a, int pieces, int pools, int64_t per_pair,
                                            int64_t total) {
  for (int64_t w = blockIdx.x; w < total; w += gridDim.x) {
    const int64_t p = w / per_pair;
    const int64_t rest = w - p * per_pair;
    const int64_t lp = rest / pieces;
    const int layer = static_cast<int>(lp / pools), pool = static_cast<int>(lp % pools);
    const int64_t at = (rest - lp * pieces) * kCopyPiece;
    const int src = a.pairs[2 * p], dst = a.pairs[2 * p + 1];
    if (src < 0 || src >= a.num_pages || dst < 0 || dst >= a.num_pages) continue;
    uint4* base = static_cast<uint4*>(pool == 0 ? a.k_pages : a.v_pages) + layer * a.layer_chunks;
    const uint4* from = base + src * a.page_chunks;
    uint4* to = base + dst * a.page_chunks;
    uint4 x[kCopyUnroll];
#pragma unroll
    for (int u = 0; u < kCopyUnroll; ++u) {
      const int64_t c = at + u * kCopyThreads + threadIdx.x;
      if (c < a.page_chunks) x[u] = load_once(from + c);
    }
#pragma unroll
    for (int u = 0; u < kCopyUnroll; ++u) {
      const int64_t c = at + u * kCopyThreads + threadIdx.x;
      if (c < a.page_chunks) store16<PAST>(x[u], to + c);
    }
  }
}

__global__ __launch_bounds__(kCopyThreads) void k_copy_pages(const CopyLaunch a, int pieces) {
  const int pools = a.v_pages != nullptr ? 2 : 1;
  const int pairs = a.count == nullptr ? a.max_pairs : min(max(*a.count, 0), a.max_pairs);
  const int64_t per_pair = static_cast<int64_t>(pieces) * pools * a.layers, total = per_pair * pairs;
  if (a.page_chunks * 16 * pools * a.layers * pairs > kPastBytes)
    copy_pieces<true>(a, pieces, pools, per_pair, total);
  else
    copy_pieces<false>(a, pieces, pools, per_pair, total);
}

// ---------------------------------------------------------------- tables
// The pool's state is a function of the tables, formed anew by every call: bitmaps of the
// pages in use, marked by atomics whose order does not matter, and ranks in them.  The k-th
// free or used page is found by a search over prefix counts that every workgroup forms for
// itself in LDS, so no list of free pages is kept or built.
constexpr int kSeqThreads = 512;


struct SeqScratch {
  uint32_t* held;  // pages that a row names without writing to them next
  uint32_t* tail;  // pages that a row will write to; null, as the next two, without new rows
  int* first;      // the lowest such row of a page of `tail`
  RowPlan* rows;
  int64_t words;
};

__device__ __forceinline__ RowPlan plan_row(const SeqGeom& g, const SeqUpdateLaunch& a, int r) {
  RowPlan p{};
  p.tail_page = -1;
  p.parent = a.parent[r];
  const int keep = a.keep == nullptr ? INT_MAX : a.keep[r], want = a.grow == nullptr ? 0 : a.grow[r];
  int tokens = 0;
  if (p.parent >= 0 && p.parent < g.N) tokens = min(max(keep, 0), clamped_len(g, p.parent));
  const int grow = max(want, 0);
  p.kept = blocks_of(g, tokens);
  if (grow > 0 && block_begun(g, tokens)) {
    const int page = g.table[static_cast<int64_t>(p.parent) * g.M + p.kept - 1];
    if (page >= 0 && page < g.num_pages) p.tail_page = page;
  }
  p.over = static_cast<int64_t>(tokens) + grow > g.cap;
  p.len = p.over ? tokens : tokens + grow;
  p.short_len = tokens;
  p.added = p.over ? 0 : blocks_of(g, p.len) - p.kept;
  return p;
}

__device__ __forceinline__ void set_bit(uint32_t* map, int page) { atomicOr(map + (page >> 5), 1u << (page & 31)); }

// An entry of a kept block: its page, or -1.
__device__ __forceinline__ int entry(const SeqGeom& g, int row, int b) {
  const int page = g.table[static_cast<int64_t>(row) * g.M + b];
  return page >= 0 && page < g.num_pages ? page : -1;
}

// Exclusive prefix sums of V values over a workgroup, and their totals; one barrier.
template <int NT, int V>
struct Scan {
  int wave[V][NT / kWave];
  __device__ __forceinline__ void operator()(int (&x)[V], int (&all)[V]) {
    const int lane = threadIdx.x % kWave, w = threadIdx.x / kWave;
    int upto[V];
#pragma unroll
    for (int v = 0; v < V; ++v) {
      upto[v] = wave_inclusive_scan(x[v]);
      if (lane == kWave - 1) wave[v][w] = upto[v];
    }
    __syncthreads();
#pragma unroll
    for (int v = 0; v < V; ++v) {
      int before = 0;
      all[v] = 0;
#pragma unroll
      for (int o = 0; o < NT / kWave; ++o) {
        if (o < w) before += wave[v][o];
        all[v] += wave[v][o];
      }
      x[v] = before + upto[v] - x[v];
    }
  }
};

// The pages of a pool that are in use, as a bitmap in one or two parts, and how many free
// ones lie in front of each thread's run of its words.
template <int NT>
struct Pages {
  const uint32_t* a;
  const uint32_t* b;  // or null
  uint32_t pages;
  int words, per;
  int* before;  // [NT], shared

  __device__ __forceinline__ Pages(const uint32_t* a_, const uint32_t* b_, int64_t pages_, int* before_)
      : a(a_), b(b_), pages(static_cast<uint32_t>(pages_)), words(static_cast<int>((pages_ + 31) / 32)),
        per((words + NT - 1) / NT), before(before_) {}
  __device__ __forceinline__ uint32_t used_in(int w) const { return b == nullptr ? a[w] : a[w] | b[w]; }
  __device__ __forceinline__ uint32_t free_in(int w) const {
    const uint32_t left = pages - static_cast<uint32_t>(w) * 32u;  // > 0
    return ~used_in(w) & (left >= 32u ? 0xffffffffu : (1u << left) - 1u);
  }
  __device__ __forceinline__ int free_of_run() const {  // in the calling thread's run
    const int lo = min(static_cast<int>(threadIdx.x) * per, words), hi = min(lo + per, words);
    int n = 0;
    for (int w = lo; w < hi; ++w) n += __popc(free_in(w));
    return n;
  }
  // free pages in front of `page`
  __device__ __forceinline__ int rank(int page) const {
    const int w = page >> 5, run = per == 1 ? w : w / per;
    int n = before[run];
    for (int x = run * per; x < w; ++x) n += __popc(free_in(x));
    return n + __popc(free_in(w) & ((1u << (page & 31)) - 1u));
  }
  // the k-th page (from 0) that is free, or in use; the caller knows that there is one
  template <bool FREE>
  __device__ __forceinline__ int select(int k) const {
    auto ahead = [&](int run) {  // pages of the kind in front of a run
      return FREE ? before[run]
                  : static_cast<int>(static_cast<uint32_t>(min(run * per, words)) * 32u) - before[run];
    };
    int run = 0;
#pragma unroll
    for (int step = NT / 2; step > 0; step >>= 1)
      if (ahead(run + step) <= k) run += step;
    k -= ahead(run);
    for (int w = run * per; w < words; ++w) {
      uint32_t bits = FREE ? free_in(w) : used_in(w);
      const int n = __popc(bits);
      if (k >= n) {
        k -= n;
        continue;
      }
      int at = 0;  // the k-th set bit, by halves
#pragma unroll
      for (int half = 16; half > 0; half >>= 1) {
        const int low = __popc(bits & ((1u << half) - 1u));
        if (k >= low) {
          k -= low;
          bits >>= half;
          at += half;
        }
      }
      return w * 32 + at;
    }
    return -1;
  }
};

__global__ __launch_bounds__(256) void k_seq_clear(const SeqGeom g, const SeqUpdateLaunch a, const SeqScratch x) {
  const int64_t id = static_cast<int64_t>(blockIdx.x) * 256 + threadIdx.x, n = static_cast<int64_t>(gridDim.x) * 256;
  for (int64_t w = id; w < x.words; w += n) {
    x.held[w] = 0;
    if (x.tail != nullptr) x.tail[w] = 0;
  }
  for (int64_t r = id; r < a.num_new; r += n) {
    const RowPlan p = plan_row(g, a, static_cast<int>(r));
    x.rows[r] = p;
    if (p.tail_page >= 0) x.first[p.tail_page] = INT_MAX;
  }
}

// y: the row, of the new ones or (compaction) of the table; x: 256 of its blocks
__global__ __launch_bounds__(256) void k_seq_mark(const SeqGeom g, const SeqUpdateLaunch a, const SeqScratch x,
                                                  int rows) {
  for (int r = blockIdx.y; r < rows; r += gridDim.y) {
    int src = r, blocks, tail = -1;
    if (a.num_new > 0) {
      const RowPlan p = x.rows[r];
      src = p.parent;
      blocks = p.kept;
      if (p.tail_page >= 0) tail = blocks - 1;
    } else {
      blocks = blocks_of(g, clamped_len(g, r));
    }
    for (int b = blockIdx.x * 256 + threadIdx.x; b < blocks; b += gridDim.x * 256) {
      const int page = entry(g, src, b);
      if (page < 0) continue;
      if (b != tail) {
        set_bit(x.held, page);
      } else {
        set_bit(x.tail, page);
        atomicMin(x.first + page, r);
      }
    }
  }
}

// New rows from marked pages, by the workgroups of a grid, `lanes` threads to a row.
// held(page): some row names the page without writing to it; first(page): the lowest row that
// writes to it; row(r): a row's plan.
template <int NT, bool FLAT, typename Held, typename First, typename Row>
__device__ __forceinline__ void write_rows(const SeqGeom& g, const SeqUpdateLaunch& a, const Pages<NT>& pool,
                                           Scan<NT, 4>& scan, int* s_want, int* s_copies, int lanes, Held held,
                                           First first, Row row) {
  const int tid = threadIdx.x;
  auto copies_page = [&](const RowPlan& p, int r) -> bool {
    return !p.over && p.tail_page >= 0 && (held(p.tail_page) || first(p.tail_page) != r);
  };
  // free pages, what the rows ask for, and rows past the capacity, by runs of words and of rows
  const int per = (a.num_new + NT - 1) / NT;
  const int lo = min(tid * per, a.num_new), hi = min(lo + per, a.num_new);
  int x[4] = {pool.free_of_run(), 0, 0, 0}, all[4];
  for (int r = lo; r < hi; ++r) {
    const RowPlan p = row(r);
    const int c = copies_page(p, r);
    x[1] += c + p.added;
    x[2] += c;
    x[3] += p.over;
  }
  scan(x, all);
  pool.before[tid] = x[0];
  s_want[tid] = x[1];
  s_copies[tid] = x[2];
  __syncthreads();
  const int room = all[0];
  const bool done = all[1] <= room && all[3] == 0;
  const int copied = done ? all[2] : 0;
  if (blockIdx.x == 0) {
    if (tid == 0) {
      a.info[0] = copied;
      a.info[1] = static_cast<int>(g.num_pages) - room + (done ? all[1] : 0);
      a.info[2] = max(all[1] - room, 0);
      a.info[3] = all[3];
    }
    for (int64_t r = copied + tid; r < a.num_new; r += NT) {
      a.pairs[2 * r] = -1;
      a.pairs[2 * r + 1] = -1;
    }
  }
  // block b of row r, whose pages begin with number `at` of those asked for
  auto block = [&](const RowPlan& p, int r, int b, int copy, int at, int nth) {
    int page = -1;
    if (b < p.kept) page = entry(g, p.parent, b);
    const int fresh = b - p.kept;  // of the row's added blocks; -1: the block that is copied
    if (done && (fresh >= 0 ? fresh < p.added : copy && fresh == -1)) {
      if (fresh < 0) {
        int32_t* pair = a.pairs + 2 * static_cast<int64_t>(nth);
        pair[0] = page;
        pair[1] = pool.template select<true>(at);
      }
      page = pool.template select<true>(at + copy + fresh);
    }
    a.out_table[static_cast<int64_t>(r) * g.M + b] = page;
    if (b == 0) a.out_lens[r] = done ? p.len : p.short_len;
  };
  if constexpr (FLAT) {  // one workgroup, no more rows than threads
    const int step_r = NT / g.M, step_b = NT - step_r * g.M;
    int r = tid / g.M, b = tid - r * g.M;
    while (r < a.num_new) {
      const RowPlan p = row(r);
      block(p, r, b, copies_page(p, r), s_want[r], s_copies[r]);
      r += step_r;
      b += step_b;
      if (b >= g.M) {
        b -= g.M;
        ++r;
      }
    }
  } else {
    const int teams = NT / lanes;
    for (int r = blockIdx.x * teams + tid / lanes; r < a.num_new; r += gridDim.x * teams) {
      const RowPlan p = row(r);
      const int run = r / per;
      int at = s_want[run], nth = s_copies[run];
      for (int y = run * per; y < r; ++y) {
        const RowPlan o = row(y);
        const int c = copies_page(o, y);
        nth += c;
        at += c + o.added;
      }
      const int copy = copies_page(p, r);
      for (int b = tid % lanes; b < g.M; b += lanes) block(p, r, b, copy, at, nth);
    }
  }
}

__global__ __launch_bounds__(kSeqThreads) void k_seq_update(const SeqGeom g, const SeqUpdateLaunch a,
                                                            const SeqScratch x, int lanes) {
  __shared__ int s_free[kSeqThreads], s_want[kSeqThreads], s_copies[kSeqThreads];
  __shared__ Scan<kSeqThreads, 4> scan;
  const Pages<kSeqThreads> pool(x.held, x.tail, g.num_pages, s_free);
  write_rows<kSeqThreads, false>(
      g, a, pool, scan, s_want, s_copies, lanes,
      [&](int page) { return (x.held[page >> 5] >> (page & 31) & 1u) != 0; }, [&](int page) { return x.first[page]; },
      [&](int r) { return x.rows[r]; });
}

// The rows and moves of a compaction; lens: the rows' blocks in LDS (FLAT: one workgroup).
template <int NT, bool FLAT>
__device__ __forceinline__ void write_compacted(const SeqGeom& g, const SeqUpdateLaunch& a, const Pages<NT>& pool,
                                                Scan<NT, 1>& scan, int max_moves, int lanes, const int* s_blocks) {
  const int tid = threadIdx.x;
  int x[1] = {pool.free_of_run()}, all[1];
  scan(x, all);
  pool.before[tid] = x[0];
  __syncthreads();
  const int pages = static_cast<int>(g.num_pages), in_use = pages - all[0];
  // free pages in front of the border, which the used ones behind it fill
  const int moves = in_use < pages ? pool.rank(in_use) : 0;
  const int in_place = in_use - moves;
  if (blockIdx.x == 0 && tid < 4) a.info[tid] = tid == 0 ? moves : tid == 1 ? in_use : 0;
  for (int64_t m = static_cast<int64_t>(blockIdx.x) * NT + tid; m < max_moves; m += static_cast<int64_t>(gridDim.x) * NT) {
    int2 move = {-1, -1};
    if (m < moves) {
      move.x = pool.template select<false>(in_place + static_cast<int>(m));
      move.y = pool.template select<true>(static_cast<int>(m));
    }
    a.pairs[2 * m] = move.x;
    a.pairs[2 * m + 1] = move.y;
  }
  auto block = [&](int r, int b, int blocks) {
    int page = b < blocks ? entry(g, r, b) : -1;
    if (page >= in_use) page = pool.template select<true>(page - pool.rank(page) - in_place);
    a.out_table[static_cast<int64_t>(r) * g.M + b] = page;
  };
  if constexpr (FLAT) {
    const int step_r = NT / g.M, step_b = NT - step_r * g.M;
    for (int r = tid / g.M, b = tid - r * g.M; r < g.N;) {
      block(r, b, s_blocks[r]);
      r += step_r;
      b += step_b;
      if (b >= g.M) {
        b -= g.M;
        ++r;
      }
    }
  } else {
    const int teams = NT / lanes;
    for (int r = blockIdx.x * teams + tid / lanes; r < g.N; r += gridDim.x * teams) {
      const int blocks = blocks_of(g, clamped_len(g, r));
      for (int b = tid % lanes; b < g.M; b += lanes) block(r, b, blocks);
    }
  }
}

__global__ __launch_bounds__(kSeqThreads) void k_seq_compact(const SeqGeom g, const SeqUpdateLaunch a,
                                                             const SeqScratch x, int max_moves, int lanes) {
  __shared__ int s_free[kSeqThreads];
  __shared__ Scan<kSeqThreads, 1> scan;
  const Pages<kSeqThreads> pool(x.held, nullptr, g.num_pages, s_free);
  write_compacted<kSeqThreads, false>(g, a, pool, scan, max_moves, lanes, nullptr);
}

// Small tables (p.one) in one workgroup and one launch, all state in LDS: a word per page, INT_MAX
// free, -1 named by a row that does not write to it, else the lowest row that does.
__device__ __forceinline__ void bitmap_of(const int* state, uint32_t* used, int pages) {
  for (int p = threadIdx.x; p < (pages + kWave - 1) / kWave * kWave; p += kOneThreads) {
    const uint64_t bits = __ballot(p < pages && state[p] != INT_MAX);
    if (threadIdx.x % kWave == 0) {
      used[p / 32] = static_cast<uint32_t>(bits);
      used[p / 32 + 1] = static_cast<uint32_t>(bits >> 32);
    }
  }
}

__global__ __launch_bounds__(kOneThreads) void k_seq_update_one(const SeqGeom g, const SeqUpdateLaunch a) {
  __shared__ int s_state[kOnePages];
  __shared__ uint32_t s_used[kOnePages / 32];
  __shared__ int s_free[kOneThreads], s_want[kOneThreads], s_copies[kOneThreads];
  __shared__ RowPlan s_rows[kOneRows];
  __shared__ Scan<kOneThreads, 4> scan;
  const int tid = threadIdx.x, pages = static_cast<int>(g.num_pages);
  if (tid < a.num_new) s_rows[tid] = plan_row(g, a, tid);
  for (int p = tid; p < pages; p += kOneThreads) s_state[p] = INT_MAX;
  __syncthreads();
  const int step_r = kOneThreads / g.M, step_b = kOneThreads - step_r * g.M;
  for (int r = tid / g.M, b = tid - r * g.M; r < a.num_new;) {
    const RowPlan& p = s_rows[r];
    const int page = b < p.kept ? entry(g, p.parent, b) : -1;
    if (page >= 0) atomicMin(&s_state[page], p.tail_page >= 0 && b == p.kept - 1 ? r : -1);
    r += step_r;
    b += step_b;
    if (b >= g.M) {
      b -= g.M;
      ++r;
    }
  }
  __syncthreads();
  bitmap_of(s_state, s_used, pages);
  __syncthreads();
  const Pages<kOneThreads> pool(s_used, nullptr, g.num_pages, s_free);
  write_rows<kOneThreads, true>(
      g, a, pool, scan, s_want, s_copies, kWave, [&](int page) { return s_state[page] < 0; },
      [&](int page) { return s_state[page]; }, [&](int r) { return s_rows[r]; });
}

__global__ __launch_bounds__(kOneThreads) void k_seq_compact_one(const SeqGeom g, const SeqUpdateLaunch a,
                                                                 int max_moves) {
  __shared__ uint32_t s_used[kOnePages / 32];
  __shared__ int s_free[kOneThreads], s_blocks[kOneRows];
  __shared__ Scan<kOneThreads, 1> scan;
  const int tid = threadIdx.x;
  for (int w = tid; w < kOnePages / 32; w += kOneThreads) s_used[w] = 0;
  if (tid < g.N) s_blocks[tid] = blocks_of(g, clamped_len(g, tid));
  __syncthreads();
  const int step_r = kOneThreads / g.M, step_b = kOneThreads - step_r * g.M;
  for (int r = tid / g.M, b = tid - r * g.M; r < g.N;) {
    const int page = b < s_blocks[r] ? entry(g, r, b) : -1;
    if (page >= 0) atomicOr(&s_used[page >> 5], 1u << (page & 31));
    r += step_r;
    b += step_b;
    if (b >= g.M) {
      b -= g.M;
      ++r;
    }
  }
  __syncthreads();
  const Pages<kOneThreads> pool(s_used, nullptr, g.num_pages, s_free);
  write_compacted<kOneThreads, true>(g, a, pool, scan, max_moves, kWave, s_blocks);
}

SeqScratch scratch_of(const SeqPlan& p, void* workspace) {
  char* ws = static_cast<char*>(workspace);
  uint32_t* held = reinterpret_cast<uint32_t*>(ws + p.off_held);
  if (!p.growing) return SeqScratch{held, nullptr, nullptr, nullptr, p.words};
  return SeqScratch{held, reinterpret_cast<uint32_t*>(ws + p.off_tail), reinterpret_cast<int*>(ws + p.off_first),
                    reinterpret_cast<RowPlan*>(ws + p.off_rows), p.words};
}

constexpr int kSeqMaxWgs = 256;

// Clears and marks; `rows` rows of the table are marked.
void mark_used(const SeqGeom& g, const SeqPlan& p, const SeqUpdateLaunch& a, const SeqScratch& x, int rows,
               hipStream_t stream, LaunchStatus& st) {
  const int64_t most = p.words > a.num_new ? p.words : a.num_new;
  const int64_t clear = (most + 255) / 256;
  if (clear > 0) st(k_seq_clear, dim3(clear < 1024 ? clear : 1024), dim3(256), 0, stream, g, a, x);
  const int wide = (g.M + 255) / 256;
  if (rows > 0)
    st(k_seq_mark, dim3(wide < 64 ? wide : 64, rows < 16384 ? rows : 16384), dim3(256), 0, stream, g, a, x, rows);
}

// Threads to a row and workgroups of the kernels that write rows: a wave for short rows, a
// workgroup for long ones.
int row_lanes(const SeqGeom& g) { return g.M <= 4 * kWave ? kWave : kSeqThreads; }
int row_wgs(int64_t rows, int lanes) {
  const int64_t teams = kSeqThreads / lanes, wgs = (rows + teams - 1) / teams;
  return static_cast<int>(wgs < 1 ? 1 : wgs < kSeqMaxWgs ? wgs : kSeqMaxWgs);
}

}  // namespace

hipError_t launch_append_kv(const SeqGeom& g, const AppendLaunch& a, hipStream_t stream) {
  constexpr int kChunks = kAppendUnroll * kAppendThreads;
  const int64_t chunks = a.tokens * a.row_chunks, wgs = (chunks + kChunks - 1) / kChunks;
  if (wgs > 0x7fffffff) return hipErrorInvalidConfiguration;
  const auto kernel = 2 * 16 * chunks > kPastBytes ? k_append_kv<true> : k_append_kv<false>;
  return launch_kernel(kernel, dim3(static_cast<unsigned>(wgs)), dim3(kAppendThreads), 0, stream, g, a);
}

hipError_t launch_copy_pages(const CopyLaunch& a, hipStream_t stream) {
  const int64_t pieces = (a.page_chunks + kCopyPiece - 1) / kCopyPiece;
  if (pieces > 0x7fffffff) return hipErrorInvalidConfiguration;
  const double units = static_cast<double>(pieces) * 2 * a.layers * a.max_pairs;
  const int wgs = units < kCopyMaxWgs ? static_cast<int>(units) : kCopyMaxWgs;
  return launch_kernel(k_copy_pages, dim3(wgs), dim3(kCopyThreads), 0, stream, a, static_cast<int>(pieces));
}

hipError_t launch_seq_update(const SeqGeom& g, const SeqPlan& p, const SeqUpdateLaunch& a, void* workspace,
                             hipStream_t stream) {
  if (p.one) return launch_kernel(k_seq_update_one, dim3(1), dim3(kOneThreads), 0, stream, g, a);
  const SeqScratch x = scratch_of(p, workspace);
  LaunchStatus st;
  mark_used(g, p, a, x, a.num_new, stream, st);
  const int lanes = row_lanes(g);
  st(k_seq_update, dim3(row_wgs(a.num_new, lanes)), dim3(kSeqThreads), 0, stream, g, a, x, lanes);
  return st.err;
}

hipError_t launch_seq_compact(const SeqGeom& g, const SeqPlan& p, const SeqUpdateLaunch& a, void* workspace,
                              hipStream_t stream) {
  const int max_moves = g.num_pages >= 2 ? static_cast<int>(g.num_pages / 2) : 1;
  if (p.one) return launch_kernel(k_seq_compact_one, dim3(1), dim3(kOneThreads), 0, stream, g, a, max_moves);
  const SeqScratch x = scratch_of(p, workspace);
  LaunchStatus st;
  mark_used(g, p, a, x, g.N, stream, st);
  const int lanes = row_lanes(g);
  const int64_t work = (static_cast<int64_t>(max_moves) + kSeqThreads - 1) / kSeqThreads;
  const int rows = row_wgs(g.N, lanes);
  const int wgs = work < rows ? rows : work < kSeqMaxWgs ? static_cast<int>(work) : kSeqMaxWgs;
  st(k_seq_compact, dim3(wgs), dim3(kSeqThreads), 0, stream, g, a, x, max_moves, lanes);
  return st.err;
}

}  // namespace omnimem
