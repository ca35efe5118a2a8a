// pages.hip -- the sequence cache's pages for gfx950: new tokens' keys and values into them,
// whole-page copies, and the tables of the next step (forks, growth, frees) and of a
// compacted pool.
#include <limits.h>

#include "device_common.h"
#include "launch.h"
#include "seq_launch.h"

namespace omnimem {
namespace {

__device__ __forceinline__ void store16(const uint4 x, void* p) { *reinterpret_cast<uint4*>(p) = x; }

__device__ __forceinline__ int blocks_of(const SeqGeom& g, int t) {  // blocks of t tokens
  return t / g.S * g.Bpc + (t % g.S + g.B - 1) / g.B;
}

__device__ __forceinline__ int clamped_len(const SeqGeom& g, int s) { return min(max(g.lens[s], 0), g.cap); }

// ---------------------------------------------------------------- append
// Copies: a token's row of H * d values becomes H pieces of d, each 16-byte chunk of it
// moved by one lane.  Chunks of all rows are numbered through; a workgroup takes
// U * 256 of them in K and in V, all loads in flight before the lookups that say where they go:
// row -> sequence (starts), its length, and the page.
constexpr int kAppendThreads = 256;

template <int U>
__global__ __launch_bounds__(kAppendThreads) void k_append_kv(const SeqGeom g, const AppendLaunch a) {
  constexpr int kChunks = U * kAppendThreads;
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
    store16(kk[u], static_cast<uint4*>(a.k_pages) + at);
    store16(vv[u], static_cast<uint4*>(a.v_pages) + at);
  }
}

// ---------------------------------------------------------------- copies of pages
// A grid that is resident at once walks pieces of 16 KB of (pair, layer, pool); the number of
// pairs is read on the device.
constexpr int kCopyThreads = 256, kCopyUnroll = 4, kCopyPiece = kCopyThreads * kCopyUnroll;
constexpr int kCopyMaxWgs = 2048;

__global__ __launch_bounds__(kCopyThreads) void k_copy_pages(const CopyLaunch a, int pieces) {
  const int pools = a.v_pages != nullptr ? 2 : 1;
  const int pairs = a.count == nullptr ? a.max_pairs : min(max(*a.count, 0), a.max_pairs);
  const int64_t per_pair = static_cast<int64_t>(pieces) * pools * a.layers;
  const int64_t total = per_pair * pairs;
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
      if (c < a.page_chunks) store16(x[u], to + c);
    }
  }
}

// ---------------------------------------------------------------- tables
// The pool's state is a function of the tables, formed anew by every call: a bitmap of the
// pages in use, marked by atomics whose order does not matter, and ranks in it.  The k-th
// free or used page is found by a search over prefix counts that every workgroup forms for
// itself in LDS, so no list of free pages is kept or built.
constexpr int kSeqThreads = 512;

struct RowPlan {  // of a new row
  int keep, grow;  // grow < 0: past the capacity
  int tail_page;   // page of the begun block that the row will write to, or -1
  int parent;      // or -1
};

struct SeqScratch {
  uint32_t* used;  // pages that a kept block names
  uint32_t* held;  // of them, pages that a row names without writing to them next
  int* first;      // lowest row that writes to a page (set for pages written to alone)
  RowPlan* rows;
  int64_t words;
};

__device__ __forceinline__ RowPlan plan_row(const SeqGeom& g, const SeqUpdateLaunch& a, int r) {
  RowPlan p{0, 0, -1, a.parent[r]};
  if (p.parent < 0 || p.parent >= g.N) p.parent = -1;
  if (p.parent >= 0) {
    const int len = clamped_len(g, p.parent);
    p.keep = a.keep == nullptr ? len : min(max(a.keep[r], 0), len);
  }
  p.grow = a.grow == nullptr ? 0 : max(a.grow[r], 0);
  if (p.grow > 0 && p.keep % g.S % g.B != 0) {
    const int page = g.table[static_cast<int64_t>(p.parent) * g.M + blocks_of(g, p.keep) - 1];
    if (page >= 0 && page < g.num_pages) p.tail_page = page;
  }
  if (static_cast<int64_t>(p.keep) + p.grow > g.cap) p.grow = -1;
  return p;
}

__device__ __forceinline__ void set_bit(uint32_t* map, int page) { atomicOr(map + (page >> 5), 1u << (page & 31)); }

// An entry of a kept block: its page, or -1.
__device__ __forceinline__ int entry(const SeqGeom& g, int row, int b) {
  const int page = g.table[static_cast<int64_t>(row) * g.M + b];
  return page >= 0 && page < g.num_pages ? page : -1;
}

// Counts of free pages in front of every thread's run of words.
template <int NT>
struct FreeRanks {
  int before[NT];
  int scan[NT / kWave];

  __device__ __forceinline__ static uint32_t free_in(const uint32_t* used, int64_t w, int64_t pages) {
    const int64_t left = pages - w * 32;
    return ~used[w] & (left >= 32 ? 0xffffffffu : (1u << left) - 1u);
  }
  __device__ __forceinline__ int count(const uint32_t* used, int64_t words, int64_t pages) {  // all threads; the free pages
    const int64_t per = (words + NT - 1) / NT;
    const int64_t lo = min(threadIdx.x * per, words), hi = min(lo + per, words);
    int n = 0;
    for (int64_t w = lo; w < hi; ++w) n += __popc(free_in(used, w, pages));
    int all;
    const int at = block_exclusive_scan<NT>(n, scan, all);
    before[threadIdx.x] = at;
    __syncthreads();
    return all;
  }
  // free pages in front of `page`
  __device__ __forceinline__ int rank(const uint32_t* used, int64_t words, int64_t pages, int page) const {
    const int64_t per = (words + NT - 1) / NT;
    const int64_t w = page >> 5;
    const int run = static_cast<int>(w / per);
    int n = before[run];
    for (int64_t x = run * per; x < w; ++x) n += __popc(free_in(used, x, pages));
    return n + __popc(free_in(used, w, pages) & ((1u << (page & 31)) - 1u));
  }
  // the k-th page (from 0) that is free, or in use; the caller knows that there is one
  template <bool FREE>
  __device__ __forceinline__ int select(const uint32_t* used, int64_t words, int64_t pages, int k) const {
    const int64_t per = (words + NT - 1) / NT;
    auto ahead = [&](int run) {  // pages of the kind in front of a run
      return FREE ? before[run] : static_cast<int>(min(run * per * 32, pages)) - before[run];
    };
    int run = 0;
#pragma unroll
    for (int step = NT / 2; step > 0; step >>= 1)
      if (ahead(run + step) <= k) run += step;
    k -= ahead(run);
    for (int64_t w = run * per; w < words; ++w) {
      uint32_t bits = free_in(used, w, pages);
      if (!FREE) bits = used[w];
      const int n = __popc(bits);
      if (k >= n) {
        k -= n;
        continue;
      }
      for (; k > 0; --k) bits &= bits - 1;
      return static_cast<int>(w * 32 + __builtin_ctz(bits));
    }
    return -1;
  }
};

__global__ __launch_bounds__(256) void k_seq_clear(const SeqGeom g, const SeqUpdateLaunch a, const SeqScratch x) {
  const int64_t id = static_cast<int64_t>(blockIdx.x) * 256 + threadIdx.x, n = static_cast<int64_t>(gridDim.x) * 256;
  for (int64_t w = id; w < x.words; w += n) {
    x.used[w] = 0;
    if (a.num_new > 0) x.held[w] = 0;
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
      blocks = blocks_of(g, p.keep);
      if (p.tail_page >= 0) tail = blocks - 1;
    } else {
      blocks = blocks_of(g, clamped_len(g, r));
    }
    for (int b = blockIdx.x * 256 + threadIdx.x; b < blocks; b += gridDim.x * 256) {
      const int page = entry(g, src, b);
      if (page < 0) continue;
      set_bit(x.used, page);
      if (a.num_new == 0) continue;
      if (b == tail) atomicMin(x.first + page, r);
      else set_bit(x.held, page);
    }
  }
}

__global__ __launch_bounds__(kSeqThreads) void k_seq_update(const SeqGeom g, const SeqUpdateLaunch a,
                                                            const SeqScratch x) {
  __shared__ FreeRanks<kSeqThreads> ranks;
  __shared__ int s_scan[kSeqThreads / kWave];
  __shared__ int s_want[kSeqThreads], s_copies[kSeqThreads];  // of the rows in front of each thread's run
  const int tid = threadIdx.x;
  const int room = ranks.count(x.used, x.words, g.num_pages);
  // what every row asks for
  auto copies_page = [&](const RowPlan& p, int r) -> bool {
    return p.grow > 0 && p.tail_page >= 0 &&
           ((x.held[p.tail_page >> 5] >> (p.tail_page & 31) & 1u) != 0 || x.first[p.tail_page] != r);
  };
  auto added = [&](const RowPlan& p) { return p.grow > 0 ? blocks_of(g, p.keep + p.grow) - blocks_of(g, p.keep) : 0; };
  const int per = (a.num_new + kSeqThreads - 1) / kSeqThreads;
  const int lo = min(tid * per, a.num_new), hi = min(lo + per, a.num_new);
  int want = 0, copies = 0, over = 0;
  for (int r = lo; r < hi; ++r) {
    const RowPlan p = x.rows[r];
    const int c = copies_page(p, r);
    copies += c;
    want += c + added(p);
    over += p.grow < 0;
  }
  int all_want, all_copies, all_over;
  const int want_before = block_exclusive_scan<kSeqThreads>(want, s_scan, all_want);
  const int copies_before = block_exclusive_scan<kSeqThreads>(copies, s_scan, all_copies);
  block_exclusive_scan<kSeqThreads>(over, s_scan, all_over);
  s_want[tid] = want_before;
  s_copies[tid] = copies_before;
  __syncthreads();
  const bool done = all_want <= room && all_over == 0;
  if (blockIdx.x == 0) {
    if (tid == 0) {
      a.info[0] = done ? all_copies : 0;
      a.info[1] = static_cast<int>(g.num_pages) - room + (done ? all_want : 0);
      a.info[2] = max(all_want - room, 0);
      a.info[3] = all_over;
    }
    for (int r = (done ? all_copies : 0) + tid; r < a.num_new; r += kSeqThreads) {
      a.pairs[2 * r] = -1;
      a.pairs[2 * r + 1] = -1;
    }
  }
  for (int r = blockIdx.x; r < a.num_new; r += gridDim.x) {
    const RowPlan p = x.rows[r];
    const int run = r / per;
    int at = s_want[run], nth = s_copies[run];
    for (int y = run * per; y < r; ++y) {
      const RowPlan o = x.rows[y];
      const int c = copies_page(o, y);
      nth += c;
      at += c + added(o);
    }
    const int kept = blocks_of(g, p.keep);
    const int copy = done && copies_page(p, r);
    const int blocks = done ? kept + added(p) : kept;
    int32_t* out = a.out_table + static_cast<int64_t>(r) * g.M;
    for (int b = tid; b < g.M; b += kSeqThreads) {
      int page = -1;
      if (b < kept) page = entry(g, p.parent, b);
      if (b >= blocks) page = -1;
      else if (b >= kept) page = ranks.template select<true>(x.used, x.words, g.num_pages, at + copy + b - kept);
      else if (copy && b == kept - 1) {
        page = ranks.template select<true>(x.used, x.words, g.num_pages, at);
        a.pairs[2 * nth] = p.tail_page;
        a.pairs[2 * nth + 1] = page;
      }
      out[b] = page;
    }
    if (tid == 0) a.out_lens[r] = p.keep + (done ? p.grow : 0);
  }
}

__global__ __launch_bounds__(kSeqThreads) void k_seq_compact(const SeqGeom g, const SeqUpdateLaunch a,
                                                             const SeqScratch x, int max_moves) {
  __shared__ FreeRanks<kSeqThreads> ranks;
  const int tid = threadIdx.x;
  const int pages = static_cast<int>(g.num_pages);
  const int in_use = pages - ranks.count(x.used, x.words, g.num_pages);
  // free pages in front of the border, which the used ones behind it fill
  const int moves = in_use < pages ? ranks.rank(x.used, x.words, g.num_pages, in_use) : 0;
  if (blockIdx.x == 0 && tid < 4) a.info[tid] = tid == 0 ? moves : tid == 1 ? in_use : 0;
  for (int64_t m = static_cast<int64_t>(blockIdx.x) * kSeqThreads + tid; m < max_moves;
       m += static_cast<int64_t>(gridDim.x) * kSeqThreads) {
    int from = -1, to = -1;
    if (m < moves) {
      from = ranks.template select<false>(x.used, x.words, g.num_pages, in_use - moves + static_cast<int>(m));
      to = ranks.template select<true>(x.used, x.words, g.num_pages, static_cast<int>(m));
    }
    a.pairs[2 * m] = from;
    a.pairs[2 * m + 1] = to;
  }
  for (int r = blockIdx.x; r < g.N; r += gridDim.x) {
    const int blocks = blocks_of(g, clamped_len(g, r));
    int32_t* out = a.out_table + static_cast<int64_t>(r) * g.M;
    for (int b = tid; b < g.M; b += kSeqThreads) {
      int page = b < blocks ? entry(g, r, b) : -1;
      if (page >= in_use) {
        // used pages in front of it, less those in front of the border
        const int nth = page - ranks.rank(x.used, x.words, g.num_pages, page) - (in_use - moves);
        page = ranks.template select<true>(x.used, x.words, g.num_pages, nth);
      }
      out[b] = page;
    }
  }
}

SeqScratch scratch_of(const SeqPlan& p, void* workspace) {
  char* ws = static_cast<char*>(workspace);
  return SeqScratch{reinterpret_cast<uint32_t*>(ws + p.off_used), reinterpret_cast<uint32_t*>(ws + p.off_held),
                    reinterpret_cast<int*>(ws + p.off_first), reinterpret_cast<RowPlan*>(ws + p.off_rows), p.words};
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

}  // namespace

hipError_t launch_append_kv(const SeqGeom& g, const AppendLaunch& a, hipStream_t stream) {
  constexpr int U = 4;
  const int64_t chunks = a.tokens * a.row_chunks;
  const int64_t wgs = (chunks + U * kAppendThreads - 1) / (U * kAppendThreads);
  if (wgs > 0x7fffffff) return hipErrorInvalidConfiguration;
  return launch_kernel(k_append_kv<U>, dim3(static_cast<unsigned>(wgs)), dim3(kAppendThreads), 0, stream, g, a);
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
  const SeqScratch x = scratch_of(p, workspace);
  LaunchStatus st;
  mark_used(g, p, a, x, a.num_new, stream, st);
  const int wgs = a.num_new < 1 ? 1 : a.num_new < kSeqMaxWgs ? a.num_new : kSeqMaxWgs;
  st(k_seq_update, dim3(wgs), dim3(kSeqThreads), 0, stream, g, a, x);
  return st.err;
}

hipError_t launch_seq_compact(const SeqGeom& g, const SeqPlan& p, const SeqUpdateLaunch& a, void* workspace,
                              hipStream_t stream) {
  const SeqScratch x = scratch_of(p, workspace);
  const int max_moves = g.num_pages >= 2 ? static_cast<int>(g.num_pages / 2) : 1;
  LaunchStatus st;
  mark_used(g, p, a, x, g.N, stream, st);
  const int64_t work = (static_cast<int64_t>(max_moves) + kSeqThreads - 1) / kSeqThreads;
  const int64_t most = work > g.N ? work : g.N;
  st(k_seq_compact, dim3(most < kSeqMaxWgs ? most : kSeqMaxWgs), dim3(kSeqThreads), 0, stream, g, a, x, max_moves);
  return st.err;
}

}  // namespace omnimem
