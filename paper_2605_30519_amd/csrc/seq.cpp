// seq.cpp -- argument checks and work plans of the sequence cache's entry points.  Pointers
// are checked for presence and alignment only; device contents (lengths, page ids, row
// numbers) are bounds-checked by the kernels.
#include "seq.h"

#include <math.h>

#include "plan.h"

namespace omnimem {
namespace {

bool aligned(const void* p, uintptr_t n) { return (reinterpret_cast<uintptr_t>(p) & (n - 1)) == 0; }

int64_t elem_bytes(int32_t dtype) { return dtype == OMNIMEM_BF16 ? 2 : 4; }

omnimem_status_t resolve_table(const omnimem_seq_table_t* st, SeqGeom& g, bool sizes_only) {
  if (st == nullptr || st->num_seqs < 0 || st->max_blocks < 1 || st->chunk_tokens < 1) return OMNIMEM_EINVAL;
  if (st->block_size != 64 && st->block_size != 128) return OMNIMEM_EUNSUPPORTED;
  if (st->num_pages < 0 || st->num_pages > 0x7fffffff) return OMNIMEM_EINVAL;
  g.N = st->num_seqs;
  g.M = st->max_blocks;
  g.B = st->block_size;
  const bool contiguous = st->chunk_tokens % g.B == 0;
  g.S = contiguous ? g.B : st->chunk_tokens;
  g.Bpc = contiguous ? 1 : st->chunk_tokens / g.B + 1;
  const int64_t rest = static_cast<int64_t>(g.M % g.Bpc) * g.B;
  const int64_t cap = static_cast<int64_t>(g.M / g.Bpc) * g.S + rest;
  if (cap > 0x7fffffff - 1024) return OMNIMEM_EINVAL;  // a block behind the last one stays in 31 bits
  g.cap = static_cast<int>(cap);
  g.num_pages = st->num_pages;
  g.table = st->page_table;
  g.lens = st->seq_lens;
  if (!sizes_only && g.N > 0 && (g.table == nullptr || g.lens == nullptr)) return OMNIMEM_EINVAL;
  if (!aligned(g.table, 4) || !aligned(g.lens, 4)) return OMNIMEM_EINVAL;
  return OMNIMEM_OK;
}

omnimem_status_t resolve_seq_cache(const omnimem_seq_cache_t* sc, SeqGeom& g, bool sizes_only) {
  if (sc == nullptr) return OMNIMEM_EINVAL;
  if (sc->dtype != OMNIMEM_BF16 && sc->dtype != OMNIMEM_F32) return OMNIMEM_EUNSUPPORTED;
  if (sc->head_dim != 64 && sc->head_dim != 128) return OMNIMEM_EUNSUPPORTED;
  if (sc->num_heads < 1 || sc->num_heads > (1 << 20)) return OMNIMEM_EINVAL;
  const omnimem_status_t st = resolve_table(&sc->seqs, g, sizes_only);
  if (st != OMNIMEM_OK) return st;
  // the pool's elements stay inside int64 index arithmetic
  if (g.num_pages > (int64_t{1} << 40) / (static_cast<int64_t>(sc->num_heads) * g.B * sc->head_dim))
    return OMNIMEM_EINVAL;
  if (!sizes_only && g.num_pages > 0 && (sc->k_pages == nullptr || sc->v_pages == nullptr)) return OMNIMEM_EINVAL;
  if (!aligned(sc->k_pages, 16) || !aligned(sc->v_pages, 16)) return OMNIMEM_EINVAL;
  return OMNIMEM_OK;
}

// A row stride in elements of `row` elements: covers the row, whole 16-byte chunks.
bool good_stride(int64_t stride, int64_t row, int64_t eb) {
  return stride >= row && stride <= (int64_t{1} << 40) && stride * eb % 16 == 0;
}

// Workgroups of a decode call, one on each of 256 CUs: its 64 KB in flight keep the memory busy,
// and fewer shares have less to join (one sequence of 100,000 tokens, 8 key heads, 71.4 us against
// 73.2 with two, three 89; 16 x 8,000 tokens, 16 heads of 64, 85.7 / 89.9).  Where there are more
// items than CUs, segments change often, and two hide each other's changes (48 ragged sequences,
// 8 key heads, 112.8 / 109.7).
constexpr int64_t kDecodeWgs = 256, kDecodeManyWgs = 512;

// A workgroup to an item, and no join, while an item is short at its longest: one sequence of 500
// tokens (18 units), 8 key heads, 7.7 us against 9.1, 64 of them 22.8 / 25.6; one of 1,000 tokens
// 16.1 / 9.8 (16.5 with eight waves: a CU takes in no more).  Many items of 1,000 tokens gain 6%
// so, and lose as much if they are ragged.
// Where there are four of them and more for each CU, a wave to an item up to 8 units: 1,024 items of
// 60 tokens, 24 query heads, 17.2 -> 11.8 us (4 query heads 10.6 -> 8.2, one fp32 17.4 -> 13.8); 512
// items 9.0 / 8.9 (5.9 / 6.8, 9.5 / 10.8), 64 items of 120 tokens 4.9 -> 9.0.
constexpr int64_t kItemUnitsMost = 20, kWaveUnitsMost = 8, kWaveItems = 1024;
constexpr int64_t kItemOverhead = 64;  // of an item's length on the line, no less than the kernel adds

omnimem_status_t plan_decode(const omnimem_seq_cache_t* sc, const SeqGeom& g, int32_t num_q_heads, int32_t window,
                             DecodePlan& p) {
  if (num_q_heads < 1 || num_q_heads % sc->num_heads != 0) return OMNIMEM_EINVAL;
  p.G = num_q_heads / sc->num_heads;
  p.tile_rows = p.G <= kDecodeHeadRows ? kDecodeHeadRows : 2 * kDecodeHeadRows;
  p.head_tiles = (p.G + p.tile_rows - 1) / p.tile_rows;
  p.rows = p.G < p.tile_rows ? p.G : p.tile_rows;
  const int64_t items = static_cast<int64_t>(g.N) * sc->num_heads * p.head_tiles;
  // Blocks and units of an item, at most.  A window reaches into window / S + 2 chunks, and
  // tokens of one run lie in no more than a B-th of them, and two, blocks.
  int64_t blocks = g.M;
  if (window > 0) {
    const int64_t runs = g.Bpc == 1 && g.S == g.B ? 1 : int64_t{window} / g.S + 2;
    blocks = window / g.B + 2 * runs < blocks ? window / g.B + 2 * runs : blocks;
  }
  const int64_t unit = sc->dtype == OMNIMEM_BF16 && sc->head_dim == 64 ? 64 : 32;
  const int64_t units = blocks * (g.B / unit);
  // a sum of the sequences' units in 31 bits, positions on the line in 40
  if (items > 0x7fffffff / 256 || static_cast<int64_t>(g.N) * (static_cast<int64_t>(g.M) * (g.B / unit) + kItemOverhead) > 0x7fffffff ||
      (items > 0 && units > (int64_t{1} << 40) / items))
    return OMNIMEM_EINVAL;
  p.split = units <= kWaveUnitsMost && items >= kWaveItems ? DecodeSplit::kWave
            : units <= kItemUnitsMost                         ? DecodeSplit::kItem
                                                              : DecodeSplit::kLine;
  const int64_t most = items * (units + kItemOverhead);
  const int64_t wgs = items > kDecodeWgs ? kDecodeManyWgs : kDecodeWgs;
  if (most > wgs * 0x7fffffff) return OMNIMEM_EINVAL;  // a workgroup's share of the line in 31 bits
  p.wgs = static_cast<int>(p.split == DecodeSplit::kLine   ? (most < wgs ? most : wgs)
                           : p.split == DecodeSplit::kItem ? items
                                                           : (items + kDecodeWaves - 1) / kDecodeWaves);
  p.join_rows = items * 16 <= p.wgs ? 1 : p.rows >= 4 ? 4 : p.rows >= 2 ? 2 : 1;
  p.slot_floats = static_cast<size_t>(p.rows) * (sc->head_dim + 2);
  p.slot_floats = (p.slot_floats + 3) / 4 * 4;
  p.off_part = 0;
  const size_t shares = p.split == DecodeSplit::kLine ? p.wgs : 0;
  p.off_starts = align256(shares * 2 * p.slot_floats * sizeof(float));
  p.total = shares == 0 ? 256 : p.off_starts + align256(shares * sizeof(DecodeStart)) + 512;
  return OMNIMEM_OK;
}

omnimem_status_t check_scratch(const void* workspace, size_t have, size_t need) {
  if (workspace == nullptr || !aligned(workspace, 256)) return OMNIMEM_EINVAL;
  return have < need ? OMNIMEM_EWORKSPACE : OMNIMEM_OK;
}

// num_new: rows of an update, or 0 for a compaction of the table's rows.
omnimem_status_t plan_seq(const SeqGeom& g, int32_t num_new, SeqPlan& p) {
  if (num_new < 0 || static_cast<int64_t>(num_new) * g.M > 0x7fffffff || static_cast<int64_t>(g.N) * g.M > 0x7fffffff)
    return OMNIMEM_EINVAL;  // entries, and the pages that rows ask for, are counted in 31 bits
  const int rows = num_new > 0 ? num_new : g.N;
  p.one = g.num_pages <= kOnePages && rows <= kOneRows && static_cast<int64_t>(rows) * g.M <= kOneEntries;
  p.growing = num_new > 0;
  p.words = (g.num_pages + 31) / 32;
  const size_t map = align256(static_cast<size_t>(p.words) * 4);
  p.off_held = 0;
  p.off_tail = map;
  p.off_first = p.off_tail + (p.growing ? map : 0);
  p.off_rows = p.off_first + (p.growing ? align256(static_cast<size_t>(g.num_pages) * 4) : 0);
  p.total = p.one ? 256 : p.off_rows + align256(static_cast<size_t>(num_new) * sizeof(RowPlan)) + 512;
  return OMNIMEM_OK;
}

}  // namespace

size_t decode_workspace_bytes(const omnimem_seq_cache_t* sc, int32_t num_q_heads, int32_t window) {
  SeqGeom g;
  DecodePlan p;
  if (window < 0 || resolve_seq_cache(sc, g, true) != OMNIMEM_OK ||
      plan_decode(sc, g, num_q_heads, window, p) != OMNIMEM_OK)
    return 0;
  return p.total;
}

size_t seq_workspace_bytes(const omnimem_seq_table_t* st, int32_t num_new) {
  SeqGeom g;
  SeqPlan p;
  if (resolve_table(st, g, true) != OMNIMEM_OK || plan_seq(g, num_new, p) != OMNIMEM_OK) return 0;
  return p.total;
}

omnimem_status_t check_decode_attn(const omnimem_seq_cache_t* sc, const void* q, int64_t q_stride, int32_t num_q_heads,
                                   int32_t window, float scale, void* out, float* lse, const void* workspace,
                                   size_t workspace_bytes, SeqGeom& g, DecodePlan& p, DecodeLaunch& a) {
  omnimem_status_t st = resolve_seq_cache(sc, g, false);
  if (st == OMNIMEM_OK) st = plan_decode(sc, g, num_q_heads, window, p);
  if (st != OMNIMEM_OK) return st;
  if (window < 0 || !isfinite(scale) || !(scale > 0.f)) return OMNIMEM_EINVAL;
  if (!good_stride(q_stride, static_cast<int64_t>(num_q_heads) * sc->head_dim, elem_bytes(sc->dtype)))
    return OMNIMEM_EINVAL;
  if (g.N == 0) return OMNIMEM_OK;
  if (q == nullptr || out == nullptr || !aligned(q, 16) || !aligned(out, 16) || !aligned(lse, 4)) return OMNIMEM_EINVAL;
  a.dtype = sc->dtype;
  a.H = sc->num_heads;
  a.D = sc->head_dim;
  a.k_pages = sc->k_pages;
  a.v_pages = sc->v_pages;
  a.q = q;
  a.q_stride = q_stride;
  a.Hq = num_q_heads;
  a.window = window;
  a.scale = scale;
  a.out = out;
  a.lse = lse;
  return p.split != DecodeSplit::kLine ? OMNIMEM_OK : check_scratch(workspace, workspace_bytes, p.total);
}

omnimem_status_t check_append_kv(const omnimem_seq_cache_t* sc, const void* k, int64_t k_stride, const void* v,
                                 int64_t v_stride, int32_t tokens, const int32_t* starts, SeqGeom& g,
                                 AppendLaunch& a) {
  const omnimem_status_t st = resolve_seq_cache(sc, g, false);
  if (st != OMNIMEM_OK) return st;
  if (tokens < 0 || (starts == nullptr && tokens != g.N) || !aligned(starts, 4)) return OMNIMEM_EINVAL;
  const int64_t row = static_cast<int64_t>(sc->num_heads) * sc->head_dim, eb = elem_bytes(sc->dtype);
  if (!good_stride(k_stride, row, eb) || !good_stride(v_stride, row, eb)) return OMNIMEM_EINVAL;
  if (tokens > 0 && (k == nullptr || v == nullptr || !aligned(k, 16) || !aligned(v, 16))) return OMNIMEM_EINVAL;
  a.row_chunks = row * eb / 16;
  a.head_chunks = static_cast<int>(sc->head_dim * eb / 16);
  a.H = sc->num_heads;
  a.k = k;
  a.v = v;
  a.k_stride = k_stride * eb / 16;
  a.v_stride = v_stride * eb / 16;
  a.tokens = tokens;
  a.starts = starts;
  a.k_pages = sc->k_pages;
  a.v_pages = sc->v_pages;
  return OMNIMEM_OK;
}

omnimem_status_t check_copy_pages(void* k_pages, void* v_pages, int64_t num_pages, int64_t page_bytes, int32_t layers,
                                  int64_t layer_stride, const int32_t* pairs, const int32_t* count, int32_t max_pairs,
                                  CopyLaunch& a) {
  if (num_pages < 0 || num_pages > 0x7fffffff || page_bytes < 16 || page_bytes % 16 != 0 || layers < 0 ||
      layer_stride < 0 || layer_stride % 16 != 0 || max_pairs < 0)
    return OMNIMEM_EINVAL;
  const int64_t limit = int64_t{1} << 44;
  if (page_bytes > limit || (num_pages > 0 && page_bytes > limit / num_pages)) return OMNIMEM_EINVAL;
  if (layers > 1 && (layer_stride < num_pages * page_bytes || layer_stride > limit)) return OMNIMEM_EINVAL;
  if (!aligned(k_pages, 16) || !aligned(v_pages, 16) || !aligned(pairs, 4) || !aligned(count, 4)) return OMNIMEM_EINVAL;
  if (layers > 0 && num_pages > 0 && max_pairs > 0 && (k_pages == nullptr || pairs == nullptr)) return OMNIMEM_EINVAL;
  a.k_pages = k_pages;
  a.v_pages = v_pages;
  a.num_pages = num_pages;
  a.page_chunks = page_bytes / 16;
  a.layer_chunks = layer_stride / 16;
  a.layers = layers;
  a.pairs = pairs;
  a.count = count;
  a.max_pairs = max_pairs;
  return OMNIMEM_OK;
}

omnimem_status_t check_seq_update(const omnimem_seq_table_t* st, int32_t num_new, const int32_t* parent,
                                  const int32_t* keep, const int32_t* grow, int32_t* out_table, int32_t* out_lens,
                                  int32_t* copies, int32_t* info, const void* workspace, size_t workspace_bytes,
                                  SeqGeom& g, SeqPlan& p, SeqUpdateLaunch& a) {
  omnimem_status_t s = resolve_table(st, g, false);
  if (s == OMNIMEM_OK) s = plan_seq(g, num_new, p);
  if (s != OMNIMEM_OK) return s;
  if (info == nullptr || !aligned(info, 4)) return OMNIMEM_EINVAL;
  if (num_new > 0 && (parent == nullptr || out_table == nullptr || out_lens == nullptr || copies == nullptr))
    return OMNIMEM_EINVAL;
  if (!aligned(parent, 4) || !aligned(keep, 4) || !aligned(grow, 4) || !aligned(out_table, 4) ||
      !aligned(out_lens, 4) || !aligned(copies, 4))
    return OMNIMEM_EINVAL;
  if (g.N > 0 && (out_table == g.table || out_lens == g.lens)) return OMNIMEM_EINVAL;
  a = SeqUpdateLaunch{num_new, parent, keep, grow, out_table, out_lens, copies, info};
  return p.one ? OMNIMEM_OK : check_scratch(workspace, workspace_bytes, p.total);
}

omnimem_status_t check_seq_compact(const omnimem_seq_table_t* st, int32_t* out_table, int32_t* moves, int32_t* info,
                                   const void* workspace, size_t workspace_bytes, SeqGeom& g, SeqPlan& p,
                                   SeqUpdateLaunch& a) {
  omnimem_status_t s = resolve_table(st, g, false);
  if (s == OMNIMEM_OK) s = plan_seq(g, 0, p);
  if (s != OMNIMEM_OK) return s;
  if (info == nullptr || moves == nullptr || !aligned(info, 4) || !aligned(moves, 4) || !aligned(out_table, 4))
    return OMNIMEM_EINVAL;
  if (g.N > 0 && (out_table == nullptr || out_table == g.table)) return OMNIMEM_EINVAL;
  a = SeqUpdateLaunch{0, nullptr, nullptr, nullptr, out_table, nullptr, moves, info};
  return p.one ? OMNIMEM_OK : check_scratch(workspace, workspace_bytes, p.total);
}

}  // namespace omnimem
