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

bool known_dtype(int32_t dtype) { return dtype == OMNIMEM_BF16 || dtype == OMNIMEM_F32; }

omnimem_status_t resolve_pools(const omnimem_seq_table_t& seqs, int32_t num_heads, int32_t head_dim, const void* k_pages,
                               const void* v_pages, SeqGeom& g, bool sizes_only) {
  if (head_dim != 64 && head_dim != 128) return OMNIMEM_EUNSUPPORTED;
  if (num_heads < 1 || num_heads > (1 << 20)) return OMNIMEM_EINVAL;
  const omnimem_status_t st = resolve_table(&seqs, g, sizes_only);
  if (st != OMNIMEM_OK) return st;
  // the pool's elements stay inside int64 index arithmetic
  if (g.num_pages > (int64_t{1} << 40) / (static_cast<int64_t>(num_heads) * g.B * head_dim)) return OMNIMEM_EINVAL;
  if (!sizes_only && g.num_pages > 0 && (k_pages == nullptr || v_pages == nullptr)) return OMNIMEM_EINVAL;
  if (!aligned(k_pages, 16) || !aligned(v_pages, 16)) return OMNIMEM_EINVAL;
  return OMNIMEM_OK;
}

omnimem_status_t resolve_seq_cache(const omnimem_seq_cache_t* sc, SeqGeom& g, bool sizes_only) {
  if (sc == nullptr) return OMNIMEM_EINVAL;
  if (!known_dtype(sc->dtype)) return OMNIMEM_EUNSUPPORTED;
  return resolve_pools(sc->seqs, sc->num_heads, sc->head_dim, sc->k_pages, sc->v_pages, g, sizes_only);
}

omnimem_status_t resolve_quant_cache(const omnimem_seq_cache_quant_t* sc, SeqGeom& g, bool sizes_only) {
  if (sc == nullptr) return OMNIMEM_EINVAL;
  const omnimem_status_t st = resolve_pools(sc->seqs, sc->num_heads, sc->head_dim, sc->k_pages, sc->v_pages, g, sizes_only);
  if (st != OMNIMEM_OK) return st;
  if (!sizes_only && g.num_pages > 0 && sc->scales == nullptr) return OMNIMEM_EINVAL;
  return aligned(sc->scales, 8) ? OMNIMEM_OK : OMNIMEM_EINVAL;
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
// Two column tiles over 8-bit pages, from this many bytes of K and V on both a wave's, which is
// then held up less by memory than by a key's and a value's widening, once for both; below, each every
// other wave's.  The bytes are what a call can read at most: of the blocks that a window leaves, half the threshold,
// since sequences are mostly longer than it; else of the table's capacity, which they seldom fill.  24 query heads a key
// head, bf16, pairs and both: 4 sequences of 60 to 90 thousand tokens, 8 key heads (704 MB of capacity) 141.6 / 114.6 us,
// 16 of 3 to 20 thousand (628 MB) 81.8 / 68.2, 16 of an eighth to all of 256 MB 42.7 / 40.8, of 192 MB 33.2 / 38.0; windows over
// tables of 1 GB and more, 16 sequences: 256 MB 78.4 / 62.7, 128 MB 46.5 / 42.2, 96 MB 36.7 / 37.5, 1,560 tokens (52 MB) 27.3 /
// 31.0; heads of 64, 16 key heads, 4,000 tokens (128 MB) 47.5 / 43.5.  fp32 queries of 128 dims hold three pieces of both
// tiles, which leaves one workgroup a CU and less to gain: 16 sequences of an eighth to all of 512 MB 74.3 / 79.0, 4 of 60
// to 90 thousand tokens (704 MB) 161.4 / 158.6; more items than CUs end more often, 40 sequences of 384 MB 61.8 / 77.0, of 768 MB
// 100.5 / 118.2; windows, 16 sequences, 192 MB 67.3 / 71.2, 384 MB 113.4 / 112.8.  Of 64 dims they are as bf16: 512 MB 74.9 / 67.2,
// windows of 128 MB 51.2 / 47.7.
constexpr double kBothBytes = 256 << 20, kBothBytesF32 = 640 << 20, kBothBytesF32Many = 1024 << 20;
constexpr int64_t kItemOverhead = 64;  // of an item's length on the line, no less than the kernel adds

// What a plan goes by, of a kind of pages: tokens of a unit; units of the longest item that is a
// workgroup's, and of one that a window bounds where there is an item for each CU; workgroups of a line
// where there are no more items than CUs and where there are; whether these are 8-bit pages, whose
// kernels have forms and joins of their own; of those, kBothBytes for the queries' type, in both places.
struct DecodeTuning {
  int64_t unit, item_units, window_units, wgs, many_wgs;
  bool eight_bit;
  double both_bytes, many_both_bytes;
};

omnimem_status_t plan_decode(int32_t num_heads, int32_t head_dim, const DecodeTuning& t, const SeqGeom& g,
                             int32_t num_q_heads, int32_t window, DecodePlan& p) {
  if (num_q_heads < 1 || num_q_heads % num_heads != 0) return OMNIMEM_EINVAL;
  p.G = num_q_heads / num_heads;
  const auto tile = [&p](int rows) {
    p.tile_rows = rows;
    p.head_tiles = (p.G + rows - 1) / rows;
    p.rows = p.G < rows ? p.G : rows;
  };
  tile(p.G <= kDecodeHeadRows ? kDecodeHeadRows : 2 * kDecodeHeadRows);
  int64_t items = static_cast<int64_t>(g.N) * num_heads * p.head_tiles;
  // Blocks and units of an item, at most.  A window reaches into window / S + 2 chunks, and
  // tokens of one run lie in no more than a B-th of them, and two, blocks.
  int64_t blocks = g.M;
  if (window > 0) {
    const int64_t runs = g.Bpc == 1 && g.S == g.B ? 1 : int64_t{window} / g.S + 2;
    blocks = window / g.B + 2 * runs < blocks ? window / g.B + 2 * runs : blocks;
  }
  const int64_t unit = t.unit, units = blocks * (g.B / unit);
  // a sum of the sequences' units in 31 bits, positions on the line in 40
  if (items > 0x7fffffff / 256 || static_cast<int64_t>(g.N) * (static_cast<int64_t>(g.M) * (g.B / unit) + kItemOverhead) > 0x7fffffff ||
      (items > 0 && units > (int64_t{1} << 40) / items))
    return OMNIMEM_EINVAL;
  const bool pair = t.eight_bit && p.tile_rows > kDecodeHeadRows;
  const int64_t item_units = window > 0 && items >= kDecodeWgs ? t.window_units : pair ? t.item_units * 2 / 3 : t.item_units;
  p.split = units <= kWaveUnitsMost && items >= kWaveItems ? DecodeSplit::kWave
            : units <= item_units                             ? DecodeSplit::kItem
                                                              : DecodeSplit::kLine;
  if (p.split == DecodeSplit::kWave && t.eight_bit) {
    tile(kDecodeHeadRows);
    items = static_cast<int64_t>(g.N) * num_heads * p.head_tiles;
  }
  const int64_t most = items * (units + kItemOverhead);
  p.eight_waves = t.eight_bit && head_dim == 64 && p.tile_rows == kDecodeHeadRows && p.split == DecodeSplit::kItem &&
                  items <= kDecodeWgs / 2 && units > 4;
  p.pair = pair && p.tile_rows > kDecodeHeadRows;
  const double bytes = 2. * g.N * blocks * num_heads * g.B * head_dim;
  const double both_bytes = items > kDecodeWgs ? t.many_both_bytes : t.both_bytes;
  const bool both = p.pair && p.split == DecodeSplit::kLine && bytes >= (blocks < g.M ? both_bytes / 2 : both_bytes);
  if (both) p.pair = false;
  const int64_t most_wgs = items > kDecodeWgs ? t.many_wgs : t.wgs;
  const int64_t wgs = both && head_dim == 128 ? kDecodeWgs : most_wgs;
  if (most > wgs * 0x7fffffff) return OMNIMEM_EINVAL;  // a workgroup's share of the line in 31 bits
  p.wgs = static_cast<int>(p.split == DecodeSplit::kLine   ? (most < wgs ? most : wgs)
                           : p.split == DecodeSplit::kItem ? items
                                                           : (items + kDecodeWaves - 1) / kDecodeWaves);
  p.long_items = t.eight_bit && items * 64 <= p.wgs;
  if (!t.eight_bit) p.join_rows = items * 16 <= p.wgs ? 1 : p.rows >= 4 ? 4 : p.rows >= 2 ? 2 : 1;
  else p.join_rows = p.long_items || p.rows == 1 ? 1 : 2;
  p.slot_floats = static_cast<size_t>(p.rows) * (head_dim + 2);
  p.slot_floats = (p.slot_floats + 3) / 4 * 4;
  p.off_part = 0;
  // of either form: the workspace's size is asked for without the queries' type
  const size_t shares = p.split != DecodeSplit::kLine ? 0 : most < most_wgs ? most : most_wgs;
  p.off_starts = align256(shares * 2 * p.slot_floats * sizeof(float));
  p.total = shares == 0 ? 256 : p.off_starts + align256(shares * sizeof(DecodeStart)) + 512;
  return OMNIMEM_OK;
}

omnimem_status_t plan_decode(const omnimem_seq_cache_t* sc, const SeqGeom& g, int32_t num_q_heads, int32_t window,
                             DecodePlan& p) {
  const DecodeTuning t{sc->dtype == OMNIMEM_BF16 && sc->head_dim == 64 ? 64 : 32, kItemUnitsMost, kItemUnitsMost, kDecodeWgs,
                       kDecodeManyWgs, false, 0, 0};
  return plan_decode(sc->num_heads, sc->head_dim, t, g, num_q_heads, window, p);
}

// 8-bit pages (the kernels' times, with the join's, in a graph).  A wave's tile of 64-dim heads is 8 KB
// instead of 16, so two workgroups a CU: 12 sequences of 4,000 to 30,000 tokens, 16 key heads, 62.7 ->
// 58.3 us; an item of one goes twice as far: a window of 1,560 tokens, 256 items 23.6 -> 12.7, 4 items
// 10.2 -> 11.6, but a launch less.  Two column tiles of 128-dim heads need a CU's registers for one workgroup:
// 16 sequences of 3,000 to 9,000 tokens, 17 query heads on each of 4, bf16, 36.0 -> 32.9 (two spill).
// Column tiles in pairs of waves leave an item two waves for each, so it is a workgroup's for two thirds of
// that length: 24 query heads, 17 units 16.7 against 14.6, 10 units 11.4 / 14.5.  A CU takes in an item of
// 128-dim heads no faster with eight waves, one of 64 does: a window of 1,560 tokens, 32 items, fp32 11.8 ->
// 10.3, bf16 10.1 -> 8.7, but 240 items 12.8 -> 13.0, 3 units 5.0 -> 5.3.
// Windows make items of one length: 256 of 2,400 tokens, bf16 heads of 128, 36.2 -> 28.1, fp32 heads of
// 64 28.3 -> 17.1, where 32 items lose (15.4 -> 20.1, 14.0 -> 15.0).
omnimem_status_t plan_decode(const omnimem_seq_cache_quant_t* sc, int32_t dtype, const SeqGeom& g, int32_t num_q_heads,
                             int32_t window, DecodePlan& p) {
  const bool f32 = dtype == OMNIMEM_F32 && sc->head_dim == 128;
  const double both = f32 ? kBothBytesF32 : kBothBytes, many_both = f32 ? kBothBytesF32Many : kBothBytes;
  const DecodeTuning t = sc->head_dim == 64 ? DecodeTuning{64, 28, 48, kDecodeManyWgs, kDecodeManyWgs, true, both, many_both}
                                            : DecodeTuning{64, 20, 48, kDecodeWgs, kDecodeManyWgs, true, both, many_both};
  return plan_decode(sc->num_heads, sc->head_dim, t, g, num_q_heads, window, p);
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

size_t decode_quant_workspace_bytes(const omnimem_seq_cache_quant_t* sc, int32_t num_q_heads, int32_t window) {
  SeqGeom g;
  DecodePlan p;
  if (window < 0 || resolve_quant_cache(sc, g, true) != OMNIMEM_OK ||
      plan_decode(sc, OMNIMEM_BF16, g, num_q_heads, window, p) != OMNIMEM_OK)
    return 0;
  return p.total;
}

size_t seq_workspace_bytes(const omnimem_seq_table_t* st, int32_t num_new) {
  SeqGeom g;
  SeqPlan p;
  if (resolve_table(st, g, true) != OMNIMEM_OK || plan_seq(g, num_new, p) != OMNIMEM_OK) return 0;
  return p.total;
}

namespace {

// Of a decode call behind its cache and plan.
omnimem_status_t check_decode(const SeqGeom& g, const DecodePlan& p, const DecodeLaunch& a, const void* workspace,
                              size_t workspace_bytes) {
  if (a.window < 0 || !isfinite(a.scale) || !(a.scale > 0.f)) return OMNIMEM_EINVAL;
  if (!good_stride(a.q_stride, static_cast<int64_t>(a.Hq) * a.D, elem_bytes(a.dtype))) return OMNIMEM_EINVAL;
  if (g.N == 0) return OMNIMEM_OK;
  if (a.q == nullptr || a.out == nullptr || !aligned(a.q, 16) || !aligned(a.out, 16) || !aligned(a.lse, 4))
    return OMNIMEM_EINVAL;
  return p.split != DecodeSplit::kLine ? OMNIMEM_OK : check_scratch(workspace, workspace_bytes, p.total);
}

}  // namespace

omnimem_status_t check_decode_attn(const omnimem_seq_cache_t* sc, const void* q, int64_t q_stride, int32_t num_q_heads,
                                   int32_t window, float scale, void* out, float* lse, const void* workspace,
                                   size_t workspace_bytes, SeqGeom& g, DecodePlan& p, DecodeLaunch& a) {
  omnimem_status_t st = resolve_seq_cache(sc, g, false);
  if (st == OMNIMEM_OK) st = plan_decode(sc, g, num_q_heads, window, p);
  if (st != OMNIMEM_OK) return st;
  a = DecodeLaunch{sc->dtype, sc->num_heads, sc->head_dim, sc->k_pages, sc->v_pages, nullptr,
                   q,         q_stride,      num_q_heads,  window,      scale,       out, lse};
  return check_decode(g, p, a, workspace, workspace_bytes);
}

omnimem_status_t check_decode_attn_quant(const omnimem_seq_cache_quant_t* sc, int32_t dtype, const void* q, int64_t q_stride,
                                         int32_t num_q_heads, int32_t window, float scale, void* out, float* lse,
                                         const void* workspace, size_t workspace_bytes, SeqGeom& g, DecodePlan& p,
                                         DecodeLaunch& a) {
  if (!known_dtype(dtype)) return OMNIMEM_EUNSUPPORTED;
  omnimem_status_t st = resolve_quant_cache(sc, g, false);
  if (st == OMNIMEM_OK) st = plan_decode(sc, dtype, g, num_q_heads, window, p);
  if (st != OMNIMEM_OK) return st;
  a = DecodeLaunch{dtype, sc->num_heads, sc->head_dim, sc->k_pages, sc->v_pages, sc->scales,
                   q,     q_stride,      num_q_heads,  window,      scale,       out, lse};
  return check_decode(g, p, a, workspace, workspace_bytes);
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
  a.scales = nullptr;
  a.page_scales = a.layer_scales = 0;
  return OMNIMEM_OK;
}

omnimem_status_t check_append_kv_quant(const omnimem_seq_cache_quant_t* sc, int32_t dtype, const void* k, int64_t k_stride,
                                       const void* v, int64_t v_stride, int32_t tokens, const int32_t* starts, SeqGeom& g,
                                       AppendQuantLaunch& a) {
  if (!known_dtype(dtype)) return OMNIMEM_EUNSUPPORTED;
  const omnimem_status_t st = resolve_quant_cache(sc, g, false);
  if (st != OMNIMEM_OK) return st;
  if (tokens < 0 || (starts == nullptr && tokens != g.N) || !aligned(starts, 4)) return OMNIMEM_EINVAL;
  const int64_t row = static_cast<int64_t>(sc->num_heads) * sc->head_dim, eb = elem_bytes(dtype);
  if (!good_stride(k_stride, row, eb) || !good_stride(v_stride, row, eb)) return OMNIMEM_EINVAL;
  if (tokens > 0 && (k == nullptr || v == nullptr || !aligned(k, 16) || !aligned(v, 16))) return OMNIMEM_EINVAL;
  a = AppendQuantLaunch{dtype,  sc->num_heads, sc->head_dim, k, v, k_stride, v_stride, tokens,
                     starts, sc->k_pages,   sc->v_pages,  sc->scales};
  return OMNIMEM_OK;
}

omnimem_status_t check_read_kv_quant(const omnimem_seq_cache_quant_t* sc, int32_t dtype, int32_t tokens, const int32_t* starts,
                                     const int32_t* first, void* out_k, void* out_v, SeqGeom& g, ReadQuantLaunch& a) {
  if (!known_dtype(dtype)) return OMNIMEM_EUNSUPPORTED;
  const omnimem_status_t st = resolve_quant_cache(sc, g, false);
  if (st != OMNIMEM_OK) return st;
  if (tokens < 0 || (starts == nullptr && tokens != g.N) || !aligned(starts, 4) || !aligned(first, 4))
    return OMNIMEM_EINVAL;
  if (tokens > 0 && (out_k == nullptr || out_v == nullptr)) return OMNIMEM_EINVAL;
  if (!aligned(out_k, 16) || !aligned(out_v, 16)) return OMNIMEM_EINVAL;
  a = ReadQuantLaunch{dtype,       sc->num_heads, sc->head_dim, tokens, starts, first,
                   sc->k_pages, sc->v_pages,   sc->scales,   out_k,  out_v};
  return OMNIMEM_OK;
}

omnimem_status_t check_copy_pages_quant(void* k_pages, void* v_pages, float* scales, int64_t num_pages, int32_t num_heads,
                                        int32_t block_size, int32_t head_dim, int32_t layers, int64_t layer_stride,
                                        int64_t scale_stride, const int32_t* pairs, const int32_t* count, int32_t max_pairs,
                                        CopyLaunch& a) {
  if ((block_size != 64 && block_size != 128) || (head_dim != 64 && head_dim != 128)) return OMNIMEM_EUNSUPPORTED;
  if (num_heads < 1 || num_heads > (1 << 20)) return OMNIMEM_EINVAL;
  const int64_t page_bytes = static_cast<int64_t>(num_heads) * block_size * head_dim;
  const omnimem_status_t st =
      check_copy_pages(k_pages, v_pages, num_pages, page_bytes, layers, layer_stride, pairs, count, max_pairs, a);
  if (st != OMNIMEM_OK) return st;
  if (scale_stride < 0 || scale_stride % 8 != 0 || !aligned(scales, 8)) return OMNIMEM_EINVAL;
  if (layers > 1 && (scale_stride < num_pages * num_heads * 8 || scale_stride > (int64_t{1} << 44))) return OMNIMEM_EINVAL;
  if (layers > 0 && num_pages > 0 && max_pairs > 0 && (v_pages == nullptr || scales == nullptr)) return OMNIMEM_EINVAL;
  a.scales = scales;
  a.page_scales = num_heads;
  a.layer_scales = scale_stride / 8;
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
