// seq.h -- host-side geometry, argument checks and work plans of the sequence cache's
// entry points (internal to the library).  No HIP here: seq.cpp builds with the host
// compiler alone, so the checks also run on a CPU under sanitizers.
#pragma once

#include <stddef.h>
#include <stdint.h>

#include "../../include/omnimem.h"

namespace omnimem {

// Rows of a sequence table: token t of a row lies in block (t / S) * Bpc + (t % S) / B.
// A contiguous sequence (S a multiple of B) is resolved to S = B, Bpc = 1.
struct SeqGeom {
  int N, M, B, S, Bpc;
  int cap;  // capacity of a row in tokens
  int64_t num_pages;
  const int32_t* table;  // [N][M]
  const int32_t* lens;   // [N]
};

// ---------------------------------------------------------------- decode
// The (sequence, key/value head, tile of query heads) items of a call, each of them its
// sequence's units of 32 tokens (64 for bf16 heads of 64 and for 8-bit pages) in turn, form one line, which `wgs`
// workgroups share evenly; or, where sequences are short, an item is a workgroup's, or a wave's.
enum class DecodeSplit { kLine, kItem, kWave };
constexpr int kDecodeWaves = 4;
constexpr int kDecodeHeadRows = 16;  // query heads of an MFMA tile

struct DecodePlan {
  int G;             // query heads of a key/value head
  int head_tiles;    // tiles of query heads of a key/value head
  int tile_rows;     // query heads of a tile: 16 or 32
  int rows;          // of them in use, min(G, tile_rows)
  int wgs;           // workgroups
  DecodeSplit split;
  int join_rows;     // query heads of a workgroup that joins shares
  bool long_items;   // 8-bit pages: items of many shares, joined by larger workgroups a head
  bool eight_waves;  // 8-bit pages: a workgroup's item is eight waves', not four
  bool pair;         // 8-bit pages: of two column tiles, each is every other wave's
  size_t off_part, off_starts, total;
  size_t slot_floats;  // one workgroup's partial result of one item: O [rows][d], max [rows], sum [rows]
};

// Where a workgroup's share of the line begins: inside an item (units > 0) that earlier
// workgroups began, or not (units = 0).
struct DecodeStart {
  int64_t first;   // the item's first position on the line
  int units;       // its units
  int seq, head;   // its sequence, its (key/value head, tile) pair
  int share;       // units of a workgroup
};

struct DecodeLaunch {
  int dtype, H, D;
  const void* k_pages;
  const void* v_pages;
  const float* scales;  // [page][head][2] of 8-bit pages, else null
  const void* q;
  int64_t q_stride;  // elements
  int Hq, window;
  float scale;
  void* out;
  float* lse;
};

// ---------------------------------------------------------------- pages
struct AppendLaunch {
  int64_t row_chunks;     // 16-byte chunks of a token's row, H * d * bytes / 16
  int head_chunks;        // of one head
  int H;
  const void* k;
  const void* v;
  int64_t k_stride, v_stride;  // chunks
  int tokens;
  const int32_t* starts;  // or null: one token per sequence
  void* k_pages;
  void* v_pages;
};

struct CopyLaunch {
  void* k_pages;
  void* v_pages;
  int64_t num_pages, page_chunks, layer_chunks;  // 16-byte chunks
  int layers;
  const int32_t* pairs;
  const int32_t* count;
  int max_pairs;
  float* scales;                       // of 8-bit pages, else null
  int64_t page_scales, layer_scales;   // (K, V) pairs
};

// ---------------------------------------------------------------- 8-bit pages
struct AppendQuantLaunch {
  int dtype, H, D;             // of k and v
  const void* k;
  const void* v;
  int64_t k_stride, v_stride;  // elements
  int tokens;
  const int32_t* starts;       // or null: one token per sequence
  void* k_pages;
  void* v_pages;
  float* scales;
};

struct ReadQuantLaunch {
  int dtype, H, D;             // of the rows
  int tokens;
  const int32_t* starts;       // or null: one token per sequence
  const int32_t* first;        // or null: each sequence's last tokens
  const void* k_pages;
  const void* v_pages;
  const float* scales;
  void* out_k;
  void* out_v;
};

// Scratch of the table updates: a bitmap of the pool's pages, and where there are new rows a
// second one, one word per page (the lowest growing row of a page) and the rows' records.
// A workgroup with its state in LDS does small tables instead.  One launch costs the host 6 us
// less than three; on the GPU, 16 rows of 18 entries take 7.1 us against 10.6 (update; compaction
// 5.2 / 8.6), 16 of 252 9.2 / 11.9 (9.3 / 13.3), 8 of 939 11.6 / 12.0 (13.4 / 11.5), 256 of 65 27 / 14
// (29 / 13): one CU's instruction rate.
constexpr int kOneThreads = 1024, kOnePages = 16384, kOneRows = 1024;
constexpr int64_t kOneEntries = 8192;

struct SeqPlan {
  bool one;
  bool growing;   // new rows may write to pages: a second bitmap, `first` and `rows` have their place
  int64_t words;  // 32-page words of a bitmap
  size_t off_held, off_tail, off_first, off_rows, total;
};

struct RowPlan {   // of a new row
  int parent;
  int kept;         // blocks it takes over
  int added;        // blocks it gets
  int tail_page;    // page of the begun block that it will write to, or -1
  int len, short_len;  // tokens with its growth and without
  int over;         // its growth would pass the capacity
  int unused;
};

struct SeqUpdateLaunch {
  int num_new;
  const int32_t* parent;
  const int32_t* keep;
  const int32_t* grow;
  int32_t* out_table;
  int32_t* out_lens;
  int32_t* pairs;  // copies or moves
  int32_t* info;
};

size_t decode_workspace_bytes(const omnimem_seq_cache_t* sc, int32_t num_q_heads, int32_t window);
size_t seq_workspace_bytes(const omnimem_seq_table_t* st, int32_t num_new);
size_t decode_quant_workspace_bytes(const omnimem_seq_cache_quant_t* sc, int32_t num_q_heads, int32_t window);

omnimem_status_t check_decode_attn(const omnimem_seq_cache_t* sc, const void* q, int64_t q_stride, int32_t num_q_heads,
                                   int32_t window, float scale, void* out, float* lse, const void* workspace,
                                   size_t workspace_bytes, SeqGeom& g, DecodePlan& p, DecodeLaunch& a);
omnimem_status_t check_append_kv(const omnimem_seq_cache_t* sc, const void* k, int64_t k_stride, const void* v,
                                 int64_t v_stride, int32_t tokens, const int32_t* starts, SeqGeom& g, AppendLaunch& a);
omnimem_status_t check_copy_pages(void* k_pages, void* v_pages, int64_t num_pages, int64_t page_bytes, int32_t layers,
                                  int64_t layer_stride, const int32_t* pairs, const int32_t* count, int32_t max_pairs,
                                  CopyLaunch& a);
omnimem_status_t check_decode_attn_quant(const omnimem_seq_cache_quant_t* sc, int32_t dtype, const void* q, int64_t q_stride,
                                         int32_t num_q_heads, int32_t window, float scale, void* out, float* lse,
                                         const void* workspace, size_t workspace_bytes, SeqGeom& g, DecodePlan& p,
                                         DecodeLaunch& a);
omnimem_status_t check_append_kv_quant(const omnimem_seq_cache_quant_t* sc, int32_t dtype, const void* k, int64_t k_stride,
                                       const void* v, int64_t v_stride, int32_t tokens, const int32_t* starts, SeqGeom& g,
                                       AppendQuantLaunch& a);
omnimem_status_t check_read_kv_quant(const omnimem_seq_cache_quant_t* sc, int32_t dtype, int32_t tokens, const int32_t* starts,
                                     const int32_t* first, void* out_k, void* out_v, SeqGeom& g, ReadQuantLaunch& a);
omnimem_status_t check_copy_pages_quant(void* k_pages, void* v_pages, float* scales, int64_t num_pages, int32_t num_heads,
                                        int32_t block_size, int32_t head_dim, int32_t layers, int64_t layer_stride,
                                        int64_t scale_stride, const int32_t* pairs, const int32_t* count, int32_t max_pairs,
                                        CopyLaunch& a);
omnimem_status_t check_seq_update(const omnimem_seq_table_t* st, int32_t num_new, const int32_t* parent,
                                  const int32_t* keep, const int32_t* grow, int32_t* out_table, int32_t* out_lens,
                                  int32_t* copies, int32_t* info, const void* workspace, size_t workspace_bytes,
                                  SeqGeom& g, SeqPlan& p, SeqUpdateLaunch& a);
omnimem_status_t check_seq_compact(const omnimem_seq_table_t* st, int32_t* out_table, int32_t* moves, int32_t* info,
                                   const void* workspace, size_t workspace_bytes, SeqGeom& g, SeqPlan& p,
                                   SeqUpdateLaunch& a);

}  // namespace omnimem
