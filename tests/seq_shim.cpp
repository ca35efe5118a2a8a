// Host-only build of the sequence cache's argument checks, for the sanitizer test (CPU only;
// never loaded next to the real library).  Each entry point runs the library's own checks
// from seq.cpp and returns their status where the library would launch its kernels.
#include <stdint.h>

#include "../include/omnimem.h"
#include "../paper_2605_30519_amd/csrc/seq.h"

using namespace omnimem;

extern "C" {

size_t omnimem_decode_workspace_bytes(const omnimem_seq_cache_t* sc, int32_t heads, int32_t window) {
  return decode_workspace_bytes(sc, heads, window);
}
size_t omnimem_seq_workspace_bytes(const omnimem_seq_table_t* st, int32_t n) { return seq_workspace_bytes(st, n); }

omnimem_status_t omnimem_decode_attn(const omnimem_seq_cache_t* sc, const void* q, int64_t q_stride, int32_t heads,
                                     int32_t window, float scale, void* out, float* lse, void* ws, size_t n, void*) {
  SeqGeom g;
  DecodePlan p;
  DecodeLaunch a;
  return check_decode_attn(sc, q, q_stride, heads, window, scale, out, lse, ws, n, g, p, a);
}

omnimem_status_t omnimem_append_kv(const omnimem_seq_cache_t* sc, const void* k, int64_t ks, const void* v, int64_t vs,
                                   int32_t tokens, const int32_t* starts, void*) {
  SeqGeom g;
  AppendLaunch a;
  return check_append_kv(sc, k, ks, v, vs, tokens, starts, g, a);
}

omnimem_status_t omnimem_copy_pages(void* k, void* v, int64_t pages, int64_t bytes, int32_t layers, int64_t step,
                                    const int32_t* pairs, const int32_t* count, int32_t most, void*) {
  CopyLaunch a;
  return check_copy_pages(k, v, pages, bytes, layers, step, pairs, count, most, a);
}

omnimem_status_t omnimem_seq_update(const omnimem_seq_table_t* st, int32_t n, const int32_t* parent, const int32_t* keep,
                                    const int32_t* grow, int32_t* rows, int32_t* lens, int32_t* copies, int32_t* info,
                                    void* ws, size_t size, void*) {
  SeqGeom g;
  SeqPlan p;
  SeqUpdateLaunch a;
  return check_seq_update(st, n, parent, keep, grow, rows, lens, copies, info, ws, size, g, p, a);
}

omnimem_status_t omnimem_seq_compact(const omnimem_seq_table_t* st, int32_t* rows, int32_t* moves, int32_t* info,
                                     void* ws, size_t size, void*) {
  SeqGeom g;
  SeqPlan p;
  SeqUpdateLaunch a;
  return check_seq_compact(st, rows, moves, info, ws, size, g, p, a);
}

}  // extern "C"
