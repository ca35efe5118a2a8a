// Host-only build of the 8-bit sequence cache's argument checks and plans, for the sanitizer and plan tests
// (CPU only; never loaded next to the real library).  Each entry point runs the library's own checks
// from seq.cpp and returns their status where the library would launch its kernels.
#include <stdint.h>

#include "../include/omnimem.h"
#include "../paper_2605_30519_amd/csrc/seq.h"

using namespace omnimem;

extern "C" {

size_t omnimem_decode_quant_workspace_bytes(const omnimem_seq_cache_quant_t* sc, int32_t heads, int32_t window) {
  return decode_quant_workspace_bytes(sc, heads, window);
}

omnimem_status_t omnimem_decode_attn_quant(const omnimem_seq_cache_quant_t* sc, int32_t dtype, const void* q,
                                           int64_t q_stride, int32_t heads, int32_t window, float scale, void* out,
                                           float* lse, void* ws, size_t n, void*) {
  SeqGeom g;
  DecodePlan p;
  DecodeLaunch a;
  return check_decode_attn_quant(sc, dtype, q, q_stride, heads, window, scale, out, lse, ws, n, g, p, a);
}

omnimem_status_t omnimem_append_kv_quant(const omnimem_seq_cache_quant_t* sc, int32_t dtype, const void* k, int64_t ks,
                                         const void* v, int64_t vs, int32_t tokens, const int32_t* starts, void*) {
  SeqGeom g;
  AppendQuantLaunch a;
  return check_append_kv_quant(sc, dtype, k, ks, v, vs, tokens, starts, g, a);
}

omnimem_status_t omnimem_read_kv_quant(const omnimem_seq_cache_quant_t* sc, int32_t dtype, int32_t tokens,
                                       const int32_t* starts, const int32_t* first, void* k, void* v, void*) {
  SeqGeom g;
  ReadQuantLaunch a;
  return check_read_kv_quant(sc, dtype, tokens, starts, first, k, v, g, a);
}

omnimem_status_t omnimem_copy_pages_quant(void* k, void* v, float* s, int64_t pages, int32_t heads, int32_t B, int32_t d,
                                          int32_t layers, int64_t step, int64_t sstep, const int32_t* pairs,
                                          const int32_t* count, int32_t most, void*) {
  CopyLaunch a;
  return check_copy_pages_quant(k, v, s, pages, heads, B, d, layers, step, sstep, pairs, count, most, a);
}

// {split (0: line), wgs, items, most units of an item, bytes of the shares, their offset, the starts' offset,
// total, bytes of the starts} of a decode call.
omnimem_status_t shim_decode_quant_plan(const omnimem_seq_cache_quant_t* sc, int32_t heads, int32_t window, int64_t* out) {
  SeqGeom g;
  DecodePlan p;
  DecodeLaunch a;
  void* const fake = reinterpret_cast<void*>(0x10000);
  const omnimem_status_t s = check_decode_attn_quant(sc, OMNIMEM_BF16, fake, static_cast<int64_t>(heads) * sc->head_dim,
                                                     heads, window, 0.1f, fake, nullptr, fake, static_cast<size_t>(1) << 62,
                                                     g, p, a);
  if (s != OMNIMEM_OK) return s;
  out[0] = static_cast<int64_t>(p.split);
  out[1] = p.wgs;
  out[2] = static_cast<int64_t>(g.N) * sc->num_heads * p.head_tiles;
  out[3] = static_cast<int64_t>(g.M) * (g.B / 64);
  out[4] = static_cast<int64_t>(p.wgs) * 2 * static_cast<int64_t>(p.slot_floats * sizeof(float));
  out[5] = static_cast<int64_t>(p.off_part);
  out[6] = static_cast<int64_t>(p.off_starts);
  out[7] = static_cast<int64_t>(p.total);
  out[8] = static_cast<int64_t>(sizeof(DecodeStart)) * p.wgs;
  return s;
}

}  // extern "C"
