// Host-only build of the sequence cache's work plans for tests/test_seq_plans.py (CPU only).
#include <stdint.h>

#include "../include/omnimem.h"
#include "../paper_2605_30519_amd/csrc/seq.h"

using namespace omnimem;

// {one, growing, words, off_held, off_tail, off_first, off_rows, total, bytes of a row's record} of an
// update to n rows; the status of its checks with that workspace.
extern "C" omnimem_status_t shim_update_plan(const omnimem_seq_table_t* st, int32_t n, int64_t* out) {
  SeqGeom g;
  SeqPlan p;
  SeqUpdateLaunch a;
  int32_t* const fake = reinterpret_cast<int32_t*>(0x10000);
  const size_t need = seq_workspace_bytes(st, n);
  const omnimem_status_t s = check_seq_update(st, n, fake, fake, fake, fake + 64, fake + 64, fake + 128, fake + 192, fake,
                                              need, g, p, a);
  if (s != OMNIMEM_OK) return s;
  const int64_t all[] = {p.one, p.growing, p.words, static_cast<int64_t>(p.off_held), static_cast<int64_t>(p.off_tail),
                         static_cast<int64_t>(p.off_first), static_cast<int64_t>(p.off_rows),
                         static_cast<int64_t>(p.total), static_cast<int64_t>(sizeof(RowPlan))};
  for (int i = 0; i < 9; ++i) out[i] = all[i];
  return s;
}

// {split (0: line), wgs, items, most units of an item} of a decode call; the units are the table's or
// the window's.
extern "C" omnimem_status_t shim_decode_plan(const omnimem_seq_cache_t* sc, int32_t heads, int32_t window, int64_t* out) {
  SeqGeom g;
  DecodePlan p;
  DecodeLaunch a;
  void* const fake = reinterpret_cast<void*>(0x10000);
  const omnimem_status_t s = check_decode_attn(sc, fake, static_cast<int64_t>(heads) * sc->head_dim, heads, window, 0.1f,
                                               fake, nullptr, fake, static_cast<size_t>(1) << 62, g, p, a);
  if (s != OMNIMEM_OK) return s;
  const int unit = sc->dtype == OMNIMEM_BF16 && sc->head_dim == 64 ? 64 : 32;
  out[0] = static_cast<int64_t>(p.split);
  out[1] = p.wgs;
  out[2] = static_cast<int64_t>(g.N) * sc->num_heads * p.head_tiles;
  out[3] = static_cast<int64_t>(g.M) * (g.B / unit);
  return s;
}
