// Host-only build of the 8-bit cache's decode plans for tests/test_quant_forms.py (CPU only).
#include <stdint.h>

#include "../include/omnimem.h"
#include "../paper_2605_30519_amd/csrc/seq.h"

using namespace omnimem;

// {split (0: line), query heads of an item, pairs of waves, workgroups, the shares' offset, their bytes, the starts'
// offset, the workspace's bytes} of a decode call.
extern "C" omnimem_status_t shim_decode_form(const omnimem_seq_cache_quant_t* sc, int32_t dtype, int32_t heads,
                                             int32_t window, int64_t* out) {
  SeqGeom g;
  DecodePlan p;
  DecodeLaunch a;
  void* const fake = reinterpret_cast<void*>(0x10000);
  const size_t need = decode_quant_workspace_bytes(sc, heads, window);
  const omnimem_status_t s = check_decode_attn_quant(sc, dtype, fake, static_cast<int64_t>(heads) * sc->head_dim, heads,
                                                     window, 0.1f, fake, nullptr, fake, need, g, p, a);
  if (s != OMNIMEM_OK) return s;
  const int64_t all[] = {static_cast<int64_t>(p.split), p.tile_rows, p.pair, p.wgs, static_cast<int64_t>(p.off_part),
                         static_cast<int64_t>(2 * p.slot_floats * sizeof(float)) * p.wgs,
                         static_cast<int64_t>(p.off_starts), static_cast<int64_t>(need)};
  for (int i = 0; i < 8; ++i) out[i] = all[i];
  return s;
}
