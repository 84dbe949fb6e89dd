// Attention of trees of many (token, head) rows, over bf16 rows and over e4m3 rows with a scale per head.
#include "ea_attend_tile.h"

namespace ea {

hipError_t launch_attend_tile_tree(const AttendArgs& a, const Dims& d, hipStream_t st) {
  if (d.kv_fp8) return d.D == 128 ? tile_of_type<128, kRowsFp8, false, true>(a, st) : tile_of_type<256, kRowsFp8, false, true>(a, st);
#define EA_CASE(DD) if (d.D == DD) return a.pm.table ? tile_of_type<DD, kRowsBf16, true, true>(a, st) : tile_of_type<DD, kRowsBf16, false, true>(a, st)
  EA_CASE(64);
  EA_CASE(128);
#undef EA_CASE
  return a.pm.table ? tile_of_type<256, kRowsBf16, true, true>(a, st) : tile_of_type<256, kRowsBf16, false, true>(a, st);
}

}  // namespace ea
