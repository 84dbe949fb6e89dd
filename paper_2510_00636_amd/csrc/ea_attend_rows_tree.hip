// Attention of few rows that form trees, over bf16 rows and over e4m3 rows with a scale per head.
#include "ea_attend_rows.h"

namespace ea {

hipError_t launch_attend_rows_tree(const AttendArgs& a, const Dims& d, hipStream_t st) {
  if (d.kv_fp8) return d.D == 128 ? rows_of_type<128, kRowsFp8, true>(a, st) : rows_of_type<256, kRowsFp8, true>(a, st);
  return d.D == 64 ? rows_of_type<64, kRowsBf16, true>(a, st)
                   : d.D == 128 ? rows_of_type<128, kRowsBf16, true>(a, st) : rows_of_type<256, kRowsBf16, true>(a, st);
}

}  // namespace ea
