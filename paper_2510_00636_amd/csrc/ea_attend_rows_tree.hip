// Attention of few rows that form trees, over bf16 rows.
#include "ea_attend_rows.h"

namespace ea {

hipError_t launch_attend_rows_tree(const AttendArgs& a, const Dims& d, hipStream_t st) {
  return d.D == 64 ? rows_of_type<64, kRowsBf16, true>(a, st)
                   : d.D == 128 ? rows_of_type<128, kRowsBf16, true>(a, st) : rows_of_type<256, kRowsBf16, true>(a, st);
}

}  // namespace ea
