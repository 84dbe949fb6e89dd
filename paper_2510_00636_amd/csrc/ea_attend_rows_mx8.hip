// Attention of few rows, chains and trees, over MX pools of 8-bit elements.
#include "ea_attend_rows.h"

namespace ea {

hipError_t launch_attend_rows_mx8(const AttendArgs& a, const Dims& d, hipStream_t st) {
  return d.D == 64 ? rows_of_type<64, kRowsMx8, true>(a, st)
                   : d.D == 128 ? rows_of_type<128, kRowsMx8, true>(a, st) : rows_of_type<256, kRowsMx8, true>(a, st);
}

}  // namespace ea
