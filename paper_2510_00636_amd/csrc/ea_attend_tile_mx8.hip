// Attention of stretches and of trees of many (token, head) rows, over MX pools of 8-bit elements.
#include "ea_attend_tile.h"

namespace ea {

hipError_t launch_attend_tile_mx8(const AttendArgs& a, const Dims& d, hipStream_t st) {
  return d.D == 64 ? tile_of_type<64, kRowsMx8, true, true>(a, st)
                   : d.D == 128 ? tile_of_type<128, kRowsMx8, true, true>(a, st) : tile_of_type<256, kRowsMx8, true, true>(a, st);
}

}  // namespace ea
