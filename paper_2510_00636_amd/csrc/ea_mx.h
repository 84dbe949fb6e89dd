// Rows of MX pools (8- or 4-bit elements, one power of two for 32 channels): what the kernels that write, read and attend to them share.
#pragma once
#include <hip/hip_runtime.h>

#include "ea_common.h"

namespace ea {

// The byte that a group's power of two is stored as, 2^(e - 127), as the float that the converting instructions take: they look at its
// exponent bits only, and make NaN of every element where those are all ones (byte 255).
__device__ __forceinline__ float mx_scale(uint32_t e) { return __uint_as_float(e << 23); }

__device__ __forceinline__ uint32_t mx8_pair(uint32_t w, float scale, bool high) {
  return high ? __builtin_bit_cast(uint32_t, __builtin_amdgcn_cvt_scalef32_pk_bf16_fp8((int)w, scale, true))
              : __builtin_bit_cast(uint32_t, __builtin_amdgcn_cvt_scalef32_pk_bf16_fp8((int)w, scale, false));
}
// eight elements of one group -> eight bf16 numbers, exactly: of 8 bits in two words, of 4 bits in one
__device__ __forceinline__ uint4 widen_mx8(uint2 w, float scale) {
  return make_uint4(mx8_pair(w.x, scale, false), mx8_pair(w.x, scale, true), mx8_pair(w.y, scale, false), mx8_pair(w.y, scale, true));
}
template <int BYTE>
__device__ __forceinline__ uint32_t mx4_pair(uint32_t w, float scale) {
  return __builtin_bit_cast(uint32_t, __builtin_amdgcn_cvt_scalef32_pk_bf16_fp4(w, scale, BYTE));
}
__device__ __forceinline__ uint4 widen_mx4(uint32_t w, float scale) {
  return make_uint4(mx4_pair<0>(w, scale), mx4_pair<1>(w, scale), mx4_pair<2>(w, scale), mx4_pair<3>(w, scale));
}

struct MxAppendArgs {
  const void *q, *k, *v;
  void *q_out, *k_pool, *v_pool;
  uint8_t *k_scale, *v_scale;
  const int32_t* pos;
  const double* inv_freq;
  const int64_t* slots;
  long long q_stride, k_stride, v_stride, num_blocks;
  int Hq, Hkv, n_tokens, sh, rope_layout, bits;
  int first;                            // token of the launch
};
hipError_t launch_append_mx(const MxAppendArgs& a, const Dims& d, hipStream_t st);

struct MxReadArgs {
  const void *k, *v;
  const uint8_t *k_scale, *v_scale;
  const int32_t* lens;
  void *k_out, *v_out;                  // either may be null
  PageMap pm;
  long long n_cap;
  int B, Hkv, n, bits;
};
hipError_t launch_read_mx(const MxReadArgs& a, const Dims& d, hipStream_t st);

}  // namespace ea
