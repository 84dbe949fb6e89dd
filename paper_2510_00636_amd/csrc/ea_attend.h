// Attention of new tokens over a cache: what its kernels share.
#pragma once
#include <hip/hip_runtime.h>

#include "ea_kernels.h"
#include "ea_lanes.h"

namespace ea {

using bf16x8 = __bf16 __attribute__((ext_vector_type(8)));
using u32x4 = uint32_t __attribute__((ext_vector_type(4)));
using f32x4 = float __attribute__((ext_vector_type(4)));
using f32x16 = float __attribute__((ext_vector_type(16)));

// One call.  Sequence b's tokens are cu[b] .. cu[b + 1] - 1; its rows lens[per_head ? b * Hkv + h : b].
struct AttendArgs {
  const void* q;
  const void *k, *v;
  const int32_t *cu, *lens;
  const float *kscale, *vscale;   // [B, Hkv] or null (8-bit rows only)
  void* out;
  float* lse;                     // or null
  char* ws;
  PageMap pm;                     // table == nullptr: contiguous, n_cap rows per head
  long long q_stride, n_cap;
  int B, Hq, Hkv, G, D;
  int n, n_tokens, per_head;
  int only_long;                  // the tile kernel leaves sequences of up to short_rows (token, head) rows to the row kernel
  int short_rows;
  float scale;                    // log2(e) / sqrt(d): weights are powers of two
  AttendPlan plan;
};

// the tokens of a sequence, clamped so that no list of prefix sums leads outside q and out
__device__ __forceinline__ int first_token(const AttendArgs& a, int b) {
  const int t = a.cu[b];
  return t < 0 ? 0 : t > a.n_tokens ? a.n_tokens : t;
}
__device__ __forceinline__ int rows_of(const AttendArgs& a, int b, int h) {
  const int t = a.lens[a.per_head ? b * a.Hkv + h : b];
  return t < 0 ? 0 : t > a.n ? a.n : t;
}

// exp2f of an argument that is -inf where a row is masked
__device__ __forceinline__ float pow2(float x) { return exp2f(x); }

__device__ __forceinline__ uint32_t pack_bf16(float lo, float hi) {
  typedef __bf16 pair __attribute__((ext_vector_type(2)));
  const pair p = {(__bf16)lo, (__bf16)hi};
  return __builtin_bit_cast(uint32_t, p);
}

// eight e4m3 bytes -> eight bf16 numbers (exact: three bits behind the point, exponents -9 .. 8)
__device__ __forceinline__ uint4 widen_fp8(uint2 w) {
  auto lo = [](uint32_t x) { return __builtin_bit_cast(uint32_t, __builtin_amdgcn_cvt_scalef32_pk_bf16_fp8((int)x, 1.0f, false)); };
  auto hi = [](uint32_t x) { return __builtin_bit_cast(uint32_t, __builtin_amdgcn_cvt_scalef32_pk_bf16_fp8((int)x, 1.0f, true)); };
  return make_uint4(lo(w.x), hi(w.x), lo(w.y), hi(w.y));
}

// Where row `row` (a multiple of 16, so that its 16 rows lie in one block) of unit (b, h) starts, in rows of the cache tensor.
// entry: the block's table entry (paged).
__device__ __forceinline__ long long row_base(const AttendArgs& a, int b, int h, int row, int entry) {
  if (!a.pm.table) return ((long long)b * a.Hkv + h) * a.n_cap + row;
  long long blk = entry;
  blk = blk < 0 ? 0 : blk >= a.pm.num_blocks ? a.pm.num_blocks - 1 : blk;
  return ((blk * a.Hkv + h) << a.pm.sh) + (row & ((1 << a.pm.sh) - 1));
}
__device__ __forceinline__ int table_entry(const AttendArgs& a, int b, int row) {
  return a.pm.table ? a.pm.table[(size_t)b * a.pm.max_blocks + (row >> a.pm.sh)] : 0;
}

template <int CTRL, int ROWS>
__device__ __forceinline__ int dpp_add_int(int x) {
  return x + __builtin_amdgcn_update_dpp(0, x, CTRL, ROWS, 0xf, true);
}
// sums of x over the lanes up to and with this one
__device__ __forceinline__ int wave_prefix(int x) {
  x = dpp_add_int<0x111, 0xf>(x);
  x = dpp_add_int<0x112, 0xf>(x);
  x = dpp_add_int<0x114, 0xf>(x);
  x = dpp_add_int<0x118, 0xf>(x);
  x = dpp_add_int<0x142, 0xa>(x);   // the last lane of rows 0 and 2 to rows 1 and 3
  return dpp_add_int<0x143, 0xc>(x);
}
__device__ __forceinline__ int last_lane(int x) { return __builtin_amdgcn_readlane(x, 63); }

__device__ __forceinline__ float max_xor32(float x) {
  const auto r = __builtin_amdgcn_permlane32_swap(__float_as_uint(x), __float_as_uint(x), false, false);
  return fmaxf(__uint_as_float(r[0]), __uint_as_float(r[1]));
}
__device__ __forceinline__ float max_xor16(float x) {
  const auto r = __builtin_amdgcn_permlane16_swap(__float_as_uint(x), __float_as_uint(x), false, false);
  return fmaxf(__uint_as_float(r[0]), __uint_as_float(r[1]));
}

// base-2 logarithm of a row's sum and maximum -> natural log-sum-exp; -inf for a row that saw nothing
__device__ __forceinline__ float natural_lse(float m, float l) {
  return l > 0.0f ? fmaf(m, 0.6931471805599453f, logf(l)) : -__builtin_inff();
}

hipError_t launch_attend(const AttendArgs& a, const Dims& d, hipStream_t st);
hipError_t launch_attend_rows(const AttendArgs& a, const Dims& d, hipStream_t st);
hipError_t launch_attend_tile(const AttendArgs& a, const Dims& d, hipStream_t st);
hipError_t launch_attend_f32(const AttendArgs& a, hipStream_t st);
hipError_t launch_attend_join(const AttendArgs& a, bool f32, hipStream_t st);

}  // namespace ea
