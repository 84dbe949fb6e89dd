// Arguments of the kernels in ea_step.hip.
#pragma once
#include <hip/hip_runtime.h>

#include "ea_common.h"

namespace ea {

struct BlockTableArgs {
  int32_t* table;
  const int32_t *len_old, *len_new, *free_in, *seen;
  int32_t *free_list, *len_out, *free_out, *cu_tokens, *pos;
  int64_t* slots;
  long long n_tokens, num_blocks;
  int B, sh, max_blocks;
};
hipError_t launch_block_tables(const BlockTableArgs& a, hipStream_t st);

struct AppendArgs {
  const void *q, *k, *v;
  void *q_out, *k_cache, *v_cache;
  const int32_t *pos, *cu, *lens;
  const double* inv_freq;
  const int64_t* slots;                 // or null: rows by cu and lens [B, Hkv], n_cap per head
  const float *k_scale, *v_scale;
  long long q_stride, k_stride, v_stride, n_cap, num_blocks;
  int B, Hq, Hkv, n_tokens, sh, rope_layout;
  int first;                            // token of the launch
};
hipError_t launch_append(const AppendArgs& a, const Dims& d, hipStream_t st);

}  // namespace ea
