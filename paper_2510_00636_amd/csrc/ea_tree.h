// Arguments of the kernels in ea_tree.hip: what a step does with its drafted trees besides attention.
#pragma once
#include <hip/hip_runtime.h>

#include "ea_common.h"

namespace ea {

struct TreeArgs {
  const int32_t *cu, *parents, *seen, *tokens, *target;
  uint64_t* sees;
  int32_t *pos, *path, *n_path, *next;
  int B, n_tokens, words, max_new;
};
hipError_t launch_tree_masks(const TreeArgs& a, hipStream_t st);
hipError_t launch_tree_accept(const TreeArgs& a, hipStream_t st);

// What moves with a row: `count` tensors of row_bytes[i] bytes a row, rows of a head next to each other (paged: within a block).
struct KeepArgs {
  char* at[4];
  int row_bytes[4];
  int count;
  const int32_t *cu, *path, *n_path, *lens;
  int32_t* len_out;
  const int64_t* slots;                 // or null
  PageMap pm;                           // table == nullptr: contiguous, n_cap rows per head
  long long n_cap;
  int B, Hkv, n_tokens, max_new, per_head;
};
hipError_t launch_keep_path(const KeepArgs& a, hipStream_t st);

}  // namespace ea
