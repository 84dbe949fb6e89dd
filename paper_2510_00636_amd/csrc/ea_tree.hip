// Drafted trees: masks and positions from parents, the branch that the model confirms, and its rows moved together.  Latency bounds
// all three: a few words per token, and the rows of one branch.
#include "ea_kernels.h"
#include "ea_tree.h"

namespace ea {

namespace {

constexpr int kTreeMost = EA_TREE_MAX;

__device__ __forceinline__ int token_bound(const int32_t* cu, int b, int most) {
  const int t = cu[b];
  return t < 0 ? 0 : t < most ? t : most;
}

}  // namespace

// A workgroup per sequence, a thread per token.  The set of those above a token doubles its reach with every round: what it sees, and
// what the highest token that it has reached sees; a round for every bit of the tree's depth.
__global__ __launch_bounds__(kTreeMost) void k_tree_masks(TreeArgs a) {
  __shared__ uint64_t set[2][kTreeMost / 64][kTreeMost];
  __shared__ int top[2][kTreeMost];             // the parent of the highest token reached, -1: it has none
  const int b = blockIdx.x, i = threadIdx.x, t0 = token_bound(a.cu, b, a.n_tokens);
  const int m = min(token_bound(a.cu, b + 1, a.n_tokens) - t0, 64 * a.words);
  if (m < 1) return;
  int up = -1;
  uint64_t mine[kTreeMost / 64] = {};
  if (i < m) {
    up = a.parents[t0 + i];
    if (up < 0 || up >= i) up = -1;
#pragma unroll
    for (int w = 0; w < kTreeMost / 64; ++w) mine[w] = i >> 6 == w ? 1ull << (i & 63) : 0;
  }
  for (int turn = 0;; turn ^= 1) {
    top[turn][i] = up;
#pragma unroll
    for (int w = 0; w < kTreeMost / 64; ++w) set[turn][w][i] = mine[w];
    if (!__syncthreads_or(up >= 0)) break;
    if (up >= 0) {
#pragma unroll
      for (int w = 0; w < kTreeMost / 64; ++w) mine[w] |= set[turn][w][up];
      up = top[turn][up];
    }
  }
  if (i >= m) return;
  int above = -1;
#pragma unroll
  for (int w = 0; w < kTreeMost / 64; ++w) {
    above += __popcll(mine[w]);
    if (w < a.words) a.sees[(long long)(t0 + i) * a.words + w] = mine[w];
  }
  if (a.pos) a.pos[t0 + i] = (a.seen ? a.seen[b] : 0) + above;
}

// A wavefront per sequence, up to four tokens to a lane.
__global__ __launch_bounds__(64) void k_tree_accept(TreeArgs a) {
  constexpr int kPer = kTreeMost / 64;
  const int b = blockIdx.x, lane = threadIdx.x, t0 = token_bound(a.cu, b, a.n_tokens);
  const int all = token_bound(a.cu, b + 1, a.n_tokens) - t0, m = min(min(all, a.max_new), kTreeMost);
  if (m < 1) {
    if (lane == 0) a.n_path[b] = 0, a.next[b] = -1;
    return;
  }
  int parent[kPer], token[kPer], target[kPer];
#pragma unroll
  for (int k = 0; k < kPer; ++k) {
    const int i = k * 64 + lane, at = t0 + min(i, m - 1);
    parent[k] = i < m && a.parents[at] < i ? a.parents[at] : -1;
    token[k] = a.tokens[at];
    target[k] = a.target[at];
  }
  auto answer = [&](int i) {            // behind token i
    int x = 0;
#pragma unroll
    for (int k = 0; k < kPer; ++k)
      if (i >> 6 == k) x = __builtin_amdgcn_readlane(target[k], i & 63);
    return x;
  };
  int at = 0, count = 1, want = answer(0);
  if (lane == 0) a.path[(long long)b * a.max_new] = 0;
  for (;;) {
    int found = -1;
#pragma unroll
    for (int k = kPer - 1; k >= 0; --k) {
      const uint64_t in = __ballot(parent[k] == at && token[k] == want);
      if (in) found = k * 64 + __builtin_ctzll(in);
    }
    if (found < 0) break;
    at = found;
    if (lane == 0) a.path[(long long)b * a.max_new + count] = at;
    ++count;
    want = answer(at);
  }
  if (lane == 0) a.n_path[b] = count, a.next[b] = want;
}

// A workgroup per KV head.  A thread has 16 bytes (or what a shorter row has) of every row that moves, and takes them in order: numbers
// ascend, so that no row is written before it is read.
__global__ __launch_bounds__(128) void k_keep_path(KeepArgs a) {
  __shared__ long long src[kTreeMost], dst[kTreeMost];
  const int unit = blockIdx.x, b = unit / a.Hkv, h = unit - b * a.Hkv, tid = threadIdx.x, lane = tid & 63;
  const int t0 = token_bound(a.cu, b, a.n_tokens), m = max(token_bound(a.cu, b + 1, a.n_tokens) - t0, 0);
  const int given = a.lens[a.per_head ? unit : b], len = max(given, 0);
  const bool served = m > 0 && !(a.slots && a.slots[t0] < 0);
  int n = served ? min(min(a.n_path[b], a.max_new), min(m, kTreeMost)) : 0;
  n = max(n, 0);
  const int32_t* path = a.path + (long long)b * a.max_new;
  // the path ends in front of its first number that makes no sense
  for (int base = 0; base < n; base += 64) {
    const int j = base + lane;
    bool wrong = false;
    if (j < n) {
      const int x = path[j];
      wrong = x >= m || x < 0 || (j > 0 && path[j - 1] >= x);
    }
    const uint64_t some = __ballot(wrong);
    if (some) n = base + __builtin_ctzll(some);
  }
  if (tid == 0 && (a.per_head || h == 0)) a.len_out[a.per_head ? unit : b] = served ? max(len - m + n, 0) : given;
  auto row_at = [&](long long r) -> long long {      // -1: there is none
    if (r < 0) return -1;
    if (!a.pm.table) return r < a.n_cap ? (long long)unit * a.n_cap + r : -1;
    const long long j = r >> a.pm.sh;
    if (j >= a.pm.max_blocks) return -1;
    long long blk = a.pm.table[(long long)b * a.pm.max_blocks + j];
    blk = blk < 0 ? 0 : blk < a.pm.num_blocks ? blk : a.pm.num_blocks - 1;
    return ((blk * a.Hkv + h) << a.pm.sh) + (r & ((1 << a.pm.sh) - 1));
  };
  for (int j = tid; j < n; j += 128) {
    const long long first = (long long)len - m;
    src[j] = row_at(first + path[j]);
    dst[j] = row_at(first + j);
  }
  __syncthreads();
  // rows in front that stay where they are, or that are not there, are passed over
  int from = 0;
  while (from < n && (src[from] == dst[from] || src[from] < 0 || dst[from] < 0)) ++from;
  if (from == n) return;
  int item = tid;
  for (int i = 0; i < a.count; ++i) {
    const int bytes = a.row_bytes[i], each = bytes < 16 ? bytes : 16, pieces = bytes / each;
    for (; item < pieces; item += 128) {
      char* base = a.at[i] + item * each;
      for (int j = from; j < n; ++j) {
        if (src[j] < 0 || dst[j] < 0) continue;
        const char* s = base + src[j] * bytes;
        char* t = base + dst[j] * bytes;
        if (each == 16) *(uint4*)t = *(const uint4*)s;
        else if (each == 8) *(uint2*)t = *(const uint2*)s;
        else if (each == 4) *(uint32_t*)t = *(const uint32_t*)s;
        else *(uint16_t*)t = *(const uint16_t*)s;
      }
    }
    item -= pieces;
  }
}

hipError_t launch_tree_masks(const TreeArgs& a, hipStream_t st) {
  k_tree_masks<<<(unsigned)a.B, kTreeMost, 0, st>>>(a);
  return hipGetLastError();
}
hipError_t launch_tree_accept(const TreeArgs& a, hipStream_t st) {
  k_tree_accept<<<(unsigned)a.B, 64, 0, st>>>(a);
  return hipGetLastError();
}
hipError_t launch_keep_path(const KeepArgs& a, hipStream_t st) {
  k_keep_path<<<(unsigned)(a.B * a.Hkv), 128, 0, st>>>(a);
  return hipGetLastError();
}

}  // namespace ea
