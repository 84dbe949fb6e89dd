// Drafted trees: masks and positions from parents, the branch that the model confirms, and its rows moved together.  Latency bounds
// all three: a few words per token, and the rows of one branch.  One tree of 16 tokens 2.5, 2.2 and 4.2 us, 48 of 61 tokens 4.4, 4.8
// and 4.7 (launched one after the other the host takes longer: 14 to 16 us for the three).
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

// A wavefront per sequence, up to four tokens to a lane: a step down the tree is a vote over what the lanes hold, without memory.
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

// A workgroup per KV head.  What says which rows move is asked for together (lengths, counts, the path), then the table's entries, then
// as many rows as the threads have room for, 16 bytes (or what a shorter row has) to a piece: three round trips to memory for a
// branch (row after row, each waiting for the one in front: 48 trees 13.1 us, so 4.7).  Numbers ascend, so a round that is written leaves
// the rows of the next ones alone.
__global__ __launch_bounds__(256) void k_keep_path(KeepArgs a) {
  using u32x4 = uint32_t __attribute__((ext_vector_type(4)));
  using u32x2 = uint32_t __attribute__((ext_vector_type(2)));
  constexpr int kThreads = 256, kPer = 4;
  __shared__ long long src[kTreeMost], dst[kTreeMost];
  const int unit = blockIdx.x, b = unit / a.Hkv, h = unit - b * a.Hkv, tid = threadIdx.x, lane = tid & 63;
  const int32_t* path = a.path + (long long)b * a.max_new;
  const int t0 = token_bound(a.cu, b, a.n_tokens), m = max(token_bound(a.cu, b + 1, a.n_tokens) - t0, 0);
  const int given = a.lens[a.per_head ? unit : b], len = max(given, 0), count = a.n_path[b];
  const int x0 = lane < a.max_new ? path[lane] : -1;
  const bool served = m > 0 && !(a.slots && a.slots[t0] < 0);
  int n = served ? max(min(min(count, a.max_new), min(m, kTreeMost)), 0) : 0;
  // the path ends in front of its first number that makes no sense
  int before = -1;
  for (int base = 0; base < n; base += 64) {
    const int j = base + lane, x = base == 0 ? x0 : j < n ? path[j] : -1;
    const int left = lane == 0 ? before : __shfl_up(x, 1);
    before = __shfl(x, 63);
    const uint64_t wrong = __ballot(j < n && (x >= m || x < 0 || x <= left));
    if (wrong) n = base + __builtin_ctzll(wrong);
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
  // rows that stay where they are, or that are not there, are passed over
  const long long first = (long long)len - m;
  for (int j = tid; j < n; j += kThreads) {
    const int x = j == lane ? x0 : path[j];
    const long long s = x == j ? -1 : row_at(first + x), t = s < 0 ? -1 : row_at(first + j);
    src[j] = t < 0 ? -1 : s;
    dst[j] = t;
  }
  __syncthreads();
  // A thread's pieces of the rows of a round: read, and written behind the barrier.
  int pieces = 0;
#pragma unroll
  for (int i = 0; i < 4; ++i)
    if (i < a.count) pieces += a.row_bytes[i] < 16 ? 1 : a.row_bytes[i] / 16;
  const int per_round = kPer * kThreads / pieces;          // rows (a row has up to 128 pieces)
  for (int j0 = 0; j0 < n; j0 += per_round) {
    const int rows = min(per_round, n - j0);
    u32x4 x[kPer];
    char* to[kPer];
    int bytes[kPer];
#pragma unroll
    for (int k = 0; k < kPer; ++k) {
      const int at = k * kThreads + tid, j = at / pieces;
      bytes[k] = 0;
      if (j >= rows || src[j0 + j] < 0) continue;
      int piece = at - j * pieces, row_bytes = 0;
      char* base = nullptr;
#pragma unroll
      for (int i = 3; i >= 0; --i) {                        // the tensors from the last on, pieces in that order
        if (i >= a.count || row_bytes) continue;
        const int mine = a.row_bytes[i] < 16 ? 1 : a.row_bytes[i] / 16;
        if (piece < mine) base = a.at[i], row_bytes = a.row_bytes[i];
        else piece -= mine;
      }
      const char* from = base + src[j0 + j] * row_bytes + piece * 16;
      to[k] = base + dst[j0 + j] * row_bytes + piece * 16;
      bytes[k] = row_bytes < 16 ? row_bytes : 16;
      if (bytes[k] == 16) x[k] = *(const u32x4*)from;
      else if (bytes[k] == 8) x[k] = u32x4{((const uint32_t*)from)[0], ((const uint32_t*)from)[1], 0, 0};
      else x[k] = u32x4{bytes[k] == 4 ? *(const uint32_t*)from : *(const uint16_t*)from, 0, 0, 0};
    }
    __syncthreads();
#pragma unroll
    for (int k = 0; k < kPer; ++k) {
      if (bytes[k] == 16) *(u32x4*)to[k] = x[k];
      else if (bytes[k] == 8) *(u32x2*)to[k] = u32x2{x[k].x, x[k].y};
      else if (bytes[k] == 4) *(uint32_t*)to[k] = x[k].x;
      else if (bytes[k] == 2) *(uint16_t*)to[k] = (uint16_t)x[k].x;
    }
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
  k_keep_path<<<(unsigned)(a.B * a.Hkv), 256, 0, st>>>(a);
  return hipGetLastError();
}

}  // namespace ea
