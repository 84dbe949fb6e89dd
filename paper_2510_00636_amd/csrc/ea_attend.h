// Attention of new tokens over a cache: what its kernels share.
#pragma once
#include <hip/hip_runtime.h>

#include "ea_kernels.h"
#include "ea_lanes.h"
#include "ea_mx.h"

namespace ea {

using bf16x8 = __bf16 __attribute__((ext_vector_type(8)));
using u32x4 = uint32_t __attribute__((ext_vector_type(4)));
using u32x2 = uint32_t __attribute__((ext_vector_type(2)));
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
  const uint8_t *kscale8, *vscale8;       // MX pools: a byte for 32 channels of a row
  int mx;                         // bits of an element of such pools, 0: others
  const uint64_t* sees;           // trees: which of its sequence's new rows a token sees, `words` words each; null: those up to its own
  int words;
  int by_head;                    // stretches are cut along the keys head by head (trees over caches with a length per head)
  AttendPlan plan;
};

// what cached rows are: bf16 numbers, e4m3 bytes with a scale per head, MX rows
enum Rows { kRowsBf16, kRowsFp8, kRowsMx8, kRowsMx4 };
enum { kKindF32 = -1 };                 // and fp32 ones, for add_not_finite()
constexpr int kind_of(Rows r) { return (int)r; }

// the tokens of a sequence, clamped so that no list of prefix sums leads outside q and out
__device__ __forceinline__ int clamped(int t, int most) { return t < 0 ? 0 : t > most ? most : t; }
__device__ __forceinline__ int first_token(const AttendArgs& a, int b) { return clamped(a.cu[b], a.n_tokens); }
__device__ __forceinline__ int rows_of(const AttendArgs& a, int b, int h) { return clamped(a.lens[a.per_head ? b * a.Hkv + h : b], a.n); }

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

// Where row `row` of unit (b, h) starts, in rows of the cache tensor (the 16 rows from a multiple of 16 on lie in one block).
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

// largest x of the wavefront, of either sign, in every lane
__device__ __forceinline__ float wave_max_any(float x) {
#pragma unroll
  for (int d = 1; d < 64; d *= 2) x = fmaxf(x, __shfl_xor(x, d));
  return x;
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

// ---- Stretches: which piece a workgroup takes.
// A sequence's (token, head) rows come in tiles of ROWS; tiles of few, long sequences are cut along the keys as well, so that the
// pieces fill the chip's slots evenly.  How finely follows from the lengths on the device: every lane looks at one way to cut the
// longest (and with it the others, into pieces of at most as many keys), and the one that is done first is taken.  All workgroups
// come to the same result, and the first of a sequence writes down for the joining launch how it was cut.  In steps of 64 keys:
// a piece costs kPieceSteps besides its own (its queries, its first tile, its results), a cut one kCutSteps more of a slot
// (its partial result written and read again, 5 TB/s for all), cutting at all kJoinSteps (the launch that joins).
constexpr int kPieceSteps = 3, kCutSteps = 6, kJoinSteps = 4, kLeastSteps = 4, kLongSteps = 64;
struct Piece {
  int b, h, tile, split;        // tile < 0: none
  int tiles, nsplit, chunk;     // of the sequence, and keys of a stretch
  int t0, m;
  bool first;
};
__device__ __forceinline__ int ceil_div(int x, int by) {      // x < 2^24, both sides exact in fp32
  int k = (int)((float)(x + by - 1) * __builtin_amdgcn_rcpf((float)by));
  if (k * by > x + by - 1) --k;
  if ((k + 1) * by <= x + by - 1) ++k;
  return k;
}
// WAVES > 1: that many wavefronts, the workgroup's, share out the sequences between them, their sums through LDS (24 sequences: 4.2 us of a piece's time -> 2.8).
// PER_HEAD: heads have lengths of their own (a.per_head).  HEADS: with a.by_head what is cut is such a head, not a sequence.
template <int ROWS, bool PER_HEAD, int WAVES = 1, bool HEADS = false>
__device__ __forceinline__ Piece find_piece(const AttendArgs& a, int index, float (*sums)[3][64] = nullptr) {
  const int lane = threadIdx.x & 63;
  const bool by_head = PER_HEAD && HEADS && a.by_head;
  const int supers = by_head ? a.B * a.Hkv : a.B, heads = by_head ? 1 : a.Hkv;      // that are cut each for itself, and heads of one
  auto look = [&](int b, int& tiles, int& steps) {
    const int su = min(b, supers - 1), at = by_head ? su / a.Hkv : su;
    const bool one = !PER_HEAD || by_head;      // length to look at
    int len = one ? rows_of(a, at, by_head ? su - at * a.Hkv : 0) : 0;
    const int rows = b < supers ? (first_token(a, at + 1) - first_token(a, at)) * a.G : 0;
    const bool none = rows < 1 || (a.only_long && rows <= a.short_rows);
    if (!one && !none) {
      // A line of memory for each head and lane: only of sequences that are this kernel's, and four at a time (16 of 100 sequences of 8
      // heads add 40 tokens, the others one, at d = 128: of all sequences, one by one, 133 us, so 111).
      int h = 0;
      for (; h + 4 <= a.Hkv; h += 4) len = max(len, max(max(rows_of(a, at, h), rows_of(a, at, h + 1)), max(rows_of(a, at, h + 2), rows_of(a, at, h + 3))));
      for (; h < a.Hkv; ++h) len = max(len, rows_of(a, at, h));
    }
    tiles = none ? 0 : (rows + ROWS - 1) / ROWS;
    steps = none ? 0 : len > 0 ? (len + 63) >> 6 : 1;
  };
  int tiles, steps;
  look(lane, tiles, steps);
  const int tiles0 = tiles, steps0 = steps;
  int q = 1 << 24;              // most steps of a piece
  if (a.plan.most_pieces > 0) {
    int most = (int)wave_max((float)steps);
    for (int base = 64; base < supers; base += 64) {
      look(base + lane, tiles, steps);
      most = max(most, (int)wave_max((float)steps));
    }
    q = max(ceil_div(most, lane + 1), min(kLeastSteps, most));
    float pieces = 0.0f, cut = 0.0f, work = 0.0f;
    for (int base = 0; base < supers; base += 64) {
      if (base > 0) look(base + lane, tiles, steps); else tiles = tiles0, steps = steps0;
      uint64_t left = __ballot(tiles > 0);
      if constexpr (WAVES > 1) left &= (~0ull / ((1ull << WAVES) - 1)) << (threadIdx.x >> 6);      // every WAVES-th
      for (; left; left &= left - 1) {
        const int l = __builtin_ctzll(left), n = __builtin_amdgcn_readlane(tiles, l) * heads, each = __builtin_amdgcn_readlane(steps, l);
        const int k = ceil_div(each, q);
        pieces += (float)(n * k);
        cut += k > 1 ? (float)(n * k) : 0.0f;
        work += (float)n * (float)each;
      }
    }
    if constexpr (WAVES > 1) {
      const int wave = threadIdx.x >> 6;
      sums[wave][0][lane] = pieces;
      sums[wave][1][lane] = cut;
      sums[wave][2][lane] = work;
      __syncthreads();
      pieces = cut = work = 0.0f;
#pragma unroll
      for (int w = 0; w < WAVES; ++w) {
        pieces += sums[w][0][lane];
        cut += sums[w][1][lane];
        work += sums[w][2][lane];
      }
      __syncthreads();      // what else stands there may be written again
    }
    // one round: its longest piece.  More: the work shared out, with a quarter of a piece at the end, but whole rounds where all
    // pieces are alike
    const float longest = (float)(q + kPieceSteps), per_slot = a.plan.per_slot;
    float cost = longest;
    if (pieces * per_slot > 1.0f) {
      cost = (work + pieces * kPieceSteps) * per_slot + 0.25f * longest;
      if (work > 0.9f * pieces * (float)q) cost = fmaxf(cost, ceilf(pieces * per_slot) * longest);
    }
    if (cut > 0.0f) cost = pieces > (float)a.plan.most_pieces ? 3e38f : cost + kJoinSteps + cut * per_slot * kCutSteps;
    const float least = -wave_max_any(-cost);
    q = __builtin_amdgcn_readlane(q, __builtin_ctzll(__ballot(cost == least)));
  }
  Piece p;
  p.tile = -1;
  int have = 0;
  // sequences of long pieces first, so that short ones fill up the end
  const int blocks = (supers + 63) >> 6;
  for (int turn = 0; turn < 2 * blocks; ++turn) {
    const int base = (turn >= blocks ? turn - blocks : turn) * 64;
    if (blocks > 1) look(base + lane, tiles, steps); else tiles = tiles0, steps = steps0;
    const int cuts = ceil_div(steps, q);
    if ((2 * ceil_div(steps, max(cuts, 1)) >= min(q, kLongSteps)) != (turn < blocks)) tiles = 0;
    const int mine = tiles * cuts * heads, pre = wave_prefix(mine);
    const uint64_t in = __ballot(have + pre > index);
    if (in) {
      const int l = __builtin_ctzll(in);
      p.b = by_head ? (base + l) / a.Hkv : base + l;
      p.tiles = __builtin_amdgcn_readlane(tiles, l);
      p.nsplit = __builtin_amdgcn_readlane(cuts, l);
      p.chunk = ceil_div(__builtin_amdgcn_readlane(steps, l), p.nsplit) * 64;
      const int at = index - have - (__builtin_amdgcn_readlane(pre, l) - __builtin_amdgcn_readlane(mine, l));
      // heads next to each other (they run on different dies), the last tiles, which see most keys, first
      p.h = by_head ? base + l - p.b * a.Hkv : at % a.Hkv;
      const int rest = at / heads;
      p.split = rest % p.nsplit;
      p.tile = p.tiles - 1 - rest / p.nsplit;
      p.first = at == 0;
      p.t0 = __builtin_amdgcn_readfirstlane(first_token(a, p.b));
      p.m = __builtin_amdgcn_readfirstlane(first_token(a, p.b + 1)) - p.t0;
      return p;
    }
    have += last_lane(pre);
  }
  return p;
}
// where the rows of a piece's partial result stand, and what the joining launch needs to find them
template <bool HEADS = false>
__device__ __forceinline__ void note_cuts(const AttendArgs& a, const Piece& p, int index) {
  if (a.plan.most_pieces > 0 && p.first && threadIdx.x == 0) ((int4*)(a.ws + a.plan.cuts))[HEADS && a.by_head ? p.b * a.Hkv + p.h : p.b] = make_int4(index, p.nsplit, p.chunk, p.tiles);
}

// ---- Values that a row does not see.  Behind the last cached row they are taken for zeros; but a step's own rows are seen by some of
// its tokens and not by others, and a weight of zero times an infinity or a NaN there is a NaN.  So where such rows stand, values
// that are not finite are taken for zeros too, and the kernel remembers that there was one: then, at the end, every row is given
// those that it does see (their weights are positive, so what comes of them is the value itself).
__device__ __forceinline__ bool not_finite(float x) { return (__float_as_uint(x) & 0x7f800000u) == 0x7f800000u; }
// the bf16 pair w without its numbers that are not finite; `any` is set where there was one
__device__ __forceinline__ uint32_t finite_pair(uint32_t w, bool& any) {
  const bool lo = (w & 0x7f80u) == 0x7f80u, hi = (w & 0x7f800000u) == 0x7f800000u;
  any |= lo || hi;
  return (lo ? 0u : w & 0xffffu) | (hi ? 0u : w & 0xffff0000u);
}
// adds to x the four values at `channel` of those rows lo .. hi - 1 for which seen(row) that are not finite; kind one of Rows, or fp32
struct SeenAll { __device__ __forceinline__ bool operator()(int) const { return true; } };
template <int D, int KIND, class SEEN = SeenAll>
__device__ __forceinline__ void add_not_finite(const AttendArgs& a, int b, int h, int lo, int hi, int channel, float* x, SEEN seen = {}) {
  for (int key = lo; key < hi; ++key) {
    if (!seen(key)) continue;
    const long long row = row_base(a, b, h, key, table_entry(a, b, key)), at = row * D + channel;
    float v[4];
    if constexpr (KIND == kKindF32) {
      const float4 w = *(const float4*)((const float*)a.v + at);
      v[0] = w.x; v[1] = w.y; v[2] = w.z; v[3] = w.w;
    } else {
      uint2 w;
      if constexpr (KIND == kRowsBf16) {
        w = *(const uint2*)((const __bf16*)a.v + at);
      } else if constexpr (KIND == kRowsFp8) {
        const uint4 t = widen_fp8(make_uint2(*(const uint32_t*)((const char*)a.v + at), 0u));
        w = make_uint2(t.x, t.y);
      } else {
        const float scale = mx_scale(a.vscale8[row * (D / 32) + channel / 32]);
        const uint4 t = KIND == kRowsMx8 ? widen_mx8(make_uint2(*(const uint32_t*)((const char*)a.v + at), 0u), scale)
                                         : widen_mx4(*(const uint16_t*)((const char*)a.v + at / 2), scale);
        w = make_uint2(t.x, t.y);
      }
      v[0] = __uint_as_float(w.x << 16); v[1] = __uint_as_float(w.x & 0xffff0000u);
      v[2] = __uint_as_float(w.y << 16); v[3] = __uint_as_float(w.y & 0xffff0000u);
    }
#pragma unroll
    for (int i = 0; i < 4; ++i)
      if (not_finite(v[i])) x[i] += v[i];
  }
}

// ---- Weights.  The maximum that a row's are taken against moves only when a logit passes it by more than kLag powers of two, which
// saves most of the products that a move costs.  So that no weight passes one all the same (a value times 2^8 can pass the end of
// fp32 where the value itself, and the result, do not) a weight is 2^-kLag of the power of two: the sums of weights and of weighted
// values have the factor alike, and only the logarithm of the sum has to take it out again.
constexpr float kLag = 8.0f;
// the largest logit of a row as the reference that its weights are taken against: one that stays the same number plus and minus kLag
__device__ __forceinline__ float reference(float top) { return (top + kLag) - kLag; }
// what is subtracted from a row's logits: its reference and kLag; -inf (nothing seen so far) is taken for zero
__device__ __forceinline__ float subtrahend(float m) { return m == -__builtin_inff() ? 0.0f : m + kLag; }

// base-2 logarithm of a row's sum and maximum -> natural log-sum-exp; -inf for a row that saw nothing (and for no other: a sum
// that is not a number has no logarithm either).  The sum is 2^-kLag of what it stands for.
__device__ __forceinline__ float natural_lse(float m, float l) {
  return l == 0.0f ? -__builtin_inff() : fmaf(m, 0.6931471805599453f, logf(l * 256.0f));
}

// four channels of a finished row, whose values have the scale vs
template <int D>
__device__ __forceinline__ void write_row(const AttendArgs& a, int t0, int h, int tok, int hd, int c4, float vs, float top, float sum, float4 acc) {
  const long long at = (long long)(t0 + tok) * a.Hq + h * a.G + hd;
  const bool any = sum > 0.0f || sum != sum;
  const float f = vs / sum;
  *(uint2*)((__bf16*)a.out + at * D + c4) =
      any ? make_uint2(pack_bf16(acc.x * f, acc.y * f), pack_bf16(acc.z * f, acc.w * f)) : make_uint2(0u, 0u);
  if (a.lse && c4 == 0) a.lse[at] = natural_lse(top, sum);
}

hipError_t launch_attend(const AttendArgs& a, const Dims& d, hipStream_t st);
hipError_t launch_attend_rows_tree(const AttendArgs& a, const Dims& d, hipStream_t st);
hipError_t launch_attend_rows_mx8(const AttendArgs& a, const Dims& d, hipStream_t st);
hipError_t launch_attend_rows_mx4(const AttendArgs& a, const Dims& d, hipStream_t st);
hipError_t launch_attend_tile_tree(const AttendArgs& a, const Dims& d, hipStream_t st);
hipError_t launch_attend_tile_mx8(const AttendArgs& a, const Dims& d, hipStream_t st);
hipError_t launch_attend_tile_mx4(const AttendArgs& a, const Dims& d, hipStream_t st);
hipError_t launch_attend_rows_join(const AttendArgs& a, hipStream_t st);
hipError_t launch_attend_rows(const AttendArgs& a, const Dims& d, hipStream_t st);
hipError_t launch_attend_tile(const AttendArgs& a, const Dims& d, hipStream_t st);
hipError_t launch_attend_f32(const AttendArgs& a, hipStream_t st);
hipError_t launch_attend_f32_tree(const AttendArgs& a, hipStream_t st);
hipError_t launch_attend_join(const AttendArgs& a, bool f32, hipStream_t st);

}  // namespace ea
