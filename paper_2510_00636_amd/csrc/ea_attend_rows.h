// Attention of few (token, head) rows per KV head, up to 16, 32 or 64: single tokens, and stretches of a few.
//
// The cache is read once and that bounds it (4 G d operations for 4 d bytes of a pair; 4 sequences of 131k rows 349 us, 6.15 TB/s of
// the 6.16 that a large read has on this card), so the whole chip reads all the time:
// the call's heads are laid end to end in groups of 128 rows and every workgroup takes an equal, contiguous share of them,
// from the lengths that stand on the device.  A head that falls into several shares leaves a partial result (maximum, sum,
// weighted values) of each, which a second launch joins in the order of the shares.
// (One launch, with the workgroup that arrives last joining, was slower: it waits for its stores, for a counter across the dies
// and, alone, for all the pieces: 40 query heads over 4097 rows 20.6 us against 9.3 and 4.2.)
//
// S^T = K Q^T and O^T = V^T P^T by v_mfma_f32_16x16x32_bf16, 32 keys at a time and wavefront.  A lane of group g (of four) then
// holds of its query row the keys 4 g + r of either half of the tile, which is a set of eight keys that the second product
// may take as its operand just as it stands: the contraction runs over keys in any order as long as V^T has the same.  V^T
// comes out of registers, too: a lane loads a stretch of channels of its eight keys and pairs them with v_perm.
// So nothing passes through LDS but the four wavefronts' results at the end, and a wavefront's loads are only bound by its
// registers: one tile of K and one of V in flight, 16 KiB at d = 128.
//
// MX rows: a lane's scale bytes come with its rows, and elements are widened (exactly) just where a product takes them: 4 sequences of 131k
// rows of 4 bits 105 us, 5.4 TB/s; 48 of 17 to 4419 rows of 8 bits 20.
//
// What a part of a head needs besides its tiles does not fit the scalar registers: 118 to 155 of them wait in lanes of vector registers,
// where a part begins and ends, without memory.
//
// The kernel by itself; the files that include it say for which rows and sizes it is made.
#pragma once
#include <type_traits>

#include "ea_attend.h"
#include "ea_mx.h"

namespace ea {

namespace {

constexpr int kGroup = kAttendGroup;    // rows of a group: 32 for each wavefront

// Super-unit su (a sequence where heads share a length, else a head): its first token, tokens, cached rows and groups (none if it
// is not this kernel's).
struct Super { int t0, m, len, grp; };
__device__ __forceinline__ Super super_unit(const AttendArgs& a, int su, int supers) {
  Super s = {0, 0, 0, 0};
  if (su >= supers) return s;
  const int b = a.per_head ? su / a.Hkv : su;
  s.len = rows_of(a, b, a.per_head ? su - b * a.Hkv : 0);
  s.t0 = first_token(a, b);
  s.m = first_token(a, b + 1) - s.t0;
  if (s.m >= 1 && s.m * a.G <= a.short_rows) s.grp = s.len < 1 ? 1 : (s.len + kGroup - 1) / kGroup;
  return s;
}
// element i of what no launch writes while it is read, the same for the whole wavefront
template <class T>
__device__ __forceinline__ T scalar(const T* p, long long i) { return ((const __attribute__((address_space(4))) T*)p)[i]; }
__device__ __forceinline__ int from_lane(int x, int l) { return __builtin_amdgcn_readlane(x, l); }

template <int D, Rows R>
struct RowShape {
  static constexpr bool kWide = R == kRowsBf16, kMx = R == kRowsMx8 || R == kRowsMx4;
  static constexpr int kBits = kWide ? 16 : R == kRowsMx4 ? 4 : 8;
  static constexpr int kBytes = D * kBits / 8;           // of a cached row
  static constexpr int kSteps = D / 32;                  // of the first product
  static constexpr int kKCpl = kWide ? 8 : R == kRowsMx4 && D > 64 ? 32 : 16;      // channels per lane and load of K
  static constexpr int kKPer = kKCpl / 8, kKLoads = D / (4 * kKCpl);               // steps that such a load serves; loads
  static constexpr int kCpl = D == 64 ? 4 : !kWide && D == 256 ? 16 : 8;           // channels per lane and load of V
  static constexpr int kLoads = D / (16 * kCpl);
  static constexpr int kTiles = D / 16;                  // output tiles of 16 channels
  static constexpr int kScales = D / 32;                 // MX: scale bytes of a row
};

// BYTES of a row as a lane loads them
template <int BYTES> struct Raw { uint32_t w[BYTES < 4 ? 1 : BYTES / 4]; };
template <int BYTES>
__device__ __forceinline__ Raw<BYTES> load_raw(__amdgpu_buffer_rsrc_t from, int at) {
  Raw<BYTES> r;
  if constexpr (BYTES == 16) {
    const u32x4 x = __builtin_amdgcn_raw_buffer_load_b128(from, at, 0, 0);
    r.w[0] = x.x; r.w[1] = x.y; r.w[2] = x.z; r.w[3] = x.w;
  } else if constexpr (BYTES == 8) {
    const u32x2 x = __builtin_amdgcn_raw_buffer_load_b64(from, at, 0, 0);
    r.w[0] = x.x; r.w[1] = x.y;
  } else if constexpr (BYTES == 4) {
    r.w[0] = __builtin_amdgcn_raw_buffer_load_b32(from, at, 0, 0);
  } else {
    r.w[0] = __builtin_amdgcn_raw_buffer_load_b16(from, at, 0, 0);
  }
  return r;
}

// Scale bytes: those of one row (K), or of the four rows next to each other that a lane has of each half (V)
template <int D> struct RowScales { Raw<D / 32> x; };
// (d = 256: a byte each, since registers are scarce)
template <int D> struct FourScales { Raw<D / 8> x; };
template <> struct FourScales<256> { uint32_t x[4]; };
// byte i of a row's scales, i the lane's own
__device__ __forceinline__ uint32_t byte_of(uint32_t lo, int i) { return __builtin_amdgcn_ubfe(lo, i * 8, 8); }
__device__ __forceinline__ uint32_t byte_of(uint32_t lo, uint32_t hi, int i) { return __builtin_amdgcn_ubfe(i & 4 ? hi : lo, (i & 3) * 8, 8); }

// a loaded piece of V as bf16, all its channels
template <int D, Rows R, int BYTES>
__device__ __forceinline__ void widen_piece(const Raw<BYTES>& p, uint32_t* o) {
  if constexpr (R == kRowsBf16) {
#pragma unroll
    for (int i = 0; i < BYTES / 4; ++i) o[i] = p.w[i];
  } else {
#pragma unroll
    for (int i = 0; i < BYTES / 8; ++i) {
      const uint4 t = widen_fp8(make_uint2(p.w[2 * i], p.w[2 * i + 1]));
      o[4 * i] = t.x; o[4 * i + 1] = t.y; o[4 * i + 2] = t.z; o[4 * i + 3] = t.w;
    }
  }
}
// narrow rows with masks, and MX rows: its channels 2 x, 2 x + 1
template <Rows R>
__device__ __forceinline__ uint32_t mx_pair(const uint32_t* w, int x, float scale) {
  if constexpr (R != kRowsMx4) return mx8_pair(w[x >> 1], scale, x & 1);
  switch (x & 3) {
    case 0: return mx4_pair<0>(w[x >> 2], scale);
    case 1: return mx4_pair<1>(w[x >> 2], scale);
    case 2: return mx4_pair<2>(w[x >> 2], scale);
    default: return mx4_pair<3>(w[x >> 2], scale);
  }
}
// A word's elements without those that widen to no finite number under scale byte e (not 255, which makes NaN of all of them): e4m3's
// bytes of all ones, and elements of 2^(255 - e) and more, which are infinities as bf16.  Codes ascend with what they stand for, so
// those begin at one code: e4m3's (262 - e) * 8, from e = 247 on, e2m1's 8 - 2 (e - 252), from 253 on.  `any` is set where there was one.
template <Rows R>
__device__ __forceinline__ uint32_t finite_elements(uint32_t w, uint32_t e, bool& any) {
  if constexpr (R == kRowsMx4) {
    const uint32_t up = e > 252 ? 2 * (e - 252) : 0;        // from the least such code to the sign bit
    const uint32_t past = ((w & 0x77777777u) + up * 0x11111111u) & 0x88888888u;
    any |= past != 0;
    return w & ~((past >> 3) * 0xfu);
  }
  const uint32_t up = R == kRowsMx8 && e > 246 ? 8 * (e - 246) : 1;
  const uint32_t past = ((w & 0x7f7f7f7fu) + up * 0x01010101u) & 0x80808080u;
  any |= past != 0;
  return w & ~((past >> 7) * 0xffu);
}

// eight channels of K for the products' step `sub` of those that the load serves
template <int D, Rows R, int BYTES>
__device__ __forceinline__ bf16x8 key_operand(const Raw<BYTES>& p, float scale, int sub) {
  using S = RowShape<D, R>;
  uint4 t;
  if constexpr (S::kWide) t = make_uint4(p.w[0], p.w[1], p.w[2], p.w[3]);
  else if constexpr (R == kRowsFp8) t = widen_fp8(sub ? make_uint2(p.w[2], p.w[3]) : make_uint2(p.w[0], p.w[1]));
  else if constexpr (R == kRowsMx8) t = widen_mx8(sub ? make_uint2(p.w[2], p.w[3]) : make_uint2(p.w[0], p.w[1]), scale);
  else t = widen_mx4(p.w[sub], scale);
  return __builtin_bit_cast(bf16x8, t);
}

}  // namespace

// A head's (or its part's) results of one wavefront: [wavefront][row][channel], rows four floats apart from a whole number of
// 64 banks; behind them maxima and sums.
template <int D, int MT> constexpr int rows_lds_floats() { return 4 * 16 * MT * (D + 4) + 4 * 16 * MT * 2; }

// workgroups on a CU
template <int D, Rows R, int MT> constexpr int rows_groups() {
  return D * MT > 256 || (D == 256 && R == kRowsBf16) ? 1 : (R == kRowsMx8 || R == kRowsMx4) && MT == 1 && D < 256 ? 3 : 2;
}

// TREE: what a token sees of its sequence's new rows (no more than 64 of them, or the sequence is not this kernel's) is a mask of them, its own or
// the chain's; else a number of rows.
template <int D, Rows R, int MT, bool TREE>
__global__ __launch_bounds__(256, (rows_groups<D, R, MT>())) void k_attend_rows(AttendArgs a) {
  using S = RowShape<D, R>;
  constexpr int kKeys = 32, kSubs = 2, kStride = 4 * kKeys;      // of a tile: keys, 16 rows at a time; from tile to tile of a wavefront
  constexpr bool kHeadScale = R == kRowsFp8;
  // What a head costs besides its groups, in groups: shares are equal in both, or one of four short heads is done when the others have long
  // been.  48 sequences of 17 .. 4419 rows of 8 bits: none 30.8 us, one group 24.6, two 25.0 (16-bit rows, 8 tokens each: 66.5, 54.5, 54.2;
  // d = 256, 8 bits: 46.4, 40.3, 42.1); 8 sequences of 4608 rows 21.8, 22.7, 22.7.
  constexpr int kLead = TREE ? 1 : 0;
  auto units_of = [](int grp) { return grp > 0 ? grp + kLead : 0; };
  constexpr int kM = 16 * MT, kPitch = D + 4;
  extern __shared__ __attribute__((aligned(16))) float lds[];
  float* pass_o = lds;
  float2* pass_ml = (float2*)(lds + 4 * kM * kPitch);
  __shared__ int bad[2];   // a value that is not finite in a row that some of the part's tokens do not see: this part's, the next one's
  const int tid = threadIdx.x, lane = tid & 63, wave = __builtin_amdgcn_readfirstlane(tid >> 6);
  const int n16 = lane & 15, g = lane >> 4;
  const int supers = a.per_head ? a.B * a.Hkv : a.B, mult = a.per_head ? 1 : a.Hkv;

  // ---- the share: total of all groups, then the super-unit in which this workgroup's begins.  A lane holds one of 64 of them.
  Super mine = super_unit(a, lane, supers);
  int pre = wave_prefix(units_of(mine.grp)), total = last_lane(pre), block = 0;
  for (int base = 64; base < supers; base += 64) total += last_lane(wave_prefix(units_of(super_unit(a, base + lane, supers).grp)));
  const long long all = (long long)total * mult, wgs = all < gridDim.x ? all : gridDim.x;
  // for the joining launch, of a head that begins here: the head, this workgroup, and to how many the head falls from here on; by
  // heads, or by workgroups, in which no more than one head goes on behind the end (-1: none does)
  int4* info = (int4*)(a.ws + a.plan.info);
  auto nothing = [&]() {
    if (a.plan.by_share && tid == 0) info[blockIdx.x] = make_int4(-1, 0, 0, 0);
  };
  if (blockIdx.x >= wgs) return nothing();            // (a head's pieces are those of neighbours: no share in between is empty)
  // all w / wgs without a 64-bit division where there is none to do
  const bool small = all < (1ll << 31);
  const long long each = small ? (long long)((uint32_t)all / (uint32_t)wgs) : all / wgs;
  const uint32_t extra = (uint32_t)(all - each * wgs);
  auto share_at = [&](uint32_t w) { return each * w + extra * w / (uint32_t)wgs; };      // extra < wgs <= kAttendShares
  const long long x0 = share_at(blockIdx.x), x1 = share_at(blockIdx.x + 1);

  // ---- a part of a head that falls into the share
  struct Part {
    int su, have;             // super-unit, groups in front of it
    int grp, t0, m, len;      // its groups, first token, tokens, rows
    int b, h, off, take;      // sequence, KV head, first group of the part and how many (none: the share ends in front of them)
    int lead;                 // of what the head costs besides, how much lies in the share
  };
  long long x = x0;
  auto fill = [&](Part& c) {
    const int l = c.su - block;
    c.grp = from_lane(mine.grp, l);
    c.t0 = from_lane(mine.t0, l);
    c.m = from_lane(mine.m, l);
    c.len = from_lane(mine.len, l);
    const int rel = (int)(x - (long long)c.have * mult), hh = a.per_head ? 0 : rel / (c.grp + kLead);
    c.off = rel - hh * (c.grp + kLead) - kLead;
    c.lead = c.off < 0 ? -c.off : 0;
    c.off = c.off < 0 ? 0 : c.off;
    c.take = (int)(x1 - x - c.lead < c.grp - c.off ? x1 - x - c.lead : c.grp - c.off);
    c.b = a.per_head ? c.su / a.Hkv : c.su;
    c.h = a.per_head ? c.su - c.b * a.Hkv : hh;
  };
  Part cur;
  cur.su = -1;
  cur.have = 0;
  for (;;) {
    const uint64_t in = __ballot((long long)(cur.have + pre) * mult > x0);
    if (in) {
      const int l = __builtin_ctzll(in);
      cur.su = block + l;
      cur.have += from_lane(pre, l) - units_of(from_lane(mine.grp, l));
      break;
    }
    cur.have += last_lane(pre);
    block += 64;
    if (block >= supers) return nothing();
    mine = super_unit(a, block + lane, supers);
    pre = wave_prefix(units_of(mine.grp));
  }
  fill(cur);
  if (kLead > 0 && cur.take <= 0) return nothing();

  // ---- What is in flight: always a tile of K and behind it a tile of V, of this part or, at its end, of the next one; the next part's
  // queries in front of them.  Loads are waited for in order, and the compiler counts what may be on its way behind the one that it
  // waits for on the path with the fewest: so no path asks for fewer (a wavefront whose part of a head is over or empty asks for none
  // of a tile's rows, by the same loads), and what else is read on the way comes by scalar loads.  Against waits for all that is on
  // its way: five tokens of 8 sequences over 16k rows 117 -> 107 us, 256 sequences of 100 rows 39.5 -> 32.
  struct Blocks { int e[kSubs]; };      // table entries of a tile's 16 rows
  auto last_sub = [](const Part& c, int at) {           // the 16 rows from `at` on, or the head's last ones
    const int last = c.len > 0 ? (c.len - 1) & ~15 : 0;
    return at < last ? at : last;
  };
  auto look_up = [&](const Part& c, int at) {
    Blocks e = {};
    if (a.pm.table) {
      const int32_t* t = a.pm.table + (long long)c.b * a.pm.max_blocks;
#pragma unroll
      for (int i = 0; i < kSubs; ++i) e.e[i] = scalar(t, last_sub(c, at + 16 * i) >> a.pm.sh);
    }
    return e;
  };
  constexpr int kPiece = S::kCpl * S::kBits / 8, kKPiece = S::kKCpl * S::kBits / 8;        // bytes of a lane's load of V and of K
  Raw<kKPiece> kraw[kSubs][S::kKLoads];
  Raw<kPiece> vraw[4 * kSubs][S::kLoads];
  RowScales<D> kscales[kSubs];
  FourScales<D> vscales[kSubs];
  // Rows come through descriptors of the 16 rows at a time that a tile has: those behind the last one are zeros, and are not asked for.
  // MX: these are made where they are used, of the first row's number and how many there are (four tensors' would take more scalar
  // registers than there are).
  __amdgpu_buffer_rsrc_t k_rows[S::kMx ? 1 : kSubs], v_rows[S::kMx ? 1 : kSubs];
  long long first_row[kSubs];
  int row_count[kSubs];
  auto place = [&](const Part& c, int at, int hi, Blocks e) {      // the tile at row `at`, none of it from row hi on
#pragma unroll
    for (int t = 0; t < kSubs; ++t) {
      const int r = last_sub(c, at + t * 16), n = at + t * 16 < hi ? min(c.len - r, 16) : 0;
      const long long row = row_base(a, c.b, c.h, r, e.e[t]), base = row * S::kBytes;
      if constexpr (S::kMx) {
        first_row[t] = row;
        row_count[t] = n;
      } else {
        k_rows[t] = __builtin_amdgcn_make_buffer_rsrc((void*)((const char*)a.k + base), 0, n * S::kBytes, 0x27000);
        v_rows[t] = __builtin_amdgcn_make_buffer_rsrc((void*)((const char*)a.v + base), 0, n * S::kBytes, 0x27000);
      }
    }
  };
  auto place_none = [&]() {
#pragma unroll
    for (int t = 0; t < kSubs; ++t) {
      if constexpr (S::kMx) {
        first_row[t] = 0;
        row_count[t] = 0;
      } else {
        k_rows[t] = __builtin_amdgcn_make_buffer_rsrc((void*)a.k, 0, 0, 0x27000);
        v_rows[t] = __builtin_amdgcn_make_buffer_rsrc((void*)a.v, 0, 0, 0x27000);
      }
    }
  };
  auto rows_at = [&](const void* base, int t, int row_bytes) {
    return __builtin_amdgcn_make_buffer_rsrc((void*)((const char*)base + first_row[t] * row_bytes), 0, row_count[t] * row_bytes, 0x27000);
  };
  const int k_at = n16 * S::kBytes + g * kKPiece, v_at = 4 * g * S::kBytes + n16 * kPiece;
  auto load_k = [&]() {
#pragma unroll
    for (int t = 0; t < kSubs; ++t) {
      __amdgpu_buffer_rsrc_t from;
      if constexpr (S::kMx) kscales[t].x = load_raw<S::kScales>(rows_at(a.kscale8, t, S::kScales), n16 * S::kScales);
      if constexpr (S::kMx) from = rows_at(a.k, t, S::kBytes);
      else from = k_rows[t];
#pragma unroll
      for (int s = 0; s < S::kKLoads; ++s) kraw[t][s] = load_raw<kKPiece>(from, k_at + s * 4 * kKPiece);
    }
  };
  auto load_v = [&]() {
    if constexpr (S::kMx)
#pragma unroll
      for (int t = 0; t < kSubs; ++t) {
        // (at d = 64 a word has the scales of two rows, and a part of it would be refused: with an odd number of rows one row more)
        const auto from = __builtin_amdgcn_make_buffer_rsrc((void*)(a.vscale8 + first_row[t] * S::kScales), 0, (row_count[t] * S::kScales + 3) & ~3, 0x27000);
#pragma unroll
        for (int i = 0; i < (D == 256 ? 4 : 1); ++i) {
          if constexpr (D == 256) vscales[t].x[i] = __builtin_amdgcn_raw_buffer_load_b8(from, (4 * g + i) * S::kScales + n16 * S::kCpl / 32, 0, 0);
          else vscales[t].x = load_raw<D / 8>(from, 4 * g * S::kScales);
        }
      }
#pragma unroll
    for (int t = 0; t < kSubs; ++t) {
      __amdgpu_buffer_rsrc_t from;
      if constexpr (S::kMx) from = rows_at(a.v, t, S::kBytes);
      else from = v_rows[t];
#pragma unroll
      for (int j = 0; j < 4; ++j)
#pragma unroll
        for (int u = 0; u < S::kLoads; ++u) vraw[4 * t + j][u] = load_raw<kPiece>(from, v_at + j * S::kBytes + u * 16 * kPiece);
    }
  };
  // the lane's scale of K for load s of 16 rows, and its scale byte of V for row j of its own
  auto key_scale = [&](int t, int s) {
    if constexpr (!S::kMx) return 1.0f;
    else {
      const uint32_t *w = kscales[t].x.w, lo = w[0];
      const int i = (s * 4 * S::kKCpl + g * S::kKCpl) / 32;
      if constexpr (D < 256) return mx_scale(byte_of(lo, i));
      else return mx_scale(byte_of(lo, w[1], i));
    }
  };
  auto value_scale = [&](int j) -> uint32_t {
    if constexpr (!S::kMx) {
      return 0;
    } else if constexpr (D == 64) {
      const uint32_t w = vscales[j >> 2].x.w[(j & 3) >> 1];
      return __builtin_amdgcn_ubfe(w, (j & 1) * 16 + n16 * S::kCpl / 32 * 8, 8);
    } else if constexpr (D == 128) {
      return byte_of(vscales[j >> 2].x.w[j & 3], n16 * S::kCpl / 32);
    } else {
      return vscales[j >> 2].x[j & 3];
    }
  };
  const uint32_t g_inverse = (65535u + a.G) / a.G;       // rows / G by a product: exact for rows and G up to 64
  auto over_g = [&](int row) { return (int)((uint32_t)row * g_inverse >> 16); };
  // the step's own rows that token `tok` of a sequence sees
  auto mask_of = [&](int t0, int tok) { return a.sees ? a.sees[(long long)(t0 + tok) * a.words] : (2ull << tok) - 1; };
  // the query operand: row n16 (+ 16) of the head's rows (token, head of the group), channels as the keys' operand has them
  u32x4 q[MT][S::kSteps];
  // with them: what the rows' tokens see (TREE; no more tokens than rows), which waits in LDS until the tiles that ask for it
  using Mask = std::conditional_t<MT == 4, uint64_t, uint32_t>;
  constexpr int kMaskBits = 8 * sizeof(Mask);
  Mask masks[MT];
  __shared__ Mask see[TREE ? 4 : 1][TREE ? kM : 1];
  auto load_q = [&](const Part& c) {
#pragma unroll
    for (int t = 0; t < MT; ++t) {
      const int row = t * 16 + n16, in = row < c.m * a.G ? row : 0, tok = over_g(in), hd = in - tok * a.G;
      const __bf16* src = (const __bf16*)a.q + (long long)(c.t0 + tok) * a.q_stride + (c.h * a.G + hd) * D;
#pragma unroll
      for (int s = 0; s < S::kSteps; ++s)
        q[t][s] = *(const u32x4*)(src + s / S::kKPer * 4 * S::kKCpl + g * S::kKCpl + s % S::kKPer * 8);
      if constexpr (TREE) masks[t] = (Mask)mask_of(c.t0, tok);
    }
  };
  auto begin = [&](const Part& c, Blocks e) {
    const int at = c.off * kGroup + wave * kKeys;
    load_q(c);
    place(c, at, c.len, e);
    load_k();
    load_v();
  };
  begin(cur, look_up(cur, cur.off * kGroup + wave * kKeys));
  if (tid == 0) bad[0] = 0;
  __syncthreads();

  for (int parity = 0;; parity ^= 1) {
    x += cur.lead + cur.take;
    // ---- the part behind this one, and the entries of its blocks
    Part next = cur;
    Blocks first = {}, following_blocks = {};
    if (cur.take * kGroup > kStride) following_blocks = look_up(cur, cur.off * kGroup + kStride + wave * kKeys);
    bool go_on = x < x1;
    if (go_on) {
      if (x >= (long long)(cur.have + units_of(cur.grp)) * mult) {      // the next super-unit that has groups
        next.have += units_of(cur.grp);
        ++next.su;
        for (;;) {
          const uint64_t some = next.su - block < 64 ? __ballot(mine.grp > 0) >> (next.su - block) : 0;
          if (some) {
            next.su += __builtin_ctzll(some);
            break;
          }
          block += 64;
          next.su = block;
          if (block >= supers) break;
          mine = super_unit(a, block + lane, supers);
        }
        go_on = next.su < supers;
      }
      if (go_on) {
        fill(next);
        if (kLead > 0 && next.take <= 0) go_on = false;
        else first = look_up(next, next.off * kGroup + wave * kKeys);
      }
    }
    const int rows = cur.m * a.G, unit = cur.b * a.Hkv + cur.h, len = cur.len;
    const bool whole = cur.take == cur.grp;
    const bool begins = cur.off == 0;
    if (tid == 0 && (begins || !go_on)) {
      int pieces = 1;
      if (begins && !whole) {     // the last one is the last of those that begin at or in front of its last group
        const long long end = x - cur.take + cur.grp;
        int w = (int)blockIdx.x + (int)((cur.grp - cur.take) / (each + 1));
        while (share_at(w + 1) < end) ++w;
        pieces = w - (int)blockIdx.x + 1;
      }
      if (!a.plan.by_share) {
        if (begins) info[unit] = make_int4(unit, (int)blockIdx.x, pieces, 0);
      } else if (!go_on) {
        info[blockIdx.x] = make_int4(pieces > 1 ? unit : -1, (int)blockIdx.x, pieces, 0);
      }
    }
    const float qk = a.scale * (kHeadScale && a.kscale ? scalar(a.kscale, unit) : 1.0f), vs = kHeadScale && a.vscale ? scalar(a.vscale, unit) : 1.0f;
    const int new_rows = len - cur.m;                  // where the step's own begin
    const int some = new_rows + (TREE ? 0 : 1);        // and those that not all of its tokens see
    int vis[MT];            // keys that the row sees
#pragma unroll
    for (int t = 0; t < MT; ++t) {
      const int row = t * 16 + n16, tok = over_g(row);
      vis[t] = row < rows ? len - (cur.m - 1 - tok) : len;
      if constexpr (TREE) see[wave][row] = masks[t] & (Mask)(~(Mask)0 >> (kMaskBits - cur.m));
    }
    bool any_bad = false;
    f32x4 o[MT][S::kTiles];
    float mx[MT], l[MT];
#pragma unroll
    for (int t = 0; t < MT; ++t) {
      mx[t] = -__builtin_inff();
      l[t] = 0.0f;
#pragma unroll
      for (int c = 0; c < S::kTiles; ++c) o[t][c] = (f32x4)0.0f;
    }
    const int row_hi = min((cur.off + cur.take) * kGroup, len);
    int row = cur.off * kGroup + wave * kKeys;
    const bool no_tile = row >= row_hi;
    while (row < row_hi) {
      const int following = row + kStride;
      // ---- S^T: 16 keys x 16 rows each
      f32x4 s[MT][kSubs];
#pragma unroll
      for (int t = 0; t < MT; ++t)
#pragma unroll
        for (int i = 0; i < kSubs; ++i) s[t][i] = (f32x4)0.0f;
#pragma unroll
      for (int c = 0; c < S::kSteps; ++c)
#pragma unroll
        for (int t = 0; t < kSubs; ++t) {
          const bf16x8 w = key_operand<D, R>(kraw[t][c / S::kKPer], key_scale(t, c / S::kKPer), c % S::kKPer);
#pragma unroll
          for (int i = 0; i < MT; ++i)
            s[i][t] = __builtin_amdgcn_mfma_f32_16x16x32_bf16(w, __builtin_bit_cast(bf16x8, q[i][c]), s[i][t], 0, 0, 0);
        }
      const bool over = following >= row_hi && go_on;
      if (over) load_q(next);
      if (over) place(next, next.off * kGroup + wave * kKeys, next.len, first);
      else if (following < row_hi) place(cur, following, row_hi, following_blocks);
      else place_none();
      load_k();
      if (following + kStride < row_hi) following_blocks = look_up(cur, following + kStride);
      __builtin_amdgcn_sched_barrier(0);
      // ---- weights (see kLag).
      // A weight reaches the second product as two bf16 numbers, which together are as good as fp32 next to the values' eight
      // bits: the matrix cores have time for it here.
      const bool ragged = row + kKeys > some;
      uint32_t p[MT][4], plo[MT][4];
#pragma unroll
      for (int t = 0; t < MT; ++t) {
#pragma unroll
        for (int i = 0; i < kSubs; ++i) s[t][i] *= qk;
        if constexpr (TREE) {
          if (ragged) {
            // bit i: key row + i is seen (row + kKeys > new_rows)
            const Mask mask = see[wave][t * 16 + n16];
            const int from = row - new_rows;
            const uint32_t bits = from >= kMaskBits ? 0 : from >= 0 ? (uint32_t)(mask >> (from & (kMaskBits - 1)))
                                                                    : (uint32_t)mask << (-from & 31) | ((1u << (-from & 31)) - 1);
#pragma unroll
            for (int i = 0; i < kSubs; ++i) {
              const uint32_t mine = bits >> 16 * i >> 4 * g;
#pragma unroll
              for (int r = 0; r < 4; ++r) s[t][i][r] = mine >> r & 1 ? s[t][i][r] : -__builtin_inff();
            }
          }
        } else if (ragged) {
#pragma unroll
          for (int i = 0; i < 4 * kSubs; ++i)
            if (row + (i >> 2) * 16 + 4 * g + (i & 3) >= vis[t]) s[t][i >> 2][i & 3] = -__builtin_inff();
        }
        float top = fmaxf(fmaxf(s[t][0][0], s[t][0][1]), fmaxf(s[t][0][2], s[t][0][3]));
#pragma unroll
        for (int i = 1; i < kSubs; ++i) top = fmaxf(top, fmaxf(fmaxf(s[t][i][0], s[t][i][1]), fmaxf(s[t][i][2], s[t][i][3])));
        if (__any(top > mx[t] + kLag)) {
          top = reference(fmaxf(max_xor16(max_xor32(top)), mx[t]));
          const float f = mx[t] == -__builtin_inff() ? 0.0f : pow2(mx[t] - top);
          mx[t] = top;
          l[t] *= f;
#pragma unroll
          for (int c = 0; c < S::kTiles; ++c) o[t][c] *= f;
        }
        const float from = subtrahend(mx[t]);
#pragma unroll
        for (int i = 0; i < 4; ++i) {
          const float lo = pow2(s[t][i >> 1][(i & 1) * 2] - from), hi = pow2(s[t][i >> 1][(i & 1) * 2 + 1] - from);
          l[t] += lo + hi;
          p[t][i] = pack_bf16(lo, hi);
          plo[t][i] = pack_bf16(lo - __uint_as_float(p[t][i] << 16), hi - __uint_as_float(p[t][i] & 0xffff0000u));
        }
      }
      // ---- O^T
#pragma unroll
      for (int u = 0; u < S::kLoads; ++u) {
        // Narrow rows with masks: a pair of channels is widened where it is needed (all of them at once take 64 registers at d = 256), so what
        // is not finite goes in front of that
        constexpr bool kPairs = S::kMx || (TREE && R == kRowsFp8);
        uint32_t w[8][kPairs ? 1 : S::kCpl / 2];
        float scale[8];
        if constexpr (kPairs) {
          uint32_t e[8];
#pragma unroll
          for (int j = 0; j < 8; ++j) e[j] = value_scale(j);
          if (ragged) {
#pragma unroll
            for (int j = 0; j < 8; ++j) {
              const int key = row + (j >> 2) * 16 + 4 * g + (j & 3);
              const bool none = S::kMx && key >= some && e[j] == 255;
              any_bad |= none && key < len;
              e[j] = none ? 0 : e[j];
#pragma unroll
              for (int i = 0; i < (int)(sizeof(Raw<kPiece>) / 4); ++i) {
                bool bad_element = false;
                const uint32_t x = vraw[j][u].w[i], y = finite_elements<R>(x, e[j], bad_element);
                any_bad |= bad_element && key >= some;
                vraw[j][u].w[i] = none ? 0 : key >= some ? y : x;
              }
            }
          }
#pragma unroll
          for (int j = 0; j < 8; ++j) scale[j] = S::kMx ? mx_scale(e[j]) : 1.0f;
        } else {
#pragma unroll
          for (int j = 0; j < 8; ++j) {
            widen_piece<D, R>(vraw[j][u], w[j]);
            if ((TREE || cur.m > 1) && ragged && row + (j >> 2) * 16 + 4 * g + (j & 3) >= some)
#pragma unroll
              for (int c = 0; c < S::kCpl / 2; ++c) w[j][c] = finite_pair(w[j][c], any_bad);
          }
        }
#pragma unroll
        for (int c = 0; c < S::kCpl; ++c) {
          const uint32_t sel = c & 1 ? 0x07060302u : 0x05040100u;
          const int at = kPairs ? 0 : c >> 1;
          if constexpr (kPairs)
            if (c % 2 == 0)
#pragma unroll
              for (int j = 0; j < 8; ++j) w[j][0] = mx_pair<R>(vraw[j][u].w, c >> 1, scale[j]);
          const uint4 v = make_uint4(__builtin_amdgcn_perm(w[1][at], w[0][at], sel), __builtin_amdgcn_perm(w[3][at], w[2][at], sel),
                                     __builtin_amdgcn_perm(w[5][at], w[4][at], sel), __builtin_amdgcn_perm(w[7][at], w[6][at], sel));
#pragma unroll
          for (int t = 0; t < MT; ++t) {
            f32x4& acc = o[t][u * S::kCpl + c];
            const uint32_t *hi = p[t], *lo = plo[t];
            acc = __builtin_amdgcn_mfma_f32_16x16x32_bf16(__builtin_bit_cast(bf16x8, v), __builtin_bit_cast(bf16x8, make_uint4(lo[0], lo[1], lo[2], lo[3])), acc, 0, 0, 0);
            acc = __builtin_amdgcn_mfma_f32_16x16x32_bf16(__builtin_bit_cast(bf16x8, v), __builtin_bit_cast(bf16x8, make_uint4(hi[0], hi[1], hi[2], hi[3])), acc, 0, 0, 0);
          }
        }
      }
      load_v();
      __builtin_amdgcn_sched_barrier(0);
      row = following;
    }
    // the next part's first tile is on its way while this one's results are put together
    if (go_on && no_tile) begin(next, first);
    __builtin_amdgcn_sched_barrier(0);

    // ---- the four wavefronts' results through LDS, once; then every thread makes four channels of a row of them
#pragma unroll
    for (int t = 0; t < MT; ++t) {
      l[t] = sum_xor16(sum_halves(l[t]));
      const int r = t * 16 + n16;
      if (r < rows) {
        if (g == 0) pass_ml[wave * kM + r] = make_float2(mx[t], l[t]);
        float* dst = pass_o + (wave * kM + r) * kPitch;
        // channel u 16 cpl + (4 g + r) cpl + c is o[u cpl + c][r]
#pragma unroll
        for (int u = 0; u < S::kLoads; ++u)
#pragma unroll
          for (int i = 0; i < 4; ++i)
#pragma unroll
            for (int c = 0; c < S::kCpl; c += 4) {
              const f32x4* w = &o[t][u * S::kCpl + c];
              *(float4*)(dst + u * 16 * S::kCpl + (4 * g + i) * S::kCpl + c) = make_float4(w[0][i], w[1][i], w[2][i], w[3][i]);
            }
      }
    }
    if (any_bad) bad[parity] = 1;
    __syncthreads();
    if (tid == 0) bad[parity ^ 1] = 0;      // nobody looks at it until the next barrier
    // slot 0 of a workgroup: a head that began in front of it; slot 1: one that goes on behind it
    const long long slot = ((long long)blockIdx.x * 2 + (cur.off == 0 ? 1 : 0)) * kM;
    float* part_o = (float*)(a.ws + a.plan.part_o) + slot * D;
    float2* part_ml = (float2*)(a.ws + a.plan.part_ml) + slot;
    constexpr int kLanes = D / 4;
    const int c4 = tid % kLanes * 4;
    for (int r = tid / kLanes; r < rows; r += 256 / kLanes) {
      float2 ml[4];
#pragma unroll
      for (int w = 0; w < 4; ++w) ml[w] = pass_ml[w * kM + r];
      const float top = fmaxf(fmaxf(ml[0].x, ml[1].x), fmaxf(ml[2].x, ml[3].x)), from = top == -__builtin_inff() ? 0.0f : top;
      float4 acc = make_float4(0, 0, 0, 0);
      float sum = 0.0f;
#pragma unroll
      for (int w = 0; w < 4; ++w) {
        const float f = pow2(ml[w].x - from);
        const float4 y = *(const float4*)(pass_o + (w * kM + r) * kPitch + c4);
        sum += ml[w].y * f;
        acc.x += y.x * f; acc.y += y.y * f; acc.z += y.z * f; acc.w += y.w * f;
      }
      if (bad[parity]) {
        float y[4] = {acc.x, acc.y, acc.z, acc.w};
        const int seen = TREE ? len : len - (cur.m - 1 - over_g(r));
        const int lo = max(max(some, cur.off * kGroup), 0), hi = min(seen, row_hi);
        if constexpr (TREE) {
          const uint64_t mask = mask_of(cur.t0, over_g(r));
          add_not_finite<D, kind_of(R)>(a, cur.b, cur.h, lo, hi, c4, y, [&](int key) { return key - new_rows < 64 && (mask >> (key - new_rows) & 1); });
        } else {
          add_not_finite<D, kind_of(R)>(a, cur.b, cur.h, lo, hi, c4, y);
        }
        acc = make_float4(y[0], y[1], y[2], y[3]);
      }
      if (whole) {
        write_row<D>(a, cur.t0, cur.h, over_g(r), r - over_g(r) * a.G, c4, vs, top, sum, acc);
      } else {
        *(float4*)(part_o + (long long)r * D + c4) = acc;
        if (c4 == 0) part_ml[r] = make_float2(top, sum);
      }
    }
    if (!go_on) return;
    __syncthreads();      // the next part's results go through the same LDS
    cur = next;
  }
}

template <int D, Rows R, int MT, bool TREE>
static hipError_t rows_of_height(const AttendArgs& a, hipStream_t st) {
  static LdsOptIn opt;
  const size_t bytes = rows_lds_floats<D, MT>() * sizeof(float);
  const hipError_t e = opt.ensure((const void*)k_attend_rows<D, R, MT, TREE>, bytes);
  if (e != hipSuccess) return e;
  k_attend_rows<D, R, MT, TREE><<<a.plan.shares, 256, bytes, st>>>(a);
  const hipError_t e2 = hipGetLastError();
  return e2 != hipSuccess ? e2 : launch_attend_rows_join(a, st);
}
template <int D, Rows R, bool TREE>
static hipError_t rows_of_type(const AttendArgs& a, hipStream_t st) {
  if constexpr (D < 256)
    if (a.plan.mt == 4) return rows_of_height<D, R, 4, TREE>(a, st);
  if (a.plan.mt == 2) return rows_of_height<D, R, 2, TREE>(a, st);
  return rows_of_height<D, R, 1, TREE>(a, st);
}

}  // namespace ea
