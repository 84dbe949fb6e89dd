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
#include "ea_attend.h"

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

template <int D, bool FP8>
struct RowShape {
  static constexpr int kBytes = D * (FP8 ? 1 : 2);       // of a cached row
  static constexpr int kSteps = D / 32;                  // of the first product
  static constexpr int kCpl = D == 64 ? 4 : FP8 && D == 256 ? 16 : 8;    // channels per lane and load of V
  static constexpr int kLoads = D / (16 * kCpl);
  static constexpr int kTiles = D / 16;                  // output tiles of 16 channels
};

// a row of V as it is loaded: kCpl channels
template <int D, bool FP8> struct VPiece { u32x4 w; };
template <> struct VPiece<64, false> { u32x2 w; };
template <> struct VPiece<128, true> { u32x2 w; };

// channels 2 x, 2 x + 1 of a loaded piece as bf16
template <int D, bool FP8>
__device__ __forceinline__ void widen_piece(const VPiece<D, FP8>& p, uint32_t* o) {
  if constexpr (!FP8 && D == 64) {
    o[0] = p.w.x; o[1] = p.w.y;
  } else if constexpr (!FP8) {
    o[0] = p.w.x; o[1] = p.w.y; o[2] = p.w.z; o[3] = p.w.w;
  } else if constexpr (D == 128) {
    const uint4 t = widen_fp8(make_uint2(p.w.x, p.w.y));
    o[0] = t.x; o[1] = t.y; o[2] = t.z; o[3] = t.w;
  } else {
    const uint4 t = widen_fp8(make_uint2(p.w.x, p.w.y)), u = widen_fp8(make_uint2(p.w.z, p.w.w));
    o[0] = t.x; o[1] = t.y; o[2] = t.z; o[3] = t.w;
    o[4] = u.x; o[5] = u.y; o[6] = u.z; o[7] = u.w;
  }
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

}  // namespace

// A head's (or its part's) results of one wavefront: [wavefront][row][channel], rows four floats apart from a whole number of
// 64 banks; behind them maxima and sums.
template <int D, int MT> constexpr int rows_lds_floats() { return 4 * 16 * MT * (D + 4) + 4 * 16 * MT * 2; }

template <int D, bool FP8, int MT>
__global__ __launch_bounds__(256, (D * MT > 256 || (D == 256 && !FP8) ? 1 : 2)) void k_attend_rows(AttendArgs a) {
  using S = RowShape<D, FP8>;
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
  int pre = wave_prefix(mine.grp), total = last_lane(pre), block = 0;
  for (int base = 64; base < supers; base += 64) total += last_lane(wave_prefix(super_unit(a, base + lane, supers).grp));
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
    int b, h, off, take;      // sequence, KV head, first group of the part and how many
  };
  long long x = x0;
  auto fill = [&](Part& c) {
    const int l = c.su - block;
    c.grp = from_lane(mine.grp, l);
    c.t0 = from_lane(mine.t0, l);
    c.m = from_lane(mine.m, l);
    c.len = from_lane(mine.len, l);
    const int rel = (int)(x - (long long)c.have * mult), hh = a.per_head ? 0 : rel / c.grp;
    c.off = rel - hh * c.grp;
    c.take = (int)(x1 - x < c.grp - c.off ? x1 - x : c.grp - c.off);
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
      cur.have += from_lane(pre, l) - from_lane(mine.grp, l);
      break;
    }
    cur.have += last_lane(pre);
    block += 64;
    if (block >= supers) return nothing();
    mine = super_unit(a, block + lane, supers);
    pre = wave_prefix(mine.grp);
  }
  fill(cur);

  // ---- What is in flight: always a tile of K and behind it a tile of V, of this part or, at its end, of the next one; the next part's
  // queries in front of them.  Loads are waited for in order, and the compiler counts what may be on its way behind the one that it
  // waits for on the path with the fewest: so no path asks for fewer (a wavefront whose part of a head is over or empty asks for none
  // of a tile's rows, by the same loads), and what else is read on the way comes by scalar loads.  Against waits for all that is on
  // its way: five tokens of 8 sequences over 16k rows 117 -> 107 us, 256 sequences of 100 rows 39.5 -> 32.
  struct Blocks { int e0, e1; };      // table entries of a tile's halves
  auto last_sub = [](const Part& c, int at) {           // the 16 rows from `at` on, or the head's last ones
    const int last = c.len > 0 ? (c.len - 1) & ~15 : 0;
    return at < last ? at : last;
  };
  auto look_up = [&](const Part& c, int at) {
    Blocks e = {0, 0};
    if (a.pm.table) {
      const int32_t* t = a.pm.table + (long long)c.b * a.pm.max_blocks;
      e.e0 = scalar(t, last_sub(c, at) >> a.pm.sh);
      e.e1 = scalar(t, last_sub(c, at + 16) >> a.pm.sh);
    }
    return e;
  };
  u32x4 kraw[2][FP8 ? S::kSteps / 2 : S::kSteps];
  VPiece<D, FP8> vraw[8][S::kLoads];
  // Rows come through descriptors of the 16 rows that a tile's half has: those behind the last one are zeros, and are not asked for.
  __amdgpu_buffer_rsrc_t k_rows[2], v_rows[2];
  auto place = [&](const Part& c, int at, int hi, Blocks e) {      // the tile at row `at`, none of it from row hi on
#pragma unroll
    for (int t = 0; t < 2; ++t) {
      const int r = last_sub(c, at + t * 16), n = at + t * 16 < hi ? min(c.len - r, 16) : 0;
      const long long base = row_base(a, c.b, c.h, r, t ? e.e1 : e.e0) * S::kBytes;
      k_rows[t] = __builtin_amdgcn_make_buffer_rsrc((void*)((const char*)a.k + base), 0, n * S::kBytes, 0x27000);
      v_rows[t] = __builtin_amdgcn_make_buffer_rsrc((void*)((const char*)a.v + base), 0, n * S::kBytes, 0x27000);
    }
  };
  auto place_none = [&]() {
#pragma unroll
    for (int t = 0; t < 2; ++t) {
      k_rows[t] = __builtin_amdgcn_make_buffer_rsrc((void*)a.k, 0, 0, 0x27000);
      v_rows[t] = __builtin_amdgcn_make_buffer_rsrc((void*)a.v, 0, 0, 0x27000);
    }
  };
  constexpr int kPiece = S::kCpl * (FP8 ? 1 : 2);        // bytes of a lane's load of V
  const int k_at = n16 * S::kBytes + g * 16, v_at = 4 * g * S::kBytes + n16 * kPiece;
  auto load_k = [&]() {
#pragma unroll
    for (int t = 0; t < 2; ++t)
#pragma unroll
      for (int s = 0; s < (FP8 ? S::kSteps / 2 : S::kSteps); ++s)
        kraw[t][s] = __builtin_amdgcn_raw_buffer_load_b128(k_rows[t], k_at + s * 64, 0, 0);
  };
  auto load_v = [&]() {
#pragma unroll
    for (int j = 0; j < 8; ++j)
#pragma unroll
      for (int u = 0; u < S::kLoads; ++u) {
        const int at = v_at + (j & 3) * S::kBytes + u * 16 * kPiece;
        if constexpr (kPiece == 16) vraw[j][u].w = __builtin_amdgcn_raw_buffer_load_b128(v_rows[j >> 2], at, 0, 0);
        else vraw[j][u].w = __builtin_amdgcn_raw_buffer_load_b64(v_rows[j >> 2], at, 0, 0);
      }
  };
  const uint32_t g_inverse = (65535u + a.G) / a.G;       // rows / G by a product: exact for rows and G up to 64
  auto over_g = [&](int row) { return (int)((uint32_t)row * g_inverse >> 16); };
  // the query operand: row n16 (+ 16) of the head's rows (token, head of the group), channels as the keys' operand has them
  u32x4 q[MT][S::kSteps];
  auto load_q = [&](const Part& c) {
#pragma unroll
    for (int t = 0; t < MT; ++t) {
      const int row = t * 16 + n16, in = row < c.m * a.G ? row : 0, tok = over_g(in), hd = in - tok * a.G;
      const __bf16* src = (const __bf16*)a.q + (long long)(c.t0 + tok) * a.q_stride + (c.h * a.G + hd) * D;
#pragma unroll
      for (int s = 0; s < S::kSteps; ++s)
        q[t][s] = *(const u32x4*)(src + (FP8 ? (s >> 1) * 64 + g * 16 + (s & 1) * 8 : s * 32 + g * 8));
    }
  };
  auto begin = [&](const Part& c, Blocks e) {
    const int at = c.off * kGroup + wave * 32;
    load_q(c);
    place(c, at, c.len, e);
    load_k();
    load_v();
  };
  begin(cur, look_up(cur, cur.off * kGroup + wave * 32));
  if (tid == 0) bad[0] = 0;
  __syncthreads();

  for (int parity = 0;; parity ^= 1) {
    x += cur.take;
    // ---- the part behind this one, and the entries of its blocks
    Part next = cur;
    Blocks first = {0, 0}, following_blocks = {0, 0};
    if (cur.take > 1) following_blocks = look_up(cur, (cur.off + 1) * kGroup + wave * 32);
    bool go_on = x < x1;
    if (go_on) {
      if (x >= (long long)(cur.have + cur.grp) * mult) {      // the next super-unit that has groups
        next.have += cur.grp;
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
        first = look_up(next, next.off * kGroup + wave * 32);
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
    const float qk = a.scale * (FP8 && a.kscale ? scalar(a.kscale, unit) : 1.0f), vs = FP8 && a.vscale ? scalar(a.vscale, unit) : 1.0f;
    int vis[MT];            // keys that the row sees
#pragma unroll
    for (int t = 0; t < MT; ++t) {
      const int row = t * 16 + n16, tok = over_g(row);
      vis[t] = row < rows ? len - (cur.m - 1 - tok) : len;
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
    int row = cur.off * kGroup + wave * 32;
    const bool no_tile = row >= row_hi;
    while (row < row_hi) {
      const int following = row + kGroup;
      // ---- S^T: 32 keys x 16 rows
      f32x4 s[MT][2];
#pragma unroll
      for (int t = 0; t < MT; ++t) s[t][0] = s[t][1] = (f32x4)0.0f;
#pragma unroll
      for (int c = 0; c < S::kSteps; ++c)
#pragma unroll
        for (int t = 0; t < 2; ++t) {
          bf16x8 w;
          if constexpr (FP8) {
            const u32x4 p = kraw[t][c >> 1];
            w = __builtin_bit_cast(bf16x8, c & 1 ? widen_fp8(make_uint2(p[2], p[3])) : widen_fp8(make_uint2(p[0], p[1])));
          } else {
            w = __builtin_bit_cast(bf16x8, kraw[t][c]);
          }
#pragma unroll
          for (int i = 0; i < MT; ++i)
            s[i][t] = __builtin_amdgcn_mfma_f32_16x16x32_bf16(w, __builtin_bit_cast(bf16x8, q[i][c]), s[i][t], 0, 0, 0);
        }
      const bool over = following >= row_hi && go_on;
      if (over) load_q(next);
      if (over) place(next, next.off * kGroup + wave * 32, next.len, first);
      else if (following < row_hi) place(cur, following, row_hi, following_blocks);
      else place_none();
      load_k();
      if (following + kGroup < row_hi) following_blocks = look_up(cur, following + kGroup);
      __builtin_amdgcn_sched_barrier(0);
      // ---- weights (see kLag).
      // A weight reaches the second product as two bf16 numbers, which together are as good as fp32 next to the values' eight
      // bits: the matrix cores have time for it here.
      const bool ragged = row + 32 > len - (cur.m - 1);
      uint32_t p[MT][4], plo[MT][4];
#pragma unroll
      for (int t = 0; t < MT; ++t) {
        s[t][0] *= qk;
        s[t][1] *= qk;
        if (ragged)
#pragma unroll
          for (int i = 0; i < 8; ++i)
            if (row + (i >> 2) * 16 + 4 * g + (i & 3) >= vis[t]) s[t][i >> 2][i & 3] = -__builtin_inff();
        float top = fmaxf(fmaxf(fmaxf(s[t][0][0], s[t][0][1]), fmaxf(s[t][0][2], s[t][0][3])),
                          fmaxf(fmaxf(s[t][1][0], s[t][1][1]), fmaxf(s[t][1][2], s[t][1][3])));
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
        uint32_t w[8][S::kCpl / 2];
#pragma unroll
        for (int j = 0; j < 8; ++j) {
          widen_piece<D, FP8>(vraw[j][u], w[j]);
          if (cur.m > 1 && ragged && row + (j >> 2) * 16 + 4 * g + (j & 3) >= len - (cur.m - 1))
#pragma unroll
            for (int c = 0; c < S::kCpl / 2; ++c) w[j][c] = finite_pair(w[j][c], any_bad);
        }
#pragma unroll
        for (int c = 0; c < S::kCpl; ++c) {
          const uint32_t sel = c & 1 ? 0x07060302u : 0x05040100u;
          const uint4 v = make_uint4(__builtin_amdgcn_perm(w[1][c >> 1], w[0][c >> 1], sel), __builtin_amdgcn_perm(w[3][c >> 1], w[2][c >> 1], sel),
                                     __builtin_amdgcn_perm(w[5][c >> 1], w[4][c >> 1], sel), __builtin_amdgcn_perm(w[7][c >> 1], w[6][c >> 1], sel));
#pragma unroll
          for (int t = 0; t < MT; ++t) {
            f32x4& acc = o[t][u * S::kCpl + c];
            acc = __builtin_amdgcn_mfma_f32_16x16x32_bf16(
                __builtin_bit_cast(bf16x8, v), __builtin_bit_cast(bf16x8, make_uint4(plo[t][0], plo[t][1], plo[t][2], plo[t][3])), acc, 0, 0, 0);
            acc = __builtin_amdgcn_mfma_f32_16x16x32_bf16(
                __builtin_bit_cast(bf16x8, v), __builtin_bit_cast(bf16x8, make_uint4(p[t][0], p[t][1], p[t][2], p[t][3])), acc, 0, 0, 0);
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
        const int seen = len - (cur.m - 1 - over_g(r));
        add_not_finite<D, FP8 ? 1 : 0>(a, cur.b, cur.h, max(max(len - (cur.m - 1), cur.off * kGroup), 0), min(seen, row_hi), c4, y);
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

// The heads that fell into several shares: a workgroup per (head, row), 256 / (D / 4) pieces at a time and eight rounds of them
// requested together, so that what takes the time is one round trip for where the pieces are and one for them.
template <int D>
__global__ __launch_bounds__(256) void k_attend_rows_join(AttendArgs a) {
  constexpr int kLanes = D / 4, kWays = 256 / kLanes, kRounds = 8;
  __shared__ float4 pass[kWays][kLanes];
  __shared__ float2 pass_ml[kWays];
  const int nth = blockIdx.x / a.short_rows, row = blockIdx.x - nth * a.short_rows;
  const int4 info = ((const int4*)(a.ws + a.plan.info))[nth];
  const int unit = a.plan.by_share ? info.x : nth;
  if (unit < 0) return;
  const int b = unit / a.Hkv, h = unit - b * a.Hkv;
  const int t0 = first_token(a, b), m = first_token(a, b + 1) - t0;
  if (m < 1 || m * a.G > a.short_rows || row >= m * a.G) return;
  const int pieces = info.z;
  if (pieces <= 1) return;
  const float vs = a.vscale ? a.vscale[unit] : 1.0f;
  const int way = threadIdx.x / kLanes, c4 = threadIdx.x % kLanes * 4;
  const float* po = (const float*)(a.ws + a.plan.part_o) + c4;
  const float2* part_ml = (const float2*)(a.ws + a.plan.part_ml);
  float top = -__builtin_inff(), sum = 0.0f;
  float4 acc = make_float4(0, 0, 0, 0);
  auto take = [&](float2 ml, float4 y) {
    const float t = fmaxf(top, ml.x), from = t == -__builtin_inff() ? 0.0f : t;
    const float f = pow2(top - from), n = pow2(ml.x - from);
    top = t;
    sum = sum * f + ml.y * n;
    acc.x = acc.x * f + y.x * n; acc.y = acc.y * f + y.y * n; acc.z = acc.z * f + y.z * n; acc.w = acc.w * f + y.w * n;
  };
  for (int i0 = way; i0 < pieces; i0 += kWays * kRounds) {
    float2 ml[kRounds];
    float4 y[kRounds];
#pragma unroll
    for (int k = 0; k < kRounds; ++k) {
      const int i = i0 + k * kWays < pieces ? i0 + k * kWays : i0;
      const long long slot = ((long long)(info.y + i) * 2 + (i == 0 ? 1 : 0)) * a.plan.piece_rows + row;
      ml[k] = part_ml[slot];
      y[k] = *(const float4*)(po + slot * D);
    }
#pragma unroll
    for (int k = 0; k < kRounds; ++k)
      if (i0 + k * kWays < pieces) take(ml[k], y[k]);
  }
  if (c4 == 0) pass_ml[way] = make_float2(top, sum);
  pass[way][c4 / 4] = acc;
  __syncthreads();
  if (way != 0) return;
#pragma unroll
  for (int w = 1; w < kWays; ++w) take(pass_ml[w], pass[w][c4 / 4]);
  write_row<D>(a, t0, h, row / a.G, row % a.G, c4, vs, top, sum, acc);
}

template <int D, bool FP8, int MT>
static hipError_t rows_of_height(const AttendArgs& a, hipStream_t st) {
  static LdsOptIn opt;
  const size_t bytes = rows_lds_floats<D, MT>() * sizeof(float);
  const hipError_t e = opt.ensure((const void*)k_attend_rows<D, FP8, MT>, bytes);
  if (e != hipSuccess) return e;
  k_attend_rows<D, FP8, MT><<<a.plan.shares, 256, bytes, st>>>(a);
  const hipError_t e2 = hipGetLastError();
  if (e2 != hipSuccess) return e2;
  k_attend_rows_join<D><<<(a.plan.by_share ? a.plan.shares : a.B * a.Hkv) * a.short_rows, 256, 0, st>>>(a);
  return hipGetLastError();
}
template <int D, bool FP8>
static hipError_t rows_of_type(const AttendArgs& a, hipStream_t st) {
  if constexpr (D < 256)
    if (a.plan.mt == 4) return rows_of_height<D, FP8, 4>(a, st);
  if (a.plan.mt == 2) return rows_of_height<D, FP8, 2>(a, st);
  return rows_of_height<D, FP8, 1>(a, st);
}

hipError_t launch_attend_rows(const AttendArgs& a, const Dims& d, hipStream_t st) {
  if (d.kv_fp8) return d.D == 128 ? rows_of_type<128, true>(a, st) : rows_of_type<256, true>(a, st);
  return d.D == 64 ? rows_of_type<64, false>(a, st) : d.D == 128 ? rows_of_type<128, false>(a, st) : rows_of_type<256, false>(a, st);
}

}  // namespace ea
