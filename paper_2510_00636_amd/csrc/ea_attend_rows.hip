// Attention of few (token, head) rows per KV head: single tokens, and stretches of a few.
//
// The cache is read once and that bounds it (4 G d operations for 4 d bytes of a pair), so the whole chip reads all the time:
// the call's heads are laid end to end in groups of 128 rows and every workgroup takes an equal, contiguous share of them,
// from the lengths that stand on the device.  A head that falls into several shares leaves partial results (maximum, sum,
// weighted values) that a second launch joins in the order of the shares.
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

// the groups of super-unit su (a sequence where heads share a length, else a head): none if it is not this kernel's
__device__ __forceinline__ int groups_of(const AttendArgs& a, int su) {
  const int b = a.per_head ? su / a.Hkv : su;
  const int m = first_token(a, b + 1) - first_token(a, b);
  if (m < 1 || m * a.G > a.short_rows) return 0;
  const int len = rows_of(a, b, a.per_head ? su - b * a.Hkv : 0);
  return len < 1 ? 1 : (len + kGroup - 1) / kGroup;
}

template <int D, bool FP8>
struct RowShape {
  static constexpr int kBytes = D * (FP8 ? 1 : 2);       // of a cached row
  static constexpr int kSteps = D / 32;                  // of the first product
  static constexpr int kCpl = D == 64 ? 4 : FP8 && D == 256 ? 16 : 8;    // channels per lane and load of V
  static constexpr int kLoads = D / (16 * kCpl);
  static constexpr int kTiles = D / 16;                  // output tiles of 16 channels
};

// a row of V as it is loaded: kCpl channels
template <int D, bool FP8> struct VPiece { uint4 w; };
template <> struct VPiece<64, false> { uint2 w; };
template <> struct VPiece<128, true> { uint2 w; };

// channels 2 x, 2 x + 1 of a loaded piece as bf16
template <int D, bool FP8>
__device__ __forceinline__ void widen_piece(const VPiece<D, FP8>& p, uint32_t* o) {
  if constexpr (!FP8 && D == 64) {
    o[0] = p.w.x; o[1] = p.w.y;
  } else if constexpr (!FP8) {
    o[0] = p.w.x; o[1] = p.w.y; o[2] = p.w.z; o[3] = p.w.w;
  } else if constexpr (D == 128) {
    const uint4 t = widen_fp8(p.w);
    o[0] = t.x; o[1] = t.y; o[2] = t.z; o[3] = t.w;
  } else {
    const uint4 t = widen_fp8(make_uint2(p.w.x, p.w.y)), u = widen_fp8(make_uint2(p.w.z, p.w.w));
    o[0] = t.x; o[1] = t.y; o[2] = t.z; o[3] = t.w;
    o[4] = u.x; o[5] = u.y; o[6] = u.z; o[7] = u.w;
  }
}

}  // namespace

template <int D, bool FP8, int MT>
__global__ __launch_bounds__(256, (D * MT > 128 ? 1 : 2)) void k_attend_rows(AttendArgs a) {
  using S = RowShape<D, FP8>;
  constexpr int kM = 16 * MT;
  __shared__ float pass_o[2][MT * S::kTiles * 4][64];
  __shared__ float pass_ml[4][2][kM];
  const int lane = threadIdx.x & 63, wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
  const int n16 = lane & 15, g = lane >> 4;
  const int supers = a.per_head ? a.B * a.Hkv : a.B, mult = a.per_head ? 1 : a.Hkv;

  // ---- the share: total of all groups, then the super-unit in which this workgroup's begins
  int mine = lane < supers ? groups_of(a, lane) : 0;
  int pre = wave_prefix(mine);
  int total = last_lane(pre);
  for (int base = 64; base < supers; base += 64)
    total += last_lane(wave_prefix(base + lane < supers ? groups_of(a, base + lane) : 0));
  const long long all = (long long)total * mult;
  const long long per = (all + gridDim.x - 1) / gridDim.x;
  const long long x0 = per * blockIdx.x, x1 = x0 + per < all ? x0 + per : all;
  if (x0 >= x1) return;
  int su = 0, have = 0;     // `have`: groups in front of super-unit su
  for (int base = 0; base < supers; base += 64) {
    if (base > 0) pre = wave_prefix(mine = base + lane < supers ? groups_of(a, base + lane) : 0);
    const uint64_t in = __ballot((long long)(have + pre) * mult > x0);
    if (in) {
      const int l = __builtin_ctzll(in);
      su = base + l;
      have += __builtin_amdgcn_readlane(pre, l) - __builtin_amdgcn_readlane(mine, l);
      break;
    }
    have += last_lane(pre);
  }
  int grp = groups_of(a, su);
  grp = __builtin_amdgcn_readfirstlane(grp);
  if (grp == 0) return;

  long long x = x0;
  while (x < x1) {
    const int rel = (int)(x - (long long)have * mult);
    const int hh = rel / grp, off = rel - hh * grp;
    const int take = (int)(x1 - x < grp - off ? x1 - x : grp - off);
    const int b = a.per_head ? su / a.Hkv : su, h = a.per_head ? su - b * a.Hkv : hh;
    const int t0 = __builtin_amdgcn_readfirstlane(first_token(a, b));
    const int m = __builtin_amdgcn_readfirstlane(first_token(a, b + 1)) - t0;
    const int len = __builtin_amdgcn_readfirstlane(rows_of(a, b, h));
    const int rows = m * a.G;

    // the query operand: row n16 (+ 16) of the head's rows (token, head of the group), channels as the keys' operand has them
    bf16x8 q[MT][S::kSteps];
    int vis[MT];            // keys that the row sees
#pragma unroll
    for (int t = 0; t < MT; ++t) {
      const int row = t * 16 + n16, tok = row / a.G, hd = row - tok * a.G;
      const bool in = row < rows;
      vis[t] = in ? len - (m - 1 - tok) : len;
      const __bf16* src = (const __bf16*)a.q + (long long)(t0 + (in ? tok : 0)) * a.q_stride + (h * a.G + (in ? hd : 0)) * D;
#pragma unroll
      for (int s = 0; s < S::kSteps; ++s) {
        const int c = FP8 ? (s >> 1) * 64 + g * 16 + (s & 1) * 8 : s * 32 + g * 8;
        bf16x8 w = *(const bf16x8*)(src + c);
        if (!in) w = (bf16x8)(__bf16)0.0f;
        q[t][s] = w;
      }
    }
    const float qk = a.scale * (FP8 && a.kscale ? a.kscale[b * a.Hkv + h] : 1.0f);

    f32x4 o[MT][S::kTiles];
    float mx[MT], l[MT];
#pragma unroll
    for (int t = 0; t < MT; ++t) {
      mx[t] = -__builtin_inff();
      l[t] = 0.0f;
#pragma unroll
      for (int c = 0; c < S::kTiles; ++c) o[t][c] = (f32x4)0.0f;
    }

    const int row_lo = off * kGroup, row_hi = min((off + take) * kGroup, len);
    int row = row_lo + wave * 32;
    // table entries of the wavefront's next 32 tiles, two per tile, one in each lane
    int entries = 0, window = row;
    auto load_window = [&](int from) {
      const int r = from + (lane >> 1) * kGroup + (lane & 1) * 16;
      entries = table_entry(a, b, r < len ? r : len - 1);
      window = from;
    };
    uint4 kraw[2][FP8 ? S::kSteps / 2 : S::kSteps];
    VPiece<D, FP8> vraw[8][S::kLoads];
    long long base[2];
    int lim[2];
    auto place = [&](int at) {      // the two halves of the tile at row `at`: where they start, and their last row
#pragma unroll
      for (int t = 0; t < 2; ++t) {
        const int r = at + t * 16 < len ? at + t * 16 : at;
        const int e = __builtin_amdgcn_readlane(entries, (at - window) / kGroup * 2 + (r != at ? 1 : 0));
        base[t] = row_base(a, b, h, r, e) * S::kBytes;
        lim[t] = len - 1 - r < 15 ? len - 1 - r : 15;
      }
    };
    auto load_k = [&]() {
#pragma unroll
      for (int t = 0; t < 2; ++t) {
        const char* p = (const char*)a.k + base[t];
        const int at = (n16 < lim[t] ? n16 : lim[t]) * S::kBytes + g * 16;
#pragma unroll
        for (int s = 0; s < (FP8 ? S::kSteps / 2 : S::kSteps); ++s) kraw[t][s] = *(const uint4*)(p + at + s * 64);
      }
    };
    auto load_v = [&]() {
#pragma unroll
      for (int j = 0; j < 8; ++j) {
        const char* p = (const char*)a.v + base[j >> 2];
        const int r = 4 * g + (j & 3), last = lim[j >> 2];
        const int at = (r < last ? r : last) * S::kBytes + n16 * (S::kCpl * (FP8 ? 1 : 2));
#pragma unroll
        for (int u = 0; u < S::kLoads; ++u)
          vraw[j][u] = *(const VPiece<D, FP8>*)(p + at + u * (16 * S::kCpl * (FP8 ? 1 : 2)));
      }
    };
    if (row < row_hi) {
      load_window(row);
      place(row);
      load_k();
      load_v();
    }
    while (row < row_hi) {
      const int next = row + kGroup;
      // ---- S^T: 32 keys x 16 rows
      f32x4 s[MT][2];
#pragma unroll
      for (int t = 0; t < MT; ++t) s[t][0] = s[t][1] = (f32x4)0.0f;
#pragma unroll
      for (int c = 0; c < S::kSteps; ++c)
#pragma unroll
        for (int t = 0; t < 2; ++t) {
          uint4 w;
          if constexpr (FP8) {
            const uint4 p = kraw[t][c >> 1];
            w = c & 1 ? widen_fp8(make_uint2(p.z, p.w)) : widen_fp8(make_uint2(p.x, p.y));
          } else {
            w = kraw[t][c];
          }
#pragma unroll
          for (int i = 0; i < MT; ++i)
            s[i][t] = __builtin_amdgcn_mfma_f32_16x16x32_bf16(__builtin_bit_cast(bf16x8, w), q[i][c], s[i][t], 0, 0, 0);
        }
      const bool more = next < row_hi;
      if (more) {
        if (next - window >= 32 * kGroup) load_window(next);
        place(next);
        load_k();
      }
      __builtin_amdgcn_sched_barrier(0);
      // ---- weights.  The maximum that they are taken against moves only when a row's passes it by more than 2^8: their sum and
      // the weighted values stay far from either end of fp32 then, and the division at the end takes the factor out again.
      const bool ragged = row + 32 > len - (m - 1);
      uint32_t p[MT][4];
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
        if (__any(top > mx[t] + 8.0f)) {
          top = fmaxf(max_xor16(max_xor32(top)), mx[t]);
          const float f = mx[t] == -__builtin_inff() ? 0.0f : pow2(mx[t] - top);
          mx[t] = top;
          l[t] *= f;
#pragma unroll
          for (int c = 0; c < S::kTiles; ++c) o[t][c] *= f;
        }
        const float from = mx[t] == -__builtin_inff() ? 0.0f : mx[t];
#pragma unroll
        for (int i = 0; i < 4; ++i) {
          const float lo = pow2(s[t][i >> 1][(i & 1) * 2] - from), hi = pow2(s[t][i >> 1][(i & 1) * 2 + 1] - from);
          l[t] += lo + hi;
          p[t][i] = pack_bf16(lo, hi);
        }
      }
      // ---- O^T
#pragma unroll
      for (int u = 0; u < S::kLoads; ++u) {
        uint32_t w[8][S::kCpl / 2];
#pragma unroll
        for (int j = 0; j < 8; ++j) {
          widen_piece<D, FP8>(vraw[j][u], w[j]);
          // rows behind the last one weigh nothing, whatever they hold
          if (row + 32 > len && row + (j >> 2) * 16 + 4 * g + (j & 3) >= len)
#pragma unroll
            for (int c = 0; c < S::kCpl / 2; ++c) w[j][c] = 0u;
        }
#pragma unroll
        for (int c = 0; c < S::kCpl; ++c) {
          const uint32_t sel = c & 1 ? 0x07060302u : 0x05040100u;
          const uint4 v = make_uint4(__builtin_amdgcn_perm(w[1][c >> 1], w[0][c >> 1], sel), __builtin_amdgcn_perm(w[3][c >> 1], w[2][c >> 1], sel),
                                     __builtin_amdgcn_perm(w[5][c >> 1], w[4][c >> 1], sel), __builtin_amdgcn_perm(w[7][c >> 1], w[6][c >> 1], sel));
#pragma unroll
          for (int t = 0; t < MT; ++t)
            o[t][u * S::kCpl + c] = __builtin_amdgcn_mfma_f32_16x16x32_bf16(
                __builtin_bit_cast(bf16x8, v), __builtin_bit_cast(bf16x8, make_uint4(p[t][0], p[t][1], p[t][2], p[t][3])),
                o[t][u * S::kCpl + c], 0, 0, 0);
        }
      }
      if (more) load_v();
      __builtin_amdgcn_sched_barrier(0);
      row = next;
    }

    // ---- the four wavefronts' results: one maximum per row, then sums over wavefronts 2 + 0 and 3 + 1, then the two
#pragma unroll
    for (int t = 0; t < MT; ++t) {
      l[t] = sum_xor16(sum_halves(l[t]));
      if (g == 0) {
        pass_ml[wave][0][t * 16 + n16] = mx[t];
        pass_ml[wave][1][t * 16 + n16] = l[t];
      }
    }
    __syncthreads();
    float top[MT], sum[MT];
#pragma unroll
    for (int t = 0; t < MT; ++t) {
      const int r = t * 16 + n16;
      top[t] = fmaxf(fmaxf(pass_ml[0][0][r], pass_ml[1][0][r]), fmaxf(pass_ml[2][0][r], pass_ml[3][0][r]));
      const float from = top[t] == -__builtin_inff() ? 0.0f : top[t];
      sum[t] = 0.0f;
#pragma unroll
      for (int w = 0; w < 4; ++w) sum[t] += pass_ml[w][1][r] * pow2(pass_ml[w][0][r] - from);
      const float f = pow2(mx[t] - from);
#pragma unroll
      for (int c = 0; c < S::kTiles; ++c) o[t][c] *= f;
    }
    if (wave >= 2)
#pragma unroll
      for (int t = 0; t < MT; ++t)
#pragma unroll
        for (int c = 0; c < S::kTiles; ++c)
#pragma unroll
          for (int r = 0; r < 4; ++r) pass_o[wave - 2][(t * S::kTiles + c) * 4 + r][lane] = o[t][c][r];
    __syncthreads();
    if (wave < 2)
#pragma unroll
      for (int t = 0; t < MT; ++t)
#pragma unroll
        for (int c = 0; c < S::kTiles; ++c)
#pragma unroll
          for (int r = 0; r < 4; ++r) {
            o[t][c][r] += pass_o[wave][(t * S::kTiles + c) * 4 + r][lane];
            if (wave == 1) pass_o[1][(t * S::kTiles + c) * 4 + r][lane] = o[t][c][r];
          }
    __syncthreads();
    if (wave == 0) {
#pragma unroll
      for (int t = 0; t < MT; ++t)
#pragma unroll
        for (int c = 0; c < S::kTiles; ++c)
#pragma unroll
          for (int r = 0; r < 4; ++r) o[t][c][r] += pass_o[1][(t * S::kTiles + c) * 4 + r][lane];
      const int unit = b * a.Hkv + h;
      const bool whole = take == grp;
      if (off == 0 && lane == 0) {      // the pieces of this head: the workgroups from this one on, for the joining launch
        const long long end = x + grp - 1;
        ((int2*)(a.ws + a.plan.info))[unit] = make_int2((int)blockIdx.x, (int)(end / per - blockIdx.x) + 1);
      }
      // channel u 16 cpl + (4 g + r) cpl + c of row n16 is o[u cpl + c][r]
      if (whole) {
        const float vs = FP8 && a.vscale ? a.vscale[unit] : 1.0f;
#pragma unroll
        for (int t = 0; t < MT; ++t) {
          const int rw = t * 16 + n16, tok = rw / a.G, hd = rw - tok * a.G;
          if (rw < rows) {
            const long long at = (long long)(t0 + tok) * a.Hq + h * a.G + hd;
            const float f = vs / sum[t];
            __bf16* dst = (__bf16*)a.out + at * D;
#pragma unroll
            for (int u = 0; u < S::kLoads; ++u)
#pragma unroll
              for (int r = 0; r < 4; ++r) {
                const int c0 = u * 16 * S::kCpl + (4 * g + r) * S::kCpl;
#pragma unroll
                for (int c = 0; c < S::kCpl; c += 4) {
                  const f32x4* w = &o[t][u * S::kCpl + c];
                  *(uint2*)(dst + c0 + c) = sum[t] > 0.0f || sum[t] != sum[t]
                      ? make_uint2(pack_bf16(w[0][r] * f, w[1][r] * f), pack_bf16(w[2][r] * f, w[3][r] * f)) : make_uint2(0u, 0u);
                }
              }
            if (a.lse && g == 0) a.lse[at] = natural_lse(top[t], sum[t]);
          }
        }
      } else {
        // slot 0 of a workgroup: a head that began in front of it; slot 1: one that goes on behind it
        const long long slot = ((long long)blockIdx.x * 2 + (off == 0 ? 1 : 0)) * kM;
        float* po = (float*)(a.ws + a.plan.part_o) + slot * D;
        float2* ml = (float2*)(a.ws + a.plan.part_ml) + slot;
#pragma unroll
        for (int t = 0; t < MT; ++t) {
          const int rw = t * 16 + n16;
          if (rw < rows) {
#pragma unroll
            for (int u = 0; u < S::kLoads; ++u)
#pragma unroll
              for (int r = 0; r < 4; ++r) {
                const int c0 = u * 16 * S::kCpl + (4 * g + r) * S::kCpl;
#pragma unroll
                for (int c = 0; c < S::kCpl; c += 4) {
                  const f32x4* w = &o[t][u * S::kCpl + c];
                  *(float4*)(po + (long long)rw * D + c0 + c) = make_float4(w[0][r], w[1][r], w[2][r], w[3][r]);
                }
              }
            if (g == 0) ml[rw] = make_float2(top[t], sum[t]);
          }
        }
      }
    }
    x += take;
    if (x < x1) {
      __syncthreads();      // the next head's results go through the same LDS
      if (x >= (long long)(have + grp) * mult) {
        have += grp;
        do {
          if (++su >= supers) return;
          grp = __builtin_amdgcn_readfirstlane(groups_of(a, su));
        } while (grp == 0);
      }
    }
  }
}

// The heads that fell into several shares: one workgroup per (head, row), four pieces at a time.
template <int D>
__global__ __launch_bounds__(256) void k_attend_rows_join(AttendArgs a) {
  constexpr int kLanes = D / 4, kWays = 256 / kLanes;
  __shared__ float4 pass[kWays][kLanes];
  __shared__ float pass_l[kWays];
  const int unit = blockIdx.x / a.short_rows, row = blockIdx.x - unit * a.short_rows;
  const int b = unit / a.Hkv, h = unit - b * a.Hkv;
  const int t0 = first_token(a, b), m = first_token(a, b + 1) - t0;
  if (m < 1 || m * a.G > a.short_rows || row >= m * a.G) return;
  const int2 info = ((const int2*)(a.ws + a.plan.info))[unit];
  const int pieces = info.y;
  if (pieces <= 1) return;
  const int way = threadIdx.x / kLanes, c = threadIdx.x % kLanes;
  const float* po = (const float*)(a.ws + a.plan.part_o);
  const float2* ml = (const float2*)(a.ws + a.plan.part_ml);
  auto slot = [&](int i) { return ((long long)(info.x + i) * 2 + (i == 0 ? 1 : 0)) * a.plan.piece_rows + row; };
  float top = -__builtin_inff();
  for (int i = threadIdx.x & 63; i < pieces; i += 64) top = fmaxf(top, ml[slot(i)].x);
#pragma unroll
  for (int i = 1; i < 64; i *= 2) top = fmaxf(top, __shfl_xor(top, i));
  const float from = top == -__builtin_inff() ? 0.0f : top;
  float4 acc = make_float4(0, 0, 0, 0);
  float sum = 0.0f;
  for (int i = way; i < pieces; i += kWays) {
    const long long s = slot(i);
    const float2 w = ml[s];
    const float4 x = *(const float4*)(po + s * D + c * 4);
    const float f = pow2(w.x - from);
    sum += w.y * f;
    acc.x += x.x * f; acc.y += x.y * f; acc.z += x.z * f; acc.w += x.w * f;
  }
  pass[way][c] = acc;
  if (c == 0) pass_l[way] = sum;
  __syncthreads();
  if (way != 0) return;
  for (int w = 1; w < kWays; ++w) {
    const float4 x = pass[w][c];
    acc.x += x.x; acc.y += x.y; acc.z += x.z; acc.w += x.w;
    sum += pass_l[w];
  }
  const int tok = row / a.G, hd = row - tok * a.G;
  const long long at = (long long)(t0 + tok) * a.Hq + h * a.G + hd;
  const float f = (a.vscale ? a.vscale[unit] : 1.0f) / sum;
  const bool any = sum > 0.0f || sum != sum;
  *(uint2*)((__bf16*)a.out + at * D + c * 4) =
      any ? make_uint2(pack_bf16(acc.x * f, acc.y * f), pack_bf16(acc.z * f, acc.w * f)) : make_uint2(0u, 0u);
  if (a.lse && c == 0) a.lse[at] = natural_lse(top, sum);
}

template <int D, bool FP8>
static hipError_t rows_of_type(const AttendArgs& a, hipStream_t st) {
  if (D == 256 || a.plan.mt == 1) k_attend_rows<D, FP8, 1><<<a.plan.shares, 256, 0, st>>>(a);
  else if constexpr (D < 256) k_attend_rows<D, FP8, 2><<<a.plan.shares, 256, 0, st>>>(a);
  hipError_t e = hipGetLastError();
  if (e != hipSuccess) return e;
  k_attend_rows_join<D><<<a.B * a.Hkv * a.short_rows, 256, 0, st>>>(a);
  return hipGetLastError();
}

hipError_t launch_attend_rows(const AttendArgs& a, const Dims& d, hipStream_t st) {
  if (d.kv_fp8) return d.D == 128 ? rows_of_type<128, true>(a, st) : rows_of_type<256, true>(a, st);
  return d.D == 64 ? rows_of_type<64, false>(a, st) : d.D == 128 ? rows_of_type<128, false>(a, st) : rows_of_type<256, false>(a, st);
}

}  // namespace ea
