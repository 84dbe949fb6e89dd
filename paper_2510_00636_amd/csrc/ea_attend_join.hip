// The joining launch of stretches that are cut along the keys (bf16, 8-bit and fp32 rows).
#include "ea_attend.h"

namespace ea {

// The pieces of every (token, head) row together.  Few rows (WIDE) have a workgroup each, whose 256 threads request all the pieces at
// once.  Many: D / 4 threads have one row after the other, kJoinRows in all, so that what leads to a row (its sequence, how that was
// cut) is looked up once and not once a row.  Two pieces each of 22k rows at d = 256: 20 us with two or four rows, 22 with eight, 33
// with sixteen or one; the bytes alone take 13.
constexpr int kJoinRows = 4;
template <int D, bool F32, bool WIDE>
__global__ __launch_bounds__(256) void k_attend_join(AttendArgs a) {
  constexpr int kLanes = D / 4, kRounds = WIDE ? 8 : 4, kWays = WIDE ? 256 / kLanes : 1, kRows = WIDE ? 1 : kJoinRows, kGroups = 256 / kLanes;
  __shared__ float4 pass[kWays][kLanes];
  __shared__ float2 pass_ml[kWays];
  const int lane = threadIdx.x & 63, c4 = threadIdx.x % kLanes * 4, way = WIDE ? threadIdx.x / kLanes : 0;
  const uint32_t at0 = WIDE ? blockIdx.x : blockIdx.x * (kGroups * kRows) + threadIdx.x / kLanes, hq = a.Hq;
  const int all = first_token(a, a.B);
  // the sequence of the wavefront's first token: behind those that end in front of it
  const int token0 = __builtin_amdgcn_readfirstlane((int)(at0 / hq));
  int b = 0;
  for (int base = 0; base < a.B; base += 64) b += __popcll(__ballot(base + lane < a.B && first_token(a, min(base + lane, a.B - 1) + 1) <= token0));
  if (b >= a.B) return;      // tokens behind the last one are nobody's
  int t0 = first_token(a, b), m = first_token(a, b + 1) - t0;
  int4 cut = ((const int4*)(a.ws + a.plan.cuts))[b];      // its first piece, cuts, keys of a stretch, tiles
  const float* po = (const float*)(a.ws + a.plan.split_o) + c4;
  const float2* part_ml = (const float2*)(a.ws + a.plan.split_ml);
#pragma unroll 1
  for (int nth = 0; nth < kRows; ++nth) {
    const uint32_t at = at0 + nth * kGroups;
    const int token = (int)(at / hq), head = (int)(at - token * hq), h = head / a.G;
    if (token >= all) return;
    if (token >= t0 + m) {
      while (b + 1 < a.B && first_token(a, b + 1) <= token) ++b;
      t0 = first_token(a, b);
      m = first_token(a, b + 1) - t0;
      cut = ((const int4*)(a.ws + a.plan.cuts))[b];
    }
    if (token < t0 || token >= t0 + m || (a.only_long && m * a.G <= a.short_rows) || cut.y <= 1) continue;
    const int row = (token - t0) * a.G + (head - h * a.G), tile = row / a.plan.tile_rows;
    const int vis = rows_of(a, b, h) - (m - 1 - (token - t0));
    int n = (vis + cut.z - 1) / cut.z;
    n = n < 1 ? 0 : n > cut.y ? cut.y : n;
    const int first = cut.x + (cut.w - 1 - tile) * cut.y * a.Hkv + h;
    // (prefix sums that do not ascend can count more pieces than there are: none is looked for outside the workspace)
    if (cut.y > a.plan.most_pieces || first < 0 || first + (n - 1) * a.Hkv >= a.plan.most_pieces) continue;
    float top = -__builtin_inff(), sum = 0.0f;
    float4 acc = make_float4(0, 0, 0, 0);
    auto take = [&](float2 ml, float4 y) {
      const float t = fmaxf(top, ml.x), from = t == -__builtin_inff() ? 0.0f : t;
      const float f = pow2(top - from), w = pow2(ml.x - from);
      top = t;
      sum = sum * f + ml.y * w;
      acc.x = acc.x * f + y.x * w; acc.y = acc.y * f + y.y * w; acc.z = acc.z * f + y.z * w; acc.w = acc.w * f + y.w * w;
    };
    for (int i0 = way; i0 < n; i0 += kRounds * kWays) {
      float2 ml[kRounds];
      float4 y[kRounds];
#pragma unroll
      for (int k = 0; k < kRounds; ++k) {
        const int i = i0 + k * kWays;
        if (i >= n) break;
        const long long slot = (long long)(first + i * a.Hkv) * a.plan.tile_rows + (row - tile * a.plan.tile_rows);
        ml[k] = part_ml[slot];
        y[k] = *(const float4*)(po + slot * D);
      }
#pragma unroll
      for (int k = 0; k < kRounds; ++k)
        if (i0 + k * kWays < n) take(ml[k], y[k]);
    }
    if constexpr (WIDE) {
      if (c4 == 0) pass_ml[way] = make_float2(top, sum);
      pass[way][c4 / 4] = acc;
      __syncthreads();
      if (way != 0) return;
#pragma unroll
      for (int w = 1; w < kWays; ++w) take(pass_ml[w], pass[w][c4 / 4]);
    }
    const bool any = sum > 0.0f || sum != sum;
    const float f = (a.vscale ? a.vscale[b * a.Hkv + h] : 1.0f) / sum;
    const size_t to = (size_t)at * D + c4;
    if (F32)
      *(float4*)((float*)a.out + to) = any ? make_float4(acc.x * f, acc.y * f, acc.z * f, acc.w * f) : make_float4(0, 0, 0, 0);
    else
      *(uint2*)((__bf16*)a.out + to) = any ? make_uint2(pack_bf16(acc.x * f, acc.y * f), pack_bf16(acc.z * f, acc.w * f)) : make_uint2(0u, 0u);
    if (a.lse && c4 == 0) a.lse[at] = natural_lse(top, sum);
  }
}

template <int D, bool F32>
static hipError_t join_of_type(const AttendArgs& a, hipStream_t st) {
  const long long rows = (long long)a.n_tokens * a.Hq, per = 256 / (D / 4) * kJoinRows;
  // a workgroup per row as long as those are not many rounds of the chip's: d = 128, rows of 64 pieces 512 rows 5.8 us (else 77), of
  // 32 pieces 2048 rows 9.6 (51), of 16 pieces 8192 rows 21.8 (12.7)
  if (rows <= 4096) k_attend_join<D, F32, true><<<(unsigned)rows, 256, 0, st>>>(a);
  else k_attend_join<D, F32, false><<<(unsigned)((rows + per - 1) / per), 256, 0, st>>>(a);
  return hipGetLastError();
}
hipError_t launch_attend_join(const AttendArgs& a, bool f32, hipStream_t st) {
#define EA_CASE(DD) if (a.D == DD) return f32 ? join_of_type<DD, true>(a, st) : join_of_type<DD, false>(a, st)
  EA_CASE(64);
  EA_CASE(128);
#undef EA_CASE
  return f32 ? join_of_type<256, true>(a, st) : join_of_type<256, false>(a, st);
}

}  // namespace ea
