// The joining launch of few rows.
#include "ea_attend.h"

namespace ea {

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

hipError_t launch_attend_rows_join(const AttendArgs& a, hipStream_t st) {
  const unsigned grid = (unsigned)((a.plan.by_share ? a.plan.shares : a.B * a.Hkv) * a.short_rows);
  if (a.D == 64) k_attend_rows_join<64><<<grid, 256, 0, st>>>(a);
  else if (a.D == 128) k_attend_rows_join<128><<<grid, 256, 0, st>>>(a);
  else k_attend_rows_join<256><<<grid, 256, 0, st>>>(a);
  return hipGetLastError();
}

}  // namespace ea
