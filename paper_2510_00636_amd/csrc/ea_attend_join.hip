// The joining launch of stretches that are cut along the keys (16-, 8-, 4-bit and fp32 rows).
#include "ea_attend.h"

namespace ea {

// The pieces of every (token, head) row together.  What leads to a row (its sequence, how that was cut, its length) is asked for at once, a
// lane for a sequence where there are no more than lanes; then pieces.  WIDE: a workgroup per row, whose 256 threads request all the
// pieces at once.  Else D / 4 threads have ROWS rows, of which they request ROUNDS pieces each at a time.
template <int D, bool F32, bool WIDE, int ROWS, int ROUNDS>
__global__ __launch_bounds__(256) void k_attend_join(AttendArgs a) {
  constexpr int kLanes = D / 4, kRounds = ROUNDS, kWays = WIDE ? 256 / kLanes : 1, kRows = ROWS, kGroups = 256 / kLanes;
  __shared__ float4 pass[kWays][kLanes];
  __shared__ float2 pass_ml[kWays];
  const int lane = threadIdx.x & 63, c4 = threadIdx.x % kLanes * 4, way = WIDE ? threadIdx.x / kLanes : 0;
  const uint32_t at0 = WIDE ? blockIdx.x : blockIdx.x * (kGroups * kRows) + threadIdx.x / kLanes, hq = a.Hq;
  const int all = first_token(a, a.B);
  const int4* cuts = (const int4*)(a.ws + a.plan.cuts);      // of a sequence: its first piece, cuts, keys of a stretch, tiles
  const int mine = min(lane, a.B - 1), my_first = first_token(a, mine), my_end = first_token(a, mine + 1);
  const int my_len = a.per_head ? 0 : rows_of(a, mine, 0);
  const int4 my_cut = cuts[mine];
  // the sequence of the wavefront's first token: behind those that end in front of it
  const int token0 = __builtin_amdgcn_readfirstlane((int)(at0 / hq));
  int b = __popcll(__ballot(lane < a.B && my_end <= token0));
  for (int base = 64; base < a.B; base += 64) b += __popcll(__ballot(base + lane < a.B && first_token(a, min(base + lane, a.B - 1) + 1) <= token0));
  if (b >= a.B) return;      // tokens behind the last one are nobody's
  int t0, m, len;
  int4 sequence_cut;
  auto sequence = [&]() {
    if (a.B <= 64) {
      t0 = __shfl(my_first, b);
      m = __shfl(my_end, b) - t0;
      len = __shfl(my_len, b);
      sequence_cut = make_int4(__shfl(my_cut.x, b), __shfl(my_cut.y, b), __shfl(my_cut.z, b), __shfl(my_cut.w, b));
    } else {
      t0 = first_token(a, b);
      m = first_token(a, b + 1) - t0;
      len = a.per_head ? 0 : rows_of(a, b, 0);
      sequence_cut = cuts[b];
    }
  };
  sequence();
  const float* po = (const float*)(a.ws + a.plan.split_o) + c4;
  const float2* part_ml = (const float2*)(a.ws + a.plan.split_ml);
  const int apart = a.by_head ? 1 : a.Hkv;      // pieces next to each other in a row's order
  // where a row's pieces stand: how many (-1: none of this launch's rows), the first one's slot
  auto find = [&](uint32_t at, int& unit, int& n) -> long long {
    const int token = (int)(at / hq), head = (int)(at - token * hq), h = head / a.G;
    n = -1;
    unit = 0;
    // (all lanes go on together: they look at each other's)
    while (__any(token < all && token >= t0 + m && b + 1 < a.B)) {
      if (token < all && token >= t0 + m && b + 1 < a.B) ++b;
      sequence();
    }
    if (token >= all) return 0;
    if (token < t0 || token >= t0 + m || (a.only_long && m * a.G <= a.short_rows)) return 0;
    const int4 cut = a.by_head ? cuts[b * a.Hkv + h] : sequence_cut;
    if (cut.y <= 1) return 0;
    const int row = (token - t0) * a.G + (head - h * a.G), tile = row / a.plan.tile_rows;
    const int vis = (a.per_head ? rows_of(a, b, h) : len) - (a.sees ? 0 : m - 1 - (token - t0));
    int k = (vis + cut.z - 1) / cut.z;
    k = k < 1 ? 0 : k > cut.y ? cut.y : k;
    const int first = cut.x + (cut.w - 1 - tile) * cut.y * apart + (a.by_head ? 0 : h);
    // (prefix sums that do not ascend can count more pieces than there are: none is looked for outside the workspace)
    if (cut.y > a.plan.most_pieces || first < 0 || first + (k - 1) * apart >= a.plan.most_pieces) return 0;
    n = k;
    unit = b * a.Hkv + h;
    return (long long)first * a.plan.tile_rows + (row - tile * a.plan.tile_rows);
  };
  const long long step = (long long)apart * a.plan.tile_rows;      // from piece to piece of a row
  long long slot[kRows];
  int unit[kRows], n[kRows], most = 0;
#pragma unroll
  for (int r = 0; r < kRows; ++r) {
    slot[r] = find(at0 + r * kGroups, unit[r], n[r]);
    most = max(most, n[r]);
  }
  float top[kRows], sum[kRows];
  float4 acc[kRows];
#pragma unroll
  for (int r = 0; r < kRows; ++r) {
    top[r] = -__builtin_inff();
    sum[r] = 0.0f;
    acc[r] = make_float4(0, 0, 0, 0);
  }
  auto take = [&](int r, float2 ml, float4 y) {
    const float t = fmaxf(top[r], ml.x), from = t == -__builtin_inff() ? 0.0f : t;
    const float f = pow2(top[r] - from), w = pow2(ml.x - from);
    top[r] = t;
    sum[r] = sum[r] * f + ml.y * w;
    acc[r].x = acc[r].x * f + y.x * w; acc[r].y = acc[r].y * f + y.y * w; acc[r].z = acc[r].z * f + y.z * w; acc[r].w = acc[r].w * f + y.w * w;
  };
  for (int i0 = way; i0 < most; i0 += kRounds * kWays) {
    float2 ml[kRows][kRounds];
    float4 y[kRows][kRounds];
#pragma unroll
    for (int r = 0; r < kRows; ++r)
#pragma unroll
      for (int k = 0; k < kRounds; ++k) {
        const int i = min(i0 + k * kWays, n[r] - 1);          // (one that is there, asked for once more, if the row has no such piece)
        const long long at = n[r] > 0 ? slot[r] + i * step : 0;
        ml[r][k] = part_ml[at];
        y[r][k] = *(const float4*)(po + at * D);
      }
#pragma unroll
    for (int r = 0; r < kRows; ++r)
#pragma unroll
      for (int k = 0; k < kRounds; ++k)
        if (i0 + k * kWays < n[r]) take(r, ml[r][k], y[r][k]);
  }
  if constexpr (WIDE) {
    if (n[0] < 0) return;
    if (c4 == 0) pass_ml[way] = make_float2(top[0], sum[0]);
    pass[way][c4 / 4] = acc[0];
    __syncthreads();
    if (way != 0) return;
#pragma unroll
    for (int w = 1; w < kWays; ++w) take(0, pass_ml[w], pass[w][c4 / 4]);
  }
#pragma unroll
  for (int r = 0; r < kRows; ++r) {
    if (n[r] < 0) continue;
    const bool any = sum[r] > 0.0f || sum[r] != sum[r];
    const float f = (a.vscale ? a.vscale[unit[r]] : 1.0f) / sum[r];
    const size_t row = at0 + r * kGroups, to = row * D + c4;
    if (F32)
      *(float4*)((float*)a.out + to) = any ? make_float4(acc[r].x * f, acc[r].y * f, acc[r].z * f, acc[r].w * f) : make_float4(0, 0, 0, 0);
    else
      *(uint2*)((__bf16*)a.out + to) = any ? make_uint2(pack_bf16(acc[r].x * f, acc[r].y * f), pack_bf16(acc[r].z * f, acc[r].w * f)) : make_uint2(0u, 0u);
    if (a.lse && c4 == 0) a.lse[row] = natural_lse(top[r], sum[r]);
  }
}

template <int D, bool F32>
static hipError_t join_of_type(const AttendArgs& a, hipStream_t st) {
  const long long rows = (long long)a.n_tokens * a.Hq, per = 256 / (D / 4);
  // a workgroup per row as long as those are not many rounds of the chip's: d = 128, rows of 64 pieces 512 rows 5.8 us (else 77), of
  // 32 pieces 2048 rows 9.6 (51), of 16 pieces 8192 rows 21.8 (12.7).  Rows one by one while they are few for the chip, else four to
  // what leads to them.
  if (rows <= 4096) k_attend_join<D, F32, true, 1, 8><<<(unsigned)rows, 256, 0, st>>>(a);
  else if (rows <= 16384) k_attend_join<D, F32, false, 1, 8><<<(unsigned)((rows + per - 1) / per), 256, 0, st>>>(a);
  else if (rows <= 65536) k_attend_join<D, F32, false, 2, 4><<<(unsigned)((rows + 2 * per - 1) / (2 * per)), 256, 0, st>>>(a);
  else k_attend_join<D, F32, false, 4, 2><<<(unsigned)((rows + 4 * per - 1) / (4 * per)), 256, 0, st>>>(a);
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
