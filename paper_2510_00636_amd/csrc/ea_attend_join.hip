// The joining launch of stretches that are cut along the keys (16-, 8-, 4-bit and fp32 rows).
#include "ea_attend.h"

namespace ea {

// The pieces of every (token, head) row together, ROUNDS of them at a time.  WIDE: a workgroup per row, whose 256 threads request all the
// pieces at once; else D / 4 threads have ROWS, one after the other, so that a workgroup's lookups serve them all.  What leads to a row
// (its sequence, how that was cut, its length) is asked for at once where a group has one row, a lane for a sequence while there are no more than lanes; a
// workgroup's one row (640 to 2080 rows 0.3 to 0.7 us longer that way), and the first of several, look it up as they need it.
template <int D, bool F32, bool WIDE, int ROUNDS, int ROWS>
__global__ __launch_bounds__(256) void k_attend_join(AttendArgs a) {
  constexpr int kLanes = D / 4, kWays = WIDE ? 256 / kLanes : 1, kGroups = 256 / kLanes;
  __shared__ float4 pass[kWays][kLanes];
  __shared__ float2 pass_ml[kWays];
  const int lane = threadIdx.x & 63, c4 = threadIdx.x % kLanes * 4, way = WIDE ? threadIdx.x / kLanes : 0;
  const uint32_t at0 = WIDE ? blockIdx.x : blockIdx.x * (kGroups * ROWS) + threadIdx.x / kLanes, hq = a.Hq;
  const int all = first_token(a, a.B);
  const int4* cuts = (const int4*)(a.ws + a.plan.cuts);      // of a sequence: its first piece, cuts, keys of a stretch, tiles
  constexpr bool kAtOnce = !WIDE && ROWS == 1;
  const int mine = min(lane, a.B - 1), my_end = first_token(a, mine + 1);
  int my_first = 0, my_len = 0;
  int4 my_cut = make_int4(0, 0, 0, 0);
  if constexpr (kAtOnce) {
    my_first = first_token(a, mine);
    my_len = a.per_head ? 0 : rows_of(a, mine, 0);
    my_cut = cuts[mine];
  }
  // the sequence of the wavefront's first token: behind those that end in front of it
  const int token0 = __builtin_amdgcn_readfirstlane((int)(at0 / hq));
  int b = __popcll(__ballot(lane < a.B && my_end <= token0));
  for (int base = 64; base < a.B; base += 64) b += __popcll(__ballot(base + lane < a.B && first_token(a, min(base + lane, a.B - 1) + 1) <= token0));
  if (b >= a.B) return;      // tokens behind the last one are nobody's
  int t0, m, len;
  int4 cut;
  auto sequence = [&]() {
    if (kAtOnce && a.B <= 64) {
      t0 = __shfl(my_first, b);
      m = __shfl(my_end, b) - t0;
      len = __shfl(my_len, b);
      cut = make_int4(__shfl(my_cut.x, b), __shfl(my_cut.y, b), __shfl(my_cut.z, b), __shfl(my_cut.w, b));
    } else {
      t0 = first_token(a, b);
      m = first_token(a, b + 1) - t0;
      len = a.per_head ? 0 : rows_of(a, b, 0);
      cut = cuts[b];
    }
  };
  sequence();
#pragma unroll 1
  for (int nth = 0; nth < ROWS; ++nth) {
    const uint32_t at = at0 + nth * kGroups;      // token, head
    const int token = (int)(at / hq), head = (int)(at - token * hq), h = head / a.G;
    if constexpr (kAtOnce) {      // (all lanes go on together: they look at each other's)
      while (__any(token < all && token >= t0 + m && b + 1 < a.B)) {
        if (token < all && token >= t0 + m && b + 1 < a.B) ++b;
        sequence();
      }
    } else if (token < all && token >= t0 + m) {
      while (b + 1 < a.B && first_token(a, b + 1) <= token) ++b;
      sequence();
    }
    if (token >= all || token < t0 || token >= t0 + m || (a.only_long && m * a.G <= a.short_rows)) continue;
    const int unit = b * a.Hkv + h;
    const int4 c = a.by_head ? cuts[unit] : cut;
    if (c.y <= 1) continue;
    const int apart = a.by_head ? 1 : a.Hkv;      // pieces next to each other in a row's order
    const int row = (token - t0) * a.G + (head - h * a.G), tile = row / a.plan.tile_rows;
    const int vis = (a.per_head ? rows_of(a, b, h) : len) - (a.sees ? 0 : m - 1 - (token - t0));
    int n = (vis + c.z - 1) / c.z;
    n = n < 1 ? 0 : n > c.y ? c.y : n;
    const int first = c.x + (c.w - 1 - tile) * c.y * apart + (a.by_head ? 0 : h);
    // (prefix sums that do not ascend can count more pieces than there are: none is looked for outside the workspace)
    if (c.y > a.plan.most_pieces || first < 0 || first + (n - 1) * apart >= a.plan.most_pieces) continue;
    const long long slot = (long long)first * a.plan.tile_rows + (row - tile * a.plan.tile_rows), step = (long long)apart * a.plan.tile_rows;
    const float* po = (const float*)(a.ws + a.plan.split_o) + c4;
    const float2* part_ml = (const float2*)(a.ws + a.plan.split_ml);
    float top = -__builtin_inff(), sum = 0.0f;
    float4 acc = make_float4(0, 0, 0, 0);
    auto take = [&](float2 ml, float4 y) {
      const float t = fmaxf(top, ml.x), from = t == -__builtin_inff() ? 0.0f : t;
      const float f = pow2(top - from), w = pow2(ml.x - from);
      top = t;
      sum = sum * f + ml.y * w;
      acc.x = acc.x * f + y.x * w; acc.y = acc.y * f + y.y * w; acc.z = acc.z * f + y.z * w; acc.w = acc.w * f + y.w * w;
    };
    for (int i0 = way; i0 < n; i0 += ROUNDS * kWays) {
      float2 ml[ROUNDS];
      float4 y[ROUNDS];
#pragma unroll
      for (int k = 0; k < ROUNDS; ++k) {
        const long long from = slot + min(i0 + k * kWays, n - 1) * step;      // (the last one once more where there is none)
        ml[k] = part_ml[from];
        y[k] = *(const float4*)(po + from * D);
      }
#pragma unroll
      for (int k = 0; k < ROUNDS; ++k)
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
    const float f = (a.vscale ? a.vscale[unit] : 1.0f) / sum;
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
  const long long rows = (long long)a.n_tokens * a.Hq, per = 256 / (D / 4);
  // A workgroup per row while rows are few (whole calls, d = 128: 640 rows over 16k keys 29.1 us, else 33.6; 1024 over 131k 84.6 and 87.4, over
  // 4096 22.0 and 21.4; 2048 over 4096 31.8 and 28.0; 4096 over 16k 78.8 and 66.1).  Calls that have neither masks nor MX rows take it
  // up to 4096 rows: the order of their sums, and with it their last bits, stays what it was.
  // Eight pieces at a time up to 8192 rows, four behind that, when the chip is full (2048 rows over 16k keys 43.2 and 43.9 us, 4096 66.1 and
  // 67.2, 8128 61.0 and 60.7, 16k 87.4 and 85.9, 32k 93.7 and 89.3).
  // Four rows to a group of threads from 32768 on, where workgroups come in many rounds: two pieces each of 160k rows 35 us, so 21 (whole
  // calls, one and four: 38k rows 65.5 and 65.2, 61k 71.9 and 71.3, 160k 187 and 181, at d = 256 263 and 252, 460k 181 and 182; 17k 48.2 and
  // 51.0, 32k 70.9 and 72.5).
  constexpr int kMany = 4;
  auto groups = [&](int each) { return (unsigned)((rows + per * each - 1) / (per * each)); };
  if (rows <= (a.sees || a.mx ? 1024 : 4096)) k_attend_join<D, F32, true, 8, 1><<<(unsigned)rows, 256, 0, st>>>(a);
  else if (rows <= 8192) k_attend_join<D, F32, false, 8, 1><<<groups(1), 256, 0, st>>>(a);
  else if (rows <= 32768) k_attend_join<D, F32, false, 4, 1><<<groups(1), 256, 0, st>>>(a);
  else k_attend_join<D, F32, false, 4, kMany><<<groups(kMany), 256, 0, st>>>(a);
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
