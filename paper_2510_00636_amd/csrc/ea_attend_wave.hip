// Attention of a wavefront per (token, head) row: MX pools and drafted trees, every type and size, nothing shared between rows.
#include "ea_attend.h"
#include "ea_mx.h"

namespace ea {

namespace {

// D / 64 channels of row `row` of unit (b, h), of K or V
template <int D>
__device__ __forceinline__ void load_row(const AttendArgs& a, bool values, int b, int h, int row, int lane, float* x) {
  constexpr int kPer = D / 64;
  const long long at = row_base(a, b, h, row, table_entry(a, b, row));
  const void* base = values ? a.v : a.k;
#pragma unroll
  for (int i = 0; i < kPer; ++i) {
    const int c = lane * kPer + i;
    if (a.mx) {
      const float scale = mx_scale((values ? a.vscale8 : a.kscale8)[at * (D / 32) + c / 32]);
      const uint32_t w = a.mx == 8 ? ((const uint8_t*)base)[at * D + c] : ((const uint8_t*)base)[(at * D + c) / 2] >> (c & 1) * 4;
      x[i] = __uint_as_float((a.mx == 8 ? mx8_pair(w, scale, false) : mx4_pair<0>(w, scale)) << 16);
    } else if (a.f32) {
      x[i] = ((const float*)base)[at * D + c];
    } else {
      x[i] = (float)((const __bf16*)base)[at * D + c];
    }
  }
}

}  // namespace

template <int D>
__global__ __launch_bounds__(64) void k_attend_wave(AttendArgs a) {
  constexpr int kPer = D / 64;
  const int lane = threadIdx.x, token = blockIdx.x / a.Hq, head = blockIdx.x % a.Hq, h = head / a.G;
  if (token >= first_token(a, a.B)) return;
  int b = 0;
  while (b < a.B && first_token(a, b + 1) <= token) ++b;
  if (b >= a.B || token < first_token(a, b)) return;
  const int t0 = first_token(a, b), m = first_token(a, b + 1) - t0, len = rows_of(a, b, h), old = len - m;
  if (a.only_long && m * a.G <= a.short_rows) return;
  float q[kPer], o[kPer] = {};
#pragma unroll
  for (int i = 0; i < kPer; ++i) {
    const long long at = (long long)token * a.q_stride + head * D + lane * kPer + i;
    q[i] = a.f32 ? ((const float*)a.q)[at] : (float)((const __bf16*)a.q)[at];
  }
  float top = -__builtin_inff(), sum = 0.0f;
  for (int row = 0; row < len; ++row) {
    const int j = row - old;
    const bool seen = j < 0 || (a.sees ? j < 64 * a.words && (a.sees[(long long)token * a.words + (j >> 6)] >> (j & 63) & 1) : j <= token - t0);
    if (!seen) continue;
    float x[kPer], s = 0.0f;
    load_row<D>(a, false, b, h, row, lane, x);
#pragma unroll
    for (int i = 0; i < kPer; ++i) s = fmaf(x[i], q[i], s);
#pragma unroll
    for (int d = 1; d < 64; d *= 2) s += __shfl_xor(s, d);
    s *= a.scale;
    if (s == -__builtin_inff()) continue;
    const float t = fmaxf(top, s), f = top == -__builtin_inff() ? 0.0f : exp2f(top - t), w = exp2f(s - t);
    top = t;
    sum = sum * f + w;
    load_row<D>(a, true, b, h, row, lane, x);
#pragma unroll
    for (int i = 0; i < kPer; ++i) o[i] = o[i] * f + w * x[i];
  }
  const bool any = sum > 0.0f || sum != sum;
  const long long at = (long long)token * a.Hq + head;
#pragma unroll
  for (int i = 0; i < kPer; ++i) {
    const float y = any ? o[i] / sum : 0.0f;
    if (a.f32) ((float*)a.out)[at * D + lane * kPer + i] = y;
    else ((__bf16*)a.out)[at * D + lane * kPer + i] = (__bf16)y;
  }
  if (a.lse && lane == 0) a.lse[at] = any ? fmaf(top, 0.6931471805599453f, logf(sum)) : -__builtin_inff();
}

hipError_t launch_attend_wave(const AttendArgs& a, const Dims& d, hipStream_t st) {
  const unsigned grid = (unsigned)a.n_tokens * a.Hq;
  if (d.D == 64) k_attend_wave<64><<<grid, 64, 0, st>>>(a);
  else if (d.D == 128) k_attend_wave<128><<<grid, 64, 0, st>>>(a);
  else k_attend_wave<256><<<grid, 64, 0, st>>>(a);
  return hipGetLastError();
}

}  // namespace ea
