// Attention over fp32 caches: everything in fp32, on v_mfma_f32_16x16x4_f32.
//
// A workgroup takes 16 (token, head) rows of a KV head, its four wavefronts every fourth 16 keys.  A lane loads 16 bytes of a key
// (channels 16 s + 4 g ..) and of four values (channels 4 i ..): both products take their contraction, and the second its
// channels, in the order that such loads bring them, so nothing is staged.
#include "ea_attend.h"

namespace ea {

template <int D>
__global__ __launch_bounds__(256, (D == 256 ? 1 : 2)) void k_attend_f32(AttendArgs a) {
  constexpr int kSteps = D / 16, kLoads = D / 64, kM = kAttendF32Rows;
  __shared__ float pass_o[2][D / 4][64];
  __shared__ float pass_ml[4][2][kM];
  const int lane = threadIdx.x & 63, wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
  const int n16 = lane & 15, g = lane >> 4;
  const Piece piece = find_piece<kM>(a, blockIdx.x);
  if (piece.tile < 0) return;
  note_cuts(a, piece, blockIdx.x);
  const int b = piece.b, h = piece.h, t0 = piece.t0, m = piece.m, rows = m * a.G, row0 = piece.tile * kM;
  const int len = rows_of(a, b, h);
  int key_hi = len - (m - 1 - (min(row0 + kM, rows) - 1) / a.G);
  key_hi = key_hi < 0 ? 0 : key_hi;
  const int key_lo = piece.split * piece.chunk;
  if (piece.nsplit > 1) {
    if (key_lo >= key_hi) return;
    key_hi = min(key_hi, key_lo + piece.chunk);
  }
  const int row = row0 + n16, tok = row / a.G, hd = row - tok * a.G;
  const bool in = row < rows;
  const int vis = in ? len - (m - 1 - tok) : len, vis_min = len - (m - 1 - row0 / a.G);
  float4 q[kSteps];
  {
    const float* src = (const float*)a.q + (long long)(t0 + (in ? tok : 0)) * a.q_stride + (h * a.G + (in ? hd : 0)) * D;
#pragma unroll
    for (int s = 0; s < kSteps; ++s) {
      const float4 w = *(const float4*)(src + s * 16 + g * 4);
      q[s] = in ? w : make_float4(0, 0, 0, 0);
    }
  }
  const long long head = ((long long)b * a.Hkv + h) * a.n_cap;
  const float* kp = (const float*)a.k + head * D + g * 4;
  const float* vp = (const float*)a.v + head * D + n16 * 4;
  f32x4 o[D / 16];
#pragma unroll
  for (int c = 0; c < D / 16; ++c) o[c] = (f32x4)0.0f;
  float mx = -__builtin_inff(), l = 0.0f;
  for (int key = key_lo + wave * 16; key < key_hi; key += 64) {
    float4 k[kSteps], v[4][kLoads];
    const long long kr = (long long)min(key + n16, key_hi - 1) * D;
#pragma unroll
    for (int s = 0; s < kSteps; ++s) k[s] = *(const float4*)(kp + kr + s * 16);
#pragma unroll
    for (int r = 0; r < 4; ++r) {
      const int vk = key + 4 * g + r;
      const long long vr = (long long)min(vk, key_hi - 1) * D;
#pragma unroll
      for (int u = 0; u < kLoads; ++u) {
        v[r][u] = *(const float4*)(vp + vr + u * 64);
        if (vk >= key_hi) v[r][u] = make_float4(0, 0, 0, 0);
      }
    }
    f32x4 s0 = (f32x4)0.0f, s1 = (f32x4)0.0f;
#pragma unroll
    for (int s = 0; s < kSteps; ++s) {
      s0 = __builtin_amdgcn_mfma_f32_16x16x4f32(k[s].x, q[s].x, s0, 0, 0, 0);
      s1 = __builtin_amdgcn_mfma_f32_16x16x4f32(k[s].y, q[s].y, s1, 0, 0, 0);
      s0 = __builtin_amdgcn_mfma_f32_16x16x4f32(k[s].z, q[s].z, s0, 0, 0, 0);
      s1 = __builtin_amdgcn_mfma_f32_16x16x4f32(k[s].w, q[s].w, s1, 0, 0, 0);
    }
    s0 += s1;
    s0 *= a.scale;
    if (key + 16 > vis_min || key + 16 > key_hi)
#pragma unroll
      for (int r = 0; r < 4; ++r)
        if (key + 4 * g + r >= vis || key + 4 * g + r >= key_hi) s0[r] = -__builtin_inff();
    float top = fmaxf(fmaxf(s0[0], s0[1]), fmaxf(s0[2], s0[3]));
    if (__any(top > mx + 8.0f)) {
      top = fmaxf(max_xor16(max_xor32(top)), mx);
      const float f = mx == -__builtin_inff() ? 0.0f : pow2(mx - top);
      mx = top;
      l *= f;
#pragma unroll
      for (int c = 0; c < D / 16; ++c) o[c] *= f;
    }
    const float from = mx == -__builtin_inff() ? 0.0f : mx;
    float p[4];
#pragma unroll
    for (int r = 0; r < 4; ++r) {
      p[r] = pow2(s0[r] - from);
      l += p[r];
    }
#pragma unroll
    for (int r = 0; r < 4; ++r)
#pragma unroll
      for (int u = 0; u < kLoads; ++u) {
        o[u * 4 + 0] = __builtin_amdgcn_mfma_f32_16x16x4f32(v[r][u].x, p[r], o[u * 4 + 0], 0, 0, 0);
        o[u * 4 + 1] = __builtin_amdgcn_mfma_f32_16x16x4f32(v[r][u].y, p[r], o[u * 4 + 1], 0, 0, 0);
        o[u * 4 + 2] = __builtin_amdgcn_mfma_f32_16x16x4f32(v[r][u].z, p[r], o[u * 4 + 2], 0, 0, 0);
        o[u * 4 + 3] = __builtin_amdgcn_mfma_f32_16x16x4f32(v[r][u].w, p[r], o[u * 4 + 3], 0, 0, 0);
      }
  }
  // ---- the four wavefronts' results, as in the row kernel
  l = sum_xor16(sum_halves(l));
  if (g == 0) {
    pass_ml[wave][0][n16] = mx;
    pass_ml[wave][1][n16] = l;
  }
  __syncthreads();
  const float top = fmaxf(fmaxf(pass_ml[0][0][n16], pass_ml[1][0][n16]), fmaxf(pass_ml[2][0][n16], pass_ml[3][0][n16]));
  const float from = top == -__builtin_inff() ? 0.0f : top;
  float sum = 0.0f;
#pragma unroll
  for (int w = 0; w < 4; ++w) sum += pass_ml[w][1][n16] * pow2(pass_ml[w][0][n16] - from);
  const float f = pow2(mx - from);
#pragma unroll
  for (int c = 0; c < D / 16; ++c) o[c] *= f;
  if (wave >= 2)
#pragma unroll
    for (int c = 0; c < D / 16; ++c)
#pragma unroll
      for (int r = 0; r < 4; ++r) pass_o[wave - 2][c * 4 + r][lane] = o[c][r];
  __syncthreads();
  if (wave < 2)
#pragma unroll
    for (int c = 0; c < D / 16; ++c)
#pragma unroll
      for (int r = 0; r < 4; ++r) {
        o[c][r] += pass_o[wave][c * 4 + r][lane];
        if (wave == 1) pass_o[1][c * 4 + r][lane] = o[c][r];
      }
  __syncthreads();
  if (wave != 0 || !in) return;
  const long long at = (long long)(t0 + tok) * a.Hq + h * a.G + hd;
  const long long slot = (long long)blockIdx.x * kM + n16;
  const bool whole = piece.nsplit == 1, any = sum > 0.0f || sum != sum;
  float* dst = whole ? (float*)a.out + at * D : (float*)(a.ws + a.plan.split_o) + slot * D;
  const float by = !whole ? 1.0f : 1.0f / sum;
  // channel u 64 + (4 g + r) 4 + j of row n16 is o[u 4 + j][r]
#pragma unroll
  for (int u = 0; u < kLoads; ++u)
#pragma unroll
    for (int r = 0; r < 4; ++r) {
      float4 x = make_float4(0, 0, 0, 0);
      const int c = u * 4;
      if (!whole || any)
        x = make_float4((o[c][r] + pass_o[1][c * 4 + r][lane]) * by, (o[c + 1][r] + pass_o[1][c * 4 + 4 + r][lane]) * by,
                        (o[c + 2][r] + pass_o[1][c * 4 + 8 + r][lane]) * by, (o[c + 3][r] + pass_o[1][c * 4 + 12 + r][lane]) * by);
      *(float4*)(dst + u * 64 + (4 * g + r) * 4) = x;
    }
  if (g == 0) {
    if (!whole) ((float2*)(a.ws + a.plan.split_ml))[slot] = make_float2(top, sum);
    else if (a.lse) a.lse[at] = natural_lse(top, sum);
  }
}

hipError_t launch_attend_f32(const AttendArgs& a, hipStream_t st) {
  const unsigned grid = (unsigned)a.plan.grid;
  if (a.D == 64) k_attend_f32<64><<<grid, 256, 0, st>>>(a);
  else if (a.D == 128) k_attend_f32<128><<<grid, 256, 0, st>>>(a);
  else k_attend_f32<256><<<grid, 256, 0, st>>>(a);
  const hipError_t e = hipGetLastError();
  return e != hipSuccess || a.plan.most_pieces == 0 ? e : launch_attend_join(a, true, st);
}

}  // namespace ea
