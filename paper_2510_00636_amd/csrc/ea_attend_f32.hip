// Attention over fp32 caches: everything in fp32, on v_mfma_f32_16x16x4_f32.
//
// A wavefront takes 16 (token, head) rows of a KV head and 16 keys at a time.  A lane loads 16 bytes of a key (channels 16 s + 4 g ..)
// and of four values (channels 4 i ..): both products take their contraction, and the second its channels, in the order that such
// loads bring them, so nothing is staged.  Where there are rows enough for the chip, the four wavefronts of a workgroup have 16 of them
// each and walk the same keys, which come to them out of the L1 cache; else all have the same rows and every eighth (d = 256: fourth)
// 16 keys, and put their results together through LDS.  The matrix cores and the reads between their instructions bound it: 2 x 256
// tokens of 32 heads of 64 channels over 8192 rows 359 us, 94 TFLOP/s.  At d = 128 two workgroups are on a CU, by their registers: three
// take each other's keys out of the L1 cache (4 x 300 tokens of 32 heads over 2048 rows 534 us, so 429).
#include "ea_attend.h"

namespace ea {

namespace {
template <int D, bool KEYS> constexpr int f32_waves() { return KEYS && D < 256 ? 8 : 4; }
template <int D, bool KEYS> constexpr int f32_rows() { return KEYS ? kAttendF32Rows : kAttendF32LongRows; }
}  // namespace

template <int D, bool KEYS>
__global__ __launch_bounds__((64 * f32_waves<D, KEYS>()), (D == 256 ? 1 : 2)) void k_attend_f32(AttendArgs a) {
  constexpr int kSteps = D / 16, kLoads = D / 64, kM = f32_rows<D, KEYS>(), kNW = f32_waves<D, KEYS>(), kPitch = D + 4;
  extern __shared__ __attribute__((aligned(16))) float pass_o[];          // KEYS: [wavefront][row][channel], and behind it maxima and sums
  const int lane = threadIdx.x & 63, wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
  const int n16 = lane & 15, g = lane >> 4;
  const Piece piece = find_piece<kM, true>(a, blockIdx.x);
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
  const int all_see = len - (m - 1 - row0 / a.G);        // rows from here on some of the tile's tokens do not see
  bool bad = false;                                     // one of those has a value that is not finite
  const int my_rows = row0 + (KEYS ? 0 : wave * 16);
  const int row = my_rows + n16, tok = row / a.G, hd = row - tok * a.G;
  const bool in = row < rows;
  const int vis = in ? len - (m - 1 - tok) : len, vis_min = len - (m - 1 - my_rows / a.G);
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
  // the next keys are on their way from the products that took the last ones on, and so the next values
  float4 k[kSteps], v[4][kLoads];
  auto load_k = [&](int key) {
    const long long kr = (long long)min(key + n16, key_hi - 1) * D;
#pragma unroll
    for (int s = 0; s < kSteps; ++s) k[s] = *(const float4*)(kp + kr + s * 16);
  };
  auto load_v = [&](int key) {
#pragma unroll
    for (int r = 0; r < 4; ++r) {
      const long long vr = (long long)min(key + 4 * g + r, key_hi - 1) * D;
#pragma unroll
      for (int u = 0; u < kLoads; ++u) v[r][u] = *(const float4*)(vp + vr + u * 64);
    }
  };
  const int first = key_lo + (KEYS ? wave * 16 : 0), stride = KEYS ? kNW * 16 : 16;
  if (first < key_hi) {
    load_k(first);
    load_v(first);
  }
  for (int key = first; key < key_hi; key += stride) {
    const bool more = key + stride < key_hi;
    // Either block of products begins at a line of 64 bytes of the code (the first one 4 bytes behind it): where they came to stand else, by
    // what the compiler made of the lines above, moved the time by up to 7 % (520 tokens of 32 heads over 2048 rows at d = 128 333 to 357 us,
    // so 321).
    if constexpr (D < 256) {
      __builtin_amdgcn_sched_barrier(0);
      asm volatile(".p2align 6\n\ts_nop 0");
      __builtin_amdgcn_sched_barrier(0);
    }
    f32x4 s0 = (f32x4)0.0f, s1 = (f32x4)0.0f;
#pragma unroll
    for (int s = 0; s < kSteps; ++s) {
      s0 = __builtin_amdgcn_mfma_f32_16x16x4f32(k[s].x, q[s].x, s0, 0, 0, 0);
      s1 = __builtin_amdgcn_mfma_f32_16x16x4f32(k[s].y, q[s].y, s1, 0, 0, 0);
      s0 = __builtin_amdgcn_mfma_f32_16x16x4f32(k[s].z, q[s].z, s0, 0, 0, 0);
      s1 = __builtin_amdgcn_mfma_f32_16x16x4f32(k[s].w, q[s].w, s1, 0, 0, 0);
    }
    if (more) load_k(key + stride);
    __builtin_amdgcn_sched_barrier(0);
    s0 += s1;
    s0 *= a.scale;
    if (key + 16 > vis_min || key + 16 > key_hi)
#pragma unroll
      for (int r = 0; r < 4; ++r)
        if (key + 4 * g + r >= vis || key + 4 * g + r >= key_hi) s0[r] = -__builtin_inff();
    float top = fmaxf(fmaxf(s0[0], s0[1]), fmaxf(s0[2], s0[3]));
    if (__any(top > mx + kLag)) {
      top = fmaxf(max_xor16(max_xor32(top)), mx);
      const float f = mx == -__builtin_inff() ? 0.0f : pow2(mx - top);
      mx = top;
      l *= f;
#pragma unroll
      for (int c = 0; c < D / 16; ++c) o[c] *= f;
    }
    // (2^-kLag as a factor of its own: logits close to their maximum lose no bits to it)
    const float from = mx == -__builtin_inff() ? 0.0f : mx;
    float p[4];
#pragma unroll
    for (int r = 0; r < 4; ++r) {
      p[r] = pow2(s0[r] - from) * 0.00390625f;
      l += p[r];
    }
    // rows behind the last one weigh nothing, whatever they hold
    if (key + 16 > (all_see < key_hi ? all_see : key_hi))
#pragma unroll
      for (int r = 0; r < 4; ++r)
#pragma unroll
        for (int u = 0; u < kLoads; ++u) {
          const bool there = key + 4 * g + r < key_hi, some = key + 4 * g + r >= all_see;
          auto tame = [&](float& x) {
            if (there && some && not_finite(x)) bad = true;
            if (!there || (some && not_finite(x))) x = 0.0f;
          };
          tame(v[r][u].x); tame(v[r][u].y); tame(v[r][u].z); tame(v[r][u].w);
        }
    if constexpr (D < 256) asm volatile(".p2align 6");
#pragma unroll
    for (int r = 0; r < 4; ++r)
#pragma unroll
      for (int u = 0; u < kLoads; ++u) {
        o[u * 4 + 0] = __builtin_amdgcn_mfma_f32_16x16x4f32(v[r][u].x, p[r], o[u * 4 + 0], 0, 0, 0);
        o[u * 4 + 1] = __builtin_amdgcn_mfma_f32_16x16x4f32(v[r][u].y, p[r], o[u * 4 + 1], 0, 0, 0);
        o[u * 4 + 2] = __builtin_amdgcn_mfma_f32_16x16x4f32(v[r][u].z, p[r], o[u * 4 + 2], 0, 0, 0);
        o[u * 4 + 3] = __builtin_amdgcn_mfma_f32_16x16x4f32(v[r][u].w, p[r], o[u * 4 + 3], 0, 0, 0);
      }
    if (more) load_v(key + stride);
    __builtin_amdgcn_sched_barrier(0);
  }
  l = sum_xor16(sum_halves(l));
  // channel u 64 + (4 g + r) 4 + j of row n16 is o[u 4 + j][r]
  const bool whole = piece.nsplit == 1;
  bool one_bad = false;
  auto store = [&](int r, int c4, float top, float sum, float4 x) {      // four channels of a row of the tile
    const int rw = row0 + r, tk = rw / a.G;
    if (one_bad) {
      float y[4] = {x.x, x.y, x.z, x.w};
      add_not_finite<D, kKindF32>(a, b, h, max(max(all_see, key_lo), 0), min(len - (m - 1 - tk), key_hi), c4, y);
      x = make_float4(y[0], y[1], y[2], y[3]);
    }
    const bool any = sum > 0.0f || sum != sum;
    const float by = 1.0f / sum;
    const long long at = (long long)(t0 + tk) * a.Hq + h * a.G + (rw - tk * a.G), slot = (long long)blockIdx.x * kM + r;
    if (whole) {
      *(float4*)((float*)a.out + at * D + c4) = any ? make_float4(x.x * by, x.y * by, x.z * by, x.w * by) : make_float4(0, 0, 0, 0);
      if (a.lse && c4 == 0) a.lse[at] = natural_lse(top, sum);
    } else {
      *(float4*)((float*)(a.ws + a.plan.split_o) + slot * D + c4) = x;
      if (c4 == 0) ((float2*)(a.ws + a.plan.split_ml))[slot] = make_float2(top, sum);
    }
  };
  if constexpr (!KEYS) {
    one_bad = __any(bad);      // of the wavefront, whose rows are its own
    if (!in) return;
#pragma unroll
    for (int u = 0; u < kLoads; ++u)
#pragma unroll
      for (int r = 0; r < 4; ++r)
        store(row - row0, u * 64 + (4 * g + r) * 4, mx, l, make_float4(o[u * 4][r], o[u * 4 + 1][r], o[u * 4 + 2][r], o[u * 4 + 3][r]));
  } else {
    float2* pass_ml = (float2*)(pass_o + kNW * kM * kPitch);
    if (g == 0) pass_ml[wave * kM + n16] = make_float2(mx, l);
#pragma unroll
    for (int u = 0; u < kLoads; ++u)
#pragma unroll
      for (int r = 0; r < 4; ++r)
        *(float4*)(pass_o + (wave * kM + n16) * kPitch + u * 64 + (4 * g + r) * 4) =
            make_float4(o[u * 4][r], o[u * 4 + 1][r], o[u * 4 + 2][r], o[u * 4 + 3][r]);
    one_bad = __syncthreads_or(bad);
    constexpr int kLanes = D / 4;
    for (int i = threadIdx.x; i < min(kM, rows - row0) * kLanes; i += kNW * 64) {
      const int r = i / kLanes, c4 = i % kLanes * 4;
      float top = -__builtin_inff(), sum = 0.0f;
#pragma unroll
      for (int w = 0; w < kNW; ++w) top = fmaxf(top, pass_ml[w * kM + r].x);
      const float from = top == -__builtin_inff() ? 0.0f : top;
      float4 acc = make_float4(0, 0, 0, 0);
#pragma unroll
      for (int w = 0; w < kNW; ++w) {
        const float2 ml = pass_ml[w * kM + r];
        const float f = pow2(ml.x - from);
        const float4 y = *(const float4*)(pass_o + (w * kM + r) * kPitch + c4);
        sum += ml.y * f;
        acc.x += y.x * f; acc.y += y.y * f; acc.z += y.z * f; acc.w += y.w * f;
      }
      store(r, c4, top, sum, acc);
    }
  }
}

template <int D, bool KEYS>
static hipError_t f32_of_shape(const AttendArgs& a, hipStream_t st) {
  static LdsOptIn opt;
  constexpr int kNW = f32_waves<D, KEYS>(), kM = f32_rows<D, KEYS>();
  const size_t lds = KEYS ? (size_t)kNW * kM * (D + 4 + 2) * sizeof(float) : 0;
  hipError_t e = opt.ensure((const void*)k_attend_f32<D, KEYS>, lds);
  if (e != hipSuccess) return e;
  k_attend_f32<D, KEYS><<<(unsigned)a.plan.grid, kNW * 64, lds, st>>>(a);
  e = hipGetLastError();
  return e != hipSuccess || a.plan.most_pieces == 0 ? e : launch_attend_join(a, true, st);
}

hipError_t launch_attend_f32(const AttendArgs& a, hipStream_t st) {
#define EA_CASE(DD) if (a.D == DD) return a.plan.tile_rows == kAttendF32Rows ? f32_of_shape<DD, true>(a, st) : f32_of_shape<DD, false>(a, st)
  EA_CASE(64);
  EA_CASE(128);
#undef EA_CASE
  return a.plan.tile_rows == kAttendF32Rows ? f32_of_shape<256, true>(a, st) : f32_of_shape<256, false>(a, st);
}

}  // namespace ea
