// Attention of drafted trees over fp32 caches: the kernel of ea_attend_f32.hip, where which of its sequence's new rows a token sees is a mask.
// Masks are read where a tile reaches the step's own rows; 4 trees of 12 tokens of 18 heads over 40k rows 297 us, 1 GB at 3.4 TB/s, 61
// TFLOP/s.
//
// A kernel of its own because of registers: as one with that of steps without masks, whose lanes have one row, it left that one 158 of them at
// d = 128, which let three workgroups on a CU and put addresses into the registers that their loads write (4 x 300 tokens of 32 heads
// over 2048 rows without masks 534 us, so 429).
#include "ea_attend.h"

namespace ea {

namespace {
template <int D, bool KEYS, int MT> constexpr int f32_waves() { return KEYS && D < 256 && MT == 1 ? 8 : 4; }
template <bool KEYS, int MT> constexpr int f32_rows() { return KEYS ? kAttendF32Rows * MT : kAttendF32LongRows; }
}  // namespace

// MT > 1: a wavefront has MT times 16 rows, for which the keys are read once (four at d = 64 and 128; at d = 256 registers hold two).
template <int D, bool KEYS, int MT>
__global__ __launch_bounds__((64 * f32_waves<D, KEYS, MT>()), (D == 256 || (D == 128 && MT > 1) ? 1 : 2)) void k_attend_f32_tree(AttendArgs a) {
  constexpr int kSteps = D / 16, kLoads = D / 64, kM = f32_rows<KEYS, MT>(), kNW = f32_waves<D, KEYS, MT>(), kPitch = D + 4;
  extern __shared__ __attribute__((aligned(16))) float pass_o[];          // KEYS: [wavefront][row][channel], and behind it maxima and sums
  const int lane = threadIdx.x & 63, wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
  const int n16 = lane & 15, g = lane >> 4;
  const Piece piece = find_piece<kM, true, 1, true>(a, blockIdx.x);
  if (piece.tile < 0) return;
  note_cuts<true>(a, piece, blockIdx.x);
  const int b = piece.b, h = piece.h, t0 = piece.t0, m = piece.m, rows = m * a.G, row0 = piece.tile * kM;
  const int len = rows_of(a, b, h);
  const int new_rows = len - m;                          // where the step's own begin
  int key_hi = len;
  const int key_lo = piece.split * piece.chunk;
  if (piece.nsplit > 1) {
    if (key_lo >= key_hi) return;
    key_hi = min(key_hi, key_lo + piece.chunk);
  }
  bool bad = false;                                     // one of those has a value that is not finite
  const int my_rows = row0 + (KEYS ? 0 : wave * 16);
  const int live = MT > 1 ? min((rows - row0 + 15) >> 4, MT) : 1;        // sixteens of rows that there are
  int row[MT], tok[MT], hd[MT];
  bool in[MT];
#pragma unroll
  for (int t = 0; t < MT; ++t) {
    row[t] = my_rows + t * 16 + n16;
    tok[t] = row[t] / a.G;
    hd[t] = row[t] - tok[t] * a.G;
    in[t] = row[t] < rows;
  }
  // bits of the mask of token `of` from the one of row `key` on
  auto seen_from = [&](int of, int key) -> uint64_t {
    const uint64_t* mask = a.sees + (long long)(t0 + of) * a.words;
    auto word = [&](int w) -> uint64_t {
      const int left = m - 64 * w;
      const uint64_t x = w < a.words && left > 0 ? mask[w] : 0;
      return left >= 64 || left <= 0 ? x : x & ((1ull << left) - 1);
    };
    const int from = key - new_rows, w = from >> 6, shift = from & 63;
    if (from < 0) return from <= -64 ? ~0ull : word(0) << (-from & 63) | ((1ull << (-from & 63)) - 1);
    return word(w) >> shift | (shift > 0 ? word(w + 1) << (64 - shift) : 0);
  };
  float4 q[MT][kSteps];
#pragma unroll
  for (int t = 0; t < MT; ++t) {
    const float* src = (const float*)a.q + (long long)(t0 + (in[t] ? tok[t] : 0)) * a.q_stride + (h * a.G + (in[t] ? hd[t] : 0)) * D;
#pragma unroll
    for (int s = 0; s < kSteps; ++s) {
      const float4 w = *(const float4*)(src + s * 16 + g * 4);
      q[t][s] = in[t] ? w : make_float4(0, 0, 0, 0);
    }
  }
  const long long head = ((long long)b * a.Hkv + h) * a.n_cap;
  const float* kp = (const float*)a.k + head * D + g * 4;
  const float* vp = (const float*)a.v + head * D + n16 * 4;
  f32x4 o[MT][D / 16];
  float mx[MT], l[MT];
#pragma unroll
  for (int t = 0; t < MT; ++t) {
#pragma unroll
    for (int c = 0; c < D / 16; ++c) o[t][c] = (f32x4)0.0f;
    mx[t] = -__builtin_inff();
    l[t] = 0.0f;
  }
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
    f32x4 s[MT];
#pragma unroll
    for (int t = 0; t < MT; ++t) {
      if (MT > 1 && t >= live) break;
      f32x4 s0 = (f32x4)0.0f, s1 = (f32x4)0.0f;
#pragma unroll
      for (int c = 0; c < kSteps; ++c) {
        s0 = __builtin_amdgcn_mfma_f32_16x16x4f32(k[c].x, q[t][c].x, s0, 0, 0, 0);
        s1 = __builtin_amdgcn_mfma_f32_16x16x4f32(k[c].y, q[t][c].y, s1, 0, 0, 0);
        s0 = __builtin_amdgcn_mfma_f32_16x16x4f32(k[c].z, q[t][c].z, s0, 0, 0, 0);
        s1 = __builtin_amdgcn_mfma_f32_16x16x4f32(k[c].w, q[t][c].w, s1, 0, 0, 0);
      }
      s[t] = s0 + s1;
    }
    if (more) load_k(key + stride);
    __builtin_amdgcn_sched_barrier(0);
    float p[MT][4];
#pragma unroll
    for (int t = 0; t < MT; ++t) {
      if (MT > 1 && t >= live) break;
      f32x4& s0 = s[t];
      s0 *= a.scale;
      if (key + 16 > new_rows || key + 16 > key_hi) {
        const uint32_t bits = key < key_hi ? (uint32_t)seen_from(in[t] ? tok[t] : 0, key) & (key + 16 > key_hi ? (1u << (key_hi - key)) - 1 : 0xffffu) : 0;
#pragma unroll
        for (int r = 0; r < 4; ++r) s0[r] = bits >> (4 * g + r) & 1 ? s0[r] : -__builtin_inff();
      }
      float top = fmaxf(fmaxf(s0[0], s0[1]), fmaxf(s0[2], s0[3]));
      if (__any(top > mx[t] + kLag)) {
        top = fmaxf(max_xor16(max_xor32(top)), mx[t]);
        const float f = mx[t] == -__builtin_inff() ? 0.0f : pow2(mx[t] - top);
        mx[t] = top;
        l[t] *= f;
#pragma unroll
        for (int c = 0; c < D / 16; ++c) o[t][c] *= f;
      }
      // (2^-kLag as a factor of its own: logits close to their maximum lose no bits to it)
      const float from = mx[t] == -__builtin_inff() ? 0.0f : mx[t];
#pragma unroll
      for (int r = 0; r < 4; ++r) {
        p[t][r] = pow2(s0[r] - from) * 0.00390625f;
        l[t] += p[t][r];
      }
    }
    // rows behind the last one weigh nothing, whatever they hold
    if (key + 16 > (new_rows < key_hi ? new_rows : key_hi))
#pragma unroll
      for (int r = 0; r < 4; ++r)
#pragma unroll
        for (int u = 0; u < kLoads; ++u) {
          const bool there = key + 4 * g + r < key_hi, some = key + 4 * g + r >= new_rows;
          auto tame = [&](float& x) {
            if (there && some && not_finite(x)) bad = true;
            if (!there || (some && not_finite(x))) x = 0.0f;
          };
          tame(v[r][u].x); tame(v[r][u].y); tame(v[r][u].z); tame(v[r][u].w);
        }
#pragma unroll
    for (int t = 0; t < MT; ++t) {
      if (MT > 1 && t >= live) break;
#pragma unroll
      for (int r = 0; r < 4; ++r)
#pragma unroll
        for (int u = 0; u < kLoads; ++u) {
          f32x4* acc = &o[t][u * 4];
          acc[0] = __builtin_amdgcn_mfma_f32_16x16x4f32(v[r][u].x, p[t][r], acc[0], 0, 0, 0);
          acc[1] = __builtin_amdgcn_mfma_f32_16x16x4f32(v[r][u].y, p[t][r], acc[1], 0, 0, 0);
          acc[2] = __builtin_amdgcn_mfma_f32_16x16x4f32(v[r][u].z, p[t][r], acc[2], 0, 0, 0);
          acc[3] = __builtin_amdgcn_mfma_f32_16x16x4f32(v[r][u].w, p[t][r], acc[3], 0, 0, 0);
        }
    }
    if (more) load_v(key + stride);
    __builtin_amdgcn_sched_barrier(0);
  }
#pragma unroll
  for (int t = 0; t < MT; ++t) l[t] = sum_xor16(sum_halves(l[t]));
  // channel u 64 + (4 g + r) 4 + j of row n16 is o[u 4 + j][r]
  const bool whole = piece.nsplit == 1;
  bool one_bad = false;
  auto store = [&](int r, int c4, float top, float sum, float4 x) {      // four channels of a row of the tile
    const int rw = row0 + r, tk = rw / a.G;
    if (one_bad) {
      float y[4] = {x.x, x.y, x.z, x.w};
      const int lo = max(max(new_rows, key_lo), 0);
      add_not_finite<D, kKindF32>(a, b, h, lo, key_hi, c4, y, [&](int key) { return seen_from(tk, key) & 1; });
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
    if (!in[0]) return;
#pragma unroll
    for (int u = 0; u < kLoads; ++u)
#pragma unroll
      for (int r = 0; r < 4; ++r)
        store(row[0] - row0, u * 64 + (4 * g + r) * 4, mx[0], l[0], make_float4(o[0][u * 4][r], o[0][u * 4 + 1][r], o[0][u * 4 + 2][r], o[0][u * 4 + 3][r]));
  } else {
    float2* pass_ml = (float2*)(pass_o + kNW * 16 * kPitch);
#pragma unroll
    for (int t = 0; t < MT; ++t) {      // sixteen rows at a time
      if (MT > 1 && t >= live) break;
      if (t > 0) __syncthreads();
      if (g == 0) pass_ml[wave * 16 + n16] = make_float2(mx[t], l[t]);
#pragma unroll
      for (int u = 0; u < kLoads; ++u)
#pragma unroll
        for (int r = 0; r < 4; ++r)
          *(float4*)(pass_o + (wave * 16 + n16) * kPitch + u * 64 + (4 * g + r) * 4) =
              make_float4(o[t][u * 4][r], o[t][u * 4 + 1][r], o[t][u * 4 + 2][r], o[t][u * 4 + 3][r]);
      one_bad = __syncthreads_or(bad);
      constexpr int kLanes = D / 4;
      for (int i = threadIdx.x; i < min(16, rows - row0 - t * 16) * kLanes; i += kNW * 64) {
        const int r = i / kLanes, c4 = i % kLanes * 4;
        float top = -__builtin_inff(), sum = 0.0f;
#pragma unroll
        for (int w = 0; w < kNW; ++w) top = fmaxf(top, pass_ml[w * 16 + r].x);
        const float from = top == -__builtin_inff() ? 0.0f : top;
        float4 acc = make_float4(0, 0, 0, 0);
#pragma unroll
        for (int w = 0; w < kNW; ++w) {
          const float2 ml = pass_ml[w * 16 + r];
          const float f = pow2(ml.x - from);
          const float4 y = *(const float4*)(pass_o + (w * 16 + r) * kPitch + c4);
          sum += ml.y * f;
          acc.x += y.x * f; acc.y += y.y * f; acc.z += y.z * f; acc.w += y.w * f;
        }
        store(t * 16 + r, c4, top, sum, acc);
      }
    }
  }
}

template <int D, bool KEYS, int MT = 1>
static hipError_t f32_of_shape(const AttendArgs& a, hipStream_t st) {
  static LdsOptIn opt;
  constexpr int kNW = f32_waves<D, KEYS, MT>();
  const size_t lds = KEYS ? (size_t)kNW * 16 * (D + 4 + 2) * sizeof(float) : 0;
  hipError_t e = opt.ensure((const void*)k_attend_f32_tree<D, KEYS, MT>, lds);
  if (e != hipSuccess) return e;
  k_attend_f32_tree<D, KEYS, MT><<<(unsigned)a.plan.grid, kNW * 64, lds, st>>>(a);
  e = hipGetLastError();
  return e != hipSuccess || a.plan.most_pieces == 0 ? e : launch_attend_join(a, true, st);
}
template <int D>
static hipError_t f32_of_size(const AttendArgs& a, hipStream_t st) {
  if (!a.plan.keys) return f32_of_shape<D, false>(a, st);
  return a.plan.tile_rows == kAttendF32Rows ? f32_of_shape<D, true>(a, st) : f32_of_shape<D, true, D == 256 ? 2 : 4>(a, st);
}

hipError_t launch_attend_f32_tree(const AttendArgs& a, hipStream_t st) {
  return a.D == 64 ? f32_of_size<64>(a, st) : a.D == 128 ? f32_of_size<128>(a, st) : f32_of_size<256>(a, st);
}

}  // namespace ea
