// Rows into MX pools and back: quantised as they are written, read back as bf16 tensors.
//
// Both are copies: 8192 tokens of 8 heads of 128 channels in 4 bits are written in 41 us (their bytes at a copy's 4.89 TB/s take 38) and
// read back in 10, 131k rows of 8 bits are read back in 157 us (166).  The rotation's fp64 hides under the copy; one token of each of 48
// sequences takes 3.9 us, one launch.
#include "ea_mx.h"

namespace ea {

namespace {

// largest of |x| over this lane and its neighbours 1 (and 2, 3 where FOUR) of a group of four lanes
template <bool FOUR>
__device__ __forceinline__ float max_of_group(float x) {
  x = fmaxf(x, __int_as_float(__builtin_amdgcn_update_dpp(0, __float_as_int(x), 0xB1, 0xf, 0xf, true)));
  if (FOUR) x = fmaxf(x, __int_as_float(__builtin_amdgcn_update_dpp(0, __float_as_int(x), 0x4E, 0xf, 0xf, true)));
  return x;
}

// The exponent byte of a group whose largest |x| is top (finite): the least e >= 10 with top <= most * 2^(e - 127), most being
// 1.75 * 2^8 (e4m3) or 1.5 * 2^2 (e2m1), from the bits of top.  Below 2^-117 nothing is resolved, so that no element stands for
// a number below 2^-126.
template <int BITS>
__device__ __forceinline__ int group_exponent(float top) {
  const uint32_t w = __float_as_uint(top), frac = w & 0x7fffff;
  const int e = (int)(w >> 23) - (BITS == 8 ? 8 : 2) + (frac > (BITS == 8 ? 0x600000u : 0x400000u) ? 1 : 0);
  return e < 10 ? 10 : e;
}
// the largest element of a group with exponent byte e: the format's, but where that would stand for more than bf16's largest number
template <int BITS>
__device__ __forceinline__ float largest_element(int e) {
  if (BITS == 8) return e == 247 ? 240.0f : 448.0f;
  return e == 253 ? 3.0f : 6.0f;
}

}  // namespace

// A workgroup takes 256 stretches of one token's rows, as k_append does; here angles, and the keys' rotation, are fp64, so that what is
// quantised is the exact key rounded once to fp32.  A lane has eight channels of either half of a head (or sixteen next to each other), so
// the largest of 32 comes from four lanes (two) by row moves without LDS, and elements leave by the instructions that convert pairs,
// which round to nearest even.  (Rows asked for in front of the angles: 51 registers and not 41, and no faster.)
template <int D, int BITS>
__global__ __launch_bounds__(256) void k_append_mx(MxAppendArgs a) {
  __shared__ double2 turn[D / 2];
  const int tid = threadIdx.x, token = a.first + blockIdx.x;
  const long long slot = a.slots[token];
  if (slot < 0 || slot >= (a.num_blocks << a.sh)) return;
  const long long blk = slot >> a.sh;
  const int off = (int)(slot & ((1 << a.sh) - 1));
  if (a.inv_freq) {
    for (int c = tid; c < D / 2; c += 256) {
#pragma clang fp contract(off)
      // the fp64 angle in half turns, whole turns taken out, with what its product with 1 / pi rounded away
      const double angle = (double)a.pos[token] * a.inv_freq[c], inv_pi = 0.31830988618379067154, inv_pi_lo = -1.9678676675182485e-17;
      const double turns = angle * inv_pi, whole = 2.0 * rint(0.5 * turns);
      const double rest = (turns - whole) + fma(angle, inv_pi_lo, fma(angle, inv_pi, -turns));
      double si, co;
      sincospi(rest, &si, &co);
      turn[c] = make_double2(co, si);
    }
    __syncthreads();
  }
  constexpr int kPieces = D / 16;                      // of 8 channel pairs in a head: four or more lanes next to each other
  const int q_heads = a.q ? a.Hq : 0, heads = q_heads + 2 * a.Hkv;
  for (int it = blockIdx.y * 256 + tid; it < heads * kPieces; it += gridDim.y * 256) {
    const int head = it / kPieces, c = it % kPieces;
    const bool is_q = head < q_heads, is_v = head >= q_heads + a.Hkv;
    const int h = is_q ? head : is_v ? head - q_heads - a.Hkv : head - q_heads;
    const __bf16* src = is_q ? (const __bf16*)a.q + token * a.q_stride : is_v ? (const __bf16*)a.v + token * a.v_stride : (const __bf16*)a.k + token * a.k_stride;
    const int c0 = a.rope_layout ? c * 16 : c * 8, c1 = a.rope_layout ? c0 + 8 : c0 + D / 2;
    const uint4 w0 = *(const uint4*)(src + h * D + c0), w1 = *(const uint4*)(src + h * D + c1);
    const uint32_t w[8] = {w0.x, w0.y, w0.z, w0.w, w1.x, w1.y, w1.z, w1.w};
    float x[16];
#pragma unroll
    for (int i = 0; i < 8; ++i) {
      x[2 * i] = __uint_as_float(w[i] << 16);
      x[2 * i + 1] = __uint_as_float(w[i] & 0xffff0000u);
    }
    if (a.inv_freq && !is_v) {
      const double2* t = &turn[c * 8];
#pragma unroll
      for (int i = 0; i < 8; ++i) {
        const int lo = a.rope_layout ? 2 * i : i, hi = a.rope_layout ? 2 * i + 1 : i + 8;
        const double p = x[lo], r = x[hi];
        x[lo] = (float)fma(p, t[i].x, -r * t[i].y);
        x[hi] = (float)fma(p, t[i].y, r * t[i].x);
      }
    }
    if (is_q) {
      typedef __bf16 pair __attribute__((ext_vector_type(2)));
      uint32_t o[8];
#pragma unroll
      for (int i = 0; i < 8; ++i) {
        const pair p = {(__bf16)x[2 * i], (__bf16)x[2 * i + 1]};
        o[i] = __builtin_bit_cast(uint32_t, p);
      }
      __bf16* dst = (__bf16*)a.q_out + ((long long)token * a.Hq + h) * D;
      *(uint4*)(dst + c0) = make_uint4(o[0], o[1], o[2], o[3]);
      *(uint4*)(dst + c1) = make_uint4(o[4], o[5], o[6], o[7]);
      continue;
    }
    // ---- the largest of each half's group, which a number that is not finite makes infinite
    float top[2];
#pragma unroll
    for (int s = 0; s < 2; ++s) {
      top[s] = 0.0f;
#pragma unroll
      for (int i = 0; i < 8; ++i) {
        const float y = fabsf(x[8 * s + i]);
        top[s] = fmaxf(top[s], y == y ? y : __builtin_inff());
      }
    }
    if (a.rope_layout) top[0] = top[1] = max_of_group<false>(fmaxf(top[0], top[1]));
    else top[0] = max_of_group<true>(top[0]), top[1] = max_of_group<true>(top[1]);
    const long long row = ((blk * a.Hkv + h) << a.sh) + off;
    uint8_t* dst = (uint8_t*)(is_v ? a.v_pool : a.k_pool) + row * (D * BITS / 8);
    uint8_t* scales = (is_v ? a.v_scale : a.k_scale) + row * (D / 32);
#pragma unroll
    for (int s = 0; s < 2; ++s) {
      const int at = s ? c1 : c0, e = group_exponent<BITS>(top[s]);
      const bool finite = top[s] < __builtin_inff();
      const float by = __uint_as_float((uint32_t)(254 - e) << 23), most = largest_element<BITS>(e);      // 2^(127 - e), 127 - e >= -126
      float y[8];
#pragma unroll
      for (int i = 0; i < 8; ++i) y[i] = finite ? fminf(fmaxf(x[8 * s + i] * by, -most), most) : 0.0f;
      if constexpr (BITS == 8) {
        int lo = __builtin_amdgcn_cvt_pk_fp8_f32(y[0], y[1], 0, false), hi = __builtin_amdgcn_cvt_pk_fp8_f32(y[4], y[5], 0, false);
        lo = __builtin_amdgcn_cvt_pk_fp8_f32(y[2], y[3], lo, true);
        hi = __builtin_amdgcn_cvt_pk_fp8_f32(y[6], y[7], hi, true);
        *(uint2*)(dst + at) = make_uint2((uint32_t)lo, (uint32_t)hi);
      } else {
        uint32_t o = __builtin_amdgcn_cvt_scalef32_pk_fp4_f32(0, y[0], y[1], 1.0f, 0);
        o = __builtin_amdgcn_cvt_scalef32_pk_fp4_f32(o, y[2], y[3], 1.0f, 1);
        o = __builtin_amdgcn_cvt_scalef32_pk_fp4_f32(o, y[4], y[5], 1.0f, 2);
        o = __builtin_amdgcn_cvt_scalef32_pk_fp4_f32(o, y[6], y[7], 1.0f, 3);
        *(uint32_t*)(dst + at / 2) = o;
      }
      if (at % 32 == 0) scales[at / 32] = (uint8_t)(finite ? e : 255);
    }
  }
}

hipError_t launch_append_mx(const MxAppendArgs& given, const Dims& d, hipStream_t st) {
  MxAppendArgs a = given;
  const int items = ((a.q ? a.Hq : 0) + 2 * a.Hkv) * (d.D / 16);
  constexpr int kMost = 1 << 23;      // (2^32 threads to a launch)
  for (a.first = 0; a.first < a.n_tokens; a.first += kMost) {
    const dim3 grid(a.n_tokens - a.first < kMost ? a.n_tokens - a.first : kMost, items < 65535 * 256 ? (items + 255) / 256 : 65535);
#define EA_CASE(DD)                                                       \
    if (d.D == DD) {                                                        \
      if (a.bits == 8) k_append_mx<DD, 8><<<grid, 256, 0, st>>>(a);           \
      else k_append_mx<DD, 4><<<grid, 256, 0, st>>>(a);                       \
    }
    EA_CASE(64) EA_CASE(128) EA_CASE(256)
#undef EA_CASE
    const hipError_t e = hipGetLastError();
    if (e != hipSuccess) return e;
  }
  return hipSuccess;
}

// A lane reads eight channels of a row back and writes 16 bytes: the conversion takes the scale along and is exact.  A workgroup has
// stretches of a head's rows, one after the other; a lane asks for its four rows of one together (one by one: 131k rows 164 us, so 157).
// Those behind the head's length are asked for as the last one and not written.
namespace {
template <int D> constexpr int read_rows() { return 256 * 4 / (D / 8); }
}
template <int D, int BITS>
__global__ __launch_bounds__(256) void k_read_mx(MxReadArgs a) {
  constexpr int kLanes = D / 8, kRows = read_rows<D>();
  const int stretches = (a.n + kRows - 1) / kRows;
  const long long total = (long long)a.B * a.Hkv * stretches;
  for (long long w = blockIdx.x; w < total; w += gridDim.x) {
    const int unit = (int)(w / stretches), row0 = (int)(w - (long long)unit * stretches) * kRows, b = unit / a.Hkv, h = unit - b * a.Hkv;
    const int len = min(a.lens[b], a.n);
    if (row0 >= len) continue;
    // a lane's rows together: their blocks, their elements and scales, and then what they stand for
    constexpr int kPer = kRows * kLanes / 256;
    const int r0 = row0 + threadIdx.x / kLanes, c = threadIdx.x % kLanes * 8;
    long long from[kPer];
#pragma unroll
    for (int i = 0; i < kPer; ++i) {
      const int row = min(r0 + i * (256 / kLanes), len - 1);
      from[i] = a.pm.table[(long long)b * a.pm.max_blocks + (row >> a.pm.sh)];
    }
#pragma unroll
    for (int i = 0; i < kPer; ++i) {
      const int row = min(r0 + i * (256 / kLanes), len - 1);
      const long long blk = from[i] < 0 ? 0 : from[i] < a.pm.num_blocks ? from[i] : a.pm.num_blocks - 1;
      from[i] = ((blk * a.Hkv + h) << a.pm.sh) + (row & ((1 << a.pm.sh) - 1));
    }
#pragma unroll
    for (int s = 0; s < 2; ++s) {
      __bf16* out = (__bf16*)(s ? a.v_out : a.k_out);
      if (!out) continue;
      const char* pool = (const char*)(s ? a.v : a.k);
      const uint8_t* scales = s ? a.v_scale : a.k_scale;
      uint2 x[kPer];
      uint32_t e[kPer];
#pragma unroll
      for (int i = 0; i < kPer; ++i) {
        e[i] = scales[from[i] * (D / 32) + c / 32];
        if constexpr (BITS == 8) x[i] = *(const uint2*)(pool + from[i] * D + c);
        else x[i].x = *(const uint32_t*)(pool + (from[i] * D + c) / 2);
      }
#pragma unroll
      for (int i = 0; i < kPer; ++i) {
        const int row = r0 + i * (256 / kLanes);
        if (row >= len) continue;
        const long long to = ((long long)unit * a.n_cap + row) * D + c;
        if constexpr (BITS == 8) *(uint4*)(out + to) = widen_mx8(x[i], mx_scale(e[i]));
        else *(uint4*)(out + to) = widen_mx4(x[i].x, mx_scale(e[i]));
      }
    }
  }
}

template <int D, int BITS>
static hipError_t read_of_type(const MxReadArgs& a, hipStream_t st) {
  const long long total = (long long)a.B * a.Hkv * ((a.n + read_rows<D>() - 1) / read_rows<D>());
  k_read_mx<D, BITS><<<(unsigned)(total < 8192 ? total : 8192), 256, 0, st>>>(a);
  return hipGetLastError();
}
hipError_t launch_read_mx(const MxReadArgs& a, const Dims& d, hipStream_t st) {
#define EA_CASE(DD) if (d.D == DD) return a.bits == 8 ? read_of_type<DD, 8>(a, st) : read_of_type<DD, 4>(a, st)
  EA_CASE(64);
  EA_CASE(128);
#undef EA_CASE
  return a.bits == 8 ? read_of_type<256, 8>(a, st) : read_of_type<256, 4>(a, st);
}

}  // namespace ea
