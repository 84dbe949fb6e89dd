// What a model's step does to its cache before attention: the blocks that its tokens need, and their rows.
#include <hip/hip_runtime.h>

#include <type_traits>

#include "ea_lanes.h"
#include "ea_step.h"

namespace ea {

// ------------------------------------------------------------------------------- block tables
// Everything follows from the lengths: prefix sums of the blocks wanted, the blocks given back and the tokens, which every
// workgroup makes for itself (48 KiB of LDS for the largest batch), so that none waits for another.  The i-th block taken is
// the i-th one given back, or else comes off the list's end; one given back and not taken goes onto it.  What is read (table
// entries in front of the old ends, the list below its old end) is nowhere written, so the launch needs no order within.
// Latency bounds it: lengths, sums, a search, a table entry, a store.  48 sequences of a token each 3.5 us, 512 sequences with 370k
// tokens 11 us.
namespace {

constexpr int kTableThreads = 256, kTableTokens = 256;

__device__ __forceinline__ int count_le(const int* sums, int n, int x) {     // how many of n ascending sums are <= x
  int lo = 0;
  while (n > 0) {
    const int half = n >> 1;
    if (sums[lo + half] <= x) { lo += half + 1; n -= half + 1; } else n = half;
  }
  return lo;
}

}  // namespace

__global__ __launch_bounds__(kTableThreads) void k_block_tables(BlockTableArgs a) {
  extern __shared__ int sums[];      // three lists of B sums up to and with a sequence: wanted, given back, tokens
  __shared__ long long wave_sum[3][4];
  int *want_to = sums, *back_to = sums + a.B, *tok_to = sums + 2 * a.B;
  const int tid = threadIdx.x, lane = tid & 63, wave = tid >> 6;
  const long long bs = 1ll << a.sh;
  auto held_of = [&](int b) {
    const long long x = a.len_old[b], h = x > 0 ? (x + bs - 1) >> a.sh : 0;
    return h < a.max_blocks ? h : (long long)a.max_blocks;
  };
  auto need_of = [&](int b) {
    const long long x = a.len_new[b];
    return x > 0 ? (x + bs - 1) >> a.sh : 0ll;
  };
  const int per = (a.B + kTableThreads - 1) / kTableThreads, b0 = min(tid * per, a.B), b1 = min(b0 + per, a.B);
  long long x[3] = {0, 0, 0};
  auto add = [&](int b) {
    const long long held = held_of(b), need = need_of(b), more = (long long)max(a.len_new[b], 0) - max(a.len_old[b], 0);
    x[0] += need > held && need <= a.max_blocks ? need - held : 0;
    x[1] += held > need ? held - need : 0;
    x[2] += more > 0 ? more : 0;
  };
  for (int b = b0; b < b1; ++b) add(b);
  long long incl[3];
#pragma unroll
  for (int i = 0; i < 3; ++i) {
    // 40 bits (16 sequences of 2^31 each) as two numbers whose sums over a wavefront fit 32
    incl[i] = ((long long)wave_prefix((int)(x[i] >> 20)) << 20) + wave_prefix((int)(x[i] & 0xfffff));
    if (lane == 63) wave_sum[i][wave] = incl[i];
  }
  __syncthreads();
#pragma unroll
  for (int i = 0; i < 3; ++i) {
    long long s = incl[i] - x[i];
    for (int w = 0; w < wave; ++w) s += wave_sum[i][w];
    x[i] = s;
  }
  const long long top = 0x7fffffffll;
  for (int b = b0; b < b1; ++b) {
    add(b);
    want_to[b] = (int)min(x[0], top);
    back_to[b] = (int)min(x[1], top);
    tok_to[b] = (int)min(x[2], top);
  }
  long long total[3];
#pragma unroll
  for (int i = 0; i < 3; ++i) total[i] = wave_sum[i][0] + wave_sum[i][1] + wave_sum[i][2] + wave_sum[i][3];
  long long count = *a.free_in;
  count = count < 0 ? 0 : count > a.num_blocks ? a.num_blocks : count;
  const long long back = total[1], there = min(count + back, top - 1);
  __syncthreads();

  // served: what it wants is there and fits its row of the table
  auto served = [&](int b) {
    const long long held = held_of(b), need = need_of(b);
    return need <= a.max_blocks && (need <= held || want_to[b] <= there);
  };
  // blocks taken: the sums of the wanting sequences that are served are the first ones
  const int reach = count_le(want_to, a.B, (int)there);
  const long long taken = reach > 0 ? want_to[reach - 1] : 0;
  auto given = [&](int r) {          // the r-th block given back
    const int b = count_le(back_to, a.B, r);
    return a.table[(long long)b * a.max_blocks + need_of(b) + (r - (b > 0 ? back_to[b - 1] : 0))];
  };
  auto block_taken = [&](long long i) { return i < back ? given((int)i) : a.free_list[count - 1 - (i - back)]; };
  const long long first = (long long)blockIdx.x * kTableThreads + tid, step = (long long)gridDim.x * kTableThreads;
  for (long long i = first; i < taken; i += step) {
    const int b = count_le(want_to, a.B, (int)i);
    a.table[(long long)b * a.max_blocks + held_of(b) + (i - (b > 0 ? want_to[b - 1] : 0))] = block_taken(i);
  }
  for (long long r = taken + first; r < back; r += step) {
    const long long at = count + back - 1 - r;
    if (at < a.num_blocks) a.free_list[at] = given((int)r);
  }
  // slots and positions: a wavefront takes 256 tokens next to each other, whose first sequence is found once
  const long long tokens = a.n_tokens < total[2] ? a.n_tokens : total[2];
  for (long long t0 = ((long long)blockIdx.x * 4 + wave) * kTableTokens; t0 < a.n_tokens; t0 += (long long)gridDim.x * 4 * kTableTokens) {
    const int b_first = t0 < tokens ? count_le(tok_to, a.B, (int)t0) : 0;
    const long long t_last = min(t0 + kTableTokens, tokens) - 1;
    const int span = t0 < tokens ? b_first + count_le(tok_to + b_first, a.B - b_first, (int)t_last) - b_first + 1 : 0;
#pragma unroll
    for (int k = 0; k < kTableTokens / 64; ++k) {
      const long long t = t0 + k * 64 + lane;
      if (t >= a.n_tokens) break;
      if (t >= tokens) {
        a.slots[t] = -1;
        continue;
      }
      const int b = b_first + count_le(tok_to + b_first, span, (int)t);
      const long long i = t - (b > 0 ? tok_to[b - 1] : 0), old = max(a.len_old[b], 0), row = old + i, j = row >> a.sh, held = held_of(b);
      long long slot = -1;
      if (served(b)) {
        const long long block = j < held ? a.table[(long long)b * a.max_blocks + j]
                                         : block_taken((b > 0 ? want_to[b - 1] : 0) + (j - held));
        slot = (block << a.sh) + (row & (bs - 1));
      }
      a.slots[t] = slot;
      a.pos[t] = (int)((a.seen ? (long long)a.seen[b] : old) + i);
    }
  }
  if (blockIdx.x == 0) {
    for (int b = tid; b < a.B; b += kTableThreads) {
      a.len_out[b] = served(b) ? max(a.len_new[b], 0) : max(a.len_old[b], 0);
      a.cu_tokens[b + 1] = tok_to[b];
    }
    if (tid == 0) {
      a.cu_tokens[0] = 0;
      const long long left = count + back - taken;
      *a.free_out = (int)(left > a.num_blocks ? a.num_blocks : left);
    }
  }
}

hipError_t launch_block_tables(const BlockTableArgs& a, hipStream_t st) {
  // a workgroup per 1024 tokens, or per 2048 blocks that may move
  long long wgs = (a.n_tokens + 4 * kTableTokens - 1) / (4 * kTableTokens);
  const long long blocks = (long long)a.B * a.max_blocks, moved = ((blocks < a.num_blocks ? blocks : a.num_blocks) + 2047) / 2048;
  if (wgs < moved) wgs = moved;
  wgs = wgs < 1 ? 1 : wgs > 512 ? 512 : wgs;
  k_block_tables<<<(unsigned)wgs, kTableThreads, (size_t)a.B * 3 * sizeof(int), st>>>(a);
  return hipGetLastError();
}

// ---------------------------------------------------------------------------------- new rows
// A workgroup takes 256 stretches of one token's rows: the token's angles go through LDS once (fp64 product and reduction to one turn,
// fp32 sine and cosine), then every thread turns 8 pairs of channels of a head and stores them.  Values take the same way unturned.
// Memory bounds long calls: every row is read and written once, 16 bytes a lane (8192 tokens of 32 + 8 + 8 heads of 128 channels 40.6
// us with cold caches, 4.96 TB/s, where a large copy has 4.89; 201 MB, which the last-level cache holds, in a row 32.5, four tokens to
// a workgroup 35.8); latency the short ones (48 tokens 3 us).
namespace {

template <typename T> struct Eight;                  // eight channels as they stand in memory
template <> struct Eight<__bf16> { uint4 w; };
template <> struct Eight<float> { float4 w[2]; };

__device__ __forceinline__ void widen(const Eight<__bf16>& e, float* x) {
  const uint32_t w[4] = {e.w.x, e.w.y, e.w.z, e.w.w};
#pragma unroll
  for (int i = 0; i < 4; ++i) {
    x[2 * i] = __uint_as_float(w[i] << 16);
    x[2 * i + 1] = __uint_as_float(w[i] & 0xffff0000u);
  }
}
__device__ __forceinline__ void widen(const Eight<float>& e, float* x) {
#pragma unroll
  for (int i = 0; i < 2; ++i) { x[4 * i] = e.w[i].x; x[4 * i + 1] = e.w[i].y; x[4 * i + 2] = e.w[i].z; x[4 * i + 3] = e.w[i].w; }
}
__device__ __forceinline__ uint32_t two_bf16(float lo, float hi) {
  typedef __bf16 pair __attribute__((ext_vector_type(2)));
  const pair p = {(__bf16)lo, (__bf16)hi};
  return __builtin_bit_cast(uint32_t, p);
}
__device__ __forceinline__ Eight<__bf16> narrow(const float* x, __bf16) {
  return {make_uint4(two_bf16(x[0], x[1]), two_bf16(x[2], x[3]), two_bf16(x[4], x[5]), two_bf16(x[6], x[7]))};
}
__device__ __forceinline__ Eight<float> narrow(const float* x, float) {
  return {{make_float4(x[0], x[1], x[2], x[3]), make_float4(x[4], x[5], x[6], x[7])}};
}
// eight numbers as e4m3 bytes: to nearest even, saturating (a NaN stays one)
__device__ __forceinline__ uint2 bytes_of(const float* x) {
  float y[8];
#pragma unroll
  for (int i = 0; i < 8; ++i) y[i] = x[i] != x[i] ? x[i] : fminf(fmaxf(x[i], -448.0f), 448.0f);
  int lo = __builtin_amdgcn_cvt_pk_fp8_f32(y[0], y[1], 0, false), hi = __builtin_amdgcn_cvt_pk_fp8_f32(y[4], y[5], 0, false);
  lo = __builtin_amdgcn_cvt_pk_fp8_f32(y[2], y[3], lo, true);
  hi = __builtin_amdgcn_cvt_pk_fp8_f32(y[6], y[7], hi, true);
  return make_uint2((uint32_t)lo, (uint32_t)hi);
}

}  // namespace

template <int D, typename T, bool FP8>
__global__ __launch_bounds__(256) void k_append(AppendArgs a) {
  __shared__ float2 turn[D / 2];
  const int tid = threadIdx.x, token = a.first + blockIdx.x;
  long long blk = 0;
  int off = 0, b = 0, behind = 0;
  if (a.slots) {
    const long long slot = a.slots[token];
    if (slot < 0 || slot >= (a.num_blocks << a.sh)) return;
    blk = slot >> a.sh;
    off = (int)(slot & ((1 << a.sh) - 1));
  } else {
    int lo = 0, hi = a.B;                            // the token's sequence: cu[lo] <= token < cu[hi]
    if (token < a.cu[0] || token >= a.cu[a.B]) return;
    while (hi - lo > 1) {
      const int mid = (lo + hi) >> 1;
      if (a.cu[mid] <= token) lo = mid; else hi = mid;
    }
    b = lo;
    behind = a.cu[lo + 1] - token;
  }
  if (a.inv_freq) {
    for (int c = tid; c < D / 2; c += 256) {
#pragma clang fp contract(off)
      // The angle is the fp64 product.  Its whole turns, in halves, go out in fp64, with what the product with 1 / pi rounded away and what fp64
      // leaves of that number: without, an angle near 2^31 is off by 2^-24 of a turn.  What is left goes in as an fp32 number and its
      // remainder, by which sine and cosine turn on, so that they are off by those functions' own error at any position.
      const double angle = (double)a.pos[token] * a.inv_freq[c], inv_pi = 0.31830988618379067154, inv_pi_lo = -1.9678676675182485e-17;
      const double turns = angle * inv_pi, whole = 2.0 * rint(0.5 * turns);
      const double rest = (turns - whole) + fma(angle, inv_pi_lo, fma(angle, inv_pi, -turns));
      const float half_turns = (float)rest, more = (float)(rest - (double)half_turns) * 3.14159265f;
      float si, co;
      sincospif(half_turns, &si, &co);
      turn[c] = make_float2(fmaf(-si, more, co), fmaf(co, more, si));
    }
    __syncthreads();
  }
  constexpr int kPieces = D / 16;                      // of 8 channel pairs in a head
  const int heads = (a.q ? a.Hq : 0) + 2 * a.Hkv, q_heads = a.q ? a.Hq : 0;
  for (int it = blockIdx.y * 256 + tid; it < heads * kPieces; it += gridDim.y * 256) {
    const int head = it / kPieces, c = it % kPieces;
    // channels: halves apart or next to each other
    const bool is_q = head < q_heads, is_v = head >= q_heads + a.Hkv;
    const int h = is_q ? head : is_v ? head - q_heads - a.Hkv : head - q_heads;
    const T* src = is_q ? (const T*)a.q + token * a.q_stride : is_v ? (const T*)a.v + token * a.v_stride : (const T*)a.k + token * a.k_stride;
    const int c0 = a.rope_layout ? c * 16 : c * 8, c1 = a.rope_layout ? c0 + 8 : c0 + D / 2;
    const Eight<T> e0 = *(const Eight<T>*)(src + h * D + c0), e1 = *(const Eight<T>*)(src + h * D + c1);
    float x[16], y[16];
    widen(e0, x);
    widen(e1, x + 8);
    if (a.inv_freq && !is_v) {
      const float2* w = &turn[c * 8];
      if (a.rope_layout) {
#pragma unroll
        for (int i = 0; i < 8; ++i) {
          y[2 * i] = fmaf(x[2 * i], w[i].x, -x[2 * i + 1] * w[i].y);
          y[2 * i + 1] = fmaf(x[2 * i], w[i].y, x[2 * i + 1] * w[i].x);
        }
      } else {
#pragma unroll
        for (int i = 0; i < 8; ++i) {
          y[i] = fmaf(x[i], w[i].x, -x[i + 8] * w[i].y);
          y[i + 8] = fmaf(x[i], w[i].y, x[i + 8] * w[i].x);
        }
      }
    } else {
#pragma unroll
      for (int i = 0; i < 16; ++i) y[i] = x[i];
    }
    if (is_q) {
      T* dst = (T*)a.q_out + ((long long)token * a.Hq + h) * D;
      *(Eight<T>*)(dst + c0) = narrow(y, T());
      *(Eight<T>*)(dst + c1) = narrow(y + 8, T());
      continue;
    }
    long long row;
    if (a.slots) {
      row = ((blk * a.Hkv + h) << a.sh) + off;
    } else {
      const long long r = (long long)a.lens[b * a.Hkv + h] - behind;
      if (r < 0 || r >= a.n_cap) continue;
      row = ((long long)b * a.Hkv + h) * a.n_cap + r;
    }
    if constexpr (FP8) {
      const float* scale = is_v ? a.v_scale : a.k_scale;
      if (scale) {
        const float s = scale[b * a.Hkv + h];
#pragma unroll
        for (int i = 0; i < 16; ++i) y[i] /= s;
      }
      uint8_t* dst = (uint8_t*)(is_v ? a.v_cache : a.k_cache) + row * D;
      *(uint2*)(dst + c0) = bytes_of(y);
      *(uint2*)(dst + c1) = bytes_of(y + 8);
    } else {
      T* dst = (T*)(is_v ? a.v_cache : a.k_cache) + row * D;
      *(Eight<T>*)(dst + c0) = narrow(y, T());
      *(Eight<T>*)(dst + c1) = narrow(y + 8, T());
    }
  }
}

hipError_t launch_append(const AppendArgs& given, const Dims& d, hipStream_t st) {
  AppendArgs a = given;
  const int items = ((a.q ? a.Hq : 0) + 2 * a.Hkv) * (d.D / 16);
  constexpr int kMost = 1 << 23;      // (2^32 threads to a launch)
  for (a.first = 0; a.first < a.n_tokens; a.first += kMost) {
    const dim3 grid(a.n_tokens - a.first < kMost ? a.n_tokens - a.first : kMost, items < 65535 * 256 ? (items + 255) / 256 : 65535);
#define EA_CASE(DD)                                                       \
    if (d.D == DD) {                                                        \
      if (d.kv_fp8) {                                                       \
        if constexpr (DD > 64) k_append<DD, __bf16, true><<<grid, 256, 0, st>>>(a);   \
      } else if (d.dtype == EA_BF16) k_append<DD, __bf16, false><<<grid, 256, 0, st>>>(a); \
      else k_append<DD, float, false><<<grid, 256, 0, st>>>(a);             \
  }
    EA_CASE(64) EA_CASE(128) EA_CASE(256)
#undef EA_CASE
    const hipError_t e = hipGetLastError();
    if (e != hipSuccess) return e;
  }
  return hipSuccess;
}

}  // namespace ea
