// Attention of long stretches of new tokens (prompts read in pieces): the matrix cores bound it.
//
// A workgroup takes 256 (token, head) rows of a KV head, 32 for each wavefront, or 128 where no sequence has more, and walks the keys
// in tiles that all wavefronts share through LDS, the next tiles requested while one is worked on.  S^T = K Q^T and O^T = V^T P^T by v_mfma_f32_32x32x16_bf16: a
// lane then holds half of the keys of its row, and what it holds is, as it stands, the operand of the second product if V^T has
// its keys in the same order.  V^T comes out of the row-major tile by ds_read_b64_tr_b16.
//
// 2048 tokens of 32 heads over 32k rows, d = 128: 997 us (980 to 1046 from card to card), 1137 TFLOP/s of the 1189 that a large library
// product has; the matrix cores are busy in 54 % of the cycles at the 1.85 GHz that the chip's power leaves.  d = 256 1030 TFLOP/s (1100 without block
// tables), d = 64 780 (its exponentials cost as much as its products), 8-bit rows 980.
#include "ea_attend.h"

namespace ea {

namespace {

using s16x4 = short __attribute__((ext_vector_type(4)));

// A tile in LDS.  bf16 rows come straight from memory, 1 KiB per wavefront and load, lanes in order, so what would make rows meet in
// the 64 banks has to be taken out by gaps between such loads and by the order of the 16-byte pieces in a row.  K is read sixteen rows
// at a time, 16 bytes of each: 64 bytes of gap behind every KiB, and piece c stands at c ^ k_piece(row).  V is read (transposing) four
// rows at a time, 64 bytes of each: no gaps, piece c at c ^ v_piece(row).  8-bit rows pass through registers, are widened there, and
// have rows four banks apart for K, sixteen for V.
template <int D, bool FP8> constexpr int k_pitch() { return D * 2 + (FP8 ? 16 : 0); }
template <int D, bool FP8> constexpr int v_pitch() { return D * 2 + (FP8 ? 64 : 0); }
template <int D, bool FP8, int NW> constexpr int tile_keys() { return D == 256 || (D == 128 && NW == 4 && !FP8) ? 32 : 64; }
template <int D, bool FP8, int NW> constexpr int k_bytes() {
  return FP8 ? tile_keys<D, FP8, NW>() * k_pitch<D, true>() : tile_keys<D, FP8, NW>() * D * 2 / 1024 * 1088;
}
// Tiles in LDS at once.  bf16: two that are worked on and two on their way, and a barrier for every two: of the two wavefronts on a
// SIMD one is always ahead (it gets the matrix cores first, and the vector unit while the other has those), and where they meet it
// waits for the other.  8-bit rows: one of each.
template <bool FP8> constexpr int stages() { return FP8 ? 2 : 4; }
template <int D, bool FP8, int NW> constexpr int buffer_bytes() { return k_bytes<D, FP8, NW>() + tile_keys<D, FP8, NW>() * v_pitch<D, FP8>(); }
// (the row's bits that its place in its KiB and the gap in front of that leave over)
template <int D> __device__ __forceinline__ int k_piece(int row) { return D == 64 ? row >> 1 & 3 : D == 128 ? row & 3 : (row & 1) | (row >> 2 & 2); }
template <int D> __device__ __forceinline__ int v_piece(int row) { return D == 64 ? (row >> 1 & 1) * 4 : (row & 3) * 4; }
// where row `row` of K begins
template <int D, bool FP8> __host__ __device__ constexpr int k_row(int row) {
  return FP8 ? row * k_pitch<D, true>() : row / (512 / D) * 1088 + row % (512 / D) * D * 2;
}

// 16 bytes per lane from base + at to LDS address `to` and on, lanes in order.  Nothing waits for it but the s_waitcnt in front of
// the barrier behind which the tile is read; the compiler, told of such a load, would wait at the next read of any LDS.  m0,
// which the load takes its address from when it is issued, is left as it was: the compiler does not let it be named as changed.
__device__ __forceinline__ void to_lds(uint32_t to, const void* base, uint32_t at) {
  uint32_t m0;
  asm volatile("s_mov_b32 %0, m0\n\ts_mov_b32 m0, %1\n\ts_nop 0\n\tglobal_load_lds_dwordx4 %2, %3\n\ts_mov_b32 m0, %0"
               : "=&s"(m0) : "s"(to), "v"(at), "s"(base) : "memory");
}

// The order in which a block's instructions are issued: operands from LDS a few products ahead (left to itself the compiler
// reads one, waits for it, multiplies), and the next weights between the products.
template <int PRODUCTS, int kAhead>
__device__ __forceinline__ void order_products() {
  __builtin_amdgcn_sched_group_barrier(0x100, kAhead, 0);
#pragma unroll
  for (int i = 0; i < PRODUCTS - kAhead; ++i) {
    __builtin_amdgcn_sched_group_barrier(0x008, 1, 0);
    __builtin_amdgcn_sched_group_barrier(0x100, 1, 0);
  }
  __builtin_amdgcn_sched_group_barrier(0x008, kAhead, 0);
  __builtin_amdgcn_sched_barrier(0);
}
// 16 keys: their products, each with two reads for the next 16 keys and a share of the next weights behind it
template <int TILES>
__device__ __forceinline__ void order_weighted() {
#pragma unroll
  for (int i = 0; i < TILES; ++i) {
    __builtin_amdgcn_sched_group_barrier(0x008, 1, 0);
    __builtin_amdgcn_sched_group_barrier(0x100, 2, 0);
    __builtin_amdgcn_sched_group_barrier(0x002, (16 + TILES - 1) / TILES, 0);
    __builtin_amdgcn_sched_group_barrier(0x400, (8 + TILES - 1) / TILES, 0);
  }
  __builtin_amdgcn_sched_barrier(0);
}

}  // namespace

template <int D, bool FP8, bool PAGED, int NW>
__global__ __launch_bounds__(NW * 64, 2) void k_attend_tile(AttendArgs a) {
  constexpr int kM = NW * 32;
  constexpr int kN = tile_keys<D, FP8, NW>(), kKt = kN / 32, kSteps = D / 16, kCt = D / 32;
  constexpr int kRowBytes = D * (FP8 ? 1 : 2);
  constexpr int kPer = 1024 / kRowBytes;                 // rows that a wavefront's load covers
  constexpr int kPasses = kN / (NW * kPer);               // of the workgroup's loads over a tile
  constexpr int kChunks = kRowBytes / 16;
  constexpr int kKPitch = k_pitch<D, FP8>(), kKBytes = k_bytes<D, FP8, NW>(), kVPitch = v_pitch<D, FP8>(), kBuffer = buffer_bytes<D, FP8, NW>();
  constexpr int kStages = stages<FP8>();
  constexpr bool kOrdered = D < 256;                     // at d = 256 the registers are all taken without an order
  extern __shared__ __attribute__((aligned(1024))) char lds[];
  const int lane = threadIdx.x & 63, wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
  const int n32 = lane & 31, hi = lane >> 5;

  const Piece piece = find_piece<kM>(a, blockIdx.x);
  if (piece.tile < 0) return;
  note_cuts(a, piece, blockIdx.x);
  const int b = piece.b, h = piece.h, t0 = piece.t0, m = piece.m, rows = m * a.G, row0 = piece.tile * kM;
  const int len = __builtin_amdgcn_readfirstlane(rows_of(a, b, h));
  const int last_row = min(row0 + kM, rows) - 1;
  int key_hi = len - (m - 1 - last_row / a.G);           // keys that the tile's last token sees
  key_hi = key_hi < 0 ? 0 : key_hi;
  const int key_lo = piece.split * piece.chunk;
  if (piece.nsplit > 1) {
    if (key_lo >= key_hi) return;                        // (the joining launch does not ask for it)
    key_hi = min(key_hi, key_lo + piece.chunk);
  }
  const int unit = b * a.Hkv + h;
  const int all_see = len - (m - 1 - row0 / a.G);        // rows from here on some of the tile's tokens do not see
  __shared__ int bad;                                   // one of those has a value that is not finite
  if (threadIdx.x == 0) bad = 0;

  const int row = row0 + wave * 32 + n32, tok = row / a.G, hd = row - tok * a.G;
  const bool in = row < rows;
  const int vis = in ? len - (m - 1 - tok) : len;
  const int vis_min = len - (m - 1 - (row0 + wave * 32) / a.G);      // of the wavefront's rows
  // (a scale's sign goes to the queries, so that logits order like their products, and a scale of zero leaves masked ones -inf; so
  // does a scale that is not a number, which goes to the queries, too)
  const float scale = FP8 && a.kscale ? a.kscale[unit] : 1.0f, qk = a.scale * fmaxf(fabsf(scale), 1e-30f);
  bf16x8 q[kSteps];
  {
    const __bf16* src = (const __bf16*)a.q + (long long)(t0 + (in ? tok : 0)) * a.q_stride + (h * a.G + (in ? hd : 0)) * D;
#pragma unroll
    for (int s = 0; s < kSteps; ++s) {
      bf16x8 w = *(const bf16x8*)(src + s * 16 + hi * 8);
      if (!in) w = (bf16x8)(__bf16)0.0f;
      if (FP8 && scale < 0.0f) w = -w;
      if (FP8 && scale != scale) w = (bf16x8)(__bf16)scale;
      q[s] = w;
    }
  }

  // ---- loads of a tile: pass i of wavefront w covers rows (NW i + w) kPer .., which lie in one block.  Rows behind the last one are
  // asked for as the last one.  A tile's places are made while the tile in front of it is worked on, and their blocks looked up one
  // tile before that (by scalar loads: a vector load's wait would be one for all the rows on their way).
  const char* kp = (const char*)a.k + (PAGED ? ((long long)h << a.pm.sh) : ((long long)b * a.Hkv + h) * a.n_cap) * kRowBytes;
  const char* vp = (const char*)a.v + (kp - (const char*)a.k);
  const int32_t* table = PAGED ? a.pm.table + (long long)b * a.pm.max_blocks : nullptr;
  const uint32_t block_bytes = PAGED ? ((uint32_t)a.Hkv << a.pm.sh) * (uint32_t)kRowBytes : 0;     // (less than 2^32: the host sees to it)
  const int in_block = PAGED ? (1 << a.pm.sh) - 1 : ~0, last_block = (int)(a.pm.num_blocks - 1), last_sub = (len - 1) & ~15;
  const int my_row = wave * kPer + lane / kChunks, my_piece = lane % kChunks;      // of the tile, in pass 0
  const int last_tile = key_lo + (key_hi - 1 - key_lo) / kN * kN;
  int entry[kPasses];                // of the tile behind the one whose places stand in `place`
  long long place[kPasses];
  uint32_t k_off[kPasses], v_off[kPasses];
  auto first_row = [&](int at, int i) {                  // of the 16 rows that the pass's lie in
    const int sub = (at + (NW * i + wave) * kPer) & ~15;
    return sub < last_sub ? sub : last_sub;
  };
  auto look_up = [&](int at) {
    at = at < last_tile ? at : last_tile;
#pragma unroll
    for (int i = 0; i < (PAGED ? kPasses : 0); ++i)
      entry[i] = ((const __attribute__((address_space(4))) int32_t*)table)[first_row(at, i) >> a.pm.sh];
  };
  auto make_places = [&](int at) {
    at = at < last_tile ? at : last_tile;
#pragma unroll
    for (int i = 0; i < kPasses; ++i) {
      const int from = first_row(at, i), r0 = at + (NW * i + wave) * kPer, in_tile = NW * i * kPer + my_row;
      const int r = min(r0 - (r0 & ~15) + lane / kChunks, len - 1 - from);
      k_off[i] = r * kRowBytes + (FP8 ? my_piece : my_piece ^ k_piece<D>(in_tile)) * 16;
      v_off[i] = r * kRowBytes + (FP8 ? my_piece : my_piece ^ v_piece<D>(in_tile)) * 16;
      place[i] = (long long)(from & in_block) * kRowBytes;
      if (PAGED) {
        const int blk = entry[i] < 0 ? 0 : entry[i] < last_block ? entry[i] : last_block;      // a bad entry leads into the pool
        place[i] += (long long)((uint64_t)(uint32_t)blk * block_bytes);
      }
    }
  };
  u32x4 kraw[FP8 ? kPasses : 1], vraw[FP8 ? kPasses : 1];
  const uint32_t lds_at = (uint32_t)(uintptr_t)(__attribute__((address_space(3))) char*)lds;
  auto request = [&](int buf) {      // the tile at `place`
#pragma unroll
    for (int i = 0; i < kPasses; ++i) {
      if constexpr (FP8) {
        kraw[i] = *(const u32x4*)(kp + place[i] + k_off[i]);
        vraw[i] = *(const u32x4*)(vp + place[i] + v_off[i]);
      } else {
        const uint32_t to = lds_at + buf * kBuffer;
        to_lds(to + (NW * i + wave) * 1088, kp + place[i], k_off[i]);
        to_lds(to + kKBytes + (NW * i + wave) * 1024, vp + place[i], v_off[i]);
      }
    }
  };
  // 8-bit rows: from registers to LDS
  auto stage = [&](int buf) {
#pragma unroll
    for (int i = 0; i < (FP8 ? kPasses : 0); ++i) {
      const int r = (NW * i) * kPer + my_row;
      char* kd = lds + buf * kBuffer + r * kKPitch + my_piece * 32;
      char* vd = lds + buf * kBuffer + kKBytes + r * kVPitch + my_piece * 32;
      *(uint4*)kd = widen_fp8(make_uint2(kraw[i].x, kraw[i].y));
      *(uint4*)(kd + 16) = widen_fp8(make_uint2(kraw[i].z, kraw[i].w));
      *(uint4*)vd = widen_fp8(make_uint2(vraw[i].x, vraw[i].y));
      *(uint4*)(vd + 16) = widen_fp8(make_uint2(vraw[i].z, vraw[i].w));
    }
  };
  // The tiles from `at` on, kRound of them from buffer `buf`, stand in LDS where all wavefronts see them.  Values behind the last row
  // become zeros there, and of those that not all tokens see the ones that are not finite.
  constexpr int kRound = FP8 ? 1 : 2;
  auto arrived = [&](int at, int buf) {
    if constexpr (!FP8) asm volatile("s_waitcnt vmcnt(0)" ::: "memory");
    __syncthreads();
    if (at + kRound * kN > (all_see < key_hi ? all_see : key_hi)) {
      bool any = false;
      for (int i = threadIdx.x; i < kRound * kN * (D / 8); i += NW * 64) {
        const int nth = i / (kN * (D / 8)), in_tile = i % (kN * (D / 8)), row = in_tile / (D / 8), r = at + nth * kN + row;
        u32x4* v = (u32x4*)(lds + (buf + nth) * kBuffer + kKBytes + row * kVPitch) + in_tile % (D / 8);
        if (r >= key_hi) {
          *v = (u32x4)0u;
        } else if (r >= all_see) {
          const u32x4 w = *v;
          *v = u32x4{finite_pair(w.x, any), finite_pair(w.y, any), finite_pair(w.z, any), finite_pair(w.w, any)};
        }
      }
      if (any) bad = 1;
      __syncthreads();
    }
  };

  f32x16 o[kCt];
#pragma unroll
  for (int c = 0; c < kCt; ++c) o[c] = (f32x16)0.0f;
  float mx = -__builtin_inff(), l = 0.0f;
  constexpr int kFirst = FP8 ? 1 : 2;      // tiles asked for in front of the loop
  if (key_lo < key_hi) {
    look_up(key_lo);
#pragma unroll
    for (int t = 0; t < kFirst; ++t) {
      make_places(key_lo + t * kN);
      look_up(key_lo + (t + 1) * kN);
      request(t);
    }
    make_places(key_lo + kFirst * kN);
    look_up(key_lo + (kFirst + 1) * kN);
    if constexpr (FP8) {
      stage(0);
      request(1);
      make_places(key_lo + 2 * kN);
    }
    arrived(key_lo, 0);
  }
  // where the lane's operands stand: K's row n32, pieces 2 c + hi; V's rows 4 hi + .., 64-byte stretches c
  const int v_row = 4 * hi + ((lane & 15) >> 2);
  constexpr int kKWays = FP8 ? 1 : 2, kVWays = FP8 ? 1 : D == 64 ? 2 : 4;
  uint32_t k_at[kKWays], v_at[kVWays];
#pragma unroll
  for (int c = 0; c < kKWays; ++c) k_at[c] = k_row<D, FP8>(n32) + ((2 * c + hi) ^ (FP8 ? 0 : k_piece<D>(n32))) * 16;
#pragma unroll
  for (int c = 0; c < kVWays; ++c)
    v_at[c] = kKBytes + v_row * kVPitch + ((c * 4) ^ (FP8 ? 0 : v_piece<D>(v_row))) * 16 + ((lane >> 4) & 1) * 32 + (lane & 3) * 8;
  int buf = 0;
  for (int key = key_lo; key < key_hi; key += kN, buf = buf + 1 < kStages ? buf + 1 : 0) {
    const char* kt = lds + buf * kBuffer;
    const int next = key + kN;
    const int next_buf = buf + 1 < kStages ? buf + 1 : 0;
    if constexpr (!FP8) request(buf ^ 2);                  // the tile behind the next one
    __builtin_amdgcn_s_setprio(1);
    f32x16 s[kKt];
#pragma unroll
    for (int t = 0; t < kKt; ++t) {
      s[t] = (f32x16)0.0f;
#pragma unroll
      for (int c = 0; c < kSteps; ++c) {
        const bf16x8 w = *(const bf16x8*)(kt + k_at[c % kKWays] + t * k_row<D, FP8>(32) + c / kKWays * kKWays * 32);
        s[t] = __builtin_amdgcn_mfma_f32_32x32x16_bf16(w, q[c], s[t], 0, 0, 0);
      }
    }
    if constexpr (kOrdered) order_products<kKt * kSteps, 6>();
    __builtin_amdgcn_s_setprio(0);
    // V^T's operands, kRing of them ahead of the products.  Lanes 16 j .. of a group of 16 read four rows of 16 channels, and get one
    // channel of the four rows each
    constexpr int kRing = D == 256 ? 1 : 4, kOperands = kKt * 2 * kCt;
    bf16x8 vf[kRing];
    auto read_v = [&](int f) {
      const int c = f % kCt;
      const char* at = kt + v_at[c % kVWays] + (f / kCt) * 16 * kVPitch + c / kVWays * kVWays * 64;
      using lds_s16x4 = __attribute__((address_space(3))) s16x4;
      const s16x4 w0 = __builtin_amdgcn_ds_read_tr16_b64_v4i16((lds_s16x4*)at);
      const s16x4 w1 = __builtin_amdgcn_ds_read_tr16_b64_v4i16((lds_s16x4*)(at + 8 * kVPitch));
      vf[f % kRing] = __builtin_bit_cast(bf16x8, __builtin_shufflevector(w0, w1, 0, 1, 2, 3, 4, 5, 6, 7));
    };
#pragma unroll
    for (int f = 0; f < kRing; ++f) read_v(f);
    // key of s[t][r]: t 32 + (r / 4) 8 + hi 4 + r % 4
    if (key + kN > vis_min)
#pragma unroll
      for (int t = 0; t < kKt; ++t)
#pragma unroll
        for (int r = 0; r < 16; ++r)
          if (key + t * 32 + (r >> 2) * 8 + hi * 4 + (r & 3) >= vis) s[t][r] = -__builtin_inff();
    float top = s[0][0];
#pragma unroll
    for (int t = 0; t < kKt; ++t)
#pragma unroll
      for (int r = 0; r < 16; ++r) top = fmaxf(top, s[t][r]);
    top *= qk;
    if (__any(top > mx + kLag)) {
      top = reference(fmaxf(max_xor32(top), mx));
      const float f = mx == -__builtin_inff() ? 0.0f : pow2(mx - top);
      mx = top;
      l *= f;
#pragma unroll
      for (int c = 0; c < kCt; ++c) o[c] *= f;
    }
    const float from = subtrahend(mx);
    // Weights of 16 keys at a time, one block ahead of the products that take them, each rounded to one bf16 number; the sum is of the
    // unrounded ones.  The matrix cores bound this kernel, and they have no product of wider weights with bf16 values: as the sum of
    // two numbers (as in the kernel of few rows, which the cache's bytes bound) 2048 tokens over 34k rows take 1422 us and not 997, 2 x
    // 1024 over 4096 rows 121 and not 93 at d = 64, 190 and not 147 at d = 256.  What one number costs in turn is 2^-8 of the weighted
    // mean of |v| at most, and measured errors of 1.3 to 1.4 times those of results that are only rounded at the end.
    uint32_t p[kKt * 2][4];
    auto weigh = [&](int kb) {
#pragma unroll
      for (int r = 0; r < 4; ++r) {
        const float s0 = s[kb >> 1][(kb & 1) * 8 + 2 * r], s1 = s[kb >> 1][(kb & 1) * 8 + 2 * r + 1];
        const float x = pow2(fmaf(s0, qk, -from)), y = pow2(fmaf(s1, qk, -from));
        l += x + y;
        p[kb][r] = pack_bf16(x, y);
      }
    };
    weigh(0);
    __builtin_amdgcn_s_setprio(1);
    if constexpr (kOrdered) __builtin_amdgcn_sched_barrier(0);
#pragma unroll
    for (int kb = 0; kb < kKt * 2; ++kb) {
      const bf16x8 pv = __builtin_bit_cast(bf16x8, make_uint4(p[kb][0], p[kb][1], p[kb][2], p[kb][3]));
#pragma unroll
      for (int c = 0; c < kCt; ++c) {
        const int f = kb * kCt + c;
        o[c] = __builtin_amdgcn_mfma_f32_32x32x16_bf16(vf[f % kRing], pv, o[c], 0, 0, 0);
        if (f + kRing < kOperands) read_v(f + kRing);
      }
      if (kb + 1 < kKt * 2) weigh(kb + 1);
      if (!FP8 && kb == 0) make_places(key + 3 * kN);
      if (!FP8 && kb == 1) look_up(key + 4 * kN);
      if constexpr (kOrdered) order_weighted<kCt>();
    }
    __builtin_amdgcn_s_setprio(0);
    if (next < key_hi) {
      if constexpr (FP8) {
        stage(next_buf);
        request(0);
        make_places(next + 2 * kN);
      }
      if (FP8 || (buf & 1)) arrived(next, next_buf);
    }
  }
  if constexpr (!FP8) asm volatile("s_waitcnt vmcnt(0)" ::: "memory");      // nothing writes to LDS behind the workgroup's end

  l = sum_halves(l);
  __syncthreads();
  if (!in) return;
  if (bad)
#pragma unroll
    for (int c = 0; c < kCt; ++c)
#pragma unroll
      for (int r = 0; r < 16; r += 4) {
        float x[4] = {o[c][r], o[c][r + 1], o[c][r + 2], o[c][r + 3]};
        add_not_finite<D, FP8 ? 1 : 0>(a, b, h, max(max(all_see, key_lo), 0), min(vis, key_hi), c * 32 + r * 2 + hi * 4, x);
        o[c][r] = x[0]; o[c][r + 1] = x[1]; o[c][r + 2] = x[2]; o[c][r + 3] = x[3];
      }
  const long long at = (long long)(t0 + tok) * a.Hq + h * a.G + hd;
  // channel c 32 + (r / 4) 8 + hi 4 + r % 4 is o[c][r]
  if (piece.nsplit == 1) {
    const bool any = l > 0.0f || l != l;
    const float f = (FP8 && a.vscale ? a.vscale[unit] : 1.0f) / l;
    __bf16* dst = (__bf16*)a.out + at * D;
#pragma unroll
    for (int c = 0; c < kCt; ++c)
#pragma unroll
      for (int r = 0; r < 16; r += 4)
        *(uint2*)(dst + c * 32 + r * 2 + hi * 4) = any ? make_uint2(pack_bf16(o[c][r] * f, o[c][r + 1] * f), pack_bf16(o[c][r + 2] * f, o[c][r + 3] * f))
                                                       : make_uint2(0u, 0u);
    if (a.lse && hi == 0) a.lse[at] = natural_lse(mx, l);
  } else {
    const long long slot = (long long)blockIdx.x * kM + (row - row0);
    float* po = (float*)(a.ws + a.plan.split_o) + slot * D;
#pragma unroll
    for (int c = 0; c < kCt; ++c)
#pragma unroll
      for (int r = 0; r < 16; r += 4)
        *(float4*)(po + c * 32 + r * 2 + hi * 4) = make_float4(o[c][r], o[c][r + 1], o[c][r + 2], o[c][r + 3]);
    if (hi == 0) ((float2*)(a.ws + a.plan.split_ml))[slot] = make_float2(mx, l);
  }
}

template <int D, bool FP8, bool PAGED, int NW>
static hipError_t tile_of_width(const AttendArgs& a, hipStream_t st) {
  static LdsOptIn opt;
  const size_t lds = stages<FP8>() * buffer_bytes<D, FP8, NW>();
  hipError_t e = opt.ensure((const void*)k_attend_tile<D, FP8, PAGED, NW>, lds);
  if (e != hipSuccess) return e;
  k_attend_tile<D, FP8, PAGED, NW><<<(unsigned)a.plan.grid, NW * 64, lds, st>>>(a);
  e = hipGetLastError();
  if (e != hipSuccess || a.plan.most_pieces == 0) return e;
  return launch_attend_join(a, false, st);
}
template <int D, bool FP8, bool PAGED>
static hipError_t tile_of_type(const AttendArgs& a, hipStream_t st) {
  if constexpr (D < 256)
    if (a.plan.tile_rows == 128) return tile_of_width<D, FP8, PAGED, 4>(a, st);
  return tile_of_width<D, FP8, PAGED, 8>(a, st);
}

hipError_t launch_attend_tile(const AttendArgs& a, const Dims& d, hipStream_t st) {
  if (d.kv_fp8) return d.D == 128 ? tile_of_type<128, true, false>(a, st) : tile_of_type<256, true, false>(a, st);
#define EA_CASE(DD) if (d.D == DD) return a.pm.table ? tile_of_type<DD, false, true>(a, st) : tile_of_type<DD, false, false>(a, st)
  EA_CASE(64);
  EA_CASE(128);
#undef EA_CASE
  return a.pm.table ? tile_of_type<256, false, true>(a, st) : tile_of_type<256, false, false>(a, st);
}

}  // namespace ea
