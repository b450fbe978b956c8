// The kernel behind sttm_queries.h; compiled once for each element type (sttm_queries_*.hip).
#pragma once
#include "sttm_queries.h"

#include <cmath>

namespace sttm {
namespace {

typedef float f32x16 __attribute__((vector_size(64)));
typedef uint32_t w4 __attribute__((vector_size(16)));
typedef uint32_t w2 __attribute__((vector_size(8)));

// ---- products on the matrix cores ---------------------------------------------------------------------------
// D[m][n] += sum_k A[m][k] B[k][n], m, n < 32. Lane (i = lane % 32, g = lane / 32) holds A[i][*] and B[*][i] for the k of its half
// g: eight 16-bit ones (v_mfma_f32_32x32x16) or one fp32 (v_mfma_f32_32x32x2), and D[8 (r / 4) + 4 g + r % 4][i], r < 16. Which k a
// place stands for is free as long as A and B agree.
// tr_load: sixteen lanes name a 4 x 16 piece of 16-bit numbers in LDS, lane l the four of row l / 4 from column 4 (l % 4) on,
// and lane l gets the four of column l (ds_read_b64_tr_b16).
#ifndef STTM_HOST_EMULATION
template <int DT> __device__ inline f32x16 mma16(w4 a, w4 b, f32x16 c) {
  typedef float v16 __attribute__((ext_vector_type(16)));
  if constexpr (DT == 1) {
    typedef __bf16 v8 __attribute__((ext_vector_type(8)));
    return __builtin_bit_cast(f32x16, __builtin_amdgcn_mfma_f32_32x32x16_bf16(__builtin_bit_cast(v8, a), __builtin_bit_cast(v8, b), __builtin_bit_cast(v16, c), 0, 0, 0));
  } else {
    typedef _Float16 v8 __attribute__((ext_vector_type(8)));
    return __builtin_bit_cast(f32x16, __builtin_amdgcn_mfma_f32_32x32x16_f16(__builtin_bit_cast(v8, a), __builtin_bit_cast(v8, b), __builtin_bit_cast(v16, c), 0, 0, 0));
  }
}
__device__ inline f32x16 mma32(float a, float b, f32x16 c) {
  typedef float v16 __attribute__((ext_vector_type(16)));
  return __builtin_bit_cast(f32x16, __builtin_amdgcn_mfma_f32_32x32x2f32(a, b, __builtin_bit_cast(v16, c), 0, 0, 0));
}
__device__ inline w2 tr_load(const char* at) {
  typedef short v4 __attribute__((ext_vector_type(4)));
  return __builtin_bit_cast(w2, __builtin_amdgcn_ds_read_tr16_b64_v4i16((__attribute__((address_space(3))) v4*)at));
}
// Wait states between matrix products and what reads their results behind a branch (19 for the longest of them): the compiler (ROCm 7.2)
// puts none across one.
__device__ inline void settle() {
  __builtin_amdgcn_sched_barrier(0);
  asm volatile("s_nop 15\n\ts_nop 7");
  __builtin_amdgcn_sched_barrier(0);
}
// Sixteen bytes from memory to LDS, past the registers: lane i's to base + 16 i (base the same in all lanes). Lanes that do not take part leave
// their place as it is. arrived(): all of this wavefront's are there.
__device__ inline void to_lds(const char* from, char* base) {
  __builtin_amdgcn_global_load_lds((const __attribute__((address_space(1))) void*)from, (__attribute__((address_space(3))) void*)base, 16, 0, 0);
}
__device__ inline void arrived() { asm volatile("s_waitcnt vmcnt(0)" ::: "memory"); }
#else
struct EmulTiles { w4 a[64], b[64]; };
inline EmulTiles& emul_tiles() {
  static EmulTiles of_wave[16];
  return of_wave[threadIdx.x >> 6];
}
template <int DT> inline f32x16 mma16(w4 a, w4 b, f32x16 c) {
  EmulTiles& e = emul_tiles();
  const int lane = threadIdx.x & 63;
  e.a[lane] = a;
  e.b[lane] = b;
  hip_emul::wave_sync();
  for (int r = 0; r < 16; ++r) {
    float sum = c[r];
    for (int g = 0; g < 2; ++g)
      for (int w = 0; w < 4; ++w) {
        const uint32_t x = e.a[g * 32 + 8 * (r / 4) + 4 * (lane / 32) + r % 4][w], y = e.b[g * 32 + lane % 32][w];
        sum += low_half<DT>(x) * low_half<DT>(y) + high_half<DT>(x) * high_half<DT>(y);
      }
    c[r] = sum;
  }
  hip_emul::wave_sync();
  return c;
}
inline f32x16 mma32(float a, float b, f32x16 c) {
  EmulTiles& e = emul_tiles();
  const int lane = threadIdx.x & 63;
  e.a[lane][0] = __float_as_uint(a);
  e.b[lane][0] = __float_as_uint(b);
  hip_emul::wave_sync();
  for (int r = 0; r < 16; ++r)
    for (int g = 0; g < 2; ++g)
      c[r] += __uint_as_float(e.a[g * 32 + 8 * (r / 4) + 4 * (lane / 32) + r % 4][0]) * __uint_as_float(e.b[g * 32 + lane % 32][0]);
  hip_emul::wave_sync();
  return c;
}
inline w2 tr_load(const char* at) {
  EmulTiles& e = emul_tiles();
  const int lane = threadIdx.x & 63, i = lane & 15;
  memcpy(&e.a[lane], at, 8);
  hip_emul::wave_sync();
  uint16_t x[4];
  for (int k = 0; k < 4; ++k) memcpy(&x[k], reinterpret_cast<const char*>(&e.a[(lane & 48) + 4 * k + i / 4]) + 2 * (i % 4), 2);
  hip_emul::wave_sync();
  w2 r;
  memcpy(&r, x, 8);
  return r;
}
inline void settle() {}
inline void to_lds(const char* from, char* base) { memcpy(base + 16 * (threadIdx.x & 63), from, 16); }
inline void arrived() {}
#define __builtin_amdgcn_sched_barrier(x) ((void)0)
#define __builtin_amdgcn_readlane(x, i) __shfl(x, i)
#endif

// A row has CH pieces of 16 bytes in LDS (a power of two), in an order of its own, so that the lanes that read a column of pieces (keys:
// sixteen rows; values: four rows of 64 bytes) find them in different banks.
template <int CH> __device__ inline int key_order(int row) { return CH >= 16 ? row & 15 : (row >> 1) & 7; }
template <int DT, int CH> __device__ inline int value_order(int row) {
  if constexpr (DT == 0) return CH >= 16 ? 8 * ((row >> 2) & 1) : 0;
  return CH >= 16 ? 4 * (row & 3) : 4 * ((row >> 1) & 1);
}

// Of a word with two 16-bit numbers (fp32: one), those that are neither infinite nor NaN.
template <int DT> __device__ inline uint32_t finite_only(uint32_t x) {
  if constexpr (DT == 0) return (x & 0x7f800000u) == 0x7f800000u ? 0u : x;
  constexpr uint32_t E = DT == 1 ? 0x7f80u : 0x7c00u;
  return ((x & E) == E ? 0u : x & 0xffffu) | ((x >> 16 & E) == E ? 0u : x & 0xffff0000u);
}

// How a workgroup is made up: wavefronts (two buffers each have to fit LDS where a wavefront has blocks of its own), keys of a block, sixteen-byte
// pieces that a thread brings of it.
constexpr int query_waves(int dt, int dp, bool few) { return few && query_row_bytes(dp, dt == 0 ? 4 : 2) > 256 ? 2 : kQueryWaves; }
constexpr int query_blocks_a_unit(int dt, int dp, bool few) { return few || query_row_bytes(dp, dt == 0 ? 4 : 2) > 256 ? 1 : 2; }
template <int DT, int DP, bool FEW> struct Shape {
  static constexpr int ES = DT == 0 ? 4 : 2, M = DP / 32, NQ = DP * ES / 32;
  static constexpr int ROW = query_row_bytes(DP, ES), CH = ROW / 16;
  static constexpr int WAVES = query_waves(DT, DP, FEW), THREADS = WAVES * kWave;
  static constexpr int SHARE = FEW ? 1 : WAVES;           // wavefronts that share a block of keys
  static constexpr int SETS = WAVES / SHARE;
  static constexpr int NK = !FEW && ROW <= 256 ? 64 : 32, KT = NK / 32;
  static constexpr int AT_ONCE = kWave / CH;              // rows of one load of a wavefront
  static constexpr int PER = NK / (AT_ONCE * SHARE);      // loads of a wavefront for a block's keys
  static constexpr int TILE = kRowTile * SHARE;
};

// One workgroup: a tile of rows (a token and a head of the kv head's group each) of one segment, one chunk of the segment's keys. FEW: 32
// rows, the four wavefronts take blocks of 32 keys in turn, each with its own running maximum and sum, joined in LDS at the
// end. Else 128 rows, 32 a wavefront, that share blocks of NK keys.
//
// Both products are laid out so that nothing changes lanes between them: S^T = K Q^T has keys as rows and query rows as columns, a lane
// ends up with the keys 8 i + 4 g + 0..3 of its own query row, and these are the k of its half in O^T = V^T P^T. Maximum and sum are taken
// in a lane and once across the two halves. Keys are read from LDS as they lie, values transposed on the way.
//
// P is rounded to 16 bits for 16-bit values (half a step of the type: as much as the rounding of the result, which the sum over keys
// mostly averages away); the sum that divides is that of the unrounded ones, in 32 bits. In fp16 it is 2^15 P, so that a weight is
// off by no more than 2^-40 of the largest one where fp16 runs out of exponents.
template <int DT, int DP, bool FEW>
__global__ void __launch_bounds__(query_waves(DT, DP, FEW) * kWave, query_blocks_a_unit(DT, DP, FEW)) k_query_tiles(QueryArgs a, KeyArgs kk) {
  using S = Shape<DT, DP, FEW>;
  constexpr int ES = S::ES, ROW = S::ROW, CH = S::CH, NQ = S::NQ, M = S::M, SETS = S::SETS, NK = S::NK, KT = S::KT;
  constexpr int AT_ONCE = S::AT_ONCE, PER = S::PER, TILE = S::TILE, THREADS = S::THREADS;
  constexpr float LIFT = DT == 2 ? 15.f : 0.f;
  constexpr float UNLIFT = DT == 2 ? 1.f / 32768.f : 1.f;
  constexpr bool WIDE = DP * ES > 256;                    // one way for all blocks: the registers that two ways take are not there
  static_assert(CH >= 8 && CH <= 64 && NK % (AT_ONCE * S::SHARE) == 0 && (!FEW || SETS * 2 * NK * ROW * 2 >= S::WAVES * 4096), "tiles");

  __shared__ __align__(16) char tiles[SETS][2][2][NK * ROW];  // of each set two buffers of keys and of values
  __shared__ __align__(16) float adds[SETS][2][NK];       // what is added to a key's score: its bias; -inf: it does not count
  __shared__ float stat_m[SETS][kRowTile], stat_l[SETS][kRowTile];
  __shared__ int odd_value;                               // a value that is not finite in a block whose keys not all rows see

  const int tid = threadIdx.x, wave = __builtin_amdgcn_readfirstlane(tid >> 6), lane = tid & 63, i32 = lane & 31, g = lane >> 5;
  const int tile = blockIdx.x, h = blockIdx.y, chunk = blockIdx.z;
  // Segment s has the tiles from first_token * group / TILE + s on: no two share one, and each has as many as it needs.
  const int s = last_not_above(a.segments, tile, [&](int i) { return first_token_of_segment(a, i) * a.group / TILE + i; });
  const long long token0 = first_token_of_segment(a, s);
  const long long rows = max(first_token_of_segment(a, s + 1) - token0, 0ll) * a.group;
  const long long row0 = (tile - (token0 * a.group / TILE + s)) * TILE;
  if (row0 < 0 || row0 >= rows) return;
  long long key0;
  const int length = segment_length(kk, s, &key0);
  const int first = chunk * kk.chunk;
  if (first >= length && chunk > 0) return;               // (an empty segment's first chunk is gone through: its result is written)

  // This lane's row.
  const int set = FEW ? wave : 0, share = FEW ? 0 : wave;
  const long long row = row0 + share * kRowTile + i32;
  const bool mine = row < rows;
  const long long in_row = min(row, rows - 1), in_token = in_row / a.group, token = token0 + in_token;
  const int head = h * a.group + (int)(in_row - in_token * a.group);
  int limit = length, end = min(length, first + kk.chunk), least = length;   // slots that the row, any row of the tile, all of them see
  if (kk.causal) {
    const long long behind = length - rows / a.group + 1;
    limit = (int)max(behind + in_token, 0ll);
    least = (int)max(behind + row0 / a.group, 0ll);
    end = (int)min((long long)end, max(behind + (min(row0 + TILE, rows) - 1) / a.group, 0ll));
  }

  w4 q[NQ];
  {
    const char* at = a.q + token * a.q_stride + (long long)head * a.d * ES;
#pragma unroll
    for (int c = 0; c < NQ; ++c) {
      const int o = (2 * c + g) * 16;
      uint4 x = make_uint4(0u, 0u, 0u, 0u);
      if (mine && o < kk.pool.row) x = *reinterpret_cast<const uint4*>(at + o);
      q[c] = w4{x.x, x.y, x.z, x.w};
    }
  }

  const float* bias = kk.bias ? kk.bias + s * kk.bias_segment + h * kk.bias_head + key0 : nullptr;
  const int32_t* table = kk.table ? kk.table + s * kk.table_stride : nullptr;
  const int page_mask = (1 << kk.pool.shift) - 1;
  const long long base = h * kk.pool.head_stride + key0 * kk.token_stride;
  const int stride = (int)kk.token_stride;                // (a block's rows lie within 2 GiB)

  // The pieces of LDS that this lane fills with load i: of row brought + AT_ONCE * SHARE * i (+ its own row of the AT_ONCE of a load), which lie
  // in one page. Pieces behind a head's channels stay zero.
  const int brought = __builtin_amdgcn_readfirstlane(share * AT_ONCE), own_row = lane / CH;
  int key_from[PER], value_from[PER];
#pragma unroll
  for (int i = 0; i < PER; ++i) {
    const int r = brought + AT_ONCE * S::SHARE * i + own_row;
    key_from[i] = 16 * (lane % CH ^ key_order<CH>(r));
    value_from[i] = 16 * (lane % CH ^ value_order<DT, CH>(r));
  }
  const bool full = kk.pool.row == ROW;
  // Lane i: the page of the block's key i, looked up a block ahead, and what is added to its score. Keys from the end on: the page of the
  // last one, whose other slots may be read.
  int page_next = 0;
  float add_next = 0.f;
  auto look_up = [&](int s0) {
    if (table) page_next = table[min(s0 + min(lane, NK - 1), end - 1) >> kk.pool.shift];
  };
  auto load = [&](int s0, int buffer) {
    const bool there = !table || (unsigned)page_next < (unsigned)kk.pool.pages;
    add_next = bias ? bias[min(s0 + min(lane, NK - 1), end - 1)] : 0.f;
    if (lane >= NK || s0 + lane >= end || !there) add_next = -INFINITY;
    const int page = there ? page_next : 0;               // (what is read of a page that is not there does not count)
    char* const to = tiles[set][buffer][0] + brought * ROW;
#pragma unroll
    for (int i = 0; i < PER; ++i) {
      const int r = brought + AT_ONCE * S::SHARE * i;
      long long from;
      int row = own_row * stride;
      if (table) {
        from = __builtin_amdgcn_readlane(page, r) * kk.pool.page_stride + base + ((s0 + r) & page_mask) * stride;
      } else {
        from = base + (s0 + r) * kk.token_stride;
        if (s0 + NK > end) {                              // (rows from the end on: the last one)
          from = base + s0 * kk.token_stride;
          row = min(r + own_row, end - 1 - s0) * stride;
        }
      }
      char* const at = to + AT_ONCE * S::SHARE * i * ROW;
      if (full) {
        to_lds(kk.pool.k + from + (unsigned)(row + key_from[i]), at);
        to_lds(kk.pool.v + from + (unsigned)(row + value_from[i]), at + NK * ROW);
      } else {
        if (key_from[i] < kk.pool.row) to_lds(kk.pool.k + from + (unsigned)(row + key_from[i]), at);
        if (value_from[i] < kk.pool.row) to_lds(kk.pool.v + from + (unsigned)(row + value_from[i]), at + NK * ROW);
      }
    }
  };

  // Where this lane reads in LDS: the parts of an address that rows of a fixed distance have in common.
  constexpr int P = CH >= 16 ? 16 : 8, NK_AT = NQ < P / 2 ? NQ : P / 2, NV_AT = DT != 0 ? M : M < 2 || CH < 16 ? 1 : 2;
  int key_at[NK_AT], value_at[NV_AT];
#pragma unroll
  for (int i = 0; i < NK_AT; ++i) key_at[i] = i32 * ROW + 16 * ((2 * i + g) ^ key_order<CH>(i32));
#pragma unroll
  for (int i = 0; i < NV_AT; ++i) {
    if constexpr (DT == 0) value_at[i] = 4 * g * ROW + 16 * ((8 * i + i32 / 4) ^ value_order<DT, CH>(4 * g)) + 4 * (i32 % 4);
    else {
      const int r = 4 * g + (lane & 15) / 4;
      value_at[i] = r * ROW + 16 * ((4 * i + 2 * ((lane >> 4) & 1) + (lane & 3) / 2) ^ value_order<DT, CH>(r)) + 8 * (lane & 1);
    }
  }

  f32x16 acc[M];
#pragma unroll
  for (int n = 0; n < M; ++n)
#pragma unroll
    for (int r = 0; r < 16; ++r) acc[n][r] = 0.f;
  // Scores that have no bias stay as the product gives them, the scale is part of the exponent's factor.
  constexpr float kWide = 65536.f;                        // (times 2^-24 is what the rounding of `from` may leave in an exponent)
  float m = -INFINITY, from = 0.f, l = 0.f;  // from: m as an exponent of two; l: of this lane's keys
  const float times = kk.scaled ? kLog2e : a.scale * kLog2e, scaled = kk.scaled ? a.scale : 1.f;
  if (tid == 0) odd_value = 0;
  if (!full) {                                            // pieces of LDS that nothing is loaded into
    for (int i = tid; i < (int)sizeof(tiles) / 16; i += THREADS) reinterpret_cast<w4*>(tiles)[i] = w4{0u, 0u, 0u, 0u};
    __syncthreads();
  }
  const int start = first + set * NK, step = SETS * NK;
  if (start < end) {
    look_up(start);
    load(start, 0);
    look_up(start + step);
  }
  int buffer = 0;
  for (int s0 = start; s0 < end; s0 += step, buffer ^= 1) {
    char* const keys = tiles[set][buffer][0];
    char* const values = tiles[set][buffer][1];
    arrived();
    const unsigned long long alive = __ballot(add_next != -INFINITY);
    const bool whole = alive == (NK == 64 ? ~0ull : 0xffffffffull);
    const bool diagonal = s0 + NK > least && least < length, added = WIDE || kk.scaled || !whole;
    if (diagonal || !whole) {                             // (this wavefront's own pieces: it sees what it loaded)
      __builtin_amdgcn_wave_barrier();
      bool odd = false;
#pragma unroll
      for (int i = 0; i < PER; ++i) {
        const int r = brought + AT_ONCE * S::SHARE * i;
        w4* at = reinterpret_cast<w4*>(values + r * ROW + 16 * lane);
        if (!(alive >> (r + own_row) & 1)) {              // a key that does not count: nothing of it may be infinite or NaN
          *at = w4{0u, 0u, 0u, 0u};
          *reinterpret_cast<w4*>(keys + r * ROW + 16 * lane) = w4{0u, 0u, 0u, 0u};
        } else if (diagonal) {
          w4 y = *at;
#pragma unroll
          for (int e = 0; e < 4; ++e) {
            const uint32_t f = finite_only<DT>(y[e]);
            odd |= f != y[e];
            y[e] = f;
          }
          *at = y;
        }
      }
      if (odd) odd_value = 1;
    }
    if (share == 0 && lane < NK && added) adds[set][buffer][lane] = add_next;
    if constexpr (FEW) __builtin_amdgcn_wave_barrier();
    else __syncthreads();
    if (s0 + step < end) {
      load(s0 + step, buffer ^ 1);
      look_up(s0 + 2 * step);
    }

    f32x16 x[KT];
#pragma unroll
    for (int t = 0; t < KT; ++t)
#pragma unroll
      for (int r = 0; r < 16; ++r) x[t][r] = 0.f;
#pragma unroll
    for (int c = 0; c < NQ; ++c) {
      if (DP * ES > 256 && c % 4 == 0) __builtin_amdgcn_sched_barrier(0);   // (not all reads before the first product: registers)
#pragma unroll
      for (int t = 0; t < KT; ++t) {
        const w4 k = *reinterpret_cast<const w4*>(keys + key_at[c % NK_AT] + (32 * t * ROW + c / NK_AT * NK_AT * 32));
        if constexpr (DT == 0) {
#pragma unroll
          for (int e = 0; e < 4; ++e) x[t] = mma32(__uint_as_float(k[e]), __uint_as_float(q[c][e]), x[t]);
        } else {
          x[t] = mma16<DT>(k, q[c], x[t]);
        }
      }
    }
    settle();
    if (added) {
#pragma unroll
      for (int t = 0; t < KT; ++t)
#pragma unroll
        for (int r4 = 0; r4 < 4; ++r4) {
          const float4 add = *reinterpret_cast<const float4*>(&adds[set][buffer][32 * t + 8 * r4 + 4 * g]);
          const float of[4] = {add.x, add.y, add.z, add.w};
#pragma unroll
          for (int e = 0; e < 4; ++e) x[t][4 * r4 + e] = fmaf(x[t][4 * r4 + e], scaled, of[e]);
        }
    }
    if (diagonal) {
#pragma unroll
      for (int t = 0; t < KT; ++t)
#pragma unroll
        for (int r = 0; r < 16; ++r)
          if (s0 + 32 * t + 8 * (r / 4) + 4 * g + r % 4 >= limit) x[t][r] = -INFINITY;
    }
    float top = x[0][0];
#pragma unroll
    for (int t = 0; t < KT; ++t)
#pragma unroll
      for (int r = 0; r < 16; ++r) top = fmaxf(top, x[t][r]);
    top = fmaxf(top, __shfl_xor(top, 32, 64));
    if (__ballot(top > m) != 0) {  // (seldom after the first blocks)
      const float before = m, from_before = m == -INFINITY ? -INFINITY : from;
      m = fmaxf(m, top);
      from = m == -INFINITY ? 0.f : m * times;
      const float shrink = exp2_fast(fabsf(from) < kWide ? from_before - from : (before - m) * times);
      l *= shrink;
#pragma unroll
      for (int n = 0; n < M; ++n)
#pragma unroll
        for (int r = 0; r < 16; ++r) acc[n][r] *= shrink;
    }
    float less = LIFT - from;
    if (WIDE || __ballot(!(fabsf(from) < kWide)) != 0) {  // large scores: no multiple of theirs, only of their differences
      less = LIFT;
#pragma unroll
      for (int t = 0; t < KT; ++t)
#pragma unroll
        for (int r = 0; r < 16; ++r) x[t][r] -= m == -INFINITY ? 0.f : m;
    }
#pragma unroll
    for (int t = 0; t < KT; ++t)
#pragma unroll
      for (int r = 0; r < 16; ++r) {
        x[t][r] = exp2_fast(fmaf(x[t][r], times, less));
        l += x[t][r];
      }
    if constexpr (DT == 0) {
#pragma unroll
      for (int t = 0; t < KT; ++t)
#pragma unroll
        for (int r = 0; r < 16; ++r) {
          if (r % 2 == 0) __builtin_amdgcn_sched_barrier(0);
#pragma unroll
          for (int n = 0; n < M; ++n) {
            const char* at = values + value_at[n % NV_AT] + ((32 * t + 8 * (r / 4) + r % 4) * ROW + n / NV_AT * NV_AT * 128);
            acc[n] = mma32(*reinterpret_cast<const float*>(at), x[t][r], acc[n]);
          }
        }
    } else {
#pragma unroll
      for (int j = 0; j < NK / 16; ++j) {
        __builtin_amdgcn_sched_barrier(0);
        w4 p;
#pragma unroll
        for (int w = 0; w < 4; ++w) p[w] = pack2<DT>(x[j / 2][8 * (j % 2) + 2 * w], x[j / 2][8 * (j % 2) + 2 * w + 1]);
#pragma unroll
        for (int n = 0; n < M; ++n) {
          const w2 lo = tr_load(values + value_at[n] + 16 * j * ROW), hi = tr_load(values + value_at[n] + (16 * j + 8) * ROW);
          acc[n] = mma16<DT>(w4{lo[0], lo[1], hi[0], hi[1]}, p, acc[n]);
        }
      }
    }
  }
  settle();

  l += __shfl_xor(l, 32, 64);
  l *= UNLIFT;
  if (!kk.scaled && m != -INFINITY) m *= a.scale;
  float top = m, total = l, mine_of = UNLIFT;
  if constexpr (FEW) {  // the wavefronts on a common maximum
    if (lane < kRowTile) {
      stat_m[wave][lane] = m;
      stat_l[wave][lane] = l;
    }
    __syncthreads();
    for (int w = 0; w < SETS; ++w) top = fmaxf(top, stat_m[w][i32]);
    total = 0.f;
    for (int w = 0; w < SETS; ++w) total += stat_l[w][i32] * query_factor(stat_m[w][i32], top);
    mine_of = query_factor(m, top) * UNLIFT;
  }
  const long long index = token * (a.kv_heads * a.group) + head;
  if (mine && g == 0 && set == 0) {
    if (a.part) a.stat[index * a.parts + a.first_part + chunk] = make_float2(top, total);
    else if (a.lse) a.lse[index] = top + logf(total);
  }
  const float inverse = a.part ? 1.f : total == 0.f ? 0.f : 1.f / total;
  float* part = a.part ? a.part + (index * a.parts + a.first_part + chunk) * a.d : nullptr;
  char* out = a.part ? nullptr : a.out + token * a.out_stride + (long long)head * a.d * ES;
  auto store = [&](int c, float4 y) {                     // four channels of this lane's row
    if (part) {
      *reinterpret_cast<float4*>(part + c) = y;
    } else {
      const float z[4] = {y.x * inverse, y.y * inverse, y.z * inverse, y.w * inverse};
      if constexpr (DT == 0) *reinterpret_cast<float4*>(out + 4 * c) = make_float4(z[0], z[1], z[2], z[3]);
      else *reinterpret_cast<uint2*>(out + 2 * c) = make_uint2(pack2<DT>(z[0], z[1]), pack2<DT>(z[2], z[3]));
    }
  };
  if constexpr (!FEW) {
#pragma unroll
    for (int n = 0; n < M; ++n)
#pragma unroll
      for (int j = 0; j < 4; ++j) {
        const int c = 32 * n + 8 * j + 4 * g;
        if (mine && c < a.d) store(c, make_float4(acc[n][4 * j] * mine_of, acc[n][4 * j + 1] * mine_of, acc[n][4 * j + 2] * mine_of, acc[n][4 * j + 3] * mine_of));
      }
  } else {
    // 32 channels at a time: every wavefront leaves its four runs of four channels a lane, wavefront w adds the runs w, w + SETS .. up.
    float4* joined = reinterpret_cast<float4*>(tiles);    // [wave][j][lane]
#pragma unroll
    for (int n = 0; n < M; ++n) {
      __syncthreads();
#pragma unroll
      for (int j = 0; j < 4; ++j)
        joined[(wave * 4 + j) * kWave + lane] = make_float4(acc[n][4 * j] * mine_of, acc[n][4 * j + 1] * mine_of, acc[n][4 * j + 2] * mine_of, acc[n][4 * j + 3] * mine_of);
      __syncthreads();
#pragma unroll
      for (int j = wave; j < 4; j += SETS) {
        const int c = 32 * n + 8 * j + 4 * g;
        if (!mine || c >= a.d) continue;
        float4 y = joined[j * kWave + lane];
        for (int w = 1; w < SETS; ++w) {
          const float4 z = joined[(w * 4 + j) * kWave + lane];
          y.x += z.x; y.y += z.y; y.z += z.z; y.w += z.w;
        }
        store(c, y);
      }
    }
  }
  if (kk.causal) __syncthreads();                         // (odd_value, of all wavefronts)
  if (kk.causal && odd_value) {
    // Values that are not finite were left out where some rows see them and others do not (a weight of zero does not make them
    // zero): the rows that see them get them here. What is infinite or NaN already stays so.
#pragma unroll 1
    for (int c = FEW ? 8 * wave + 4 * g : 4 * g; c < a.d && mine; c += FEW ? 8 * SETS : 8) {
      float add[4] = {0.f, 0.f, 0.f, 0.f};
#pragma unroll 1
      for (int i = max(first, least - NK + 1); i < min(end, limit); ++i) {
        const int page = table ? table[i >> kk.pool.shift] : 0;
        if ((table && (unsigned)page >= (unsigned)kk.pool.pages) || (bias && bias[i] == -INFINITY)) continue;
        const long long at = base + (table ? page * kk.pool.page_stride + (i & page_mask) * stride : i * kk.token_stride);
        for (int e = 0; e < 4; ++e) {
          float v;
          if constexpr (DT == 0) v = *reinterpret_cast<const float*>(kk.pool.v + at + 4 * (c + e));
          else v = low_half<DT>(*reinterpret_cast<const uint16_t*>(kk.pool.v + at + 2 * (c + e)));
          if (!(fabsf(v) < INFINITY)) add[e] += v;
        }
      }
      for (int e = 0; e < 4; ++e) {
        if (add[e] == 0.f) continue;
        if (part) part[c + e] += add[e];
        else if constexpr (DT == 0) reinterpret_cast<float*>(out)[c + e] += add[e];
        else {
          uint16_t* to = reinterpret_cast<uint16_t*>(out) + c + e;
          *to = (uint16_t)pack2<DT>(low_half<DT>(*to) + add[e], 0.f);
        }
      }
    }
  }
}

template <int DT, int DP>
void launch_tiles(const QueryArgs& a, const KeyArgs& k, bool few, hipStream_t s) {
  constexpr int ROW = DP * (DT == 0 ? 4 : 2);
  const dim3 grid((unsigned)(a.tokens * a.group / query_tile(few) + a.segments), a.kv_heads, k.chunks);
  if constexpr (ROW <= 512) {
    if (few) {
      hipLaunchKernelGGL((k_query_tiles<DT, DP, true>), grid, dim3(Shape<DT, DP, true>::THREADS), 0, s, a, k);
      return;
    }
  }
  hipLaunchKernelGGL((k_query_tiles<DT, DP, false>), grid, dim3(Shape<DT, DP, false>::THREADS), 0, s, a, k);
}

}  // namespace

template <int DT> void launch_queries(const QueryArgs& a, const KeyArgs& k, bool few_rows, hipStream_t s) {
  if (a.d <= 32) launch_tiles<DT, 32>(a, k, few_rows, s);
  else if (a.d <= 64) launch_tiles<DT, 64>(a, k, few_rows, s);
  else if (a.d <= 96) launch_tiles<DT, 96>(a, k, few_rows, s);
  else if (a.d <= 128) launch_tiles<DT, 128>(a, k, few_rows, s);
  else if (a.d <= 192) launch_tiles<DT, 192>(a, k, few_rows, s);
  else launch_tiles<DT, 256>(a, k, few_rows, s);
}

}  // namespace sttm
