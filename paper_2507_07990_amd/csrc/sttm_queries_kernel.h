// The kernel behind sttm_queries.h; compiled once for each element type (sttm_queries_*.hip).
#pragma once
#include "sttm_queries.h"

#include <cmath>
#include <type_traits>

// (for lambdas: one that is not inlined has its captures in memory)
#define STTM_INLINE __attribute__((always_inline))

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
// The larger of a lane's number and that of the lane 32 further.
__device__ inline float of_halves(float x) {
  const auto r = __builtin_amdgcn_permlane32_swap(__float_as_uint(x), __float_as_uint(x), false, false);
  return fmaxf(__uint_as_float(r[0]), __uint_as_float(r[1]));
}
// Wait states between matrix products and what reads their results behind a branch (19 for the longest of them): the compiler (ROCm 7.2)
// puts none across one.
__device__ inline void settle() {
  __builtin_amdgcn_sched_barrier(0);
  asm volatile("s_nop 15\n\ts_nop 7");
  __builtin_amdgcn_sched_barrier(0);
}
// Sixteen bytes from memory to LDS, past the registers: lane i's to base + 16 i (base the same in all lanes). Lanes that do not take part leave
// their place as it is. arrived(): all of this wavefront's are there but the last LATER loads.
__device__ inline void to_lds(const char* from, char* base) {
  __builtin_amdgcn_global_load_lds((const __attribute__((address_space(1))) void*)from, (__attribute__((address_space(3))) void*)base, 16, 0, 0);
}
template <int LATER> __device__ inline void arrived() {
  static_assert(LATER < 64, "a counter of six bits");
  asm volatile("" ::: "memory");
  __builtin_amdgcn_s_waitcnt((LATER & 15) | 7 << 4 | 15 << 8 | (LATER >> 4) << 14);  // (the other counters as they are)
  asm volatile("" ::: "memory");
}
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
inline float of_halves(float x) { return fmaxf(x, __shfl_xor(x, 32, 64)); }
inline void to_lds(const char* from, char* base) { memcpy(base + 16 * (threadIdx.x & 63), from, 16); }
template <int LATER> inline void arrived() {}
#define __builtin_amdgcn_sched_barrier(x) ((void)0)
#define __builtin_amdgcn_s_setprio(x) ((void)0)
#define __builtin_amdgcn_sched_group_barrier(kinds, count, group) ((void)0)
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

__device__ __align__(16) const char kZeros[16] = {};

// How a workgroup is made up: wavefronts (two buffers each have to fit LDS where a wavefront has blocks of its own), keys of a block, sixteen-byte
// pieces that a thread brings of it.
constexpr int query_waves(int dt, int dp, bool few) { return few && query_row_bytes(dp, dt == 0 ? 4 : 2) > 256 ? 2 : kQueryWaves; }
constexpr int query_waves_a_simd(int dt, int dp) { return dp * (dt == 0 ? 4 : 2) > 256 ? 1 : 2; }
template <int DT, int DP, bool FEW> struct Shape {
  static constexpr int ES = DT == 0 ? 4 : 2, M = DP / 32, NQ = DP * ES / 32;
  static constexpr int ROW = query_row_bytes(DP, ES), CH = ROW / 16;
  static constexpr int WAVES = query_waves(DT, DP, FEW), THREADS = WAVES * kWave;
  static constexpr int SHARE = FEW ? 1 : WAVES;           // wavefronts that share a block of keys
  static constexpr int SETS = WAVES / SHARE, BUFFERS = FEW ? 1 : 2;
  static constexpr int NK = !FEW && ROW <= 256 ? 64 : 32, KT = NK / 32;
  static constexpr int AT_ONCE = kWave / CH;              // rows of one load of a wavefront
  static constexpr int PER = NK / (AT_ONCE * SHARE);      // loads of a wavefront for a block's keys
  static constexpr int TILE = kRowTile * SHARE;
};

// Held in a register, the same in all lanes: the compiler would read an argument anew in every block, and wait for it.
template <class T> __device__ inline T held(T x) {
#ifdef __HIP_DEVICE_COMPILE__
  asm("" : "+s"(x));
#endif
  return x;
}

// Which of n pieces of work, tiles fastest, workgroup id takes. Workgroups go to the eight dies in turn, and each die has an L2 of its own: the tiles of one
// head and chunk, which read the same keys, go to one die; what is left over of eight of these, in eight runs (whole calls, us, against tiles in turn:
// one prompt on 43,264 keys 275 against 302, ragged prompts 164 / 195, 32 answers behind 14,672 slots 60 / 65). Few rows share no keys.
template <bool FEW> __device__ inline unsigned in_dies(unsigned id, unsigned n, unsigned tiles) {
  constexpr unsigned DIES = 8;
  if (FEW) return id;
  const unsigned whole = n / (DIES * tiles) * (DIES * tiles);
  unsigned run = tiles, begin = 0;
  if (id >= whole) {
    begin = whole;
    run = (n - whole) / DIES;
    if (id >= begin + run * DIES) return id;
  }
  const unsigned turn = (id - begin) / DIES, round = turn / run;
  return begin + (round * DIES + (id - begin) % DIES) * run + (turn - round * run);
}

// One workgroup: a tile of rows (a token and a head of the kv head's group each) of one segment, one chunk of the segment's keys. FEW: 32
// rows, the four wavefronts take blocks of 32 keys in turn, each with its own running maximum and sum, joined in LDS at the
// end. Else 128 rows, 32 a wavefront, that share blocks of NK keys.
//
// What bounds it. Few rows: memory (32 sequences of 1,013 to 8,117 keys, 64 heads on 8 of 128 bf16 channels: 454 MB in 97 us, 4.7 TB/s), and where the keys
// are few the chain of dependent loads (257 keys: 8 us). Many rows: the two products and the softmax between them; a compute unit's registers and LDS
// hold two workgroups, whose wavefronts take turns (331 tokens on 43,264 keys, 28 heads on 4: 205 GFLOP in 258 us, 0.79 PFLOP/s, matrix cores busy
// 38 % of the time, vector units 49 %; without the loads 0.82, without the exponentials 0.90, without either product 0.86 of the time). A tile of
// 128 rows reads each key from the die's L2 once; 32 rows a wavefront leave registers for two wavefronts a SIMD. Rows have a power of two of
// bytes in LDS, their pieces in an order of their own: no bank conflicts.
//
// Both products are laid out so that nothing changes lanes between them: S^T = K Q^T has keys as rows and query rows as columns, a lane
// ends up with the keys 8 i + 4 g + 0..3 of its own query row, and these are the k of its half in O^T = V^T P^T. Maximum and sum are taken
// in a lane and once across the two halves. Keys are read from LDS as they lie, values transposed on the way.
//
// P is rounded to 16 bits for 16-bit values (half a step of the type: as much as the rounding of the result, which the sum over keys
// mostly averages away); the sum that divides is that of the unrounded ones, in 32 bits. In fp16 it is 2^15 P, so that a weight is
// off by no more than 2^-40 of the largest one where fp16 runs out of exponents.
template <int DT, int DP, bool FEW, bool PAGED, bool FULL>
__global__ void __launch_bounds__(query_waves(DT, DP, FEW) * kWave, query_waves_a_simd(DT, DP)) k_query_tiles(QueryJobs jobs) {
  using S = Shape<DT, DP, FEW>;
  constexpr int ES = S::ES, ROW = S::ROW, CH = S::CH, NQ = S::NQ, M = S::M, SETS = S::SETS, BUFFERS = S::BUFFERS, NK = S::NK, KT = S::KT;
  constexpr int AT_ONCE = S::AT_ONCE, PER = S::PER, TILE = S::TILE;
  constexpr bool CAUSAL = PAGED;                          // (or may be)
  constexpr float LIFT = DT == 2 ? 15.f : 0.f;
  // (as a weight up to 16, which costs sums that much of their range; fp16: 2^15.9, what it can hold; fp32 products take longer than the rescaling)
  constexpr float SLACK = DT == 0 ? 0.f : DT == 1 ? 2.75f : 0.62f;
  constexpr float UNLIFT = DT == 2 ? 1.f / 32768.f : 1.f;
  constexpr int K_AHEAD = DT == 0 ? 2 : 4, V_AHEAD = 2;  // pieces of keys, steps of values read ahead
  constexpr bool ONE_WAY = DP * ES > 256;                 // (the registers that two ways take are not there)
  static_assert(CH >= 8 && CH <= 64 && NK % (AT_ONCE * S::SHARE) == 0 && (!FEW || SETS * NK * ROW >= S::WAVES * 4096), "tiles");

  // Keys and values, two buffers where wavefronts share them. (Arrays of their own: the compiler waits for all loads to LDS before it reads what they
  // might have written to.)
  __shared__ __align__(16) char keys0[SETS * NK * ROW], values0[SETS * NK * ROW], keys1[BUFFERS == 2 ? NK * ROW : 16], values1[BUFFERS == 2 ? NK * ROW : 16];
  __shared__ __align__(16) float adds[SETS][BUFFERS][NK];  // what is added to a key's score: its bias; -inf: it does not count
  __shared__ float stat_m[SETS][kRowTile], stat_l[SETS][kRowTile];
  __shared__ int odd_value;                               // a value that is not finite in a block whose keys not all rows see

  const int tid = threadIdx.x, wave = __builtin_amdgcn_readfirstlane(tid >> 6), lane = tid & 63, i32 = lane & 31, g = lane >> 5;
  const unsigned id = blockIdx.y * gridDim.x + blockIdx.x;
  if (id >= jobs.all) return;
  const unsigned which = PAGED && id >= jobs.first;
  const QueryArgs& a = jobs.q[which];
  const KeyArgs& kk = jobs.k[which];
  const unsigned tiles = jobs.tiles[which], at = in_dies<FEW>(id - (which ? jobs.first : 0u), (which ? jobs.all - jobs.first : jobs.first), tiles);
  const unsigned in_heads = at / tiles;
  const int chunk = (int)(in_heads / (unsigned)a.kv_heads), h = (int)(in_heads - (unsigned)chunk * a.kv_heads), tile = (int)(at - in_heads * tiles);
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
  if (CAUSAL && kk.causal) {
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
  const int32_t* table = PAGED ? kk.table + s * kk.table_stride : nullptr;
  const long long base = h * kk.pool.head_stride + key0 * kk.token_stride;
  const int stride = (int)held(kk.token_stride);          // (a block's rows lie within 2 GiB)
  const float scale = held(a.scale);
  const int page_shift = held(kk.pool.shift), pages = held(kk.pool.pages), slot_mask = held(kk.slot_mask);
  const long long page_stride = held(kk.pool.page_stride);

  // The pieces of LDS that this lane fills with load i: of row brought + AT_ONCE * SHARE * i (+ its own row of the AT_ONCE of a load), which lie
  // in one page. Pieces behind a head's channels stay zero.
  const int brought = __builtin_amdgcn_readfirstlane(share * AT_ONCE), own_row = lane / CH;
  auto key_from = [&](int i) STTM_INLINE { return 16 * (lane % CH ^ key_order<CH>(brought + AT_ONCE * S::SHARE * i + own_row)); };
  auto value_from = [&](int i) STTM_INLINE { return 16 * (lane % CH ^ value_order<DT, CH>(brought + AT_ONCE * S::SHARE * i + own_row)); };
  // Lane i: the page of key i of the block that is loaded next and its bias, looked up a block ahead; of the block on its way, what is added to the
  // key's score and where its row is. Keys from the end on: the page of the last one, whose other slots may be read.
  int page_next = 0;
  float bias_next = 0.f, add_now = 0.f;
  unsigned long long from_now = 0;                        // (packed: of the block's first row, the same in all lanes)
  int last_now = 0;                                       // (packed: of the last row there is, as seen from the block's first, or further)
  auto look_up = [&](int s0) STTM_INLINE {
    const int slot = min(s0 + min(lane, NK - 1), end - 1);
    if constexpr (PAGED) page_next = table[slot >> page_shift];
    if (bias) bias_next = bias[slot];
  };
  const char *const k_base = kk.pool.k + base, *const v_base = kk.pool.v + base;
  auto next_block = [&](int s0) STTM_INLINE {
    const bool there = !PAGED || (unsigned)page_next < (unsigned)pages;
    add_now = lane >= NK || s0 + lane >= end || !there ? -INFINITY : bias_next;
    if constexpr (PAGED) {                                // (what is read of a page that is not there does not count)
      const int slot = min(s0 + min(lane, NK - 1), end - 1) & slot_mask;
      from_now = (unsigned long long)(unsigned)(there ? page_next : 0) * (unsigned long long)page_stride + (unsigned long long)(unsigned)slot * (unsigned)stride;
    } else {
      from_now = (unsigned long long)(unsigned)s0 * (unsigned long long)kk.token_stride;
      last_now = min(end - 1 - s0, NK) * stride;
    }
  };
  // Load i of a block's keys, values. As many loads whatever the width, for the sake of those that count them: pieces behind a head's channels come
  // from a place of zeros. Pages: from the start of the load's rows, which lie in one page. Packed: from the block's first row, rows from the end on
  // the last one.
  const int own_from = own_row * stride;
  auto load_one = [&](auto what, int i, char* keys_to, char* values_to) STTM_INLINE {
    constexpr bool KEYS = decltype(what)::value & 1, VALUES = decltype(what)::value & 2;
    const int r = brought + AT_ONCE * S::SHARE * i, at = (set * NK + r) * ROW;
    unsigned long long from = from_now;
    unsigned row = own_from;
    if constexpr (PAGED) {
      from = (unsigned)__builtin_amdgcn_readlane((int)(unsigned)from_now, r) |
             (unsigned long long)(unsigned)__builtin_amdgcn_readlane((int)(unsigned)(from_now >> 32), r) << 32;
    } else {
      row = (unsigned)min(own_from + r * stride, last_now);
    }
    const char *k_from = k_base + from, *v_from = v_base + from;
    if constexpr (KEYS) to_lds(FULL || key_from(i) < kk.pool.row ? k_from + (row + key_from(i)) : kZeros, keys_to + at);
    if constexpr (VALUES) to_lds(FULL || value_from(i) < kk.pool.row ? v_from + (row + value_from(i)) : kZeros, values_to + at);
  };
  auto load = [&](auto what, char* keys_to, char* values_to) STTM_INLINE {
#pragma unroll
    for (int i = 0; i < PER; ++i) load_one(what, i, keys_to, values_to);
  };
  using Keys = std::integral_constant<int, 1>;
  using Values = std::integral_constant<int, 2>;
  using Both = std::integral_constant<int, 3>;

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
  float m = -INFINITY, from = 0.f, l = 0.f;  // from: m as an exponent of two; l: of this lane's keys
  if (tid == 0) odd_value = 0;
  const int start = first + set * NK, step = SETS * NK;
  if (start < end) {
    look_up(start);
    next_block(start);
    if constexpr (FEW) load(Keys(), keys0, values0);
    else load(Both(), keys0, values0);
    look_up(start + step);
    if constexpr (FEW) load(Values(), keys0, values0);
  }
  arrived<0>();                                           // (the queries, too, which the compiler would wait for with every block else)
  // A block's keys (values) that count for none of the rows, or values that are not finite where not all rows see them: nothing of those may be
  // infinite or NaN. Each wavefront sees to the pieces that it has loaded.
  auto mend = [&](char* at, unsigned long long alive, bool finite) STTM_INLINE {
    bool odd = false;
#pragma unroll
    for (int i = 0; i < PER; ++i) {
      const int r = brought + AT_ONCE * S::SHARE * i;
      w4* piece = reinterpret_cast<w4*>(at + r * ROW + 16 * lane);
      if (!(alive >> (r + own_row) & 1)) {
        *piece = w4{0u, 0u, 0u, 0u};
      } else if (finite) {
        w4 y = *piece;
#pragma unroll
        for (int e = 0; e < 4; ++e) {
          const uint32_t f = finite_only<DT>(y[e]);
          odd |= f != y[e];
          y[e] = f;
        }
        *piece = y;
      }
    }
    if (odd) odd_value = 1;
  };
  // One block. FEW: a wavefront has its block to itself, one buffer for keys and one for values; the next keys are on their way from the first
  // product on, the next values from the second.
  auto block = [&](int s0, bool more, bool diagonal, bool whole, unsigned long long alive, const char* keys, char* values, const float* added,
                   char* next_keys, char* next_values) STTM_INLINE {
    // Values, the first ones on their way while the softmax goes on: of step j the keys that one product takes (16, fp32: 1 a half).
    constexpr int STEPS = DT == 0 ? 16 * KT : NK / 16;
    w4 v[V_AHEAD][DT == 0 ? (M + 3) / 4 : M];
    auto read_values = [&](int j) STTM_INLINE {
#pragma unroll
      for (int n = 0; n < M; ++n) {
        if constexpr (DT == 0) {
          const char* at = values + value_at[n % NV_AT] + ((8 * (j / 4) + j % 4) * ROW + n / NV_AT * NV_AT * 128);
          v[j % V_AHEAD][n / 4][n % 4] = *reinterpret_cast<const uint32_t*>(at);
        } else {
          const w2 lo = tr_load(values + value_at[n] + 16 * j * ROW), hi = tr_load(values + value_at[n] + (16 * j + 8) * ROW);
          v[j % V_AHEAD][n] = w4{lo[0], lo[1], hi[0], hi[1]};
        }
      }
    };
    // S^T. The pieces of keys are read a few products ahead (a read takes as long as four of them).
    f32x16 x[KT];
#pragma unroll
    for (int t = 0; t < KT; ++t)
#pragma unroll
      for (int r = 0; r < 16; ++r) x[t][r] = 0.f;
    w4 k[K_AHEAD][KT];
    float4 add[KT * 4];
    auto read_keys = [&](int c) STTM_INLINE {
#pragma unroll
      for (int t = 0; t < KT; ++t)
        k[c % K_AHEAD][t] = *reinterpret_cast<const w4*>(keys + key_at[c % NK_AT] + (32 * t * ROW + c / NK_AT * NK_AT * 32));
    };
#pragma unroll
    for (int c = 0; c < K_AHEAD; ++c) read_keys(c);
    if constexpr (!FEW) __builtin_amdgcn_s_setprio(1);    // (products first: the SIMD's other wavefront does its softmax behind them)
#pragma unroll
    for (int c = 0; c < NQ; ++c) {
      __builtin_amdgcn_sched_barrier(0);
#pragma unroll
      for (int t = 0; t < KT; ++t) {
        if constexpr (DT == 0) {
#pragma unroll
          for (int e = 0; e < 4; ++e) x[t] = mma32(__uint_as_float(k[c % K_AHEAD][t][e]), __uint_as_float(q[c][e]), x[t]);
        } else {
          x[t] = mma16<DT>(k[c % K_AHEAD][t], q[c], x[t]);
        }
      }
      __builtin_amdgcn_sched_barrier(0);
      if (c + K_AHEAD < NQ) {
        read_keys(c + K_AHEAD);
      } else {                                            // (then what the softmax and the first product of values begin with)
#pragma unroll
        for (int i = 0; i < KT * 4; ++i)
          if (i * K_AHEAD / (KT * 4) == c + K_AHEAD - NQ) add[i] = *reinterpret_cast<const float4*>(&added[8 * i + 4 * g]);
        if (!FEW && c == NQ - 2) read_values(0);
      }
      if constexpr (!FEW) {                               // (the next block's loads while products go on)
#pragma unroll
        for (int i = 0; i < PER; ++i)
          if (i * NQ / PER == c) load_one(Both(), i, next_keys, next_values);
      }
    }
    if constexpr (!FEW) __builtin_amdgcn_s_setprio(0);
    if constexpr (FEW) {
      __builtin_amdgcn_sched_barrier(0);
      __builtin_amdgcn_wave_barrier();
      if (more) {
        next_block(s0 + step);
        load(Keys(), keys0, values0);
      }
    }
#pragma unroll
    for (int t = 0; t < KT; ++t)
#pragma unroll
      for (int r4 = 0; r4 < 4; ++r4) {
        x[t][4 * r4] = fmaf(x[t][4 * r4], scale, add[4 * t + r4].x);
        x[t][4 * r4 + 1] = fmaf(x[t][4 * r4 + 1], scale, add[4 * t + r4].y);
        x[t][4 * r4 + 2] = fmaf(x[t][4 * r4 + 2], scale, add[4 * t + r4].z);
        x[t][4 * r4 + 3] = fmaf(x[t][4 * r4 + 3], scale, add[4 * t + r4].w);
      }
    if (CAUSAL && diagonal) {
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
    top = of_halves(top);
    // What weights are relative to follows the maximum where that has risen by SLACK: of 32 rows one has a new maximum in most blocks.
    // (The difference, not the sum: that one is rounded, to m + 1 where scores are 2^23. -inf less -inf is no rise.)
    const bool rises = __ballot(top - m > SLACK) != 0;
    const float before = m, from_before = m == -INFINITY ? -INFINITY : from;
    m = rises ? fmaxf(m, top) : m;
    from = m == -INFINITY ? 0.f : m * kLog2e;
    // Large scores: no multiple of theirs, only of their differences. (A rounding of `from` times 2^-24 is what an exponent may be off else.)
    float less = LIFT - from;
    if (ONE_WAY || __ballot(!(fabsf(from) < 65536.f)) != 0) {
      less = LIFT;
#pragma unroll
      for (int t = 0; t < KT; ++t)
#pragma unroll
        for (int r = 0; r < 16; ++r) x[t][r] -= m == -INFINITY ? 0.f : m;
    }
    if (rises) {
      const float by = exp2_fast(fabsf(from) < 65536.f ? from_before - from : (before - m) * kLog2e);
      l *= by;
#pragma unroll
      for (int n = 0; n < M; ++n)
#pragma unroll
        for (int r = 0; r < 16; ++r) acc[n][r] *= by;
    }
    if constexpr (FEW) {
      if (more) arrived<PER>();                   // (all but the keys that come next)
      else arrived<0>();
      if (diagonal || !whole) {
        __builtin_amdgcn_wave_barrier();
        mend(values, alive, diagonal);
      }
      __builtin_amdgcn_wave_barrier();
      read_values(0);
    }
    // O^T, the exponentials of a step while the products of the one before it go on.
    constexpr int EACH = DT == 0 ? 1 : 8;                 // scores a lane has of one step
    w4 p[2];
    auto weigh = [&](int j) STTM_INLINE {
#pragma unroll
      for (int e = 0; e < EACH; ++e) {
        const int at = j * EACH % 16 + e;
        x[j * EACH / 16][at] = exp2_fast(fmaf(x[j * EACH / 16][at], kLog2e, less));
        l += x[j * EACH / 16][at];
      }
      if constexpr (DT != 0) {
#pragma unroll
        for (int w = 0; w < 4; ++w) p[j % 2][w] = pack2<DT>(x[j / 2][8 * (j % 2) + 2 * w], x[j / 2][8 * (j % 2) + 2 * w + 1]);
      }
    };
    weigh(0);
    if constexpr (!FEW) __builtin_amdgcn_s_setprio(1);
#pragma unroll
    for (int j = 0; j < STEPS; ++j) {
      __builtin_amdgcn_sched_barrier(0);
      if (j + 1 < STEPS) read_values(j + 1);
#pragma unroll
      for (int n = 0; n < M; ++n) {
        if constexpr (DT == 0) acc[n] = mma32(__uint_as_float(v[j % V_AHEAD][n / 4][n % 4]), x[j / 16][j % 16], acc[n]);
        else acc[n] = mma16<DT>(v[j % V_AHEAD][n], p[j % 2], acc[n]);
      }
      if (j + 1 < STEPS) weigh(j + 1);
      // (reads, then a product and what two of the next step's scores take, in turn)
      __builtin_amdgcn_sched_group_barrier(0x100, DT == 0 ? M : 2 * M, 0);
#pragma unroll
      for (int n = 0; n < M; ++n) {
        __builtin_amdgcn_sched_group_barrier(0x8, 1, 0);
        __builtin_amdgcn_sched_group_barrier(0x402, DT == 0 ? 4 : (28 + M - 1) / M, 0);
      }
    }
    if constexpr (!FEW) __builtin_amdgcn_s_setprio(0);
  };
  auto one = [&](int s0, char* keys, char* values, char* next_keys, char* next_values, float* added) STTM_INLINE {
    keys += set * NK * ROW;
    values += set * NK * ROW;
    const bool more = s0 + step < end;
    if (FEW) arrived<PER>();                              // (all but the values)
    else arrived<0>();
    const unsigned long long alive = __ballot(add_now != -INFINITY);
    const bool whole = alive == (NK == 64 ? ~0ull : 0xffffffffull);
    const bool diagonal = CAUSAL && s0 + NK > least && least < length;
    if (diagonal || !whole) {
      __builtin_amdgcn_wave_barrier();
      if (!whole) mend(keys, alive, false);
      if (!FEW) mend(values, alive, diagonal);
    }
    if (share == 0 && lane < NK) added[lane] = add_now;
    if constexpr (FEW) {
      __builtin_amdgcn_wave_barrier();
    } else {
      __syncthreads();
      next_block(more ? s0 + step : s0);                  // (behind the last block comes that one again: no way of its own for it)
    }
    block(s0, more, diagonal, whole, alive, keys, values, added, next_keys, next_values);
    if constexpr (!FEW) {
      look_up(s0 + 2 * step);
    } else {
      __builtin_amdgcn_sched_barrier(0);
      __builtin_amdgcn_wave_barrier();
      if (more) {
        look_up(s0 + 2 * step);
        load(Values(), keys0, values0);
      }
    }
  };
  if constexpr (FEW) {
    for (int s0 = start; s0 < end; s0 += step) one(s0, keys0, values0, nullptr, nullptr, adds[set][0]);
  } else {
    for (int s0 = start; s0 < end; s0 += 2 * step) {
      one(s0, keys0, values0, keys1, values1, adds[0][0]);
      if (s0 + step < end) one(s0 + step, keys1, values1, keys0, values0, adds[0][BUFFERS - 1]);
    }
  }
  arrived<0>();                                           // (nothing may come into LDS any more)
  settle();

  const bool parted = a.part && !(a.alone && length <= kk.chunk);
  l += __shfl_xor(l, 32, 64);
  l *= UNLIFT;
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
    if (parted) a.stat[index * a.parts + a.first_part + chunk] = make_float2(top, total);
    else if (a.lse) a.lse[index] = top + logf(total);
  }
  const float inverse = parted ? 1.f : total == 0.f ? 0.f : 1.f / total;
  float* part = parted ? a.part + (index * a.parts + a.first_part + chunk) * a.d : nullptr;
  char* out = parted ? nullptr : a.out + token * a.out_stride + (long long)head * a.d * ES;
  auto store = [&](int c, float4 y) STTM_INLINE {                     // four channels of this lane's row
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
    float4* joined = reinterpret_cast<float4*>(keys0);    // [wave][j][lane]
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
  if constexpr (CAUSAL) __syncthreads();                         // (odd_value, of all wavefronts)
  if (CAUSAL && odd_value) {
    // Values that are not finite were left out where some rows see them and others do not (a weight of zero does not make them
    // zero): the rows that see them get them here. What is infinite or NaN already stays so.
#pragma unroll 1
    for (int c = FEW ? 8 * wave + 4 * g : 4 * g; c < a.d && mine; c += FEW ? 8 * SETS : 8) {
      float add[4] = {0.f, 0.f, 0.f, 0.f};
#pragma unroll 1
      for (int i = max(first, least - NK + 1); i < min(end, limit); ++i) {
        const int page = PAGED ? table[i >> page_shift] : 0;
        if ((PAGED && (unsigned)page >= (unsigned)pages) || (bias && bias[i] == -INFINITY)) continue;
        const long long at = base + (PAGED ? page * page_stride + (i & slot_mask) * stride : i * kk.token_stride);
#pragma unroll
        for (int e = 0; e < 4; ++e) {
          float v;
          if constexpr (DT == 0) v = *reinterpret_cast<const float*>(kk.pool.v + at + 4 * (c + e));
          else v = low_half<DT>(*reinterpret_cast<const uint16_t*>(kk.pool.v + at + 2 * (c + e)));
          if (!(fabsf(v) < INFINITY)) add[e] += v;
        }
      }
      float* to = part ? part : DT == 0 ? reinterpret_cast<float*>(out) : nullptr;
      if (to) {
        const float4 y = *reinterpret_cast<const float4*>(to + c);
        *reinterpret_cast<float4*>(to + c) = make_float4(y.x + add[0], y.y + add[1], y.z + add[2], y.w + add[3]);
      } else if constexpr (DT != 0) {
        const uint2 y = *reinterpret_cast<const uint2*>(out + 2 * c);
        *reinterpret_cast<uint2*>(out + 2 * c) = make_uint2(pack2<DT>(low_half<DT>(y.x) + add[0], high_half<DT>(y.x) + add[1]),
                                                            pack2<DT>(low_half<DT>(y.y) + add[2], high_half<DT>(y.y) + add[3]));
      }
    }
  }
}

template <int DT, int DP, bool FEW, bool PAGED>
void launch_tiles(const QueryJobs& jobs, hipStream_t s) {
  const unsigned wide = std::min(jobs.all, 1u << 20);     // (fewer than 2^32 threads along a side of the grid)
  const dim3 grid(wide, (jobs.all + wide - 1) / wide), block(Shape<DT, DP, FEW>::THREADS);
  if (jobs.k[0].pool.row == Shape<DT, DP, FEW>::ROW) hipLaunchKernelGGL((k_query_tiles<DT, DP, FEW, PAGED, true>), grid, block, 0, s, jobs);
  else hipLaunchKernelGGL((k_query_tiles<DT, DP, FEW, PAGED, false>), grid, block, 0, s, jobs);
}

template <int DT, int DP>
void launch_width(const QueryJobs& jobs, bool few, hipStream_t s) {
  const bool paged = !jobs.k[0].offsets;
  if (few) paged ? launch_tiles<DT, DP, true, true>(jobs, s) : launch_tiles<DT, DP, true, false>(jobs, s);
  else paged ? launch_tiles<DT, DP, false, true>(jobs, s) : launch_tiles<DT, DP, false, false>(jobs, s);
}

}  // namespace

template <int DT> void launch_queries(QueryJobs& jobs, bool few_rows, hipStream_t s) {
  jobs.all = 0;
  for (int i = 0; i < jobs.count; ++i) {
    const QueryArgs& a = jobs.q[i];
    jobs.tiles[i] = (unsigned)(a.tokens * a.group / query_tile(few_rows) + a.segments);
    jobs.first = jobs.all;
    jobs.all += jobs.tiles[i] * a.kv_heads * jobs.k[i].chunks;
  }
  if (jobs.count == 1) jobs.first = jobs.all;
  const int d = jobs.q[0].d;
  if (d <= 64) launch_width<DT, 64>(jobs, few_rows, s);
  else if (d <= 96) launch_width<DT, 96>(jobs, few_rows, s);
  else if (d <= 128) launch_width<DT, 128>(jobs, few_rows, s);
  else if (d <= 192) launch_width<DT, 192>(jobs, few_rows, s);
  else launch_width<DT, 256>(jobs, few_rows, s);
}

}  // namespace sttm
