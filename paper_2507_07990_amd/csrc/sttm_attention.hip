// Attention of one new token of every sequence over a paged cache, split over the cache's length and joined.
#include "sttm_cache.h"

#include <algorithm>
#include <cmath>

namespace sttm {
namespace {

constexpr int kAttnThreads = 256, kAttnWaves = kAttnThreads / kWave;
constexpr int kQTile = 16;      // heads of a group that one matrix product takes
// Slots of one workgroup at most. (A host-thread build of the tests sets fewer, for many chunks of short sequences.)
#ifndef STTM_CHUNK_MAX
#define STTM_CHUNK_MAX 512
#endif
constexpr int kChunkMax = STTM_CHUNK_MAX, kChunkMid = kChunkMax / 2, kChunkLeast = kChunkMax / 4;
constexpr float kLog2e = 1.4426950408889634f;

typedef float f32x4 __attribute__((vector_size(16)));
typedef uint32_t u32x4 __attribute__((vector_size(16)));

// ---- products on the matrix cores ---------------------------------------------------------------------------
// D[m][n] += sum_k A[m][k] B[k][n], m, n < 16. A lane (i = lane % 16, g = lane / 16) holds A[i][*] and B[*][i] for the k of
// its group g: eight 16-bit ones (v_mfma_f32_16x16x32) or one fp32 (v_mfma_f32_16x16x4), and D[4g + r][i], r < 4. Which k a
// place stands for is free as long as A and B agree.
#ifndef STTM_HOST_EMULATION
template <int DT> __device__ inline f32x4 mma16(u32x4 a, u32x4 b, f32x4 c) {
  typedef float v4 __attribute__((ext_vector_type(4)));
  if constexpr (DT == 1) {
    typedef __bf16 v8 __attribute__((ext_vector_type(8)));
    return __builtin_bit_cast(f32x4, __builtin_amdgcn_mfma_f32_16x16x32_bf16(__builtin_bit_cast(v8, a), __builtin_bit_cast(v8, b), __builtin_bit_cast(v4, c), 0, 0, 0));
  } else {
    typedef _Float16 v8 __attribute__((ext_vector_type(8)));
    return __builtin_bit_cast(f32x4, __builtin_amdgcn_mfma_f32_16x16x32_f16(__builtin_bit_cast(v8, a), __builtin_bit_cast(v8, b), __builtin_bit_cast(v4, c), 0, 0, 0));
  }
}
__device__ inline f32x4 mma32(float a, float b, f32x4 c) {
  typedef float v4 __attribute__((ext_vector_type(4)));
  return __builtin_bit_cast(f32x4, __builtin_amdgcn_mfma_f32_16x16x4f32(a, b, __builtin_bit_cast(v4, c), 0, 0, 0));
}
// (a's and b's 16-bit halves of one kind side by side, a's first)
__device__ inline uint32_t low_halves(uint32_t a, uint32_t b) { return __builtin_amdgcn_perm(b, a, 0x05040100u); }
__device__ inline uint32_t high_halves(uint32_t a, uint32_t b) { return __builtin_amdgcn_perm(b, a, 0x07060302u); }
#else
struct EmulOperands { u32x4 a[64], b[64]; };
inline EmulOperands& emul_operands() {
  static EmulOperands of_wave[16];
  return of_wave[threadIdx.x >> 6];
}
template <int DT> inline f32x4 mma16(u32x4 a, u32x4 b, f32x4 c) {
  EmulOperands& e = emul_operands();
  const int lane = threadIdx.x & 63;
  e.a[lane] = a;
  e.b[lane] = b;
  hip_emul::wave_sync();
  for (int r = 0; r < 4; ++r) {
    float sum = c[r];
    for (int g = 0; g < 4; ++g)
      for (int w = 0; w < 4; ++w) {
        const uint32_t x = e.a[g * 16 + 4 * (lane / 16) + r][w], y = e.b[g * 16 + lane % 16][w];
        sum += low_half<DT>(x) * low_half<DT>(y) + high_half<DT>(x) * high_half<DT>(y);
      }
    c[r] = sum;
  }
  hip_emul::wave_sync();
  return c;
}
inline f32x4 mma32(float a, float b, f32x4 c) {
  EmulOperands& e = emul_operands();
  const int lane = threadIdx.x & 63;
  e.a[lane][0] = __float_as_uint(a);
  e.b[lane][0] = __float_as_uint(b);
  hip_emul::wave_sync();
  for (int r = 0; r < 4; ++r)
    for (int g = 0; g < 4; ++g)
      c[r] += __uint_as_float(e.a[g * 16 + 4 * (lane / 16) + r][0]) * __uint_as_float(e.b[g * 16 + lane % 16][0]);
  hip_emul::wave_sync();
  return c;
}
inline uint32_t low_halves(uint32_t a, uint32_t b) { return (a & 0xffffu) | (b << 16); }
inline uint32_t high_halves(uint32_t a, uint32_t b) { return (a >> 16) | (b & 0xffff0000u); }
#endif

struct AttnArgs {
  Pool pool;
  Seqs seqs;
  const char* q;
  char* out;
  long long q_stride, out_stride;  // bytes
  const float *bias, *weights_in;
  float *weights_out, *lse;
  long long slot_stride;
  float* logits;     // [batch, kv_heads, max_len, group]: s_j (weights wanted), else NULL
  float* part;       // [batch, q_heads, chunks, d]: unnormalised sums of the chunks (more than one chunk), else NULL
  float2* stat;      // [batch, q_heads, chunks]: largest s and sum of exponentials of a chunk
  float scale;
  int kv_heads, group, d, chunk, chunks, tiles;
};

// Softmax statistics of one head over several parts of the slots. (s is kept as it is and differences are multiplied by log2(e): s
// itself may be the lowest fp32 number, or near the largest, and has no multiple then.)
__device__ inline float factor(float m, float top) { return exp2_fast((m - (top == -INFINITY ? 0.f : top)) * kLog2e); }

// The logarithm of a sum of exponentials (-inf: of none; the largest s does not show a NaN, the sum does).
__device__ inline float log_sum(float m, float total) { return m + logf(total); }

// A slot's elements as one lane takes them, in loads of 16 bytes (8 bytes: VW == 4 of 16 bits). ONCE: marked as used once; only
// where rows are made of whole lines, which sixteen lanes take at a time. A lane whose share lies beyond the row takes the
// row's start in its place: what it makes of that is not written.
template <int DT, int VW> struct ValueRow {
  static constexpr int WORDS = DT == 0 ? VW : VW / 2;
  uint32_t w[WORDS];
  template <bool ONCE = false> __device__ inline void load(const char* row, int i, int bytes) {  // i: lane % 16
    if constexpr (DT != 0 && VW == 4) {
      const uint2 x = *reinterpret_cast<const uint2*>(row + (i * 8 < bytes ? i * 8 : 0));
      w[0] = x.x; w[1] = x.y;
    } else {
#pragma unroll
      for (int h = 0; h < WORDS / 4; ++h) {
        const int o = i * 16 + h * 256;
        const uint4* at = reinterpret_cast<const uint4*>(row + (o < bytes ? o : 0));
        const uint4 x = ONCE ? load_once(at) : *at;
        w[4 * h] = x.x; w[4 * h + 1] = x.y; w[4 * h + 2] = x.z; w[4 * h + 3] = x.w;
      }
    }
  }
  __device__ inline void clear() {
#pragma unroll
    for (int i = 0; i < WORDS; ++i) w[i] = 0u;
  }
};

// Where the sum of channel c (a multiple of 4; the three channels after it are 4 lines further each) is among what a
// wavefront leaves in LDS, 64 * line + lane of head 0: lane m of sixteen holds a row's channels m*RUN .. in a load, channel
// m*RUN + n is row m of product n, and row 4g + r of product n is line 4n + r of lanes 16g ...
template <int DT, int VW> __device__ inline int value_place(int c) {
  constexpr int RUN = DT == 0 || VW == 4 ? 4 : 8;
  const int m = c % (16 * RUN) / RUN, n = c / (16 * RUN) * RUN + c % RUN;
  return 64 * (4 * n + m % 4) + 16 * (m / 4);
}

template <int DT> __device__ inline void store_channels(char* at, const float (&x)[4]) {
  if constexpr (DT == 0) *reinterpret_cast<float4*>(at) = make_float4(x[0], x[1], x[2], x[3]);
  else *reinterpret_cast<uint2*>(at) = make_uint2(pack2<DT>(x[0], x[1]), pack2<DT>(x[2], x[3]));
}

// One workgroup: one chunk of the slots of one (sequence, kv head, tile of 16 of the group's heads). Its wavefronts take
// blocks of 32 slots (fp32: 16) in turn, each with its own running maximum and sum; at the end the four are joined in LDS.
//
// Both products are laid out so that nothing changes lanes between them: S = K Q^T has slots as rows and heads as columns,
// a lane ends up with the slots 4g + r of each tile of 16 for head lane % 16; these are the k of its group in the second
// product, O^T = V^T P^T, whose A operand a lane fills from the rows of the same slots, loaded as they lie in memory (16
// lanes a row): channel lane * 8 + n is row `lane` of product n. The 16-bit transposition that is left is between registers
// of one lane, one v_perm for two elements.
//
// P is handed on as the sum of two 16-bit numbers (16 bits of mantissa with bf16; 22 with fp16, and as 2^15 P, so that a weight is
// off by no more than 2^-40 of the largest one where fp16 runs out of exponents), one product each: rounding it to one alone would
// cost as much accuracy as the result's own rounding. (The smaller number may be zero or negative, and makes NaN of
// an infinite value: where a sum is NaN the infinite values of its channel are looked up at the end. Nothing else is spent on them.)
//
// Keys of the next block are loaded once this one's are used up, values likewise: no second set of registers, and there
// are always some on their way. Up to 128 channels two wavefronts a SIMD bound the registers to 256, which keeps the sums out of
// the accumulation registers that only copies reach. Above, one wavefront a SIMD has them there in part (8 sequences of 16,384 slots,
// 4 kv heads of 256 channels: bf16 137 us, bound to 256 registers 139; fp32 226 and 310; but bf16 heads of 192 119 and 93).
//
// Bound by memory: 24 sequences of 901 to 25,977 slots, 64 heads on 8 of 128 bf16 channels, are 760 MB in 142 us (5.3 TB/s; the
// matrix units are busy a twentieth of the time); one of 43,328 slots, 28 heads on 4, with scores kept, 90 MB in 21 us.
template <int DT, int NQ, int VW, bool BIAS>
__global__ void __launch_bounds__(kAttnThreads, VW == 16 ? 1 : 2) k_paged_attention(AttnArgs a) {
  constexpr int ES = DT == 0 ? 4 : 2, TILES = DT == 0 ? 1 : 2, BLOCK = 16 * TILES, PART = VW < 8 ? VW : 8;
  constexpr int PIECES = DT == 0 ? NQ / 2 : NQ;  // (of 32 channels; the shortest row this instance is chosen for:)
  // Values past the caches where a head's row is a number of whole lines (146 us against 155 on the ragged batch of 24
  // sequences; fp32 rows of 288 bytes took 32 against 23). Not the keys: their pieces of 64 bytes come by a line twice.
  constexpr bool ONCE = DT != 0 && PIECES != 1 && PIECES != 3 && PIECES != 6;
  constexpr float LIFT = DT == 2 ? 15.f : 0.f;  // the largest weight is 2^LIFT while it is summed up (fp16 ends at 2^16)
  constexpr int LEAST = ES * (PIECES <= 4 ? 32 * PIECES - 24 : PIECES == 6 ? 136 : 200);

  __shared__ long long page_at[kChunkMax / 8];        // byte offset of every page of the chunk, -1: not in the pool
  __shared__ float joined[kAttnWaves][PART * 4][kWave];  // the wavefronts' sums, a part of the channels at a time
  __shared__ float stat_m[kAttnWaves][kQTile], stat_l[kAttnWaves][kQTile];
  __shared__ float2 all_heads[kQTile];  // maximum and reciprocal sum

  const int b = blockIdx.z, h = blockIdx.y / a.tiles, tile = blockIdx.y % a.tiles, chunk = blockIdx.x;
  const int length = seq_length(a.seqs, b);
  const int first = chunk * a.chunk;
  if (first >= length && chunk > 0) return;  // (an empty sequence's first chunk is gone through: its result is written)
  const int end = min(length, first + a.chunk);
  const int tid = threadIdx.x, wave = __builtin_amdgcn_readfirstlane(tid >> 6), lane = tid & 63, i16 = lane & 15, g = lane >> 4;
  const int head0 = tile * kQTile, heads = min(kQTile, a.group - head0);

  for (int p = tid; p << a.pool.shift < end - first; p += kAttnThreads) {
    const int page = a.seqs.table[b * a.seqs.table_stride + (first >> a.pool.shift) + p];
    const bool ok = page >= 0 && page < a.pool.pages;
    page_at[p] = ok ? page * a.pool.page_stride + h * a.pool.head_stride : -1;
  }

  // The tile's queries, as the B operand: column i16, the k of group g.
  u32x4 q[NQ];
  {
    const char* row = a.q + b * a.q_stride + ((long long)h * a.group + head0 + min(i16, heads - 1)) * a.d * ES;
#pragma unroll
    for (int c = 0; c < NQ; ++c) {
      const int o = (c * 4 + g) * 16;
      uint4 x = make_uint4(0u, 0u, 0u, 0u);
      if (i16 < heads && o < a.pool.row) x = *reinterpret_cast<const uint4*>(row + o);
      q[c] = u32x4{x.x, x.y, x.z, x.w};
    }
  }
  __syncthreads();

  f32x4 acc[VW];
#pragma unroll
  for (int n = 0; n < VW; ++n) acc[n] = f32x4{0.f, 0.f, 0.f, 0.f};
  float m = -INFINITY, l = 0.f;  // l: of this lane's slots
  const int page_mask = (1 << a.pool.shift) - 1;
  const float* bias = BIAS ? a.bias + ((long long)b * a.kv_heads + h) * a.slot_stride : nullptr;
  float* logits = a.logits ? a.logits + ((long long)b * a.kv_heads + h) * a.seqs.max_len * a.group + head0 : nullptr;

  // keys: lane i16 has the row of slot s0 + 16t + i16, its group's channels; values: slots s0 + 16t + 4g + r. Slots from the
  // end on are read as the last one. Loads stand without a branch around them: they are on their way together.
  u32x4 k[TILES][NQ];
  ValueRow<DT, VW> v[TILES][4];
  bool outside = false, dead_next[TILES][4];
  float add_next[TILES][4];
  auto load_keys = [&](int s0) {
    outside = false;
#pragma unroll
    for (int t = 0; t < TILES; ++t)
#pragma unroll
      for (int r = 0; r < 4; ++r) {
        const int slot = s0 + 16 * t + 4 * g + r;
        add_next[t][r] = BIAS ? bias[min(slot, end - 1)] : 0.f;
        dead_next[t][r] = slot >= end;
      }
#pragma unroll
    for (int t = 0; t < TILES; ++t) {
      const int slot = min(s0 + 16 * t + i16, end - 1);
      const long long at = page_at[(slot - first) >> a.pool.shift];
      outside |= at < 0;
      const char* row = a.pool.k + (at < 0 ? 0 : at) + (slot & page_mask) * a.pool.token_stride;
#pragma unroll
      for (int c = 0; c < NQ; ++c) {
        const int o = (c * 4 + g) * 16;
        const bool part = (c + 1) * 64 > LEAST;  // (the row may end in this piece)
        const uint4 x = *reinterpret_cast<const uint4*>(row + (part && o >= a.pool.row ? 0 : o));
        k[t][c] = u32x4{x.x, x.y, x.z, x.w};
        if (part && o >= a.pool.row) k[t][c] = u32x4{0u, 0u, 0u, 0u};
      }
    }
  };
  bool gone[TILES][4];
  auto load_values = [&](int s0) {
#pragma unroll
    for (int t = 0; t < TILES; ++t)
#pragma unroll
      for (int r = 0; r < 4; ++r) {
        const int slot = s0 + 16 * t + 4 * g + r, in = min(slot, end - 1);
        const long long at = page_at[(in - first) >> a.pool.shift];
        gone[t][r] = at < 0;
        v[t][r].template load<ONCE>(a.pool.v + (at < 0 ? 0 : at) + (in & page_mask) * a.pool.token_stride, i16, a.pool.row);
      }
  };
  const int start = first + wave * BLOCK;
  if (start < end) {
    load_keys(start);
    load_values(start);
  }
  for (int s0 = start; s0 < end; s0 += kAttnWaves * BLOCK) {
    const bool careful = BIAS || s0 + BLOCK > end || __ballot(outside) != 0;  // (the same in all lanes: masked slots among these)
    bool dead[TILES][4];
    float add[TILES][4];
#pragma unroll
    for (int t = 0; t < TILES; ++t)
#pragma unroll
      for (int r = 0; r < 4; ++r) {
        add[t][r] = add_next[t][r];
        dead[t][r] = dead_next[t][r] || gone[t][r] || (BIAS && add[t][r] == -INFINITY);
      }
    auto clear_dead = [&]() {
#pragma unroll
      for (int t = 0; t < TILES; ++t)
#pragma unroll
        for (int r = 0; r < 4; ++r)
          if (dead[t][r]) v[t][r].clear();
    };
    if (!BIAS && careful) clear_dead();  // (no branch between the products and what reads them: this compiler puts no wait
                                         // states across one, and the result would be read before it is there)
    f32x4 s[TILES];
#pragma unroll
    for (int t = 0; t < TILES; ++t) {
      s[t] = f32x4{0.f, 0.f, 0.f, 0.f};
      f32x4 part[2] = {s[t], s[t]};  // (fp32: two chains of products, each waits for its own)
#pragma unroll
      for (int c = 0; c < NQ; ++c) {
        if constexpr (DT == 0) {
#pragma unroll
          for (int j = 0; j < 4; ++j) part[j % 2] = mma32(__uint_as_float(k[t][c][j]), __uint_as_float(q[c][j]), part[j % 2]);
        } else {
          s[t] = mma16<DT>(k[t][c], q[c], s[t]);
        }
      }
      if constexpr (DT == 0) s[t] = part[0] + part[1];
    }
    load_keys(s0 + kAttnWaves * BLOCK);  // (the next block's, while this one goes on; past the end the last slot)
    float top = -INFINITY;
#pragma unroll
    for (int t = 0; t < TILES; ++t)
#pragma unroll
      for (int r = 0; r < 4; ++r) {
        float x = BIAS ? fmaf(s[t][r], a.scale, add[t][r]) : s[t][r] * a.scale;
        if (careful && dead[t][r]) x = -INFINITY;
        s[t][r] = x;
        top = fmaxf(top, x);
      }
    if (logits) {
#pragma unroll
      for (int t = 0; t < TILES; ++t)
#pragma unroll
        for (int r = 0; r < 4; ++r)
          if (i16 < heads && s0 + 16 * t + 4 * g + r < end) logits[(long long)(s0 + 16 * t + 4 * g + r) * a.group + i16] = s[t][r];
    }
    top = fmaxf(top, __shfl_xor(top, 16, 64));
    top = fmaxf(top, __shfl_xor(top, 32, 64));
    if (__ballot(top > m) != 0) {  // (seldom after the first blocks)
      const float m2 = fmaxf(m, top), shrink = factor(m, m2);
      m = m2;
      l *= shrink;
#pragma unroll
      for (int n = 0; n < VW; ++n)
#pragma unroll
        for (int r = 0; r < 4; ++r) acc[n][r] *= shrink;
    }
    const float base = m == -INFINITY ? 0.f : m;
    float p[TILES][4];
#pragma unroll
    for (int t = 0; t < TILES; ++t)
#pragma unroll
      for (int r = 0; r < 4; ++r) {
        p[t][r] = exp2_fast(DT == 2 ? fmaf(s[t][r] - base, kLog2e, LIFT) : (s[t][r] - base) * kLog2e);
        l += p[t][r];
      }
    if constexpr (BIAS) clear_dead();
    if constexpr (DT == 0) {
#pragma unroll
      for (int n = 0; n < VW; ++n)
#pragma unroll
        for (int r = 0; r < 4; ++r) acc[n] = mma32(__uint_as_float(v[0][r].w[n]), p[0][r], acc[n]);
    } else {
      u32x4 hi, lo;
#pragma unroll
      for (int j = 0; j < 4; ++j) {
        const float x = p[j / 2][j % 2 * 2], y = p[j / 2][j % 2 * 2 + 1];
        hi[j] = pack2<DT>(x, y);
        lo[j] = pack2<DT>(x - low_half<DT>(hi[j]), y - high_half<DT>(hi[j]));
      }
#pragma unroll
      for (int n = 0; n < VW; ++n) {
        u32x4 x;
#pragma unroll
        for (int j = 0; j < 4; ++j) {
          const uint32_t e = v[j / 2][j % 2 * 2].w[n / 2], f = v[j / 2][j % 2 * 2 + 1].w[n / 2];
          x[j] = n % 2 ? high_halves(e, f) : low_halves(e, f);
        }
        acc[n] = mma16<DT>(x, hi, acc[n]);
        acc[n] = mma16<DT>(x, lo, acc[n]);
      }
    }
    load_values(s0 + kAttnWaves * BLOCK);
  }

  // Four channels' sums, some of them NaN though no weight is: those get their infinite values in slots that count (whose weights are
  // above zero), if they have any. (One short loop out of the way: code that is seldom run, unrolled in place, cost every call 0.5 us.)
  auto look_up_infinite = [&](int channel, float (&x)[4]) {
    float sum[4] = {0.f, 0.f, 0.f, 0.f};
#pragma unroll 1
    for (int slot = first; slot < end; ++slot) {
      const long long at = page_at[(slot - first) >> a.pool.shift];
      const uint2 v4 = *reinterpret_cast<const uint2*>(a.pool.v + (at < 0 ? 0 : at) + (slot & page_mask) * a.pool.token_stride + channel * 2);
      const float f[4] = {low_half<DT>(v4.x), high_half<DT>(v4.x), low_half<DT>(v4.y), high_half<DT>(v4.y)};
      const bool masked = at < 0 || (BIAS && bias[slot] == -INFINITY);
#pragma unroll
      for (int e = 0; e < 4; ++e) sum[e] += masked || fabsf(f[e]) < INFINITY ? 0.f : f[e];
    }
#pragma unroll
    for (int e = 0; e < 4; ++e)
      if (x[e] != x[e] && sum[e] != 0.f) x[e] = sum[e];
  };

  // The wavefronts' sums on a common maximum, added up in their order.
  constexpr float UNLIFT = DT == 2 ? 1.f / 32768.f : 1.f;
  l += __shfl_xor(l, 16, 64);
  l += __shfl_xor(l, 32, 64);
  l *= UNLIFT;
  if (lane < kQTile) {
    stat_m[wave][lane] = m;
    stat_l[wave][lane] = l;
  }
  __syncthreads();
  float top = stat_m[0][i16];
#pragma unroll
  for (int w = 1; w < kAttnWaves; ++w) top = fmaxf(top, stat_m[w][i16]);
  const float mine = factor(m, top) * UNLIFT;
  float total = 0.f;
#pragma unroll
  for (int w = 0; w < kAttnWaves; ++w) total += stat_l[w][i16] * factor(stat_m[w][i16], top);
  const long long head = ((long long)b * a.kv_heads + h) * a.group + head0 + i16;
  if (tid < heads) {
    if (a.stat) a.stat[head * a.chunks + chunk] = make_float2(top, total);
    if (!a.part && a.lse) a.lse[head] = log_sum(top, total);
  }
  const float share = a.part ? 1.f : total == 0.f ? 0.f : 1.f / total;
  if (logits && !a.stat) {  // one chunk and one tile: every slot's weight from here
    if (tid < heads) all_heads[tid] = make_float2(top == -INFINITY ? 0.f : top, share);
    __syncthreads();
    const long long slots = ((long long)b * a.kv_heads + h) * a.slot_stride;
    for (int slot = tid; slot < end; slot += kAttnThreads) {
      float sum = 0.f;
      for (int i = 0; i < heads; ++i) sum = fmaf(exp2_fast((logits[(long long)slot * a.group + i] - all_heads[i].x) * kLog2e), all_heads[i].y, sum);
      a.weights_out[slots + slot] = (a.weights_in ? a.weights_in[slots + slot] : 0.f) + sum;
    }
  }
#pragma unroll
  for (int n0 = 0; n0 < VW; n0 += PART) {
    if (n0) __syncthreads();
#pragma unroll
    for (int n = 0; n < PART; ++n)
#pragma unroll
      for (int r = 0; r < 4; ++r) joined[wave][n * 4 + r][lane] = acc[n0 + n][r] * mine;
    __syncthreads();
    // four channels a thread, head i16 as before
    for (int u = tid >> 4; u < 4 * PART; u += kAttnThreads / 16) {
      const int channel = 16 * n0 + 4 * u, place = value_place<DT, VW>(4 * u);
      if (i16 >= heads || channel >= a.d) continue;
      float x[4];
#pragma unroll
      for (int e = 0; e < 4; ++e) {
        x[e] = 0.f;
#pragma unroll
        for (int w = 0; w < kAttnWaves; ++w) x[e] += joined[w][(place >> 6) + 4 * e][(place & 63) + i16];
        x[e] *= share;
      }
      if constexpr (DT != 0) {
        const float all = (x[0] + x[1]) + (x[2] + x[3]);
        if (__builtin_expect(all != all && total == total, 0)) look_up_infinite(channel, x);
      }
      if (a.part) *reinterpret_cast<float4*>(a.part + (head * a.chunks + chunk) * a.d + channel) = make_float4(x[0], x[1], x[2], x[3]);
      else store_channels<DT>(a.out + b * a.out_stride + (((long long)h * a.group + head0 + i16) * a.d + channel) * ES, x);
    }
  }
}

// The sum over the sixteen lanes of a row, the same bits in each of them.
__device__ inline float row16_sum(float v) {
#ifndef STTM_HOST_EMULATION
  v += __uint_as_float(__builtin_amdgcn_update_dpp(0, __float_as_uint(v), 0x128, 0xF, 0xF, true));  // row_ror:8
  v += __uint_as_float(__builtin_amdgcn_update_dpp(0, __float_as_uint(v), 0x124, 0xF, 0xF, true));
  v += __uint_as_float(__builtin_amdgcn_update_dpp(0, __float_as_uint(v), 0x122, 0xF, 0xF, true));
  v += __uint_as_float(__builtin_amdgcn_update_dpp(0, __float_as_uint(v), 0x121, 0xF, 0xF, true));
#else
  for (int o = 8; o > 0; o >>= 1) v += __shfl_xor(v, o, 64);
#endif
  return v;
}

// fp32 with one or two heads a kv head: of the sixteen columns of a matrix product one or two would be of use, and in fp32
// that is what bounds it (56 products of 32 cycles for 16 slots of 72 channels). Here sixteen lanes have a slot's row, keys and
// values alike, a wavefront four rows at a time, and each sixteen lanes their own running maximum and sum over their slots.
// 5 sequences of 333 to 4,979 slots, 16 heads of 72 with counts: 92 MB in 23 us, 32 by matrix products.
template <int HEADS, int VW, bool BIAS>
__global__ void __launch_bounds__(kAttnThreads, 2) k_paged_attention_rows(AttnArgs a) {
  constexpr int ROWS = 4, BLOCK = 4 * ROWS;  // rows of sixteen lanes under way together
  __shared__ long long page_at[kChunkMax / 8];
  __shared__ float joined[kAttnWaves][HEADS][VW][16];
  __shared__ float stat_m[4 * kAttnWaves][HEADS], stat_l[4 * kAttnWaves][HEADS];
  __shared__ float2 all_heads[HEADS];
  const int b = blockIdx.z, h = blockIdx.y, chunk = blockIdx.x;
  const int length = seq_length(a.seqs, b), first = chunk * a.chunk;
  if (first >= length && chunk > 0) return;
  const int end = min(length, first + a.chunk);
  const int tid = threadIdx.x, wave = __builtin_amdgcn_readfirstlane(tid >> 6), lane = tid & 63, i16 = lane & 15, g = lane >> 4;
  for (int p = tid; p << a.pool.shift < end - first; p += kAttnThreads) {
    const int page = a.seqs.table[b * a.seqs.table_stride + (first >> a.pool.shift) + p];
    const bool ok = page >= 0 && page < a.pool.pages;
    page_at[p] = ok ? page * a.pool.page_stride + h * a.pool.head_stride : -1;
  }
  // Channel 64 * (n / 4) + 4 * i16 + n % 4 of each head; zero beyond the row, and for a head that is not there.
  float q[HEADS][VW], acc[HEADS][VW], m[HEADS], l[HEADS];
#pragma unroll
  for (int e = 0; e < HEADS; ++e) {
    const char* row = a.q + b * a.q_stride + ((long long)h * a.group + min(e, a.group - 1)) * a.d * 4;
    ValueRow<0, VW> x;
    x.load(row, i16, a.pool.row);
#pragma unroll
    for (int n = 0; n < VW; ++n) {
      q[e][n] = 64 * (n / 4) + 4 * i16 < a.d ? __uint_as_float(x.w[n]) : 0.f;
      acc[e][n] = 0.f;
    }
    m[e] = -INFINITY;
    l[e] = 0.f;
  }
  __syncthreads();
  const int page_mask = (1 << a.pool.shift) - 1;
  const float* bias = BIAS ? a.bias + ((long long)b * a.kv_heads + h) * a.slot_stride : nullptr;
  float* logits = a.logits ? a.logits + ((long long)b * a.kv_heads + h) * a.seqs.max_len * a.group : nullptr;
  ValueRow<0, VW> k[ROWS], v[ROWS];
  float add[ROWS];
  bool dead[ROWS];
  auto load = [&](int s0) {  // (slots from the end on are read as the last one)
#pragma unroll
    for (int r = 0; r < ROWS; ++r) {
      const int slot = s0 + ROWS * g + r, in = min(slot, end - 1);
      const long long at = page_at[(in - first) >> a.pool.shift];
      const long long off = (at < 0 ? 0 : at) + (in & page_mask) * a.pool.token_stride;
      add[r] = BIAS ? bias[in] : 0.f;
      dead[r] = slot >= end || at < 0;
      k[r].load(a.pool.k + off, i16, a.pool.row);
      v[r].load(a.pool.v + off, i16, a.pool.row);
    }
  };
  const int start = first + wave * BLOCK;
  if (start < end) load(start);
  for (int s0 = start; s0 < end; s0 += kAttnWaves * BLOCK) {
    float s[HEADS][ROWS], p[HEADS][ROWS];
    bool gone[ROWS];
#pragma unroll
    for (int r = 0; r < ROWS; ++r) {
      gone[r] = dead[r] || (BIAS && add[r] == -INFINITY);
#pragma unroll
      for (int e = 0; e < HEADS; ++e) {
        float x = 0.f;
#pragma unroll
        for (int n = 0; n < VW; ++n)
          x = fmaf(64 * (n / 4) + 4 * i16 < a.d ? __uint_as_float(k[r].w[n]) : 0.f, q[e][n], x);
        x = row16_sum(x);
        x = BIAS ? fmaf(x, a.scale, add[r]) : x * a.scale;
        s[e][r] = gone[r] ? -INFINITY : x;
      }
    }
    if (logits) {
#pragma unroll
      for (int r = 0; r < ROWS; ++r)
#pragma unroll
        for (int e = 0; e < HEADS; ++e)
          if (i16 == e && e < a.group && s0 + ROWS * g + r < end) logits[(long long)(s0 + ROWS * g + r) * a.group + e] = s[e][r];
    }
#pragma unroll
    for (int e = 0; e < HEADS; ++e) {
      float top = m[e];
#pragma unroll
      for (int r = 0; r < ROWS; ++r) top = fmaxf(top, s[e][r]);
      if (__ballot(top > m[e]) != 0) {  // (seldom after the first blocks)
        const float shrink = factor(m[e], top);
        m[e] = top;
        l[e] *= shrink;
#pragma unroll
        for (int n = 0; n < VW; ++n) acc[e][n] *= shrink;
      }
      const float base = m[e] == -INFINITY ? 0.f : m[e];
#pragma unroll
      for (int r = 0; r < ROWS; ++r) {
        p[e][r] = exp2_fast((s[e][r] - base) * kLog2e);
        l[e] += p[e][r];
      }
    }
#pragma unroll
    for (int r = 0; r < ROWS; ++r)
#pragma unroll
      for (int n = 0; n < VW; ++n) {
        const float x = gone[r] ? 0.f : __uint_as_float(v[r].w[n]);
#pragma unroll
        for (int e = 0; e < HEADS; ++e) acc[e][n] = fmaf(p[e][r], x, acc[e][n]);
      }
    load(s0 + kAttnWaves * BLOCK);
  }

  // Sixteen sums a head (four wavefronts of four rows) on a common maximum: the rows by lanes, the wavefronts in their order.
  if (i16 == 0) {
#pragma unroll
    for (int e = 0; e < HEADS; ++e) {
      stat_m[4 * wave + g][e] = m[e];
      stat_l[4 * wave + g][e] = l[e];
    }
  }
  __syncthreads();
  float share[HEADS];
#pragma unroll
  for (int e = 0; e < HEADS; ++e) {
    float top = -INFINITY, total = 0.f;
    for (int w = 0; w < 4 * kAttnWaves; ++w) top = fmaxf(top, stat_m[w][e]);
    for (int w = 0; w < 4 * kAttnWaves; ++w) total += stat_l[w][e] * factor(stat_m[w][e], top);
    const float mine = factor(m[e], top);
#pragma unroll
    for (int n = 0; n < VW; ++n) {
      float x = acc[e][n] * mine;
      x += __shfl_xor(x, 16, 64);
      x += __shfl_xor(x, 32, 64);
      if (g == 0) joined[wave][e][n][i16] = x;
    }
    share[e] = a.part ? 1.f : total == 0.f ? 0.f : 1.f / total;
    if (tid == 0 && e < a.group) {
      const long long head = ((long long)b * a.kv_heads + h) * a.group + e;
      if (a.stat) a.stat[head * a.chunks + chunk] = make_float2(top, total);
      if (!a.part && a.lse) a.lse[head] = log_sum(top, total);
      all_heads[e] = make_float2(top == -INFINITY ? 0.f : top, share[e]);
    }
  }
  __syncthreads();
  if (logits && !a.stat) {
    const long long slots = ((long long)b * a.kv_heads + h) * a.slot_stride;
    for (int slot = tid; slot < end; slot += kAttnThreads) {
      float sum = 0.f;
      for (int e = 0; e < a.group; ++e) sum = fmaf(exp2_fast((logits[(long long)slot * a.group + e] - all_heads[e].x) * kLog2e), all_heads[e].y, sum);
      a.weights_out[slots + slot] = (a.weights_in ? a.weights_in[slots + slot] : 0.f) + sum;
    }
  }
#pragma unroll
  for (int e = 0; e < HEADS; ++e) {
    if (e >= a.group) continue;
    const long long head = ((long long)b * a.kv_heads + h) * a.group + e;
    for (int c = tid; c < a.d; c += kAttnThreads) {
      const int n = c / 64 * 4 + c % 4, i = c % 64 / 4;
      float x = 0.f;
#pragma unroll
      for (int w = 0; w < kAttnWaves; ++w) x += joined[w][e][n][i];
      x *= share[e];
      if (a.part) a.part[(head * a.chunks + chunk) * a.d + c] = x;
      else *reinterpret_cast<float*>(a.out + b * a.out_stride + (((long long)h * a.group + e) * a.d + c) * 4) = x;
    }
  }
}

// Maximum and sum of one head over its chunks, the same in all lanes of a wavefront.
__device__ inline float2 join_stats(const float2* stat, int chunks, int lane) {
  float top = -INFINITY, total = 0.f;
  for (int c0 = 0; c0 < chunks; c0 += 4 * kWave) {
    float2 x[4];
    float most = top;
#pragma unroll
    for (int k = 0; k < 4; ++k) {
      const int c = c0 + k * kWave + lane;
      x[k] = c < chunks ? stat[c] : make_float2(-INFINITY, 0.f);
    }
#pragma unroll
    for (int k = 0; k < 4; ++k) most = fmaxf(most, x[k].x);
    total *= factor(top, most);
#pragma unroll
    for (int k = 0; k < 4; ++k) total = fmaf(x[k].y, factor(x[k].x, most), total);
    top = most;
  }
  float all = top;
#pragma unroll
  for (int o = 32; o > 0; o >>= 1) all = fmaxf(all, __shfl_xor(all, o, 64));
  return make_float2(all, wave_sum(total * factor(top, all)));
}

constexpr int kFinishThreads = 256;

// The chunks' sums of one head on a common maximum: four channels a thread, the chunks dealt out among as many groups of
// threads as there are, added up in a fixed order.
template <int DT> __device__ inline void join_head(const AttnArgs& a, int b, int h, float4* sums) {
  constexpr int ES = DT == 0 ? 4 : 2;
  const int tid = threadIdx.x;
  const long long head = (long long)b * a.kv_heads * a.group + h;
  const int chunks = (seq_length(a.seqs, b) + a.chunk - 1) / a.chunk;
  const float2* stat = a.stat + head * a.chunks;
  const float2 all = join_stats(stat, chunks, tid & 63);
  if (tid == 0 && a.lse) a.lse[head] = log_sum(all.x, all.y);
  const int units = a.d / 4, slices = kFinishThreads / units, unit = tid % units, slice = tid / units;
  float4 x = make_float4(0.f, 0.f, 0.f, 0.f);
  if (slice < slices) {
    const float* part = a.part + head * a.chunks * a.d + 4 * unit;
#pragma unroll 8
    for (int c = slice; c < chunks; c += slices) {
      const float4 y = *reinterpret_cast<const float4*>(part + (long long)c * a.d);
      const float f = factor(stat[c].x, all.x);
      x.x = fmaf(y.x, f, x.x); x.y = fmaf(y.y, f, x.y); x.z = fmaf(y.z, f, x.z); x.w = fmaf(y.w, f, x.w);
    }
  }
  sums[tid] = x;
  __syncthreads();
  if (slice != 0) return;
  for (int i = 1; i < slices; ++i) {
    const float4 y = sums[i * units + unit];
    x.x += y.x; x.y += y.y; x.z += y.z; x.w += y.w;
  }
  const float inverse = all.y == 0.f ? 0.f : 1.f / all.y;
  const float y[4] = {x.x * inverse, x.y * inverse, x.z * inverse, x.w * inverse};
  store_channels<DT>(a.out + b * a.out_stride + ((long long)h * a.d + 4 * unit) * ES, y);
}

// The weights of some slots of one kv head, summed over the group's heads, from the stored s: one slot a thread. The first
// few s are on their way while the statistics are put together.
__device__ inline void add_weights(const AttnArgs& a, int b, int h, int first, float2* of_head) {
  constexpr int AHEAD = 8;
  const int tid = threadIdx.x, length = seq_length(a.seqs, b);
  if (first >= length) return;
  const long long row = (long long)b * a.kv_heads + h;
  const int chunks = (length + a.chunk - 1) / a.chunk, slot = min(first + tid, length - 1);
  const float* x = a.logits + (row * a.seqs.max_len + slot) * a.group;
  const long long at = row * a.slot_stride + slot;
  float ahead[AHEAD], before = 0.f;
#pragma unroll
  for (int q = 0; q < AHEAD; ++q) ahead[q] = x[min(q, a.group - 1)];
  if (a.weights_in) before = a.weights_in[at];
  for (int q = tid / kWave; q < a.group; q += kFinishThreads / kWave) {
    const float2 r = join_stats(a.stat + (row * a.group + q) * a.chunks, chunks, tid & 63);
    if ((tid & 63) == 0) of_head[q] = make_float2(r.x == -INFINITY ? 0.f : r.x, r.y == 0.f ? 0.f : 1.f / r.y);
  }
  __syncthreads();
  float sum = 0.f;
#pragma unroll
  for (int q = 0; q < AHEAD; ++q)
    if (q < a.group) sum = fmaf(exp2_fast((ahead[q] - of_head[q].x) * kLog2e), of_head[q].y, sum);
  for (int q = AHEAD; q < a.group; ++q) sum = fmaf(exp2_fast((x[q] - of_head[q].x) * kLog2e), of_head[q].y, sum);
  if (first + tid < length) a.weights_out[at] = before + sum;
}

// What is left when every chunk is done (7 us for 170 chunks and 43,328 weights, half of it the launch): blocks 0 .. joins - 1
// of a kv head put its heads' sums together, the others add the weights up.
template <int DT>
__global__ void __launch_bounds__(kFinishThreads) k_attention_finish(AttnArgs a, int joins) {
  __shared__ float4 shared[kFinishThreads];
  const int x = blockIdx.x, h = blockIdx.y, b = blockIdx.z;
  if (x < joins) join_head<DT>(a, b, h * a.group + x, shared);
  else add_weights(a, b, h, (x - joins) * kFinishThreads, reinterpret_cast<float2*>(shared));
}

// ---- launches -----------------------------------------------------------------------------------------------------

struct Plan {
  int tiles, chunk, chunks;
  bool whole;                 // a workgroup sees all of a kv head: nothing is left to do behind it
  size_t part, stat, logits, bytes;  // offsets in the workspace
};

Plan make_plan(const sttm_cache* c, const sttm_sequences* s, int q_heads, bool weights) {
  Plan p;
  const int group = q_heads / c->kv_heads, max_len = make_seqs(c, s).max_len;
  p.tiles = (group + kQTile - 1) / kQTile;
  // One chunk for short sequences: a second launch costs more than the few blocks that follow each other (in a graph, 4 kv heads of
  // 128 bf16 channels: 257 slots 8.6 us, as three chunks 9.6; 64 sequences of 512 slots 17 and 24. One sequence alone would gain
  // from 400 slots on, 512: 12 and 9.7, and with weights from 257 on, 11.7 and 10.2). Else chunks of 256 or 512 slots, the longer ones where there are enough of them for every compute unit to
  // have several of unequal sequences (the batch 142 us, by 256 153, by 1,024 148; one sequence of 43,328 slots by 256 21);
  // of 128 only where 256 would leave compute units without any (that sequence by 128: 24).
  // Whole calls in a graph, bf16 heads of 128 channels, by 128 / 256 / 512 slots, us: 4,096 slots in all rows 10.1 / 12.0 / 15.7;
  // 32,768 12.5 / 14.4 / 17.5; 65,536 16.2 / 15.2 / 18.4; 131,072 24.8 / 21.4 / 20.6; 262,144 41 / 36 / 32; 524,288 69 / 61 / 57;
  // 1,048,576 128 / 111 / 99; 2,097,152 246 / 212 / 192. fp32 rows of 72, 398,320 slots: 49.6 / 49.8 / 52.3; 2,097,152: 217 / 213 / 209.
  // (So between the two bounds 512 is up to a tenth faster for 16-bit rows, and 256 for short fp32 ones.)
  const long long rows = (long long)std::max(s->batch, 1) * c->kv_heads * p.tiles, len = std::max(max_len, 1);
  p.chunk = len <= kChunkMax || rows * len >= kChunkMax * 4096ll ? kChunkMax : rows * len >= kChunkMid * 256ll ? kChunkMid : kChunkLeast;
  p.chunks = (int)((len + p.chunk - 1) / p.chunk);
  size_t off = 0;
  auto take = [&](size_t bytes) { size_t o = off; off = (off + bytes + 255) / 256 * 256; return o; };
  const size_t heads = (size_t)s->batch * q_heads;
  p.part = take(p.chunks > 1 ? heads * p.chunks * c->head_dim * sizeof(float) : 0);
  p.whole = p.chunks == 1 && p.tiles == 1;
  p.stat = take(p.chunks > 1 || (weights && !p.whole) ? heads * p.chunks * sizeof(float2) : 0);
  p.logits = take(weights ? heads * (size_t)max_len * sizeof(float) : 0);
  p.bytes = std::max(off, (size_t)256);
  return p;
}

int check_attention(sttm_ctx* ctx, const sttm_cache* cache, const sttm_sequences* seqs, int q_heads) {
  int rc = check_cache(ctx, cache);
  if (rc == STTM_OK) rc = check_sequences(ctx, cache, seqs);
  if (rc != STTM_OK) return rc;
  if (q_heads < 1 || q_heads % cache->kv_heads || q_heads / cache->kv_heads > 256 || q_heads > 65535)
    return ctx_fail(ctx, STTM_ERR_SHAPE, "need q_heads a multiple of kv_heads, at most 256 a kv head, q_heads <= 65535");
  if ((double)seqs->batch * q_heads * make_seqs(cache, seqs).max_len > 1e14) return ctx_fail(ctx, STTM_ERR_SHAPE, "batch * q_heads * max_len too large");
  return STTM_OK;
}

template <int HEADS, int VW>
void launch_rows(const AttnArgs& a, dim3 grid, hipStream_t s) {
  if (a.bias) hipLaunchKernelGGL((k_paged_attention_rows<HEADS, VW, true>), grid, dim3(kAttnThreads), 0, s, a);
  else hipLaunchKernelGGL((k_paged_attention_rows<HEADS, VW, false>), grid, dim3(kAttnThreads), 0, s, a);
}

template <int DT, int NQ, int VW>
void launch_blocks(const AttnArgs& a, dim3 grid, hipStream_t s) {
  if constexpr (DT == 0) {
    if (a.group == 1) return launch_rows<1, VW>(a, grid, s);
    if (a.group == 2) return launch_rows<2, VW>(a, grid, s);
  }
  if (a.bias) hipLaunchKernelGGL((k_paged_attention<DT, NQ, VW, true>), grid, dim3(kAttnThreads), 0, s, a);
  else hipLaunchKernelGGL((k_paged_attention<DT, NQ, VW, false>), grid, dim3(kAttnThreads), 0, s, a);
}

// One instance for each way a head's channels fill the products: 64 bytes of a key and 16 lanes' shares of a value.
template <int DT>
void launch_attention(const AttnArgs& a, int batch, hipStream_t s) {
  const dim3 grid(a.chunks, a.kv_heads * a.tiles, batch);
  constexpr int W = DT == 0 ? 2 : 1;  // fp32 rows have twice the bytes
  if (a.d <= 32) launch_blocks<DT, W, 4>(a, grid, s);
  else if (a.d <= 64) launch_blocks<DT, 2 * W, 4>(a, grid, s);
  else if (a.d <= 96) launch_blocks<DT, 3 * W, 8>(a, grid, s);
  else if (a.d <= 128) launch_blocks<DT, 4 * W, 8>(a, grid, s);
  else if (a.d <= 192) launch_blocks<DT, 6 * W, 16>(a, grid, s);
  else launch_blocks<DT, 8 * W, 16>(a, grid, s);
  const int joins = a.part ? a.group : 0, weights = a.weights_out && a.stat ? (a.seqs.max_len + kFinishThreads - 1) / kFinishThreads : 0;
  if (joins + weights)
    hipLaunchKernelGGL((k_attention_finish<DT>), dim3(joins + weights, a.kv_heads, batch), dim3(kFinishThreads), 0, s, a, joins);
}

}  // namespace
}  // namespace sttm

using namespace sttm;

extern "C" size_t sttm_paged_attention_workspace_bytes(const sttm_cache* cache, const sttm_sequences* seqs, int q_heads, int weights) {
  if (check_attention(nullptr, cache, seqs, q_heads) != STTM_OK) return 0;
  return make_plan(cache, seqs, q_heads, weights != 0).bytes;
}

extern "C" int sttm_paged_attention(sttm_ctx* ctx, const sttm_cache* cache, const sttm_sequences* seqs, int q_heads, float scale,
                                    const void* q, int64_t q_stride, const float* key_bias, const float* weights_in,
                                    float* weights_out, int64_t slot_stride, void* out, int64_t out_stride, float* lse,
                                    void* workspace, size_t workspace_bytes) {
  if (!ctx) return STTM_ERR_NULL;
  int rc = check_attention(ctx, cache, seqs, q_heads);
  if (rc != STTM_OK) return rc;
  const int es = elem_bytes(cache->dtype), align = 16 / es;
  const int64_t row = (int64_t)q_heads * cache->head_dim, most = (int64_t)1 << 40;
  if (q_stride < row || out_stride < row || q_stride > most || out_stride > most || q_stride % align || out_stride % align)
    return ctx_fail(ctx, STTM_ERR_SHAPE, "q_stride, out_stride: multiples of 16 bytes, no less than a row");
  AttnArgs a{};
  a.seqs = make_seqs(cache, seqs);
  if ((key_bias || weights_out) && (slot_stride < a.seqs.max_len || slot_stride > most))
    return ctx_fail(ctx, STTM_ERR_SHAPE, "slot_stride must be no less than max_len");
  if (!(std::fabs(scale) <= 3e38f)) return ctx_fail(ctx, STTM_ERR_ARG, "scale must be a finite number");
  if (weights_in && !weights_out) return ctx_fail(ctx, STTM_ERR_ARG, "weights_in without weights_out");
  if (seqs->batch == 0) return STTM_OK;
  if (!q || !out) return ctx_fail(ctx, STTM_ERR_NULL, "q or out is NULL");
  if (!aligned16(q) || !aligned16(out)) return ctx_fail(ctx, STTM_ERR_ARG, "q and out must be 16-byte aligned");
  const Plan p = make_plan(cache, seqs, q_heads, weights_out != nullptr);
  rc = check_workspace(ctx, workspace, workspace_bytes, p.bytes);
  if (rc != STTM_OK) return rc;
  char* ws = static_cast<char*>(workspace);
  a.pool = make_pool(cache);
  a.q = static_cast<const char*>(q);
  a.out = static_cast<char*>(out);
  a.q_stride = q_stride * es;
  a.out_stride = out_stride * es;
  a.bias = key_bias;
  a.weights_in = weights_in;
  a.weights_out = weights_out;
  a.lse = lse;
  a.slot_stride = slot_stride;
  if (weights_out) a.logits = reinterpret_cast<float*>(ws + p.logits);
  if (p.chunks > 1) a.part = reinterpret_cast<float*>(ws + p.part);
  if (p.chunks > 1 || (weights_out && !p.whole)) a.stat = reinterpret_cast<float2*>(ws + p.stat);
  a.scale = scale;
  a.kv_heads = cache->kv_heads;
  a.group = q_heads / cache->kv_heads;
  a.d = cache->head_dim;
  a.chunk = p.chunk;
  a.chunks = p.chunks;
  a.tiles = p.tiles;
  rc = ctx_device(ctx);
  if (rc != STTM_OK) return rc;
  const hipStream_t s = ctx_stream(ctx);
  if (cache->dtype == STTM_F32) launch_attention<0>(a, seqs->batch, s);
  else if (cache->dtype == STTM_BF16) launch_attention<1>(a, seqs->batch, s);
  else launch_attention<2>(a, seqs->batch, s);
  return ctx_after_launch(ctx);
}
