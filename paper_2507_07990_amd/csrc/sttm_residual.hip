// What follows a block of a layer: norm of its result, gate, residual sum, and the norm before the next block, one pass over the rows.
#include "sttm_cache.h"

#include <algorithm>
#include <cmath>

namespace sttm {
namespace {

constexpr int kResidualThreads = 256;

struct NormArgs {
  const char *weight, *bias;     // NULL: none
  float eps;
  int kind;                      // -1: no norm, 0: root of the mean square, 1: mean and variance
};

struct ResidualArgs {
  const char *x, *y, *gate;
  char *r, *h;
  long long x_stride, y_stride, gate_stride, r_stride, h_stride;  // bytes
  long long n;
  NormArgs post, pre;
  float scale, mean;             // mean = 1 / width
  int units;                     // of 16 bytes in a row
  int gate_wide, gate_tanh;
};

// Sixteen bytes of a row as numbers.
template <int DT> struct Unit {
  static constexpr int N = DT == 0 ? 4 : 8;
  __device__ static inline void get(const uint4& w, float (&x)[N]) {
    if constexpr (DT == 0) {
      x[0] = __uint_as_float(w.x); x[1] = __uint_as_float(w.y); x[2] = __uint_as_float(w.z); x[3] = __uint_as_float(w.w);
    } else {
      x[0] = low_half<DT>(w.x); x[1] = high_half<DT>(w.x); x[2] = low_half<DT>(w.y); x[3] = high_half<DT>(w.y);
      x[4] = low_half<DT>(w.z); x[5] = high_half<DT>(w.z); x[6] = low_half<DT>(w.w); x[7] = high_half<DT>(w.w);
    }
  }
  __device__ static inline uint4 of(const float (&x)[N]) {
    if constexpr (DT == 0) return make_uint4(__float_as_uint(x[0]), __float_as_uint(x[1]), __float_as_uint(x[2]), __float_as_uint(x[3]));
    else return make_uint4(pack2<DT>(x[0], x[1]), pack2<DT>(x[2], x[3]), pack2<DT>(x[4], x[5]), pack2<DT>(x[6], x[7]));
  }
};

// The hyperbolic tangent, within three steps of fp32: its Taylor series up to a half, where the other form would lose digits, and 1 - 2 / (e^2x + 1).
__device__ inline float tanh_of(float x) {
  const float s = x * x, y = fabsf(x);
  float p = -929569.f / 638512875.f;
  p = fmaf(p, s, 21844.f / 6081075.f);
  p = fmaf(p, s, -1382.f / 155925.f);
  p = fmaf(p, s, 62.f / 2835.f);
  p = fmaf(p, s, -17.f / 315.f);
  p = fmaf(p, s, 2.f / 15.f);
  p = fmaf(p, s, -1.f / 3.f);
  const float far = copysignf(1.f - 2.f / (exp2_fast(y * 2.8853900817779268f) + 1.f), x);
  return y < 0.5f ? fmaf(x * s, p, x) : far;
}

// The sum over the lanes that have a row, the same bits in each of them. of_wave: a place that no other sum of this row uses, nor the same one
// of the next row.
template <int LANES> __device__ inline float row_sum(float v, float* of_wave) {
#pragma unroll
  for (int o = 32; o > 0; o >>= 1) v += __shfl_xor(v, o, 64);
  if constexpr (LANES > kWave) {
    if ((threadIdx.x & 63) == 0) of_wave[threadIdx.x >> 6] = v;
    __syncthreads();
    v = of_wave[0];
#pragma unroll
    for (int w = 1; w < LANES / kWave; ++w) v += of_wave[w];
  }
  return v;
}

// LANES lanes (a wavefront where rows are short, all four of a workgroup else) have a row, U units of 16 bytes a lane at most, kept in registers
// from the one read to the two writes; so are the weights, for all the rows that the lanes come by. The next row is on its way while this one is
// worked on. Sums of squares are those of differences from the mean, which is known by then.
// Bound by memory: 43,264 rows of 3,584 bf16 channels with two norms and a gate are 1.24 GB in 237 us, 5.2 TB/s (a wavefront a row, its weights from the
// caches with every row: 362). ONCE: what is written is more than the caches are good for and goes past them.
template <int DT, int LANES, int U, bool ONCE>
__global__ void __launch_bounds__(kResidualThreads) k_residual_norm(ResidualArgs a) {
  constexpr int N = Unit<DT>::N, ROWS = kResidualThreads / LANES;
  constexpr bool KEEP = U <= 2;                           // weights in registers, the next row ahead (where there are registers for that)
  __shared__ float of_wave[2][4][kResidualThreads / kWave];
  const int lane = threadIdx.x & (LANES - 1);
  auto read = [&](const char* from, int i) __attribute__((always_inline)) {
    const int at = lane + i * LANES;
    uint4 w = make_uint4(0u, 0u, 0u, 0u);
    if (at < a.units) w = *reinterpret_cast<const uint4*>(from + 16 * at);
    return w;
  };
  uint4 kept[5][KEEP ? U : 1];
  if constexpr (KEEP) {
#pragma unroll
    for (int k = 0; k < 5; ++k)
#pragma unroll
      for (int i = 0; i < U; ++i) kept[k][i] = make_uint4(0u, 0u, 0u, 0u);
#pragma unroll
    for (int i = 0; i < U; ++i) {
      if (a.post.weight) kept[0][i] = read(a.post.weight, i);
      if (a.post.bias) kept[1][i] = read(a.post.bias, i);
      if (a.pre.weight) kept[2][i] = read(a.pre.weight, i);
      if (a.pre.bias) kept[3][i] = read(a.pre.bias, i);
      if (a.gate_wide && !a.gate_stride) kept[4][i] = read(a.gate, i);
    }
  }
  auto weight = [&](int k, int i, float (&f)[N]) __attribute__((always_inline)) {
    if constexpr (KEEP) Unit<DT>::get(kept[k][i], f);
    else Unit<DT>::get(read(k == 0 ? a.post.weight : k == 1 ? a.post.bias : k == 2 ? a.pre.weight : k == 3 ? a.pre.bias : a.gate, i), f);
  };
  const long long step = (long long)gridDim.x * ROWS;
  long long row = blockIdx.x * (long long)ROWS + threadIdx.x / LANES;
  uint4 x_next[U], y_next[U];
  auto fetch = [&](long long r) __attribute__((always_inline)) {
#pragma unroll
    for (int i = 0; i < U; ++i) {
      x_next[i] = read(a.x + r * a.x_stride, i);
      y_next[i] = make_uint4(0u, 0u, 0u, 0u);
      if (a.y) y_next[i] = read(a.y + r * a.y_stride, i);
    }
  };
  if (KEEP && row < a.n) fetch(row);
  for (int parity = 0; row < a.n; row += step, parity ^= 1) {  // (all lanes of a row)
    float v[U][N], f[N];
    uint4 x[U];
    if (!KEEP) fetch(row);
#pragma unroll
    for (int i = 0; i < U; ++i) {
      x[i] = x_next[i];
      Unit<DT>::get(y_next[i], v[i]);
    }
    if (KEEP && row + step < a.n) fetch(row + step);
    // (x - mean) / root of (variance + eps), or without a mean; weight and bias.
    auto norm = [&](const NormArgs& by, int which) __attribute__((always_inline)) {
      float mean = 0.f, sum = 0.f;
      if (by.kind == 1) {
#pragma unroll
        for (int i = 0; i < U; ++i)
#pragma unroll
          for (int e = 0; e < N; ++e) sum += v[i][e];
        mean = row_sum<LANES>(sum, of_wave[parity][2 * which]) * a.mean;
        sum = 0.f;
      }
#pragma unroll
      for (int i = 0; i < U; ++i)
#pragma unroll
        for (int e = 0; e < N; ++e) {
          const float d = v[i][e] - mean;
          if (lane + i * LANES < a.units) sum = fmaf(d, d, sum);
        }
      const float by_root = 1.f / sqrtf(fmaf(row_sum<LANES>(sum, of_wave[parity][2 * which + 1]), a.mean, by.eps));
#pragma unroll
      for (int i = 0; i < U; ++i) {
#pragma unroll
        for (int e = 0; e < N; ++e) v[i][e] = lane + i * LANES < a.units ? (v[i][e] - mean) * by_root : 0.f;
        if (by.weight) {
          weight(2 * which, i, f);
#pragma unroll
          for (int e = 0; e < N; ++e) v[i][e] *= f[e];
        }
        if (by.bias) {
          weight(2 * which + 1, i, f);
#pragma unroll
          for (int e = 0; e < N; ++e) v[i][e] += f[e];
        }
      }
    };
    auto put = [&](char* to, int i) __attribute__((always_inline)) {
      const int at = lane + i * LANES;
      if (at >= a.units) return;
      const uint4 w = Unit<DT>::of(v[i]);
      if constexpr (ONCE) store_once(reinterpret_cast<uint4*>(to + 16 * at), w);
      else *reinterpret_cast<uint4*>(to + 16 * at) = w;
    };
    if (a.post.kind >= 0) norm(a.post, 0);
    float one = 1.f;
    if (a.gate && !a.gate_wide) {
      const char* gate = a.gate + row * a.gate_stride;
      if constexpr (DT == 0) one = *reinterpret_cast<const float*>(gate);
      else one = low_half<DT>(*reinterpret_cast<const uint16_t*>(gate));
      if (a.gate_tanh) one = tanh_of(one);
    }
#pragma unroll
    for (int i = 0; i < U; ++i) {
      if (a.gate && a.gate_wide) {
        if (a.gate_stride) Unit<DT>::get(read(a.gate + row * a.gate_stride, i), f);
        else weight(4, i, f);
#pragma unroll
        for (int e = 0; e < N; ++e) v[i][e] *= a.gate_tanh ? tanh_of(f[e]) : f[e];
      } else if (a.gate) {
#pragma unroll
        for (int e = 0; e < N; ++e) v[i][e] *= one;
      }
      Unit<DT>::get(x[i], f);
#pragma unroll
      for (int e = 0; e < N; ++e) v[i][e] = a.y ? fmaf(f[e], a.scale, v[i][e]) : f[e] * a.scale;
      if (a.r) put(a.r + row * a.r_stride, i);
    }
    if (!a.h) continue;
    if (a.pre.kind >= 0) norm(a.pre, 1);
#pragma unroll
    for (int i = 0; i < U; ++i) put(a.h + row * a.h_stride, i);
  }
}

// Rows follow one another in as many workgroups: twelve a compute unit, which holds three or four at once, so that they come out even (43,264
// rows of 3,584 bf16 channels by 3 / 4 / 8 / 10 / 11 / 12 / 14 a compute unit and one a row: 235 / 292 / 246 / 254 / 243 / 237 / 240 / 280 us; 16,384 of
// 1,152 in fp32 75 / 67 / 68 / 71 / 68 / 69 / 69 / 78).
constexpr int64_t kResidualBlocks = 12 * 256;

template <int DT, int LANES, int U> void launch_rows(const ResidualArgs& a, bool once, hipStream_t s) {
  const int64_t blocks = (a.n + kResidualThreads / LANES - 1) / (kResidualThreads / LANES);
  const dim3 grid((unsigned)std::min(blocks, kResidualBlocks)), block(kResidualThreads);
  if (once) hipLaunchKernelGGL((k_residual_norm<DT, LANES, U, true>), grid, block, 0, s, a);
  else hipLaunchKernelGGL((k_residual_norm<DT, LANES, U, false>), grid, block, 0, s, a);
}

template <int DT> void launch_residual(const ResidualArgs& a, bool once, hipStream_t s) {
  if (a.units <= kWave) launch_rows<DT, 64, 1>(a, once, s);
  else if (a.units <= 2 * kWave) launch_rows<DT, 64, 2>(a, once, s);
  else if (a.units <= kResidualThreads) launch_rows<DT, 256, 1>(a, once, s);
  else if (a.units <= 2 * kResidualThreads) launch_rows<DT, 256, 2>(a, once, s);
  else if (a.units <= 4 * kResidualThreads) launch_rows<DT, 256, 4>(a, once, s);
  else if (a.units <= 8 * kResidualThreads) launch_rows<DT, 256, 8>(a, once, s);
  else if constexpr (DT == 0) launch_rows<DT, 256, 16>(a, once, s);
}

int check_norm(sttm_ctx* ctx, const sttm_norm* n, NormArgs* out) {
  out->kind = -1;
  if (!n) return STTM_OK;
  if (n->kind != STTM_NORM_RMS && n->kind != STTM_NORM_LAYER) return ctx_fail(ctx, STTM_ERR_ARG, "kind of a norm must be STTM_NORM_RMS or STTM_NORM_LAYER");
  if (!(n->eps >= 0.f)) return ctx_fail(ctx, STTM_ERR_ARG, "eps must be a number >= 0");
  if (!aligned16(n->weight) || !aligned16(n->bias)) return ctx_fail(ctx, STTM_ERR_ARG, "weights of norms must be 16-byte aligned");
  *out = {static_cast<const char*>(n->weight), static_cast<const char*>(n->bias), n->eps, n->kind == STTM_NORM_LAYER};
  return STTM_OK;
}

constexpr int64_t kOnceBytes = 32 << 20;  // what the eight L2 of the card hold together

}  // namespace
}  // namespace sttm

using namespace sttm;

extern "C" int sttm_residual_norm(sttm_ctx* ctx, int dtype, int64_t n, int width, const void* x, int64_t x_stride, const void* y, int64_t y_stride,
                                  const sttm_norm* post, const void* gate, int64_t gate_stride, int gate_width, int gate_tanh, float scale, void* r,
                                  int64_t r_stride, const sttm_norm* pre, void* h, int64_t h_stride) {
  if (!ctx) return STTM_ERR_NULL;
  if (dtype != STTM_F32 && dtype != STTM_BF16 && dtype != STTM_F16)
    return ctx_fail(ctx, STTM_ERR_DTYPE, "dtype must be STTM_F32, STTM_BF16 or STTM_F16");
  if (n < 0 || n > (1ll << 25) || width < 8 || width > 16384 || width % 8)
    return ctx_fail(ctx, STTM_ERR_SHAPE, "need 0 <= n <= 2^25, width % 8 == 0, 8 <= width <= 16384");
  const int64_t es = elem_bytes(dtype), align = 16 / es, most = (int64_t)1 << 36;
  auto bad = [&](const void* p, int64_t stride) { return p && (stride < width || stride > most || stride % align); };
  if (bad(x, x_stride) || bad(y, y_stride) || bad(r, r_stride) || bad(h, h_stride))
    return ctx_fail(ctx, STTM_ERR_SHAPE, "row strides: multiples of 16 bytes, no less than a row");
  if (gate && (gate_width != 1 && gate_width != width)) return ctx_fail(ctx, STTM_ERR_SHAPE, "gate_width must be 1 or width");
  if (gate && (gate_stride < 0 || gate_stride > most || (gate_stride && gate_stride < gate_width) || (gate_width > 1 && gate_stride % align)))
    return ctx_fail(ctx, STTM_ERR_SHAPE, "gate_stride: zero, or no less than gate_width (and a multiple of 16 bytes where that is width)");
  if (!(std::fabs(scale) <= 3e38f)) return ctx_fail(ctx, STTM_ERR_ARG, "scale must be a finite number");
  ResidualArgs a{};
  int rc = check_norm(ctx, post, &a.post);
  if (rc == STTM_OK) rc = check_norm(ctx, pre, &a.pre);
  if (rc != STTM_OK) return rc;
  if (!y && (post || gate)) return ctx_fail(ctx, STTM_ERR_ARG, "a norm or a gate for y without y");
  if (!h && pre) return ctx_fail(ctx, STTM_ERR_ARG, "a norm for h without h");
  if (r && r == h) return ctx_fail(ctx, STTM_ERR_ARG, "r and h must not be the same rows");
  if (n == 0) return STTM_OK;
  if (!x || (!r && !h)) return ctx_fail(ctx, STTM_ERR_NULL, "x, or both r and h, are NULL");
  if (!aligned16(x) || !aligned16(y) || !aligned16(r) || !aligned16(h) || (gate_width > 1 && !aligned16(gate)))
    return ctx_fail(ctx, STTM_ERR_ARG, "rows must be 16-byte aligned");
  a.x = static_cast<const char*>(x); a.y = static_cast<const char*>(y); a.gate = static_cast<const char*>(gate);
  a.r = static_cast<char*>(r); a.h = static_cast<char*>(h);
  a.x_stride = x_stride * es; a.y_stride = y_stride * es; a.gate_stride = gate_stride * es;
  a.r_stride = r_stride * es; a.h_stride = h_stride * es;
  a.n = n;
  a.scale = scale; a.mean = 1.f / (float)width;
  a.units = (int)(width * es / 16);
  a.gate_wide = gate_width > 1; a.gate_tanh = gate_tanh != 0;
  rc = ctx_device(ctx);
  if (rc != STTM_OK) return rc;
  const hipStream_t s = ctx_stream(ctx);
  const bool once = n * width * es * ((r != nullptr) + (h != nullptr)) > kOnceBytes;
  if (dtype == STTM_F32) launch_residual<0>(a, once, s);
  else if (dtype == STTM_BF16) launch_residual<1>(a, once, s);
  else launch_residual<2>(a, once, s);
  return ctx_after_launch(ctx);
}
