// Norm of queries and keys per head, rotation by position and the write into the paged cache, one pass over the rows; the
// argument checks the cache's operators share.
#include "sttm_cache.h"

#include <cstdio>

namespace sttm {

int check_cache(sttm_ctx* c, const sttm_cache* p) {
  if (!p || !p->k || !p->v) return ctx_fail(c, STTM_ERR_NULL, "the cache, or its k or v, is NULL");
  if (p->dtype != STTM_F32 && p->dtype != STTM_BF16 && p->dtype != STTM_F16)
    return ctx_fail(c, STTM_ERR_DTYPE, "dtype must be STTM_F32, STTM_BF16 or STTM_F16");
  if (p->head_dim < 8 || p->head_dim > 256 || p->head_dim % 8 || p->kv_heads < 1 || p->kv_heads > 1024 || p->pages < 1 ||
      p->pages >= (1ll << 31) || p->page_size < 8 || p->page_size > 1024 || (p->page_size & (p->page_size - 1)))
    return ctx_fail(c, STTM_ERR_SHAPE, "need head_dim % 8 == 0, 8 <= head_dim <= 256, 1 <= kv_heads <= 1024, page_size a power of two in 8 .. 1024, 1 <= pages < 2^31");
  const int64_t align = 16 / elem_bytes(p->dtype), most = (int64_t)1 << 40;
  if (p->page_stride < 0 || p->head_stride < 0 || p->token_stride < p->head_dim || p->page_stride > most || p->head_stride > most ||
      p->token_stride > (1 << 20) || p->page_stride % align || p->head_stride % align || p->token_stride % align)
    return ctx_fail(c, STTM_ERR_SHAPE, "cache strides: multiples of 16 bytes, not negative, token_stride from head_dim to 2^20");
  if (p->page_size * p->token_stride * elem_bytes(p->dtype) >= (1ll << 31))
    return ctx_fail(c, STTM_ERR_SHAPE, "the slots of a page must lie within 2 GiB of each other");
  if (!aligned16(p->k) || !aligned16(p->v)) return ctx_fail(c, STTM_ERR_ARG, "k and v must be 16-byte aligned");
  return STTM_OK;
}

int check_sequences(sttm_ctx* c, const sttm_cache* p, const sttm_sequences* s) {
  if (!s) return ctx_fail(c, STTM_ERR_NULL, "seqs is NULL");
  if (s->batch < 0 || s->batch > 65535 || s->max_pages < 0 || s->max_len < 0 || s->table_stride < s->max_pages)
    return ctx_fail(c, STTM_ERR_SHAPE, "need 0 <= batch <= 65535, max_pages >= 0, max_len >= 0, table_stride >= max_pages");
  if ((int64_t)s->max_pages * p->page_size >= (1ll << 31)) return ctx_fail(c, STTM_ERR_SHAPE, "need max_pages * page_size < 2^31");
  // (slots are numbered in 32 bits, and the numbers run on by up to as many: behind the new length, past the end in whole blocks)
  if (make_seqs(p, s).max_len > 1 << 30) return ctx_fail(c, STTM_ERR_SHAPE, "need no more than 2^30 slots a sequence (max_len, or max_pages * page_size)");
  if (s->batch && (!s->lengths || (!s->block_table && s->max_pages && s->max_len)))
    return ctx_fail(c, STTM_ERR_NULL, "block_table or lengths is NULL");
  return STTM_OK;
}

int check_workspace(sttm_ctx* c, const void* ws, size_t have, size_t need) {
  if (ws && have >= need && (reinterpret_cast<uintptr_t>(ws) & 255) == 0) return STTM_OK;
  char buf[160];
  snprintf(buf, sizeof buf, "workspace: need %zu bytes, 256-byte aligned; have %zu at %p", need, have, ws);
  return ctx_fail(c, STTM_ERR_WORKSPACE, buf);
}

Pool make_pool(const sttm_cache* c) {
  const long long es = elem_bytes(c->dtype);
  Pool p;
  p.k = static_cast<char*>(c->k);
  p.v = static_cast<char*>(c->v);
  p.page_stride = c->page_stride * es;
  p.head_stride = c->head_stride * es;
  p.token_stride = (int)(c->token_stride * es);
  p.pages = (int)c->pages;
  p.shift = __builtin_ctz((unsigned)c->page_size);
  p.row = (int)(c->head_dim * es);
  return p;
}

Seqs make_seqs(const sttm_cache* c, const sttm_sequences* s) {
  const int64_t slots = (int64_t)s->max_pages * c->page_size;
  return {s->block_table, s->lengths, s->table_stride, (int)(s->max_len < slots ? s->max_len : slots)};
}

namespace {

struct RopeArgs {
  const char *q, *k, *v;
  char *q_out, *k_out;
  long long q_stride, k_stride, v_stride, q_out_stride, k_out_stride;  // bytes
  const void *q_weight, *k_weight;
  const long long* slots;
  const void* positions;
  const float* inv_freq;
  long long pos_stride;
  long long n;
  long long total_slots;     // of the pool
  Pool pool;
  float eps, mean;           // mean = 1 / d
  int q_heads, kv_heads, d;
  int pairs, cut1, cut2;     // pair i belongs to axis (i >= cut1) + (i >= cut2)
  int pos_float, interleaved, cached;
  int parts;                 // wavefronts that share a row of q, k and v
};

// Eight elements of a row: two runs of four.
template <int DT> struct Run;
template <> struct Run<0> {
  float4 a, b;
  __device__ inline void load(const char* p, int o0, int o1) {
    a = *reinterpret_cast<const float4*>(p + o0);
    b = *reinterpret_cast<const float4*>(p + o1);
  }
  __device__ inline void get(float (&x)[8]) const {
    x[0] = a.x; x[1] = a.y; x[2] = a.z; x[3] = a.w;
    x[4] = b.x; x[5] = b.y; x[6] = b.z; x[7] = b.w;
  }
  __device__ static inline Run of(const float (&x)[8]) {
    return {make_float4(x[0], x[1], x[2], x[3]), make_float4(x[4], x[5], x[6], x[7])};
  }
  template <bool ONCE> __device__ inline void store(char* p, int o0, int o1) const {
    if constexpr (ONCE) {
      store_once(reinterpret_cast<float4*>(p + o0), a);
      store_once(reinterpret_cast<float4*>(p + o1), b);
    } else {
      *reinterpret_cast<float4*>(p + o0) = a;
      *reinterpret_cast<float4*>(p + o1) = b;
    }
  }
};
template <int DT> struct Run {
  uint2 a, b;
  __device__ inline void load(const char* p, int o0, int o1) {
    a = *reinterpret_cast<const uint2*>(p + o0);
    b = *reinterpret_cast<const uint2*>(p + o1);
  }
  __device__ inline void get(float (&x)[8]) const {
    x[0] = low_half<DT>(a.x); x[1] = high_half<DT>(a.x); x[2] = low_half<DT>(a.y); x[3] = high_half<DT>(a.y);
    x[4] = low_half<DT>(b.x); x[5] = high_half<DT>(b.x); x[6] = low_half<DT>(b.y); x[7] = high_half<DT>(b.y);
  }
  __device__ static inline Run of(const float (&x)[8]) {
    return {make_uint2(pack2<DT>(x[0], x[1]), pack2<DT>(x[2], x[3])), make_uint2(pack2<DT>(x[4], x[5]), pack2<DT>(x[6], x[7]))};
  }
  template <bool ONCE> __device__ inline void store(char* p, int o0, int o1) const {
    if constexpr (ONCE) {
      store_once8(p + o0, a);
      store_once8(p + o1, b);
    } else {
      *reinterpret_cast<uint2*>(p + o0) = a;
      *reinterpret_cast<uint2*>(p + o1) = b;
    }
  }
};

constexpr int kRopeThreads = 256;
// Wavefronts: two a SIMD; more of them work the angles out more often (4,915 tokens by 4,915 wavefronts 35 us, by 9,830 40). Bytes
// that the eight L2 of the card hold together. (A host-thread build of the tests sets 1 and 0: a wavefront has many rows of heads,
// which go past the caches.)
#ifndef STTM_ROPE_WAVES
#define STTM_ROPE_WAVES 2048
#define STTM_ROPE_ONCE_BYTES (32 << 20)
#endif
constexpr int kRopeWaves = STTM_ROPE_WAVES;
constexpr int64_t kOnceBytes = STTM_ROPE_ONCE_BYTES;

// LANES lanes share a head's row, eight channels a lane: the two runs of four that its four pairs consist of (or eight
// channels in a row where pairs are neighbours, and behind the rotated part). A wavefront has 64 / LANES rows of the same
// token side by side, so that cos and sin of a lane's pairs serve all heads it comes by.
// The angle is position * frequency in turns, in 64 bits, where whole turns are taken off exactly: in 32 bits position 43,264
// would leave an angle 2^-9 off.
// Bound by memory: 43,264 tokens of 28 + 4 heads of 128 bf16 channels are 798 MB in 155 us where launches follow each other,
// 5.1 TB/s, the rate of a copy (in the first ones after idle up to 169). ONCE:
// what is written is more than the caches are good for and goes past them (4,915 fp32 tokens 28 us against 36).
template <int DT, int LANES, bool ONCE>
__global__ void __launch_bounds__(kRopeThreads) k_qk_norm_rope(RopeArgs a) {
  constexpr int ES = DT == 0 ? 4 : 2, ROWS = kWave / LANES;
  const unsigned wave = blockIdx.x * (kRopeThreads / kWave) + __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
  const unsigned in_n = wave / (unsigned)a.parts;
  const long long row = in_n;
  if (row >= a.n) return;  // (the same in all lanes)
  const int part = (int)(wave - in_n * (unsigned)a.parts), lane = threadIdx.x & 63, unit = lane & (LANES - 1), sub = lane / LANES;
  const bool there = unit < a.d / 8, turns = unit < a.pairs / 4;
  const int o0 = ES * (turns && !a.interleaved ? 4 * unit : 8 * unit);
  const int o1 = ES * (turns && !a.interleaved ? a.pairs + 4 * unit : 8 * unit + 4);
  float cs[4] = {1.f, 1.f, 1.f, 1.f}, sn[4] = {0.f, 0.f, 0.f, 0.f};
  if (there && turns) {
#pragma unroll
    for (int i = 0; i < 4; ++i) {
      const int pair = 4 * unit + i;
      const long long at = row * a.pos_stride + (pair >= a.cut1) + (pair >= a.cut2);
      const double pos = a.pos_float ? (double)static_cast<const float*>(a.positions)[at] : (double)static_cast<const int*>(a.positions)[at];
      const double t = pos * ((double)a.inv_freq[pair] * 0.15915494309189533577);  // in turns
      const float r = 2.f * (float)(t - rint(t));                                   // in half turns, -1 .. 1
      sincos_half_turns(r, &sn[i], &cs[i]);
    }
  }
  float wq[8], wk[8];
#pragma unroll
  for (int i = 0; i < 8; ++i) wq[i] = wk[i] = 1.f;
  Run<DT> w;
  if (there && a.q_weight) { w.load(static_cast<const char*>(a.q_weight), o0, o1); w.get(wq); }
  if (there && a.k_weight) { w.load(static_cast<const char*>(a.k_weight), o0, o1); w.get(wk); }
  long long at = -1;  // of the row's slot in the pool
  if (a.cached) {
    const long long slot = a.slots[row];
    if (slot >= 0 && slot < a.total_slots)
      at = (slot >> a.pool.shift) * a.pool.page_stride + (slot & ((1 << a.pool.shift) - 1)) * a.pool.token_stride;
  }
  const int heads = a.q_heads + (a.cached ? 2 : 1) * a.kv_heads;
  const int bytes = a.d * ES;
  for (int h0 = part * ROWS; h0 < heads; h0 += a.parts * ROWS) {
    const int h = h0 + sub;
    const bool mine = there && h < heads;
    const int kind = h < a.q_heads ? 0 : h < a.q_heads + a.kv_heads ? 1 : 2;
    const int hh = kind == 0 ? h : kind == 1 ? h - a.q_heads : h - a.q_heads - a.kv_heads;
    Run<DT> x;
    float f[8];
#pragma unroll
    for (int i = 0; i < 8; ++i) f[i] = 0.f;
    if (mine) {
      const char* from = kind == 0 ? a.q + row * a.q_stride : kind == 1 ? a.k + row * a.k_stride : a.v + row * a.v_stride;
      x.load(from + (long long)hh * bytes, o0, o1);
      x.get(f);
    }
    float sum = 0.f;
#pragma unroll
    for (int i = 0; i < 8; ++i) sum = fmaf(f[i], f[i], sum);
#pragma unroll
    for (int o = LANES / 2; o > 0; o >>= 1) sum += __shfl_xor(sum, o, 64);
    if (!mine) continue;
    if (kind < 2) {
      const bool norm = kind == 0 ? a.q_weight != nullptr : a.k_weight != nullptr;
      if (norm) {
        const float scale = 1.f / sqrtf(fmaf(sum, a.mean, a.eps));
#pragma unroll
        for (int i = 0; i < 8; ++i) f[i] = f[i] * scale * (kind == 0 ? wq[i] : wk[i]);
      }
      if (turns) {
        float y[8];
        if (a.interleaved) {
#pragma unroll
          for (int i = 0; i < 4; ++i) {
            y[2 * i] = f[2 * i] * cs[i] - f[2 * i + 1] * sn[i];
            y[2 * i + 1] = f[2 * i] * sn[i] + f[2 * i + 1] * cs[i];
          }
        } else {
#pragma unroll
          for (int i = 0; i < 4; ++i) {
            y[i] = f[i] * cs[i] - f[i + 4] * sn[i];
            y[i + 4] = f[i] * sn[i] + f[i + 4] * cs[i];
          }
        }
        x = Run<DT>::of(y);
      } else if (norm) {
        x = Run<DT>::of(f);
      }
    }
    if (kind == 0) x.template store<ONCE>(a.q_out + row * a.q_out_stride + (long long)hh * bytes, o0, o1);
    if (kind == 1 && a.k_out) x.template store<ONCE>(a.k_out + row * a.k_out_stride + (long long)hh * bytes, o0, o1);
    if (kind != 0 && at >= 0) x.template store<ONCE>((kind == 1 ? a.pool.k : a.pool.v) + at + hh * a.pool.head_stride, o0, o1);
  }
}

template <int DT, bool ONCE>
void launch_rope(const RopeArgs& a, int lanes, hipStream_t s) {
  const long long waves = a.n * a.parts;
  const dim3 grid((unsigned)((waves + kRopeThreads / kWave - 1) / (kRopeThreads / kWave))), block(kRopeThreads);
  if (lanes == 8) hipLaunchKernelGGL((k_qk_norm_rope<DT, 8, ONCE>), grid, block, 0, s, a);
  else if (lanes == 16) hipLaunchKernelGGL((k_qk_norm_rope<DT, 16, ONCE>), grid, block, 0, s, a);
  else hipLaunchKernelGGL((k_qk_norm_rope<DT, 32, ONCE>), grid, block, 0, s, a);
}

}  // namespace
}  // namespace sttm

using namespace sttm;

extern "C" int sttm_qk_norm_rope(sttm_ctx* ctx, int dtype, int64_t n, int q_heads, int kv_heads, int head_dim, const void* q,
                                 int64_t q_stride, const void* k, int64_t k_stride, const void* v, int64_t v_stride,
                                 const void* q_weight, const void* k_weight, float eps, const sttm_rope* rope, void* q_out,
                                 int64_t q_out_stride, void* k_out, int64_t k_out_stride, const sttm_cache* cache,
                                 const int64_t* slots) {
  if (!ctx) return STTM_ERR_NULL;
  if (dtype != STTM_F32 && dtype != STTM_BF16 && dtype != STTM_F16)
    return ctx_fail(ctx, STTM_ERR_DTYPE, "dtype must be STTM_F32, STTM_BF16 or STTM_F16");
  if (n < 0 || n > (1ll << 25) || q_heads < 1 || kv_heads < 1 || q_heads > 4096 || kv_heads > 1024 || q_heads + 2 * kv_heads > 4096 ||
      head_dim < 8 || head_dim > 256 || head_dim % 8)
    return ctx_fail(ctx, STTM_ERR_SHAPE, "need 0 <= n <= 2^25, heads >= 1, q_heads + 2 * kv_heads <= 4096, head_dim % 8 == 0, 8 <= head_dim <= 256");
  const int es = elem_bytes(dtype), align = 16 / es;
  const int64_t q_row = (int64_t)q_heads * head_dim, kv_row = (int64_t)kv_heads * head_dim, most = (int64_t)1 << 40;
  auto bad = [&](int64_t stride, int64_t row) { return stride < row || stride > most || stride % align; };
  if (bad(q_stride, q_row) || bad(k_stride, kv_row) || bad(q_out_stride, q_row) || (k_out && bad(k_out_stride, kv_row)) ||
      (cache && bad(v_stride, kv_row)))
    return ctx_fail(ctx, STTM_ERR_SHAPE, "row strides: multiples of 16 bytes, no less than a row");
  if (!(eps >= 0.f)) return ctx_fail(ctx, STTM_ERR_ARG, "eps must be a number >= 0");
  RopeArgs a{};
  a.cut1 = a.cut2 = 1 << 30;
  if (rope) {
    for (int i = 0; i < 3; ++i)
      if (rope->sections[i] < 0 || rope->sections[i] > head_dim / 2) return ctx_fail(ctx, STTM_ERR_SHAPE, "sections: between 0 and head_dim / 2");
    a.cut1 = rope->sections[0];
    a.cut2 = a.cut1 + rope->sections[1];
    a.pairs = a.cut2 + rope->sections[2];
    if (a.pairs % 4 || 2 * a.pairs > head_dim)
      return ctx_fail(ctx, STTM_ERR_SHAPE, "the sections' sum must be a multiple of 4 and at most head_dim / 2");
    if (a.pairs) {
      if (n && (!rope->positions || !rope->inv_freq)) return ctx_fail(ctx, STTM_ERR_NULL, "positions or inv_freq is NULL");
      const int axes = rope->sections[2] ? 3 : rope->sections[1] ? 2 : 1;
      if (rope->pos_stride < axes || rope->pos_stride > most) return ctx_fail(ctx, STTM_ERR_SHAPE, "pos_stride: no less than the axes in use");
      a.positions = rope->positions;
      a.inv_freq = rope->inv_freq;
      a.pos_stride = rope->pos_stride;
      a.pos_float = rope->pos_float != 0;
      a.interleaved = rope->interleaved != 0;
    }
  }
  if (cache) {
    int rc = check_cache(ctx, cache);
    if (rc != STTM_OK) return rc;
    if (cache->dtype != dtype) return ctx_fail(ctx, STTM_ERR_DTYPE, "the cache has another dtype");
    if (cache->kv_heads != kv_heads || cache->head_dim != head_dim) return ctx_fail(ctx, STTM_ERR_SHAPE, "the cache has other heads");
    a.pool = make_pool(cache);
    a.total_slots = cache->pages * cache->page_size;
    a.cached = 1;
  }
  if (n == 0) return STTM_OK;
  if (!q || !k || !q_out || (cache && (!v || !slots))) return ctx_fail(ctx, STTM_ERR_NULL, "q, k, q_out, or v or slots with a cache, is NULL");
  if (!aligned16(q) || !aligned16(k) || !aligned16(v) || !aligned16(q_out) || !aligned16(k_out) || !aligned16(q_weight) || !aligned16(k_weight))
    return ctx_fail(ctx, STTM_ERR_ARG, "rows and weights must be 16-byte aligned");
  a.q = static_cast<const char*>(q); a.k = static_cast<const char*>(k); a.v = static_cast<const char*>(v);
  a.q_out = static_cast<char*>(q_out); a.k_out = static_cast<char*>(k_out);
  a.q_stride = q_stride * es; a.k_stride = k_stride * es; a.v_stride = v_stride * es;
  a.q_out_stride = q_out_stride * es; a.k_out_stride = k_out_stride * es;
  a.q_weight = q_weight; a.k_weight = k_weight;
  a.slots = reinterpret_cast<const long long*>(slots);
  a.n = n;
  a.eps = eps; a.mean = 1.f / (float)head_dim;
  a.q_heads = q_heads; a.kv_heads = kv_heads; a.d = head_dim;
  const int lanes = head_dim <= 64 ? 8 : head_dim <= 128 ? 16 : 32;
  const int steps = (q_heads + 2 * kv_heads + kWave / lanes - 1) / (kWave / lanes);  // rows of heads a token has
  // Few tokens: their heads are spread over wavefronts until there are some for every SIMD.
  a.parts = 1;
  while (a.parts < steps && n * a.parts < kRopeWaves) a.parts *= 2;
  if (a.parts > steps) a.parts = steps;
  const bool once = n * (int64_t)(q_heads + (k_out ? kv_heads : 0) + (cache ? 2 * kv_heads : 0)) * head_dim * es > kOnceBytes;
  int rc = ctx_device(ctx);
  if (rc != STTM_OK) return rc;
  const hipStream_t s = ctx_stream(ctx);
  if (dtype == STTM_F32) once ? launch_rope<0, true>(a, lanes, s) : launch_rope<0, false>(a, lanes, s);
  else if (dtype == STTM_BF16) once ? launch_rope<1, true>(a, lanes, s) : launch_rope<1, false>(a, lanes, s);
  else once ? launch_rope<2, true>(a, lanes, s) : launch_rope<2, false>(a, lanes, s);
  return ctx_after_launch(ctx);
}
