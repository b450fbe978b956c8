// Entry points of the attention of several queries: over the packed rows of a batch, and over a prefix that sequences of a paged cache share.
#include "sttm_queries.h"

#include <algorithm>
#include <cmath>

namespace sttm {
namespace {

constexpr int kJoinThreads = 256, kJoinHeads = 4, kJoinWaves = 4096;  // (rows from which on a wavefront each)

// The sequence, and for a launch over groups its segment, that a token belongs to; -1: none.
__device__ inline int sequence_of(const QueryArgs& a, long long token) {
  if (a.batch == 0) return -1;
  const int b = last_not_above(a.batch, token, [&](int i) { return first_token(a, i); });
  return first_token(a, b) <= token && token < first_token(a, b + 1) ? b : -1;
}
__device__ inline int segment_of(const QueryArgs& a, int b) {
  if (!a.cuts) return b;
  if (a.segments == 0) return -1;
  const int s = last_not_above(a.segments, b, [&](int i) { return clamped(a.cuts[i], a.batch); });
  return clamped(a.cuts[s], a.batch) <= b && b < clamped(a.cuts[s + 1], a.batch) ? s : -1;
}
__device__ inline int parts_of(const QueryArgs& a, const KeyArgs& k, int b) {
  const int s = segment_of(a, b);
  if (s < 0) return 0;
  long long first;
  const int length = segment_length(k, s, &first);
  return max((length + k.chunk - 1) / k.chunk, 1);
}

// A row's parts on a common maximum: those of the prefix, then its own, added up in a fixed order. Tokens of no sequence stay
// as they are, and rows whose only part is their result already.
// LANES lanes have a row, four channels each, the parts dealt out among as many groups of lanes as there are. A workgroup where there are few rows (their
// parts come from all over memory at once: 32 tokens, 28 heads, 58 parts of 128 channels 9 us), a wavefront with four of a token's heads in turn else.
template <int DT, int LANES>
__global__ void __launch_bounds__(kJoinThreads) k_query_join(QueryArgs a, KeyArgs ka, QueryArgs b, KeyArgs kb) {
  __shared__ float4 sums[kJoinThreads];
  constexpr int ES = DT == 0 ? 4 : 2, HEADS = LANES == kJoinThreads ? 1 : kJoinHeads;
  const long long token = blockIdx.x;
  const int tid = threadIdx.x, lane = tid & 63, u = tid & (LANES - 1);
  const int seq = sequence_of(b, token);
  if (seq < 0) return;
  const int of_a = ka.chunks ? parts_of(a, ka, seq) : 0, of_b = parts_of(b, kb, seq), n = of_a + of_b, heads = b.kv_heads * b.group;
  if (b.alone && n == 1) return;
  const int units = b.d / 4, slices = LANES / units, unit = u % units, slice = u / units;
  auto at = [&](int i) { return i < of_a ? i : b.first_part + i - of_a; };
  for (int i = 0; i < HEADS; ++i) {
    const int head = (blockIdx.y * (kJoinThreads / LANES) + tid / LANES) * HEADS + i;
    if (head >= heads) return;                            // (all lanes of a row)
    const long long index = token * heads + head;
    const float2* stat = b.stat + index * b.parts;
    float top = -INFINITY, total = 0.f;
    for (int p = lane; p < n; p += kWave) top = fmaxf(top, stat[at(p)].x);
#pragma unroll
    for (int o = 32; o > 0; o >>= 1) top = fmaxf(top, __shfl_xor(top, o, 64));
    for (int p = lane; p < n; p += kWave) total = fmaf(stat[at(p)].y, query_factor(stat[at(p)].x, top), total);
#pragma unroll
    for (int o = 32; o > 0; o >>= 1) total += __shfl_xor(total, o, 64);
    if (u == 0 && b.lse) b.lse[index] = top + logf(total);
    float4 x = make_float4(0.f, 0.f, 0.f, 0.f);
    if (slice < slices) {
#pragma unroll 4
      for (int p = slice; p < n; p += slices) {
        const float4 y = *reinterpret_cast<const float4*>(b.part + (index * b.parts + at(p)) * b.d + 4 * unit);
        const float f = query_factor(stat[at(p)].x, top);
        x.x = fmaf(y.x, f, x.x); x.y = fmaf(y.y, f, x.y); x.z = fmaf(y.z, f, x.z); x.w = fmaf(y.w, f, x.w);
      }
    }
    sums[tid] = x;
    if constexpr (LANES == kJoinThreads) __syncthreads();
    else __builtin_amdgcn_wave_barrier();
    if (slice == 0) {
      for (int p = 1; p < slices; ++p) {
        const float4 y = sums[tid - u + p * units + unit];
        x.x += y.x; x.y += y.y; x.z += y.z; x.w += y.w;
      }
      const float f = total == 0.f ? 0.f : 1.f / total;
      char* out = b.out + token * b.out_stride + ((long long)head * b.d + 4 * unit) * ES;
      if constexpr (DT == 0) *reinterpret_cast<float4*>(out) = make_float4(x.x * f, x.y * f, x.z * f, x.w * f);
      else *reinterpret_cast<uint2*>(out) = make_uint2(pack2<DT>(x.x * f, x.y * f), pack2<DT>(x.z * f, x.w * f));
    }
    if constexpr (LANES != kJoinThreads) __builtin_amdgcn_wave_barrier();
  }
}

// ---- launches -----------------------------------------------------------------------------------------------------

// In blocks of 64 keys (2 us): a workgroup's beginning and end, of the last one's time, a second launch, a channel of a part written and read again.
constexpr double kEnds = 3, kTail = 0.75, kJoin = 2, kPart = 7e-7;

// How the keys of one kind of segment are cut.
struct Cut {
  int chunk, chunks;
};
bool few_rows(int64_t tokens, int group, int segments) { return tokens * group <= (int64_t)kRowTile * segments; }
Cut make_cut(bool few, int64_t tokens, int group, int segments, int kv_heads, int64_t max_len, int d, int es) {
  Cut c{64, 1};
  if (segments < 1) return c;
  const int64_t rows = tokens * group, row_bytes = query_row_bytes(d, es);
  // Workgroups of one chunk each: at most one a tile more than the rows fill, and a compute unit holds two (few rows, wide rows: one).
  const int64_t tiles = (rows / query_tile(few) + std::min<int64_t>(segments, rows)) * kv_heads, slots = row_bytes > 512 || (!few && row_bytes > 256) ? 256 : 512;
  if (few) {
    // Bound by memory and by how even the load is: chunks of 1,024 keys, shorter ones where those would not make three or four rounds (whole calls by
    // 256 / 512 / 1,024 / 2,048, us: 32 sequences of 1,013 to 8,117 keys, 64 heads on 8 of 128 bf16 channels 125 / 110 / 106 / 119; 5 of 333 to 4,979,
    // 16 heads of 72, fp32 85 / 91 / 109 / 204); one for short ones, where a second launch costs more than blocks that follow each other (257
    // keys 10.0, as two chunks 13.1).
    c.chunk = 1024;
    while (c.chunk > 256 && tiles * ((max_len + c.chunk - 1) / c.chunk) < 1800) c.chunk /= 2;
    if (max_len <= 512) c.chunk = 512;
    while ((int64_t)segments * ((max_len + c.chunk - 1) / c.chunk) > 1 << 20) c.chunk *= 2;      // (a grid has fewer than 2^32 workgroups)
    c.chunks = (int)std::max<int64_t>(1, (max_len + c.chunk - 1) / c.chunk);
    return c;
  }
  // The cut with the least time, in units of a block of 64 keys: workgroups in rounds (one length), or all their work dealt out and the longest one
  // behind it (lengths of half the largest on average), which has a compute unit to itself by then, each with a beginning and an end; a second launch, and what
  // it takes to write and read each part of a row. Whole calls with chunks of 1,024 / 2,048 / 4,096 keys / one chunk, us: one prompt of 331 tokens on
  // 43,264 keys, 28 heads on 4, 326 / 308 / 284 / 1,015 (the rule: 3,328, 272); ten of 19 to 160 on up to 6,491, 64 on 8, 181 / 165 / 165 / 158; eight of
  // 13 to 211 behind two of up to 8,191 slots, 28 on 4, 126 / 111 / 179 / 252 (1,536: 140); 32 of one behind 43,264 slots 67 / 81 / 138 / 1,284 (the rule: 704, 60).
  const int64_t blocks = (max_len + 63) / 64;
  double best = 0;
  for (int64_t n = 1; n <= std::min<int64_t>(blocks, 256); ++n) {
    const int64_t chunk = (blocks + n - 1) / n;
    if ((blocks + chunk - 1) / chunk != n) continue;      // (as many blocks each as with fewer)
    const double work = (double)tiles * n * (chunk + kEnds) / slots;
    const double time = segments == 1 ? std::ceil((double)tiles * n / slots) * (chunk + kEnds) : work / 2 + (chunk + kEnds) * kTail;
    const double cost = time + (n > 1 ? kJoin + (double)rows * kv_heads * n * d * kPart : 0);
    if (n == 1 || cost < best) {
      best = cost;
      c.chunk = (int)chunk * 64;
      c.chunks = (int)n;
    }
  }
  return c;
}

struct Plan {
  bool few;
  Cut a, b;          // segments of several sequences (none: no chunks), segments of one
  int parts;
  size_t part, stat, bytes;
};
Plan make_plan(bool few, Cut a, Cut b, int64_t tokens, int q_heads, int d) {
  Plan p{few, a, b, a.chunks + b.chunks, 0, 0, 0};
  size_t off = 0;
  auto take = [&](size_t bytes) { size_t o = off; off = (off + bytes + 255) / 256 * 256; return o; };
  const size_t rows = p.parts > 1 ? (size_t)tokens * q_heads * p.parts : 0;
  p.part = take(rows * d * sizeof(float));
  p.stat = take(rows * sizeof(float2));
  p.bytes = std::max(off, (size_t)256);
  return p;
}

int check_queries(sttm_ctx* ctx, int64_t tokens, int q_heads, int kv_heads, int64_t max_len) {
  if (tokens < 0 || tokens > (1ll << 22)) return ctx_fail(ctx, STTM_ERR_SHAPE, "need 0 <= tokens <= 2^22");
  if (q_heads < 1 || q_heads % kv_heads || q_heads / kv_heads > 256 || q_heads > 65535)
    return ctx_fail(ctx, STTM_ERR_SHAPE, "need q_heads a multiple of kv_heads, at most 256 a kv head, q_heads <= 65535");
  if (tokens * (q_heads / kv_heads) > (1ll << 28)) return ctx_fail(ctx, STTM_ERR_SHAPE, "need tokens * q_heads / kv_heads <= 2^28");
  if ((double)tokens * q_heads * max_len > 1e15) return ctx_fail(ctx, STTM_ERR_SHAPE, "tokens * q_heads * keys too large");
  return STTM_OK;
}

int check_states(sttm_ctx* c, const sttm_states* s) {
  if (!s) return ctx_fail(c, STTM_ERR_NULL, "states is NULL");
  if (s->dtype != STTM_F32 && s->dtype != STTM_BF16 && s->dtype != STTM_F16)
    return ctx_fail(c, STTM_ERR_DTYPE, "dtype must be STTM_F32, STTM_BF16 or STTM_F16");
  if (s->head_dim < 8 || s->head_dim > 256 || s->head_dim % 8 || s->kv_heads < 1 || s->kv_heads > 1024 || s->rows < 0 || s->rows > (1ll << 40) ||
      s->batch < 0 || s->batch > 65535 || s->max_rows < 0 || s->max_rows > 1 << 30)
    return ctx_fail(c, STTM_ERR_SHAPE, "need head_dim % 8 == 0, 8 <= head_dim <= 256, 1 <= kv_heads <= 1024, 0 <= rows <= 2^40, 0 <= batch <= 65535, 0 <= max_rows <= 2^30");
  const int64_t align = 16 / elem_bytes(s->dtype), most = (int64_t)1 << 40;
  if (s->row_stride < 0 || s->head_stride < 0 || s->row_stride > 1 << 22 || s->head_stride > most || s->row_stride % align || s->head_stride % align)
    return ctx_fail(c, STTM_ERR_SHAPE, "strides of the states: multiples of 16 bytes, not negative, row_stride at most 2^22");
  if (s->batch && !s->offsets) return ctx_fail(c, STTM_ERR_NULL, "offsets is NULL");
  if (s->batch && s->rows && s->max_rows && (!s->k || !s->v)) return ctx_fail(c, STTM_ERR_NULL, "k or v of the states is NULL");
  if (!aligned16(s->k) || !aligned16(s->v)) return ctx_fail(c, STTM_ERR_ARG, "k and v must be 16-byte aligned");
  return STTM_OK;
}

// What both calls ask of queries, results and scale, in the order in which they are looked at.
int check_rows(sttm_ctx* ctx, int dtype, int head_dim, int q_heads, int64_t tokens, int batch, const void* q, int64_t q_stride, const void* out,
               int64_t out_stride, const int64_t* q_offsets, float scale) {
  const int64_t align = 16 / elem_bytes(dtype), row = (int64_t)q_heads * head_dim, most = (int64_t)1 << 40;
  if (q_stride < row || out_stride < row || q_stride > most || out_stride > most || q_stride % align || out_stride % align)
    return ctx_fail(ctx, STTM_ERR_SHAPE, "q_stride, out_stride: multiples of 16 bytes, no less than a row");
  if (!q_offsets && tokens != batch) return ctx_fail(ctx, STTM_ERR_SHAPE, "without q_offsets there is one token for each sequence");
  if (!(std::fabs(scale) <= 3e38f)) return ctx_fail(ctx, STTM_ERR_ARG, "scale must be a finite number");
  if (tokens && batch && (!q || !out)) return ctx_fail(ctx, STTM_ERR_NULL, "q or out is NULL");
  if (!aligned16(q) || !aligned16(out)) return ctx_fail(ctx, STTM_ERR_ARG, "q and out must be 16-byte aligned");
  return STTM_OK;
}

Plan plan_cross(const sttm_states* s, int64_t tokens, int q_heads) {
  const int group = q_heads / s->kv_heads;
  const bool few = few_rows(tokens, group, s->batch);
  const Cut b = make_cut(few, tokens, group, s->batch, s->kv_heads, std::min<int64_t>(s->max_rows, s->rows), s->head_dim, elem_bytes(s->dtype));
  return make_plan(few, Cut{1, 0}, b, tokens, q_heads, s->head_dim);
}

// (Prefixes and own slots in one launch, with tiles of one size: those of the prefixes, whose rows are more.)
Plan plan_shared(const sttm_cache* c, const sttm_sequences* prefixes, const sttm_sequences* seqs, int64_t tokens, int q_heads) {
  const int group = q_heads / c->kv_heads, es = elem_bytes(c->dtype), groups = prefixes ? prefixes->batch : 0;
  const bool few = few_rows(tokens, group, groups ? groups : seqs->batch) && few_rows(tokens, group, seqs->batch);
  Cut a{1, 0};
  if (groups) a = make_cut(few, tokens, group, groups, c->kv_heads, make_seqs(c, prefixes).max_len, c->head_dim, es);
  return make_plan(few, a, make_cut(few, tokens, group, seqs->batch, c->kv_heads, make_seqs(c, seqs).max_len, c->head_dim, es), tokens, q_heads, c->head_dim);
}

template <int DT> void launch_all(QueryArgs a, KeyArgs ka, QueryArgs b, KeyArgs kb, const Plan& p, hipStream_t s) {
  QueryJobs jobs{};
  if (p.a.chunks) {
    jobs.q[0] = a;
    jobs.k[0] = ka;
    jobs.count = 1;
  }
  jobs.q[jobs.count] = b;
  jobs.k[jobs.count++] = kb;
  launch_queries<DT>(jobs, p.few, s);
  if (p.parts < 2) return;
  const unsigned tokens = (unsigned)b.tokens, heads = b.kv_heads * b.group, some = kJoinHeads * (kJoinThreads / kWave);
  if ((int64_t)tokens * heads < kJoinWaves) hipLaunchKernelGGL((k_query_join<DT, kJoinThreads>), dim3(tokens, heads), dim3(kJoinThreads), 0, s, a, ka, b, kb);
  else hipLaunchKernelGGL((k_query_join<DT, kWave>), dim3(tokens, (heads + some - 1) / some), dim3(kJoinThreads), 0, s, a, ka, b, kb);
}

int launch(sttm_ctx* ctx, int dtype, QueryArgs a, KeyArgs ka, QueryArgs b, KeyArgs kb, const Plan& p, char* ws) {
  const auto tiles = [&](const QueryArgs& x) { return x.tokens * x.group / query_tile(p.few) + x.segments; };
  if ((tiles(a) * p.a.chunks + tiles(b) * p.b.chunks) * b.kv_heads >= 1ll << 32) return ctx_fail(ctx, STTM_ERR_SHAPE, "more than 2^32 pieces of work");
  const int rc = ctx_device(ctx);
  if (rc != STTM_OK) return rc;
  if (p.parts > 1) {
    a.part = b.part = reinterpret_cast<float*>(ws + p.part);
    a.stat = b.stat = reinterpret_cast<float2*>(ws + p.stat);
  }
  a.parts = b.parts = p.parts;
  b.alone = p.a.chunks == 0;
  a.first_part = 0;
  b.first_part = p.a.chunks;
  ka.chunk = p.a.chunk; ka.chunks = p.a.chunks;
  kb.chunk = p.b.chunk; kb.chunks = p.b.chunks;
  const hipStream_t s = ctx_stream(ctx);
  if (dtype == STTM_F32) launch_all<0>(a, ka, b, kb, p, s);
  else if (dtype == STTM_BF16) launch_all<1>(a, ka, b, kb, p, s);
  else launch_all<2>(a, ka, b, kb, p, s);
  return ctx_after_launch(ctx);
}

QueryArgs make_queries(int dtype, int64_t tokens, int batch, int q_heads, int kv_heads, int head_dim, float scale, const void* q, int64_t q_stride,
                       const int64_t* q_offsets, void* out, int64_t out_stride, float* lse) {
  QueryArgs a{};
  a.q = static_cast<const char*>(q);
  a.out = static_cast<char*>(out);
  a.lse = lse;
  a.q_stride = q_stride * elem_bytes(dtype);
  a.out_stride = out_stride * elem_bytes(dtype);
  a.offsets = reinterpret_cast<const long long*>(q_offsets);
  a.tokens = tokens;
  a.batch = a.segments = batch;
  a.kv_heads = kv_heads;
  a.group = q_heads / kv_heads;
  a.d = head_dim;
  a.scale = scale;
  return a;
}

KeyArgs make_paged(const sttm_cache* c, const sttm_sequences* s, const float* bias, int64_t slots) {
  KeyArgs k{};
  const Seqs seqs = make_seqs(c, s);
  k.pool = make_pool(c);
  k.table = seqs.table;
  k.lengths = seqs.lengths;
  k.table_stride = seqs.table_stride;
  k.max_len = seqs.max_len;
  k.token_stride = k.pool.token_stride;
  k.slot_mask = c->page_size - 1;
  k.bias = bias;
  k.bias_segment = c->kv_heads * slots;
  k.bias_head = slots;
  return k;
}

}  // namespace
}  // namespace sttm

using namespace sttm;

extern "C" size_t sttm_cross_attention_workspace_bytes(const sttm_states* states, int64_t tokens, int q_heads) {
  if (check_states(nullptr, states) != STTM_OK) return 0;
  if (check_queries(nullptr, tokens, q_heads, states->kv_heads, std::min<int64_t>(states->max_rows, states->rows)) != STTM_OK) return 0;
  return plan_cross(states, tokens, q_heads).bytes;
}

extern "C" int sttm_cross_attention(sttm_ctx* ctx, const sttm_states* states, int64_t tokens, int q_heads, float scale, const void* q,
                                    int64_t q_stride, const int64_t* q_offsets, const float* key_bias, int64_t bias_stride, void* out,
                                    int64_t out_stride, float* lse, void* workspace, size_t workspace_bytes) {
  if (!ctx) return STTM_ERR_NULL;
  int rc = check_states(ctx, states);
  if (rc != STTM_OK) return rc;
  const int64_t max_len = std::min<int64_t>(states->max_rows, states->rows);
  rc = check_queries(ctx, tokens, q_heads, states->kv_heads, max_len);
  if (rc == STTM_OK) rc = check_rows(ctx, states->dtype, states->head_dim, q_heads, tokens, states->batch, q, q_stride, out, out_stride, q_offsets, scale);
  if (rc != STTM_OK) return rc;
  if (key_bias && bias_stride != 0 && (bias_stride < states->rows || bias_stride > (1ll << 40)))
    return ctx_fail(ctx, STTM_ERR_SHAPE, "bias_stride: zero, or no less than rows");
  if (tokens == 0 || states->batch == 0) return STTM_OK;
  const Plan p = plan_cross(states, tokens, q_heads);
  rc = check_workspace(ctx, workspace, workspace_bytes, p.bytes);
  if (rc != STTM_OK) return rc;
  const QueryArgs b = make_queries(states->dtype, tokens, states->batch, q_heads, states->kv_heads, states->head_dim, scale, q, q_stride, q_offsets, out,
                                   out_stride, lse);
  const int64_t es = elem_bytes(states->dtype);
  KeyArgs k{};
  k.pool.k = static_cast<char*>(const_cast<void*>(states->k));
  k.pool.v = static_cast<char*>(const_cast<void*>(states->v));
  k.pool.head_stride = states->head_stride * es;
  k.pool.row = (int)(states->head_dim * es);
  k.offsets = reinterpret_cast<const long long*>(states->offsets);
  k.rows = states->rows;
  k.max_len = (int)max_len;
  k.token_stride = states->row_stride * es;
  k.bias = key_bias;
  k.bias_head = bias_stride;
  return launch(ctx, states->dtype, QueryArgs{}, KeyArgs{}, b, k, p, static_cast<char*>(workspace));
}

extern "C" size_t sttm_shared_attention_workspace_bytes(const sttm_cache* cache, const sttm_sequences* prefixes, const sttm_sequences* seqs,
                                                        int64_t tokens, int q_heads) {
  if (check_cache(nullptr, cache) != STTM_OK || (prefixes && check_sequences(nullptr, cache, prefixes) != STTM_OK) ||
      check_sequences(nullptr, cache, seqs) != STTM_OK)
    return 0;
  const int64_t max_len = (int64_t)make_seqs(cache, seqs).max_len + (prefixes ? make_seqs(cache, prefixes).max_len : 0);
  if (check_queries(nullptr, tokens, q_heads, cache->kv_heads, max_len) != STTM_OK) return 0;
  return plan_shared(cache, prefixes, seqs, tokens, q_heads).bytes;
}

extern "C" int sttm_shared_attention(sttm_ctx* ctx, const sttm_cache* cache, const sttm_sequences* prefixes, const int32_t* group_offsets,
                                     const sttm_sequences* seqs, int64_t tokens, int q_heads, float scale, const void* q, int64_t q_stride,
                                     const int64_t* q_offsets, const float* prefix_bias, int64_t prefix_slots, const float* key_bias,
                                     int64_t key_slots, void* out, int64_t out_stride, float* lse, void* workspace, size_t workspace_bytes) {
  if (!ctx) return STTM_ERR_NULL;
  int rc = check_cache(ctx, cache);
  if (rc == STTM_OK && prefixes) rc = check_sequences(ctx, cache, prefixes);
  if (rc == STTM_OK) rc = check_sequences(ctx, cache, seqs);
  if (rc != STTM_OK) return rc;
  const int64_t prefix_len = prefixes ? make_seqs(cache, prefixes).max_len : 0, own_len = make_seqs(cache, seqs).max_len, most = (int64_t)1 << 40;
  rc = check_queries(ctx, tokens, q_heads, cache->kv_heads, prefix_len + own_len);
  if (rc == STTM_OK) rc = check_rows(ctx, cache->dtype, cache->head_dim, q_heads, tokens, seqs->batch, q, q_stride, out, out_stride, q_offsets, scale);
  if (rc != STTM_OK) return rc;
  if ((prefix_bias && (prefix_slots < prefix_len || prefix_slots > most)) || (key_bias && (key_slots < own_len || key_slots > most)))
    return ctx_fail(ctx, STTM_ERR_SHAPE, "a bias needs no fewer slots than the max_len of its sequences");
  if (prefix_bias && !prefixes) return ctx_fail(ctx, STTM_ERR_ARG, "prefix_bias without prefixes");
  if (prefixes && prefixes->batch && !group_offsets) return ctx_fail(ctx, STTM_ERR_NULL, "group_offsets is NULL");
  if (tokens == 0 || seqs->batch == 0) return STTM_OK;
  const Plan p = plan_shared(cache, prefixes, seqs, tokens, q_heads);
  rc = check_workspace(ctx, workspace, workspace_bytes, p.bytes);
  if (rc != STTM_OK) return rc;
  const QueryArgs b = make_queries(cache->dtype, tokens, seqs->batch, q_heads, cache->kv_heads, cache->head_dim, scale, q, q_stride, q_offsets, out,
                                   out_stride, lse);
  KeyArgs kb = make_paged(cache, seqs, key_bias, key_slots), ka{};
  kb.causal = 1;
  QueryArgs a = b;
  if (p.a.chunks) {
    a.cuts = group_offsets;
    a.segments = prefixes->batch;
    ka = make_paged(cache, prefixes, prefix_bias, prefix_slots);
  }
  return launch(ctx, cache->dtype, a, ka, b, kb, p, static_cast<char*>(workspace));
}
