// Eviction from a paged cache by accumulated attention weight: which slots stay, and the rows that move for it.
#include "sttm_cache.h"

#include <algorithm>

namespace sttm {
namespace {

// A survivor from behind the new length, with its entries in the tables.
struct Mover {
  int32_t slot, id;
  float weight, bias;
};

struct EvictArgs {
  Pool pool;
  Seqs seqs;
  const int32_t *keep, *total;
  long long slot_stride;
  const float *weights_in, *bias_in;
  const int32_t* ids_in;
  float *weights_out, *bias_out;
  int32_t *ids_out, *lengths_out;
  int kv_heads, sink, recent;
  Mover* movers;    // [batch, kv_heads, max_len]
  int32_t* holes;   // [batch, kv_heads, max_len]
  int2* counts;     // [batch, kv_heads]: movers (= holes), new length
};

// The order of the slots as a 64-bit number, larger ones stay: the class and weight, then the lower number.
__device__ inline unsigned long long rank_key(float w, int id, int total, const EvictArgs& a) {
  unsigned hi;
  if (id < a.sink || (long long)id >= (long long)total - a.recent) hi = 0xffffffffu;
  else if (w != w) hi = 0u;
  else hi = float_key(w == 0.f ? 0.f : w);   // (0x007fffff .. 0xff800000; both zeros alike)
  return (unsigned long long)hi << 32 | ~(unsigned)id;
}

constexpr int kEvictThreads = 1024, kEvictWaves = kEvictThreads / kWave;

// One workgroup a (sequence, kv head). The new length's largest keys are found digit by digit from the top (eight bits a
// pass, until the digits so far cut off exactly as many as stay); one more pass deals out holes and movers in the order of
// their slots and writes the tables.
__global__ void __launch_bounds__(kEvictThreads) k_evict_select(EvictArgs a) {
  __shared__ unsigned hist[256];
  __shared__ unsigned long long prefix_s;
  __shared__ int left_s, done_s;
  __shared__ int wave_holes[kEvictWaves], wave_movers[kEvictWaves];
  const int h = blockIdx.x, b = blockIdx.y, tid = threadIdx.x, lane = tid & 63, wave = tid >> 6;
  const long long row = (long long)b * a.kv_heads + h, at = row * a.slot_stride;
  const int length = seq_length(a.seqs, b), total = a.total ? a.total[b] : length;
  const int stay = min(length, max(a.keep[b], 0));
  auto number = [&](int i) {
    const int id = a.ids_in ? a.ids_in[at + i] : -1;
    return id < 0 ? total - length + i : id;
  };

  // Keys that agree with `prefix` in the bits above `shift` are still open; `left` of them stay.
  unsigned long long prefix = 0;
  int shift = 64, left = stay;
  bool done = stay == length || stay == 0;
  while (!done) {
    shift -= 8;
    for (int i = tid; i < 256; i += kEvictThreads) hist[i] = 0;
    __syncthreads();
    for (int i = tid; i < length; i += kEvictThreads) {
      const unsigned long long k = rank_key(a.weights_in[at + i], number(i), total, a);
      if (shift == 56 || (k >> (shift + 8)) == (prefix >> (shift + 8))) atomicAdd(&hist[(k >> shift) & 255], 1u);
    }
    __syncthreads();
    if (tid == 0) {
      int rest = left, digit = 255;
      while (digit > 0 && (int)hist[digit] < rest) rest -= (int)hist[digit--];
      prefix_s = prefix | (unsigned long long)digit << shift;
      left_s = rest;
      done_s = (int)hist[digit] == rest || shift == 0;
    }
    __syncthreads();
    prefix = prefix_s;
    left = left_s;
    done = done_s != 0;
    __syncthreads();
  }
  // stays: key >= prefix (in the bits from `shift` up)
  const bool all = stay == length, none = stay == 0;
  int holes = 0, movers = 0;
  for (int i0 = 0; i0 < length; i0 += kEvictThreads) {
    const int i = i0 + tid;
    const bool in = i < length;
    float w = 0.f, bias = 0.f;
    int id = 0;
    bool stays = false;
    if (in) {
      w = a.weights_in[at + i];
      id = number(i);
      if (a.bias_in) bias = a.bias_in[at + i];
      stays = all || (!none && rank_key(w, id, total, a) >= prefix);
    }
    const bool hole = in && i < stay && !stays, mover = in && i >= stay && stays;
    const unsigned long long hole_mask = __ballot(hole), mover_mask = __ballot(mover);
    if (lane == 0) {
      wave_holes[wave] = __popcll(hole_mask);
      wave_movers[wave] = __popcll(mover_mask);
    }
    __syncthreads();
    int my_hole = holes, my_mover = movers;
    for (int v = 0; v < kEvictWaves; ++v) {
      if (v < wave) { my_hole += wave_holes[v]; my_mover += wave_movers[v]; }
      holes += wave_holes[v];
      movers += wave_movers[v];
    }
    __syncthreads();
    const unsigned long long below = (1ull << lane) - 1;
    if (hole) a.holes[row * a.seqs.max_len + my_hole + __popcll(hole_mask & below)] = i;
    if (mover) a.movers[row * a.seqs.max_len + my_mover + __popcll(mover_mask & below)] = Mover{i, id, w, bias};
    if (in && !hole) {
      const bool gone = i >= stay;
      a.weights_out[at + i] = gone ? 0.f : w;
      a.ids_out[at + i] = gone ? -1 : id;
      if (a.bias_out) a.bias_out[at + i] = gone ? 0.f : bias;
    }
  }
  if (tid == 0) a.counts[row] = make_int2(movers, stay);
}

// The j-th mover's rows go to the j-th hole: 2^LOG_LANES lanes a row, 16 bytes a lane.
constexpr int kMoveThreads = 256;
template <int LANES>
__global__ void __launch_bounds__(kMoveThreads) k_evict_move(EvictArgs a) {
  const int h = blockIdx.y, b = blockIdx.z, tid = threadIdx.x, unit = tid & (LANES - 1);
  const long long row = (long long)b * a.kv_heads + h, at = row * a.slot_stride;
  const int2 count = a.counts[row];
  if (blockIdx.x == 0 && h == 0 && tid == 0) a.lengths_out[b] = count.y;
  const int step = gridDim.x * (kMoveThreads / LANES), mask = (1 << a.pool.shift) - 1;
  for (int j = blockIdx.x * (kMoveThreads / LANES) + tid / LANES; j < count.x; j += step) {
    const Mover m = a.movers[row * a.seqs.max_len + j];
    const int hole = a.holes[row * a.seqs.max_len + j];
    if (unit == 0) {
      a.weights_out[at + hole] = m.weight;
      a.ids_out[at + hole] = m.id;
      if (a.bias_out) a.bias_out[at + hole] = m.bias;
    }
    const int p = a.seqs.table[b * a.seqs.table_stride + (m.slot >> a.pool.shift)];
    const int q = a.seqs.table[b * a.seqs.table_stride + (hole >> a.pool.shift)];
    if (p < 0 || p >= a.pool.pages || q < 0 || q >= a.pool.pages || unit * 16 >= a.pool.row) continue;
    const long long from = p * a.pool.page_stride + h * a.pool.head_stride + (long long)(m.slot & mask) * a.pool.token_stride + unit * 16;
    const long long to = q * a.pool.page_stride + h * a.pool.head_stride + (long long)(hole & mask) * a.pool.token_stride + unit * 16;
    const uint4 k = *reinterpret_cast<const uint4*>(a.pool.k + from), v = *reinterpret_cast<const uint4*>(a.pool.v + from);
    *reinterpret_cast<uint4*>(a.pool.k + to) = k;
    *reinterpret_cast<uint4*>(a.pool.v + to) = v;
  }
}

struct Plan {
  size_t movers, holes, counts, bytes;
};
Plan make_plan(const sttm_cache* c, const sttm_sequences* s) {
  Plan p;
  size_t off = 0;
  auto take = [&](size_t bytes) { size_t o = off; off = (off + bytes + 255) / 256 * 256; return o; };
  const size_t rows = (size_t)s->batch * c->kv_heads, slots = (size_t)make_seqs(c, s).max_len;
  p.movers = take(rows * slots * sizeof(Mover));
  p.holes = take(rows * slots * sizeof(int32_t));
  p.counts = take(rows * sizeof(int2));
  p.bytes = std::max(off, (size_t)256);
  return p;
}

int check_evict(sttm_ctx* ctx, const sttm_cache* cache, const sttm_sequences* seqs) {
  int rc = check_cache(ctx, cache);
  if (rc == STTM_OK) rc = check_sequences(ctx, cache, seqs);
  if (rc != STTM_OK) return rc;
  if ((double)seqs->batch * cache->kv_heads * seqs->max_len > 1e13) return ctx_fail(ctx, STTM_ERR_SHAPE, "batch * kv_heads * max_len too large");
  return STTM_OK;
}

}  // namespace
}  // namespace sttm

using namespace sttm;

extern "C" size_t sttm_cache_evict_workspace_bytes(const sttm_cache* cache, const sttm_sequences* seqs) {
  if (check_evict(nullptr, cache, seqs) != STTM_OK) return 0;
  return make_plan(cache, seqs).bytes;
}

extern "C" int sttm_cache_evict(sttm_ctx* ctx, const sttm_cache* cache, const sttm_sequences* seqs, const int32_t* keep,
                                const int32_t* total, int sink, int recent, int64_t slot_stride, const float* weights_in,
                                float* weights_out, const int32_t* ids_in, int32_t* ids_out, const float* bias_in,
                                float* bias_out, int32_t* lengths_out, void* workspace, size_t workspace_bytes) {
  if (!ctx) return STTM_ERR_NULL;
  int rc = check_evict(ctx, cache, seqs);
  if (rc != STTM_OK) return rc;
  EvictArgs a{};
  a.seqs = make_seqs(cache, seqs);
  if (slot_stride < a.seqs.max_len || slot_stride > ((int64_t)1 << 40)) return ctx_fail(ctx, STTM_ERR_SHAPE, "slot_stride must be no less than max_len");
  if (sink < 0 || recent < 0) return ctx_fail(ctx, STTM_ERR_ARG, "sink and recent must not be negative");
  if (!bias_in != !bias_out) return ctx_fail(ctx, STTM_ERR_ARG, "bias_in and bias_out: both or neither");
  if (seqs->batch == 0) return STTM_OK;
  if (!keep || !weights_in || !weights_out || !ids_out || !lengths_out)
    return ctx_fail(ctx, STTM_ERR_NULL, "keep, weights_in, weights_out, ids_out or lengths_out is NULL");
  const Plan p = make_plan(cache, seqs);
  rc = check_workspace(ctx, workspace, workspace_bytes, p.bytes);
  if (rc != STTM_OK) return rc;
  char* ws = static_cast<char*>(workspace);
  a.pool = make_pool(cache);
  a.keep = keep;
  a.total = total;
  a.slot_stride = slot_stride;
  a.weights_in = weights_in; a.weights_out = weights_out;
  a.ids_in = ids_in; a.ids_out = ids_out;
  a.bias_in = bias_in; a.bias_out = bias_out;
  a.lengths_out = lengths_out;
  a.kv_heads = cache->kv_heads;
  a.sink = sink;
  a.recent = recent;
  a.movers = reinterpret_cast<Mover*>(ws + p.movers);
  a.holes = reinterpret_cast<int32_t*>(ws + p.holes);
  a.counts = reinterpret_cast<int2*>(ws + p.counts);
  rc = ctx_device(ctx);
  if (rc != STTM_OK) return rc;
  const hipStream_t s = ctx_stream(ctx);
  hipLaunchKernelGGL(k_evict_select, dim3(a.kv_heads, seqs->batch), dim3(kEvictThreads), 0, s, a);
  const int lanes = a.pool.row <= 128 ? 8 : a.pool.row <= 256 ? 16 : a.pool.row <= 512 ? 32 : 64;
  // At most half of the slots move; some eight rows for a group of lanes.
  const int groups = kMoveThreads / lanes;
  const dim3 grid(std::max(1, (a.seqs.max_len / 2 + 8 * groups - 1) / (8 * groups)), a.kv_heads, seqs->batch), block(kMoveThreads);
  if (lanes == 8) hipLaunchKernelGGL((k_evict_move<8>), grid, block, 0, s, a);
  else if (lanes == 16) hipLaunchKernelGGL((k_evict_move<16>), grid, block, 0, s, a);
  else if (lanes == 32) hipLaunchKernelGGL((k_evict_move<32>), grid, block, 0, s, a);
  else hipLaunchKernelGGL((k_evict_move<64>), grid, block, 0, s, a);
  return ctx_after_launch(ctx);
}
