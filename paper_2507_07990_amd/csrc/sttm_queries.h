// Attention of several queries: the rows of a segment's tokens over the segment's keys, in the packed rows of a batch or in the pages of a
// cache. One kernel for all element types and head sizes; the entry points (sttm_queries.hip) launch it once and put parts
// together.
#pragma once
#include "sttm_cache.h"

namespace sttm {

constexpr int kQueryThreads = 256, kQueryWaves = kQueryThreads / kWave;
constexpr int kRowTile = 32;    // query rows of a wavefront
constexpr float kLog2e = 1.4426950408889634f;

// Where the queries and results of a batch lie. A row of a matrix product is one token and one of the q heads of a kv head.
struct QueryArgs {
  const char* q;
  char* out;                     // of the whole attention (one part), else NULL
  float* lse;                    // may be NULL
  long long q_stride, out_stride;  // bytes
  const long long* offsets;      // [batch + 1], NULL: one token each
  long long tokens;
  int batch;
  const int32_t* cuts;           // [segments + 1]: segment s has the sequences cuts[s] .. cuts[s + 1] - 1; NULL: sequence s alone
  int segments;
  int kv_heads, group, d;
  float scale;
  float* part;                   // [tokens, q_heads, parts, d]: unnormalised sums (more than one part), else NULL
  float2* stat;                  // [tokens, q_heads, parts]: largest score and sum of exponentials of a part
  int alone;                     // no other kind has parts of these rows: a segment of one chunk has its result right away
  int parts, first_part;         // parts of a row in all, and where this kind's chunks begin among them
};

// Where the segments' keys and values lie: in pages (table) or one segment after the other (offsets).
struct KeyArgs {
  Pool pool;                     // packed rows: a page for each segment that begins at its first row
  const int32_t* table;
  const int32_t* lengths;
  long long table_stride;
  const long long* offsets;      // [segments + 1]
  long long rows;
  int max_len;
  long long token_stride;        // bytes
  int slot_mask;                 // the slots of a page less one
  const float* bias;             // NULL: none. Of slot i: bias[segment * bias_segment + h * bias_head + i] (packed: + the first row)
  long long bias_segment, bias_head;
  int causal;                    // (pages) token j of a segment's n sees the slots before length - (n - 1 - j)
  int chunk, chunks;
};

// What one launch does: up to two kinds of segments, the workgroups of the first one in front.
struct QueryJobs {
  QueryArgs q[2];
  KeyArgs k[2];
  int count;
  unsigned tiles[2];             // tiles of rows
  unsigned first, all;           // workgroups of the first kind, of both
};

__device__ inline long long clamped(long long x, long long most) { return min(max(x, 0ll), most); }

// First token of sequence b (b == batch: behind the last one).
__device__ inline long long first_token(const QueryArgs& a, long long b) {
  return a.offsets ? clamped(a.offsets[b], a.tokens) : min(b, a.tokens);
}
__device__ inline long long first_token_of_segment(const QueryArgs& a, int s) {
  return first_token(a, a.cuts ? clamped(a.cuts[s], a.batch) : s);
}

// The last i in 0 .. n - 1 for which at(i) <= x holds, at ascending (0 if there is none): 64 probes at a time, the same in all lanes.
template <class F> __device__ inline int last_not_above(int n, long long x, F at) {
  const int lane = threadIdx.x & 63;
  int lo = 0;
  while (n > 1) {
    const int step = (n + kWave - 1) / kWave, i = lane * step;
    const bool yes = i < n && at(lo + min(i, n - 1)) <= x;
    const int found = __popcll(__ballot(yes)), skip = max(found - 1, 0) * step;
    lo += skip;
    n = min(step, n - skip);
  }
  return lo;
}

// Rows first .. of a segment's keys: how many there are, and where the first one is (in rows; pages: 0).
__device__ inline int segment_length(const KeyArgs& k, int s, long long* first) {
  if (k.table || !k.offsets) {
    *first = 0;
    return k.lengths ? min(max(k.lengths[s], 0), k.max_len) : 0;
  }
  const long long from = clamped(k.offsets[s], k.rows), to = clamped(k.offsets[s + 1], k.rows);
  *first = from;
  return (int)min(max(to - from, 0ll), (long long)k.max_len);
}

// Softmax statistics of one row over several parts. (Differences are formed before they are multiplied by log2(e): a score may be the
// lowest fp32 number, or near the largest, and has no multiple then.)
__device__ inline float query_factor(float m, float top) { return exp2_fast((m - (top == -INFINITY ? 0.f : top)) * kLog2e); }

// One launch of the kernel. few_rows: a workgroup has 32 rows, its four wavefronts take blocks of keys in
// turn; else 128 rows that share the blocks.
template <int DT> void launch_queries(QueryJobs& jobs, bool few_rows, hipStream_t s);
// Rows of a workgroup's tile for this kind.
inline int query_tile(bool few_rows) { return few_rows ? kRowTile : kRowTile * kQueryWaves; }
// Bytes of a head's row in LDS: a power of two; above 512 a tile of its own for each wavefront would not fit.
constexpr int query_row_bytes(int d, int es) { return d * es <= 128 ? 128 : d * es <= 256 ? 256 : d * es <= 512 ? 512 : 1024; }

}  // namespace sttm
