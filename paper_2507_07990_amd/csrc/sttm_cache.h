// Shared declarations of the operators on a paged key-value cache (sttm_rope.hip, sttm_attention.hip, sttm_evict.hip).
#pragma once
#include "sttm_dev.h"
#include "../../include/sttm.h"

namespace sttm {

// ---- the context, for entry points outside sttm_api.hip ------------------------------------------------------
int ctx_fail(sttm_ctx* c, int code, const char* msg);  // sets the message (up to 255 characters), returns code
int ctx_device(sttm_ctx* c);                           // makes the context's device the current one
int ctx_after_launch(sttm_ctx* c);
hipStream_t ctx_stream(const sttm_ctx* c);

// ---- argument checks shared by the operators (sttm_rope.hip) ---------------------------------------------------
int check_cache(sttm_ctx* c, const sttm_cache* cache);
int check_sequences(sttm_ctx* c, const sttm_cache* cache, const sttm_sequences* seqs);
int check_workspace(sttm_ctx* c, const void* ws, size_t have, size_t need);

// The pool of pages as kernels see it. Strides in bytes.
struct Pool {
  char* k;
  char* v;
  long long page_stride, head_stride;
  int token_stride;
  int pages;     // page numbers are below this
  int shift;     // log2 of the page size
  int row;       // bytes of a row
};
Pool make_pool(const sttm_cache* c);

struct Seqs {
  const int32_t* table;
  const int32_t* lengths;
  long long table_stride;
  int max_len;   // at most the slots of a table row
};
Seqs make_seqs(const sttm_cache* c, const sttm_sequences* s);

__device__ inline int seq_length(const Seqs& s, int b) { return min(max(s.lengths[b], 0), s.max_len); }

inline int elem_bytes(int dtype) { return dtype == STTM_F32 ? 4 : 2; }
inline bool aligned16(const void* p) { return (reinterpret_cast<uintptr_t>(p) & 15) == 0; }

// ---- 16-bit numbers ----------------------------------------------------------------------------------------------
template <int DT> __device__ inline uint32_t pack2(float a, float b) { return DT == 1 ? pack2_bf16(a, b) : pack2_f16(a, b); }
template <int DT> __device__ inline float low_half(uint32_t w) {
  return DT == 1 ? __uint_as_float(w << 16) : __half2float(__ushort_as_half((unsigned short)(w & 0xffffu)));
}
template <int DT> __device__ inline float high_half(uint32_t w) {
  return DT == 1 ? __uint_as_float(w & 0xffff0000u) : __half2float(__ushort_as_half((unsigned short)(w >> 16)));
}

// 2^x (v_exp_f32: within an ulp; results below 2^-126 are zero).
__device__ inline float exp2_fast(float x) {
#ifndef STTM_HOST_EMULATION
  return __builtin_amdgcn_exp2f(x);
#else
  return exp2f(x);
#endif
}

// An 8-byte store past the caches (see store_once).
__device__ inline void store_once8(char* p, const uint2& v) {
#ifndef STTM_HOST_EMULATION
  typedef unsigned int u32x2 __attribute__((ext_vector_type(2)));
  const u32x2 x = {v.x, v.y};
  __builtin_nontemporal_store(x, reinterpret_cast<u32x2*>(p));
#else
  *reinterpret_cast<uint2*>(p) = v;
#endif
}

// sin and cos of pi * x, |x| <= 1.
__device__ inline void sincos_half_turns(float x, float* s, float* c) {
#ifndef STTM_HOST_EMULATION
  sincospif(x, s, c);
#else
  *s = (float)sin(3.14159265358979323846 * x);
  *c = (float)cos(3.14159265358979323846 * x);
#endif
}

}  // namespace sttm
