// What the operators on a paged cache use beyond hip_runtime.h of this folder.
#pragma once
#include <hip/hip_runtime.h>

struct float2 { float x, y; };
struct int2 { int x, y; };
inline float2 make_float2(float a, float b) { return {a, b}; }
inline int2 make_int2(int a, int b) { return {a, b}; }
inline unsigned atomicOr(unsigned* p, unsigned v) { return __atomic_fetch_or(p, v, __ATOMIC_SEQ_CST); }
inline unsigned atomicAnd(unsigned* p, unsigned v) { return __atomic_fetch_and(p, v, __ATOMIC_SEQ_CST); }
inline int __clzll(long long v) { return v ? __builtin_clzll((unsigned long long)v) : 64; }
