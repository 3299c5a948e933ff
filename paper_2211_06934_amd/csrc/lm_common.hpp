// Shared pieces of the language-model operators (distill, qknorm, linattn):
// element types, vectors at any alignment, reductions, argument checks.
#pragma once

#include <hip/hip_runtime.h>

#include <cmath>
#include <cstdint>

#include "common.hpp"

namespace diffopt {

using bf16 = __bf16;
typedef float f32x4 __attribute__((ext_vector_type(4)));
typedef bf16 bf16x4 __attribute__((ext_vector_type(4)));
typedef bf16 bf16x8 __attribute__((ext_vector_type(8)));

// 16 bytes of elements as memory holds them: aligned to the element only (the
// hardware takes 128-bit accesses at any address).
template <class E>
struct Vec {
  static constexpr int N = 16 / (int)sizeof(E);
  typedef E type __attribute__((ext_vector_type(16 / sizeof(E)), aligned(alignof(E))));
};

template <class E>
__device__ __forceinline__ typename Vec<E>::type load_vec(const E* p) {
  return *reinterpret_cast<const typename Vec<E>::type*>(p);
}

template <class E>
__device__ __forceinline__ void load_floats(const E* p, float* x) {
  const typename Vec<E>::type v = load_vec(p);
#pragma unroll
  for (int i = 0; i < Vec<E>::N; ++i) x[i] = (float)v[i];
}

template <class E>
__device__ __forceinline__ void store_vec(E* p, const float* x) {
  typedef float wide __attribute__((ext_vector_type(16 / sizeof(E))));
  typedef E whole __attribute__((ext_vector_type(16 / sizeof(E))));
  wide w;
#pragma unroll
  for (int i = 0; i < Vec<E>::N; ++i) w[i] = x[i];
  *reinterpret_cast<typename Vec<E>::type*>(p) = __builtin_convertvector(w, whole);  // pairs in one instruction
}

constexpr float kInf = __builtin_inff();
constexpr float kNan = __builtin_nanf("");

template <int WIDTH = 64>
__device__ __forceinline__ float wave_sum(float x) {
#pragma unroll
  for (int o = WIDTH / 2; o > 0; o >>= 1) x += __shfl_xor(x, o, 64);
  return x;
}

// fmaxf drops a NaN operand; a NaN logit has to reach the row's results, which
// it does through the sum.
__device__ __forceinline__ float wave_max(float x) {
#pragma unroll
  for (int o = 32; o > 0; o >>= 1) x = fmaxf(x, __shfl_xor(x, o, 64));
  return x;
}

// A [B][T][heads][width] operand: strides in elements.
struct HeadArr {
  void* p;
  int64_t sb, st, sh;
};

inline bool dtype_ok(int32_t dtype) { return dtype == DIFFOPT_F32 || dtype == DIFFOPT_BF16; }
inline int64_t elem_size(int32_t dtype) { return dtype == DIFFOPT_F32 ? 4 : 2; }
inline bool aligned_to(const void* p, int64_t bytes) { return (reinterpret_cast<uintptr_t>(p) & (uintptr_t)(bytes - 1)) == 0; }

inline int check_heads(const char* who, const char* what, const diffopt_heads* h, int32_t dtype, HeadArr* out) {
  if (!h || !h->data) return fail(DIFFOPT_EINVAL, "%s: null %s", who, what);
  if (!aligned_to(h->data, elem_size(dtype))) return fail(DIFFOPT_EINVAL, "%s: %s is not aligned to its elements", who, what);
  *out = HeadArr{h->data, h->stride_b, h->stride_t, h->stride_h};
  return DIFFOPT_OK;
}

// Whether a and b (either may be NULL) share bytes.
inline bool overlap(const void* a, int64_t a_bytes, const void* b, int64_t b_bytes) {
  if (!a || !b) return false;
  const uintptr_t x = reinterpret_cast<uintptr_t>(a), y = reinterpret_cast<uintptr_t>(b);
  return x < y + (uint64_t)b_bytes && y < x + (uint64_t)a_bytes;
}

}  // namespace diffopt
