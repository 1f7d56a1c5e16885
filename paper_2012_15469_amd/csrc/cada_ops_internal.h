// What the operators' translation units share (declared and documented in cada_ops.h): element types, unaligned vectors, argument checks.
#pragma once

#include "cada_internal.h"
#include "cada_ops_sizes.h"

namespace cada {

struct bf16 { uint16_t bits; };      // storage type
template <typename T> struct Elem;
template <> struct Elem<bf16> { static constexpr int kPer16 = 8; };
template <> struct Elem<float> { static constexpr int kPer16 = 4; };

__device__ __forceinline__ float to_f32(bf16 x) { return bf2f(x.bits); }
__device__ __forceinline__ float to_f32(float x) { return x; }
template <typename T> __device__ __forceinline__ T from_f32(float x);
template <> __device__ __forceinline__ bf16 from_f32<bf16>(float x) { return bf16{f2bf(x)}; }
template <> __device__ __forceinline__ float from_f32<float>(float x) { return x; }

// 16 bytes at an address that is a multiple of the element's size only (one access: the target runs in its unaligned mode).
typedef uint32_t u32x4a2 __attribute__((ext_vector_type(4), aligned(2)));
typedef uint32_t u32x4a4 __attribute__((ext_vector_type(4), aligned(4)));
typedef uint32_t u32x4v __attribute__((ext_vector_type(4)));
template <typename T> struct Vec16;
template <> struct Vec16<bf16> { typedef u32x4a2 type; };
template <> struct Vec16<float> { typedef u32x4a4 type; };
template <typename T> __device__ __forceinline__ u32x4v load16(const T *p) { return *reinterpret_cast<const typename Vec16<T>::type *>(p); }
template <typename T> __device__ __forceinline__ void store16(T *p, u32x4v x) { *reinterpret_cast<typename Vec16<T>::type *>(p) = x; }

// The first `n` elements at p (n may be anything; none if n <= 0), the others zero.
template <typename T> __device__ __forceinline__ u32x4v load16_n(const T *p, int64_t n) {
  constexpr int E = Elem<T>::kPer16;
  if (n >= E) return load16(p);
  u32x4v x = {0, 0, 0, 0};
  if constexpr (E == 8) {
#pragma unroll
    for (int i = 0; i < 8; ++i) if (i < n) x[i >> 1] |= (uint32_t)p[i].bits << (16 * (i & 1));
  } else {
#pragma unroll
    for (int i = 0; i < 4; ++i) if (i < n) x[i] = __float_as_uint(p[i]);
  }
  return x;
}

// A piece of 16 bytes as float32 values, and back.
template <typename T> __device__ __forceinline__ void unpack(u32x4v x, float (&f)[Elem<T>::kPer16]) {
#pragma unroll
  for (int i = 0; i < 4; ++i) {
    if constexpr (Elem<T>::kPer16 == 8) { f[2 * i] = __uint_as_float(x[i] << 16); f[2 * i + 1] = __uint_as_float(x[i] & 0xFFFF0000u); }
    else f[i] = __uint_as_float(x[i]);
  }
}
template <typename T> __device__ __forceinline__ u32x4v pack(const float (&f)[Elem<T>::kPer16]) {
  if constexpr (Elem<T>::kPer16 == 8) return u32x4v{f2bf_pk(f[0], f[1]), f2bf_pk(f[2], f[3]), f2bf_pk(f[4], f[5]), f2bf_pk(f[6], f[7])};
  else return u32x4v{__float_as_uint(f[0]), __float_as_uint(f[1]), __float_as_uint(f[2]), __float_as_uint(f[3])};
}

// Eight consecutive values as float32, from and to memory; only the first n exist.
template <typename T> __device__ __forceinline__ void load8_n(const T *p, int64_t n, float (&f)[8]) {
  if constexpr (Elem<T>::kPer16 == 8) {
    const u32x4v x = load16_n(p, n);
#pragma unroll
    for (int i = 0; i < 4; ++i) { f[2 * i] = __uint_as_float(x[i] << 16); f[2 * i + 1] = __uint_as_float(x[i] & 0xFFFF0000u); }
  } else {
    const u32x4v x = load16_n(p, n), y = load16_n(p + 4, n - 4);
#pragma unroll
    for (int i = 0; i < 4; ++i) { f[i] = __uint_as_float(x[i]); f[4 + i] = __uint_as_float(y[i]); }
  }
}
template <typename T> __device__ __forceinline__ void store8_n(T *p, int64_t n, const float (&f)[8]) {
  if (n >= 8) {
    if constexpr (Elem<T>::kPer16 == 8) {
      store16(p, u32x4v{f2bf_pk(f[0], f[1]), f2bf_pk(f[2], f[3]), f2bf_pk(f[4], f[5]), f2bf_pk(f[6], f[7])});
    } else {
      store16(p, u32x4v{__float_as_uint(f[0]), __float_as_uint(f[1]), __float_as_uint(f[2]), __float_as_uint(f[3])});
      store16(p + 4, u32x4v{__float_as_uint(f[4]), __float_as_uint(f[5]), __float_as_uint(f[6]), __float_as_uint(f[7])});
    }
    return;
  }
#pragma unroll
  for (int i = 0; i < 8; ++i) if (i < n) p[i] = from_f32<T>(f[i]);
}

// Activations and their derivatives, in float32: with the library's functions for float32 tables, for bf16 ones with the hardware's exp2 and reciprocal (an
// ulp or two) and, for the normal distribution, formula 7.1.26 of Abramowitz and Stegun's handbook (|error of erf| <= 1.5e-7, far below bf16's 2^-9; erff is a
// third of the time of a 4096 x 4096 layer's epilogue).  Phi(-|z|) is formed without the 1 that would cancel.
__device__ __forceinline__ float fast_exp(float x) { return __builtin_amdgcn_exp2f(x * 1.4426950408889634f); }
// Phi(z), and e = exp(-z^2 / 2)
__device__ __forceinline__ float fast_phi(float z, float &e) {
  const float x = fabsf(z) * 0.70710678118654752f, t = __builtin_amdgcn_rcpf(fmaf(0.3275911f, x, 1.f));
  e = fast_exp(-x * x);
  const float tail = t * fmaf(t, fmaf(t, fmaf(t, fmaf(t, 1.061405429f * 0.5f, -1.453152027f * 0.5f), 1.421413741f * 0.5f), -0.284496736f * 0.5f), 0.254829592f * 0.5f) * e;
  return z < 0.f ? tail : 1.f - tail;
}
template <typename T> __device__ __forceinline__ float activation(float z, int act) {
  constexpr bool FAST = sizeof(T) == 2;
  float e;
  switch (act) {
    case CADA_ACT_RELU: return z < 0.f ? 0.f : z;          // (NaN stays NaN)
    case CADA_ACT_GELU: return z * (FAST ? fast_phi(z, e) : 0.5f * (1.f + erff(z * 0.70710678118654752f)));
    case CADA_ACT_SILU: return FAST ? z * __builtin_amdgcn_rcpf(1.f + fast_exp(-z)) : z / (1.f + expf(-z));
    default: return z;
  }
}
template <typename T> __device__ __forceinline__ float activation_slope(float z, int act) {
  constexpr bool FAST = sizeof(T) == 2;
  switch (act) {
    case CADA_ACT_RELU: return z > 0.f ? 1.f : 0.f;
    case CADA_ACT_GELU: {
      float e, phi;
      if constexpr (FAST) phi = fast_phi(z, e);
      else { phi = 0.5f * (1.f + erff(z * 0.70710678118654752f)); e = expf(-0.5f * z * z); }
      return fmaf(z * 0.39894228040143268f, e, phi);
    }
    case CADA_ACT_SILU: {
      const float s = FAST ? __builtin_amdgcn_rcpf(1.f + fast_exp(-z)) : 1.f / (1.f + expf(-z));
      return s * fmaf(z, 1.f - s, 1.f);
    }
    default: return 1.f;
  }
}

// ---- host ----
// Whether an output shares no memory with another table, which an error names otherwise.  Columns side by side of one wider table (one row length, or a single row among them) are apart.
struct Span { const char *name; const void *at; int64_t rows, ld, cols; };      // (in bytes)
inline Span span(const char *name, const void *at, int64_t rows, int64_t ld, int64_t cols, size_t elem) { return Span{name, at, rows, ld * (int64_t)elem, cols * (int64_t)elem}; }
inline Span span(const char *name, const void *at, size_t bytes) { return Span{name, bytes > 0 ? at : nullptr, 1, (int64_t)bytes, (int64_t)bytes}; }
bool ops_apart(const Span &out, const Span &other);      // cada_linear.hip
// The same of any number of ranges of memory: no written one shares memory with another.  `index`: which tensor of a list, or -1.
struct Range { const char *name; int index; const void *at; size_t bytes; bool written; };
bool ops_apart(Range *ranges, size_t n);      // cada_linear.hip (puts them in order; none may throw)
int ops_check_workspace(const void *ws, size_t given, size_t need);      // cada_linear.hip
int ops_launched(const char *what);

}  // namespace cada
