// Element types of the sequence operators: fp32 beside the two 16-bit formats of common.hpp.  Arithmetic is fp32; a value
// is rounded (to nearest even) where it is stored.
#pragma once
#include "../../include/rampde.h"
#include "common.hpp"

namespace rampde {

struct F32 {};

template <class T>
struct Elem {  // F16, BF16
  typedef uint16_t S;
  __device__ static inline float up(S s) { return Low<T>::to_f32(s); }
  __device__ static inline S down(float v) { return (S)Low<T>::pack2(v, v); }
};
template <>
struct Elem<F32> {
  typedef float S;
  __device__ static inline float up(S s) { return s; }
  __device__ static inline S down(float v) { return v; }
};

// f with the tag of a type that the caller has checked
template <class F>
int by_type(rampde_dtype t, F&& f) {
  if (t == RAMPDE_F32) return f(F32{});
  if (t == RAMPDE_F16) return f(F16{});
  return f(BF16{});
}

// 8 neighbouring elements as they lie in memory
template <class T>
struct Raw8 {
  u16x8 v;
};
template <>
struct Raw8<F32> {
  f32x4 v[2];
};

// The first n of 8 neighbouring elements (the others read as zero): whole ones in words of 16 bytes, on whatever element they start
// (global accesses need no alignment; one that crosses a cache line takes both).
template <class T>
__device__ inline Raw8<T> load8(const typename Elem<T>::S* p, int n) {
  Raw8<T> r;
  if (n >= 8) {
    __builtin_memcpy(&r, p, sizeof r);
  } else {
    typename Elem<T>::S e[8];
#pragma unroll
    for (int i = 0; i < 8; ++i) e[i] = i < n ? p[i] : (typename Elem<T>::S)0;
    r = __builtin_bit_cast(Raw8<T>, e);
  }
  return r;
}
template <class T>
__device__ inline void unpack8(const Raw8<T>& r, float (&f)[8]) {
  if constexpr (sizeof(typename Elem<T>::S) == 4) {
#pragma unroll
    for (int i = 0; i < 8; ++i) f[i] = r.v[i >> 2][i & 3];
  } else {
#pragma unroll
    for (int i = 0; i < 8; ++i) f[i] = Elem<T>::up(r.v[i]);
  }
}
template <class T>
__device__ inline void store8(typename Elem<T>::S* p, int n, const float (&f)[8]) {
  Raw8<T> r;
  if constexpr (sizeof(typename Elem<T>::S) == 4) {
#pragma unroll
    for (int i = 0; i < 8; ++i) r.v[i >> 2][i & 3] = f[i];
  } else {
    uint32_t w[4];
#pragma unroll
    for (int i = 0; i < 4; ++i) w[i] = Low<T>::pack2(f[2 * i], f[2 * i + 1]);
    r = __builtin_bit_cast(Raw8<T>, w);
  }
  if (n >= 8) {
    __builtin_memcpy(p, &r, sizeof r);
  } else {
    struct { typename Elem<T>::S e[8]; } a = __builtin_bit_cast(decltype(a), r);
#pragma unroll
    for (int i = 0; i < 8; ++i)
      if (i < n) p[i] = a.e[i];
  }
}

// e = exp(-z) and s = 1 / (1 + e) on the hardware exp2 and reciprocal; s is 0 where e overflows.  1 - s is e s, to as many places: by
// subtraction, that of an open gate has lost 12 of 24 at z = 8 and all of them at 17.
//
// Relative error about 2e-7, and that of the exponent's rounding, |z| 5e-8 (1e-6 at 20, 4e-6 at 80).  The latter is as if z were off by
// half a unit in its last place, if z is fp32, and far less than that for z in 16 bits, which take it; fp32 operands, whose results are
// held to 24 places, get what the product has dropped as a factor behind the exponential: six instructions of some 40 an element (4 x
// 4096 x 2048 in fp32 87.2 instead of 86.3 us forward, join of 65536 x 64 17.3 instead of 16.4).
struct Gate {
  float e, s;
};
template <class T>
__device__ inline Gate gate_of(float z) {
  const float L = -1.44269504f, t = z * L;
  float e = __builtin_amdgcn_exp2f(t);
  if constexpr (sizeof(typename Elem<T>::S) == 4) {
    const float dropped = fmaf(z, -1.92596299e-8f, fmaf(z, L, -t)), f = fmaf(e, dropped * 0.693147181f, e);  // (log2(e) in two parts)
    e = fabsf(z) < 88.f ? f : e;  // (beyond, e or z may be infinite)
  }
  return {e, __builtin_amdgcn_rcpf(1.f + e)};
}
template <class T>
__device__ inline float logistic(float z) {
  return gate_of<T>(z).s;
}

}  // namespace rampde
