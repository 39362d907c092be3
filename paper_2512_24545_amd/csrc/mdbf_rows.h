// Rows of 16- and 32-bit numbers in pieces of eight, of any stride, for the kernels around the projections.
#pragma once
#include "mdbf_internal.h"

namespace mdbf {

typedef uint32_t U32x2 __attribute__((ext_vector_type(2)));
typedef uint32_t U32x4 __attribute__((ext_vector_type(4)));
typedef float F32x2 __attribute__((ext_vector_type(2)));
typedef float F32x4 __attribute__((ext_vector_type(4)));
typedef _Float16 F16x2 __attribute__((ext_vector_type(2)));
typedef __bf16 Bf16x2 __attribute__((ext_vector_type(2)));
// the same at the alignment of an element: rows of odd strides take the wide instructions too
typedef U32x4 U32x4u __attribute__((aligned(2)));
typedef F32x4 F32x4u __attribute__((aligned(4)));

inline bool row_dtype(int d) { return d == MDBF_F16 || d == MDBF_BF16 || d == MDBF_F32; }
inline bool ptr_aligned(const void* p, size_t n) { return reinterpret_cast<uintptr_t>(p) % n == 0; }

// eight elements as they lie
template <int DT>
struct Raw8 {
  U32x4 w[DT == MDBF_F32 ? 2 : 1];
};

// elements at .. at + 7, of which `count` (1 .. 8) are there; the others are zeros
template <int DT>
__device__ __forceinline__ void load_raw8(const void* base, int64_t at, int count, Raw8<DT>& r) {
  if (DT == MDBF_F32) {
    const MDBF_GLOBAL float* p = (const MDBF_GLOBAL float*)base + at;
    if (count >= 8) {
      r.w[0] = __builtin_bit_cast(U32x4, *(const MDBF_GLOBAL F32x4u*)p);
      r.w[DT == MDBF_F32] = __builtin_bit_cast(U32x4, *(const MDBF_GLOBAL F32x4u*)(p + 4));
    } else {
#pragma unroll
      for (int i = 0; i < 8; ++i) r.w[i / 4 * (DT == MDBF_F32)][i % 4] = i < count ? __builtin_bit_cast(uint32_t, p[i]) : 0u;
    }
  } else {
    const MDBF_GLOBAL uint16_t* p = (const MDBF_GLOBAL uint16_t*)base + at;
    if (count >= 8) {
      r.w[0] = *(const MDBF_GLOBAL U32x4u*)p;
    } else {
#pragma unroll
      for (int i = 0; i < 4; ++i)
        r.w[0][i] = (2 * i < count ? (uint32_t)p[2 * i] : 0u) | (2 * i + 1 < count ? (uint32_t)p[2 * i + 1] << 16 : 0u);
    }
  }
}

template <int DT>
__device__ __forceinline__ void to_float8(const Raw8<DT>& r, float (&x)[8]) {
#pragma unroll
  for (int i = 0; i < 4; ++i) {
    if (DT == MDBF_F32) {
      const uint32_t a = r.w[0][i], b = r.w[DT == MDBF_F32][i];
      x[i] = __builtin_bit_cast(float, a);
      x[4 + i] = __builtin_bit_cast(float, b);
    } else {
      const uint32_t w = r.w[0][i];
      if (DT == MDBF_F16) {
        const F16x2 h = __builtin_bit_cast(F16x2, w);
        x[2 * i] = (float)h[0];
        x[2 * i + 1] = (float)h[1];
      } else {
        x[2 * i] = __builtin_bit_cast(float, w << 16);
        x[2 * i + 1] = __builtin_bit_cast(float, w & 0xffff0000u);
      }
    }
  }
}

// two values rounded to nearest in the 16-bit type
template <int DT>
__device__ __forceinline__ uint32_t round2(float a, float b) {
  const F32x2 v = {a, b};
  if (DT == MDBF_F16) return __builtin_bit_cast(uint32_t, __builtin_convertvector(v, F16x2));
  return __builtin_bit_cast(uint32_t, __builtin_convertvector(v, Bf16x2));
}

// STREAM: past the caches, for results that are more than they hold for a reader (a template's argument: of two stores to one place
// the compiler makes one, without the hint)
template <int DT, bool STREAM>
__device__ __forceinline__ void store_float8(void* base, int64_t at, int count, const float (&x)[8]) {
  if (DT == MDBF_F32) {
    MDBF_GLOBAL float* p = (MDBF_GLOBAL float*)base + at;
    if (count >= 8) {
      const F32x4 a = {x[0], x[1], x[2], x[3]}, b = {x[4], x[5], x[6], x[7]};
      if (STREAM) {
        __builtin_nontemporal_store(a, (MDBF_GLOBAL F32x4u*)p);
        __builtin_nontemporal_store(b, (MDBF_GLOBAL F32x4u*)(p + 4));
      } else {
        *(MDBF_GLOBAL F32x4u*)p = a;
        *(MDBF_GLOBAL F32x4u*)(p + 4) = b;
      }
    } else {
#pragma unroll
      for (int i = 0; i < 8; ++i)
        if (i < count) p[i] = x[i];
    }
  } else {
    MDBF_GLOBAL uint16_t* p = (MDBF_GLOBAL uint16_t*)base + at;
    U32x4 v;
#pragma unroll
    for (int i = 0; i < 4; ++i) v[i] = round2<DT>(x[2 * i], x[2 * i + 1]);
    if (count >= 8) {
      if (STREAM) __builtin_nontemporal_store(v, (MDBF_GLOBAL U32x4u*)p);
      else *(MDBF_GLOBAL U32x4u*)p = v;
    } else {
#pragma unroll
      for (int i = 0; i < 8; ++i)
        if (i < count) p[i] = (uint16_t)(v[i / 2] >> (16 * (i % 2)));
    }
  }
}

}  // namespace mdbf
