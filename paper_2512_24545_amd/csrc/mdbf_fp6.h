// Conversions between fp32 and fp6 (e2m3), the format of the limbs that the block-scaled matrix-core products read.
#pragma once
#include "mdbf_internal.h"

namespace mdbf {

// ---------------------------------------------------------------------------------------------------
// fp6 e2m3: 1 sign, 2 exponent (bias 1), 3 mantissa bits: 0, 0.125 .. 0.875, 1 .. 1.875, 2 .. 3.75, 4 .. 7.5.
// v_cvt_scalef32_2xpk16_fp6_f32 converts 32 floats at once: divides by the power of two in the exponent
// field of `scale`, rounds to nearest even, saturates at +-7.5; element 2i of the result comes from the
// first source's element i, element 2i+1 from the second's; element j sits at bits [6j, 6j+6) -- the order
// the matrix-core instruction reads.  v_cvt_scalef32_pk32_f32_fp6 is the inverse (times the scale).
// ---------------------------------------------------------------------------------------------------
typedef float v16f __attribute__((ext_vector_type(16)));
typedef float v32f __attribute__((ext_vector_type(32)));
typedef unsigned v6u __attribute__((ext_vector_type(6)));

__device__ __forceinline__ v6u fp6_encode32(const float (&v)[32], float scale) {
  v16f even, odd;
#pragma unroll
  for (int i = 0; i < 16; ++i) {
    even[i] = v[2 * i];
    odd[i] = v[2 * i + 1];
  }
  // The result must not share registers with the sources: with a destination inside the second source's
  // range the instruction gave wrong limbs (seen in a build whose register allocation produced that
  // overlap; the compiler's builtin does not exclude it).  Hence the instruction is written out with an
  // early-clobber result; the idle cycle after it covers the wait a conversion's result may need before
  // an ordinary vector instruction reads it, which the compiler cannot add around opaque text.
  v6u out;
  asm("v_cvt_scalef32_2xpk16_fp6_f32 %0, %1, %2, %3\n\ts_nop 1" : "=&v"(out) : "v"(even), "v"(odd), "v"(scale));
  return out;
}

// the inverse (32 floats from one limb), with the same precaution
__device__ __forceinline__ v32f fp6_decode32(v6u limb, float scale) {
  v32f out;
  asm("v_cvt_scalef32_pk32_f32_fp6 %0, %1, %2\n\ts_nop 1" : "=&v"(out) : "v"(limb), "v"(scale));
  return out;
}

}  // namespace mdbf
