// Rotary positions: the turn of a pair of dims, and the pairs of either layout.
//
//   (a, b) -> scale * (a cos t - b sin t, b cos t + a sin t),  t = position * inv_freq[i]
//
// The angle is formed in 64 bits, in turns: a position of 2^31 and a frequency of 1 leave
// 2^-22 of a turn's fraction, where 32 bits would leave nothing of it.  Its fraction goes on
// in fp32 (2^-25 of a turn).
#pragma once

#include <hip/hip_runtime.h>
#include <stdint.h>

#include "echo.h"

namespace echo {
namespace {

// scale * (cos, sin) of the angle.
__device__ __forceinline__ float2 rope_turn(int position, double inv_freq, float scale) {
  double turns = double(position) * (inv_freq * 0.15915494309189535);  // 1 / (2 pi)
  turns -= __builtin_rint(turns);
  float s, c;
  sincospif(2.0f * float(turns), &s, &c);
  return make_float2(c * scale, s * scale);
}

__device__ __forceinline__ float2 rope_pair(float a, float b, float2 cs) {
  return make_float2(__builtin_fmaf(a, cs.x, -(b * cs.y)), __builtin_fmaf(b, cs.x, a * cs.y));
}

__device__ __forceinline__ float bf16_lo(uint32_t w) { return __uint_as_float(w << 16); }
__device__ __forceinline__ float bf16_hi(uint32_t w) { return __uint_as_float(w & 0xFFFF0000u); }

typedef float rope_floatx2 __attribute__((ext_vector_type(2)));
typedef __bf16 rope_bf16x2 __attribute__((ext_vector_type(2)));
// Two floats rounded to bfloat16 (to nearest even).
__device__ __forceinline__ uint32_t rope_pack(float lo, float hi) {
  return __builtin_bit_cast(uint32_t, __builtin_convertvector(rope_floatx2{lo, hi}, rope_bf16x2));
}

// The rows of a call: num_rows, or *row_count of them; -1 if there cannot be so many.
__device__ __forceinline__ int rope_rows(const int32_t* row_count, int num_rows) {
  if (row_count == nullptr) return num_rows;
  const int n = row_count[0];
  return n < 0 || n > num_rows ? -1 : n;
}

}  // namespace
}  // namespace echo
