// The 8-bit paged KV cache: its layout, its scales and its number formats.
//
// Pages are [num_pages][Hkv][page_size][128] bytes, scales
// [num_pages][Hkv][page_size / 32] floats: a block is 32 consecutive tokens of one
// head, 4 KB in one piece, and stands for byte value x scale.  The writers take
// powers of two for scales.  The values are floating, so that a scale that is up to
// twice too large costs none of their bits (only the range's lower end moves), and
// bytes that are scaled again, where a part-filled block's scale grows, keep their
// value exactly unless they become subnormal.  A block is the attention's tile, so
// that a tile has one scale.
#pragma once

#include "echo_device.h"
#include "echo_internal.h"

namespace echo {
namespace {

constexpr int kBlockTokens = ECHO_KV_BLOCK;                     // 32
constexpr int kBlockBytes = ECHO_KV_BLOCK * ECHO_HEAD_DIM;      // 4 KB
constexpr int kScaleExpMin = -60, kScaleExpMax = 60;            // the writers' scales

typedef float floatx2v __attribute__((ext_vector_type(2)));

template <int kFmt>
struct Fmt8;
template <>
struct Fmt8<ECHO_KV_E4M3> {
  static constexpr float kMax = 448.0f;  // 1.75 * 2^8
  static constexpr int kMaxExp = 8;
};
template <>
struct Fmt8<ECHO_KV_E5M2> {
  static constexpr float kMax = 57344.0f;  // 1.75 * 2^15
  static constexpr int kMaxExp = 15;
};

// Four values to four bytes, rounded to nearest even; beyond the largest value (an
// infinity) that value, NaN stays NaN.
template <int kFmt>
__device__ __forceinline__ uint32_t encode4(float a, float b, float c, float d) {
  const auto sat = [](float x) {  // (a comparison with NaN is false: NaN passes)
    x = x > Fmt8<kFmt>::kMax ? Fmt8<kFmt>::kMax : x;
    return x < -Fmt8<kFmt>::kMax ? -Fmt8<kFmt>::kMax : x;
  };
  int w = 0;
  if (kFmt == ECHO_KV_E4M3) {
    w = __builtin_amdgcn_cvt_pk_fp8_f32(sat(a), sat(b), w, false);
    w = __builtin_amdgcn_cvt_pk_fp8_f32(sat(c), sat(d), w, true);
  } else {
    w = __builtin_amdgcn_cvt_pk_bf8_f32(sat(a), sat(b), w, false);
    w = __builtin_amdgcn_cvt_pk_bf8_f32(sat(c), sat(d), w, true);
  }
  return uint32_t(w);
}

// The four values of a word's bytes, times ratio, as bytes again.
template <int kFmt>
__device__ __forceinline__ uint32_t rescale4(uint32_t w, float ratio) {
  floatx2v lo, hi;
  if (kFmt == ECHO_KV_E4M3) {
    lo = __builtin_amdgcn_cvt_pk_f32_fp8(int(w), false);
    hi = __builtin_amdgcn_cvt_pk_f32_fp8(int(w), true);
  } else {
    lo = __builtin_amdgcn_cvt_pk_f32_bf8(int(w), false);
    hi = __builtin_amdgcn_cvt_pk_f32_bf8(int(w), true);
  }
  return encode4<kFmt>(lo[0] * ratio, lo[1] * ratio, hi[0] * ratio, hi[1] * ratio);
}

// The smallest scale 2^e, of those with kScaleExpMin <= e <= kScaleExpMax, that brings a
// largest magnitude, given as bfloat16 bits, into the format's range.
template <int kFmt>
__device__ __forceinline__ float block_scale(uint32_t amax_bits) {
  int e = int(amax_bits >> 7) - 127 - Fmt8<kFmt>::kMaxExp + ((amax_bits & 0x7Fu) > 0x60u ? 1 : 0);
  e = min(max(e, kScaleExpMin), kScaleExpMax);
  return __uint_as_float(uint32_t(e + 127) << 23);
}

// Two magnitudes in the bfloat16 pair of a word, those that are not finite as 0.
__device__ __forceinline__ uint32_t finite_mag2(uint32_t w) {
  const uint32_t lo = w & 0x7FFFu, hi = (w >> 16) & 0x7FFFu;
  return max(lo < 0x7F80u ? lo : 0u, hi < 0x7F80u ? hi : 0u);
}

// 16 bytes that are read once, past the caches' reuse order (prompts of three batches in
// turn, 252 MB each: 57.7 -> 54.8 us).
__device__ __forceinline__ uint4 load_once(const uint4* p) {
  typedef uint32_t uint4w __attribute__((ext_vector_type(4)));
  const uint4w w = __builtin_nontemporal_load(reinterpret_cast<const uint4w*>(p));
  return make_uint4(w[0], w[1], w[2], w[3]);
}

// One wave appends n rows (1..32) of a head to a block whose first o rows hold tokens
// (o + n <= 32): the block's scale is the larger of the one it has (if o > 0) and the
// one that the new rows need; where it grows, the o rows are scaled again.  Rows
// behind the new ones are left as they are.  src(i): row i's 128 bfloat16 values.
template <int kFmt, typename Src>
__device__ __forceinline__ void append_block(const Src& src, int n, int o, uint8_t* block,
                                             float* scale) {
  const int lane = threadIdx.x & (kWave - 1);
  const int row = lane >> 4, col = lane & 15;  // row of four, 16-byte chunk of eight values
  uint4 x[8];
#pragma unroll
  for (int j = 0; j < 8; ++j) {
    x[j] = make_uint4(0, 0, 0, 0);
    if (4 * j < n) {  // uniform
      if (4 * j + row < n) x[j] = load_once(reinterpret_cast<const uint4*>(src(4 * j + row)) + col);
    }
  }
  // the block's old bytes, should they need another scale, in the same round trip
  uint4 old[4];
  const float was = o > 0 ? *scale : 0.0f;
#pragma unroll
  for (int j = 0; j < 4; ++j)
    if (8 * j < o) old[j] = reinterpret_cast<const uint4*>(block)[64 * j + lane];
  uint32_t m = 0u;
#pragma unroll
  for (int j = 0; j < 8; ++j)
    if (4 * j < n)
      m = max(m, max(max(finite_mag2(x[j].x), finite_mag2(x[j].y)),
                     max(finite_mag2(x[j].z), finite_mag2(x[j].w))));
  const float need = block_scale<kFmt>(wave_max(m));
  const float now = o > 0 && was > need ? was : need;
  if (o > 0 && was != now) {
    const float ratio = was / now;
#pragma unroll
    for (int j = 0; j < 4; ++j)
      if (8 * j < o && 8 * j + (lane >> 3) < o)
        reinterpret_cast<uint4*>(block)[64 * j + lane] =
            make_uint4(rescale4<kFmt>(old[j].x, ratio), rescale4<kFmt>(old[j].y, ratio),
                       rescale4<kFmt>(old[j].z, ratio), rescale4<kFmt>(old[j].w, ratio));
  }
  const bool pow2 = (__float_as_uint(now) & 0x7FFFFFu) == 0u;  // the product is the quotient
  const float inv = 1.0f / now;
  const auto value = [&](uint32_t w, int half) {
    const float v = __uint_as_float(half ? (w & 0xFFFF0000u) : (w << 16));
    return pow2 ? v * inv : v / now;
  };
#pragma unroll
  for (int j = 0; j < 8; ++j)
    if (4 * j < n && 4 * j + row < n) {
      const uint2 b = make_uint2(
          encode4<kFmt>(value(x[j].x, 0), value(x[j].x, 1), value(x[j].y, 0), value(x[j].y, 1)),
          encode4<kFmt>(value(x[j].z, 0), value(x[j].z, 1), value(x[j].w, 0), value(x[j].w, 1)));
      reinterpret_cast<uint2*>(block + (o + 4 * j + row) * ECHO_HEAD_DIM)[col] = b;
    }
  if (lane == 0 && !(o > 0 && was == now)) *scale = now;
}

// Where the 8-bit cache is (see the layout above).
struct CacheQ8 {
  uint8_t* k_pages;
  uint8_t* v_pages;
  float* k_scale;
  float* v_scale;
  long long num_pages;
  int page_size, page_shift, hkv;
};

// Index of the block (and of its scale) that holds token `off` of a page for a head.
__device__ __forceinline__ size_t block_index(const CacheQ8& c, long long page, int head, int off) {
  return (size_t(page) * c.hkv + head) * size_t(c.page_size / kBlockTokens) +
         size_t(off / kBlockTokens);
}

}  // namespace
}  // namespace echo
