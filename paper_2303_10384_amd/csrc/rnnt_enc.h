// Shared by the operators of an encoder's layers (include/rnnt_encoder_mi355x.h).
#pragma once

#include "rnnt_encoder_mi355x.h"
#include "rnnt_net.h"

namespace rnnt {

// Rows of a call fit a launch of a few blocks for each (the limit that the header states).
constexpr int64_t kEncRows = (int64_t{1} << 31) / 128;

// elements of a 16-byte access
template <typename T>
constexpr int kVec = sizeof(T) == 4 ? 4 : 8;

// The larger magnitude by its bits: infinity is above every number, and NaN above infinity.
struct MaxBitsOp {
  __device__ static __forceinline__ float apply(float a, float b) {
    const uint32_t x = __float_as_uint(a), y = __float_as_uint(b);
    return __uint_as_float(x > y ? x : y);
  }
};

// ---- rows in 8 bits -----------------------------------------------------------
// q = 127 v / most, correctly rounded before it goes to an integer wherever the quotient is one of
// float32's: a half, which values of 16 bits meet often, is then a half and goes to the even side.  (A product
// with 127 / most, rounded, would put halves on either side.)
struct Quantizer {
  float factor, most, inverse;

  // most: the row's largest magnitude, by its bits
  __device__ __forceinline__ explicit Quantizer(float m) {
    // 127 v stays in float32's range; powers of two change no digit
    const bool large = m > 0x1p100f;
    factor = large ? 127.f * 0x1p-64f : 127.f;
    most = large ? m * 0x1p-64f : m;
    inverse = __builtin_amdgcn_rcpf(most);
    if (!(m >= 0x1p-100f && m < __builtin_inff())) factor = inverse = 0.f;  // zeros, or no number: q = 0
  }
  // the scale of a row whose values are v * unit
  __device__ __forceinline__ static float scale(float m, float unit) {
    if (m < 0x1p-100f) return 0.f;
    const float s = m * unit * (1.f / 127.f);
    return s < __builtin_inff() && m < __builtin_inff() ? s : __builtin_nanf("");
  }
  __device__ __forceinline__ int quantize(float v) const {
    const float p = inverse == 0.f ? 0.f : v * factor, t = p * inverse;
    const float q = __builtin_fmaf(__builtin_fmaf(-t, most, p), inverse, t);
    return static_cast<int>(__builtin_rintf(inverse == 0.f ? 0.f : q));
  }
};

// four integers of -127 .. 127 as bytes, the first one lowest
__device__ __forceinline__ uint32_t pack4_i8(int a, int b, int c, int d) {
  return (a & 0xff) | (b & 0xff) << 8 | (c & 0xff) << 16 | static_cast<uint32_t>(d) << 24;
}

}  // namespace rnnt
