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

// What the lanes of a wave stored into LDS before this is there for its other lanes behind it, and what they read before it
// is read.  A wave's accesses to LDS keep their order, so it takes no instruction: it is the compiler that must not move any
// of them across, which nothing else forbids where the addresses of two lanes differ.
__device__ __forceinline__ void wave_exchange() {
  __builtin_amdgcn_fence(__ATOMIC_RELEASE, "wavefront", "local");
  __builtin_amdgcn_wave_barrier();
  __builtin_amdgcn_fence(__ATOMIC_ACQUIRE, "wavefront", "local");
}

// ---- rows in 8 bits -----------------------------------------------------------
// q = 127 v / most, correctly rounded before it goes to an integer wherever the quotient is one of
// float32's: a half, which values of 16 bits meet often, is then a half and goes to the even side.  (A product
// with 127 / most, rounded, would put halves on either side.)
struct Quantizer {
  float factor, most, inverse;
  uint32_t keep;  // no bits for a row of zeros, or one that holds no number

  // m: the row's largest magnitude, by its bits
  __device__ __forceinline__ explicit Quantizer(float m) {
    // 127 v stays in float32's range; powers of two change no digit
    const bool large = m > 0x1p100f;
    factor = large ? 127.f * 0x1p-64f : 127.f;
    most = large ? m * 0x1p-64f : m;
    inverse = __builtin_amdgcn_rcpf(most);
    keep = m >= 0x1p-100f && m < __builtin_inff() ? 0xffffffffu : 0u;
  }
  // the scale of a row whose values are v * unit
  __device__ __forceinline__ static float scale(float m, float unit) {
    if (m < 0x1p-100f && unit < __builtin_inff()) return 0.f;  // a norm of zeros without eps is 0 / 0
    const float s = m * unit * (1.f / 127.f);
    return s < __builtin_inff() && m < __builtin_inff() ? s : __builtin_nanf("");
  }
  // the integer of v, in the low byte
  __device__ __forceinline__ uint32_t one(float v) const {
    const float p = v * factor, t = p * inverse;
    const float q = __builtin_fmaf(__builtin_fmaf(-t, most, p), inverse, t);
    return __float_as_uint(q + 12582912.f);  // 1.5 * 2^23: the sum's last digit is 1
  }
  // four as bytes, the first one lowest
  __device__ __forceinline__ uint32_t four(const float* v) const {
    const uint32_t low = __builtin_amdgcn_perm(one(v[1]), one(v[0]), 0x0c0c0400u);
    const uint32_t high = __builtin_amdgcn_perm(one(v[3]), one(v[2]), 0x0c0c0400u);
    return __builtin_amdgcn_perm(high, low, 0x05040100u) & keep;
  }
};

// The largest magnitude of 16-bit elements, two at a time on their bits.
typedef unsigned short u16x2 __attribute__((ext_vector_type(2)));
__device__ __forceinline__ void raise_most16(uint32_t& most, uint32_t two) {
  most = __builtin_bit_cast(uint32_t, __builtin_elementwise_max(__builtin_bit_cast(u16x2, most), __builtin_bit_cast(u16x2, two & 0x7fff7fffu)));
}
template <typename T>
__device__ __forceinline__ float most16(uint32_t most) {
  return ElemTraits<T>::from_bits((most & 0xffffu) > most >> 16 ? most & 0xffffu : most >> 16);
}

}  // namespace rnnt
