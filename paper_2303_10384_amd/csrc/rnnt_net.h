// Shared by the operators between an encoder and the loss (include/rnnt_network_mi355x.h):
// element access of any width, the gate and activation functions, the random numbers of
// dropout, and the host's checks and workspaces.
#pragma once

#include <hip/hip_runtime.h>

#include <cstdint>

#include "rnnt_device.h"
#include "rnnt_network_mi355x.h"
#include "rnnt_workspace.h"

namespace rnnt {

// ---- VEC consecutive elements as floats -------------------------------------
// One access of 2, 4, 8 or 16 bytes (32 bytes are two of 16) at the alignment of an element: the
// hardware takes vector accesses to global memory at any address, so a row of odd length needs no
// narrow form, only its last elements do.

template <int BYTES, int ALIGN>
struct __attribute__((packed, aligned(ALIGN))) Words {
  uint32_t w[BYTES / 4];
};

template <int ALIGN>
struct LooseVector;
template <>
struct LooseVector<2> {
  typedef u32x4 type __attribute__((aligned(2)));
};
template <>
struct LooseVector<4> {
  typedef u32x4 type __attribute__((aligned(4)));
};

template <typename T, int VEC>
struct Pack {
  static constexpr int kBytes = VEC * static_cast<int>(sizeof(T));
  static constexpr int kWords = (kBytes + 3) / 4;
  using Memory = Words<kWords * 4, static_cast<int>(sizeof(T))>;
  uint32_t w[kWords];

  __device__ __forceinline__ void load(const T* p) {
    if constexpr (kBytes == 2) {
      w[0] = *reinterpret_cast<const uint16_t*>(p);
    } else {
      const Memory m = *reinterpret_cast<const Memory*>(p);
#pragma unroll
      for (int i = 0; i < kWords; ++i) w[i] = m.w[i];
    }
  }
  // a load of what is read once: it does not push lines out that are still to be written or read
  __device__ __forceinline__ void load_once(const T* p) {
    if constexpr (kBytes % 16 != 0) return load(p);
    using loose = LooseVector<sizeof(T)>;
#pragma unroll
    for (int i = 0; i < kBytes / 16; ++i) {
      const u32x4 v = __builtin_nontemporal_load(reinterpret_cast<const typename loose::type*>(p) + i);
      w[4 * i] = v.x;
      w[4 * i + 1] = v.y;
      w[4 * i + 2] = v.z;
      w[4 * i + 3] = v.w;
    }
  }
  __device__ __forceinline__ void store(T* p) const {
    if constexpr (kBytes == 2) {
      *reinterpret_cast<uint16_t*>(p) = static_cast<uint16_t>(w[0]);
    } else {
      Memory m;
#pragma unroll
      for (int i = 0; i < kWords; ++i) m.w[i] = w[i];
      *reinterpret_cast<Memory*>(p) = m;
    }
  }
  // a store that leaves the caches to others, for results that no cache holds until they are read
  __device__ __forceinline__ void store_away(T* p) const {
    if constexpr (kBytes % 16 != 0) return store(p);
    using loose = LooseVector<sizeof(T)>;
#pragma unroll
    for (int i = 0; i < kBytes / 16; ++i) {
      const u32x4 v = {w[4 * i], w[4 * i + 1], w[4 * i + 2], w[4 * i + 3]};
      __builtin_nontemporal_store(v, reinterpret_cast<typename loose::type*>(p) + i);
    }
  }
  // the first n (0 .. VEC) elements alone, the others 0 / not written
  __device__ __forceinline__ void load_part(const T* p, int n) {
    zero();
#pragma unroll
    for (int i = 0; i < VEC; ++i) {
      if (i < n) {
        if constexpr (sizeof(T) == 4) w[i] = *reinterpret_cast<const uint32_t*>(p + i);
        else w[i / 2] |= static_cast<uint32_t>(*reinterpret_cast<const uint16_t*>(p + i)) << (16 * (i & 1));
      }
    }
  }
  __device__ __forceinline__ void store_part(T* p, int n) const {
#pragma unroll
    for (int i = 0; i < VEC; ++i) {
      if (i < n) {
        if constexpr (sizeof(T) == 4) *reinterpret_cast<uint32_t*>(p + i) = w[i];
        else *reinterpret_cast<uint16_t*>(p + i) = static_cast<uint16_t>(w[i / 2] >> (16 * (i & 1)));
      }
    }
  }
  __device__ __forceinline__ void zero() {
#pragma unroll
    for (int i = 0; i < kWords; ++i) w[i] = 0;
  }
  __device__ __forceinline__ void get(float* f) const {
    if constexpr (kBytes == 2) f[0] = ElemTraits<T>::from_bits(w[0]);
    else ElemTraits<T>::template unpack_words<kWords>(w, f);
  }
  __device__ __forceinline__ void set(const float* f) {
    if constexpr (sizeof(T) == 4) {
#pragma unroll
      for (int i = 0; i < VEC; ++i) w[i] = __float_as_uint(f[i]);
    } else if constexpr (kBytes == 2) {
      T t;
      ElemTraits<T>::store1(&t, f[0]);
      w[0] = t.bits;
    } else {
#pragma unroll
      for (int i = 0; i < VEC / 2; ++i) w[i] = pack2(f[2 * i], f[2 * i + 1]);
    }
  }
  __device__ static __forceinline__ uint32_t pack2(float a, float b) {
    if constexpr (__is_same(T, f16_t)) return pack2_f16(a, b);
    else return pack2_bf16(a, b);
  }
};

// Eight elements a lane as two accesses of 16 bytes would meet every other 16 bytes of memory.  For float32 the
// lanes of a pair exchange halves instead, so that an access covers 32 bytes of a pair and 1 KB of a wave (dropout
// of 512 MB: 5.2 TB/s without, 5.8 with; the joint's stores gained nothing).  Both lanes of the pair hold whole neighbouring groups, p the lane's own.
__device__ __forceinline__ uint32_t swap_pair(uint32_t x) {
  return static_cast<uint32_t>(__builtin_amdgcn_mov_dpp(static_cast<int>(x), dpp::kQuadSwap1, 0xf, 0xf, false));
}
__device__ __forceinline__ void exchange_halves(uint32_t* w) {  // even lanes: own low, partner's low; odd: own high, partner's
  const bool odd = threadIdx.x & 1;
#pragma unroll
  for (int i = 0; i < 4; ++i) {
    const uint32_t got = swap_pair(odd ? w[i] : w[4 + i]);
    w[4 + i] = odd ? w[4 + i] : got;
    w[i] = odd ? got : w[i];
  }
}
template <typename T>
__device__ __forceinline__ void load_pair(Pack<T, 8>& k, const T* p) {
  if constexpr (sizeof(T) == 4) {
    const T* q = p - ((threadIdx.x & 1) ? 4 : 0);
    Pack<T, 4> a, b;
    a.load(q);
    b.load(q + 8);
#pragma unroll
    for (int i = 0; i < 4; ++i) {
      k.w[i] = a.w[i];
      k.w[4 + i] = b.w[i];
    }
    exchange_halves(k.w);
  } else {
    k.load(p);
  }
}
template <typename T>
__device__ __forceinline__ void store_pair(Pack<T, 8> k, T* p) {
  if constexpr (sizeof(T) == 4) {
    exchange_halves(k.w);
    T* q = p - ((threadIdx.x & 1) ? 4 : 0);
    Pack<T, 4> a, b;
#pragma unroll
    for (int i = 0; i < 4; ++i) {
      a.w[i] = k.w[i];
      b.w[i] = k.w[4 + i];
    }
    a.store(q);
    b.store(q + 8);
  } else {
    k.store(p);
  }
}

// ---- functions of one float ---------------------------------------------------

// e^-y for y >= 0 within 2 ulp: the product with log2 e in two parts, so that a large y does
// not cost its digits (|y| log2 e rounded alone would be off by up to 5e-6 of the result at
// y = 80).  A y past 104, infinity included, gives 0; NaN stays.
__device__ __forceinline__ float exp_neg(float y) {
  y = y > 104.f ? 104.f : y;
  const float t = -y * kLog2eF;
  const float lo = __builtin_fmaf(-y, kLog2eF, -t) - y * 1.925963033500e-8f;  // log2 e - float(log2 e)
  const float r = fast_exp2(t);
  return __builtin_fmaf(r, lo * kLn2F, r);
}

// a = sigmoid(z) and g = 1 - a = sigmoid(-z), each to float32's relative accuracy (1 - a as a
// difference would lose it where the gate is nearly open).  For z of 16 bits the exponent's own rounding,
// |z| 2^-24 of the small one of the two, is left in: z is known to 2^-12 of itself at best.
template <typename T>
__device__ __forceinline__ void gate(float z, float& a, float& g) {
  if constexpr (sizeof(T) == 4) {
    const float e = exp_neg(__builtin_fabsf(z)), small = e * __builtin_amdgcn_rcpf(1.f + e), big = 1.f - small;
    a = z < 0.f ? small : big;
    g = z < 0.f ? big : small;
  } else {
    const float e = fast_exp2(z * -kLog2eF);
    a = __builtin_amdgcn_rcpf(1.f + e);
    g = z < 0.f ? 1.f - a : e * a;
  }
}

template <int ACT>
struct Activation;

template <>
struct Activation<RNNT_ACT_RELU> {
  template <typename T>
  __device__ static __forceinline__ float value(float s) { return s < 0.f ? 0.f : s; }  // NaN stays
  __device__ static __forceinline__ float slope(float s) { return s > 0.f ? 1.f : 0.f; }
};

// tanh s = 1 - 2 / (1 + e^2s), which ends at -1 and 1 whatever overflows; near 0, where the difference loses
// digits, an odd polynomial.  For float32 of |s|, as at negative s the quotient would be near 1 and its rounding
// twice the value's, and from 0.6 on; the polynomial goes through s^11 (least relative error, 3e-9, fitted by
// reweighted least squares).  For a result of 16 bits (h is rounded to 2^-12 or 2^-9) of s itself, and from 0.3 on,
// through s^9: off by up to 8e-7, 271 -> 253 us for B=32 T=250 U=80 H=640 bf16 with dropout.  The slope is 4u / (1 + u)^2
// with u = e^-2|s|.  The rounding of the exponent, 2|s| 2^-24 of the exponential, needs no correction: where it
// grows, little of the value is left to it, and in the slope it is what the rounding of s itself costs.
template <>
struct Activation<RNNT_ACT_TANH> {
  __device__ static __forceinline__ float u_of(float s) { return fast_exp2(__builtin_fabsf(s) * (-2.f * kLog2eF)); }
  template <typename T>
  __device__ static __forceinline__ float value(float s) {
    constexpr bool F32 = sizeof(T) == 4;
    const float q = s * s, y = F32 ? __builtin_fabsf(s) : s;
    const float big = __builtin_fmaf(-2.f, __builtin_amdgcn_rcpf(1.f + fast_exp2(y * (2.f * kLog2eF))), 1.f);
    float p;
    if constexpr (F32) {
      p = __builtin_fmaf(q, -5.895158276e-3f, 2.079597116e-2f);
      p = __builtin_fmaf(q, p, -5.378383026e-2f);
      p = __builtin_fmaf(q, p, 1.333192438e-1f);
      p = __builtin_fmaf(q, p, -3.333329856e-1f);
    } else {
      p = __builtin_fmaf(q, 62.f / 2835.f, -17.f / 315.f);
      p = __builtin_fmaf(q, p, 2.f / 15.f);
      p = __builtin_fmaf(q, p, -1.f / 3.f);
    }
    return __builtin_fabsf(s) < (F32 ? 0.6f : 0.3f) ? __builtin_fmaf(q * p, s, s) : F32 ? __builtin_copysignf(big, s) : big;
  }
  __device__ static __forceinline__ float slope(float s) {
    const float u = u_of(s), r = __builtin_amdgcn_rcpf(1.f + u);
    return u * r * r * 4.f;
  }
};

// ---- random numbers -----------------------------------------------------------

// Philox4x32 (Salmon et al., SC 2011): a round multiplies two of the counter's four words by
// constants into 64 bits and folds the other two and the key, which advances by the Weyl
// constants, into the high halves.  Seven rounds are the fewest that the paper finds to pass
// every statistical test of its battery; the customary ten cost 3/7 more, and the rounds'
// multiplies (quarter rate) are what the dropout of 16-bit data would wait for.
struct Rng {
  uint32_t seed_lo, seed_hi, offset_lo, offset_hi;
};

__device__ __forceinline__ Rng load_rng(const int64_t* p) {
  const uint64_t s = static_cast<uint64_t>(p[0]), o = static_cast<uint64_t>(p[1]);
  return Rng{static_cast<uint32_t>(s), static_cast<uint32_t>(s >> 32), static_cast<uint32_t>(o),
             static_cast<uint32_t>(o >> 32)};
}

__device__ __forceinline__ uint32_t xor3(uint32_t a, uint32_t b, uint32_t c) {  // one instruction
  return static_cast<uint32_t>(__builtin_amdgcn_bitop3_b32(static_cast<int>(a), static_cast<int>(b), static_cast<int>(c), 0x96));
}

__device__ __forceinline__ uint4 random_block(const Rng& g, uint64_t block) {
  uint32_t c0 = static_cast<uint32_t>(block), c1 = static_cast<uint32_t>(block >> 32);
  uint32_t c2 = g.offset_lo, c3 = g.offset_hi, k0 = g.seed_lo, k1 = g.seed_hi;
#pragma unroll
  for (int r = 0; r < 7; ++r) {
    const uint64_t p0 = static_cast<uint64_t>(c0) * 0xD2511F53u, p1 = static_cast<uint64_t>(c2) * 0xCD9E8D57u;
    c0 = xor3(static_cast<uint32_t>(p1 >> 32), c1, k0);
    c1 = static_cast<uint32_t>(p1);
    c2 = xor3(static_cast<uint32_t>(p0 >> 32), c3, k1);
    c3 = static_cast<uint32_t>(p0);
    k0 += 0x9E3779B9u;
    k1 += 0xBB67AE85u;
  }
  return make_uint4(c0, c1, c2, c3);
}

// the 16-bit number of element i (0..7) of a block
__device__ __forceinline__ uint32_t random16(const uint4& b, int i) {
  const uint32_t w = i < 4 ? (i < 2 ? b.x : b.y) : (i < 6 ? b.z : b.w);
  return (i & 1) ? w >> 16 : w & 0xffffu;
}

// Which of the eight elements of a block are dropped: sixteen 1 bits each, two to a word, low half
// first.  A number x < q is found two at a time: both moved to the signed range, subtracted with
// saturation, and the sign spread.
typedef short i16x2 __attribute__((ext_vector_type(2)));
struct Dropped {
  uint32_t m[4];

  __device__ __forceinline__ void none() {
#pragma unroll
    for (int i = 0; i < 4; ++i) m[i] = 0;
  }
  // only the sign bits of the halves
  __device__ __forceinline__ void signs_below(const uint4& b, uint32_t q) {
    const uint32_t w[4] = {b.x, b.y, b.z, b.w}, limit = (q ^ 0x8000u) * 0x10001u;
#pragma unroll
    for (int i = 0; i < 4; ++i) {
      const i16x2 x = __builtin_bit_cast(i16x2, w[i] ^ 0x80008000u);
      m[i] = __builtin_bit_cast(uint32_t, __builtin_elementwise_sub_sat(x, __builtin_bit_cast(i16x2, limit)));
    }
  }
  __device__ __forceinline__ void below(const uint4& b, uint32_t q) {
    signs_below(b, q);
#pragma unroll
    for (int i = 0; i < 4; ++i) m[i] = spread(m[i]);
  }
  __device__ static __forceinline__ uint32_t spread(uint32_t signs) {
    return __builtin_bit_cast(uint32_t, __builtin_bit_cast(i16x2, signs) >> static_cast<short>(15));
  }
  // eight elements in memory form, the dropped ones 0
  template <typename T>
  __device__ __forceinline__ void clear(Pack<T, 8>& k) const {
    if constexpr (sizeof(T) == 2) {
#pragma unroll
      for (int i = 0; i < 4; ++i) k.w[i] &= ~m[i];
    } else {
#pragma unroll
      for (int i = 0; i < 8; ++i) k.w[i] &= ~static_cast<uint32_t>(static_cast<int32_t>((i & 1) ? m[i / 2] : m[i / 2] << 16) >> 31);
    }
  }
  // the sign bits as eight bits, and back
  __device__ __forceinline__ uint32_t bits() const {
    uint32_t out = 0;
#pragma unroll
    for (int i = 0; i < 4; ++i) out |= ((m[i] >> 15 & 1u) | (m[i] >> 30 & 2u)) << (2 * i);
    return out;
  }
  __device__ __forceinline__ void from_bits(uint32_t b) {
#pragma unroll
    for (int i = 0; i < 4; ++i) m[i] = (b >> (2 * i) & 1u) << 15 | (b >> (2 * i) & 2u) << 30;
  }
};

// dropout by numbers below `threshold`; kept elements are multiplied by `scale`
struct DropParams {
  uint32_t threshold;  // 0: nothing is dropped
  float scale;
  const int64_t* rng;  // {seed, offset} on the device, read when threshold > 0
};

// ---- host ---------------------------------------------------------------------

constexpr int64_t kMaxRows = 0x7fffffff;
// Results from here on are stored past the caches: half the 256 MB memory-side cache.  An embedding and the
// product that reads it, ordinary and streaming stores (us): 16 MB 15.5 and 17.5, 66 MB 38 and 41, 131 MB 72
// and 72, 262 MB 164 and 158, of which the embedding alone 88 and 47.
constexpr int64_t kStoreAway = int64_t{1} << 27;

inline size_t net_align256(size_t x) { return (x + 255) & ~static_cast<size_t>(255); }
inline bool net_dtype_known(int dt) { return dt == RNNT_DTYPE_F32 || dt == RNNT_DTYPE_BF16 || dt == RNNT_DTYPE_F16; }
inline int64_t net_elem_bytes(int dt) { return dt == RNNT_DTYPE_F32 ? 4 : 2; }
inline bool multiple_of(int64_t bytes, const void* p) { return reinterpret_cast<uintptr_t>(p) % bytes == 0; }

// p in [0, 1) as a threshold of 16-bit numbers; false for any other p (NaN included).
inline bool drop_params(double p, const int64_t* rng, DropParams* out) {
  if (!(p >= 0.0 && p < 1.0)) return false;
  const double q = __builtin_rint(p * 65536.0);
  out->threshold = q > 65535.0 ? 65535u : static_cast<uint32_t>(q);
  out->scale = static_cast<float>(65536.0 / (65536.0 - out->threshold));
  out->rng = rng;
  return true;
}

inline rnnt_status_t launched() { return hipGetLastError() == hipSuccess ? RNNT_OK : RNNT_ERR_HIP; }

// f called with a value of the dtype's element type
template <typename F>
rnnt_status_t with_dtype(rnnt_dtype_t dt, F&& f) {
  switch (dt) {
    case RNNT_DTYPE_F32: return f(float{});
    case RNNT_DTYPE_BF16: return f(bf16_t{});
    default: return f(f16_t{});
  }
}

}  // namespace rnnt
