// Rotary positions (contract in include/rnnt_encoder_mi355x.h).
#include <hip/hip_runtime.h>

#include <cstdint>

#include "rnnt_enc.h"

namespace rnnt {
namespace {

// A block takes a few tokens.  Their angles' cosines and sines are formed once, for all heads, and kept in LDS;
// then a thread takes eight pairs of a head, or eight of the channels that are copied.  Bound by waiting: B=32 L=250 of 16
// heads of 64, 32 of them turned, bf16, takes 13.5 us for 29 MB (2.2 TB/s; a copy would be 5), 66 % of the waves waiting:
// lengths, positions and angles lie before the first load of x.
struct RotaryParams {
  const void* x;
  void* y;
  const double* freq;
  const int32_t *start, *lens;
  int64_t stride_b, stride_t, stride_h, tokens;
  int32_t L, H, D, R;
  int32_t block_tokens, pair_items, items;   // of a block; of a head
  uint32_t items_magic, token_magic;         // division by items and by items * H
  float sign;
};

constexpr int kTablePairs = 4096;  // pairs of a block's tokens

// n / d of n, d < 2^16, by the high word of a product
__host__ __device__ constexpr uint32_t magic_of(uint32_t d) { return d == 1 ? 0 : static_cast<uint32_t>((uint64_t{1} << 32) / d + 1); }
__device__ __forceinline__ uint32_t divided(uint32_t n, uint32_t magic) { return magic ? __umulhi(n, magic) : n; }

template <typename T>
__device__ __forceinline__ void load8(Pack<T, 8>& k, const T* p, int n) {
  if (n == 8) k.load(p);
  else k.load_part(p, n);
}
template <typename T>
__device__ __forceinline__ void store8(const Pack<T, 8>& k, T* p, int n) {
  if (n == 8) k.store(p);
  else k.store_part(p, n);
}

template <typename T, bool INTERLEAVED>
__global__ __launch_bounds__(256) void enc_rotary(RotaryParams p) {
  __shared__ float2 table[kTablePairs];
  const int64_t first = static_cast<int64_t>(blockIdx.x) * p.block_tokens;
  const int half = p.R / 2, tokens = static_cast<int>(min(static_cast<int64_t>(p.block_tokens), p.tokens - first));
  for (int i = static_cast<int>(threadIdx.x); i < tokens * half; i += 256) {
    const int token = i / half, pair = i - token * half;
    const int64_t row = first + token;
    const int b = static_cast<int>(row / p.L), t = static_cast<int>(row - static_cast<int64_t>(b) * p.L);
    // whole turns go away in float64; what is left of the angle, in half turns, needs no more than float32
    const double turns = (static_cast<double>(p.start ? p.start[b] : 0) + t) * p.freq[pair] * 0.15915494309189533577;
    const float f = static_cast<float>(turns - __builtin_rint(turns)) * 2.f;
    float s, c;
    sincospif(f, &s, &c);
    table[i] = make_float2(c, s * p.sign);
  }
  __syncthreads();
  const int total = tokens * p.H * p.items;
  for (int i = static_cast<int>(threadIdx.x); i < total; i += 256) {
    const int head_of_all = static_cast<int>(divided(static_cast<uint32_t>(i), p.items_magic)), item = i - head_of_all * p.items;
    const int token = static_cast<int>(divided(static_cast<uint32_t>(i), p.token_magic)), h = head_of_all - token * p.H;
    const int64_t row = first + token;
    const int b = static_cast<int>(row / p.L), t = static_cast<int>(row - static_cast<int64_t>(b) * p.L);
    const T* x = static_cast<const T*>(p.x) + b * p.stride_b + t * p.stride_t + h * p.stride_h;
    T* y = static_cast<T*>(p.y) + (row * p.H + h) * p.D;
    const int n = p.lens ? p.lens[b] : p.L;
    const bool bad = n < 0 || n > p.L, valid = !bad && t < n;
    const float fill = bad && p.sign > 0.f ? __builtin_nanf("") : 0.f;  // gradients of a bad length are 0
    if (item < p.pair_items) {
      // the last eight pairs begin early, and write what they share with their neighbours twice alike
      const int count = min(half, 8), at = min(item * 8, half - count);
      float a[8], c[8];
      Pack<T, 8> ka, kb;
      const int at_a = INTERLEAVED ? 2 * at : at, at_b = INTERLEAVED ? 2 * at + 8 : at + half;
      const int n_a = INTERLEAVED ? min(2 * count, 8) : count, n_b = INTERLEAVED ? max(2 * count - 8, 0) : count;
      if (valid) {
        load8(ka, x + at_a, n_a);
        load8(kb, x + at_b, n_b);
        ka.get(a);
        kb.get(c);
        const float2* turn = table + token * half + at;
#pragma unroll
        for (int j = 0; j < 8; ++j) {
          if (j >= count) continue;
          const float2 cs = turn[j];
          float &u = INTERLEAVED ? (j < 4 ? a[2 * j] : c[2 * j - 8]) : a[j];
          float &v = INTERLEAVED ? (j < 4 ? a[2 * j + 1] : c[2 * j - 7]) : c[j];
          const float p0 = u * cs.x - v * cs.y, p1 = u * cs.y + v * cs.x;
          u = p0;
          v = p1;
        }
      } else {
#pragma unroll
        for (int j = 0; j < 8; ++j) a[j] = c[j] = fill;
      }
      ka.set(a);
      kb.set(c);
      store8(ka, y + at_a, n_a);
      store8(kb, y + at_b, n_b);
    } else {
      const int rest = p.D - p.R, count = min(rest, 8), at = p.R + min((item - p.pair_items) * 8, rest - count);
      Pack<T, 8> k;
      if (valid) {
        load8(k, x + at, count);
      } else {
        float f[8];
#pragma unroll
        for (int j = 0; j < 8; ++j) f[j] = fill;
        k.set(f);
      }
      store8(k, y + at, count);
    }
  }
}

}  // namespace
}  // namespace rnnt

using namespace rnnt;

extern "C" rnnt_status_t rnnt_rotary(const void* x, rnnt_rotary_shape_t shape, const double* freq, const int32_t* start,
                                     const int32_t* lens, int32_t inverse, void* y, hipStream_t stream) {
  const rnnt_rotary_shape_t& s = shape;
  if (s.B < 1 || s.L < 0 || s.H < 1 || s.D < 1 || s.R < 2 || s.R % 2 != 0 || s.R > s.D || s.stride_b < 0 ||
      s.stride_t < 0 || s.stride_h < 0)
    return RNNT_ERR_BAD_SHAPE;
  if (!net_dtype_known(s.dtype)) return RNNT_ERR_BAD_DTYPE;
  RotaryParams q{};
  q.tokens = static_cast<int64_t>(s.B) * s.L;
  if (static_cast<int64_t>(s.H) * s.D > (1 << 16) || s.R > 1024 || q.tokens >= kEncRows) return RNNT_ERR_UNSUPPORTED;
  if (!freq || (q.tokens > 0 && (!x || !y))) return RNNT_ERR_NULL_PTR;
  const int64_t e = net_elem_bytes(s.dtype);
  if (!multiple_of(e, x) || !multiple_of(e, y) || !multiple_of(8, freq)) return RNNT_ERR_ALIGNMENT;
  if (q.tokens == 0) return RNNT_OK;
  q.x = x;
  q.y = y;
  q.freq = freq;
  q.start = start;
  q.lens = lens;
  q.stride_b = s.stride_b;
  q.stride_t = s.stride_t;
  q.stride_h = s.stride_h;
  q.L = s.L;
  q.H = s.H;
  q.D = s.D;
  q.R = s.R;
  q.sign = inverse ? -1.f : 1.f;
  q.pair_items = (s.R / 2 + 7) / 8;
  q.items = q.pair_items + (s.D - s.R + 7) / 8;
  q.items_magic = magic_of(static_cast<uint32_t>(q.items));
  q.token_magic = magic_of(static_cast<uint32_t>(q.items * s.H));
  // a token to a block while that leaves CUs idle, else up to 8192 elements: one round of angles for several of data
  int64_t most = 8192 / (static_cast<int64_t>(s.H) * s.D), by_table = kTablePairs / (s.R / 2), by_grid = q.tokens / 1024;
  int64_t per = most < by_table ? most : by_table;
  per = per < by_grid ? per : by_grid;
  q.block_tokens = static_cast<int32_t>(per < 1 ? 1 : per);
  const int64_t blocks = (q.tokens + q.block_tokens - 1) / q.block_tokens;
  return with_dtype(s.dtype, [&](auto t) {
    using T = decltype(t);
    const dim3 grid(static_cast<uint32_t>(blocks));
    if (s.interleaved) hipLaunchKernelGGL((enc_rotary<T, true>), grid, dim3(256), 0, stream, q);
    else hipLaunchKernelGGL((enc_rotary<T, false>), grid, dim3(256), 0, stream, q);
    return launched();
  });
}
