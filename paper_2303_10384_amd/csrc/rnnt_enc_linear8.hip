// The product in 8-bit integers (contract in include/rnnt_encoder_mi355x.h).
#include <hip/hip_runtime.h>

#include <cstdint>

#include "rnnt_enc.h"

namespace rnnt {
namespace {

typedef int i32x4 __attribute__((ext_vector_type(4)));
typedef int i32x16 __attribute__((ext_vector_type(16)));

struct Linear8Params {
  const int8_t *x, *w;
  const float *x_scale, *w_scale;
  const void* bias;
  void* y;
  int64_t x_pitch, w_pitch;
  int32_t M, N, K, n_tiles;
};

constexpr int kTile = 128;  // rows of x and of w to a block
constexpr int kStep = 128;  // bytes of k to a step

// bytes k .. k + 15 of a row, 0 from K on
__device__ __forceinline__ u32x4 load_bytes(const int8_t* row, int k, int K) {
  u32x4 v = {0, 0, 0, 0};
  if (k >= K) return v;
  v = *reinterpret_cast<const u32x4*>(row + k);
  const int left = K - k;
  if (left < 16) {
#pragma unroll
    for (int i = 0; i < 4; ++i) {
      const int n = left - 4 * i;
      v[i] = n >= 4 ? v[i] : n <= 0 ? 0u : v[i] & ((1u << (8 * n)) - 1u);
    }
  }
  return v;
}

// A tile of 128 x 128 results to a block, 64 x 64 to a wave.  Steps of 128 bytes of k go through registers into two
// buffers of LDS in turn; the 16-byte pieces of a row lie at (piece ^ row % 8), so that the 32 rows that a matrix
// instruction reads at one piece meet all banks.
template <typename T>
__global__ __launch_bounds__(256) void enc_linear8(Linear8Params p) {
  __shared__ u32x4 lds[2][2][kTile * kStep / 16];
  const int thread = static_cast<int>(threadIdx.x), lane = thread & 63, wave = thread >> 6;
  const int64_t m0 = static_cast<int64_t>(blockIdx.x / p.n_tiles) * kTile;
  const int n0 = static_cast<int>(blockIdx.x % p.n_tiles) * kTile;
  const int piece = thread & 7, row = thread >> 3;
  const int8_t *from[2][4];
#pragma unroll
  for (int i = 0; i < 4; ++i) {
    const int64_t m = min(m0 + row + 32 * i, static_cast<int64_t>(p.M) - 1);
    const int n = min(n0 + row + 32 * i, p.N - 1);
    from[0][i] = p.x + m * p.x_pitch;
    from[1][i] = p.w + n * p.w_pitch;
  }
  i32x16 acc[2][2];
#pragma unroll
  for (int i = 0; i < 2; ++i)
#pragma unroll
    for (int j = 0; j < 2; ++j)
#pragma unroll
      for (int e = 0; e < 16; ++e) acc[i][j][e] = 0;
  u32x4 hold[2][4];
  const int steps = (p.K + kStep - 1) / kStep;
  const auto fetch = [&](int step) {
#pragma unroll
    for (int s = 0; s < 2; ++s)
#pragma unroll
      for (int i = 0; i < 4; ++i) hold[s][i] = load_bytes(from[s][i], step * kStep + piece * 16, p.K);
  };
  fetch(0);
  const int half = lane >> 5, r = lane & 31;
  const int m_wave = (wave >> 1) * 64, n_wave = (wave & 1) * 64;
  for (int step = 0; step < steps; ++step) {
    const int buf = step & 1;
#pragma unroll
    for (int s = 0; s < 2; ++s)
#pragma unroll
      for (int i = 0; i < 4; ++i) lds[buf][s][(row + 32 * i) * 8 + (piece ^ (row & 7))] = hold[s][i];
    if (step + 1 < steps) fetch(step + 1);
    __syncthreads();
#pragma unroll
    for (int k = 0; k < 4; ++k) {
      i32x4 a[2], b[2];
#pragma unroll
      for (int i = 0; i < 2; ++i) {
        const int ra = m_wave + 32 * i + r, rb = n_wave + 32 * i + r, at = (2 * k + half) ^ (r & 7);
        a[i] = __builtin_bit_cast(i32x4, lds[buf][0][ra * 8 + at]);
        b[i] = __builtin_bit_cast(i32x4, lds[buf][1][rb * 8 + at]);
      }
#pragma unroll
      for (int i = 0; i < 2; ++i)
#pragma unroll
        for (int j = 0; j < 2; ++j) acc[i][j] = __builtin_amdgcn_mfma_i32_32x32x32_i8(a[i], b[j], acc[i][j], 0, 0, 0);
    }
  }
#pragma unroll
  for (int j = 0; j < 2; ++j) {
    const int n = n0 + n_wave + 32 * j + r;
    if (n >= p.N) continue;
    const float ws = p.w_scale[n], bias = p.bias ? ElemTraits<T>::load1(static_cast<const T*>(p.bias) + n) : 0.f;
#pragma unroll
    for (int i = 0; i < 2; ++i)
#pragma unroll
      for (int e = 0; e < 16; ++e) {
        const int64_t m = m0 + m_wave + 32 * i + 8 * (e / 4) + 4 * half + e % 4;
        if (m >= p.M) continue;
        const float v = static_cast<float>(acc[i][j][e]) * p.x_scale[m] * ws;
        ElemTraits<T>::store1(static_cast<T*>(p.y) + m * p.N + n, v + bias);
      }
  }
}

// ---- host ---------------------------------------------------------------------

int64_t tiles_of(const rnnt_linear8_shape_t& s) {
  return (static_cast<int64_t>(s.M) + kTile - 1) / kTile * ((static_cast<int64_t>(s.N) + kTile - 1) / kTile);
}

bool bad_pitch(int64_t pitch) { return pitch % 16 != 0; }

rnnt_status_t check(const rnnt_linear8_shape_t& s, bool dynamic) {
  if (s.M < 0 || s.N < 1 || s.K < 1 || s.w_pitch < s.K || (!dynamic && s.x_pitch < s.K)) return RNNT_ERR_BAD_SHAPE;
  if (!net_dtype_known(s.dtype)) return RNNT_ERR_BAD_DTYPE;
  if (bad_pitch(s.w_pitch) || (!dynamic && bad_pitch(s.x_pitch))) return RNNT_ERR_ALIGNMENT;
  const int most = dynamic ? (s.dtype == RNNT_DTYPE_F32 ? 16384 : 32768) : (1 << 17) - 1;
  if (s.K > most || s.M >= kEncRows || s.N > (1 << 21) || s.w_pitch >= (1 << 20) ||
      (!dynamic && s.x_pitch >= (1 << 20)) || tiles_of(s) > kMaxRows / 256)
    return RNNT_ERR_UNSUPPORTED;
  return RNNT_OK;
}

rnnt_status_t check_memory(const rnnt_linear8_shape_t& s, const int8_t* w, const float* w_scale, const void* bias,
                           const void* y) {
  if (!w || !w_scale || (s.M > 0 && !y)) return RNNT_ERR_NULL_PTR;
  const int64_t e = net_elem_bytes(s.dtype);
  if (!multiple_of(16, w) || !multiple_of(4, w_scale) || !multiple_of(e, bias) || !multiple_of(e, y))
    return RNNT_ERR_ALIGNMENT;
  return RNNT_OK;
}

rnnt_status_t launch(const Linear8Params& q, const rnnt_linear8_shape_t& s, hipStream_t stream) {
  if (s.M == 0) return RNNT_OK;
  return with_dtype(s.dtype, [&](auto t) {
    hipLaunchKernelGGL((enc_linear8<decltype(t)>), dim3(static_cast<uint32_t>(tiles_of(s))), dim3(256), 0, stream, q);
    return launched();
  });
}

Linear8Params params_of(const rnnt_linear8_shape_t& s, const int8_t* w, const float* w_scale, const void* bias, void* y) {
  Linear8Params q{};
  q.w = w;
  q.w_scale = w_scale;
  q.bias = bias;
  q.y = y;
  q.w_pitch = s.w_pitch;
  q.M = s.M;
  q.N = s.N;
  q.K = s.K;
  q.n_tiles = (s.N + kTile - 1) / kTile;
  return q;
}

int64_t own_pitch(const rnnt_linear8_shape_t& s) { return (static_cast<int64_t>(s.K) + 15) / 16 * 16; }

}  // namespace
}  // namespace rnnt

using namespace rnnt;

extern "C" {

rnnt_status_t rnnt_linear8(const int8_t* x, const float* x_scale, const int8_t* w, const float* w_scale,
                           rnnt_linear8_shape_t shape, const void* bias, void* y, hipStream_t stream) {
  rnnt_status_t st = check(shape, false);
  if (st != RNNT_OK) return st;
  if (shape.M > 0 && (!x || !x_scale)) return RNNT_ERR_NULL_PTR;
  st = check_memory(shape, w, w_scale, bias, y);
  if (st != RNNT_OK) return st;
  if (!multiple_of(16, x) || !multiple_of(4, x_scale)) return RNNT_ERR_ALIGNMENT;
  Linear8Params q = params_of(shape, w, w_scale, bias, y);
  q.x = x;
  q.x_scale = x_scale;
  q.x_pitch = shape.x_pitch;
  return launch(q, shape, stream);
}

size_t rnnt_linear8_dynamic_workspace_bytes(rnnt_linear8_shape_t shape) {
  if (check(shape, true) != RNNT_OK) return 0;
  return net_align256(static_cast<size_t>(shape.M) * own_pitch(shape)) + net_align256(static_cast<size_t>(shape.M) * 4);
}

rnnt_status_t rnnt_linear8_dynamic(const void* x, const int8_t* w, const float* w_scale, rnnt_linear8_shape_t shape,
                                   const void* bias, void* y, void* workspace, size_t workspace_bytes,
                                   hipStream_t stream) {
  rnnt_status_t st = check(shape, true);
  if (st != RNNT_OK) return st;
  if (shape.M > 0 && !x) return RNNT_ERR_NULL_PTR;
  st = check_memory(shape, w, w_scale, bias, y);
  if (st != RNNT_OK) return st;
  if (!multiple_of(net_elem_bytes(shape.dtype), x)) return RNNT_ERR_ALIGNMENT;
  Workspace ws;
  st = ws.take(workspace, workspace_bytes, rnnt_linear8_dynamic_workspace_bytes(shape), stream);
  if (st != RNNT_OK) return st;
  Linear8Params q = params_of(shape, w, w_scale, bias, y);
  q.x_pitch = own_pitch(shape);
  int8_t* rows = reinterpret_cast<int8_t*>(ws.ptr);
  float* scale = reinterpret_cast<float*>(ws.ptr + net_align256(static_cast<size_t>(shape.M) * q.x_pitch));
  st = rnnt_quantize_rows(x, shape.M, shape.K, shape.dtype, rows, q.x_pitch, scale, stream);
  if (st != RNNT_OK) return st;
  q.x = rows;
  q.x_scale = scale;
  return launch(q, shape, stream);
}

}  // extern "C"
