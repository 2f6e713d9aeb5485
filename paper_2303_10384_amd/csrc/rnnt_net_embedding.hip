// Label embedding and its gradient (contract in include/rnnt_network_mi355x.h).
#include <hip/hip_runtime.h>

#include <cstdint>

#include "rnnt_net.h"

namespace rnnt {
namespace {

// Where the token of an output row comes from: row r = (b, i) of B x n1 rows.
struct TokenSource {
  const int32_t* labels;  // (B, N)
  const int32_t* lens;    // (B) or null
  int32_t B, N, n1, V, start;
};
constexpr int32_t kPaddingRow = -1;  // behind the utterance's length
constexpr int32_t kBadRow = -2;      // a label outside [0, V), or a length outside [0, N]

__device__ __forceinline__ int32_t token_at(const TokenSource& s, int32_t r) {
  const int32_t b = static_cast<int32_t>(static_cast<uint32_t>(r) / static_cast<uint32_t>(s.n1));
  const int32_t i = r - b * s.n1;
  const int32_t len = s.lens ? s.lens[b] : s.N;
  if (len < 0 || len > s.N) return kBadRow;
  const int32_t first = s.n1 - s.N;  // 1 with a start row
  if (i < first) return s.start;
  if (i - first >= len) return kPaddingRow;
  const int32_t v = s.labels[static_cast<int64_t>(b) * s.N + (i - first)];
  return static_cast<uint32_t>(v) < static_cast<uint32_t>(s.V) ? v : kBadRow;
}

struct EmbeddingParams {
  TokenSource src;
  const void* weight;
  void* out;
  float scale;
  int32_t D, rows, lanes;  // lanes: threads to a row, a power of two
};

template <typename T, int VEC>
__global__ __launch_bounds__(256) void net_embedding(EmbeddingParams p) {
  const int row = static_cast<int>(blockIdx.x) * (256 / p.lanes) + static_cast<int>(threadIdx.x) / p.lanes;
  if (row >= p.rows) return;
  const int32_t v = token_at(p.src, row);
  const T* w = static_cast<const T*>(p.weight) + static_cast<int64_t>(v) * p.D;
  T* o = static_cast<T*>(p.out) + static_cast<int64_t>(row) * p.D;
  for (int c = (static_cast<int>(threadIdx.x) & (p.lanes - 1)) * VEC; c < p.D; c += p.lanes * VEC) {
    float f[VEC];
    Pack<T, VEC> k;
    if (v >= 0) {
      k.load(w + c);
      k.get(f);
#pragma unroll
      for (int j = 0; j < VEC; ++j) f[j] *= p.scale;
    } else {
#pragma unroll
      for (int j = 0; j < VEC; ++j) f[j] = v == kBadRow ? __builtin_nanf("") : 0.f;
    }
    k.set(f);
    k.store(o + c);
  }
}

struct EmbeddingGradParams {
  TokenSource src;
  const void* dout;
  void* dweight;
  float scale;
  int32_t D, rows;
};

// One block to a weight row: it looks at every token and adds the rows of its own, in order.
template <typename T, int VEC>
__global__ __launch_bounds__(256) void net_embedding_grad(EmbeddingGradParams p) {
  const int32_t v = static_cast<int32_t>(blockIdx.x);
  __shared__ int32_t found[256];
  __shared__ int32_t count[4];
  for (int c0 = 0; c0 < p.D; c0 += 256 * VEC) {
    const int c = c0 + static_cast<int>(threadIdx.x) * VEC;
    float sum[VEC] = {};
    for (int r0 = 0; r0 < p.rows; r0 += 256) {
      const int r = r0 + static_cast<int>(threadIdx.x);
      const bool hit = r < p.rows && token_at(p.src, r) == v;
      const uint64_t votes = __ballot(hit);
      const int wave = static_cast<int>(threadIdx.x) >> 6, lane = static_cast<int>(threadIdx.x) & 63;
      if (lane == 0) count[wave] = __popcll(votes);
      __syncthreads();
      int at = __popcll(votes & ((uint64_t{1} << lane) - 1)), n = 0;
      for (int w = 0; w < 4; ++w) {
        at += w < wave ? count[w] : 0;
        n += count[w];
      }
      if (hit) found[at] = r;
      __syncthreads();
      if (c < p.D) {
        for (int i = 0; i < n; ++i) {
          float f[VEC];
          Pack<T, VEC> k;
          k.load(static_cast<const T*>(p.dout) + static_cast<int64_t>(found[i]) * p.D + c);
          k.get(f);
#pragma unroll
          for (int j = 0; j < VEC; ++j) sum[j] += f[j];
        }
      }
      __syncthreads();
    }
    if (c < p.D) {
#pragma unroll
      for (int j = 0; j < VEC; ++j) sum[j] *= p.scale;
      Pack<T, VEC> k;
      k.set(sum);
      k.store(static_cast<T*>(p.dweight) + static_cast<int64_t>(v) * p.D + c);
    }
  }
}

rnnt_status_t check(const int32_t* labels, const rnnt_embedding_shape_t& s, TokenSource* src, const int32_t* lens) {
  if (s.B < 1 || s.N < 0 || s.V < 1 || s.D < 1 || s.start < -1 || s.start >= s.V) return RNNT_ERR_BAD_SHAPE;
  if (!net_dtype_known(s.dtype)) return RNNT_ERR_BAD_DTYPE;
  const int64_t n1 = static_cast<int64_t>(s.N) + (s.start >= 0);
  if (n1 * s.B > kMaxRows) return RNNT_ERR_UNSUPPORTED;
  if (!labels && s.N > 0) return RNNT_ERR_NULL_PTR;
  *src = TokenSource{labels, lens, s.B, s.N, static_cast<int32_t>(n1), s.V, s.start};
  return RNNT_OK;
}

// rows that start on 16 bytes take 16-byte accesses
bool wide_rows(int D, rnnt_dtype_t dt, const void* a, const void* b) {
  return D * net_elem_bytes(dt) % 16 == 0 && multiple_of(16, a) && multiple_of(16, b);
}

int lanes_for(int chunks) {
  int n = 1;
  while (n < 256 && n < chunks) n *= 2;
  return n;
}

}  // namespace
}  // namespace rnnt

using namespace rnnt;

extern "C" {

rnnt_status_t rnnt_label_embedding(const int32_t* labels, const int32_t* lens, rnnt_embedding_shape_t shape,
                                   const void* weight, float scale, void* out, hipStream_t stream) {
  EmbeddingParams p{};
  const rnnt_status_t st = check(labels, shape, &p.src, lens);
  if (st != RNNT_OK) return st;
  p.rows = p.src.n1 * shape.B;
  if (p.rows == 0) return RNNT_OK;
  if (!weight || !out) return RNNT_ERR_NULL_PTR;
  const int64_t e = net_elem_bytes(shape.dtype);
  if (!multiple_of(e, weight) || !multiple_of(e, out)) return RNNT_ERR_ALIGNMENT;
  p.weight = weight;
  p.out = out;
  p.scale = scale;
  p.D = shape.D;
  const bool wide = wide_rows(shape.D, shape.dtype, weight, out);
  return with_dtype(shape.dtype, [&](auto t) {
    using T = decltype(t);
    constexpr int VEC = 16 / sizeof(T);
    p.lanes = lanes_for(wide ? shape.D / VEC : shape.D);
    const int per = 256 / p.lanes;
    const dim3 grid(static_cast<uint32_t>((static_cast<int64_t>(p.rows) + per - 1) / per));
    if (wide) hipLaunchKernelGGL((net_embedding<T, VEC>), grid, dim3(256), 0, stream, p);
    else hipLaunchKernelGGL((net_embedding<T, 1>), grid, dim3(256), 0, stream, p);
    return launched();
  });
}

size_t rnnt_label_embedding_grad_workspace_bytes(rnnt_embedding_shape_t shape) {
  TokenSource src;
  int32_t any;
  return check(&any, shape, &src, nullptr) == RNNT_OK ? 256 : 0;
}

rnnt_status_t rnnt_label_embedding_grad(const int32_t* labels, const int32_t* lens, rnnt_embedding_shape_t shape,
                                        const void* dout, float scale, void* dweight, void* workspace,
                                        size_t workspace_bytes, hipStream_t stream) {
  EmbeddingGradParams p{};
  rnnt_status_t st = check(labels, shape, &p.src, lens);
  if (st != RNNT_OK) return st;
  p.rows = p.src.n1 * shape.B;
  if (!dweight || (!dout && p.rows > 0)) return RNNT_ERR_NULL_PTR;
  const int64_t e = net_elem_bytes(shape.dtype);
  if (!multiple_of(e, dout) || !multiple_of(e, dweight)) return RNNT_ERR_ALIGNMENT;
  NetWorkspace ws;
  st = ws.take(workspace, workspace_bytes, rnnt_label_embedding_grad_workspace_bytes(shape), stream);
  if (st != RNNT_OK) return st;
  p.dout = dout;
  p.dweight = dweight;
  p.scale = scale;
  p.D = shape.D;
  const bool wide = wide_rows(shape.D, shape.dtype, dout, dweight);
  return with_dtype(shape.dtype, [&](auto t) {
    using T = decltype(t);
    constexpr int VEC = 16 / sizeof(T);
    if (wide) hipLaunchKernelGGL((net_embedding_grad<T, VEC>), dim3(shape.V), dim3(256), 0, stream, p);
    else hipLaunchKernelGGL((net_embedding_grad<T, 1>), dim3(shape.V), dim3(256), 0, stream, p);
    return launched();
  });
}

}  // extern "C"
