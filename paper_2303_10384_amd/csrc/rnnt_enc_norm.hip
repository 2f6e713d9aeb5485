// The root-mean-square norm with the residual's addition, its gradient, and rows in 8 bits
// (contract in include/rnnt_encoder_mi355x.h).
#include <hip/hip_runtime.h>

#include <cstdint>

#include "rnnt_enc.h"

namespace rnnt {
namespace {

// A row is held by G lanes, in NV accesses of 16 bytes each, and read once: the sums need all of it before
// anything can be written.  G is as small as the row allows, so that narrow rows share a wave.  Bound by memory: with a
// residual, B=64 L=1000 D=1024 bf16 takes 73 us (465 MB, 6.4 TB/s).  In 8 bits B=32 L=1500 D=640 takes 41 us (188 MB, 4.5
// TB/s): 80 of 128 accesses of a row's lanes are there, and the vector units are busy for 87 % of the cycles.
struct RowsParams {
  const void *x, *residual, *weight;
  void *y, *sum;
  int8_t* q;
  float* scale;
  const int32_t* lens;
  int64_t pitch, rows;
  int32_t L, D;
  float eps;
};

enum RowsMode { kNorm, kNorm8, kQuantize };

// Where the i-th access of a row begins.  The last one of a row that is no whole number of them begins early: what it
// shares with its neighbour (`skip` elements) is written twice alike and counted once.
template <int VEC>
struct Place {
  int at, skip;
  bool any;
  __device__ __forceinline__ Place(int i, int D) : at(i * VEC), skip(0), any(i * VEC < D) {
    if (any && at + VEC > D && D >= VEC) {
      skip = at + VEC - D;
      at = D - VEC;
    }
  }
};

// D < VEC: one access of D elements
template <typename T>
__device__ __forceinline__ void load_row(Pack<T, kVec<T>>& k, const T* p, int D) {
  if (D >= kVec<T>) k.load(p);
  else k.load_part(p, D);
}
template <typename T>
__device__ __forceinline__ void store_row(const Pack<T, kVec<T>>& k, T* p, int D) {
  if (D >= kVec<T>) k.store(p);
  else k.store_part(p, D);
}

template <int VEC>
__device__ __forceinline__ void store_q(int8_t* p, const Words<VEC, 1>& w, int D) {
  if (D < VEC) {
    for (int j = 0; j < VEC; ++j)
      if (j < D) p[j] = static_cast<int8_t>(w.w[j / 4] >> (8 * (j % 4)));
    return;
  }
  *reinterpret_cast<Words<VEC, 1>*>(p) = w;
}

// Op over the G lanes of a row; G > 64: over the block
template <int G, typename Op>
__device__ __forceinline__ float row_reduce(float v, float* lds) {
  v = group_reduce<(G > 64 ? 64 : G), Op>(v, 0.f);
  if constexpr (G > 64) {
    if ((threadIdx.x & 63) == 0) lds[threadIdx.x >> 6] = v;
    __syncthreads();
    v = lds[0];
#pragma unroll
    for (int i = 1; i < G / 64; ++i) v = Op::apply(v, lds[i]);
  }
  return v;
}

// valid rows of row's utterance: 1 valid, 0 behind the length, -1 a bad length
__device__ __forceinline__ int row_state(const int32_t* lens, int64_t row, int L) {
  if (!lens) return 1;
  const int b = static_cast<int>(row / L), n = lens[b];
  if (n < 0 || n > L) return -1;
  return static_cast<int>(row - static_cast<int64_t>(b) * L) < n;
}

// A launch takes fewer than 2^32 threads along x, and 2^24 rows of 1024 lanes are 2^34: from here on blocks go along y.
constexpr int64_t kGridX = int64_t{1} << 21;

template <typename T, int G, int NV, int MODE>
__global__ __launch_bounds__(G > 256 ? G : 256) void enc_rows(RowsParams p) {
  constexpr int VEC = kVec<T>, kRows = G > 256 ? 1 : 256 / G;
  __shared__ float lds[2][G > 64 ? G / 64 : 1];
  const int lane = static_cast<int>(threadIdx.x) % G;
  const int64_t row = (blockIdx.y * kGridX + blockIdx.x) * kRows + threadIdx.x / G;
  const bool there = row < p.rows;
  const int state = MODE == kQuantize ? there : there ? row_state(p.lens, row, p.L) : 0;
  const int64_t base = row * p.D;
  float t[NV][VEC];
  float squares = 0.f, most = 0.f;
#pragma unroll
  for (int v = 0; v < NV; ++v) {
    const Place<VEC> at(v * G + lane, p.D);
#pragma unroll
    for (int j = 0; j < VEC; ++j) t[v][j] = 0.f;
    if (!at.any || state != 1) continue;
    Pack<T, VEC> k;
    load_row(k, static_cast<const T*>(p.x) + base + at.at, p.D);
    k.get(t[v]);
    if (MODE != kQuantize && p.residual) {
      float r[VEC];
      load_row(k, static_cast<const T*>(p.residual) + base + at.at, p.D);
      k.get(r);
#pragma unroll
      for (int j = 0; j < VEC; ++j) t[v][j] += r[j];
      k.set(t[v]);
      store_row(k, static_cast<T*>(p.sum) + base + at.at, p.D);
    }
#pragma unroll
    for (int j = 0; j < VEC; ++j)
      if (MODE != kQuantize && j >= at.skip) squares = __builtin_fmaf(t[v][j], t[v][j], squares);
    if constexpr (MODE != kQuantize) {
      float w[VEC];
      load_row(k, static_cast<const T*>(p.weight) + at.at, p.D);
      k.get(w);
#pragma unroll
      for (int j = 0; j < VEC; ++j) t[v][j] *= w[j];
    }
    if constexpr (MODE != kNorm) {
#pragma unroll
      for (int j = 0; j < VEC; ++j) most = MaxBitsOp::apply(most, __builtin_fabsf(t[v][j]));
    }
  }
  float unit = 1.f;
  if constexpr (MODE != kQuantize) {
    squares = row_reduce<G, SumOp>(squares, lds[0]);
    unit = __builtin_amdgcn_rsqf(squares / static_cast<float>(p.D) + p.eps);
  }
  if constexpr (MODE != kNorm) most = row_reduce<G, MaxBitsOp>(most, lds[1]);
  if (!there) return;
  const float nan = __builtin_nanf("");
  if constexpr (MODE != kNorm) {
    if (lane == 0) p.scale[row] = state < 0 ? nan : state == 0 ? 0.f : Quantizer::scale(most, unit);
  }
  const Quantizer quantizer(unit < __builtin_inff() ? most : 0.f);
#pragma unroll
  for (int v = 0; v < NV; ++v) {
    const Place<VEC> at(v * G + lane, p.D);
    if (!at.any) continue;
    Pack<T, VEC> k;
    if constexpr (MODE == kNorm) {
      float f[VEC];
#pragma unroll
      for (int j = 0; j < VEC; ++j) f[j] = state < 0 ? nan : t[v][j] * unit;
      k.set(f);
      if (state == 0) k.zero();
      store_row(k, static_cast<T*>(p.y) + base + at.at, p.D);
    } else {
      Words<VEC, 1> q;
#pragma unroll
      for (int j = 0; j < VEC / 4; ++j) q.w[j] = quantizer.four(t[v] + 4 * j);
      store_q<VEC>(p.q + row * p.pitch + at.at, q, p.D);
    }
    if (MODE != kQuantize && p.residual && state != 1) {
      float f[VEC];
#pragma unroll
      for (int j = 0; j < VEC; ++j) f[j] = state < 0 ? nan : 0.f;
      k.set(f);
      store_row(k, static_cast<T*>(p.sum) + base + at.at, p.D);
    }
  }
}

// ---- gradient -----------------------------------------------------------------
// A block takes every gridDim.x-th group of rows and keeps the sums of dy t r over its rows in registers; they meet in
// LDS and go out once, and enc_norm_join adds the blocks' up in their order.  t is added up again from x and the residual:
// the stored sum's rounding, of the size of dweight's own, would make dweight's error half as large again (B=64 L=1000
// D=1024 bf16: 2.6e-3 and 1.8e-3) for the 101 MB that are not read (99 and 120 us; 536 MB, 4.5 TB/s with 16 waves to a CU,
// 80 % of which wait: dsum is asked for only behind both sums of a row).  Past 8192 channels (4096 in float32) a block's
// registers do not hold the row, and spill: 4000 rows of 16384 bf16 take 439 us.

struct NormGradParams {
  const void *x, *residual, *weight, *dy, *dsum;
  void *dx, *dweight;
  float* part;  // (blocks, D)
  const int32_t* lens;
  int64_t rows;
  int32_t L, D, blocks;
  float eps;
};

template <typename T, int G, int NV>
__global__ __launch_bounds__(G > 256 ? G : 256) void enc_norm_grad(NormGradParams p) {
  constexpr int VEC = kVec<T>, kRows = G > 256 ? 1 : 256 / G, kThreads = G > 256 ? G : 256;
  constexpr bool kJoin = kRows > 1;
  __shared__ float lds[2][2][G > 64 ? G / 64 : 1];
  __shared__ float columns[kJoin ? kThreads * NV * VEC : 1];
  const int lane = static_cast<int>(threadIdx.x) % G, mine = static_cast<int>(threadIdx.x) / G;
  float w[NV][VEC], dw[NV][VEC];
#pragma unroll
  for (int v = 0; v < NV; ++v) {
    const Place<VEC> at(v * G + lane, p.D);
    Pack<T, VEC> k;
    k.zero();
    if (at.any) load_row(k, static_cast<const T*>(p.weight) + at.at, p.D);
    k.get(w[v]);
#pragma unroll
    for (int j = 0; j < VEC; ++j) dw[v][j] = 0.f;
  }
  const float inverse_d = 1.f / static_cast<float>(p.D);
  int turn = 0;
  for (int64_t first = static_cast<int64_t>(blockIdx.x) * kRows; first < p.rows; first += static_cast<int64_t>(gridDim.x) * kRows, turn ^= 1) {
    const int64_t row = first + mine, base = row * p.D;
    const bool there = row < p.rows, valid = there && row_state(p.lens, row, p.L) == 1;
    Pack<T, VEC> kt[NV], kr[NV], kg[NV];
    float squares = 0.f, dot = 0.f;
#pragma unroll
    for (int v = 0; v < NV; ++v) {
      const Place<VEC> at(v * G + lane, p.D);
      kt[v].zero();
      kr[v].zero();
      kg[v].zero();
      if (!at.any || !valid) continue;
      load_row(kt[v], static_cast<const T*>(p.x) + base + at.at, p.D);
      if (p.residual) load_row(kr[v], static_cast<const T*>(p.residual) + base + at.at, p.D);
      load_row(kg[v], static_cast<const T*>(p.dy) + base + at.at, p.D);
    }
    const auto sum_of = [&](int v, float* t) {
      float r[VEC];
      kt[v].get(t);
      kr[v].get(r);
#pragma unroll
      for (int j = 0; j < VEC; ++j) t[j] += r[j];
    };
#pragma unroll
    for (int v = 0; v < NV; ++v) {
      const Place<VEC> at(v * G + lane, p.D);
      float t[VEC], g[VEC];
      sum_of(v, t);
      kg[v].get(g);
#pragma unroll
      for (int j = 0; j < VEC; ++j) {
        if (j < at.skip) continue;
        squares = __builtin_fmaf(t[j], t[j], squares);
        dot = __builtin_fmaf(g[j] * w[v][j], t[j], dot);
      }
    }
    squares = row_reduce<G, SumOp>(squares, lds[turn][0]);
    dot = row_reduce<G, SumOp>(dot, lds[turn][1]);
    const float r = __builtin_amdgcn_rsqf(squares * inverse_d + p.eps), c = dot * inverse_d * r * r;
#pragma unroll
    for (int v = 0; v < NV; ++v) {
      const Place<VEC> at(v * G + lane, p.D);
      if (!at.any || !there) continue;
      float t[VEC], g[VEC], d[VEC];
      sum_of(v, t);
      kg[v].get(g);
      Pack<T, VEC> k;
      k.zero();
      if (p.dsum && valid) load_row(k, static_cast<const T*>(p.dsum) + base + at.at, p.D);
      k.get(d);
#pragma unroll
      for (int j = 0; j < VEC; ++j) {
        if (valid) dw[v][j] = __builtin_fmaf(g[j] * r, t[j], dw[v][j]);
        d[j] = valid ? __builtin_fmaf(r, __builtin_fmaf(-t[j], c, g[j] * w[v][j]), d[j]) : 0.f;
      }
      k.set(d);
      store_row(k, static_cast<T*>(p.dx) + base + at.at, p.D);
    }
  }
  float* part = p.part + static_cast<int64_t>(blockIdx.x) * p.D;
  if constexpr (kJoin) {
    constexpr int kWide = G * NV * VEC;
#pragma unroll
    for (int v = 0; v < NV; ++v) {
      const Place<VEC> at(v * G + lane, p.D);
#pragma unroll
      for (int j = 0; j < VEC; ++j)
        if (at.any && j >= at.skip && at.at + j < p.D) columns[mine * kWide + at.at + j] = dw[v][j];
    }
    __syncthreads();
    for (int i = static_cast<int>(threadIdx.x); i < p.D; i += kThreads) {
      float s = 0.f;
      for (int g = 0; g < kRows; ++g) s += columns[g * kWide + i];
      part[i] = s;
    }
  } else {
#pragma unroll
    for (int v = 0; v < NV; ++v) {
      const Place<VEC> at(v * G + lane, p.D);
#pragma unroll
      for (int j = 0; j < VEC; ++j)
        if (at.any && j >= at.skip && at.at + j < p.D) part[at.at + j] = dw[v][j];
    }
  }
}

// Sixteen columns to a block; thread (c, g) adds up the g-th of every sixteen blocks.
template <typename T>
__global__ __launch_bounds__(256) void enc_norm_join(NormGradParams p) {
  __shared__ float lds[16][17];
  const int c = static_cast<int>(threadIdx.x) % 16, g = static_cast<int>(threadIdx.x) / 16;
  const int col = static_cast<int>(blockIdx.x) * 16 + c;
  float s = 0.f;
  if (col < p.D)
#pragma unroll 8
    for (int i = g; i < p.blocks; i += 16) s += p.part[static_cast<int64_t>(i) * p.D + col];
  lds[g][c] = s;
  __syncthreads();
  if (g != 0 || col >= p.D) return;
  for (int i = 1; i < 16; ++i) s += lds[i][c];
  ElemTraits<T>::store1(static_cast<T*>(p.dweight) + col, s);
}

// ---- host ---------------------------------------------------------------------

// f called with the lanes of a row and its accesses to a lane as constants
template <typename F>
rnnt_status_t with_layout(int accesses, F&& f) {
  using std::integral_constant;
#define RNNT_LAYOUT(lanes, n) \
  if (accesses <= lanes * n) return f(integral_constant<int, lanes>{}, integral_constant<int, n>{});
  RNNT_LAYOUT(8, 1)
  RNNT_LAYOUT(16, 1)
  RNNT_LAYOUT(32, 1)
  RNNT_LAYOUT(64, 1)
  RNNT_LAYOUT(64, 2)
  RNNT_LAYOUT(64, 4)
  RNNT_LAYOUT(256, 4)
  RNNT_LAYOUT(1024, 4)
#undef RNNT_LAYOUT
  return RNNT_ERR_UNSUPPORTED;
}

int accesses_of(int32_t D, rnnt_dtype_t dtype) {
  const int vec = dtype == RNNT_DTYPE_F32 ? 4 : 8;
  return D / vec + (D % vec != 0);
}
int rows_of_block(int lanes) { return lanes > 256 ? 1 : 256 / lanes; }

rnnt_status_t check(const rnnt_norm_shape_t& s, float eps) {
  if (s.B < 1 || s.L < 0 || s.D < 1) return RNNT_ERR_BAD_SHAPE;
  if (!net_dtype_known(s.dtype)) return RNNT_ERR_BAD_DTYPE;
  if (!(eps >= 0.f && eps < __builtin_inff())) return RNNT_ERR_BAD_VARIANT;
  if (static_cast<int64_t>(s.B) * s.L >= kEncRows || accesses_of(s.D, s.dtype) > 4096) return RNNT_ERR_UNSUPPORTED;
  return RNNT_OK;
}

rnnt_status_t check_q(const int8_t* q, int64_t pitch, int32_t D) {
  if (!multiple_of(16, q) || pitch < D || pitch % 16 != 0) return RNNT_ERR_ALIGNMENT;
  return RNNT_OK;
}

template <int MODE>
rnnt_status_t launch_rows(const RowsParams& q, rnnt_dtype_t dtype, hipStream_t stream) {
  if (q.rows == 0) return RNNT_OK;
  return with_dtype(dtype, [&](auto t) {
    return with_layout(accesses_of(q.D, dtype), [&](auto lanes, auto n) {
      constexpr int G = decltype(lanes)::value, NV = decltype(n)::value;
      const int64_t per = rows_of_block(G), blocks = (q.rows + per - 1) / per, x = blocks < kGridX ? blocks : kGridX;
      const dim3 grid(static_cast<uint32_t>(x), static_cast<uint32_t>((blocks + x - 1) / x));
      hipLaunchKernelGGL((enc_rows<decltype(t), G, NV, MODE>), grid, dim3(G > 256 ? G : 256), 0, stream, q);
      return launched();
    });
  });
}

// Blocks of the gradient: four to a CU, or one to a group of rows
int grad_blocks(const rnnt_norm_shape_t& s) {
  int64_t per = 1;
  (void)with_layout(accesses_of(s.D, s.dtype), [&](auto lanes, auto) {
    per = rows_of_block(decltype(lanes)::value);
    return RNNT_OK;
  });
  const int64_t want = (static_cast<int64_t>(s.B) * s.L + per - 1) / per;
  return static_cast<int>(want < 1024 ? want : 1024);
}

rnnt_status_t norm_params(const void* x, const void* residual, const rnnt_norm_shape_t& s, const int32_t* lens,
                          const void* weight, float eps, void* sum, RowsParams* q) {
  const rnnt_status_t st = check(s, eps);
  if (st != RNNT_OK) return st;
  q->rows = static_cast<int64_t>(s.B) * s.L;
  if (!weight || (q->rows > 0 && (!x || (residual && !sum)))) return RNNT_ERR_NULL_PTR;
  const int64_t e = net_elem_bytes(s.dtype);
  if (!multiple_of(e, x) || !multiple_of(e, residual) || !multiple_of(e, weight) || !multiple_of(e, sum))
    return RNNT_ERR_ALIGNMENT;
  q->x = x;
  q->residual = residual;
  q->weight = weight;
  q->sum = sum;
  q->lens = lens;
  q->L = s.L;
  q->D = s.D;
  q->eps = eps;
  return RNNT_OK;
}

}  // namespace
}  // namespace rnnt

using namespace rnnt;

extern "C" {

rnnt_status_t rnnt_rms_norm(const void* x, const void* residual, rnnt_norm_shape_t shape, const int32_t* lens,
                            const void* weight, float eps, void* y, void* sum_out, hipStream_t stream) {
  RowsParams q{};
  const rnnt_status_t st = norm_params(x, residual, shape, lens, weight, eps, sum_out, &q);
  if (st != RNNT_OK) return st;
  if (q.rows > 0 && !y) return RNNT_ERR_NULL_PTR;
  if (!multiple_of(net_elem_bytes(shape.dtype), y)) return RNNT_ERR_ALIGNMENT;
  q.y = y;
  return launch_rows<kNorm>(q, shape.dtype, stream);
}

rnnt_status_t rnnt_rms_norm8(const void* x, const void* residual, rnnt_norm_shape_t shape, const int32_t* lens,
                             const void* weight, float eps, int8_t* q8, int64_t pitch, float* scale, void* sum_out,
                             hipStream_t stream) {
  RowsParams q{};
  rnnt_status_t st = norm_params(x, residual, shape, lens, weight, eps, sum_out, &q);
  if (st != RNNT_OK) return st;
  if (q.rows > 0 && (!q8 || !scale)) return RNNT_ERR_NULL_PTR;
  st = check_q(q8, pitch, shape.D);
  if (st != RNNT_OK) return st;
  if (!multiple_of(4, scale)) return RNNT_ERR_ALIGNMENT;
  q.q = q8;
  q.pitch = pitch;
  q.scale = scale;
  return launch_rows<kNorm8>(q, shape.dtype, stream);
}

rnnt_status_t rnnt_quantize_rows(const void* x, int64_t rows, int32_t D, rnnt_dtype_t dtype, int8_t* q8, int64_t pitch,
                                 float* scale, hipStream_t stream) {
  if (rows < 0 || D < 1) return RNNT_ERR_BAD_SHAPE;
  if (!net_dtype_known(dtype)) return RNNT_ERR_BAD_DTYPE;
  if (rows >= kEncRows || accesses_of(D, dtype) > 4096) return RNNT_ERR_UNSUPPORTED;
  if (rows > 0 && (!x || !q8 || !scale)) return RNNT_ERR_NULL_PTR;
  const rnnt_status_t st = check_q(q8, pitch, D);
  if (st != RNNT_OK) return st;
  if (!multiple_of(net_elem_bytes(dtype), x) || !multiple_of(4, scale)) return RNNT_ERR_ALIGNMENT;
  RowsParams q{};
  q.x = x;
  q.q = q8;
  q.pitch = pitch;
  q.scale = scale;
  q.rows = rows;
  q.L = 1;
  q.D = D;
  return launch_rows<kQuantize>(q, dtype, stream);
}

size_t rnnt_rms_norm_grad_workspace_bytes(rnnt_norm_shape_t shape) {
  if (check(shape, 0.f) != RNNT_OK) return 0;
  return net_align256(static_cast<size_t>(grad_blocks(shape)) * shape.D * sizeof(float));
}

rnnt_status_t rnnt_rms_norm_grad(const void* x, const void* residual, rnnt_norm_shape_t shape, const int32_t* lens,
                                 const void* weight, float eps, const void* dy, const void* dsum, void* dx,
                                 void* dweight, void* workspace, size_t workspace_bytes, hipStream_t stream) {
  rnnt_status_t st = check(shape, eps);
  if (st != RNNT_OK) return st;
  NormGradParams q{};
  q.rows = static_cast<int64_t>(shape.B) * shape.L;
  if (!weight || !dweight || (q.rows > 0 && (!x || !dy || !dx))) return RNNT_ERR_NULL_PTR;
  const int64_t e = net_elem_bytes(shape.dtype);
  if (!multiple_of(e, x) || !multiple_of(e, residual) || !multiple_of(e, weight) || !multiple_of(e, dy) ||
      !multiple_of(e, dsum) || !multiple_of(e, dx) || !multiple_of(e, dweight))
    return RNNT_ERR_ALIGNMENT;
  Workspace ws;
  st = ws.take(workspace, workspace_bytes, rnnt_rms_norm_grad_workspace_bytes(shape), stream);
  if (st != RNNT_OK) return st;
  q.x = x;
  q.residual = residual;
  q.weight = weight;
  q.dy = dy;
  q.dsum = dsum;
  q.dx = dx;
  q.dweight = dweight;
  q.part = reinterpret_cast<float*>(ws.ptr);
  q.lens = lens;
  q.L = shape.L;
  q.D = shape.D;
  q.eps = eps;
  q.blocks = grad_blocks(shape);
  return with_dtype(shape.dtype, [&](auto t) {
    using T = decltype(t);
    if (q.rows > 0) {
      st = with_layout(accesses_of(shape.D, shape.dtype), [&](auto lanes, auto n) {
        constexpr int G = decltype(lanes)::value, NV = decltype(n)::value;
        hipLaunchKernelGGL((enc_norm_grad<T, G, NV>), dim3(q.blocks), dim3(G > 256 ? G : 256), 0, stream, q);
        return launched();
      });
      if (st != RNNT_OK) return st;
    }
    hipLaunchKernelGGL((enc_norm_join<T>), dim3((shape.D + 15) / 16), dim3(256), 0, stream, q);
    return launched();
  });
}

}  // extern "C"
