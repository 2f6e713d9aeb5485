// Gated linear recurrence and its gradient (contract in include/rnnt_network_mi355x.h).
#include <hip/hip_runtime.h>

#include <cstdint>

#include "rnnt_net.h"

namespace rnnt {
namespace {

constexpr int kStateSteps = RNNT_RECURRENCE_STATE_STEPS;

struct RecurrenceParams {
  const void *x, *z;
  int64_t x_sb, x_st, z_sb, z_st;
  const int32_t* lens;
  const float* h0;
  void* h;
  float* last;
  float* states;  // (B, ceil(L / kStateSteps), D), or null
  int32_t B, L, D, n_states;
};

__device__ __forceinline__ int length_of(const int32_t* lens, int b, int L) { return lens ? lens[b] : L; }

// One thread to a channel, step by step.
template <typename T>
__global__ __launch_bounds__(64) void net_recurrence(RecurrenceParams p) {
  const int c = static_cast<int>(blockIdx.x) * 64 + static_cast<int>(threadIdx.x), b = static_cast<int>(blockIdx.y);
  if (c >= p.D) return;
  const int len = length_of(p.lens, b, p.L);
  const bool bad = len < 0 || len > p.L;
  const T* x = static_cast<const T*>(p.x) + b * p.x_sb + c;
  const T* z = static_cast<const T*>(p.z) + b * p.z_sb + c;
  T* h = static_cast<T*>(p.h) + static_cast<int64_t>(b) * p.L * p.D + c;
  const int64_t bc = static_cast<int64_t>(b) * p.D + c;
  float* st = p.states ? p.states + static_cast<int64_t>(b) * p.n_states * p.D + c : nullptr;
  float s = bad ? __builtin_nanf("") : p.h0 ? p.h0[bc] : 0.f;
  for (int t = 0; t < p.L; ++t) {
    if (st && t % kStateSteps == 0) st[static_cast<int64_t>(t / kStateSteps) * p.D] = s;
    float o = bad ? s : 0.f;
    if (!bad && t < len) {
      float a, g;
      gate(ElemTraits<T>::load1(z + t * p.z_st), a, g);
      s = __builtin_fmaf(g, ElemTraits<T>::load1(x + t * p.x_st) - s, s);
      o = s;
    }
    ElemTraits<T>::store1(h + static_cast<int64_t>(t) * p.D, o);
  }
  p.last[bc] = s;
}

struct RecurrenceGradParams {
  const void *x, *z;
  int64_t x_sb, x_st, z_sb, z_st;
  const int32_t* lens;
  const float* states;
  const void* dh;
  const float* dlast;
  void *dx, *dz;
  float* dh0;
  int32_t B, L, D, n_states;
};

template <typename T>
__global__ __launch_bounds__(64) void net_recurrence_grad(RecurrenceGradParams p) {
  const int c = static_cast<int>(blockIdx.x) * 64 + static_cast<int>(threadIdx.x), b = static_cast<int>(blockIdx.y);
  if (c >= p.D) return;
  int len = length_of(p.lens, b, p.L);
  const bool bad = len < 0 || len > p.L;
  if (bad) len = 0;
  const T* x = static_cast<const T*>(p.x) + b * p.x_sb + c;
  const T* z = static_cast<const T*>(p.z) + b * p.z_sb + c;
  const int64_t base = static_cast<int64_t>(b) * p.L * p.D + c, bc = static_cast<int64_t>(b) * p.D + c;
  const T* dh = p.dh ? static_cast<const T*>(p.dh) + base : nullptr;
  T *dx = static_cast<T*>(p.dx) + base, *dz = static_cast<T*>(p.dz) + base;
  float d = bad || !p.dlast ? 0.f : p.dlast[bc];
  for (int t0 = (p.L - 1) / kStateSteps * kStateSteps; t0 >= 0 && p.L > 0; t0 -= kStateSteps) {
    float before[kStateSteps], xs[kStateSteps], as[kStateSteps], gs[kStateSteps];
    float s = p.states[(static_cast<int64_t>(b) * p.n_states + t0 / kStateSteps) * p.D + c];
#pragma unroll
    for (int j = 0; j < kStateSteps; ++j) {
      before[j] = s;
      if (t0 + j < len) {
        gate(ElemTraits<T>::load1(z + (t0 + j) * p.z_st), as[j], gs[j]);
        xs[j] = ElemTraits<T>::load1(x + (t0 + j) * p.x_st);
        s = __builtin_fmaf(gs[j], xs[j] - s, s);
      }
    }
#pragma unroll
    for (int j = kStateSteps - 1; j >= 0; --j) {
      const int t = t0 + j;
      if (t >= p.L) continue;
      float ox = 0.f, oz = 0.f;
      if (t < len) {
        const float total = d + (dh ? ElemTraits<T>::load1(dh + static_cast<int64_t>(t) * p.D) : 0.f);
        ox = gs[j] * total;
        oz = total * (before[j] - xs[j]) * (as[j] * gs[j]);
        d = as[j] * total;
      }
      ElemTraits<T>::store1(dx + static_cast<int64_t>(t) * p.D, ox);
      ElemTraits<T>::store1(dz + static_cast<int64_t>(t) * p.D, oz);
    }
  }
  if (p.dh0) p.dh0[bc] = d;
}

rnnt_status_t check(const rnnt_recurrence_shape_t& s) {
  if (s.B < 1 || s.L < 0 || s.D < 1 || s.x_stride_b < 0 || s.x_stride_t < 0 || s.z_stride_b < 0 || s.z_stride_t < 0)
    return RNNT_ERR_BAD_SHAPE;
  if (!net_dtype_known(s.dtype)) return RNNT_ERR_BAD_DTYPE;
  if (s.B > 65535) return RNNT_ERR_UNSUPPORTED;
  return RNNT_OK;
}

int state_count(int L) { return (L + kStateSteps - 1) / kStateSteps; }

}  // namespace
}  // namespace rnnt

using namespace rnnt;

extern "C" {

size_t rnnt_recurrence_states_bytes(rnnt_recurrence_shape_t shape) {
  if (check(shape) != RNNT_OK) return 0;
  return static_cast<size_t>(shape.B) * state_count(shape.L) * shape.D * sizeof(float);
}

size_t rnnt_recurrence_workspace_bytes(rnnt_recurrence_shape_t shape) { return check(shape) == RNNT_OK ? 256 : 0; }

rnnt_status_t rnnt_recurrence(const void* x, const void* z, rnnt_recurrence_shape_t shape, const int32_t* lens,
                              const float* h0, void* h_out, float* last_out, void* states_out, void* workspace,
                              size_t workspace_bytes, hipStream_t stream) {
  rnnt_status_t st = check(shape);
  if (st != RNNT_OK) return st;
  if (!last_out || (shape.L > 0 && (!x || !z || !h_out))) return RNNT_ERR_NULL_PTR;
  const int64_t e = net_elem_bytes(shape.dtype);
  if (!multiple_of(e, x) || !multiple_of(e, z) || !multiple_of(e, h_out) || !multiple_of(4, h0) ||
      !multiple_of(4, last_out) || !multiple_of(16, states_out))
    return RNNT_ERR_ALIGNMENT;
  NetWorkspace ws;
  st = ws.take(workspace, workspace_bytes, rnnt_recurrence_workspace_bytes(shape), stream);
  if (st != RNNT_OK) return st;
  RecurrenceParams p{x, z, shape.x_stride_b, shape.x_stride_t, shape.z_stride_b, shape.z_stride_t, lens, h0, h_out,
                     last_out, static_cast<float*>(states_out), shape.B, shape.L, shape.D, state_count(shape.L)};
  return with_dtype(shape.dtype, [&](auto t) {
    using T = decltype(t);
    hipLaunchKernelGGL((net_recurrence<T>), dim3((shape.D + 63) / 64, shape.B), dim3(64), 0, stream, p);
    return launched();
  });
}

rnnt_status_t rnnt_recurrence_grad(const void* x, const void* z, rnnt_recurrence_shape_t shape, const int32_t* lens,
                                   const void* states, const void* dh, const float* dlast, void* dx, void* dz,
                                   float* dh0, void* workspace, size_t workspace_bytes, hipStream_t stream) {
  rnnt_status_t st = check(shape);
  if (st != RNNT_OK) return st;
  if (shape.L > 0 && (!x || !z || !states || !dx || !dz)) return RNNT_ERR_NULL_PTR;
  const int64_t e = net_elem_bytes(shape.dtype);
  if (!multiple_of(e, x) || !multiple_of(e, z) || !multiple_of(e, dh) || !multiple_of(e, dx) || !multiple_of(e, dz) ||
      !multiple_of(4, dlast) || !multiple_of(4, dh0) || !multiple_of(16, states))
    return RNNT_ERR_ALIGNMENT;
  NetWorkspace ws;
  st = ws.take(workspace, workspace_bytes, rnnt_recurrence_workspace_bytes(shape), stream);
  if (st != RNNT_OK) return st;
  RecurrenceGradParams p{x, z, shape.x_stride_b, shape.x_stride_t, shape.z_stride_b, shape.z_stride_t, lens,
                         static_cast<const float*>(states), dh, dlast, dx, dz, dh0, shape.B, shape.L, shape.D,
                         state_count(shape.L)};
  return with_dtype(shape.dtype, [&](auto t) {
    using T = decltype(t);
    hipLaunchKernelGGL((net_recurrence_grad<T>), dim3((shape.D + 63) / 64, shape.B), dim3(64), 0, stream, p);
    return launched();
  });
}

}  // extern "C"
