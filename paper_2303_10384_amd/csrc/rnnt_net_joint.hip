// Dropout and the joint's hidden layer with its gradient (contract in include/rnnt_network_mi355x.h).
#include <hip/hip_runtime.h>

#include <cstdint>

#include "rnnt_net.h"

namespace rnnt {
namespace {

struct DropoutParams {
  const void* x;
  void* y;
  int64_t n;
  DropParams drop;
  int64_t* rng_out;
};

__device__ __forceinline__ void copy_rng(const int64_t* from, int64_t* to) {
  if (to && from && blockIdx.x == 0 && blockIdx.y == 0 && threadIdx.x < 2) to[threadIdx.x] = from[threadIdx.x];
}

// One thread to a block of eight elements.
template <typename T, bool WIDE>
__global__ __launch_bounds__(256) void net_dropout(DropoutParams p) {
  copy_rng(p.drop.rng, p.rng_out);
  const int64_t block = static_cast<int64_t>(blockIdx.x) * 256 + threadIdx.x, n0 = block * 8;
  if (n0 >= p.n) return;
  uint4 bits = make_uint4(0, 0, 0, 0);
  if (p.drop.threshold) bits = random_block(load_rng(p.drop.rng), static_cast<uint64_t>(block));
  const T* x = static_cast<const T*>(p.x) + n0;
  T* y = static_cast<T*>(p.y) + n0;
  auto one = [&](float v, int j) { return random16(bits, j) >= p.drop.threshold ? v * p.drop.scale : 0.f; };
  if (WIDE && n0 + 8 <= p.n) {
    Pack<T, 8> k;
    float f[8];
    k.load(x);
    k.get(f);
#pragma unroll
    for (int j = 0; j < 8; ++j) f[j] = one(f[j], j);
    k.set(f);
    k.store(y);
  } else {
#pragma unroll
    for (int j = 0; j < 8; ++j)
      if (n0 + j < p.n) ElemTraits<T>::store1(y + j, one(ElemTraits<T>::load1(x + j), j));
  }
}

struct JointParams {
  const void *enc, *pred;
  const int32_t *logit_lens, *label_lens;
  void* h;
  DropParams drop;
  int64_t* rng_out;
  int64_t n;  // elements of h
  int32_t B, T, U1, H;
};

// One thread to eight consecutive elements of h, which may lie in several rows.
template <typename T, int ACT>
__global__ __launch_bounds__(256) void net_joint(JointParams p) {
  copy_rng(p.drop.rng, p.rng_out);
  const int64_t block = static_cast<int64_t>(blockIdx.x) * 256 + threadIdx.x, n0 = block * 8;
  if (n0 >= p.n) return;
  uint4 bits = make_uint4(0, 0, 0, 0);
  if (p.drop.threshold) bits = random_block(load_rng(p.drop.rng), static_cast<uint64_t>(block));
  int64_t row = n0 / p.H;
  int c = static_cast<int>(n0 - row * p.H);
#pragma unroll 1
  for (int j = 0; j < 8 && n0 + j < p.n; ++j) {
    const int u = static_cast<int>(row % p.U1);
    const int64_t bt = row / p.U1;
    const int t = static_cast<int>(bt % p.T), b = static_cast<int>(bt / p.T);
    const int tl = p.logit_lens[b], ul = p.label_lens[b];
    float v = 0.f;
    if (tl < 0 || tl > p.T || ul < 0 || ul >= p.U1) {
      v = __builtin_nanf("");
    } else if (t < tl && u <= ul) {
      const float s = ElemTraits<T>::load1(static_cast<const T*>(p.enc) + bt * p.H + c) +
                      ElemTraits<T>::load1(static_cast<const T*>(p.pred) + (static_cast<int64_t>(b) * p.U1 + u) * p.H + c);
      v = random16(bits, j) >= p.drop.threshold ? Activation<ACT>::value(s) * p.drop.scale : 0.f;
    }
    ElemTraits<T>::store1(static_cast<T*>(p.h) + n0 + j, v);
    if (++c == p.H) {
      c = 0;
      ++row;
    }
  }
}

struct JointGradParams {
  const void *enc, *pred, *dh;
  const int32_t *logit_lens, *label_lens;
  void *denc, *dpred;
  DropParams drop;
  int32_t B, T, U1, H;
};

// One block to a row of one of the two gradients, one thread to a channel.
template <typename T, int ACT>
__global__ __launch_bounds__(256) void net_joint_grad(JointGradParams p, bool of_enc) {
  const int rows = of_enc ? p.T : p.U1, others = of_enc ? p.U1 : p.T;
  const int b = static_cast<int>(blockIdx.x) / rows, r = static_cast<int>(blockIdx.x) % rows;
  const int tl = p.logit_lens[b], ul = p.label_lens[b];
  const bool ok = tl >= 0 && tl <= p.T && ul >= 0 && ul < p.U1;
  const int live = !ok ? 0 : of_enc ? (r < tl ? ul + 1 : 0) : (r <= ul ? tl : 0);
  Rng rng{};
  if (p.drop.threshold) rng = load_rng(p.drop.rng);
  for (int c = threadIdx.x; c < p.H; c += 256) {
    float sum = 0.f;
    for (int o = 0; o < live && o < others; ++o) {
      const int t = of_enc ? r : o, u = of_enc ? o : r;
      const int64_t bt = static_cast<int64_t>(b) * p.T + t, n = (bt * p.U1 + u) * p.H + c;
      const float s = ElemTraits<T>::load1(static_cast<const T*>(p.enc) + bt * p.H + c) +
                      ElemTraits<T>::load1(static_cast<const T*>(p.pred) + (static_cast<int64_t>(b) * p.U1 + u) * p.H + c);
      bool keep = true;
      if (p.drop.threshold)
        keep = random16(random_block(rng, static_cast<uint64_t>(n >> 3)), static_cast<int>(n & 7)) >= p.drop.threshold;
      const float d = ElemTraits<T>::load1(static_cast<const T*>(p.dh) + n);
      const float slope = Activation<ACT>::slope(s);
      if (keep && (ACT == RNNT_ACT_TANH || slope != 0.f)) sum += d * p.drop.scale * slope;
    }
    T* out = static_cast<T*>(of_enc ? p.denc : p.dpred) + (static_cast<int64_t>(b) * rows + r) * p.H + c;
    ElemTraits<T>::store1(out, sum);
  }
}

rnnt_status_t check(const rnnt_joint_shape_t& s, rnnt_activation_t act, double p, const int64_t* rng,
                    DropParams* drop) {
  if (s.B < 1 || s.T_max < 1 || s.U_max < 0 || s.H < 1) return RNNT_ERR_BAD_SHAPE;
  const int64_t rows = static_cast<int64_t>(s.T_max) * (static_cast<int64_t>(s.U_max) + 1);
  if (rows > kMaxRows || s.B > (int64_t{1} << 40) / rows || s.H > (1 << 20)) return RNNT_ERR_BAD_SHAPE;
  if (!net_dtype_known(s.dtype)) return RNNT_ERR_BAD_DTYPE;
  if (act != RNNT_ACT_RELU && act != RNNT_ACT_TANH) return RNNT_ERR_BAD_VARIANT;
  if (!drop_params(p, rng, drop)) return RNNT_ERR_BAD_VARIANT;
  if (drop->threshold && !rng) return RNNT_ERR_NULL_PTR;
  if (static_cast<int64_t>(s.B) * s.T_max > kMaxRows || static_cast<int64_t>(s.B) * (s.U_max + 1) > kMaxRows)
    return RNNT_ERR_UNSUPPORTED;
  return RNNT_OK;
}

template <typename F>
rnnt_status_t with_activation(rnnt_activation_t act, F&& f) {
  if (act == RNNT_ACT_TANH) return f(std::integral_constant<int, RNNT_ACT_TANH>{});
  return f(std::integral_constant<int, RNNT_ACT_RELU>{});
}

}  // namespace
}  // namespace rnnt

using namespace rnnt;

extern "C" {

rnnt_status_t rnnt_dropout(const void* x, int64_t n, rnnt_dtype_t dtype, double p, const int64_t* rng,
                           int64_t* rng_out, void* y, hipStream_t stream) {
  DropoutParams q{};
  if (n < 0) return RNNT_ERR_BAD_SHAPE;
  if (!net_dtype_known(dtype)) return RNNT_ERR_BAD_DTYPE;
  if (!drop_params(p, rng, &q.drop)) return RNNT_ERR_BAD_VARIANT;
  if (!rng || (n > 0 && (!x || !y))) return RNNT_ERR_NULL_PTR;
  const int64_t e = net_elem_bytes(dtype);
  if (!multiple_of(e, x) || !multiple_of(e, y) || !multiple_of(8, rng) || !multiple_of(8, rng_out))
    return RNNT_ERR_ALIGNMENT;
  q.x = x;
  q.y = y;
  q.n = n;
  q.rng_out = rng_out;
  const int64_t blocks = n / 2048 + 1;
  if (blocks > kMaxRows / 256) return RNNT_ERR_UNSUPPORTED;
  const bool wide = multiple_of(16, x) && multiple_of(16, y);
  return with_dtype(dtype, [&](auto t) {
    using T = decltype(t);
    const dim3 grid(static_cast<uint32_t>(blocks));
    if (wide) hipLaunchKernelGGL((net_dropout<T, true>), grid, dim3(256), 0, stream, q);
    else hipLaunchKernelGGL((net_dropout<T, false>), grid, dim3(256), 0, stream, q);
    return launched();
  });
}

rnnt_status_t rnnt_joint_hidden(const void* enc, const void* pred, rnnt_joint_shape_t shape,
                                const int32_t* logit_lens, const int32_t* label_lens, rnnt_activation_t act, double p,
                                const int64_t* rng, int64_t* rng_out, void* h_out, hipStream_t stream) {
  JointParams q{};
  const rnnt_status_t st = check(shape, act, p, rng, &q.drop);
  if (st != RNNT_OK) return st;
  if (!enc || !pred || !logit_lens || !label_lens || !h_out) return RNNT_ERR_NULL_PTR;
  const int64_t e = net_elem_bytes(shape.dtype);
  if (!multiple_of(e, enc) || !multiple_of(e, pred) || !multiple_of(e, h_out) || !multiple_of(8, rng) ||
      !multiple_of(8, rng_out))
    return RNNT_ERR_ALIGNMENT;
  q.enc = enc;
  q.pred = pred;
  q.logit_lens = logit_lens;
  q.label_lens = label_lens;
  q.h = h_out;
  q.rng_out = rng_out;
  q.B = shape.B;
  q.T = shape.T_max;
  q.U1 = shape.U_max + 1;
  q.H = shape.H;
  q.n = static_cast<int64_t>(shape.B) * shape.T_max * q.U1 * shape.H;
  const int64_t blocks = (q.n + 2047) / 2048;
  if (blocks > kMaxRows / 256) return RNNT_ERR_UNSUPPORTED;
  return with_dtype(shape.dtype, [&](auto t) {
    return with_activation(act, [&](auto a) {
      hipLaunchKernelGGL((net_joint<decltype(t), decltype(a)::value>), dim3(static_cast<uint32_t>(blocks)), dim3(256),
                         0, stream, q);
      return launched();
    });
  });
}

size_t rnnt_joint_hidden_grad_workspace_bytes(rnnt_joint_shape_t shape) {
  DropParams drop;
  return check(shape, RNNT_ACT_RELU, 0.0, nullptr, &drop) == RNNT_OK ? 256 : 0;
}

rnnt_status_t rnnt_joint_hidden_grad(const void* enc, const void* pred, rnnt_joint_shape_t shape,
                                     const int32_t* logit_lens, const int32_t* label_lens, rnnt_activation_t act,
                                     double p, const int64_t* rng, const void* dh, void* denc, void* dpred,
                                     void* workspace, size_t workspace_bytes, hipStream_t stream) {
  JointGradParams q{};
  rnnt_status_t st = check(shape, act, p, rng, &q.drop);
  if (st != RNNT_OK) return st;
  if (!enc || !pred || !logit_lens || !label_lens || !dh || !denc || !dpred) return RNNT_ERR_NULL_PTR;
  const int64_t e = net_elem_bytes(shape.dtype);
  if (!multiple_of(e, enc) || !multiple_of(e, pred) || !multiple_of(e, dh) || !multiple_of(e, denc) ||
      !multiple_of(e, dpred) || !multiple_of(8, rng))
    return RNNT_ERR_ALIGNMENT;
  NetWorkspace ws;
  st = ws.take(workspace, workspace_bytes, rnnt_joint_hidden_grad_workspace_bytes(shape), stream);
  if (st != RNNT_OK) return st;
  q.enc = enc;
  q.pred = pred;
  q.dh = dh;
  q.logit_lens = logit_lens;
  q.label_lens = label_lens;
  q.denc = denc;
  q.dpred = dpred;
  q.B = shape.B;
  q.T = shape.T_max;
  q.U1 = shape.U_max + 1;
  q.H = shape.H;
  return with_dtype(shape.dtype, [&](auto t) {
    return with_activation(act, [&](auto a) {
      using K = decltype(t);
      constexpr int A = decltype(a)::value;
      hipLaunchKernelGGL((net_joint_grad<K, A>), dim3(shape.B * q.T), dim3(256), 0, stream, q, true);
      if (launched() != RNNT_OK) return RNNT_ERR_HIP;
      hipLaunchKernelGGL((net_joint_grad<K, A>), dim3(shape.B * q.U1), dim3(256), 0, stream, q, false);
      return launched();
    });
  });
}

}  // extern "C"
