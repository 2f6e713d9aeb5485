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

__device__ __forceinline__ void dropped_of(const DropParams& d, const Rng& rng, uint64_t block, Dropped& out) {
  if (d.threshold) out.below(random_block(rng, block), d.threshold);
  else out.none();
}

// One thread to a block of eight elements.
template <typename T>
__global__ __launch_bounds__(256) void net_dropout(DropoutParams p) {
  copy_rng(p.drop.rng, p.rng_out);
  const int64_t block = static_cast<int64_t>(blockIdx.x) * 256 + threadIdx.x, n0 = block * 8;
  if (n0 >= p.n) return;
  const T* x = static_cast<const T*>(p.x) + n0;
  T* y = static_cast<T*>(p.y) + n0;
  Pack<T, 8> k;
  const bool whole = n0 + 8 <= p.n;
  if (whole) k.load(x);
  else k.load_part(x, static_cast<int>(p.n - n0));
  Dropped drop;
  dropped_of(p.drop, load_rng(p.drop.rng), static_cast<uint64_t>(block), drop);
  float f[8];
  k.get(f);
#pragma unroll
  for (int j = 0; j < 8; ++j) f[j] *= p.drop.scale;
  k.set(f);
  drop.clear(k);
  if (whole) k.store(y);
  else k.store_part(y, static_cast<int>(p.n - n0));
}

// ---- the joint's hidden layer -------------------------------------------------
// The rows (b, t, 0 .. U) are one run of U1 * H elements, in which element j is
// act(enc[b, t, j % H] + pred[b].flat[j]): no division but the first, pred is read along with h, and the
// valid rows are the run's first (U_b + 1) H elements.

struct JointParams {
  const void *enc, *pred;
  const int32_t *logit_lens, *label_lens;
  void* h;
  DropParams drop;
  int64_t* rng_out;
  int32_t B, T, U1, H, t_blocks;
};

constexpr int kJointFrames = 4;    // frames of a block of net_joint: pred is read once for all of them
constexpr int kJointRun = 8;       // groups of eight elements to a thread and frame
constexpr int kJointLdsH = 4096;   // widest row that net_joint_odd keeps in LDS

template <typename T, int ACT>
__device__ __forceinline__ void joint_group(const float* e, const float* q, float scale, const Dropped& drop, Pack<T, 8>& out) {
  float f[8];
#pragma unroll
  for (int i = 0; i < 8; ++i) f[i] = Activation<ACT>::value(e[i] + q[i]) * scale;
  out.set(f);
  drop.clear(out);
}

// Elements of a run valid at frame t (-1: a bad length).
__device__ __forceinline__ int64_t joint_valid(const JointParams& p, int b, int t) {
  const int tl = p.logit_lens[b], ul = p.label_lens[b];
  if (tl < 0 || tl > p.T || ul < 0 || ul >= p.U1) return -1;
  return t < tl ? static_cast<int64_t>(ul + 1) * p.H : 0;
}

template <typename T>
__device__ __forceinline__ Pack<T, 8> nan_group() {
  float f[8];
#pragma unroll
  for (int i = 0; i < 8; ++i) f[i] = __builtin_nanf("");
  Pack<T, 8> k;
  k.set(f);
  return k;
}

// H a multiple of eight: groups lie in one row, and at the same place of the run for every frame.
template <typename T, int ACT>
__global__ __launch_bounds__(256) void net_joint(JointParams p) {
  copy_rng(p.drop.rng, p.rng_out);
  const int b = static_cast<int>(blockIdx.x) / p.t_blocks, t0 = static_cast<int>(blockIdx.x) % p.t_blocks * kJointFrames;
  const int64_t total = static_cast<int64_t>(p.U1) * p.H;
  int64_t j = (static_cast<int64_t>(blockIdx.y) * kJointRun * 256 + threadIdx.x) * 8;
  int col = static_cast<int>(j % p.H);
  const int col_step = 2048 % p.H;
  const int64_t valid0 = joint_valid(p, b, t0);
  const int frames = min(kJointFrames, p.T - t0);
  const int tl = valid0 < 0 ? 0 : p.logit_lens[b];
  const int64_t valid = valid0 < 0 ? 0 : static_cast<int64_t>(p.label_lens[b] + 1) * p.H;
  Rng rng{};
  if (p.drop.threshold) rng = load_rng(p.drop.rng);
  const T* enc = static_cast<const T*>(p.enc) + (static_cast<int64_t>(b) * p.T + t0) * p.H;
  const T* pred = static_cast<const T*>(p.pred) + b * total;
  const int64_t run0 = (static_cast<int64_t>(b) * p.T + t0) * total;
  T* h = static_cast<T*>(p.h) + run0;
  for (int it = 0; it < kJointRun && j < total; ++it, j += 2048) {
    float q[8];
    Pack<T, 8> k;
    if (j < valid && t0 < tl) {
      k.load(pred + j);
      k.get(q);
    }
#pragma unroll
    for (int i = 0; i < kJointFrames; ++i) {
      if (i < frames) {
        if (valid0 < 0) {
          k = nan_group<T>();
        } else if (j < valid && t0 + i < tl) {
          float e[8];
          k.load(enc + i * p.H + col);
          k.get(e);
          Dropped drop;
          dropped_of(p.drop, rng, static_cast<uint64_t>(run0 + i * total + j) >> 3, drop);
          joint_group<T, ACT>(e, q, p.drop.scale, drop, k);
        } else {
          k.zero();
        }
        k.store(h + i * total + j);
      }
    }
    col += col_step;
    if (col >= p.H) col -= p.H;
  }
}

// Any H: one frame to a block; groups are multiples of eight in h, where the random numbers are, so a
// group may begin in one row of the run and end in the next (the frame's row, continued by its first
// eight elements, is in LDS while it fits), and the run's first and last group may be partial.
template <typename T, int ACT, bool IN_LDS>
__global__ __launch_bounds__(256) void net_joint_odd(JointParams p) {
  copy_rng(p.drop.rng, p.rng_out);
  __shared__ float row[IN_LDS ? kJointLdsH + 8 : 1];
  const int b = static_cast<int>(blockIdx.x) / p.T, t = static_cast<int>(blockIdx.x) % p.T;
  const int64_t total = static_cast<int64_t>(p.U1) * p.H, run0 = static_cast<int64_t>(blockIdx.x) * total;
  const int64_t valid = joint_valid(p, b, t);
  const T* enc = static_cast<const T*>(p.enc) + static_cast<int64_t>(blockIdx.x) * p.H;
  const T* pred = static_cast<const T*>(p.pred) + b * total;
  T* h = static_cast<T*>(p.h) + run0;
  Rng rng{};
  if (p.drop.threshold) rng = load_rng(p.drop.rng);
  if (IN_LDS && valid > 0) {
    for (int c = threadIdx.x; c < p.H + 8; c += 256) row[c] = ElemTraits<T>::load1(enc + c % p.H);
    __syncthreads();
  }
  int64_t j = (static_cast<int64_t>(blockIdx.y) * kJointRun * 256 + threadIdx.x) * 8 - (run0 & 7);
  int col = static_cast<int>((j + p.H * static_cast<int64_t>(8)) % p.H);  // j > -8
  const int col_step = 2048 % p.H;
  for (int it = 0; it < kJointRun && j < total; ++it, j += 2048) {
    Pack<T, 8> k;
    if (valid < 0) {
      k = nan_group<T>();
    } else if (j >= valid) {
      k.zero();
    } else {
      float e[8], q[8];
      const int first = j < 0 ? static_cast<int>(-j) : 0;
      if (first == 0 && j + 8 <= total) k.load(pred + j);
      else k.zero();
      k.get(q);
      if (first > 0 || j + 8 > total) {
#pragma unroll
        for (int i = 0; i < 8; ++i)
          if (i >= first && j + i < total) q[i] = ElemTraits<T>::load1(pred + j + i);
      }
      if (IN_LDS) {
#pragma unroll
        for (int i = 0; i < 8; ++i) e[i] = row[col + i];
      } else if (col + 8 <= p.H) {
        k.load(enc + col);
        k.get(e);
      } else {
#pragma unroll
        for (int i = 0; i < 8; ++i) e[i] = ElemTraits<T>::load1(enc + (col + i) % p.H);
      }
      Dropped drop;
      dropped_of(p.drop, rng, static_cast<uint64_t>(run0 + j) >> 3, drop);
      joint_group<T, ACT>(e, q, p.drop.scale, drop, k);
      if (j + 8 > valid) {  // the valid rows end inside the group
#pragma unroll
        for (int i = 0; i < 8; ++i) {
          if (j + i >= valid) {
            if constexpr (sizeof(T) == 4) k.w[i] = 0;
            else k.w[i / 2] &= (i & 1) ? 0x0000ffffu : 0xffff0000u;
          }
        }
      }
    }
    if (j >= 0 && j + 8 <= total) {
      k.store(h + j);
    } else {
#pragma unroll
      for (int i = 0; i < 8; ++i) {
        if (j + i >= 0 && j + i < total) {
          if constexpr (sizeof(T) == 4) *reinterpret_cast<uint32_t*>(h + j + i) = k.w[i];
          else *reinterpret_cast<uint16_t*>(h + j + i) = static_cast<uint16_t>(k.w[i / 2] >> (16 * (i & 1)));
        }
      }
    }
    col += col_step;
    if (col >= p.H) col -= p.H;
  }
}

// ---- its gradient -------------------------------------------------------------
// A block takes kTileT frames of an utterance and a slice of channels, and goes over the units: dh is read
// once.  A wave holds the sums over u of its eight frames in registers (denc is finished in the block);
// the sums over its frames meet in LDS, and the block's go to the workspace, one float32 row for kTileT rows
// of dh (a sixteenth of a bfloat16 dh at 32), which net_joint_join adds up in the order of the frames.

struct JointGradParams {
  const void *enc, *pred, *dh;
  const int32_t *logit_lens, *label_lens;
  void *denc, *dpred;
  float* part;  // (B, t_blocks, U1, H)
  DropParams drop;
  int32_t B, T, U1, H, t_blocks, slices, lanes;  // lanes: of a row, eight channels each (4, 8 or 16)
};

constexpr int kWaveT = 8;                     // frames of a wave
constexpr int kGradWaves = 4;
constexpr int kTileT = kWaveT * kGradWaves;   // frames of a block

template <typename T>
__device__ __forceinline__ void load_row(Pack<T, 8>& k, const T* p, int n) {  // n: channels left in the row
  if (n >= 8) k.load(p);
  else k.load_part(p, n);
}

template <typename T, int ACT, bool EIGHTS>
__global__ __launch_bounds__(64 * kGradWaves) void net_joint_grad(JointGradParams p) {
  __shared__ __attribute__((aligned(16))) float sums[2][kGradWaves][512];
  const int slice = static_cast<int>(blockIdx.x) % p.slices, bt = static_cast<int>(blockIdx.x) / p.slices;
  const int tb = bt % p.t_blocks, b = bt / p.t_blocks;
  const int wave = static_cast<int>(threadIdx.x) >> 6, lane = static_cast<int>(threadIdx.x) & 63;
  const int sub = lane / p.lanes, rows = 64 / p.lanes;
  const int c = (slice * p.lanes + (lane & (p.lanes - 1))) * 8;
  const int left = p.H - c;  // channels of this lane: min(left, 8), none when it is not positive
  int tl = p.logit_lens[b], ul = p.label_lens[b];
  if (tl < 0 || tl > p.T || ul < 0 || ul >= p.U1) tl = 0;
  const int t0 = tb * kTileT + wave * kWaveT;
  const int frames = max(0, min(kWaveT, tl - t0));
  T* denc = static_cast<T*>(p.denc) + (static_cast<int64_t>(b) * p.T + t0) * p.H + c;
  const int64_t run0 = (static_cast<int64_t>(b) * p.T + t0) * p.U1;  // row (t0, 0)
  float acc[kWaveT][8];
#pragma unroll
  for (int i = 0; i < kWaveT; ++i)
#pragma unroll
    for (int k = 0; k < 8; ++k) acc[i][k] = 0.f;

  if (tb * kTileT < tl) {
    const T* enc = static_cast<const T*>(p.enc) + (static_cast<int64_t>(b) * p.T + t0) * p.H + c;
    const T* pred = static_cast<const T*>(p.pred) + static_cast<int64_t>(b) * p.U1 * p.H + c;
    const T* dh = static_cast<const T*>(p.dh) + run0 * p.H + c;
    float* part = p.part + (static_cast<int64_t>(b) * p.t_blocks + tb) * p.U1 * p.H;
    Rng rng{};
    if (p.drop.threshold) rng = load_rng(p.drop.rng);
    Pack<T, 8> e[kWaveT];
#pragma unroll
    for (int i = 0; i < kWaveT; ++i) {
      e[i].zero();
      if (i < frames && left > 0) load_row(e[i], enc + static_cast<int64_t>(i) * p.H, left);
    }
    int buf = 0;
    for (int u0 = 0; u0 <= ul; u0 += rows, buf ^= 1) {
      const int u = u0 + sub;
      const bool live = u <= ul && left > 0;
      float ps[8] = {};
      if (live) {
        Pack<T, 8> q, d[kWaveT];
#pragma unroll
        for (int i = 0; i < kWaveT; ++i)
          if (i < frames) load_row(d[i], dh + (static_cast<int64_t>(i) * p.U1 + u) * p.H, left);
        load_row(q, pred + static_cast<int64_t>(u) * p.H, left);
        float qf[8];
        q.get(qf);
#pragma unroll
        for (int i = 0; i < kWaveT; ++i) {
          if (i < frames) {
            if (p.drop.threshold) {
              const uint64_t n = static_cast<uint64_t>((run0 + static_cast<int64_t>(i) * p.U1 + u) * p.H + c);
              Dropped drop;
              drop.below(random_block(rng, n >> 3), p.drop.threshold);
              if (!EIGHTS) {
                Dropped next;
                next.below(random_block(rng, (n >> 3) + 1), p.drop.threshold);
                drop.shift(next, static_cast<int>(n & 7));
              }
              drop.clear(d[i]);
            }
            float ef[8], w[8];
            e[i].get(ef);
            d[i].get(w);
#pragma unroll
            for (int k = 0; k < 8; ++k) {
              const float s = ef[k] + qf[k];
              if (ACT == RNNT_ACT_RELU) w[k] = s > 0.f ? w[k] : 0.f;
              else w[k] *= Activation<ACT>::slope(s);
              acc[i][k] += w[k];
              ps[k] += w[k];
            }
          }
        }
      }
      float4* mine = reinterpret_cast<float4*>(sums[buf][wave]);
      mine[lane] = make_float4(ps[0], ps[1], ps[2], ps[3]);
      mine[64 + lane] = make_float4(ps[4], ps[5], ps[6], ps[7]);
      __syncthreads();  // one to a step: the other buffer is written before the next
      const int at = static_cast<int>(threadIdx.x), from = (at >> 1) & 63;
      float2 total = make_float2(0.f, 0.f);
#pragma unroll
      for (int w = 0; w < kGradWaves; ++w) {
        const float2 v = reinterpret_cast<const float2*>(sums[buf][w])[at];
        total.x += v.x;
        total.y += v.y;
      }
      const int pu = u0 + from / p.lanes;
      const int pc = (slice * p.lanes + (from & (p.lanes - 1))) * 8 + (at >> 7) * 4 + (at & 1) * 2;
      if (pu <= ul) {
        float* o = part + static_cast<int64_t>(pu) * p.H + pc;
        if (pc < p.H) o[0] = total.x;
        if (pc + 1 < p.H) o[1] = total.y;
      }
    }
    // the rows of u that the wave's lanes shared out
    for (int off = p.lanes; off < 64; off <<= 1) {
#pragma unroll
      for (int i = 0; i < kWaveT; ++i)
#pragma unroll
        for (int k = 0; k < 8; ++k) acc[i][k] += __shfl_xor(acc[i][k], off);
    }
  }
  if (sub == 0 && left > 0) {
#pragma unroll
    for (int i = 0; i < kWaveT; ++i) {
      if (t0 + i < p.T) {
        float f[8];
#pragma unroll
        for (int k = 0; k < 8; ++k) f[k] = acc[i][k] * p.drop.scale;
        Pack<T, 8> k;
        k.set(f);
        if (left >= 8) k.store(denc + static_cast<int64_t>(i) * p.H);
        else k.store_part(denc + static_cast<int64_t>(i) * p.H, left);
      }
    }
  }
}

__device__ __forceinline__ void load_row4(Pack<float, 4>& k, const float* p, int n) {
  if (n >= 4) k.load(p);
  else k.load_part(p, n);
}

// dpred from the blocks' sums: four channels to a thread.
template <typename T>
__global__ __launch_bounds__(256) void net_joint_join(JointGradParams p) {
  const int groups = (p.H + 3) / 4;
  const int64_t at = static_cast<int64_t>(blockIdx.x) * 256 + threadIdx.x;
  const int64_t row = at / groups;
  if (row >= static_cast<int64_t>(p.B) * p.U1) return;
  const int c = static_cast<int>(at - row * groups) * 4, left = p.H - c;
  const int b = static_cast<int>(row / p.U1), u = static_cast<int>(row - static_cast<int64_t>(b) * p.U1);
  const int tl = p.logit_lens[b], ul = p.label_lens[b];
  float f[4] = {};
  if (tl >= 0 && tl <= p.T && ul < p.U1 && u <= ul) {
    const int n = (tl + kTileT - 1) / kTileT;
    const float* part = p.part + (static_cast<int64_t>(b) * p.t_blocks * p.U1 + u) * p.H + c;
    const int64_t step = static_cast<int64_t>(p.U1) * p.H;
#pragma unroll 4
    for (int i = 0; i < n; ++i) {
      Pack<float, 4> k;
      load_row4(k, part + i * step, left);
#pragma unroll
      for (int j = 0; j < 4; ++j) f[j] += __uint_as_float(k.w[j]);
    }
  }
#pragma unroll
  for (int j = 0; j < 4; ++j) f[j] *= p.drop.scale;
  Pack<T, 4> k;
  k.set(f);
  T* o = static_cast<T*>(p.dpred) + row * p.H + c;
  if (left >= 4) k.store(o);
  else k.store_part(o, left);
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

int tile_count(int T) { return static_cast<int>((static_cast<int64_t>(T) + kTileT - 1) / kTileT); }

size_t grad_bytes(const rnnt_joint_shape_t& s) {
  return net_align256(static_cast<size_t>(s.B) * tile_count(s.T_max) * (static_cast<size_t>(s.U_max) + 1) * s.H * sizeof(float));
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
  return with_dtype(dtype, [&](auto t) {
    hipLaunchKernelGGL((net_dropout<decltype(t)>), dim3(static_cast<uint32_t>(blocks)), dim3(256), 0, stream, q);
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
  const bool eights = shape.H % 8 == 0;
  q.t_blocks = eights ? (shape.T_max + kJointFrames - 1) / kJointFrames : shape.T_max;
  const int64_t groups = (static_cast<int64_t>(q.U1) * shape.H + 7) / 8 + (eights ? 0 : 1);
  const int64_t x = static_cast<int64_t>(shape.B) * q.t_blocks, y = (groups + 256 * kJointRun - 1) / (256 * kJointRun);
  if (x > kMaxRows / 256 || y > 65535) return RNNT_ERR_UNSUPPORTED;
  const dim3 grid(static_cast<uint32_t>(x), static_cast<uint32_t>(y));
  return with_dtype(shape.dtype, [&](auto t) {
    return with_activation(act, [&](auto a) {
      using T = decltype(t);
      constexpr int A = decltype(a)::value;
      if (eights) hipLaunchKernelGGL((net_joint<T, A>), grid, dim3(256), 0, stream, q);
      else if (shape.H <= kJointLdsH) hipLaunchKernelGGL((net_joint_odd<T, A, true>), grid, dim3(256), 0, stream, q);
      else hipLaunchKernelGGL((net_joint_odd<T, A, false>), grid, dim3(256), 0, stream, q);
      return launched();
    });
  });
}

size_t rnnt_joint_hidden_grad_workspace_bytes(rnnt_joint_shape_t shape) {
  DropParams drop;
  return check(shape, RNNT_ACT_RELU, 0.0, nullptr, &drop) == RNNT_OK ? grad_bytes(shape) : 0;
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
  q.part = reinterpret_cast<float*>(ws.ptr);
  q.t_blocks = tile_count(shape.T_max);
  q.lanes = shape.H <= 32 ? 4 : shape.H <= 64 ? 8 : 16;
  q.slices = (shape.H + 8 * q.lanes - 1) / (8 * q.lanes);
  const int64_t x = static_cast<int64_t>(shape.B) * q.t_blocks * q.slices;
  const int64_t joins = (static_cast<int64_t>(shape.B) * q.U1 * ((shape.H + 3) / 4) + 255) / 256;
  if (x > kMaxRows / 256 || joins > kMaxRows / 256) return RNNT_ERR_UNSUPPORTED;
  return with_dtype(shape.dtype, [&](auto t) {
    using T = decltype(t);
    const rnnt_status_t done = with_activation(act, [&](auto a) {
      constexpr int A = decltype(a)::value;
      const dim3 grid(static_cast<uint32_t>(x)), block(64 * kGradWaves);
      if (shape.H % 8 == 0) hipLaunchKernelGGL((net_joint_grad<T, A, true>), grid, block, 0, stream, q);
      else hipLaunchKernelGGL((net_joint_grad<T, A, false>), grid, block, 0, stream, q);
      return launched();
    });
    if (done != RNNT_OK) return done;
    hipLaunchKernelGGL((net_joint_join<T>), dim3(static_cast<uint32_t>(joins)), dim3(256), 0, stream, q);
    return launched();
  });
}

}  // extern "C"
