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
  const bool whole = n0 + 8 <= p.n, pair = (block | 1) * 8 + 8 <= p.n;  // the neighbour's group too
  if (pair) load_pair(k, x);
  else if (whole) k.load(x);
  else k.load_part(x, static_cast<int>(p.n - n0));
  Dropped drop;
  dropped_of(p.drop, load_rng(p.drop.rng), static_cast<uint64_t>(block), drop);
  float f[8];
  k.get(f);
#pragma unroll
  for (int j = 0; j < 8; ++j) f[j] *= p.drop.scale;
  k.set(f);
  drop.clear(k);
  if (pair) store_pair(k, y);
  else if (whole) k.store(y);
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
  int32_t B, T, U1, H, t_blocks, block_frames;
};

constexpr int kJointFrames = 4;    // frames of a block (net_joint reads pred once for all of them)
constexpr int kJointRun = 8;       // groups of eight elements to a thread and frame
constexpr int kJointLdsBytes = 64000;  // rows that net_joint_odd keeps in LDS

template <typename T, int ACT>
__device__ __forceinline__ void joint_group(const float* e, const float* q, float scale, Pack<T, 8>& out) {
  float f[8];
#pragma unroll
  for (int i = 0; i < 8; ++i) f[i] = Activation<ACT>::template value<T>(e[i] + q[i]) * scale;
  out.set(f);
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
template <typename T, int ACT, bool DROP>
__global__ __launch_bounds__(256) void net_joint(JointParams p) {
  copy_rng(p.drop.rng, p.rng_out);
  const int b = static_cast<int>(blockIdx.x) / p.t_blocks, t0 = static_cast<int>(blockIdx.x) % p.t_blocks * p.block_frames;
  const int64_t total = static_cast<int64_t>(p.U1) * p.H;
  int64_t j = (static_cast<int64_t>(blockIdx.y) * kJointRun * 256 + threadIdx.x) * 8;
  int col = static_cast<int>(j % p.H);
  const int col_step = 2048 % p.H;
  const int64_t valid0 = joint_valid(p, b, t0);
  const int frames = min(p.block_frames, p.T - t0);
  const int tl = valid0 < 0 ? 0 : p.logit_lens[b];
  const int64_t valid = valid0 < 0 ? 0 : static_cast<int64_t>(p.label_lens[b] + 1) * p.H;
  Rng rng{};
  if constexpr (DROP) rng = load_rng(p.drop.rng);
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
          joint_group<T, ACT>(e, q, p.drop.scale, k);
          if constexpr (DROP) {
            Dropped drop;
            drop.below(random_block(rng, static_cast<uint64_t>(run0 + i * total + j) >> 3), p.drop.threshold);
            drop.clear(k);
          }
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

// Any H: groups are multiples of eight in h, where the random numbers are, so a group may begin in one row of
// the run and end in the next (the frame's row, continued by its first eight elements, is in LDS while it fits),
// and the run's first and last group may be partial.
__device__ __forceinline__ int lds_at(int c) { return c + (c >> 3); }  // lanes read eight apart: nine words, no two in a bank

template <typename T, int ACT, bool IN_LDS>
__global__ __launch_bounds__(256) void net_joint_odd(JointParams p) {
  copy_rng(p.drop.rng, p.rng_out);
  extern __shared__ float rows[];  // [block_frames][lds_at(H + 8)]
  const int b = static_cast<int>(blockIdx.x) / p.t_blocks, t0 = static_cast<int>(blockIdx.x) % p.t_blocks * p.block_frames;
  const int64_t total = static_cast<int64_t>(p.U1) * p.H;
  const int frames = min(p.block_frames, p.T - t0), pitch = lds_at(p.H + 8);
  const T* pred = static_cast<const T*>(p.pred) + b * total;
  Rng rng{};
  if (p.drop.threshold) rng = load_rng(p.drop.rng);
  if (IN_LDS) {
    const T* enc = static_cast<const T*>(p.enc) + (static_cast<int64_t>(b) * p.T + t0) * p.H;
    for (int i = 0; i < frames; ++i)
      for (int c = threadIdx.x; c < p.H + 8; c += 256)
        rows[i * pitch + lds_at(c)] = ElemTraits<T>::load1(enc + static_cast<int64_t>(i) * p.H + (c < p.H ? c : c % p.H));
    __syncthreads();
  }
  const int64_t j_block = static_cast<int64_t>(blockIdx.y) * kJointRun * 2048;
  const uint32_t col_block = static_cast<uint32_t>(j_block % p.H) + threadIdx.x * 8 + 8 * static_cast<uint32_t>(p.H);
  const int col_step = 2048 % p.H;
  for (int i = 0; i < frames; ++i) {
    const int64_t frame = static_cast<int64_t>(b) * p.T + t0 + i, run0 = frame * total;
    const int64_t valid = joint_valid(p, b, t0 + i);
    const T* enc = static_cast<const T*>(p.enc) + frame * p.H;
    T* h = static_cast<T*>(p.h) + run0;
    const int shift = static_cast<int>(run0 & 7);
    int64_t j = j_block + static_cast<int>(threadIdx.x) * 8 - shift;  // > -8
    int col = static_cast<int>((col_block - static_cast<uint32_t>(shift)) % static_cast<uint32_t>(p.H));
    for (int it = 0; it < kJointRun && j < total; ++it, j += 2048) {
      Pack<T, 8> k;
      if (j < 0 || j + 8 > total) {  // the run's first or last group, one element after the other
        Dropped drop;
        dropped_of(p.drop, rng, static_cast<uint64_t>(run0 + j) >> 3, drop);
        const uint32_t dropped = drop.bits();
        int cj = col;
#pragma unroll 1
        for (int q = 0; q < 8; ++q) {
          if (j + q >= 0 && j + q < total) {
            float v = valid < 0 ? __builtin_nanf("") : 0.f;
            if (j + q < valid && !(dropped >> q & 1u))
              v = Activation<ACT>::template value<T>(ElemTraits<T>::load1(enc + cj) + ElemTraits<T>::load1(pred + j + q)) * p.drop.scale;
            ElemTraits<T>::store1(h + j + q, v);
          }
          if (++cj == p.H) cj = 0;
        }
      } else {
        if (valid < 0) {
          k = nan_group<T>();
        } else if (j >= valid) {
          k.zero();
        } else {
          float e[8], q[8];
          k.load(pred + j);
          k.get(q);
          if (IN_LDS) {
#pragma unroll
            for (int q8 = 0; q8 < 8; ++q8) e[q8] = rows[i * pitch + lds_at(col + q8)];
          } else if (col + 8 <= p.H) {
            k.load(enc + col);
            k.get(e);
          } else {
#pragma unroll
            for (int q8 = 0; q8 < 8; ++q8) e[q8] = ElemTraits<T>::load1(enc + (col + q8) % p.H);
          }
          Dropped drop;
          dropped_of(p.drop, rng, static_cast<uint64_t>(run0 + j) >> 3, drop);
          joint_group<T, ACT>(e, q, p.drop.scale, k);
          drop.clear(k);
          if (j + 8 > valid) {  // the valid rows end inside the group
#pragma unroll
            for (int q8 = 0; q8 < 8; ++q8) {
              if (j + q8 >= valid) {
                if constexpr (sizeof(T) == 4) k.w[q8] = 0;
                else k.w[q8 / 2] &= (q8 & 1) ? 0x0000ffffu : 0xffff0000u;
              }
            }
          }
        }
        k.store(h + j);
      }
      col += col_step;
      if (col >= p.H) col -= p.H;
    }
  }
}

// ---- its gradient -------------------------------------------------------------
// A block takes the frames of its waves, of one utterance, and a slice of channels, and goes over the units: dh is
// read once.  A wave holds the sums over u of its frames in registers (denc is finished in the block); the sums
// over its frames meet in LDS, and the block's go to the workspace, one float32 row for 16 rows of a 16-bit dh
// or 8 of a float32 one (an eighth of the bytes), which net_joint_join adds up in the order of the frames.

struct JointGradParams {
  const void *enc, *pred, *dh;
  const int32_t *logit_lens, *label_lens;
  void *denc, *dpred;
  float* part;  // (B, t_blocks, U1, H)
  DropParams drop;
  float factor;  // of both sums: the dropout's scale, and 4 for tanh (its slope is 4u / (1 + u)^2)
  int32_t B, T, U1, H, t_blocks, slices, lanes;  // lanes: of a row, eight channels each (4, 8 or 16)
  int32_t tile_frames;                           // frames of a block
};

constexpr int kGradWaves = 4;
template <typename T>
constexpr int kWaveFrames = sizeof(T) == 4 ? 2 : 4;  // frames of a wave (GradShape says why)

// Whether enc + pred > 0 for two 16-bit elements at a time, without the sums: the sum of two floats is
// positive exactly when enc > -pred, and the bits of a float, its lower 15 flipped where the sign is set, are
// ordered like the floats when read as a whole number.  Both zeros of enc get -1, below 0 and -1 that the
// zeros of -pred have or equal to it; a NaN on either side compares as no.
template <typename T>
struct PositiveSum {
  static constexpr uint32_t kInf = __is_same(T, f16_t) ? 0x7c007c00u : 0x7f807f80u;
  static constexpr uint32_t kNever = 0x80008000u;       // of enc: no sum is positive
  static constexpr uint32_t kNeverPred = 0x7fff7fffu;   // of -pred
  __device__ static __forceinline__ i16x2 pair(uint32_t w) { return __builtin_bit_cast(i16x2, w); }
  __device__ static __forceinline__ uint32_t nan_mask(uint32_t w) {  // magnitude past infinity
    return Dropped::spread(__builtin_bit_cast(uint32_t, pair(kInf) - pair(w & 0x7fff7fffu)));
  }
  __device__ static __forceinline__ uint32_t enc_key(uint32_t w) {
    const uint32_t o = w ^ (Dropped::spread(w) & 0x7fff7fffu), nan = nan_mask(w);
    const uint32_t zero = (o & 0xffffu ? 0u : 0xffffu) | (o >> 16 ? 0u : 0xffff0000u);
    return ((o | zero) & ~nan) | (nan & 0x80008000u);
  }
  __device__ static __forceinline__ uint32_t pred_key(uint32_t w) {  // of -pred: ~w, or w without its sign
    const uint32_t s = Dropped::spread(w), nan = nan_mask(w);
    const uint32_t o = (w ^ ~s) & ~(s & 0x80008000u);
    return (o & ~nan) | (nan & 0x7fff7fffu);
  }
  __device__ static __forceinline__ uint32_t signs(uint32_t e, uint32_t q) {  // sign bits of q - e
    return __builtin_bit_cast(uint32_t, __builtin_elementwise_sub_sat(pair(q), pair(e)));
  }
};

// The upstream elements d times their weights but for the constant factor, added to both sums.
// 16-bit relu works on keys (e, q: PositiveSum's), everything else on the values.
template <typename T, int ACT, bool DROP>
__device__ __forceinline__ void add_weighted(const Pack<T, 8>& e, const Pack<T, 8>& q, const float* qf, Pack<T, 8>& d,
                                             const Dropped& signs, float* acc, float* ps) {
  float w[8];
  if constexpr (ACT == RNNT_ACT_RELU && sizeof(T) == 2) {
#pragma unroll
    for (int k = 0; k < 4; ++k) {
      const uint32_t on = PositiveSum<T>::signs(e.w[k], q.w[k]);
      d.w[k] &= Dropped::spread(DROP ? on & ~signs.m[k] : on);
    }
    d.get(w);
  } else {
    if constexpr (DROP) {
      Dropped drop;
#pragma unroll
      for (int k = 0; k < 4; ++k) drop.m[k] = Dropped::spread(signs.m[k]);
      drop.clear(d);
    }
    float ef[8];
    e.get(ef);
    d.get(w);
#pragma unroll
    for (int k = 0; k < 8; ++k) {
      const float s = ef[k] + qf[k];
      if constexpr (ACT == RNNT_ACT_RELU) {
        w[k] = s > 0.f ? w[k] : 0.f;
      } else {
        const float u = Activation<ACT>::u_of(s), r = __builtin_amdgcn_rcpf(1.f + u);
        w[k] *= u * r * r;
      }
    }
  }
#pragma unroll
  for (int k = 0; k < 8; ++k) {
    acc[k] += w[k];
    ps[k] += w[k];
  }
}

__device__ __forceinline__ uint32_t select(uint32_t mask, uint32_t a, uint32_t b) { return (a & mask) | (b & ~mask); }

// A step's rows: the wave's frames at one unit (the lane's), and the unit's row of pred.  Every load is issued,
// at an address inside the tensors: a load under a branch would make every later wait a full drain.
template <typename T, int FRAMES>
struct GradRows {
  Pack<T, 8> d[FRAMES], q;

  // dh, pred: the same for a whole wave; at: the lane's element (32 bits: bases stay in scalar registers)
  __device__ __forceinline__ void load(const T* const (&dh)[FRAMES], const T* pred, uint32_t at) {
#pragma unroll
    for (int i = 0; i < FRAMES; ++i) d[i].load_once(dh[i] + at);
    q.load(pred + at);
  }
};

// The utterance of place r when the ones with the most units come first (ties by number).  A block's time is
// its utterance's units, and a chip takes only a few blocks to a CU: the longest ones last left it idle.  Past 64
// utterances the blocks are many and stay in order.
__device__ __forceinline__ int longest_first(const int32_t* label_lens, int B, int r) {
  if (B > 64) return r;
  const int lane = static_cast<int>(threadIdx.x) & 63, mine = label_lens[min(lane, B - 1)];
  int place = 0;
  for (int j = 0; j < B; ++j) {
    const int other = __builtin_amdgcn_readlane(mine, j);
    place += other > mine || (other == mine && j < lane);
  }
  return __builtin_ctzll(__ballot(place == r && lane < B));
}

// EIGHTS: rows are multiples of eight elements, so that a group's numbers are one block.  H is at least 8 here: the
// last group of a row that is no multiple begins at H - 8, its first channels also the group's before it, which
// computes and writes the same values.
template <typename T, int ACT, bool EIGHTS, bool DROP>
__global__ __launch_bounds__(64 * kGradWaves) void net_joint_grad(JointGradParams p) {
  constexpr bool KEYS = ACT == RNNT_ACT_RELU && sizeof(T) == 2;
  constexpr int WAVES = kGradWaves, FRAMES = kWaveFrames<T>;
  static_assert(WAVES == 4, "256 threads store a step's 512 sums");
  __shared__ __attribute__((aligned(16))) float sums[2][WAVES][512];
  const int slice = static_cast<int>(blockIdx.x) % p.slices, bt = static_cast<int>(blockIdx.x) / p.slices;
  const int tb = bt % p.t_blocks, b = longest_first(p.label_lens, p.B, bt / p.t_blocks);
  const int wave = __builtin_amdgcn_readfirstlane(static_cast<int>(threadIdx.x) >> 6), lane = static_cast<int>(threadIdx.x) & 63;
  const int sub = lane / p.lanes, rows = 64 / p.lanes;
  // groups of a slice: one fewer than the lanes where random numbers straddle groups (the blocks are one more)
  const int wide = EIGHTS || !DROP ? p.lanes : p.lanes - 1;
  const int c0 = slice * wide * 8, c = min(c0 + min(lane & (p.lanes - 1), wide - 1) * 8, p.H - 8);
  int tl = p.logit_lens[b];
  const int ul = p.label_lens[b];
  if (tl < 0 || tl > p.T || ul < 0 || ul >= p.U1) tl = 0;
  const int t0 = (tb * WAVES + wave) * FRAMES, frames = max(0, min(FRAMES, tl - t0));
  float acc[FRAMES][8];
#pragma unroll
  for (int i = 0; i < FRAMES; ++i)
#pragma unroll
    for (int k = 0; k < 8; ++k) acc[i][k] = 0.f;

  if (tb * WAVES * FRAMES < tl) {  // the block's waves meet at barriers: all or none
    const int64_t run = static_cast<int64_t>(p.U1) * p.H;
    const T* pred = static_cast<const T*>(p.pred) + b * run;
    Rng rng{};
    if (DROP) rng = load_rng(p.drop.rng);
    // a frame past the last one reads that one's rows and is left out of the sums
    const T* dh[FRAMES];
    uint64_t number[FRAMES];  // of element (b, t, 0, 0)
    Pack<T, 8> e[FRAMES];
#pragma unroll
    for (int i = 0; i < FRAMES; ++i) {
      const int64_t bt_i = static_cast<int64_t>(b) * p.T + min(t0 + i, tl - 1);
      number[i] = static_cast<uint64_t>(bt_i * run);
      dh[i] = static_cast<const T*>(p.dh) + bt_i * run;
      e[i].load(static_cast<const T*>(p.enc) + bt_i * p.H + c);
    }
    GradRows<T, FRAMES> even, odd;
    even.load(dh, pred, static_cast<uint32_t>(min(sub, ul) * p.H + c));
    __builtin_amdgcn_sched_barrier(0);  // every load is on its way before the first is waited for
    if constexpr (KEYS) {
#pragma unroll
      for (int i = 0; i < FRAMES; ++i) {
        const uint32_t off = static_cast<uint32_t>((frames - 1 - i) >> 31);
#pragma unroll
        for (int k = 0; k < 4; ++k) e[i].w[k] = select(off, PositiveSum<T>::kNever, PositiveSum<T>::enc_key(e[i].w[k]));
      }
    }
    // this thread's part of a step's 512 sums: a pair of channels, neighbours in a row of the workspace
    const __amdgpu_buffer_rsrc_t part =
        make_buffer(p.part + (static_cast<int64_t>(b) * p.t_blocks + tb) * run, run * static_cast<int64_t>(sizeof(float)));
    const int from = static_cast<int>(threadIdx.x) >> 2, pair = static_cast<int>(threadIdx.x) & 3;
    const int sums_at = ((pair >> 1) * 64 + from) * 2 + (pair & 1);  // in float2
    const int put_u = from / p.lanes, put_c = min(c0 + min(from & (p.lanes - 1), wide - 1) * 8, p.H - 8) + pair * 2;

    auto step = [&](GradRows<T, FRAMES>& now, GradRows<T, FRAMES>& next, int u0, float (*lds)[512]) {
      const int u = u0 + sub;
      // a lane past the last unit reads that unit's row again and adds nothing
      next.load(dh, pred, static_cast<uint32_t>(min(u + rows, ul) * p.H + c));
      __builtin_amdgcn_sched_barrier(0);  // the loads stay ahead of the arithmetic
      const uint32_t at = static_cast<uint32_t>(u * p.H + c);
      // No branch from here to the barrier: what does not count (a lane past the last unit, a frame past the last
      // one) is masked, in the keys where there are any, else in the upstream elements.
      const uint32_t past = static_cast<uint32_t>((ul - u) >> 31);
      float ps[8] = {}, qf[8];
      if constexpr (KEYS) {
#pragma unroll
        for (int k = 0; k < 4; ++k) now.q.w[k] = select(past, PositiveSum<T>::kNeverPred, PositiveSum<T>::pred_key(now.q.w[k]));
      } else {
        now.q.get(qf);
      }
#pragma unroll
      for (int i = 0; i < FRAMES; ++i) {
        Dropped signs;
        if constexpr (DROP && EIGHTS) {
          signs.signs_below(random_block(rng, (number[i] + at) >> 3), p.drop.threshold);
        } else if constexpr (DROP) {
          // the row's lanes form the blocks that its slice meets, one each, from the one of its first channel on
          // (H - 8 where the slice has fewer than eight); a group's numbers may be of two of them
          const uint64_t n = number[i] + at, n_row = number[i] + static_cast<uint32_t>(u * p.H + min(c0, p.H - 8));
          signs.signs_below(random_block(rng, (n_row >> 3) + (lane & (p.lanes - 1))), p.drop.threshold);
          const uint32_t bits = signs.bits();
          const int from_lane = (lane & ~(p.lanes - 1)) + static_cast<int>((n >> 3) - (n_row >> 3));
          const uint32_t here = static_cast<uint32_t>(__shfl(static_cast<int>(bits), from_lane));
          const uint32_t next = static_cast<uint32_t>(__shfl(static_cast<int>(bits), from_lane + 1));
          signs.from_bits((here | next << 8) >> (n & 7));
        }
        if constexpr (!KEYS) {
          const uint32_t off = past | static_cast<uint32_t>((frames - 1 - i) >> 31);
#pragma unroll
          for (int k = 0; k < Pack<T, 8>::kWords; ++k) now.d[i].w[k] &= ~off;
        }
        add_weighted<T, ACT, DROP>(e[i], now.q, qf, now.d[i], signs, acc[i], ps);
      }
      float4* mine = reinterpret_cast<float4*>(lds[wave]);
      mine[lane] = make_float4(ps[0], ps[1], ps[2], ps[3]);
      mine[64 + lane] = make_float4(ps[4], ps[5], ps[6], ps[7]);
      __syncthreads();  // one to a step: see the two buffers below
      float2 total = make_float2(0.f, 0.f);
#pragma unroll
      for (int w = 0; w < WAVES; ++w) {
        const float2 v = reinterpret_cast<const float2*>(lds[w])[sums_at];
        total.x += v.x;
        total.y += v.y;
      }
      // past the last unit: an offset past the buffer, where nothing is written
      const int off = u0 + put_u <= ul ? ((u0 + put_u) * p.H + put_c) * 4 : kOutOfRange;
      __builtin_amdgcn_raw_buffer_store_b64(u32x2{__float_as_uint(total.x), __float_as_uint(total.y)}, part, off, 0, 0);
    };
    // Two sets of rows and of LDS sums in turn: the next rows are on their way while a step computes, and a wave
    // that has passed a step's barrier writes the other sums, which everyone has read before that barrier.
    for (int u0 = 0;;) {
      step(even, odd, u0, sums[0]);
      u0 += rows;
      if (u0 > ul) break;
      step(odd, even, u0, sums[1]);
      u0 += rows;
      if (u0 > ul) break;
    }
    // the rows of u that the wave's lanes shared out
    for (int off = p.lanes; off < 64; off <<= 1) {
#pragma unroll
      for (int i = 0; i < FRAMES; ++i)
#pragma unroll
        for (int k = 0; k < 8; ++k) acc[i][k] += __shfl_xor(acc[i][k], off);
    }
  }
  if (lane < p.lanes && c0 + lane * 8 < p.H) {
    T* denc = static_cast<T*>(p.denc) + (static_cast<int64_t>(b) * p.T + t0) * p.H + c;
#pragma unroll
    for (int i = 0; i < FRAMES; ++i) {
      if (t0 + i < p.T) {
        float f[8];
#pragma unroll
        for (int k = 0; k < 8; ++k) f[k] = i < frames ? acc[i][k] * p.factor : 0.f;
        Pack<T, 8> k;
        k.set(f);
        k.store(denc + static_cast<int64_t>(i) * p.H);
      }
    }
  }
}

// Rows of fewer than eight channels: a thread to a channel of one row of one gradient.
template <typename T, int ACT>
__global__ __launch_bounds__(256) void net_joint_grad_narrow(JointGradParams p, bool of_enc) {
  const int rows = of_enc ? p.T : p.U1;
  const int64_t at = static_cast<int64_t>(blockIdx.x) * 256 + threadIdx.x, row = at / p.H;
  if (row >= static_cast<int64_t>(p.B) * rows) return;
  const int c = static_cast<int>(at - row * p.H), b = static_cast<int>(row / rows), r = static_cast<int>(row - static_cast<int64_t>(b) * rows);
  const int tl = p.logit_lens[b], ul = p.label_lens[b];
  const bool ok = tl >= 0 && tl <= p.T && ul >= 0 && ul < p.U1;
  const int others = !ok ? 0 : of_enc ? (r < tl ? ul + 1 : 0) : (r <= ul ? tl : 0);
  Rng rng{};
  if (p.drop.threshold) rng = load_rng(p.drop.rng);
  float sum = 0.f;
  for (int o = 0; o < others; ++o) {
    const int64_t bt = static_cast<int64_t>(b) * p.T + (of_enc ? r : o), bu = static_cast<int64_t>(b) * p.U1 + (of_enc ? o : r);
    const int64_t n = (bt * p.U1 + (of_enc ? o : r)) * p.H + c;
    const float s = ElemTraits<T>::load1(static_cast<const T*>(p.enc) + bt * p.H + c) +
                    ElemTraits<T>::load1(static_cast<const T*>(p.pred) + bu * p.H + c);
    const bool keep = !p.drop.threshold ||
                      random16(random_block(rng, static_cast<uint64_t>(n >> 3)), static_cast<int>(n & 7)) >= p.drop.threshold;
    const float w = ACT == RNNT_ACT_RELU ? Activation<ACT>::slope(s) : 0.25f * Activation<ACT>::slope(s);
    if (keep && (ACT == RNNT_ACT_TANH || w != 0.f)) sum += ElemTraits<T>::load1(static_cast<const T*>(p.dh) + n) * w;
  }
  ElemTraits<T>::store1(static_cast<T*>(of_enc ? p.denc : p.dpred) + at, sum * p.factor);
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
    const int n = (tl + p.tile_frames - 1) / p.tile_frames;
    const float* part = p.part + (static_cast<int64_t>(b) * p.t_blocks * p.U1 + u) * p.H + c;
    const int64_t step = static_cast<int64_t>(p.U1) * p.H;
#pragma unroll 4
    for (int i = 0; i < n; ++i) {
      Pack<float, 4> k;
      if (left >= 4) k.load(part + i * step);
      else k.load_part(part + i * step, left);
#pragma unroll
      for (int j = 0; j < 4; ++j) f[j] += __uint_as_float(k.w[j]);
    }
  }
#pragma unroll
  for (int j = 0; j < 4; ++j) f[j] *= p.factor;
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

// Lanes to a row (eight channels each), the slices of channels that blocks share a row out in, and their tiles of
// frames.  Few frames to a wave leave room for twice the waves, which counts for more than the float32 sums
// (an eighth of dh): eight or four frames of bfloat16 to a wave, B=32 T=250 U=80, H=320: 72 + 4 us (gradient and
// join) or 65 + 6, H=640: 110 + 7 or 101 + 10, H=1024: 176 + 9 or 159 + 14; four or two of float32,
// B=16 T=150 U=40 H=321 tanh: 46 + 4 or 40 + 6.
struct GradShape {
  int lanes, slices, tile_frames, t_blocks;

  GradShape(const rnnt_joint_shape_t& s, bool dropping) {
    lanes = s.H <= 32 ? 4 : s.H <= 64 ? 8 : 16;
    const int wide = s.H % 8 == 0 || !dropping ? lanes : lanes - 1;
    slices = (s.H + 8 * wide - 1) / (8 * wide);
    tile_frames = kGradWaves * (s.dtype == RNNT_DTYPE_F32 ? kWaveFrames<float> : kWaveFrames<bf16_t>);
    t_blocks = static_cast<int>((static_cast<int64_t>(s.T_max) + tile_frames - 1) / tile_frames);
  }
};

// The gradient's grids and its buffers of sums (a block's is one of less than 2^31 bytes), whatever p is.
bool grad_fits(const rnnt_joint_shape_t& s) {
  const GradShape cut(s, true);
  const int64_t U1 = static_cast<int64_t>(s.U_max) + 1;
  const int64_t x = static_cast<int64_t>(s.B) * cut.t_blocks * cut.slices;
  const int64_t joins = (s.B * U1 * (s.H < 8 ? s.H : (s.H + 3) / 4) + 255) / 256;
  return x <= kMaxRows / 256 && joins <= kMaxRows / 256 && U1 * s.H < (int64_t{1} << 29);
}

size_t grad_bytes(const rnnt_joint_shape_t& s) {
  if (!grad_fits(s)) return 0;
  const GradShape cut(s, true);  // the same whatever p is
  return net_align256(static_cast<size_t>(s.B) * cut.t_blocks * (static_cast<size_t>(s.U_max) + 1) * s.H * sizeof(float));
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
  const int64_t groups = (static_cast<int64_t>(q.U1) * shape.H + 7) / 8 + (eights ? 0 : 1);
  // a frame to a block where kJointFrames would leave the chip fewer than eight blocks to a CU (B=16 T=150 U=40, 600
  // blocks of four frames and 2400 of one: H=320 bf16 tanh 29 and 20 us, f32 34 and 27; B=32 T=250 U=80 H=640 bf16
  // of full lengths, 8064 blocks of four and 16000 of two: 179 and 211)
  const int64_t y = (groups + 256 * kJointRun - 1) / (256 * kJointRun);
  const int64_t full = (static_cast<int64_t>(shape.T_max) + kJointFrames - 1) / kJointFrames;
  q.block_frames = full * shape.B * y >= 2048 ? kJointFrames : 1;
  q.t_blocks = static_cast<int32_t>(q.block_frames == 1 ? shape.T_max : full);
  const int64_t x = static_cast<int64_t>(shape.B) * q.t_blocks;
  if (x > kMaxRows / 256 || y > 65535) return RNNT_ERR_UNSUPPORTED;
  const dim3 grid(static_cast<uint32_t>(x), static_cast<uint32_t>(y));
  const int64_t lds = (static_cast<int64_t>(shape.H) + 8 + (shape.H + 8) / 8) * q.block_frames * static_cast<int64_t>(sizeof(float));
  return with_dtype(shape.dtype, [&](auto t) {
    return with_activation(act, [&](auto a) {
      using T = decltype(t);
      constexpr int A = decltype(a)::value;
      if (eights && q.drop.threshold) hipLaunchKernelGGL((net_joint<T, A, true>), grid, dim3(256), 0, stream, q);
      else if (eights) hipLaunchKernelGGL((net_joint<T, A, false>), grid, dim3(256), 0, stream, q);
      else if (lds <= kJointLdsBytes) hipLaunchKernelGGL((net_joint_odd<T, A, true>), grid, dim3(256), static_cast<size_t>(lds), stream, q);
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
  if (!grad_fits(shape)) return RNNT_ERR_UNSUPPORTED;
  Workspace ws;
  st = ws.take(workspace, workspace_bytes, grad_bytes(shape), stream);
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
  q.factor = q.drop.scale * (act == RNNT_ACT_TANH ? 4.f : 1.f);
  const GradShape cut(shape, q.drop.threshold != 0);
  q.t_blocks = cut.t_blocks;
  q.lanes = cut.lanes;
  q.slices = cut.slices;
  q.tile_frames = cut.tile_frames;
  const int64_t x = static_cast<int64_t>(shape.B) * q.t_blocks * q.slices;
  const int64_t joins = (static_cast<int64_t>(shape.B) * q.U1 * ((shape.H + 3) / 4) + 255) / 256;
  return with_dtype(shape.dtype, [&](auto t) {
    using T = decltype(t);
    if (shape.H < 8) {
      return with_activation(act, [&](auto a) {
        constexpr int A = decltype(a)::value;
        const auto grid = [&](int rows) { return dim3(static_cast<uint32_t>((static_cast<int64_t>(shape.B) * rows * shape.H + 255) / 256)); };
        hipLaunchKernelGGL((net_joint_grad_narrow<T, A>), grid(q.T), dim3(256), 0, stream, q, true);
        if (launched() != RNNT_OK) return RNNT_ERR_HIP;
        hipLaunchKernelGGL((net_joint_grad_narrow<T, A>), grid(q.U1), dim3(256), 0, stream, q, false);
        return launched();
      });
    }
    const rnnt_status_t done = with_activation(act, [&](auto a) {
      const dim3 grid(static_cast<uint32_t>(x)), block(64 * kGradWaves);
      const bool drop = q.drop.threshold != 0;
      constexpr int A = decltype(a)::value;
      if (drop && shape.H % 8 != 0) hipLaunchKernelGGL((net_joint_grad<T, A, false, true>), grid, block, 0, stream, q);
      else if (drop) hipLaunchKernelGGL((net_joint_grad<T, A, true, true>), grid, block, 0, stream, q);
      else hipLaunchKernelGGL((net_joint_grad<T, A, true, false>), grid, block, 0, stream, q);
      return launched();
    });
    if (done != RNNT_OK) return done;
    hipLaunchKernelGGL((net_joint_join<T>), dim3(static_cast<uint32_t>(joins)), dim3(256), 0, stream, q);
    return launched();
  });
}

}  // extern "C"
