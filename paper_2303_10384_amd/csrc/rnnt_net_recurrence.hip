// Gated linear recurrence and its gradient (contract in include/rnnt_network_mi355x.h).
#include <hip/hip_runtime.h>

#include <cstdint>

#include "rnnt_net.h"

namespace rnnt {
namespace {

// A block of W waves takes a tile of channels of one sequence and goes over its steps W * kSteps at a time, kSteps of
// them to a wave: a wave scans its steps from a zero state and multiplies their gates up, the waves' pairs (product P
// of the gates, state S) meet in LDS, every wave finds the state P h + S that arrives at its first step, and takes its
// steps again from there.  x and z are read once, the next tile's while this one is computed.
// Where sequences and channel tiles are too few to fill the chip, the steps are cut into segments: a first kernel
// finds each segment's pair, the second one begins each block at the state that the pairs before it give.
// Bound by the bytes of x, z and h, twice x and z in segments, and for 16 bits as much by the instructions of gates and
// runs (L=60013 D=640 bf16, one sequence: 31 us at 5.0 TB/s for the pairs, 45 us at 5.1 TB/s for the states, whose
// vector instructions fill about three quarters of the time).  One pass in which a block waits for the blocks before
// it would read x and z once; not built.
constexpr int kSteps = RNNT_RECURRENCE_STATE_STEPS;
constexpr int kWaves = 16;                     // of a block where sequences are few: as many as it can have
constexpr int kTileSteps = kSteps * kWaves;    // segments are multiples of it

struct RecurrenceParams {
  const void *x, *z;
  int64_t x_sb, x_st, z_sb, z_st;
  const int32_t* lens;
  const float* h0;
  void* h;
  float* last;
  float* states;  // (B, n_states, D), or null
  // backward
  const void* dh;
  const float* dlast;
  void *dx, *dz;
  float* dh0;
  float2* pairs;  // (B, segments, D) of the segments
  int32_t B, L, D, n_states, tiles, segments, seg_steps;
};

// ---- a step, and steps joined ---------------------------------------------------
// Whatever a state is added up from, a rounding has the size of a h or of (1 - a) x: what a shut gate lets through
// keeps its digits however large the state that it drops, and what an open one holds does not drift, however long.

// A step on its own, from the nearer of h and x a small part of the way to the other: h + g (x - h) where the gate is
// open, x + a (h - x) where it is shut (x = h stays).  By the definition where the difference is no finite float.
__device__ __forceinline__ float advance(float a, float g, float x, float h) {
  const float d = x - h;
  if (__builtin_isfinite(d)) return a < g ? __builtin_fmaf(-a, d, x) : __builtin_fmaf(g, d, h);
  return __builtin_fmaf(a, h, g * x);
}

constexpr float kLeast = 0x1p-126f;  // the least normal float

// A run of steps, h -> P h + S: of states forward, of the gradient's sums backward.  Up to 2 kSteps of them go by the
// definition, h = fma(a, h, g x), whose rounded a costs 2^-24 a step.  Between runs that would grow with the gates'
// memory, as 2^-24 / (1 - a) (z = 10 over 60000 steps: 5e-4), so Q = 1 - P is added up on its own.
struct Run {
  float P = 1.f, Q = 0.f, S = 0.f;

  // one step more, to the sum `next`
  __device__ __forceinline__ void step(float a, float g, float next, bool on) {
    const float q = __builtin_fmaf(g, P, Q), p = a * P;
    Q = on ? q : Q;
    P = on ? p : P;
    S = on ? next : S;
  }
  __device__ __forceinline__ void forward(float a, float in, float g, bool on) { step(a, g, __builtin_fmaf(a, S, in), on); }
  __device__ __forceinline__ void back(float a, float d, float g, bool on) { step(a, g, a * (S + d), on); }
  // The run joined to the state h as h + (S - Q h) where Q is below 1/2, as P h + S elsewhere.  A product of gates that is
  // below the floats does not make NaN of an infinite state.
  __device__ __forceinline__ float join(float h) const {
    const float next = Q < 0.5f ? __builtin_fmaf(-Q, h, S) + h : __builtin_fmaf(P, h, S);
    return __builtin_isfinite(h) ? next : __builtin_fmaf(fmaxf(P, kLeast), h, S);
  }
  // `next` behind this one
  __device__ __forceinline__ void append(const Run& next) {
    S = next.join(S);
    Q = __builtin_fmaf(next.P, Q, next.Q);
    P = next.Q < 0.5f ? __builtin_fmaf(-next.Q, P, P) : next.P * P;
  }
  // In memory (m, S): m is P, or -Q where Q is below 1/2 (and below 0 also where Q = 0), from which the other is known
  // to its last digit.
  __device__ __forceinline__ float2 pack() const { return make_float2(Q < 0.5f ? fminf(-Q, -kLeast) : P, S); }
  __device__ __forceinline__ static Run unpack(float2 k) {
    Run r;
    r.P = k.x < 0.f ? 1.f + k.x : k.x;
    r.Q = k.x < 0.f ? -k.x : 1.f - k.x;
    r.S = k.y;
    return r;
  }
};

// Run::unpack(k).join(h) for a finite h, in three operations; not finite for one that is not, nor is any behind it.
__device__ __forceinline__ float join_finite(float2 k, float h) {
  const float keep = __builtin_amdgcn_fmed3f(k.x * -0x1p127f, 0.f, 1.f);  // 1 where m is -Q
  return __builtin_fmaf(keep, h, __builtin_fmaf(k.x, h, k.y));
}

// The part of the work that a block has, and its sequence's length.
struct Place {
  int b, tile, segment, begin, end, len;  // steps [begin, end) of the segment
  bool bad;

  __device__ __forceinline__ explicit Place(const RecurrenceParams& p) {
    const int i = static_cast<int>(blockIdx.x);
    tile = i % p.tiles;
    segment = i / p.tiles % p.segments;
    b = i / p.tiles / p.segments;
    len = p.lens ? p.lens[b] : p.L;
    bad = len < 0 || len > p.L;
    if (bad) len = 0;
    begin = segment * p.seg_steps;
    end = min(p.L - begin, p.seg_steps) + begin;
  }
};

template <typename T, int VEC>
struct Rows {
  Pack<T, VEC> r[kSteps];

  // rows t .. t + kSteps - 1, the last valid one in the place of those past it
  __device__ __forceinline__ void load(const T* base, int64_t stride, int t, int len, int c) {
#pragma unroll
    for (int j = 0; j < kSteps; ++j) r[j].load(base + min(t + j, len - 1) * stride + c);
  }
};

// rows t + j of an output of D channels, those from `end` on left out (an offset past the buffer)
template <typename T, int VEC, int W>
struct RowStore {
  __amdgpu_buffer_rsrc_t r;
  int left;   // steps from the buffer's first row to the end of the segment
  int D, c;

  // base: row `first` of a dense output, of which `left` steps belong to the segment
  __device__ __forceinline__ RowStore(T* base, int64_t first, int left_, int D_, int c_)
      : r(make_buffer(base + first * D_, static_cast<int64_t>(min(left_, W * kSteps)) * D_ * static_cast<int64_t>(sizeof(T)))),
        left(left_), D(D_), c(c_) {}
  __device__ __forceinline__ void put(int row, const float* f) const {
    Pack<T, VEC> k;
    k.set(f);
    const int off = row < left ? (row * D + c) * static_cast<int>(sizeof(T)) : kOutOfRange;
    if constexpr (Pack<T, VEC>::kBytes == 2)
      __builtin_amdgcn_raw_buffer_store_b16(static_cast<uint16_t>(k.w[0]), r, off, 0, 0);
    else
      __builtin_amdgcn_raw_buffer_store_b32(k.w[0], r, off, 0, 0);
  }
};

// The runs of a block's waves in Run::pack()'s form, two sets of them in turn.  BACK: the last wave's comes first.
template <int VEC, int W>
struct PairBoard {
  struct __attribute__((aligned(8 * VEC))) Pairs {
    float2 of[VEC];
  };
  Pairs at[2][W][64];
  float state[2][64][VEC];  // that arrives at the tile

  __device__ __forceinline__ void put(int set, int wave, int lane, const Run* run) {
    Pairs k;
#pragma unroll
    for (int v = 0; v < VEC; ++v) k.of[v] = run[v].pack();
    at[set][wave][lane] = k;
  }
  // the state that arrives at `wave`'s run, from the tile's through the runs before
  template <bool BACK>
  __device__ __forceinline__ void arrive(int set, int wave, int lane, float* h) const {
    const int n = BACK ? W - 1 - wave : wave;
    float first[VEC];
#pragma unroll
    for (int v = 0; v < VEC; ++v) h[v] = first[v] = state[set][lane][v];
#pragma unroll
    for (int i = 0; i < W - 1; ++i) {
      if (i >= n) break;
      const Pairs k = at[set][BACK ? W - 1 - i : i][lane];
#pragma unroll
      for (int v = 0; v < VEC; ++v) h[v] = join_finite(k.of[v], h[v]);
    }
    bool finite = true;
#pragma unroll
    for (int v = 0; v < VEC; ++v) finite = finite && __builtin_isfinite(h[v]);
    if (finite) return;
#pragma unroll
    for (int v = 0; v < VEC; ++v) h[v] = first[v];
#pragma unroll 1
    for (int i = 0; i < n; ++i) {
#pragma unroll
      for (int v = 0; v < VEC; ++v) h[v] = Run::unpack(at[set][BACK ? W - 1 - i : i][lane].of[v]).join(h[v]);
    }
  }
};

// carry through the pairs of the segments before (BACK: behind) a block's, the waves a stretch each
template <int VEC, bool BACK, int W>
__device__ __forceinline__ void carry_in(const RecurrenceParams& p, const Place& at, int c, int wave, int lane,
                                         PairBoard<VEC, W>& board, float* carry) {
  const int n = BACK ? p.segments - 1 - at.segment : at.segment;
  if (n == 0) return;
  const int share = (n + W - 1) / W, from = min(wave * share, n), to = min(from + share, n);
  const float2* pairs = p.pairs + (static_cast<int64_t>(at.b) * p.segments + (BACK ? at.segment + 1 : 0)) * p.D + c;
  Run run[VEC];
#pragma unroll 4
  for (int i = from; i < to; ++i) {
    const int64_t seg = BACK ? to - 1 - (i - from) : i;
#pragma unroll
    for (int v = 0; v < VEC; ++v) run[v].append(Run::unpack(pairs[seg * p.D + v]));
  }
  board.put(1, wave, lane, run);
  __syncthreads();
#pragma unroll
  for (int i = 0; i < W; ++i) {
    const auto one = board.at[1][BACK ? W - 1 - i : i][lane];
#pragma unroll
    for (int v = 0; v < VEC; ++v) carry[v] = Run::unpack(one.of[v]).join(carry[v]);
  }
}

template <typename T, int VEC, int W>
__global__ __launch_bounds__(64 * W, 4) void net_recurrence(RecurrenceParams p) {
  constexpr int TILE = W * kSteps;
  __shared__ PairBoard<VEC, W> board;
  const Place at(p);
  const int wave = __builtin_amdgcn_readfirstlane(static_cast<int>(threadIdx.x) >> 6), lane = static_cast<int>(threadIdx.x) & 63;
  const int c = min((at.tile * 64 + lane) * VEC, p.D - VEC);
  const int64_t bc = static_cast<int64_t>(at.b) * p.D + c;
  float carry[VEC];
#pragma unroll
  for (int v = 0; v < VEC; ++v) carry[v] = at.bad ? __builtin_nanf("") : p.h0 ? p.h0[bc + v] : 0.f;
  carry_in<VEC, false, W>(p, at, c, wave, lane, board, carry);
  T* h = static_cast<T*>(p.h);
  const int64_t row0 = static_cast<int64_t>(at.b) * p.L;
  int t0 = at.begin;
  if (t0 < at.len) {
    const T* x = static_cast<const T*>(p.x) + at.b * p.x_sb;
    const T* z = static_cast<const T*>(p.z) + at.b * p.z_sb;
    Rows<T, VEC> xs, zs;
    xs.load(x, p.x_st, t0 + wave * kSteps, at.len, c);
    zs.load(z, p.z_st, t0 + wave * kSteps, at.len, c);
    for (int set = 0; t0 < min(at.end, at.len); t0 += TILE, set ^= 1) {
      const int t = t0 + wave * kSteps, live = at.len - t;
      float a[kSteps][VEC], in[kSteps][VEC];  // in: (1 - a) x
      Run run[VEC];
      // the next tile's rows, on their way while this one is computed
      const Rows<T, VEC> xn = xs, zn = zs;
      if (t0 + TILE < min(at.end, at.len)) {
        xs.load(x, p.x_st, t + TILE, at.len, c);
        zs.load(z, p.z_st, t + TILE, at.len, c);
      }
      __builtin_amdgcn_sched_barrier(0);
      const bool whole = live >= kSteps;
      const auto scan = [&](auto all) {
#pragma unroll
        for (int j = 0; j < kSteps; ++j) {
          float xf[VEC], zf[VEC];
          xn.r[j].get(xf);
          zn.r[j].get(zf);
#pragma unroll
          for (int v = 0; v < VEC; ++v) {
            float g;
            gate<T>(zf[v], a[j][v], g);
            in[j][v] = g * xf[v];
            run[v].forward(a[j][v], in[j][v], g, all || j < live);
          }
          if (j == kSteps / 2 - 1) __builtin_amdgcn_sched_barrier(0);  // all gates begun at once would not fit the registers
        }
      };
      if (whole) scan(std::true_type{});
      else scan(std::false_type{});
      board.put(set, wave, lane, run);
      if (wave == W - 1) {
#pragma unroll
        for (int v = 0; v < VEC; ++v) board.state[set][lane][v] = carry[v];
      }
      __syncthreads();  // one to a tile: the other set is written before the next
      float first[VEC];
      board.template arrive<false>(set, wave, lane, first);
      if (wave == W - 1) {  // to the next tile
#pragma unroll
        for (int v = 0; v < VEC; ++v) carry[v] = run[v].join(first[v]);
      }
      if (p.states && t < at.end) {
        Pack<float, VEC> k;
        k.set(first);
        k.store(p.states + (static_cast<int64_t>(at.b) * p.n_states + t / kSteps) * p.D + c);
      }
      const RowStore<T, VEC, W> out(h, row0 + t0, at.end - t0, p.D, c);
#pragma unroll
      for (int j = 0; j < kSteps; ++j) {
        float f[VEC];
#pragma unroll
        for (int v = 0; v < VEC; ++v) {
          first[v] = __builtin_fmaf(a[j][v], first[v], in[j][v]);
          f[v] = whole || j < live ? first[v] : 0.f;
        }
        out.put(wave * kSteps + j, f);
      }
    }
  }
  for (; t0 < at.end; t0 += TILE) {  // behind the sequence
    const RowStore<T, VEC, W> out(h, row0 + t0, at.end - t0, p.D, c);
    float f[VEC];
#pragma unroll
    for (int v = 0; v < VEC; ++v) f[v] = at.bad ? __builtin_nanf("") : 0.f;
#pragma unroll
    for (int j = 0; j < kSteps; ++j) out.put(wave * kSteps + j, f);
  }
  if (at.segment == p.segments - 1 && wave == W - 1) {
#pragma unroll
    for (int v = 0; v < VEC; ++v) p.last[bc + v] = carry[v];
  }
}

// At most kSteps steps (one, for a streaming decoder): a thread to VEC channels, step by step, nothing to exchange.
// 16 sequences of 640 float32 channels: one step 2.7 us and eight 4.0, where the tiles of four waves take 3.8 and 3.9.
template <typename T, int VEC>
__global__ __launch_bounds__(64) void net_recurrence_short(RecurrenceParams p) {
  const int b = static_cast<int>(blockIdx.x) / p.tiles, tile = static_cast<int>(blockIdx.x) % p.tiles;
  const int c = min((tile * 64 + static_cast<int>(threadIdx.x)) * VEC, p.D - VEC);
  int len = p.lens ? p.lens[b] : p.L;
  const bool bad = len < 0 || len > p.L;
  if (bad) len = 0;
  const int64_t bc = static_cast<int64_t>(b) * p.D + c;
  float s[VEC];
#pragma unroll
  for (int v = 0; v < VEC; ++v) s[v] = bad ? __builtin_nanf("") : p.h0 ? p.h0[bc + v] : 0.f;
  if (p.states && p.L > 0) {
    Pack<float, VEC> k;
    k.set(s);
    k.store(p.states + static_cast<int64_t>(b) * p.n_states * p.D + c);
  }
  const T* x = static_cast<const T*>(p.x) + b * p.x_sb + c;
  const T* z = static_cast<const T*>(p.z) + b * p.z_sb + c;
  T* h = static_cast<T*>(p.h) + static_cast<int64_t>(b) * p.L * p.D + c;
  for (int t = 0; t < p.L; ++t) {
    Pack<T, VEC> k;
    float f[VEC];
#pragma unroll
    for (int v = 0; v < VEC; ++v) f[v] = bad ? s[v] : 0.f;
    if (t < len) {
      float xf[VEC], zf[VEC];
      k.load(x + t * p.x_st);
      k.get(xf);
      k.load(z + t * p.z_st);
      k.get(zf);
#pragma unroll
      for (int v = 0; v < VEC; ++v) {
        float a, g;
        gate<T>(zf[v], a, g);
        f[v] = s[v] = advance(a, g, xf[v], s[v]);
      }
    }
    k.set(f);
    k.store(h + static_cast<int64_t>(t) * p.D);
  }
#pragma unroll
  for (int v = 0; v < VEC; ++v) p.last[bc + v] = s[v];
}

// A segment's pair: forward (BACK false) of h, backward of the gradient's sums.  A wave streams a stretch of its
// steps; nothing is exchanged before the end.
template <typename T, int VEC, bool BACK>
__global__ __launch_bounds__(64 * kWaves) void net_recurrence_pairs(RecurrenceParams p) {
  __shared__ PairBoard<VEC, kWaves> board;
  const Place at(p);
  const int wave = __builtin_amdgcn_readfirstlane(static_cast<int>(threadIdx.x) >> 6), lane = static_cast<int>(threadIdx.x) & 63;
  const int c = min((at.tile * 64 + lane) * VEC, p.D - VEC);
  // its steps [from, to), whole batches of kSteps but for the sequence's end
  const int share = (p.seg_steps / kSteps + kWaves - 1) / kWaves * kSteps;
  const int stop = min(at.end, at.len);
  const int from = min(at.begin + wave * share, stop), to = min(from + share, stop);
  Run all[VEC], run[VEC];
  const int batches = max(0, (to - from + kSteps - 1) / kSteps);
  if (batches > 0) {
    const T* z = static_cast<const T*>(p.z) + at.b * p.z_sb;
    const T* x = BACK ? static_cast<const T*>(p.dh) + static_cast<int64_t>(at.b) * p.L * p.D : static_cast<const T*>(p.x) + at.b * p.x_sb;
    const int64_t x_st = BACK ? p.D : p.x_st;
    const bool with_x = !BACK || p.dh != nullptr;
    Rows<T, VEC> xs, zs;
    if (!with_x) {
#pragma unroll
      for (int j = 0; j < kSteps; ++j) xs.r[j].zero();
    }
    const auto step_of = [&](int i) { return from + (BACK ? batches - 1 - i : i) * kSteps; };
    if (with_x) xs.load(x, x_st, step_of(0), to, c);
    zs.load(z, p.z_st, step_of(0), to, c);
    for (int i = 0; i < batches; ++i) {
      const Rows<T, VEC> xn = xs, zn = zs;
      const int live = to - step_of(i);
      if (i + 1 < batches) {
        if (with_x) xs.load(x, x_st, step_of(i + 1), to, c);
        zs.load(z, p.z_st, step_of(i + 1), to, c);
      }
      const auto scan = [&](auto whole) {
#pragma unroll
        for (int k = 0; k < kSteps; ++k) {
          const int j = BACK ? kSteps - 1 - k : k;
          float xf[VEC], zf[VEC];
          xn.r[j].get(xf);
          zn.r[j].get(zf);
#pragma unroll
          for (int v = 0; v < VEC; ++v) {
            float a, g;
            gate<T>(zf[v], a, g);
            if constexpr (BACK) run[v].back(a, xf[v], g, whole || j < live);
            else run[v].forward(a, g * xf[v], g, whole || j < live);
          }
        }
      };
      if (live >= kSteps) scan(std::true_type{});
      else scan(std::false_type{});
      if ((i & 1) || i + 1 == batches) {  // two batches to a run
#pragma unroll
        for (int v = 0; v < VEC; ++v) {
          all[v].append(run[v]);
          run[v] = Run{};
        }
      }
    }
  }
  board.put(0, wave, lane, all);
  __syncthreads();
  if (wave != 0) return;
  // the waves' pairs into one
  float2* out = p.pairs + (static_cast<int64_t>(at.b) * p.segments + at.segment) * p.D + c;
#pragma unroll
  for (int v = 0; v < VEC; ++v) {
    Run one;
#pragma unroll
    for (int i = 0; i < kWaves; ++i) one.append(Run::unpack(board.at[0][BACK ? kWaves - 1 - i : i][lane].of[v]));
    out[v] = one.pack();
  }
}

// The gradient goes the other way: s_t = dh_t + a_{t+1} s_{t+1}, tile by tile from the end, its carry d = a s.  The
// states that dz needs are formed again from the one stored before the wave's first step.
template <typename T, int VEC, int W>
__global__ __launch_bounds__(64 * W, 4) void net_recurrence_grad(RecurrenceParams p) {
  constexpr int TILE = W * kSteps;
  __shared__ PairBoard<VEC, W> board;
  const Place at(p);
  const int wave = __builtin_amdgcn_readfirstlane(static_cast<int>(threadIdx.x) >> 6), lane = static_cast<int>(threadIdx.x) & 63;
  const int c = min((at.tile * 64 + lane) * VEC, p.D - VEC);
  const int64_t bc = static_cast<int64_t>(at.b) * p.D + c, row0 = static_cast<int64_t>(at.b) * p.L;
  T *dx = static_cast<T*>(p.dx), *dz = static_cast<T*>(p.dz);
  float carry[VEC];
#pragma unroll
  for (int v = 0; v < VEC; ++v) carry[v] = at.bad || !p.dlast ? 0.f : p.dlast[bc + v];
  carry_in<VEC, true, W>(p, at, c, wave, lane, board, carry);
  const int tiles = (at.end - at.begin + TILE - 1) / TILE;
  // tiles that hold steps of the sequence; the ones behind it are zero
  const int live_tiles = max(0, min(tiles, (at.len - at.begin + TILE - 1) / TILE));
  float zero[VEC];
#pragma unroll
  for (int v = 0; v < VEC; ++v) zero[v] = 0.f;
  for (int i = live_tiles; i < tiles; ++i) {
    const int t0 = at.begin + i * TILE;
    const RowStore<T, VEC, W> ox(dx, row0 + t0, at.end - t0, p.D, c), oz(dz, row0 + t0, at.end - t0, p.D, c);
#pragma unroll
    for (int j = 0; j < kSteps; ++j) {
      ox.put(wave * kSteps + j, zero);
      oz.put(wave * kSteps + j, zero);
    }
  }
  if (live_tiles > 0) {
    const T* x = static_cast<const T*>(p.x) + at.b * p.x_sb;
    const T* z = static_cast<const T*>(p.z) + at.b * p.z_sb;
    const T* dh = static_cast<const T*>(p.dh) + row0 * p.D;
    const float* states = p.states + static_cast<int64_t>(at.b) * p.n_states * p.D + c;
    const bool with_dh = p.dh != nullptr;
    Rows<T, VEC> xs, zs, ds;
    if (!with_dh) {
#pragma unroll
      for (int j = 0; j < kSteps; ++j) ds.r[j].zero();
    }
    Pack<float, VEC> st;
    const auto load = [&](int i) {
      const int t = at.begin + i * TILE + wave * kSteps;
      xs.load(x, p.x_st, t, at.len, c);
      zs.load(z, p.z_st, t, at.len, c);
      if (with_dh) ds.load(dh, p.D, t, at.len, c);
      st.load(states + static_cast<int64_t>(min(t, at.len - 1) / kSteps) * p.D);
    };
    load(live_tiles - 1);
    for (int i = live_tiles - 1, set = 0; i >= 0; --i, set ^= 1) {
      const int t0 = at.begin + i * TILE, live = at.len - t0 - wave * kSteps;
      const bool whole = live >= kSteps;
      float a[kSteps][VEC], g[kSteps][VEC], w[kSteps][VEC], s[VEC];
      st.get(s);
#pragma unroll
      for (int j = 0; j < kSteps; ++j) {
        float xf[VEC], zf[VEC];
        xs.r[j].get(xf);
        zs.r[j].get(zf);
#pragma unroll
        for (int v = 0; v < VEC; ++v) {
          gate<T>(zf[v], a[j][v], g[j][v]);
          const float in = g[j][v] * xf[v];
          // (h - x) a g, the difference of the products: that of h and x may be past the floats
          w[j][v] = __builtin_fmaf(a[j][v] * g[j][v], s[v], -(a[j][v] * in));
          s[v] = __builtin_fmaf(a[j][v], s[v], in);
        }
        if (j == kSteps / 2 - 1) __builtin_amdgcn_sched_barrier(0);  // as in net_recurrence
      }
      Rows<T, VEC> d = ds;
      if (i > 0) load(i - 1);
      Run run[VEC];
#pragma unroll
      for (int j = kSteps - 1; j >= 0; --j) {
        float df[VEC];
        d.r[j].get(df);
#pragma unroll
        for (int v = 0; v < VEC; ++v) run[v].back(a[j][v], df[v], g[j][v], whole || j < live);
      }
      board.put(set, wave, lane, run);
      if (wave == 0) {
#pragma unroll
        for (int v = 0; v < VEC; ++v) board.state[set][lane][v] = carry[v];
      }
      __syncthreads();  // one to a tile: the other set is written before the next
      float in[VEC];
      board.template arrive<true>(set, wave, lane, in);
      if (wave == 0) {  // to the tile before
#pragma unroll
        for (int v = 0; v < VEC; ++v) carry[v] = run[v].join(in[v]);
      }
      const RowStore<T, VEC, W> ox(dx, row0 + t0, at.end - t0, p.D, c), oz(dz, row0 + t0, at.end - t0, p.D, c);
      const auto gradients = [&](auto all) {
#pragma unroll
        for (int j = kSteps - 1; j >= 0; --j) {
          float df[VEC], fx[VEC], fz[VEC];
          d.r[j].get(df);
#pragma unroll
          for (int v = 0; v < VEC; ++v) {
            const bool on = all || j < live;
            const float total = in[v] + df[v];
            fx[v] = on ? g[j][v] * total : 0.f;
            fz[v] = on ? w[j][v] * total : 0.f;
            in[v] = on ? a[j][v] * total : in[v];
          }
          ox.put(wave * kSteps + j, fx);
          oz.put(wave * kSteps + j, fz);
        }
      };
      if (whole) gradients(std::true_type{});
      else gradients(std::false_type{});
    }
  }
  if (p.dh0 && at.segment == 0 && wave == 0) {
#pragma unroll
    for (int v = 0; v < VEC; ++v) p.dh0[bc + v] = at.bad ? 0.f : carry[v];
  }
}

rnnt_status_t check(const rnnt_recurrence_shape_t& s) {
  if (s.B < 1 || s.L < 0 || s.D < 1 || s.x_stride_b < 0 || s.x_stride_t < 0 || s.z_stride_b < 0 || s.z_stride_t < 0)
    return RNNT_ERR_BAD_SHAPE;
  if (!net_dtype_known(s.dtype)) return RNNT_ERR_BAD_DTYPE;
  // a tile's rows are one buffer of less than 2^31 bytes; threads of a launch are a 32-bit count
  if (s.D > (1 << 21) || s.L > (1 << 30) || static_cast<int64_t>(s.B) * ((s.D + 63) / 64) > kMaxRows / (64 * kWaves))
    return RNNT_ERR_UNSUPPORTED;
  return RNNT_OK;
}

// Whether two (B, D) float32 states share memory: blocks write the one while others, of later segments or of the next
// channels (which begin early in a row that is no multiple of a block's), still read the other.
bool overlap(const float* a, const float* b, const rnnt_recurrence_shape_t& s) {
  const uintptr_t at = reinterpret_cast<uintptr_t>(a), bt = reinterpret_cast<uintptr_t>(b);
  const uintptr_t bytes = static_cast<uintptr_t>(s.B) * s.D * sizeof(float);
  return a && b && (at < bt ? bt - at : at - bt) < bytes;
}

int state_count(int L) { return static_cast<int>((static_cast<int64_t>(L) + kSteps - 1) / kSteps); }

// Blocks to a sequence: one, or as many segments of at least two tiles as give the chip a block to a CU.  Segments read
// x and z twice (backward: z and dh) and are two launches, so they pay where a sequence is long and blocks are few.
// D=640 bf16, us in one block and in segments (pairs and states or gradients):
//                        768 steps          896                1280               2000
//   forward   5 blocks   23, 23             26, 28             36, 23
//            80          25, 26             29, 31             39, 38             59, 51
//           100, 125                        29, 37 (125)       40, 47 (125)       60, 62 (100)  61, 66 (125)
//   backward  5          28, 19             33, 25             45, 19
//            80          32, 26             36, 31             50, 40             79, 55
//           125          34, 35             38, 42             55, 52             93, 82
// At 160 blocks they lose both ways (2000 steps: 66, 113 and 99, 134).
void segments_of(const rnnt_recurrence_shape_t& s, bool back, RecurrenceParams* p) {
  const int vec = s.dtype == RNNT_DTYPE_F32 || s.D < 2 ? 1 : 2;
  p->tiles = (s.D + 64 * vec - 1) / (64 * vec);
  const int64_t blocks = static_cast<int64_t>(s.B) * p->tiles, steps = (static_cast<int64_t>(s.L) + kTileSteps - 1) / kTileSteps;
  p->segments = 1;
  p->seg_steps = s.L;
  int64_t want = 256 / blocks;
  if (want >= 3 ? steps >= (back ? 6 : 8) : back && want == 2 && steps >= 9) {
    if (want > steps / 2) want = steps / 2;
    const int64_t per = (steps + want - 1) / want;
    p->segments = static_cast<int32_t>((steps + per - 1) / per);
    p->seg_steps = static_cast<int32_t>(per * kTileSteps);
  }
}

size_t pair_bytes(const rnnt_recurrence_shape_t& s, bool back) {
  RecurrenceParams p{};
  segments_of(s, back, &p);
  return p.segments > 1 ? net_align256(static_cast<size_t>(s.B) * p.segments * s.D * sizeof(float2)) : 0;
}

// Waves of a block: sixteen while channel tiles are few, then four or one, no more than the steps have use for
// (forward, sixteen waves and these: B=8 L=20 D=640 bf16 7.1 and 4.2 us, B=64 L=81 D=1024 bf16 14.8 and 11.3,
// B=600 L=60 D=512 bf16 53 and 24, B=256 L=81 D=1024 f32 72 and 42, 6.2 TB/s).
template <typename F>
rnnt_status_t with_waves(const RecurrenceParams& p, F&& f) {
  const int64_t blocks = static_cast<int64_t>(p.B) * p.tiles * p.segments;
  if (blocks >= 2048) return f(std::integral_constant<int, 1>{});
  if (blocks >= 512 || p.L <= 4 * kSteps) return f(std::integral_constant<int, 4>{});
  return f(std::integral_constant<int, kWaves>{});
}

template <typename F>
rnnt_status_t with_vector(const rnnt_recurrence_shape_t& s, F&& f) {
  return with_dtype(s.dtype, [&](auto t) {
    using T = decltype(t);
    if constexpr (sizeof(T) == 4) return f(t, std::integral_constant<int, 1>{});
    else return s.D < 2 ? f(t, std::integral_constant<int, 1>{}) : f(t, std::integral_constant<int, 2>{});
  });
}

RecurrenceParams params_of(const void* x, const void* z, const rnnt_recurrence_shape_t& s, const int32_t* lens, bool back,
                           char* ws) {
  RecurrenceParams p{};
  p.x = x;
  p.z = z;
  p.x_sb = s.x_stride_b;
  p.x_st = s.x_stride_t;
  p.z_sb = s.z_stride_b;
  p.z_st = s.z_stride_t;
  p.lens = lens;
  p.B = s.B;
  p.L = s.L;
  p.D = s.D;
  p.n_states = state_count(s.L);
  p.pairs = reinterpret_cast<float2*>(ws);
  segments_of(s, back, &p);
  return p;
}

}  // namespace
}  // namespace rnnt

using namespace rnnt;

extern "C" {

size_t rnnt_recurrence_states_bytes(rnnt_recurrence_shape_t shape) {
  if (check(shape) != RNNT_OK) return 0;
  return static_cast<size_t>(shape.B) * state_count(shape.L) * shape.D * sizeof(float);
}

size_t rnnt_recurrence_workspace_bytes(rnnt_recurrence_shape_t shape) {
  if (check(shape) != RNNT_OK) return 0;
  const size_t forward = pair_bytes(shape, false), back = pair_bytes(shape, true);
  return forward > back ? forward : back;
}

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
  Workspace ws;
  st = ws.take(workspace, workspace_bytes, pair_bytes(shape, false), stream);
  if (st != RNNT_OK) return st;
  if (overlap(h0, last_out, shape)) return RNNT_ERR_UNSUPPORTED;
  RecurrenceParams p = params_of(x, z, shape, lens, false, ws.ptr);
  p.h0 = h0;
  p.h = h_out;
  p.last = last_out;
  p.states = static_cast<float*>(states_out);
  const dim3 grid(static_cast<uint32_t>(p.B * p.tiles * p.segments));
  return with_vector(shape, [&](auto t, auto vec) {
    using T = decltype(t);
    constexpr int VEC = decltype(vec)::value;
    if (p.L <= kSteps) {
      hipLaunchKernelGGL((net_recurrence_short<T, VEC>), grid, dim3(64), 0, stream, p);
      return launched();
    }
    if (p.segments > 1) {
      hipLaunchKernelGGL((net_recurrence_pairs<T, VEC, false>), grid, dim3(64 * kWaves), 0, stream, p);
      if (launched() != RNNT_OK) return RNNT_ERR_HIP;
    }
    return with_waves(p, [&](auto w) {
      constexpr int W = decltype(w)::value;
      hipLaunchKernelGGL((net_recurrence<T, VEC, W>), grid, dim3(64 * W), 0, stream, p);
      return launched();
    });
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
  Workspace ws;
  st = ws.take(workspace, workspace_bytes, pair_bytes(shape, true), stream);
  if (st != RNNT_OK) return st;
  if (overlap(dlast, dh0, shape)) return RNNT_ERR_UNSUPPORTED;
  RecurrenceParams p = params_of(x, z, shape, lens, true, ws.ptr);
  p.states = const_cast<float*>(static_cast<const float*>(states));
  p.dh = dh;
  p.dlast = dlast;
  p.dx = dx;
  p.dz = dz;
  p.dh0 = dh0;
  const dim3 grid(static_cast<uint32_t>(p.B * p.tiles * p.segments));
  return with_vector(shape, [&](auto t, auto vec) {
    using T = decltype(t);
    constexpr int VEC = decltype(vec)::value;
    if (p.segments > 1) {
      hipLaunchKernelGGL((net_recurrence_pairs<T, VEC, true>), grid, dim3(64 * kWaves), 0, stream, p);
      if (launched() != RNNT_OK) return RNNT_ERR_HIP;
    }
    return with_waves(p, [&](auto w) {
      constexpr int W = decltype(w)::value;
      hipLaunchKernelGGL((net_recurrence_grad<T, VEC, W>), grid, dim3(64 * W), 0, stream, p);
      return launched();
    });
  });
}

}  // extern "C"
