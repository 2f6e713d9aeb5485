// The product in 8-bit integers (contract in include/rnnt_encoder_mi355x.h).
#include <hip/hip_runtime.h>

#include <cstdint>

#include "rnnt_enc.h"

namespace rnnt {
namespace {

typedef int i32x4 __attribute__((ext_vector_type(4)));
typedef int i32x16 __attribute__((ext_vector_type(16)));
typedef float f32x4 __attribute__((ext_vector_type(4)));

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

// ---- rows held in registers ----------------------------------------------------
// For rows of up to 1024 a block of four waves keeps 128 rows of x, 32 to a wave, in registers in the matrix
// instruction's order, and passes over its share of w, 64 rows at a time through LDS.  x is read once, whatever N is,
// and taken to 8 bits on the way in, so no copy of it in 8 bits goes through memory.  LDS serves a quarter of what two
// operands from LDS would need.  Results go through LDS to whole runs of a row.
constexpr int kHeldRows = 32;     // of x to a wave
constexpr int kHeldTile = 64;     // rows of w to a turn
constexpr int kHeldWaves = 4;
constexpr int kHeldMost = 1024;   // K

struct HeldParams {
  Linear8Params l;
  int32_t m_blocks, n_splits, turns;  // turns: of all of w
};

template <typename T>
constexpr int kOutStride = kHeldTile + 16 / static_cast<int>(sizeof(T));  // elements of a row of results in LDS

// 32 rows of x as the lanes' pieces: lane l holds bytes 32 k + 16 (l / 32) .. + 15 of row l % 32.
template <typename T, int NK>
struct HeldRows {
  static constexpr int kPitch = 128 * NK + 16;  // of a row in LDS: sixteen rows at one piece meet all banks
  static constexpr int kBytes = 16 * kPitch;    // of a wave: sixteen rows at a time
  i32x4 piece[4 * NK];
  float scale;

  // rows of `T`: a wave reads whole rows, a few at a time, and takes each to 8 bits
  // (WHOLE: a row is a whole number of accesses, and none of them has a branch)
  template <bool WHOLE>
  __device__ __forceinline__ void quantize(const T* x, int64_t m0, int64_t M, int K, int8_t* lds, float* scales) {
    constexpr int VEC = kVec<T>, NV = (128 * NK + 64 * VEC - 1) / (64 * VEC), kAtOnce = NV <= 2 ? 8 : 4;
    const int lane = static_cast<int>(threadIdx.x) & 63;
#pragma unroll
    for (int pass = 0; pass < 2; ++pass) {
#pragma unroll 1
      for (int r = 0; r < 16; r += kAtOnce) {
        Pack<T, VEC> k[kAtOnce][NV];
#pragma unroll
        for (int i = 0; i < kAtOnce; ++i) {
          const int64_t m = min(m0 + 16 * pass + r + i, M - 1);
#pragma unroll
          for (int v = 0; v < NV; ++v) {
            const int at = (v * 64 + lane) * VEC;
            if constexpr (WHOLE) {
              k[i][v].load(x + m * K + min(at, K - VEC));
              continue;
            }
            k[i][v].zero();
            if (at < K) {
              if (at + VEC <= K) k[i][v].load(x + m * K + at);
              else k[i][v].load_part(x + m * K + at, K - at);
            }
          }
        }
#pragma unroll
        for (int i = 0; i < kAtOnce; ++i) {
          float most = 0.f;
#pragma unroll
          for (int v = 0; v < NV; ++v) {
            float f[VEC];
            if (WHOLE && (v * 64 + lane) * VEC >= K) k[i][v].zero();
            k[i][v].get(f);
#pragma unroll
            for (int j = 0; j < VEC; ++j) most = MaxBitsOp::apply(most, __builtin_fabsf(f[j]));
          }
          most = group_reduce<64, MaxBitsOp>(most, 0.f);
          const Quantizer quantizer(most);
          if (lane == 0) scales[16 * pass + r + i] = Quantizer::scale(most, 1.f);
#pragma unroll
          for (int v = 0; v < NV; ++v) {
            const int at = (v * 64 + lane) * VEC;
            if (at >= 128 * NK) continue;
            float f[VEC];
            k[i][v].get(f);
            int q[VEC];
#pragma unroll
            for (int j = 0; j < VEC; ++j) q[j] = quantizer.quantize(f[j]);
            Words<VEC, VEC> w;
#pragma unroll
            for (int j = 0; j < VEC / 4; ++j) w.w[j] = pack4_i8(q[4 * j], q[4 * j + 1], q[4 * j + 2], q[4 * j + 3]);
            *reinterpret_cast<Words<VEC, VEC>*>(lds + (r + i) * kPitch + at) = w;
          }
        }
      }
      if (((lane >> 4) & 1) == pass) {
#pragma unroll
        for (int k = 0; k < 4 * NK; ++k)
          piece[k] = *reinterpret_cast<const i32x4*>(lds + (lane & 15) * kPitch + 32 * k + 16 * (lane >> 5));
      }
    }
    scale = scales[lane & 31];
  }

  // rows in 8 bits
  __device__ __forceinline__ void take(const int8_t* x, int64_t pitch, const float* scales, int64_t m0, int64_t M, int K) {
    const int lane = static_cast<int>(threadIdx.x) & 63;
    const int64_t m = min(m0 + (lane & 31), M - 1);
#pragma unroll
    for (int k = 0; k < 4 * NK; ++k) piece[k] = __builtin_bit_cast(i32x4, load_bytes(x + m * pitch, 32 * k + 16 * (lane >> 5), K));
    scale = scales[m];
  }
};

template <typename T, int NK, bool DYNAMIC>
__global__ __launch_bounds__(64 * kHeldWaves, NK <= (sizeof(T) == 4 ? 5 : 7) ? 2 : 1) void enc_linear8_held(HeldParams p) {
  using Rows = HeldRows<T, NK>;
  constexpr int kTurnBytes = kHeldTile * 128 * NK, kOutBytes = kHeldRows * kOutStride<T> * static_cast<int>(sizeof(T));
  constexpr int kInBytes = kHeldWaves * Rows::kBytes, kRunBytes = kTurnBytes + kHeldWaves * kOutBytes;
  __shared__ __attribute__((aligned(16))) char lds[kInBytes > kRunBytes ? kInBytes : kRunBytes];
  __shared__ __attribute__((aligned(16))) float row_scales[kHeldWaves][kHeldRows];
  __shared__ __attribute__((aligned(16))) float columns[2][kHeldTile];  // scale and bias of a turn's columns
  const Linear8Params& l = p.l;
  const int thread = static_cast<int>(threadIdx.x), lane = thread & 63, wave = thread >> 6, half = lane >> 5;
  // blocks that share rows of x lie behind one another on one XCD
  const int id = static_cast<int>(blockIdx.x), xcds = p.m_blocks < 8 ? 1 : 8;
  const int m_block = id % xcds + xcds * (id / xcds / p.n_splits), split = id / xcds % p.n_splits;
  if (m_block >= p.m_blocks) return;
  // a wave behind the last row works on the last 32 again, and lanes behind it on the last one: what is written twice
  // is written alike, and every store is one that all waves make
  const int64_t rows_left = l.M - kHeldRows;
  const int64_t m0 = min(static_cast<int64_t>(m_block) * (kHeldRows * kHeldWaves) + wave * kHeldRows, rows_left > 0 ? rows_left : 0);
  const int begin = static_cast<int>(static_cast<int64_t>(p.turns) * split / p.n_splits);
  const int end = static_cast<int>(static_cast<int64_t>(p.turns) * (split + 1) / p.n_splits);

  const int piece = thread & 7, row = thread >> 3, key = (row >> 1) & 7;
  const int pieces = (l.K + 15) / 16;
  // x is 0 behind K, so what lies between K and the end of its last piece, or a piece in the place of one behind it, counts
  // for nothing; without a bias, a value of w in its place is not used either
  const int last_piece = 16 * min(8 * (NK - 1) + piece, pieces - 1);
  const T* bias_or_any = l.bias ? static_cast<const T*>(l.bias) : reinterpret_cast<const T*>(l.w);
  u32x4 hold[NK][2];
  float hold_scale;
  T hold_bias;
  const auto fetch = [&](int turn) {
    const int n = min(turn * kHeldTile + (thread & (kHeldTile - 1)), l.N - 1);
    hold_scale = l.w_scale[n];
    hold_bias = bias_or_any[n];
#pragma unroll
    for (int i = 0; i < 2; ++i) {
      const int8_t* from = l.w + static_cast<int64_t>(min(turn * kHeldTile + row + 32 * i, l.N - 1)) * l.w_pitch;
#pragma unroll
      for (int s = 0; s < NK; ++s)
        hold[s][i] = *reinterpret_cast<const u32x4*>(from + (s + 1 < NK ? 128 * s + 16 * piece : last_piece));
    }
  };
  if (begin < end) fetch(begin);

  Rows x;
  if constexpr (DYNAMIC) {
    const T* from = reinterpret_cast<const T*>(l.x);
    int8_t* to = reinterpret_cast<int8_t*>(lds) + wave * Rows::kBytes;
    if (l.K % kVec<T> == 0) x.template quantize<true>(from, m0, l.M, l.K, to, row_scales[wave]);
    else x.template quantize<false>(from, m0, l.M, l.K, to, row_scales[wave]);
  } else {
    x.take(l.x, l.x_pitch, l.x_scale, m0, l.M, l.K);
  }

  T* out = reinterpret_cast<T*>(lds + kTurnBytes) + wave * (kOutBytes / static_cast<int>(sizeof(T)));
  const int r = lane & 31;
  int at[4];
#pragma unroll
  for (int k = 0; k < 4; ++k) at[k] = r * 128 + (((2 * k + half) ^ ((r >> 1) & 7)) << 4);

  const auto stage = [&] {
    __syncthreads();
#pragma unroll
    for (int s = 0; s < NK; ++s)
#pragma unroll
      for (int i = 0; i < 2; ++i)
        *reinterpret_cast<u32x4*>(lds + s * (kHeldTile * 128) + (row + 32 * i) * 128 + ((piece ^ key) << 4)) = hold[s][i];
    if (thread < kHeldTile) {
      columns[0][thread] = hold_scale;
      columns[1][thread] = l.bias ? ElemTraits<T>::load1(&hold_bias) : 0.f;
    }
    __syncthreads();
  };
  // rows of w by rows: a lane's results are row lane % 32 of x and columns 8 (e / 4) + 4 half + e % 4 of the tile
  const auto finish = [&](const i32x16& acc, int tile) {
#pragma unroll
    for (int e = 0; e < 4; ++e) {
      const int c = 32 * tile + 8 * e + 4 * half;
      const f32x4 ws = *reinterpret_cast<const f32x4*>(&columns[0][c]), bias = *reinterpret_cast<const f32x4*>(&columns[1][c]);
      float v[4];
#pragma unroll
      for (int j = 0; j < 4; ++j) v[j] = static_cast<float>(acc[4 * e + j]) * x.scale * ws[j] + bias[j];
      Pack<T, 4> k;
      k.set(v);
      using Four = Words<4 * sizeof(T), 4 * sizeof(T)>;
      *reinterpret_cast<Four*>(out + r * kOutStride<T> + c) = __builtin_bit_cast(Four, k);
    }
  };
  const auto product = [&](i32x16& acc, int tile) {
#pragma unroll
    for (int k = 0; k < 4 * NK; ++k) {
      const i32x4 w = *reinterpret_cast<const i32x4*>(lds + (k / 4) * (kHeldTile * 128) + tile * 4096 + at[k % 4]);
      acc = __builtin_amdgcn_mfma_i32_32x32x32_i8(w, x.piece[k], acc, 0, 0, 0);
    }
  };
  constexpr int VEC = kVec<T>, kLanes = kHeldTile / VEC, kRowsOnce = 64 / kLanes;
  const int c = (lane % kLanes) * VEC, last_row = static_cast<int>(min(l.M - 1 - m0, static_cast<int64_t>(kHeldRows - 1)));
  const auto result = [&](int i, T*& to, Pack<T, VEC>& k) {
    const int row_out = min(i * kRowsOnce + lane / kLanes, last_row);
    const u32x4 v = *reinterpret_cast<const u32x4*>(out + row_out * kOutStride<T> + c);
#pragma unroll
    for (int j = 0; j < 4; ++j) k.w[j] = v[j];
    to = static_cast<T*>(l.y) + (m0 + row_out) * l.N + c;
  };

  // Nothing is on its way here but the first rows of w, for a while now: said so, and the loop's waits count its own
  // accesses alone (0xf70: none left, other counters as they are).
  __builtin_amdgcn_s_waitcnt(0xf70);
  // Whole turns have no branch, so that the wait for the rows of w that were asked for before the results went out is no
  // wait for the results.
  const int whole = min(end, l.N / kHeldTile);
  for (int turn = begin; turn < whole; ++turn) {
    const int n0 = turn * kHeldTile;
    stage();
    fetch(min(turn + 1, p.turns - 1));
    i32x16 acc[2];
#pragma unroll
    for (int e = 0; e < 16; ++e) acc[0][e] = acc[1][e] = 0;
#pragma unroll
    for (int k = 0; k < 4 * NK; ++k)
#pragma unroll
      for (int tile = 0; tile < 2; ++tile) {
        const i32x4 w = *reinterpret_cast<const i32x4*>(lds + (k / 4) * (kHeldTile * 128) + tile * 4096 + at[k % 4]);
        acc[tile] = __builtin_amdgcn_mfma_i32_32x32x32_i8(w, x.piece[k], acc[tile], 0, 0, 0);
      }
    finish(acc[0], 0);
    finish(acc[1], 1);
#pragma unroll
    for (int i = 0; i < kHeldRows / kRowsOnce; ++i) {
      T* to;
      Pack<T, VEC> k;
      result(i, to, k);
      k.store(to + n0);
    }
  }
  if (whole < end) {
    const int n0 = whole * kHeldTile;
    stage();
#pragma unroll 1
    for (int tile = 0; tile < 2 && n0 + 32 * tile < l.N; ++tile) {
      i32x16 acc;
#pragma unroll
      for (int e = 0; e < 16; ++e) acc[e] = 0;
      product(acc, tile);
      finish(acc, tile);
    }
    const int left = l.N - n0 - c;
#pragma unroll 1
    for (int i = 0; i < kHeldRows / kRowsOnce; ++i) {
      T* to;
      Pack<T, VEC> k;
      result(i, to, k);
      if (left >= VEC) k.store(to + n0);
      else if (left > 0) k.store_part(to + n0, left);
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

bool held(const rnnt_linear8_shape_t& s) { return s.K <= kHeldMost; }

// blocks of the held form: several to the same rows while there are few rows
HeldParams held_params(const Linear8Params& q, int64_t* blocks) {
  HeldParams h{};
  h.l = q;
  h.m_blocks = (q.M + kHeldRows * kHeldWaves - 1) / (kHeldRows * kHeldWaves);
  h.turns = (q.N + kHeldTile - 1) / kHeldTile;
  const int want = (512 + h.m_blocks - 1) / h.m_blocks;
  h.n_splits = want < h.turns ? want : h.turns;
  const int64_t groups = h.m_blocks < 8 ? h.m_blocks : (h.m_blocks + 7) / 8 * 8;
  *blocks = groups * h.n_splits;
  return h;
}

template <bool DYNAMIC>
rnnt_status_t launch_held(const Linear8Params& q, const rnnt_linear8_shape_t& s, hipStream_t stream) {
  int64_t blocks;
  const HeldParams h = held_params(q, &blocks);
  return with_dtype(s.dtype, [&](auto t) {
    using T = decltype(t);
#define RNNT_HELD(n)                                                                                                    \
  if (s.K <= 128 * n) {                                                                                                 \
    hipLaunchKernelGGL((enc_linear8_held<T, n, DYNAMIC>), dim3(static_cast<uint32_t>(blocks)), dim3(64 * kHeldWaves), 0, stream, h); \
    return launched();                                                                                                  \
  }
    RNNT_HELD(1)
    RNNT_HELD(2)
    RNNT_HELD(3)
    RNNT_HELD(4)
    RNNT_HELD(5)
    RNNT_HELD(6)
    RNNT_HELD(7)
    RNNT_HELD(8)
#undef RNNT_HELD
    return RNNT_ERR_UNSUPPORTED;
  });
}

rnnt_status_t launch(const Linear8Params& q, const rnnt_linear8_shape_t& s, hipStream_t stream) {
  if (s.M == 0) return RNNT_OK;
  if (held(s)) return launch_held<false>(q, s, stream);
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
  if (check(shape, true) != RNNT_OK || held(shape)) return 0;
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
  if (held(shape)) {
    if (shape.M == 0) return RNNT_OK;
    q.x = static_cast<const int8_t*>(x);
    return launch_held<true>(q, shape, stream);
  }
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
