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

// Rows of any length, already in 8 bits: a tile of 128 x 128 results to a block, 64 x 64 to a wave.  Steps of 128 bytes of
// k go through registers into two buffers of LDS in turn; the 16-byte pieces of a row lie at (piece ^ row % 8), so that the
// 32 rows that a matrix instruction reads at one piece meet all banks.  For rows past kHeldMost alone: at K = 640 the two
// launches, with x in 8 bits through memory between them, took 1969 us where the form below takes 800 (M = 648000).
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

// ---- rows to 8 bits on the way in --------------------------------------------------
// A wave reads a few rows at once, 32 lanes to a row and four elements to a lane, and takes each to 8 bits: 128 NK
// bytes a row, 0 from K on, and its scale.  Rows behind the last are the last again.  WHOLE: K is a multiple of four, and no load
// has a branch.
template <typename T, int NK>
constexpr int kRowsAtOnce = sizeof(T) == 4 ? (NK <= 4 ? 4 : 2) : NK <= 6 ? 8 : 4;

template <typename T, int NK, bool WHOLE>
__device__ __forceinline__ void quantize_rows_of_wave(const T* x, int64_t m0, int64_t M, int K, int8_t* to, int pitch, float* scales) {
  constexpr int kPairs = kRowsAtOnce<T, NK> / 2;
  const int lane = static_cast<int>(threadIdx.x) & 31, half = (static_cast<int>(threadIdx.x) >> 5) & 1;
  Pack<T, 4> k[kPairs][NK];
#pragma unroll
  for (int i = 0; i < kPairs; ++i) {
    const T* row = x + min(m0 + 2 * i + half, M - 1) * K;
#pragma unroll
    for (int v = 0; v < NK; ++v) {
      const int at = (v * 32 + lane) * 4;
      if constexpr (WHOLE) {
        k[i][v].load(row + min(at, K - 4));
      } else {
        k[i][v].zero();
        if (at < K) k[i][v].load_part(row + at, min(K - at, 4));
      }
    }
  }
#pragma unroll
  for (int i = 0; i < kPairs; ++i) {
    float most = 0.f;
    uint32_t most_bits = 0;
#pragma unroll
    for (int v = 0; v < NK; ++v) {
      if (WHOLE && (v * 32 + lane) * 4 >= K) k[i][v].zero();
#pragma unroll
      for (int j = 0; j < Pack<T, 4>::kWords; ++j) {
        if constexpr (sizeof(T) == 2) raise_most16(most_bits, k[i][v].w[j]);
        else most = MaxBitsOp::apply(most, __uint_as_float(k[i][v].w[j] & 0x7fffffffu));
      }
    }
    if constexpr (sizeof(T) == 2) most = most16<T>(most_bits);
    most = group_reduce<32, MaxBitsOp>(most, 0.f);
    const Quantizer quantizer(most);
    if (lane == 0) scales[2 * i + half] = Quantizer::scale(most, 1.f);
#pragma unroll
    for (int v = 0; v < NK; ++v) {
      float f[4];
      k[i][v].get(f);
      *reinterpret_cast<uint32_t*>(to + (2 * i + half) * pitch + (v * 32 + lane) * 4) = quantizer.four(f);
    }
  }
}

// ---- rows held in registers ----------------------------------------------------
// For rows of up to 1024 a block of four waves keeps 128 rows of x, 32 to a wave, in registers in the matrix
// instruction's order, and passes over its share of w, 64 rows at a time through LDS.  x is read once, whatever N is,
// and taken to 8 bits on the way in, so no copy of it in 8 bits goes through memory; results go through LDS to whole runs of
// a row.  648000 rows of 640 bf16 to 1025: 800 us, 1.06 POP/s and 2.7 TB/s, the product alone by the library 933.  The
// matrix units are busy for 32 % of 1.30 million cycles, LDS for 43 %, the vector units for 41 %: without quantizing 190 us
// less, without storing 190, without both 440 in all.  Tried, and no faster: 64 rows to a wave (half the reads of w, one wave to a
// SIMD: 900 us, with a turn's results among the next one's products too), 32 rows of w to a turn and three blocks to a CU (890-1040),
// half the blocks out of step with the others (815), results stored past the caches (1300).
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

  // rows of `T`, sixteen at a time through LDS
  template <bool WHOLE>
  __device__ __forceinline__ void quantize(const T* x, int64_t m0, int64_t M, int K, int8_t* lds, float* scales) {
    const int lane = static_cast<int>(threadIdx.x) & 63;
#pragma unroll
    for (int pass = 0; pass < 2; ++pass) {
#pragma unroll 1
      for (int r = 0; r < 16; r += kRowsAtOnce<T, NK>)
        quantize_rows_of_wave<T, NK, WHOLE>(x, m0 + 16 * pass + r, M, K, lds + r * kPitch, kPitch, scales + 16 * pass + r);
      wave_exchange();
      if (((lane >> 4) & 1) == pass) {
#pragma unroll
        for (int k = 0; k < 4 * NK; ++k)
          piece[k] = *reinterpret_cast<const i32x4*>(lds + (lane & 15) * kPitch + 32 * k + 16 * (lane >> 5));
      }
      wave_exchange();  // the next sixteen rows take their place
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
  constexpr int kTiles = kHeldTile / 32;
  u32x4 hold[NK][kTiles];
  float hold_scale;
  T hold_bias;
  const auto fetch = [&](int turn) {
    const int n = min(turn * kHeldTile + (thread & (kHeldTile - 1)), l.N - 1);
    hold_scale = l.w_scale[n];
    hold_bias = bias_or_any[n];
#pragma unroll
    for (int i = 0; i < kTiles; ++i) {
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
    if (l.K % 4 == 0) x.template quantize<true>(from, m0, l.M, l.K, to, row_scales[wave]);
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
      for (int i = 0; i < kTiles; ++i)
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
    i32x16 acc[kTiles];
#pragma unroll
    for (int tile = 0; tile < kTiles; ++tile)
#pragma unroll
      for (int e = 0; e < 16; ++e) acc[tile][e] = 0;
#pragma unroll
    for (int k = 0; k < 4 * NK; ++k)
#pragma unroll
      for (int tile = 0; tile < kTiles; ++tile) {
        const i32x4 w = *reinterpret_cast<const i32x4*>(lds + (k / 4) * (kHeldTile * 128) + tile * 4096 + at[k % 4]);
        acc[tile] = __builtin_amdgcn_mfma_i32_32x32x32_i8(w, x.piece[k], acc[tile], 0, 0, 0);
      }
#pragma unroll
    for (int tile = 0; tile < kTiles; ++tile) finish(acc[tile], tile);
    wave_exchange();  // the wave's own rows of results; the next turn's go there behind a barrier
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
    for (int tile = 0; tile < kTiles && n0 + 32 * tile < l.N; ++tile) {
      i32x16 acc;
#pragma unroll
      for (int e = 0; e < 16; ++e) acc[e] = 0;
      product(acc, tile);
      finish(acc, tile);
    }
    wave_exchange();
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

// ---- few rows ------------------------------------------------------------------
// A block takes 16 or 32 rows of x into LDS, in 8 bits, and multiplies them with a few tiles of 16 rows of w, which go from
// memory to registers and nowhere else.  Where tiles are fewer than CUs the four waves share out k, and their sums meet in
// LDS; else they share out the tiles.  The first pieces of w are asked for before x is there.  Bound by the way from launch to
// store, three round trips to memory: 16 rows of 640 f16 to 1025 take 6.9 us in one launch, 2.8 + 10.3 in two.
struct FewParams {
  Linear8Params l;
  int32_t pitch;        // of a row of x in LDS: whole steps of 64 bytes, and 16, so that sixteen rows meet all banks
  int32_t tiles, blocks, tiles_of_wave;  // of w; blocks to the same rows of x; 0: the waves share out k
};
constexpr int kFewAhead = 4;
constexpr int kFewLds = 56000;  // and the waves' sums, within the 64 KB that a launch has without asking

template <typename T, int MT, int NV, bool DYNAMIC>
__global__ __launch_bounds__(256) void enc_linear8_few(FewParams p) {
  extern __shared__ __attribute__((aligned(16))) char lds[];
  __shared__ float scales[16 * MT];
  __shared__ __attribute__((aligned(16))) i32x4 sums[4][MT * 64];
  const Linear8Params& l = p.l;
  const int thread = static_cast<int>(threadIdx.x), lane = thread & 63, wave = __builtin_amdgcn_readfirstlane(thread >> 6);
  const int64_t m0 = static_cast<int64_t>(blockIdx.x / p.blocks) * (16 * MT);
  const int block = static_cast<int>(blockIdx.x % p.blocks);
  const bool shared_k = p.tiles_of_wave == 0;
  const int steps = (l.K + 63) / 64, pieces = (l.K + 15) / 16;
  const int first = shared_k ? block : (block * 4 + wave) * p.tiles_of_wave;
  const int last = shared_k ? block + 1 : min(first + p.tiles_of_wave, p.tiles);
  const int step0 = shared_k ? wave : 0, by = shared_k ? 4 : 1;
  // x is 0 behind K: a piece in the place of one behind it counts for nothing
  const auto w_piece = [&](int tile, int step) {
    const int n = min(tile * 16 + (lane & 15), l.N - 1), piece = min(4 * step + (lane >> 4), pieces - 1);
    return *reinterpret_cast<const i32x4*>(l.w + n * l.w_pitch + 16 * piece);
  };
  i32x4 w[kFewAhead];
  const auto ahead = [&](int tile) {
#pragma unroll
    for (int i = 0; i < kFewAhead; ++i) w[i] = w_piece(min(tile, p.tiles - 1), min(step0 + i * by, steps - 1));
  };
  ahead(first);

  // x: a wave takes every fourth row, a few at once
  if constexpr (DYNAMIC) {
    constexpr int kAtOnce = NV <= 4 ? 4 : sizeof(T) == 2 ? 32 / NV : 16 / NV;
#pragma unroll 1
    for (int r0 = 0; r0 < 4 * MT; r0 += kAtOnce) {
      Pack<T, 4> k[kAtOnce][NV];
#pragma unroll
      for (int i = 0; i < kAtOnce; ++i) {
        const T* row = reinterpret_cast<const T*>(l.x) + min(m0 + 4 * (r0 + i) + wave, static_cast<int64_t>(l.M) - 1) * l.K;
#pragma unroll
        for (int v = 0; v < NV; ++v) {
          const int at = (v * 64 + lane) * 4;
          k[i][v].zero();
          if (at + 4 <= l.K) k[i][v].load(row + at);
          else if (at < l.K) k[i][v].load_part(row + at, l.K - at);
        }
      }
#pragma unroll
      for (int i = 0; i < kAtOnce; ++i) {
        const int row = 4 * (r0 + i) + wave;
        float most = 0.f;
        uint32_t most_bits = 0;
#pragma unroll
        for (int v = 0; v < NV; ++v)
#pragma unroll
          for (int j = 0; j < Pack<T, 4>::kWords; ++j) {
            if constexpr (sizeof(T) == 2) raise_most16(most_bits, k[i][v].w[j]);
            else most = MaxBitsOp::apply(most, __uint_as_float(k[i][v].w[j] & 0x7fffffffu));
          }
        if constexpr (sizeof(T) == 2) most = most16<T>(most_bits);
        most = group_reduce<64, MaxBitsOp>(most, 0.f);
        const Quantizer quantizer(most);
        if (lane == 0) scales[row] = Quantizer::scale(most, 1.f);
#pragma unroll
        for (int v = 0; v < NV; ++v) {
          const int at = (v * 64 + lane) * 4;
          float f[4];
          k[i][v].get(f);
          if (at < 64 * steps) *reinterpret_cast<uint32_t*>(lds + row * p.pitch + at) = quantizer.four(f);
        }
      }
    }
  } else {
    for (int i = thread; i < 16 * MT * 4 * steps; i += 256) {
      const int row = i / (4 * steps), piece = i - row * 4 * steps;
      const int64_t m = min(m0 + row, static_cast<int64_t>(l.M) - 1);
      *reinterpret_cast<u32x4*>(lds + row * p.pitch + 16 * piece) = load_bytes(l.x + m * l.x_pitch, 16 * piece, l.K);
    }
    if (thread < 16 * MT) scales[thread] = l.x_scale[min(m0 + thread, static_cast<int64_t>(l.M) - 1)];
  }
  __syncthreads();

  // rows of w by rows: a lane's results are row lane % 16 of x and columns 4 (lane / 16) + e
  const auto finish = [&](const i32x4& acc, int tile, int mt, int of) {
    const int64_t m = m0 + 16 * mt + (of & 15);
    const int n = tile * 16 + 4 * (of >> 4), left = l.N - n;
    if (m >= l.M || left <= 0) return;
    const float scale = scales[16 * mt + (of & 15)];
    float v[4];
#pragma unroll
    for (int e = 0; e < 4; ++e) {
      const int at = min(n + e, l.N - 1);
      const float bias = l.bias ? ElemTraits<T>::load1(static_cast<const T*>(l.bias) + at) : 0.f;
      v[e] = static_cast<float>(acc[e]) * scale * l.w_scale[at] + bias;
    }
    Pack<T, 4> k;
    k.set(v);
    T* to = static_cast<T*>(l.y) + m * l.N + n;
    if (left >= 4) k.store(to);
    else k.store_part(to, left);
  };
  const char* x = lds + (lane & 15) * p.pitch + 16 * (lane >> 4);
#pragma unroll 1
  for (int tile = first; tile < last; ++tile) {
    i32x4 acc[MT];
#pragma unroll
    for (int mt = 0; mt < MT; ++mt) acc[mt] = i32x4{0, 0, 0, 0};
#pragma unroll 1
    for (int s0 = step0; s0 < steps; s0 += by * kFewAhead) {
#pragma unroll
      for (int i = 0; i < kFewAhead; ++i) {
        const int step = s0 + i * by;
        const i32x4 now = w[i];
        const bool more = step + by * kFewAhead < steps;
        w[i] = w_piece(more ? tile : min(tile + 1, p.tiles - 1), more ? step + by * kFewAhead : min(step0 + i * by, steps - 1));
        if (step >= steps) continue;
#pragma unroll
        for (int mt = 0; mt < MT; ++mt)
          acc[mt] = __builtin_amdgcn_mfma_i32_16x16x64_i8(now, *reinterpret_cast<const i32x4*>(x + 16 * mt * p.pitch + 64 * step), acc[mt], 0, 0, 0);
      }
    }
    if (!shared_k) {
#pragma unroll
      for (int mt = 0; mt < MT; ++mt) finish(acc[mt], tile, mt, lane);
    } else {
#pragma unroll
      for (int mt = 0; mt < MT; ++mt) sums[wave][64 * mt + lane] = acc[mt];
    }
  }
  if (shared_k) {
    __syncthreads();
    if (thread < 64 * MT) {
      const i32x4 total = sums[0][thread] + sums[1][thread] + sums[2][thread] + sums[3][thread];
      finish(total, block, thread >> 6, thread & 63);
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

// The tiles of sixteen rows of x that a block of the form for few rows takes, 0: another form.  Tiles of sixteen by sixteen
// results up to which it is the faster one (us, this form and the next; K x N): 640 x 1025, M = 16 6.3 and 13.0, M = 256
// 11.7 and 13.1, M = 512 27 and 13.4; 512 x 2048, M = 256 8.7 and 11.2, M = 512 15.1 and 11.5; 1024 x 256, M = 2048 10.5 and
// 18.9; rows of two launches, 2048 x 512, M = 1024 18.9 and 29.5, M = 2048 26 and 30, M = 4096 41 and 32.
int few(const rnnt_linear8_shape_t& s) {
  const int64_t pitch = (static_cast<int64_t>(s.K) + 63) / 64 * 64 + 16, tiles = (static_cast<int64_t>(s.N) + 15) / 16;
  const int64_t all = (static_cast<int64_t>(s.M) + 15) / 16 * tiles;
  if (s.K > 256 * 16 || pitch * 16 > kFewLds || all > (held(s) ? 2048 : 4096)) return 0;
  // sixteen rows to a block, which come in one round, while that makes no more than four blocks to a CU
  return all <= 1024 || pitch * 32 > kFewLds ? 1 : 2;
}

template <bool DYNAMIC>
rnnt_status_t launch_few(const Linear8Params& q, const rnnt_linear8_shape_t& s, int mt, hipStream_t stream) {
  FewParams p{};
  p.l = q;
  p.pitch = (s.K + 63) / 64 * 64 + 16;
  p.tiles = (s.N + 15) / 16;
  const int64_t m_blocks = (s.M + 16 * mt - 1) / (16 * mt);
  // two blocks to a CU while that is not one tile to a block
  const int64_t want = m_blocks * p.tiles / 512;
  p.tiles_of_wave = want <= 1 ? 0 : static_cast<int32_t>((want + 3) / 4);
  p.blocks = p.tiles_of_wave == 0 ? p.tiles : (p.tiles + 4 * p.tiles_of_wave - 1) / (4 * p.tiles_of_wave);
  const dim3 grid(static_cast<uint32_t>(m_blocks * p.blocks));
  const size_t lds = static_cast<size_t>(p.pitch) * 16 * mt;
  return with_dtype(s.dtype, [&](auto t) {
    using T = decltype(t);
#define RNNT_FEW(n, nv)                                                                                       \
  if (mt == n && s.K <= 256 * nv) {                                                                           \
    hipLaunchKernelGGL((enc_linear8_few<T, n, nv, DYNAMIC>), grid, dim3(256), lds, stream, p);                \
    return launched();                                                                                        \
  }
    RNNT_FEW(1, 4)
    RNNT_FEW(2, 4)
    RNNT_FEW(1, 8)
    RNNT_FEW(2, 8)
    RNNT_FEW(1, 16)
#undef RNNT_FEW
    return RNNT_ERR_UNSUPPORTED;
  });
}

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
  if (const int mt = few(s)) return launch_few<false>(q, s, mt, stream);
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
  if (check(shape, true) != RNNT_OK || held(shape) || few(shape)) return 0;
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
  if (held(shape) || few(shape)) {
    if (shape.M == 0) return RNNT_OK;
    q.x = static_cast<const int8_t*>(x);
    if (const int mt = few(shape)) return launch_few<true>(q, shape, mt, stream);
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
