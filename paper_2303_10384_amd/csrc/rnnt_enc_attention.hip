// Attention of a chunk of new tokens over a paged cache (contract in include/rnnt_encoder_mi355x.h).
#include <hip/hip_runtime.h>

#include <cstdint>

#include "rnnt_enc.h"
#include "rnnt_pages.h"

namespace rnnt {
namespace {

typedef float f32x4 __attribute__((ext_vector_type(4)));
typedef _Float16 f16x8 __attribute__((ext_vector_type(8)));
typedef __bf16 bf16x8 __attribute__((ext_vector_type(8)));
typedef short i16x4 __attribute__((ext_vector_type(4)));

struct AttentionParams {
  const void *q, *k, *v;
  void *k_cache, *v_cache, *out;
  const int32_t *lens, *cached, *pages;
  float* part;  // of the splits: sums over values, then {maximum, sum of weights}
  int64_t q_stride_b, q_stride_t, q_stride_h, k_stride_b, k_stride_t, k_stride_h, v_stride_b, v_stride_t, v_stride_h;
  int32_t B, L, Hq, Hkv, G, D, shift, table, num_pages, causal, left;
  int32_t rows, tiles, splits;  // rows of a tile, tiles of an utterance's head of keys, blocks to a tile
  float scale;                  // times log2 e
};

typedef float f32x16 __attribute__((ext_vector_type(16)));

constexpr float kNegInf = -__builtin_inff();
constexpr int kRowTile = 16;  // rows (tokens times the heads that share keys) to a block
constexpr int kKeys = 32;     // keys to a wave's step
constexpr int kWaves = 4;

// Weights are rounded to the values' type for their product.  Float16 ends at 2^-24, and the many small weights of a long
// cache beside one large one would end with it, while the sum that divides them has them whole: they are formed 2^kLift times
// as large, in the product and the sum alike, which the quotient and the joins do not see.  The largest is 1 in the kernel
// of sixteen rows; in the wide one up to 2^kLag, by which the maximum may lag behind.  65504 is the end on the other side.
// (Weights of 2^-25.25 to 2^-26 beside one of 1: without the factor their share of the result is 0.)
template <typename T>
constexpr int kLift = __is_same(T, f16_t) ? 14 : 0;
template <typename T>
constexpr int kLag = __is_same(T, f16_t) ? 4 : 8;
template <typename T>
constexpr int kWideLift = __is_same(T, f16_t) ? 11 : 0;

// ---- an utterance and its tile of rows ------------------------------------------
// Row r of an utterance's head of keys is token r / G and query head h G + r % G.
struct Tile {
  int b, h, tile, split;
  int n, cached, end;    // new tokens, cached ones, all
  int state;             // 1 there are valid rows, 0 none, -1 bad lengths
  PageTable table;

  __device__ __forceinline__ Tile(const AttentionParams& p, int64_t unit, int split_) : split(split_) {
    tile = p.tiles - 1 - static_cast<int>(unit % p.tiles);  // the later ones, which see more, begin first
    const int bh = static_cast<int>(unit / p.tiles);
    b = bh / p.Hkv;
    h = bh - b * p.Hkv;
    n = p.lens ? p.lens[b] : p.L;
    cached = p.cached[b];
    table = PageTable{p.pages + static_cast<int64_t>(b) * p.table, p.table, p.num_pages, p.shift};
    const bool fits = lengths_fit(n, p.L, cached, static_cast<int64_t>(p.table) << p.shift);
    end = cached + n;
    state = !fits ? -1 : static_cast<int64_t>(tile) * p.rows < static_cast<int64_t>(n) * p.G;
  }
};

// The row of a key: of the cache, or (the top bit) the chunk's own token.
constexpr uint32_t kNewRow = 0x80000000u, kBadRow = 0xffffffffu;
__device__ __forceinline__ uint32_t row_of(const AttentionParams& p, const Tile& t, int pos) {
  const int id = t.table.page_of(pos);
  if (id < 0) return kBadRow;
  return pos >= t.cached ? kNewRow | static_cast<uint32_t>(pos - t.cached) : cache_row(id, p.Hkv, t.h, pos, p.shift);
}

// A key's row without a branch: one of two bases, and one product.  A bad row is the chunk's first, a valid address; its
// key is NaN wherever it is seen.
template <typename T>
__device__ __forceinline__ const T* row_pointer(const T* cache, const T* fresh, int64_t stride_t, uint32_t row, int D) {
  const bool own = row & kNewRow;
  const uint32_t index = row == kBadRow ? 0u : row & ~kNewRow, by = own ? static_cast<uint32_t>(stride_t) : static_cast<uint32_t>(D);
  return (own ? fresh : cache) + static_cast<uint64_t>(index) * by;
}

// ---- eight elements in a matrix instruction's order ------------------------------
// A 16 x 16 product over 32: lane l holds row (or column) l % 16 and elements 8 (l / 16) .. + 7.  Float32
// takes eight instructions over 4, which add up the same 32 in another order.
template <typename T>
struct Eight {
  u32x4 w[sizeof(T) / 2];

  __device__ __forceinline__ void zero() {
#pragma unroll
    for (auto& x : w) x = u32x4{0, 0, 0, 0};
  }
  __device__ __forceinline__ void load(const T* p) {
#pragma unroll
    for (int i = 0; i < static_cast<int>(sizeof(T) / 2); ++i) w[i] = reinterpret_cast<const u32x4*>(p)[i];
  }
  __device__ __forceinline__ void store(T* p) const {
#pragma unroll
    for (int i = 0; i < static_cast<int>(sizeof(T) / 2); ++i) reinterpret_cast<u32x4*>(p)[i] = w[i];
  }
  __device__ __forceinline__ void set(const float* f) {
    if constexpr (sizeof(T) == 4) {
#pragma unroll
      for (int i = 0; i < 8; ++i) w[i / 4][i % 4] = __float_as_uint(f[i]);
    } else {
#pragma unroll
      for (int i = 0; i < 4; ++i) w[0][i] = Pack<T, 2>::pack2(f[2 * i], f[2 * i + 1]);
    }
  }
  // (16 bits) infinities and NaN become 0
  __device__ __forceinline__ void clear_odd() {
    constexpr uint32_t kExp = __is_same(T, bf16_t) ? 0x7f80u : 0x7c00u;
#pragma unroll
    for (int i = 0; i < 4; ++i) {
      const uint32_t x = w[0][i];
      w[0][i] = ((x & kExp) == kExp ? 0u : x & 0xffffu) | ((x >> 16 & kExp) == kExp ? 0u : x & 0xffff0000u);
    }
  }
  // an infinity or NaN among them
  __device__ __forceinline__ bool odd() const {
    constexpr uint32_t kExp = sizeof(T) == 4 ? 0x7f800000u : __is_same(T, bf16_t) ? 0x7f80u : 0x7c00u;
    bool any = false;
#pragma unroll
    for (int i = 0; i < static_cast<int>(sizeof(T) / 2); ++i)
#pragma unroll
      for (int j = 0; j < 4; ++j) {
        any |= (w[i][j] & kExp) == kExp;
        if constexpr (sizeof(T) == 2) any |= (w[i][j] & (kExp << 16)) == (kExp << 16);
      }
    return any;
  }
};

template <typename T>
__device__ __forceinline__ f32x4 mma(const Eight<T>& a, const Eight<T>& b, f32x4 c) {
  if constexpr (__is_same(T, bf16_t)) {
    return __builtin_amdgcn_mfma_f32_16x16x32_bf16(__builtin_bit_cast(bf16x8, a.w[0]), __builtin_bit_cast(bf16x8, b.w[0]), c, 0, 0, 0);
  } else if constexpr (__is_same(T, f16_t)) {
    return __builtin_amdgcn_mfma_f32_16x16x32_f16(__builtin_bit_cast(f16x8, a.w[0]), __builtin_bit_cast(f16x8, b.w[0]), c, 0, 0, 0);
  } else {
#pragma unroll
    for (int i = 0; i < 8; ++i)
      c = __builtin_amdgcn_mfma_f32_16x16x4f32(__uint_as_float(a.w[i / 4][i % 4]), __uint_as_float(b.w[i / 4][i % 4]), c, 0, 0, 0);
    return c;
  }
}

// ---- values through LDS ------------------------------------------------------------
// Rows of values lie in LDS as they do in memory, each 32 bytes (16 in float32) longer, so that the four rows that a
// group of lanes reads at once, and the groups' rows, meet different banks.
template <typename T, int DT>
struct Values {
  static constexpr int kStride = DT * 32 + (sizeof(T) == 4 ? 4 : 16);  // elements
  static constexpr int kElems = kKeys * kStride;

  // values of channel 16 c + lane % 16 and the eight keys of the lane's group g: 4 g + j and 16 + 4 g + j
  __device__ __forceinline__ static Eight<T> column(const T* lds, int c, int lane) {
    Eight<T> e;
    const int g = lane >> 4, i = lane & 15;
    if constexpr (sizeof(T) == 4) {
#pragma unroll
      for (int j = 0; j < 8; ++j)
        e.w[j / 4][j % 4] = *reinterpret_cast<const uint32_t*>(lds + (16 * (j / 4) + 4 * g + j % 4) * kStride + 16 * c + i);
    } else {
      // sixteen lanes read four rows of sixteen channels, and each gets the four of its own channel
#pragma unroll
      for (int half = 0; half < 2; ++half) {
        const T* at = lds + (16 * half + 4 * g + (i >> 2)) * kStride + 16 * c + 4 * (i & 3);
        const i16x4 t = __builtin_amdgcn_ds_read_tr16_b64_v4i16((__attribute__((address_space(3))) i16x4*)at);
        const auto two = __builtin_bit_cast(uint2, t);
        e.w[0][2 * half] = two.x;
        e.w[0][2 * half + 1] = two.y;
      }
    }
    return e;
  }
};

__device__ __forceinline__ float across_groups_max(float x) {
  x = __builtin_fmaxf(x, __shfl_xor(x, 16));
  return __builtin_fmaxf(x, __shfl_xor(x, 32));
}
// the larger of a lane's and the other half's
__device__ __forceinline__ float halves_max(float x) {
  const auto r = __builtin_amdgcn_permlane32_swap(__float_as_uint(x), __float_as_uint(x), false, false);
  return __builtin_fmaxf(__uint_as_float(r[0]), __uint_as_float(r[1]));
}
__device__ __forceinline__ float across_groups_sum(float x) {
  x += __shfl_xor(x, 16);
  return x + __shfl_xor(x, 32);
}

// ---- the chunk's own keys and values, into the cache ---------------------------------
// The tokens whose first row lies in the tile, by the tile's first split.  Nothing in this launch reads them there.  They are
// asked for and stored apart: sixteen rows' come before the attention's own rows and go after its last, and neither waits for the other.
template <typename T, int N>
struct CacheWrite {
  Eight<T> k[N], v[N];
  int id[N];

  __device__ __forceinline__ static int tokens(const AttentionParams& p, const Tile& t, int& first) {
    first = (t.tile * p.rows + p.G - 1) / p.G;
    return min(((t.tile + 1) * p.rows + p.G - 1) / p.G, t.n) - first;
  }
  __device__ __forceinline__ void ask(const AttentionParams& p, const Tile& t, int round) {
    int first;
    const int pieces = p.D / 8, total = tokens(p, t, first) * pieces;
#pragma unroll
    for (int n = 0; n < N; ++n) {
      const int i = (round * N + n) * 64 * kWaves + static_cast<int>(threadIdx.x);
      if (i >= total) continue;
      const int token = first + i / pieces, c = 8 * (i % pieces);
      id[n] = t.table.pages[(t.cached + token) >> p.shift];
      k[n].load(static_cast<const T*>(p.k) + t.b * p.k_stride_b + token * p.k_stride_t + t.h * p.k_stride_h + c);
      v[n].load(static_cast<const T*>(p.v) + t.b * p.v_stride_b + token * p.v_stride_t + t.h * p.v_stride_h + c);
    }
  }
  __device__ __forceinline__ void store(const AttentionParams& p, const Tile& t, int round) const {
    int first;
    const int pieces = p.D / 8, total = tokens(p, t, first) * pieces;
#pragma unroll
    for (int n = 0; n < N; ++n) {
      const int i = (round * N + n) * 64 * kWaves + static_cast<int>(threadIdx.x);
      if (i >= total || static_cast<uint32_t>(id[n]) >= static_cast<uint32_t>(p.num_pages)) continue;
      const int token = first + i / pieces, c = 8 * (i % pieces);
      const int64_t to = static_cast<int64_t>(cache_row(id[n], p.Hkv, t.h, t.cached + token, p.shift)) * p.D + c;
      k[n].store(static_cast<T*>(p.k_cache) + to);
      v[n].store(static_cast<T*>(p.v_cache) + to);
    }
  }
};

// ---- attention ------------------------------------------------------------------------
// A block of four waves takes sixteen rows and, of their keys, every wave every fourth step of 32.  Scores are formed
// transposed, keys by rows, so that a lane holds one row's scores and the weights are already where the product with
// the values takes them: group g's eight keys are 4 g + j and 16 + 4 g + j in both.  The waves' maxima, sums and
// products meet in LDS, or, where a sequence is split among blocks, in memory.  One token of three sequences of 60013 keys,
// 2 heads of 128 f16: 39.5 us (184 MB, 4.7 TB/s; a step's pages are waited for before its rows are asked for) and 5.6 for the join; 64 chunks of 16 tokens, 8 heads of 64 bf16, 256 keys
// before them: 14 us, most of it the way lengths -> page -> rows -> products -> join of blocks that have two steps to a wave.
template <typename T, int DT>
__global__ __launch_bounds__(64 * kWaves) void enc_attention(AttentionParams p) {
  using V = Values<T, DT>;
  constexpr int kWrites = DT <= 4 ? 1 : 2;  // sixteen tokens of up to 4 DT pieces
  constexpr int kPieces = 4 * DT, kLoads = kKeys * kPieces / 64;  // 16-byte pieces of a row (float32: pairs of them)
  constexpr int kValueBytes = kWaves * V::kElems * static_cast<int>(sizeof(T));
  constexpr int kJoinBytes = kWaves * 32 * DT * 17 * 4;
  __shared__ __attribute__((aligned(16))) char lds[kValueBytes > kJoinBytes ? kValueBytes : kJoinBytes];
  __shared__ float stat[2][kWaves][16];
  const int lane = static_cast<int>(threadIdx.x) & 63, wave = __builtin_amdgcn_readfirstlane(static_cast<int>(threadIdx.x) >> 6);
  const int g = lane >> 4, col = lane & 15;
  const Tile t(p, blockIdx.x / p.splits, static_cast<int>(blockIdx.x % p.splits));
  CacheWrite<T, kWrites> write;
  const bool writes = t.split == 0 && t.state == 1;
  if (writes) write.ask(p, t, 0);

  const int rows = p.L * p.G, row0 = t.tile * kRowTile;
  float m = kNegInf, sum = 0.f;
  f32x4 acc[2 * DT];
#pragma unroll
  for (int c = 0; c < 2 * DT; ++c) acc[c] = f32x4{0.f, 0.f, 0.f, 0.f};

  if (t.state == 1) {
    const int valid_rows = min(t.n * p.G - row0, kRowTile);
    // a lane behind the last valid row works on that one again; its result is dropped
    const int my_row = row0 + min(col, valid_rows - 1), my_token = my_row / p.G;
    const Seen mine(t.cached + my_token, t.end, p.causal != 0, p.left);
    const Seen first(t.cached + row0 / p.G, t.end, p.causal != 0, p.left);
    const Seen last(t.cached + (row0 + valid_rows - 1) / p.G, t.end, p.causal != 0, p.left);
    const int lo = first.lo, hi = last.hi;        // keys that some row sees
    const int all_lo = last.lo, all_hi = first.hi;  // ... that every row sees
    const int steps = (hi - lo + kKeys - 1) / kKeys;
    const int begin = static_cast<int>(static_cast<int64_t>(steps) * t.split / p.splits) + wave;
    const int stop = static_cast<int>(static_cast<int64_t>(steps) * (t.split + 1) / p.splits);

    const T* k_new = static_cast<const T*>(p.k) + t.b * p.k_stride_b + t.h * p.k_stride_h;
    const T* v_new = static_cast<const T*>(p.v) + t.b * p.v_stride_b + t.h * p.v_stride_h;
    const T *k_cache = static_cast<const T*>(p.k_cache), *v_cache = static_cast<const T*>(p.v_cache);
    T* values = reinterpret_cast<T*>(lds) + wave * V::kElems;

    Eight<T> q[DT];
    {
      const T* from = static_cast<const T*>(p.q) + t.b * p.q_stride_b + my_token * p.q_stride_t +
                      (t.h * p.G + my_row - my_token * p.G) * p.q_stride_h;
#pragma unroll
      for (int d = 0; d < DT; ++d) {
        q[d].zero();
        if (32 * d + 8 * g < p.D) q[d].load(from + 32 * d + 8 * g);
      }
    }

    Eight<T> kk[2][DT], vv[kLoads];
    uint32_t bad = 0;  // keys of the step whose page is none
    const auto fetch = [&](int step) {
      const uint32_t row = row_of(p, t, min(lo + step * kKeys + (lane & 31), hi - 1));
      bad = static_cast<uint32_t>(__ballot(row == kBadRow));
#pragma unroll
      for (int i = 0; i < 2; ++i) {
        const T* from = row_pointer(k_cache, k_new, p.k_stride_t, __shfl(row, 16 * i + col), p.D);
#pragma unroll
        for (int d = 0; d < DT; ++d) {
          kk[i][d].zero();
          if (32 * d + 8 * g < p.D) kk[i][d].load(from + 32 * d + 8 * g);
        }
      }
#pragma unroll
      for (int i = 0; i < kLoads; ++i) {
        const int piece = i * 64 + lane, key = piece / kPieces, c = 8 * (piece % kPieces);
        const T* from = row_pointer(v_cache, v_new, p.v_stride_t, __shfl(row, key), p.D);
        vv[i].zero();
        if (c < p.D) vv[i].load(from + c);
      }
    };

    if (begin < stop) fetch(begin);
    for (int step = begin; step < stop; step += kWaves) {
      const int base = lo + step * kKeys;
      const bool mixed = base < all_lo || base + kKeys > all_hi || bad != 0;  // some row does not see some key
      const uint32_t bad_now = bad;
      f32x4 s[2];
#pragma unroll
      for (int i = 0; i < 2; ++i) {
        s[i] = f32x4{0.f, 0.f, 0.f, 0.f};
#pragma unroll
        for (int d = 0; d < DT; ++d) s[i] = mma(kk[i][d], q[d], s[i]);
      }
      bool odd = false;
      wave_exchange();  // the step before has read its values
#pragma unroll
      for (int i = 0; i < kLoads; ++i) {
        const int piece = i * 64 + lane;
        if (mixed) odd |= vv[i].odd();
        vv[i].store(values + piece / kPieces * V::kStride + 8 * (piece % kPieces));
      }
      wave_exchange();
      const bool careful = mixed && __ballot(odd) != 0;
      if (step + kWaves < stop) fetch(step + kWaves);

      float w[8], most = kNegInf;
#pragma unroll
      for (int j = 0; j < 8; ++j) {
        const int at = 16 * (j / 4) + 4 * g + j % 4;
        w[j] = s[j / 4][j % 4] * p.scale;
        if (mixed) {
          if (bad_now >> at & 1) w[j] = __builtin_nanf("");
          if (!mine.holds(base + at)) w[j] = kNegInf;
        }
        most = __builtin_fmaxf(most, w[j]);
      }
      const float grown = __builtin_fmaxf(m, across_groups_max(most)), by = grown == kNegInf ? 0.f : grown;
      if (__ballot(grown != m)) {
        const float shrink = fast_exp2(m - by);
        sum *= shrink;
#pragma unroll
        for (int c = 0; c < 2 * DT; ++c) acc[c] *= shrink;
        m = grown;
      }
#pragma unroll
      for (int j = 0; j < 8; ++j) {
        w[j] = fast_exp2(w[j] - by) * static_cast<float>(1 << kLift<T>);
        sum += w[j];
      }
      if (!careful) {
        // weights of 16 bits, as the values are: off by half a step each, which the sum over keys averages
        Eight<T> weights;
        weights.set(w);
#pragma unroll
        for (int c = 0; c < 2 * DT; ++c) acc[c] = mma(V::column(values, c, lane), weights, acc[c]);
      } else {
        // an infinity or NaN among the values, which a weight of 0 would let through: key by key, where it is seen
#pragma unroll
        for (int j = 0; j < 8; ++j)
#pragma unroll 1
          for (int group = 0; group < 4; ++group) {
            const int at = 16 * (j / 4) + 4 * group + j % 4;
            const float weight = __shfl(w[j], 16 * group + col);
            if (!mine.holds(base + at)) continue;
#pragma unroll
            for (int c = 0; c < 2 * DT; ++c)
#pragma unroll
              for (int e = 0; e < 4; ++e)
                acc[c][e] = __builtin_fmaf(weight, ElemTraits<T>::load1(values + at * V::kStride + 16 * c + 4 * g + e), acc[c][e]);
          }
      }
    }
  }

  if (writes) write.store(p, t, 0);
  // The waves' parts, joined at the largest of their maxima.
  sum = across_groups_sum(sum);
  __syncthreads();
  float* joined = reinterpret_cast<float*>(lds);
#pragma unroll
  for (int c = 0; c < 2 * DT; ++c)
#pragma unroll
    for (int e = 0; e < 4; ++e) joined[(wave * 32 * DT + 16 * c + 4 * g + e) * 17 + col] = acc[c][e];
  if (g == 0) {
    stat[0][wave][col] = m;
    stat[1][wave][col] = sum;
  }
  __syncthreads();
  const int64_t unit = blockIdx.x;
  for (int i = static_cast<int>(threadIdx.x); i < kRowTile * p.D; i += 64 * kWaves) {
    const int row = i / p.D, c = i - row * p.D;
    float top = kNegInf, total = 0.f, value = 0.f;
#pragma unroll
    for (int w = 0; w < kWaves; ++w) top = __builtin_fmaxf(top, stat[0][w][row]);
    const float by = top == kNegInf ? 0.f : top;
#pragma unroll
    for (int w = 0; w < kWaves; ++w) {
      const float shrink = fast_exp2(stat[0][w][row] - by);
      total = __builtin_fmaf(stat[1][w][row], shrink, total);
      value = __builtin_fmaf(joined[(w * 32 * DT + c) * 17 + row], shrink, value);
    }
    if (p.splits > 1) {
      if (t.state == 1) {
        p.part[(unit * kRowTile + row) * p.D + c] = value;
        if (c == 0) {
          float* stats = p.part + static_cast<int64_t>(gridDim.x) * kRowTile * p.D;
          stats[(unit * kRowTile + row) * 2] = top;
          stats[(unit * kRowTile + row) * 2 + 1] = total;
        }
      }
    } else if (row0 + row < rows) {
      const int token = (row0 + row) / p.G, head = t.h * p.G + row0 + row - token * p.G;
      const float v = t.state < 0 ? __builtin_nanf("") : token < t.n ? value / total : 0.f;
      ElemTraits<T>::store1(static_cast<T*>(p.out) + ((static_cast<int64_t>(t.b) * p.L + token) * p.Hq + head) * p.D + c, v);
    }
  }
}

// ---- many rows ------------------------------------------------------------------------------
// A block of four waves takes 128 rows, 32 to a wave, and steps of 64 keys, whose rows go through registers (asked for a
// step ahead, their pages two) into LDS, for all four waves: sixteen rows to a block would read every key
// eight times as often.  Products of 32 x 32 x 16, transposed as above; half g of a wave holds the keys 8 (e / 4) + 4 g + e % 4
// of a group of 32, in the scores and in the values alike.  8 chunks of up to 1500 tokens over up to 1000, 16 heads on 4 of 128
// bf16: 153 us, 0.57 PFLOP/s (sixteen rows to a block: 629).  The matrix units are busy for 26 % of the cycles, the vector units for 35 %
// (an exponential is four others), LDS for 21 %; two waves to a SIMD do not hide the waits between them.  A second buffer of rows with
// one barrier to a step, and tiles ordered by length over all utterances, were no faster.
constexpr int kWideRows = 32, kWideKeys = 64;

template <typename T>
__device__ __forceinline__ f32x16 mma32(const Eight<T>& a, const Eight<T>& b, f32x16 c) {
  if constexpr (__is_same(T, bf16_t))
    return __builtin_amdgcn_mfma_f32_32x32x16_bf16(__builtin_bit_cast(bf16x8, a.w[0]), __builtin_bit_cast(bf16x8, b.w[0]), c, 0, 0, 0);
  else
    return __builtin_amdgcn_mfma_f32_32x32x16_f16(__builtin_bit_cast(f16x8, a.w[0]), __builtin_bit_cast(f16x8, b.w[0]), c, 0, 0, 0);
}

template <typename T, int DT>
__global__ __launch_bounds__(64 * kWaves, DT <= 2 ? 3 : 2) void enc_attention_wide(AttentionParams p) {
  constexpr int kPitch = DT == 1 ? 4 : DT == 2 ? 8 : 16;           // 16-byte pieces of a row of keys in LDS
  constexpr int kWhole = 32 * (DT - 1);                             // channels that every D of this DT has
  constexpr int kValueStride = 32 * DT + 32;                        // elements of a row of values in LDS
  // Four threads to a key, and every fourth piece of its row to each.  Piece c of a row of keys lies at c ^ swizzle(row): the
  // sixteen rows that are read at one piece meet all banks, and so do the four rows of four pieces that are written at
  // once.  Rows of values begin 64 bytes of banks apart, for the same, at a DT of 2 and 4; at 1 every other one meets the same
  // banks, and at 3 (72 to 96 channels) all do.
  const auto swizzle = [](int row) {
    if constexpr (kPitch == 16) return (row & 3) << 2 | (row >> 2 & 3);
    else if constexpr (kPitch == 8) return (row >> 1 & 1) << 2 | (row >> 2 & 3);
    else return row >> 2 & 3;
  };
  __shared__ __attribute__((aligned(16))) u32x4 keys[kWideKeys * kPitch];
  __shared__ __attribute__((aligned(16))) T values[kWideKeys * kValueStride];
  __shared__ uint32_t flags[2][3];  // of a step, in turn: keys whose page is none, and whether a value is no number
  const int thread = static_cast<int>(threadIdx.x), lane = thread & 63, wave = __builtin_amdgcn_readfirstlane(thread >> 6);
  const int g = lane >> 5, col = lane & 31;
  const Tile t(p, blockIdx.x / p.splits, static_cast<int>(blockIdx.x % p.splits));
  const int rows = p.L * p.G, row0 = t.tile * p.rows, wave_row0 = row0 + wave * kWideRows;

  float m = kNegInf, sum = 0.f;  // the maximum before the scale
  float by = 0.f;                // and after it, less the weights' factor
  bool far = false;              // one of the wave's rows has a maximum past 2^10
  f32x16 acc[DT];
#pragma unroll
  for (int c = 0; c < DT; ++c)
#pragma unroll
    for (int e = 0; e < 16; ++e) acc[c][e] = 0.f;
  const float scale = p.scale == 0.f ? 1.f : __builtin_fabsf(p.scale);  // 0: of products with 0

  if (t.state == 1) {
    const int all_rows = t.n * p.G, last_row = min(row0 + p.rows, all_rows) - 1;
    const int my_row = min(wave_row0 + col, last_row), my_token = my_row / p.G;
    const auto seen = [&](int row) { return Seen(t.cached + row / p.G, t.end, p.causal != 0, p.left); };
    const Seen mine(t.cached + my_token, t.end, p.causal != 0, p.left);
    const Seen first = seen(row0), last = seen(last_row);
    const Seen wave_first = seen(min(wave_row0, last_row)), wave_last = seen(min(wave_row0 + kWideRows - 1, last_row));
    const int lo = first.lo, hi = last.hi;
    const int steps = (hi - lo + kWideKeys - 1) / kWideKeys;
    const int begin = static_cast<int>(static_cast<int64_t>(steps) * t.split / p.splits);
    const int stop = static_cast<int>(static_cast<int64_t>(steps) * (t.split + 1) / p.splits);

    const T* k_new = static_cast<const T*>(p.k) + t.b * p.k_stride_b + t.h * p.k_stride_h;
    const T* v_new = static_cast<const T*>(p.v) + t.b * p.v_stride_b + t.h * p.v_stride_h;
    const T *k_cache = static_cast<const T*>(p.k_cache), *v_cache = static_cast<const T*>(p.v_cache);

    Eight<T> q[2 * DT];
    {
      const T* from = static_cast<const T*>(p.q) + t.b * p.q_stride_b + my_token * p.q_stride_t +
                      (t.h * p.G + my_row - my_token * p.G) * p.q_stride_h;
      const uint32_t sign = p.scale < 0.f ? 0x80008000u : 0u;  // the largest score is then the largest product
#pragma unroll
      for (int d = 0; d < 2 * DT; ++d) {
        q[d].zero();
        if (16 * d + 8 * g < p.D && p.scale != 0.f) q[d].load(from + 16 * d + 8 * g);
        q[d].w[0] ^= u32x4{sign, sign, sign, sign};
      }
    }

    const int key = thread >> 2, piece0 = thread & 3;
    Eight<T> kk[DT], vv[DT];
    int id = 0;
    bool none = false;
    const auto place = [&](int step) { return min(lo + step * kWideKeys + key, hi - 1); };
    const auto ask = [&](int step) { id = t.table.pages[place(step) >> p.shift]; };
    const auto fetch = [&](int step) {
      const int pos = place(step);
      none = static_cast<uint32_t>(id) >= static_cast<uint32_t>(p.num_pages);
      const uint32_t there = cache_row(id, p.Hkv, t.h, pos, p.shift), own = kNewRow | static_cast<uint32_t>(pos - t.cached);
      const uint32_t row = none ? kBadRow : pos >= t.cached ? own : there;
      const T* k = row_pointer(k_cache, k_new, p.k_stride_t, row, p.D);
      const T* v = row_pointer(v_cache, v_new, p.v_stride_t, row, p.D);
#pragma unroll
      for (int i = 0; i < DT; ++i) {
        // behind D: the last piece again; a score's channels there are taken as 0, the output's are not stored
        const int c = 32 * i + 32 <= kWhole ? 8 * (piece0 + 4 * i) : min(8 * (piece0 + 4 * i), p.D - 8);
        kk[i].load(k + c);
        vv[i].load(v + c);
      }
    };
    if (thread < 6) flags[thread / 3][thread % 3] = 0;
    if (begin < stop) {
      ask(begin);
      fetch(begin);
      if (begin + 1 < stop) ask(begin + 1);
    }
    for (int step = begin; step < stop; ++step) {
      const int base = lo + step * kWideKeys, turn = (step - begin) & 1;
      const bool block_mixed = base < last.lo || base + kWideKeys > first.hi;
      __syncthreads();
      if (thread < 3) flags[turn ^ 1][thread] = 0;
#pragma unroll
      for (int i = 0; i < DT; ++i) {
        const int piece = piece0 + 4 * i;
        keys[key * kPitch + (piece ^ swizzle(key))] = 32 * i + 32 <= kWhole || 8 * piece < p.D ? kk[i].w[0] : u32x4{0, 0, 0, 0};
        if (block_mixed && vv[i].odd()) {
          flags[turn][2] = 1;
          vv[i].clear_odd();
        }
        vv[i].store(values + key * kValueStride + 8 * piece);
      }
      if (none) atomicOr(&flags[turn][key / 32], 1u << (key % 32));
      __syncthreads();
      if (step + 1 < stop) {
        fetch(step + 1);
        if (step + 2 < stop) ask(step + 2);
      }
      if (base >= wave_last.hi || base + kWideKeys <= wave_first.lo) continue;  // nothing that the wave's rows see
      const auto flag = [&](int i) { return static_cast<uint32_t>(__builtin_amdgcn_readfirstlane(static_cast<int>(flags[turn][i]))); };
      const uint32_t pageless[2] = {flag(0), flag(1)};
      const bool mixed = base < wave_last.lo || base + kWideKeys > wave_first.hi || (pageless[0] | pageless[1]) != 0;
      const bool careful = flag(2) != 0;
      f32x16 s[2];
#pragma unroll
      for (int e = 0; e < 16; ++e) s[0][e] = s[1][e] = 0.f;
      // A half's pieces are all asked for before the first product (left to itself the compiler waits for each in turn, which
      // costs more than the products), the other half's as the first one's are used.
      const auto key_piece = [&](int i, int d) {
        const int row = 32 * i + col;
        Eight<T> a;
        a.w[0] = keys[row * kPitch + ((2 * d + g) ^ swizzle(row))];
        return a;
      };
      Eight<T> pieces[2 * DT];
#pragma unroll
      for (int d = 0; d < 2 * DT; ++d) pieces[d] = key_piece(0, d);
      __builtin_amdgcn_sched_barrier(0);
#pragma unroll
      for (int d = 0; d < 2 * DT; ++d) {
        s[0] = mma32(pieces[d], q[d], s[0]);
        pieces[d] = key_piece(1, d);
      }
      __builtin_amdgcn_sched_barrier(0);
#pragma unroll
      for (int d = 0; d < 2 * DT; ++d) s[1] = mma32(pieces[d], q[d], s[1]);
      // whether the lane's row sees key `at` of the step
      const uint32_t from = static_cast<uint32_t>(base + 4 * g - mine.lo), span = static_cast<uint32_t>(mine.hi - mine.lo);
      const auto sees = [&](int i, int e) { return from + (32 * i + 8 * (e / 4) + e % 4) < span; };
      if (mixed) {
#pragma unroll
        for (int i = 0; i < 2; ++i)
#pragma unroll
          for (int e = 0; e < 16; ++e) {
            const float v = pageless[i] >> (8 * (e / 4) + 4 * g + e % 4) & 1 ? __builtin_nanf("") : s[i][e];
            s[i][e] = sees(i, e) ? v : kNegInf;
          }
      }
      float most = kNegInf;
#pragma unroll
      for (int i = 0; i < 2; ++i)
#pragma unroll
        for (int e = 0; e < 16; ++e) most = __builtin_fmaxf(most, s[i][e]);
      most = halves_max(most);
      // The maximum that the weights are taken against follows only where one of them would pass 2^kLag: its place does not
      // matter to the quotient, and most steps spare the products with the sums so far.
      const float grown = __builtin_fmaxf(m, most);
      if (far || __ballot((grown - m) * scale > static_cast<float>(kLag<T>) || (m == kNegInf && grown > m))) {
        const float shrink = m == kNegInf ? 0.f : fast_exp2((m - grown) * scale);
        sum *= shrink;
#pragma unroll
        for (int c = 0; c < DT; ++c) acc[c] *= shrink;
        m = grown;
        by = m == kNegInf ? 0.f : m * scale - static_cast<float>(kWideLift<T>);
        // A weight is 2^(s scale - by), the product exact and by rounded: past 2^24 its rounding alone would be several
        // powers of two, and past 2^31 a weight of 1 infinity or 0.  There the difference comes first.
        far = __ballot(__builtin_fabsf(by) > 1024.f) != 0;
        if (far) {
          const float top = m == kNegInf ? 0.f : m;
#pragma unroll
          for (int i = 0; i < 2; ++i)
#pragma unroll
            for (int e = 0; e < 16; ++e) s[i][e] -= top;
          by = -static_cast<float>(kWideLift<T>);
        }
      }
      // the values of channel 32 c + lane % 32 and the sixteen keys b of the step, of which the lane holds eight
      const auto column = [&](int c, int b) {
        Eight<T> a;
        const int i = lane & 15;
#pragma unroll
        for (int half = 0; half < 2; ++half) {
          const T* at = values + (16 * b + 8 * half + 4 * g + (i >> 2)) * kValueStride + 32 * c + 16 * (lane >> 4 & 1) + 4 * (i & 3);
          const i16x4 four = __builtin_amdgcn_ds_read_tr16_b64_v4i16((__attribute__((address_space(3))) i16x4*)at);
          const auto two = __builtin_bit_cast(uint2, four);
          a.w[0][2 * half] = two.x;
          a.w[0][2 * half + 1] = two.y;
        }
        return a;
      };
      // Weights of 16 bits, as the values are.  The first half's products with the values run while the second half's weights
      // are formed: one matrix instruction, then a few of the others.
      Eight<T> weights[4];
      float half_sum[2] = {0.f, 0.f};
      const auto weigh = [&](int i) {
#pragma unroll
        for (int e = 0; e < 16; ++e) {
          s[i][e] = fast_exp2(__builtin_fmaf(s[i][e], scale, -by));
          half_sum[i] += s[i][e];
        }
#pragma unroll
        for (int b = 0; b < 2; ++b) {
          float w[8];
#pragma unroll
          for (int j = 0; j < 8; ++j) w[j] = s[i][8 * b + j];
          weights[2 * i + b].set(w);
        }
      };
      weigh(0);
      __builtin_amdgcn_sched_barrier(0);
#pragma unroll
      for (int b = 0; b < 2; ++b)
#pragma unroll
        for (int c = 0; c < DT; ++c) acc[c] = mma32(column(c, b), weights[b], acc[c]);
      weigh(1);
#pragma unroll
      for (int i = 0; i < 2 * DT; ++i) {
        __builtin_amdgcn_sched_group_barrier(0x100, 2, 0);
        __builtin_amdgcn_sched_group_barrier(0x008, 1, 0);
        __builtin_amdgcn_sched_group_barrier(0x002, 72 / (2 * DT), 0);
      }
      __builtin_amdgcn_sched_barrier(0);
#pragma unroll
      for (int b = 2; b < 4; ++b)
#pragma unroll
        for (int c = 0; c < DT; ++c) acc[c] = mma32(column(c, b), weights[b], acc[c]);
      sum += half_sum[0] + half_sum[1];
      if (careful) {
        // An infinity or NaN among the values, which a weight of 0 would have let through, went into LDS as 0: it reaches the
        // rows that see its key from here.
#pragma unroll 1
        for (int pos = base; pos < min(base + kWideKeys, hi); ++pos) {
          const uint32_t row = row_of(p, t, pos);
          if (row == kBadRow || !mine.holds(pos)) continue;
          const T* from = row_pointer(v_cache, v_new, p.v_stride_t, row, p.D);
          int first_channel = 4 * g;
          asm volatile("" : "+v"(first_channel));  // the places are formed here, not kept in registers all along
#pragma unroll
          for (int c = 0; c < DT; ++c)
#pragma unroll
            for (int e = 0; e < 4; ++e) {
              Pack<T, 4> k;
              k.load(from + min(32 * c + 8 * e + first_channel, p.D - 4));
              float v[4];
              k.get(v);
#pragma unroll
              for (int j = 0; j < 4; ++j) acc[c][4 * e + j] += __builtin_isfinite(v[j]) ? 0.f : v[j];
            }
        }
      }
    }
  }

  if (t.split == 0 && t.state == 1) {
    CacheWrite<T, 2> write;
    int first;
    const int rounds = (CacheWrite<T, 2>::tokens(p, t, first) * (p.D / 8) + 128 * kWaves - 1) / (128 * kWaves);
    for (int i = 0; i < rounds; ++i) {
      write.ask(p, t, i);
      write.store(p, t, i);
    }
  }
  sum += __shfl_xor(sum, 32);
  const int row = wave_row0 + col;
  const bool ends = p.splits == 1;
  if (!ends && t.state != 1) return;
  float* part = p.part + (static_cast<int64_t>(blockIdx.x) * p.rows + wave * kWideRows + col) * p.D;
  if (!ends && g == 0) {
    float* stats = p.part + static_cast<int64_t>(gridDim.x) * p.rows * p.D +
                   (static_cast<int64_t>(blockIdx.x) * p.rows + wave * kWideRows + col) * 2;
    stats[0] = m == kNegInf ? m : m * scale;
    stats[1] = sum;
  }
  if (ends && row >= rows) return;
  const int token = row / p.G, head = t.h * p.G + row - token * p.G;
  const bool valid = t.state == 1 && token < t.n;
  const float fill = t.state < 0 ? __builtin_nanf("") : 0.f, over = 1.f / sum;
  T* out = static_cast<T*>(p.out) + ((static_cast<int64_t>(t.b) * p.L + token) * p.Hq + head) * p.D;
#pragma unroll
  for (int c = 0; c < DT; ++c)
#pragma unroll
    for (int e = 0; e < 4; ++e) {
      const int at = 32 * c + 8 * e + 4 * g;
      if (at >= p.D) continue;
      float v[4];
#pragma unroll
      for (int j = 0; j < 4; ++j) v[j] = ends ? (valid ? acc[c][4 * e + j] * over : fill) : acc[c][4 * e + j];
      if (ends) {
        Pack<T, 4> k;
        k.set(v);
        k.store(out + at);
      } else {
        *reinterpret_cast<f32x4*>(part + at) = f32x4{v[0], v[1], v[2], v[3]};
      }
    }
}

// ---- the splits of a row, joined in their order --------------------------------------------------
// A block to a row: the splits' factors in LDS, then four channels to a thread and every eighth split or so, and the
// threads' sums.  (A block to sixteen rows that went over the splits in turn took 175 us for 48 rows of 117 splits.)
constexpr int kMostSplits = 256;
template <typename T>
__global__ __launch_bounds__(256) void enc_attention_join(AttentionParams p) {
  __shared__ float factor[kMostSplits], lds[4], total_lds[4];
  __shared__ f32x4 sums[256];
  const int64_t unit = blockIdx.x / p.rows;
  const int in_tile = static_cast<int>(blockIdx.x % p.rows), thread = static_cast<int>(threadIdx.x);
  const Tile t(p, unit, 0);
  const int row = t.tile * p.rows + in_tile;
  if (row >= p.L * p.G) return;
  const int token = row / p.G, head = t.h * p.G + row - token * p.G;
  T* out = static_cast<T*>(p.out) + ((static_cast<int64_t>(t.b) * p.L + token) * p.Hq + head) * p.D;
  if (t.state < 0 || token >= t.n) {
    const float fill = t.state < 0 ? __builtin_nanf("") : 0.f;
    for (int c = thread; c < p.D; c += 256) ElemTraits<T>::store1(out + c, fill);
    return;
  }
  const int64_t first = unit * p.splits * p.rows + in_tile;  // the first split's row
  const float* stats = p.part + static_cast<int64_t>(gridDim.x) * p.splits * p.D;
  float top = kNegInf, weight = 0.f;
  if (thread < p.splits) {
    top = stats[(first + static_cast<int64_t>(thread) * p.rows) * 2];
    weight = stats[(first + static_cast<int64_t>(thread) * p.rows) * 2 + 1];
  }
  const float mine = top;
  top = group_reduce<64, MaxOp>(top, kNegInf);
  if ((thread & 63) == 0) lds[thread >> 6] = top;
  __syncthreads();
  top = __builtin_fmaxf(__builtin_fmaxf(lds[0], lds[1]), __builtin_fmaxf(lds[2], lds[3]));
  const float by = top == kNegInf ? 0.f : top, shrink = thread < p.splits ? fast_exp2(mine - by) : 0.f;
  factor[thread] = shrink;
  weight = group_reduce<64, SumOp>(weight * shrink, 0.f);
  if ((thread & 63) == 0) total_lds[thread >> 6] = weight;
  __syncthreads();
  const float total = total_lds[0] + total_lds[1] + total_lds[2] + total_lds[3];
  const int lanes = p.D / 4, groups = 256 / lanes, group = thread / lanes, c = 4 * (thread - group * lanes);
  f32x4 sum = {0.f, 0.f, 0.f, 0.f};
  if (group < groups) {
#pragma unroll 4
    for (int s = group; s < p.splits; s += groups)
      sum += factor[s] * *reinterpret_cast<const f32x4*>(p.part + (first + static_cast<int64_t>(s) * p.rows) * p.D + c);
  }
  sums[thread] = sum;
  __syncthreads();
  if (group != 0) return;
  for (int i = 1; i < groups; ++i) sum += sums[i * lanes + thread];
#pragma unroll
  for (int j = 0; j < 4; ++j) ElemTraits<T>::store1(out + c + j, sum[j] / total);
}

// The same of few splits, where rows are many and a block to a row would fetch a few hundred bytes.  Four channels of a row to a
// thread, which goes over the splits in their order.  A call with a block to a row and with this (us; streams, heads of queries on heads
// of keys, D, tokens, cached): two splits, 8 of 8 of 64, 512 over 500 79 and 32.5; five, 2 of 16 on 2 of 64, 374 over 2000 45.6 and 29.3;
// eight, 2 of 4 on 1 of 64, 600 over 500 23.8 and 17.4; sixteen, 16 of 16 on 2 of 128, one over 3000 20 and 21.2; 47 splits, 1 of 4 of 64,
// one over 6000 10.3 and 17.6.  (units x splits <= 512 keeps the indexes within 32 bits.)
constexpr int kFewSplits = 8;
template <typename T>
__global__ __launch_bounds__(256) void enc_attention_join_few(AttentionParams p) {
  const int lanes = p.D / 4, thread = static_cast<int>(blockIdx.x * 256 + threadIdx.x), at = thread / lanes, c = 4 * (thread - at * lanes);
  const int units = p.B * p.Hkv * p.tiles, unit = at / p.rows, in_tile = at - unit * p.rows;
  if (unit >= units) return;
  const Tile t(p, unit, 0);
  const int row = t.tile * p.rows + in_tile;
  if (row >= p.L * p.G) return;
  const int token = row / p.G, head = t.h * p.G + row - token * p.G;
  T* out = static_cast<T*>(p.out) + ((static_cast<int64_t>(t.b) * p.L + token) * p.Hq + head) * p.D + c;
  if (t.state < 0 || token >= t.n) {
#pragma unroll
    for (int j = 0; j < 4; ++j) ElemTraits<T>::store1(out + j, t.state < 0 ? __builtin_nanf("") : 0.f);
    return;
  }
  const int64_t first = static_cast<int64_t>(unit) * p.splits * p.rows + in_tile;  // the first split's row
  const float* stats = p.part + static_cast<int64_t>(units) * p.splits * p.rows * p.D;
  float top = kNegInf;
#pragma unroll 4
  for (int s = 0; s < p.splits; ++s) top = __builtin_fmaxf(top, stats[(first + static_cast<int64_t>(s) * p.rows) * 2]);
  const float by = top == kNegInf ? 0.f : top;
  float total = 0.f;
  f32x4 sum = {0.f, 0.f, 0.f, 0.f};
#pragma unroll 4
  for (int s = 0; s < p.splits; ++s) {
    const int64_t of = first + static_cast<int64_t>(s) * p.rows;
    const float factor = fast_exp2(stats[of * 2] - by);
    total = __builtin_fmaf(stats[of * 2 + 1], factor, total);
    sum += factor * *reinterpret_cast<const f32x4*>(p.part + of * p.D + c);
  }
#pragma unroll
  for (int j = 0; j < 4; ++j) ElemTraits<T>::store1(out + j, sum[j] / total);
}

// ---- host ---------------------------------------------------------------------

// Whether wide tiles take the rows of an utterance's head of keys: past 64 of them, or past 16 where tiles of sixteen would be more
// than two to a CU (us, sixteen rows and wide; tokens, 64 streams of 8 heads of 64 over 300: 20 24.2 and 17.5, 40 31 and 20.6, 128 79 and
// 25.8; 8 of 4 heads of 128 over 1000: 20 16.2 and 19.8, 64 22.9 and 23.8, 128 32.5 and 29.7; 1 of 4 heads of 64 over 4000: 64 13.8 and
// 13.9, 128 14.8 and 14.3).
bool wide(const rnnt_attention_shape_t& s) {
  const int64_t rows = static_cast<int64_t>(s.L) * (s.Hq / s.Hkv);
  const int64_t narrow = static_cast<int64_t>(s.B) * s.Hkv * ((rows + kRowTile - 1) / kRowTile);
  return s.dtype != RNNT_DTYPE_F32 && s.D <= 128 && (rows > 64 || (rows > 16 && narrow > 512));
}
int rows_of(const rnnt_attention_shape_t& s) { return wide(s) ? kWaves * kWideRows : kRowTile; }

int64_t units_of(const rnnt_attention_shape_t& s) {
  const int64_t rows = static_cast<int64_t>(s.L) * (s.Hq / s.Hkv), tile = rows_of(s);
  return static_cast<int64_t>(s.B) * s.Hkv * ((rows + tile - 1) / tile);
}

bool whole_stride(int64_t stride, int64_t e) { return stride * e % 16 == 0; }

rnnt_status_t check(const rnnt_attention_shape_t& s) {
  if (s.B < 1 || s.L < 0 || s.Hq < 1 || s.Hkv < 1 || s.D < 1 || s.page < 1 || s.table < 1 || s.num_pages < 1 ||
      s.Hq % s.Hkv != 0)
    return RNNT_ERR_BAD_SHAPE;
  const int64_t strides[9] = {s.q_stride_b, s.q_stride_t, s.q_stride_h, s.k_stride_b, s.k_stride_t,
                              s.k_stride_h, s.v_stride_b, s.v_stride_t, s.v_stride_h};
  for (const int64_t x : strides)
    if (x < 0) return RNNT_ERR_BAD_SHAPE;
  if (!net_dtype_known(s.dtype)) return RNNT_ERR_BAD_DTYPE;
  for (const int64_t x : strides)
    if (!whole_stride(x, net_elem_bytes(s.dtype))) return RNNT_ERR_ALIGNMENT;
  if (s.D % 8 != 0 || s.D > 256 || (s.page & (s.page - 1)) != 0 || s.page > 1024) return RNNT_ERR_UNSUPPORTED;
  if (s.k_stride_t > kMaxRows || s.v_stride_t > kMaxRows) return RNNT_ERR_UNSUPPORTED;
  if (s.num_pages > kMaxRows / s.page / s.Hkv || static_cast<int64_t>(s.L) * s.Hq > kMaxRows ||
      static_cast<int64_t>(s.table) * s.page + s.L >= (int64_t{1} << 30))
    return RNNT_ERR_UNSUPPORTED;
  if (units_of(s) >= (int64_t{1} << 23)) return RNNT_ERR_UNSUPPORTED;
  return RNNT_OK;
}

// Blocks that share a tile's keys out: few tiles over a long cache would leave most CUs idle.  No more than two to a CU, which
// is what fits of the larger kernels: 702 blocks in two rounds took 52 us where 510 in one take 45.
int splits_of(const rnnt_attention_shape_t& s) {
  const int64_t units = units_of(s);
  if (units == 0) return 1;
  int64_t keys = static_cast<int64_t>(s.table) * s.page;
  if (s.left >= 0 && static_cast<int64_t>(s.left) + s.L < keys) keys = static_cast<int64_t>(s.left) + s.L;
  // few keys: the join costs more (128 tiles over 600: 11.6 us in one block each, 15 in four); else 128 keys to a block at least (1000
  // keys, one tile: 13.2 with 512, 10.9 with 256, 9.6; 4000 keys, 8 tiles: 19.6, 16.1, 15.0; 20000, 2 tiles: 15.4, 12.9, 13.3)
  if (keys < 768) return 1;
  const int64_t by_grid = 512 / units, by_keys = keys / 128;
  const int64_t n = by_grid < by_keys ? by_grid : by_keys;
  return static_cast<int>(n < 1 ? 1 : n > kMostSplits ? kMostSplits : n);
}

size_t workspace_of(const rnnt_attention_shape_t& s) {
  const int splits = splits_of(s);
  if (splits == 1) return 0;
  return net_align256(static_cast<size_t>(units_of(s)) * splits * rows_of(s) * (s.D + 2) * sizeof(float));
}

template <typename F>
rnnt_status_t with_channels(int D, F&& f) {
  using std::integral_constant;
  if (D <= 32) return f(integral_constant<int, 1>{});
  if (D <= 64) return f(integral_constant<int, 2>{});
  if (D <= 96) return f(integral_constant<int, 3>{});
  if (D <= 128) return f(integral_constant<int, 4>{});
  return f(integral_constant<int, 8>{});
}

}  // namespace
}  // namespace rnnt

using namespace rnnt;

extern "C" {

size_t rnnt_cached_attention_workspace_bytes(rnnt_attention_shape_t shape) {
  return check(shape) == RNNT_OK ? workspace_of(shape) : 0;
}

rnnt_status_t rnnt_cached_attention(const void* q, const void* k, const void* v, rnnt_attention_shape_t shape,
                                    const int32_t* lens, const int32_t* cached, const int32_t* pages, void* k_cache,
                                    void* v_cache, float scale, void* out, void* workspace, size_t workspace_bytes,
                                    hipStream_t stream) {
  const rnnt_attention_shape_t& s = shape;
  rnnt_status_t st = check(s);
  if (st != RNNT_OK) return st;
  if (!__builtin_isfinite(scale * kLog2eF)) return RNNT_ERR_BAD_VARIANT;
  if (!cached || !pages || !k_cache || !v_cache || (s.L > 0 && (!q || !k || !v || !out))) return RNNT_ERR_NULL_PTR;
  if (!multiple_of(16, q) || !multiple_of(16, k) || !multiple_of(16, v) || !multiple_of(16, k_cache) ||
      !multiple_of(16, v_cache) || !multiple_of(net_elem_bytes(s.dtype), out))
    return RNNT_ERR_ALIGNMENT;
  if (s.L == 0) return RNNT_OK;
  Workspace ws;
  st = ws.take(workspace, workspace_bytes, workspace_of(s), stream);
  if (st != RNNT_OK) return st;
  AttentionParams p{};
  p.q = q;
  p.k = k;
  p.v = v;
  p.k_cache = k_cache;
  p.v_cache = v_cache;
  p.out = out;
  p.lens = lens;
  p.cached = cached;
  p.pages = pages;
  p.part = reinterpret_cast<float*>(ws.ptr);
  p.q_stride_b = s.q_stride_b;
  p.q_stride_t = s.q_stride_t;
  p.q_stride_h = s.q_stride_h;
  p.k_stride_b = s.k_stride_b;
  p.k_stride_t = s.k_stride_t;
  p.k_stride_h = s.k_stride_h;
  p.v_stride_b = s.v_stride_b;
  p.v_stride_t = s.v_stride_t;
  p.v_stride_h = s.v_stride_h;
  p.B = s.B;
  p.L = s.L;
  p.Hq = s.Hq;
  p.Hkv = s.Hkv;
  p.G = s.Hq / s.Hkv;
  p.D = s.D;
  p.shift = __builtin_ctz(static_cast<unsigned>(s.page));
  p.table = s.table;
  p.num_pages = s.num_pages;
  p.causal = s.causal != 0;
  p.left = s.left < 0 ? -1 : s.left;
  p.rows = rows_of(s);
  p.tiles = static_cast<int32_t>((static_cast<int64_t>(s.L) * p.G + p.rows - 1) / p.rows);
  p.splits = splits_of(s);
  p.scale = scale * kLog2eF;
  const int64_t units = units_of(s);
  return with_dtype(s.dtype, [&](auto t) {
    using T = decltype(t);
    const dim3 grid(static_cast<uint32_t>(units * p.splits)), block(64 * kWaves);
    st = with_channels(s.D, [&](auto channels) {
      constexpr int DT = decltype(channels)::value;
      if constexpr (sizeof(T) == 2 && DT <= 4) {
        if (wide(s)) {
          hipLaunchKernelGGL((enc_attention_wide<T, DT>), grid, block, 0, stream, p);
          return launched();
        }
      }
      hipLaunchKernelGGL((enc_attention<T, DT>), grid, block, 0, stream, p);
      return launched();
    });
    if (st != RNNT_OK || p.splits == 1) return st;
    if (p.splits <= kFewSplits) {
      const int64_t threads = units * p.rows * (s.D / 4);
      hipLaunchKernelGGL((enc_attention_join_few<T>), dim3(static_cast<uint32_t>((threads + 255) / 256)), dim3(256), 0, stream, p);
      return launched();
    }
    hipLaunchKernelGGL((enc_attention_join<T>), dim3(static_cast<uint32_t>(units * p.rows)), dim3(256), 0, stream, p);
    return launched();
  });
}

}  // extern "C"
