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

// Rows are covered by groups of VEC elements; the last group of a row that is no multiple of VEC begins
// VEC before its end, and what it shares with the group before is computed and written twice alike.
__device__ __forceinline__ int group_start(int group, int VEC, int D) { return min(group * VEC, D - VEC); }

struct EmbeddingParams {
  TokenSource src;
  const void* weight;
  void* out;
  float scale;
  bool away;  // store past the caches
  int32_t D, rows, lanes, groups;  // lanes: threads to a row, a power of two; groups: of VEC elements in a row
};

// Four rows to a thread: a row's label, then its weights, then the store wait for one another, the rows do not.
constexpr int kRowsAtOnce = 4;

template <typename T, int VEC>
__global__ __launch_bounds__(256) void net_embedding(EmbeddingParams p) {
  const int per = 256 / p.lanes;
  const int64_t step = static_cast<int64_t>(gridDim.x) * per * kRowsAtOnce;
  for (int64_t r0 = static_cast<int64_t>(blockIdx.x) * per * kRowsAtOnce + static_cast<int>(threadIdx.x) / p.lanes; r0 < p.rows; r0 += step) {
    int32_t v[kRowsAtOnce], row[kRowsAtOnce];
#pragma unroll
    for (int i = 0; i < kRowsAtOnce; ++i) {  // a row past the last one is the last one again
      row[i] = static_cast<int32_t>(min(r0 + i * per, static_cast<int64_t>(p.rows) - 1));
      v[i] = token_at(p.src, row[i]);
    }
    for (int g = static_cast<int>(threadIdx.x) & (p.lanes - 1); g < p.groups; g += p.lanes) {
      const int c = group_start(g, VEC, p.D);
      Pack<T, VEC> k[kRowsAtOnce];
#pragma unroll
      for (int i = 0; i < kRowsAtOnce; ++i)
        k[i].load(static_cast<const T*>(p.weight) + static_cast<int64_t>(max(v[i], 0)) * p.D + c);
#pragma unroll
      for (int i = 0; i < kRowsAtOnce; ++i) {
        float f[VEC];
        k[i].get(f);
#pragma unroll
        for (int j = 0; j < VEC; ++j) f[j] = v[i] >= 0 ? f[j] * p.scale : v[i] == kBadRow ? __builtin_nanf("") : 0.f;
        k[i].set(f);
        T* o = static_cast<T*>(p.out) + static_cast<int64_t>(row[i]) * p.D + c;
        if (p.away) k[i].store_away(o);
        else k[i].store(o);
      }
    }
  }
}

// ---- the gradient ---------------------------------------------------------------
// Four launches: the rows' tokens (not for a few thousand rows); the rows sorted by token (and by position within one); the sums of kRun sorted
// rows at a time, token by token; the tokens that lie in several runs, and the rows without a token.  A row of dout
// is read once, and every sum has one order.

constexpr int32_t kNoKey = 0x7fffffff;  // a row without a token, past every token
constexpr int kSortWaves = 16;
constexpr int kSortTokens = 384;   // most tokens of a sorting block (a thread to a token)
constexpr int kSortFound = 384;    // rows that a wave keeps
constexpr int kSortBlocks = 256;   // one to a CU, each looks at every row
// Up to here every sorting block finds the tokens itself, a launch less (gradient of V=1025 D=256, with keys and
// without: 2592 rows 15.3 and 13.6 us, 8192 15.8 and 16.3, 16384 17.9 and 21.3).
constexpr int kRowsWithoutKeys = 8192;
constexpr int kRun = 32;
constexpr int kRowsToWave = 4;
constexpr int kManyRuns = 32;  // a token of more runs is added up by four waves

struct EmbeddingGradParams {
  TokenSource src;
  const void* dout;
  void* dweight;
  float scale;
  int32_t D, rows, tiles;           // tiles: of 64 groups of columns
  int32_t per_block;                // tokens of a sorting block
  int32_t runs;                     // ceil(rows / kRun)
  int32_t* keys;                    // (rows)
  int32_t* sorted;                  // (rows) positions, by token
  int32_t* tokens;                  // (rows) their tokens
  int32_t* first;                   // (V + 1) where a token's rows begin in `sorted`
  float* sums;                      // (runs, 2, D): of a token of the run before, of one of the next run too
};

__device__ __forceinline__ int32_t key_at(const TokenSource& src, int32_t r) {
  const int32_t v = token_at(src, r);
  return v < 0 ? kNoKey : v;
}

__global__ __launch_bounds__(256) void net_embedding_keys(EmbeddingGradParams p) {
  const int64_t r = static_cast<int64_t>(blockIdx.x) * 256 + threadIdx.x;
  if (r >= p.rows) return;
  p.keys[r] = key_at(p.src, static_cast<int32_t>(r));
}

// A counting sort in which every block looks at all rows and places those of its own few tokens: no table of
// counters between blocks, one launch, and the rows of a token in order (a wave takes a stretch of the rows and
// learns how many of each token the waves before it have).  The rows are read from L2: 131072 of them are 0.5 MB
// to a block.  What a wave finds it keeps in LDS, and looks at the rows again only where that overflows (a
// token with many rows).
struct SortBoard {
  int32_t place[kSortWaves][kSortTokens];   // rows of a token in a wave's stretch, then where its next one goes
  int32_t found[kSortWaves][kSortFound];    // rows of this block's tokens, in order
  uint16_t token[kSortWaves][kSortFound];   // their tokens, less the block's first
  int32_t below[kSortWaves], sum[kSortWaves];
};

// f(row, key) for the 64 rows of every group of a stretch, the keys of eight groups on their way at once
template <bool STORED, typename F>
__device__ __forceinline__ void for_rows(const EmbeddingGradParams& p, int begin, int end, int lane, F&& f) {
  constexpr int BATCH = 8;
  int r = begin;
  if constexpr (STORED) {
    for (; r + 64 * BATCH <= end; r += 64 * BATCH) {  // whole batches: nothing to check
      const int32_t* keys = p.keys + r + lane;
      int32_t key[BATCH];
#pragma unroll
      for (int i = 0; i < BATCH; ++i) key[i] = keys[64 * i];
#pragma unroll
      for (int i = 0; i < BATCH; ++i) f(r + 64 * i + lane, key[i]);
    }
  }
  for (; r < end; r += 64) {
    int32_t key = kNoKey;
    if (r + lane < end) key = STORED ? p.keys[r + lane] : key_at(p.src, r + lane);
    f(r + lane, key);
  }
}

template <bool STORED>
__global__ __launch_bounds__(64 * kSortWaves) void net_embedding_sort(EmbeddingGradParams p) {
  __shared__ SortBoard s;
  const int wave = __builtin_amdgcn_readfirstlane(static_cast<int>(threadIdx.x) >> 6), lane = static_cast<int>(threadIdx.x) & 63;
  const int lo = static_cast<int>(blockIdx.x) * p.per_block, n = min(p.per_block, p.src.V - lo);
  for (int i = threadIdx.x; i < kSortWaves * kSortTokens; i += 64 * kSortWaves) (&s.place[0][0])[i] = 0;
  __syncthreads();
  const int64_t stretch = ((static_cast<int64_t>(p.rows) + kSortWaves - 1) / kSortWaves + 63) / 64 * 64;
  const int begin = static_cast<int>(min(wave * stretch, static_cast<int64_t>(p.rows)));
  const int end = static_cast<int>(min(begin + stretch, static_cast<int64_t>(p.rows)));
  int32_t* mine = s.place[wave];
  const uint64_t before = (uint64_t{1} << lane) - 1;
  int less = 0, kept = 0;
  for_rows<STORED>(p, begin, end, lane, [&](int32_t row, int32_t key) {
    less += __popcll(__ballot(key < lo));
    const uint32_t d = static_cast<uint32_t>(key) - static_cast<uint32_t>(lo);
    const bool here = d < static_cast<uint32_t>(n);
    const uint64_t votes = __ballot(here);
    if (votes) {
      if (here) {
        atomicAdd(&mine[d], 1);
        const int at = kept + __popcll(votes & before);
        if (at < kSortFound) {
          s.found[wave][at] = row;
          s.token[wave][at] = static_cast<uint16_t>(d);
        }
      }
      kept += __popcll(votes);
    }
  });
  if (lane == 0) s.below[wave] = less;
  __syncthreads();
  // exclusive sums over (token, wave): a thread to a token
  int base = 0;
#pragma unroll
  for (int w = 0; w < kSortWaves; ++w) base += s.below[w];
  const int t = static_cast<int>(threadIdx.x);
  int total = 0;
  if (t < n) {
#pragma unroll
    for (int w = 0; w < kSortWaves; ++w) total += s.place[w][t];
  }
  int upto = total;  // inclusive over the wave
  for (int off = 1; off < 64; off <<= 1) {
    const int v = __shfl_up(upto, off);
    if (lane >= off) upto += v;
  }
  if (lane == 63) s.sum[wave] = upto;
  __syncthreads();
  int at = base + upto - total;
  for (int w = 0; w < wave; ++w) at += s.sum[w];
  if (t < n) {
    p.first[lo + t] = at;
    if (lo + t == p.src.V - 1) p.first[p.src.V] = at + total;
#pragma unroll
    for (int w = 0; w < kSortWaves; ++w) {
      const int c = s.place[w][t];
      s.place[w][t] = at;
      at += c;
    }
  }
  __syncthreads();
  // 64 rows at a time, their tokens one by one, each with all its rows
  const auto put = [&](int32_t row, uint32_t d) {
    uint64_t left = __ballot(d < static_cast<uint32_t>(n));
    while (left) {
      const int leader = __builtin_ctzll(left);
      const uint32_t token = static_cast<uint32_t>(__builtin_amdgcn_readlane(static_cast<int>(d), leader));
      const uint64_t same = __ballot(d == token);
      const int to = mine[token];
      if (d == token) {
        const int at = to + __popcll(same & before);
        p.sorted[at] = row;
        p.tokens[at] = lo + static_cast<int32_t>(token);
      }
      if (lane == leader) mine[token] = to + __popcll(same);
      __builtin_amdgcn_fence(__ATOMIC_ACQ_REL, "wavefront");  // the next look at the counter sees it
      left &= ~same;
    }
  };
  if (kept <= kSortFound) {
    for (int i = 0; i < kept; i += 64) {
      const int at_i = min(i + lane, kept - 1);
      put(s.found[wave][at_i], i + lane < kept ? s.token[wave][at_i] : static_cast<uint32_t>(kNoKey));
    }
  } else {
    for_rows<STORED>(p, begin, end, lane, [&](int32_t row, int32_t key) { put(row, static_cast<uint32_t>(key) - static_cast<uint32_t>(lo)); });
  }
}

// A wave to a run of kRun sorted rows and a tile of 64 groups of columns: the same work whatever the tokens are, its rows
// loaded eight at a time.  A token whose rows all lie in the run is finished here; the sums of one that comes from
// the run before go to the run's first slot, of one that only goes on in the next run to its second.
template <typename T, int VEC>
__global__ __launch_bounds__(256) void net_embedding_runs(EmbeddingGradParams p) {
  const int64_t item = static_cast<int64_t>(blockIdx.x) * 4 + __builtin_amdgcn_readfirstlane(static_cast<int>(threadIdx.x) >> 6);
  const int64_t run = item / p.tiles, begin64 = run * kRun;
  const int total = p.first[p.src.V];
  if (begin64 >= total) return;
  const int begin = static_cast<int>(begin64), n = min(kRun, total - begin), lane = static_cast<int>(threadIdx.x) & 63;
  const int c = group_start(static_cast<int>(item - run * p.tiles) * 64 + lane, VEC, p.D);
  // lane i: row and token i of the run; lanes kRun and kRun + 1: the tokens around it
  const int at = lane < kRun ? begin + min(lane, n - 1) : lane == kRun ? max(begin - 1, 0) : min(begin + n, total - 1);
  const int my_row = p.sorted[at], my_token = p.tokens[at];
  const auto token_of = [&](int i) { return __builtin_amdgcn_readlane(my_token, i); };
  const bool from_before = begin > 0 && token_of(kRun) == token_of(0);
  const bool goes_on = begin + n < total && token_of(kRun + 1) == token_of(n - 1);
  float sum[VEC];
#pragma unroll
  for (int j = 0; j < VEC; ++j) sum[j] = 0.f;
  int32_t token = token_of(0);
  bool first = true;
  const auto flush = [&](bool at_end) {
    if ((first && from_before) || (at_end && goes_on)) {
      Pack<float, VEC> k;
      k.set(sum);
      k.store(p.sums + (run * 2 + (first && from_before ? 0 : 1)) * p.D + c);
    } else {
#pragma unroll
      for (int j = 0; j < VEC; ++j) sum[j] *= p.scale;
      Pack<T, VEC> k;
      k.set(sum);
      k.store(static_cast<T*>(p.dweight) + static_cast<int64_t>(token) * p.D + c);
    }
  };
  constexpr int BATCH = 8;
  for (int i = 0; i < n; i += BATCH) {
    Pack<T, VEC> k[BATCH];
#pragma unroll
    for (int b = 0; b < BATCH; ++b)  // past the run's end its last row again
      k[b].load_once(static_cast<const T*>(p.dout) + static_cast<int64_t>(__builtin_amdgcn_readlane(my_row, min(i + b, n - 1))) * p.D + c);
#pragma unroll
    for (int b = 0; b < BATCH; ++b) {
      if (i + b < n) {
        const int32_t t = token_of(i + b);
        if (t != token) {
          flush(false);
          first = false;
          token = t;
#pragma unroll
          for (int j = 0; j < VEC; ++j) sum[j] = 0.f;
        }
        float f[VEC];
        k[b].get(f);
#pragma unroll
        for (int j = 0; j < VEC; ++j) sum[j] += f[j];
      }
    }
  }
  flush(true);
}

// The sums of a token in runs r0 .. r1 (r0's second slot, the others' first), from run r0 + 1 + s0 to s1.
template <int VEC>
__device__ __forceinline__ void add_runs(const EmbeddingGradParams& p, int64_t r0, int s0, int s1, int c, float* sum) {
  const float* sums = p.sums + (r0 + 1) * 2 * p.D + c;
#pragma unroll 4
  for (int i = s0; i < s1; ++i) {
    Pack<float, VEC> k;
    float f[VEC];
    k.load(sums + static_cast<int64_t>(i) * 2 * p.D);
    k.get(f);
#pragma unroll
    for (int j = 0; j < VEC; ++j) sum[j] += f[j];
  }
}

// What the runs left: a wave to kRowsToWave weight rows and a tile, for the rows that no token has and the tokens of several
// runs; behind them a block to every run in which a token of more than kManyRuns begins.
template <typename T, int VEC>
__global__ __launch_bounds__(256) void net_embedding_rows(EmbeddingGradParams p, int32_t row_blocks) {
  __shared__ float parts[4][VEC * 64];
  const int wave = __builtin_amdgcn_readfirstlane(static_cast<int>(threadIdx.x) >> 6), lane = static_cast<int>(threadIdx.x) & 63;
  float sum[VEC];
#pragma unroll
  for (int j = 0; j < VEC; ++j) sum[j] = 0.f;
  const auto begin_sums = [&](int64_t r0, int c) {
    Pack<float, VEC> k;
    k.load(p.sums + (r0 * 2 + 1) * p.D + c);
    k.get(sum);
  };
  const auto finish = [&](int64_t v, int c) {
#pragma unroll
    for (int j = 0; j < VEC; ++j) sum[j] *= p.scale;
    Pack<T, VEC> k;
    k.set(sum);
    k.store(static_cast<T*>(p.dweight) + v * p.D + c);
  };
  if (static_cast<int>(blockIdx.x) < row_blocks) {
    const int64_t item = static_cast<int64_t>(blockIdx.x) * 4 + wave;
    const int64_t v0 = item / p.tiles * kRowsToWave;
    if (v0 >= p.src.V) return;
    const int c = group_start(static_cast<int>(item % p.tiles) * 64 + lane, VEC, p.D);
    const int bounds = p.first[min(v0 + lane, static_cast<int64_t>(p.src.V))];  // lanes 0 .. kRowsToWave: where the rows begin
    for (int i = 0; i < kRowsToWave && v0 + i < p.src.V; ++i) {
      const int from = __builtin_amdgcn_readlane(bounds, i), to = __builtin_amdgcn_readlane(bounds, i + 1);
#pragma unroll
      for (int j = 0; j < VEC; ++j) sum[j] = 0.f;
      if (from < to) {
        const int r0 = from / kRun, more = (to - 1) / kRun - r0;
        if (more == 0 || more > kManyRuns) continue;
        begin_sums(r0, c);
        add_runs<VEC>(p, r0, 0, more, c, sum);
      }
      finish(v0 + i, c);
    }
    return;
  }
  const int64_t item = static_cast<int64_t>(blockIdx.x) - row_blocks, r0 = item / p.tiles;
  const int total = p.first[p.src.V];
  const int64_t begin = r0 * kRun;
  if (begin + kRun >= total) return;
  const int32_t token = p.tokens[begin + kRun - 1];
  const int from = p.first[token], more = static_cast<int>((p.first[token + 1] - 1) / kRun - r0);
  if (from < begin || more <= kManyRuns) return;
  const int c = group_start(static_cast<int>(item - r0 * p.tiles) * 64 + lane, VEC, p.D);
  const int stretch = (more + 3) / 4, s0 = min(wave * stretch, more), s1 = min(s0 + stretch, more);
  if (wave == 0) begin_sums(r0, c);
  add_runs<VEC>(p, r0, s0, s1, c, sum);
#pragma unroll
  for (int j = 0; j < VEC; ++j) parts[wave][j * 64 + lane] = sum[j];
  __syncthreads();
  if (wave == 0) {
#pragma unroll
    for (int j = 0; j < VEC; ++j) {
      sum[j] = 0.f;
#pragma unroll
      for (int w = 0; w < 4; ++w) sum[j] += parts[w][j * 64 + lane];
    }
    finish(token, c);
  }
}

rnnt_status_t check(const int32_t* labels, const rnnt_embedding_shape_t& s, TokenSource* src, const int32_t* lens) {
  if (s.B < 1 || s.N < 0 || s.V < 1 || s.D < 1 || s.start < -1 || s.start >= s.V) return RNNT_ERR_BAD_SHAPE;
  if (!net_dtype_known(s.dtype)) return RNNT_ERR_BAD_DTYPE;
  const int64_t n1 = static_cast<int64_t>(s.N) + (s.start >= 0);
  if (n1 * s.B > kMaxRows - (1 << 16) || s.D > (1 << 30)) return RNNT_ERR_UNSUPPORTED;
  if (!labels && s.N > 0) return RNNT_ERR_NULL_PTR;
  *src = TokenSource{labels, lens, s.B, s.N, static_cast<int32_t>(n1), s.V, s.start};
  return RNNT_OK;
}

int lanes_for(int groups) {
  int n = 1;
  while (n < 256 && n < groups) n *= 2;
  return n;
}

// The gradient's grids: a wave to a run or to weight rows, times tiles of 64 groups of channels.
struct GradGrid {
  int vec, tiles;
  int64_t runs, run_items, row_blocks;

  explicit GradGrid(const rnnt_embedding_shape_t& s, int64_t rows) {
    const int wide = static_cast<int>(16 / net_elem_bytes(s.dtype));
    vec = s.D >= wide ? wide : 1;
    tiles = (s.D - 1) / (64 * vec) + 1;
    runs = (rows + kRun - 1) / kRun;
    run_items = runs * tiles;
    const int64_t row_waves = (static_cast<int64_t>(s.V) + kRowsToWave - 1) / kRowsToWave * tiles;
    row_blocks = (row_waves + 3) / 4;
  }
  bool fits() const { return row_blocks + run_items <= kMaxRows / 256; }
};

// Workspace of the gradient, 256-byte aligned pieces.
struct GradLayout {
  size_t keys, sorted, tokens, first, sums, total;
};

GradLayout grad_layout(const rnnt_embedding_shape_t& s, int64_t rows) {
  GradLayout L{};
  const size_t runs = static_cast<size_t>((rows + kRun - 1) / kRun);
  size_t o = 0;
  L.keys = o;
  o = net_align256(o + static_cast<size_t>(rows) * sizeof(int32_t));
  L.sorted = o;
  o = net_align256(o + static_cast<size_t>(rows) * sizeof(int32_t));
  L.tokens = o;
  o = net_align256(o + static_cast<size_t>(rows) * sizeof(int32_t));
  L.first = o;
  o = net_align256(o + (static_cast<size_t>(s.V) + 1) * sizeof(int32_t));
  L.sums = o;
  o = net_align256(o + runs * 2 * s.D * sizeof(float));
  L.total = o;
  return L;
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
  p.away = static_cast<int64_t>(p.rows) * shape.D * e >= kStoreAway;
  p.scale = scale;
  p.D = shape.D;
  return with_dtype(shape.dtype, [&](auto t) {
    using T = decltype(t);
    constexpr int VEC = 16 / sizeof(T);
    const bool wide = shape.D >= VEC;
    p.groups = wide ? (shape.D + VEC - 1) / VEC : shape.D;
    p.lanes = lanes_for(p.groups);
    const int64_t per = 256 / p.lanes * kRowsAtOnce, blocks = (p.rows + per - 1) / per;
    const dim3 grid(static_cast<uint32_t>(blocks < kMaxRows / 256 ? blocks : kMaxRows / 256));
    if (wide) hipLaunchKernelGGL((net_embedding<T, VEC>), grid, dim3(256), 0, stream, p);
    else hipLaunchKernelGGL((net_embedding<T, 1>), grid, dim3(256), 0, stream, p);
    return launched();
  });
}

size_t rnnt_label_embedding_grad_workspace_bytes(rnnt_embedding_shape_t shape) {
  TokenSource src;
  int32_t any;
  if (check(&any, shape, &src, nullptr) != RNNT_OK) return 0;
  const int64_t rows = static_cast<int64_t>(src.n1) * shape.B;
  return GradGrid(shape, rows).fits() ? grad_layout(shape, rows).total : 0;
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
  const GradGrid cut(shape, p.rows);
  if (!cut.fits()) return RNNT_ERR_UNSUPPORTED;
  p.tiles = cut.tiles;
  p.runs = static_cast<int32_t>(cut.runs);
  const int64_t run_items = cut.run_items, row_blocks = cut.row_blocks;
  const GradLayout L = grad_layout(shape, p.rows);
  Workspace ws;
  st = ws.take(workspace, workspace_bytes, L.total, stream);
  if (st != RNNT_OK) return st;
  p.dout = dout;
  p.dweight = dweight;
  p.scale = scale;
  p.D = shape.D;
  p.keys = reinterpret_cast<int32_t*>(ws.ptr + L.keys);
  p.sorted = reinterpret_cast<int32_t*>(ws.ptr + L.sorted);
  p.tokens = reinterpret_cast<int32_t*>(ws.ptr + L.tokens);
  p.first = reinterpret_cast<int32_t*>(ws.ptr + L.first);
  p.sums = reinterpret_cast<float*>(ws.ptr + L.sums);
  const int64_t shares = (static_cast<int64_t>(shape.V) + kSortBlocks - 1) / kSortBlocks;
  p.per_block = static_cast<int32_t>(shares < kSortTokens ? shares : kSortTokens);
  const dim3 sort_grid(static_cast<uint32_t>((static_cast<int64_t>(shape.V) + p.per_block - 1) / p.per_block));
  if (p.rows > kRowsWithoutKeys) {
    const dim3 grid(static_cast<uint32_t>((static_cast<int64_t>(p.rows) + 255) / 256));
    hipLaunchKernelGGL(net_embedding_keys, grid, dim3(256), 0, stream, p);
    if (launched() != RNNT_OK) return RNNT_ERR_HIP;
    hipLaunchKernelGGL((net_embedding_sort<true>), sort_grid, dim3(64 * kSortWaves), 0, stream, p);
  } else {
    hipLaunchKernelGGL((net_embedding_sort<false>), sort_grid, dim3(64 * kSortWaves), 0, stream, p);
  }
  if (launched() != RNNT_OK) return RNNT_ERR_HIP;
  return with_dtype(shape.dtype, [&](auto t) {
    using T = decltype(t);
    const auto rest = [&](auto v) {
      constexpr int VEC = decltype(v)::value;
      if (run_items > 0) {
        hipLaunchKernelGGL((net_embedding_runs<T, VEC>), dim3(static_cast<uint32_t>((run_items + 3) / 4)), dim3(256), 0, stream, p);
        if (launched() != RNNT_OK) return RNNT_ERR_HIP;
      }
      hipLaunchKernelGGL((net_embedding_rows<T, VEC>), dim3(static_cast<uint32_t>(row_blocks + run_items)), dim3(256), 0, stream, p,
                         static_cast<int32_t>(row_blocks));
      return launched();
    };
    return cut.vec > 1 ? rest(std::integral_constant<int, 16 / sizeof(T)>{}) : rest(std::integral_constant<int, 1>{});
  });
}

}  // extern "C"
