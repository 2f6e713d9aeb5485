// Where a token of a paged cache lies, and which keys a query sees: plain arithmetic, compiled for the host too.
#pragma once

#include <cstdint>

#if defined(__HIPCC__)
#define RNNT_PAGES_FN __host__ __device__ inline
#else
#define RNNT_PAGES_FN inline
#endif

namespace rnnt {

// The pages of one utterance; page = 1 << shift tokens.
struct PageTable {
  const int32_t* pages;
  int32_t table, num_pages, shift;

  // the page of position pos, or -1: no entry, or one that names no page
  RNNT_PAGES_FN int32_t page_of(int32_t pos) const {
    if (pos < 0 || (pos >> shift) >= table) return -1;
    const int32_t id = pages[pos >> shift];
    return id >= 0 && id < num_pages ? id : -1;
  }
};

// The row of head h in a cache (num_pages, heads, page, D), in rows of D elements.
RNNT_PAGES_FN uint32_t cache_row(int32_t page_id, int32_t heads, int32_t h, int32_t pos, int32_t shift) {
  return ((static_cast<uint32_t>(page_id) * heads + h) << shift) + (pos & ((1 << shift) - 1));
}

// Whether an utterance's lengths fit: new_tokens of at most L, all of them within the table.
RNNT_PAGES_FN bool lengths_fit(int32_t new_tokens, int32_t L, int32_t cached, int64_t capacity) {
  return new_tokens >= 0 && new_tokens <= L && cached >= 0 && static_cast<int64_t>(cached) + new_tokens <= capacity;
}

// The keys [lo, hi) that the query at position pos sees; end = cached + new tokens.
struct Seen {
  int32_t lo, hi;
  RNNT_PAGES_FN Seen(int32_t pos, int32_t end, bool causal, int32_t left)
      : lo(left < 0 || pos < left ? 0 : pos - left), hi(causal ? pos + 1 : end) {}
  RNNT_PAGES_FN bool holds(int32_t key) const { return key >= lo && key < hi; }
};

}  // namespace rnnt
