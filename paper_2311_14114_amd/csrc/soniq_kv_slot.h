// Where a cached position lives: the index arithmetic of the paged
// key/value cache, shared by the gfx950 kernels and the host (the CPU tests
// compile this header alone).  Page tables, lengths and offsets are device
// data that no call can check before it launches, so every value taken from
// them is bounded here: nothing read or written through these functions
// lies outside the cache, whatever the tables hold.
#pragma once
#include <cstdint>

#if defined(__HIPCC__)
#define SONIQ_HD __host__ __device__ __forceinline__
#else
#define SONIQ_HD inline
#endif

namespace soniq {

// A page table: row b holds the pages of sequence b, `width` of them, rows
// `ld` entries apart.
struct KvTable {
  const int32_t* page;
  int64_t ld;
  int32_t width;
  int32_t B;
};

// The cache's extents: codes [pages][heads][page_size][row_bytes], scales
// [pages][heads][page_size].
struct KvDims {
  int32_t pages, page_size, heads, head_dim, bits;
};

// Cache row of position `pos` of sequence b for head 0 of its page, -1 where
// the position has no page: outside the table, or an entry that names none.
// The row of head h is this one plus h * page_size.  The host keeps
// pages * heads * page_size below 2^31.
SONIQ_HD int32_t kv_row(const KvTable& t, const KvDims& d, int32_t b, int64_t pos) {
  if (pos < 0 || pos >= (int64_t)t.width * d.page_size) return -1;
  const uint32_t p = (uint32_t)pos / (uint32_t)d.page_size;  // width * page_size < 2^31
  const int32_t page = t.page[(int64_t)b * t.ld + p];
  if (page < 0 || page >= d.pages) return -1;
  return page * d.heads * d.page_size + (int32_t)((uint32_t)pos - p * (uint32_t)d.page_size);
}

// Rows [first, first + count) of a ragged batch of `total` rows that belong
// to sequence b, from prefix sums that may hold anything.
struct KvSpan {
  int32_t first, count;
};
SONIQ_HD KvSpan kv_span(int32_t lo, int32_t hi, int32_t total) {
  lo = lo < 0 ? 0 : lo > total ? total : lo;
  hi = hi < lo ? lo : hi > total ? total : hi;
  return {lo, hi - lo};
}

// Cached positions of a sequence: its length, as far as its table reaches.
SONIQ_HD int32_t kv_length(const KvTable& t, const KvDims& d, int32_t len) {
  const int64_t most = (int64_t)t.width * d.page_size;
  return len < 0 ? 0 : len > most ? (int32_t)most : len;
}

}  // namespace soniq
