// Index arithmetic of the paged cache, shared by its kernels: which tokens a query
// sees, where a token lies, and how a batch's tokens are cut into chunks.  Plain C++
// (no device code), so that a host build can check every index against the bounds of
// the buffers.
#pragma once

#include <stdint.h>

#if defined(__HIPCC__)
#include <hip/hip_runtime.h>
#define HSTU_HD __host__ __device__ __forceinline__
#else
#define HSTU_HD inline
#endif

namespace hstu {

// The tokens that the last one of `len` sees: the first `head` tokens, then those
// from `from` on; `count` in all.  The x-th of them is token at(x).
struct Seen {
  int32_t head, from, count;
  HSTU_HD int32_t at(int32_t x) const { return x < head ? x : from + (x - head); }
};

// window and sinks are at most 2^31 - 1 (no window: window >= len).
HSTU_HD Seen seen_by_last(int32_t len, int32_t window, int32_t sinks) {
  Seen s;
  s.from = len > window ? len - window : 0;
  s.head = sinks < s.from ? sinks : s.from;
  s.count = s.head + (len - s.from);
  return s;
}

// Length of slot `slot`, 0 where it names none; never past the table's columns.
HSTU_HD int32_t slot_len(const int32_t *lens, int32_t slots, int32_t capacity, int32_t slot) {
  if (slot < 0 || slot >= slots) return 0;
  const int32_t n = lens[slot];
  return n < 0 ? 0 : (n > capacity ? capacity : n);
}

// Row of the pools (page * page_size + place) of token `pos` given its page, -1 where
// the page is none.
HSTU_HD int32_t page_row(int32_t page, int32_t num_pages, int32_t log_page, int32_t pos) {
  if (page < 0 || page >= num_pages) return -1;
  return (page << log_page) + (pos & ((1 << log_page) - 1));
}

// Chunk length, in tokens: `total` tokens cut into about `target` chunks, a multiple
// of `step` (where it passes 31 bits, which takes many rows of one long sequence, every
// row is one chunk).
HSTU_HD int32_t chunk_len(int64_t total, int32_t target, int32_t step) {
  const int64_t c = (total + target - 1) / target;
  const int64_t r = (c + step - 1) / step * step;
  return (int32_t)(r < step ? step : r > INT32_MAX ? INT32_MAX : r);
}
// Chunks of `count` tokens; the end of the chunk that begins at x0.  Neither passes 31
// bits for any lengths.
HSTU_HD int32_t chunks_of(int32_t count, int32_t len) {
  return count > 0 ? (count - 1) / len + 1 : 0;
}
HSTU_HD int32_t chunk_end(int32_t x0, int32_t count, int32_t len) {
  return len < count - x0 ? x0 + len : count;
}

// Pages that hold `tokens` tokens.
HSTU_HD int32_t pages_of(int64_t tokens, int32_t log_page) {
  return (int32_t)((tokens + ((int64_t)1 << log_page) - 1) >> log_page);
}

}  // namespace hstu
