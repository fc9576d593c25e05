// Host-side internals of the paged cache: the checked descriptor its kernels take.
#pragma once

#include "../../include/hstu_cache.h"
#include "cache_index.h"
#include "internal.h"

namespace hstu {

struct CacheDev {
  char *k, *v;
  int64_t *ts;
  int32_t *tables, *lens, *refs, *status;
  int32_t layers, num_pages, log_page, slots, max_pages;
  int32_t capacity;              // tokens of a table
  int32_t row_bytes;             // of a token's k (or v)
  int64_t layer_bytes;           // of a layer's pool
};

// Checks every field of the descriptor that the host can see; fills `d`.
int check_cache(const hstu_cache *c, CacheDev *d);

}  // namespace hstu
